// expanded_host.h -- what the expanded form's entry point and launches share.
#pragma once

#include <algorithm>

#include "expanded.h"
#include "kv_host.h"

namespace uzip_kv {

struct ExpandedCall {
  ExpandedArgs a;
  uzip_dtype type;
  uint32_t rot, value;
  uint32_t rows;  // of a workgroup
  bool direct;    // keys and values can go to LDS as they are
  hipStream_t stream;
};

template <int DN>
uzip_status launch_expanded(const ExpandedCall &c);

}  // namespace uzip_kv
