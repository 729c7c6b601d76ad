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

// Whether 64 rows' sums, queries, scores of two tiles and weights leave a SIMD's registers for two waves: 128 rows then go
// to eight waves, each pair a quarter of the tokens.  64 + 32 and 64 channels, fp16, 7 ragged requests of 6 heads: 38 us, by four
// waves 43; 2048 tokens of 16 heads 32 and 36; 4 x 1024 39 and 40; 8 x 512 of 8 heads 18 and 17.  (64 + 64 and 64, where
// registers spill: 35 and 39, 43 and 43, 21 and 18.)
constexpr bool expanded_by_eight(uint32_t nope, uint32_t rot, uint32_t value) { return 2 * (value / 2 + (nope + rot) / 4 + 40) <= 200; }

template <int DN>
uzip_status launch_expanded(const ExpandedCall &c);

}  // namespace uzip_kv
