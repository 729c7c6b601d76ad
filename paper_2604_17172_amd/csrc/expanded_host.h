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

// Whether 128 rows go to eight waves, each pair a quarter of the tokens.  The narrowest kernel alone: two of its waves to a SIMD have
// registers for 64 rows' sums, queries, scores of two tiles and weights; 8 words that a block's beginning and end need are in memory
// meanwhile.  64 + 32 and 64 channels, fp16, 7 ragged requests of 6 heads: 38 us, by four
// waves 43; 2048 tokens of 16 heads 32 and 36; 4 x 1024 39 and 40; 8 x 512 of 8 heads 18 and 17.  (64 + 64 and 64, where the
// loop's registers spill: 35 and 39, 43 and 43, 21 and 18.)
constexpr bool expanded_by_eight(uint32_t nope, uint32_t rot, uint32_t value) { return nope == 64 && rot == 32 && value == 64; }

template <int DN>
uzip_status launch_expanded(const ExpandedCall &c);

}  // namespace uzip_kv
