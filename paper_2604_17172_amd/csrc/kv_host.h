// kv_host.h -- argument checks shared by the key/value cache's entry points.
#pragma once

#include <string.h>

#include "uzip_kv.h"

namespace uzip_kv {

// The current device is a gfx950; its number of compute units.
uzip_status device(int *cus);

inline bool pow2_between(uint32_t x, uint32_t lo, uint32_t hi) { return x >= lo && x <= hi && (x & (x - 1)) == 0; }
inline bool valid_page(uint32_t p) { return pow2_between(p, 16, 256); }
inline bool valid_dim(uint32_t d) { return d == 64 || d == 96 || d == 128 || d == 192 || d == 256; }
inline bool valid_type(uzip_dtype t) { return t == UZIP_BF16 || t == UZIP_FP16 || t == UZIP_FP32; }
inline uint32_t type_bytes(uzip_dtype t) { return t == UZIP_FP32 ? 4 : 2; }
inline bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

inline bool valid_cache(const uzip_kv_cache *c) {
  return c && c->k && c->v && c->k_exp && c->v_exp && aligned(c->k, 16) && aligned(c->v, 16) && c->n_pages > 0 &&
         c->n_heads > 0 && c->n_heads <= 65535 && valid_dim(c->head_dim) && valid_page(c->page_tokens) &&
         (uint64_t)c->n_pages * c->page_tokens < (1ull << 31) && (c->dtype == UZIP_E4M3FN || c->dtype == UZIP_E5M2);
}

// Rows at element strides, as far as the host can see: `heads` heads of `dim`
// values in each of at most 2^22 rows stay within 63 bits.
inline bool valid_rows(const void *p, int64_t row, int64_t head, uint32_t bytes) {
  const int64_t most = 1ll << 31;
  return p && aligned(p, bytes) && row >= -most && row <= most && head >= -most && head <= most;
}

}  // namespace uzip_kv
