// latent_host.h -- what the latent cache's entry points share.
#pragma once

#include "kv_host.h"
#include "latent.h"

namespace uzip_kv {

constexpr uint32_t kLatentUnits = 256;  // workgroups that the workspace is sized for, whatever the device

struct LatentCall {
  LatentArgs a;
  uzip_dtype type, code;
  uint32_t units, rows;
  hipStream_t stream;
};

// Rows of a block, by the rows of the longest list.
inline uint32_t latent_rows(uint32_t n_rows, uint32_t heads, uint32_t max_new) {
  const uint64_t list = (uint64_t)(max_new < n_rows ? max_new : n_rows) * heads;
  return list <= 32 ? 32 : 64;
}

template <int DC>
uzip_status launch_latent(LatentCall &c);

inline bool valid_latent_cache(const uzip_latent_cache *c) {
  return c && c->codes && c->exps && aligned(c->codes, 16) && aligned(c->exps, 2) && c->n_pages > 0 &&
         (c->latent == 256 || c->latent == 512) && (c->rot == 32 || c->rot == 64) && valid_page(c->page_tokens) &&
         (uint64_t)c->n_pages * c->page_tokens < (1ull << 31) && (c->dtype == UZIP_E4M3FN || c->dtype == UZIP_E5M2);
}

}  // namespace uzip_kv
