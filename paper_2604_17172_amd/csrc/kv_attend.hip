// kv_attend.hip -- attention of new tokens over the 8-bit pages.
#include <algorithm>
#include <cmath>

#include "kv_attend.h"
#include "kv_host.h"

namespace uzip_kv {
namespace {

bool attend_sizes(uzip_dtype dtype, uint32_t n_rows, uint32_t n_q_heads, uint32_t n_heads, uint32_t head_dim,
                  uint32_t n_reqs) {
  return valid_type(dtype) && valid_dim(head_dim) && n_heads > 0 && n_q_heads > 0 && n_q_heads % n_heads == 0 &&
         n_heads <= 1024 && n_rows <= UZIP_KV_MAX_ROWS && n_reqs <= UZIP_KV_MAX_REQUESTS &&
         (uint64_t)n_rows * n_q_heads <= UZIP_KV_MAX_ROW_HEADS;
}

}  // namespace
}  // namespace uzip_kv

using namespace uzip_kv;

extern "C" {

size_t uzip_kv_attend_workspace(uzip_dtype dtype, uint32_t n_rows, uint32_t n_q_heads, uint32_t n_heads,
                                uint32_t head_dim, uint32_t n_reqs, uint32_t max_new) {
  if (!attend_sizes(dtype, n_rows, n_q_heads, n_heads, head_dim, n_reqs)) return 0;
  const Layout at = layout(dtype, head_dim, n_heads, n_q_heads / n_heads, n_reqs, max_new);
  return (size_t)(kMostUnits * at.rows_for_one * (head_dim + 2) * sizeof(float));
}

uzip_status uzip_kv_attend(const uzip_kv_cache *cache, uzip_dtype dtype, const void *d_q, int64_t q_row,
                           int64_t q_head, uint32_t n_rows, uint32_t n_q_heads, const int32_t *d_table,
                           uint32_t max_pages, const int32_t *d_lens, const int32_t *d_q_start, uint32_t n_reqs,
                           uint32_t max_new, float scale, uint32_t window, void *d_out, int64_t out_row,
                           int64_t out_head, float *d_lse, void *d_ws, size_t ws_bytes, hipStream_t stream) {
  if (!valid_cache(cache) || !attend_sizes(dtype, n_rows, n_q_heads, cache->n_heads, cache->head_dim, n_reqs))
    return UZIP_EINVAL;
  const uint32_t bytes = type_bytes(dtype);
  if (n_rows && (!valid_rows(d_q, q_row, q_head, bytes) || !valid_rows(d_out, out_row, out_head, bytes) || !d_q_start))
    return UZIP_EINVAL;
  if (n_rows && n_reqs && (!d_lens || (max_pages && !d_table))) return UZIP_EINVAL;
  if (!aligned(d_table, 4) || !aligned(d_lens, 4) || !aligned(d_q_start, 4) || !aligned(d_lse, 4) ||
      !aligned(d_ws, 16) || max_pages > INT32_MAX || !(scale - scale == 0))
    return UZIP_EINVAL;
  const size_t need = uzip_kv_attend_workspace(dtype, n_rows, n_q_heads, cache->n_heads, cache->head_dim, n_reqs, max_new);
  if (n_rows == 0) return UZIP_OK;
  if (!d_ws || ws_bytes < need) return UZIP_ENOSPC;
  int cus = 0;
  if (const uzip_status s = device(&cus); s != UZIP_OK) return s;
  AttendCall call{};
  AttendArgs &a = call.a;
  a.c = {cache->k, cache->v, cache->k_exp, cache->v_exp, cache->n_pages, cache->n_heads, cache->head_dim,
         cache->page_tokens, (uint32_t)__builtin_ctz(cache->page_tokens)};
  a.q = d_q;
  a.out = d_out;
  a.lse = d_lse;
  a.q_row = q_row;
  a.q_head = q_head;
  a.out_row = out_row;
  a.out_head = out_head;
  a.table = d_table;
  a.lens = d_lens;
  a.q_start = d_q_start;
  a.n_rows = n_rows;
  a.n_q_heads = n_q_heads;
  a.group = n_q_heads / cache->n_heads;
  a.max_pages = max_pages;
  a.n_reqs = n_reqs;
  a.window = window;
  a.units = std::min((uint32_t)std::max(cus, 1), kMostUnits);
  a.scale_log2 = std::fabs(scale) * 1.4426950408889634f;
  a.negate = scale < 0;
  auto at_multiples = [&](const void *p, int64_t row, int64_t head, int64_t of) {
    return aligned(p, of) && row * bytes % of == 0 && head * bytes % of == 0;
  };
  a.q_vec = at_multiples(d_q, q_row, q_head, 16);
  a.out_vec = at_multiples(d_out, out_row, out_head, 4 * bytes);
  a.part_acc = (float *)d_ws;
  a.part_ml = a.part_acc + (size_t)kMostUnits * layout(dtype, cache->head_dim, cache->n_heads, a.group, n_reqs, max_new).rows_for_one * cache->head_dim;
  call.type = dtype;
  call.code = cache->dtype;
  call.max_new = max_new;
  call.stream = stream;
  switch (cache->head_dim) {
    case 64: return launch_attend<64>(call);
    case 96: return launch_attend<96>(call);
    case 128: return launch_attend<128>(call);
    case 192: return launch_attend<192>(call);
    default: return launch_attend<256>(call);
  }
}

}  // extern "C"
