// kv_attend.hip -- attention of new tokens over the 8-bit pages.
#include <algorithm>

#include "kv_device.h"
#include "kv_host.h"

namespace uzip_kv {
namespace {

struct AttendArgs {
  Cache c;
  const void *q;
  void *out;
  float *lse;
  int64_t q_row, q_head, out_row, out_head;
  const int32_t *table, *lens, *q_start;
  uint32_t n_rows, n_q_heads, group, max_pages, n_reqs, window;
  float scale;
};

constexpr int kWaves = 4;

// One wave for a row and a query head: 64 tokens at a time, a lane the score
// of one, then the channels of all.
template <int T, int CODE>
__global__ __launch_bounds__(64 * kWaves) void attend_kernel(AttendArgs a) {
  typedef typename Elem<T>::type Value;
  __shared__ float qs[kWaves][256];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = a.c.dim, P = a.c.page;
  const uint64_t items = (uint64_t)a.n_rows * a.n_q_heads;
  for (uint64_t item = (uint64_t)blockIdx.x * kWaves + wave; item < items; item += (uint64_t)gridDim.x * kWaves) {
    const uint32_t r = (uint32_t)(item / a.n_q_heads), ah = (uint32_t)(item % a.n_q_heads), h = ah / a.group;
    int64_t first = 0, last = 0;
    uint32_t req = 0;
    if (a.n_reqs && (int64_t)r < a.q_start[a.n_reqs]) {
      uint32_t top = a.n_reqs;
      while (top - req > 1) {
        const uint32_t mid = (req + top) / 2;
        if (a.q_start[mid] <= (int64_t)r) req = mid;
        else top = mid;
      }
      const int64_t len = min((int64_t)max(a.lens[req], 0), (int64_t)a.max_pages * P);
      const int64_t p = len - a.q_start[req + 1] + r;
      last = min(p + 1, len);
      if (a.window) first = max((int64_t)0, p + 1 - a.window);
    }
    const Value *q = (const Value *)a.q + (int64_t)r * a.q_row + (int64_t)ah * a.q_head;
    for (uint32_t d = lane; d < D; d += 64) qs[wave][d] = (float)q[d];
    __builtin_amdgcn_wave_barrier();
    float m = -INFINITY, l = 0, acc[4] = {0, 0, 0, 0};
    for (int64_t t0 = first & ~(int64_t)63; t0 < last; t0 += 64) {
      const int64_t t = t0 + lane;
      float s = -INFINITY, vs = 0;
      int64_t vo = 0;
      if (t >= first && t < last) {
        const int32_t page = a.table[(size_t)req * a.max_pages + (t >> a.c.page_shift)];
        if ((uint32_t)page < a.c.n_pages) {
          const size_t ph = (size_t)page * a.c.heads + h;
          const uint8_t *k = a.c.k + ph * P * D + (t & (P - 1)) * D;
          float dot = 0;
          for (uint32_t d = 0; d < D; ++d) dot += qs[wave][d] * decode<CODE>(k[d]);
          s = dot * pow2(a.c.k_exp[ph]) * a.scale;
          vs = pow2(a.c.v_exp[ph]);
          vo = (int64_t)(ph * P * D + (t & (P - 1))) + 1;
        }
      }
      float top = s;
#pragma unroll
      for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
      const float m2 = fmaxf(m, top), base = m2 == -INFINITY ? 0.0f : m2;
      const float p = vo ? expf(s - base) : 0.0f, shrink = expf(m - base);
      m = m2;
      float sum = p;
#pragma unroll
      for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
      l = l * shrink + sum;
      for (int i = 0; i < 4; ++i) acc[i] *= shrink;
      for (int j = 0; j < 64; ++j) {
        const int64_t at = __shfl(vo, j);
        const float pj = __shfl(p * vs, j);
        if (at == 0) continue;
        for (uint32_t i = 0, d = lane; d < D; ++i, d += 64) acc[i] += pj * decode<CODE>(a.c.v[at - 1 + (int64_t)d * P]);
      }
    }
    Value *out = (Value *)a.out + (int64_t)r * a.out_row + (int64_t)ah * a.out_head;
    for (uint32_t i = 0, d = lane; d < D; ++i, d += 64) out[d] = (Value)(l == 0 ? 0.0f : acc[i] / l);
    if (a.lse && lane == 0) a.lse[item] = l == 0 ? -INFINITY : m + logf(l);
    __builtin_amdgcn_wave_barrier();
  }
}

bool attend_sizes(uzip_dtype dtype, uint32_t n_rows, uint32_t n_q_heads, uint32_t n_heads, uint32_t head_dim,
                  uint32_t n_reqs) {
  return valid_type(dtype) && valid_dim(head_dim) && n_heads > 0 && n_q_heads > 0 && n_q_heads % n_heads == 0 &&
         n_q_heads <= 65535 && n_rows <= UZIP_KV_MAX_ROWS && n_reqs <= UZIP_KV_MAX_REQUESTS;
}

}  // namespace
}  // namespace uzip_kv

using namespace uzip_kv;

extern "C" {

size_t uzip_kv_attend_workspace(uzip_dtype dtype, uint32_t n_rows, uint32_t n_q_heads, uint32_t n_heads,
                                uint32_t head_dim, uint32_t n_reqs, uint32_t max_new) {
  (void)max_new;
  return attend_sizes(dtype, n_rows, n_q_heads, n_heads, head_dim, n_reqs) ? 256 : 0;
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
  if (const uzip_status s = device(nullptr); s != UZIP_OK) return s;
  AttendArgs a{{cache->k, cache->v, cache->k_exp, cache->v_exp, cache->n_pages, cache->n_heads, cache->head_dim,
                cache->page_tokens, (uint32_t)__builtin_ctz(cache->page_tokens)},
               d_q, d_out, d_lse, q_row, q_head, out_row, out_head, d_table, d_lens, d_q_start,
               n_rows, n_q_heads, n_q_heads / cache->n_heads, max_pages, n_reqs, window, scale};
  void (*fn)(AttendArgs) = nullptr;
  const bool e5 = cache->dtype == UZIP_E5M2;
  switch (dtype) {
    case UZIP_BF16: fn = e5 ? attend_kernel<UZIP_BF16, UZIP_E5M2> : attend_kernel<UZIP_BF16, UZIP_E4M3FN>; break;
    case UZIP_FP16: fn = e5 ? attend_kernel<UZIP_FP16, UZIP_E5M2> : attend_kernel<UZIP_FP16, UZIP_E4M3FN>; break;
    default: fn = e5 ? attend_kernel<UZIP_FP32, UZIP_E5M2> : attend_kernel<UZIP_FP32, UZIP_E4M3FN>; break;
  }
  const uint64_t blocks = ((uint64_t)n_rows * n_q_heads + kWaves - 1) / kWaves;
  fn<<<(uint32_t)std::min<uint64_t>(blocks, 65536), 64 * kWaves, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? UZIP_OK : UZIP_EHIP;
}

}  // extern "C"
