// rotary.hip -- places of rows, rotary positions, and turned keys into 8-bit pages.
#include <algorithm>

#include "rotary.h"

namespace uzip_kv {
namespace {

// ------------------------------------------------------------------ places
__global__ __launch_bounds__(256) void positions_kernel(const int32_t *lens, const int32_t *q_start, uint32_t n_reqs, uint32_t n_rows, int32_t *out) {
  const uint32_t r = blockIdx.x * 256 + threadIdx.x;
  if (r >= n_rows) return;
  int32_t place = -1;
  uint32_t i = 0, top = n_reqs;  // the requests that begin at or before r: the last of them
  while (i < top) {
    const uint32_t mid = (i + top) / 2;
    if (q_start[mid] <= (int32_t)r) i = mid + 1;
    else top = mid;
  }
  if (i > 0) {
    const int64_t end = q_start[i], first = q_start[i - 1];
    const int64_t p = (int64_t)lens[i - 1] - (end - r);
    if ((int64_t)r < end && first >= 0 && p >= 0) place = (int32_t)p;
  }
  out[r] = place;
}

// ------------------------------------------------------------------ rotate
template <int T>
__global__ __launch_bounds__(kTurnThreads) void rotate_kernel(TurnRows a, Turn t) {
  __shared__ CosSin table[kTurnTable];
  turn_rows<T>(a, t, blockIdx.x, table);
}

// ------------------------------------------------------------------ turned keys into pages
// One run of keys of a head: as store_run, of units of eight pairs that are turned as they come.  What a
// thread turned first stays in registers until the page's exponent is known.
template <int T, int CODE, int THREADS>
__device__ __forceinline__ void store_turned_run(const StoreArgs &a, const Turn &t, bool vec, uint32_t run, uint32_t h, uint32_t tid, float *part) {
  typedef typename Elem<T>::type Value;
  const uint32_t D = a.c.dim, P = a.c.page, per = D / 16;
  const int32_t row = a.runs[2 * (size_t)run];
  int32_t n = a.runs[2 * (size_t)run + 1];
  if (row < 0 || n <= 0 || (uint32_t)row >= a.n_rows) return;
  const int64_t slot = a.slots[row];
  if (slot < 0 || (uint64_t)slot >= (uint64_t)a.c.n_pages << a.c.page_shift) return;
  const uint32_t page = (uint32_t)(slot >> a.c.page_shift), off = (uint32_t)slot & (P - 1);
  n = min((uint32_t)n, min(P - off, a.n_rows - (uint32_t)row));
  const Value *x = (const Value *)a.x[0] + (int64_t)row * a.row[0] + (int64_t)h * a.head[0];
  const size_t ph = (size_t)page * a.c.heads + h;
  uint8_t *codes = a.c.k + (ph * P + off) * D;
  const uint32_t was = off ? a.c.k_exp[ph] : 0, count = (uint32_t)n * per;

  auto load = [&](uint32_t i, float *v) {
    const uint32_t j = i / per, u = i - j * per;
    const Value *from = x + (int64_t)j * a.row[0];
    if (vec) {
      const Groups g = groups_of<8>(t, u);
      Eight<T> e[2];
      e[0].load(from + g.a, true);
      e[1].load(from + g.b, true);
      e[0].get(v);
      e[1].get(v + 8);
      if (g.turned) {
        const int32_t place = t.positions[row + (int32_t)j];
        turn_unit<8>(t, v, [&](int k) {
          return turn_of(t, place, 8 * u + k);
        });
      }
    } else {  // pair by pair; v[2 k] and v[2 k + 1]
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t p = 8 * u + k;
        v[2 * k] = (float)from[channel_of(t, p, 0)];
        v[2 * k + 1] = (float)from[channel_of(t, p, 1)];
        if (p < t.half) turn_pair(turn_of(t, t.positions[row + (int32_t)j], p), v[2 * k], v[2 * k + 1]);
      }
    }
  };
  float amax = 0;
  bool odd = false;
  auto scan = [&](const float *v) {
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const float f = fabsf(v[k]);
      const bool finite = f < INFINITY;
      odd = odd || !finite;
      amax = fmaxf(amax, finite ? f : 0.0f);
    }
  };
  constexpr uint32_t kKeep = 2;
  float held[kKeep][16];
#pragma unroll
  for (uint32_t k = 0; k < kKeep; ++k)
    if (tid + k * THREADS < count) {
      load(tid + k * THREADS, held[k]);
      scan(held[k]);
    }
  for (uint32_t i = tid + kKeep * THREADS; i < count; i += THREADS) {
    float v[16];
    load(i, v);
    scan(v);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
  odd = __any(odd);
  if (THREADS > 64) {
    if ((tid & 63) == 0) {
      part[tid >> 6] = amax;
      part[4 + (tid >> 6)] = odd ? 1.0f : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      amax = fmaxf(amax, part[w]);
      odd = odd || part[4 + w] != 0;
    }
  }
  const uint32_t e = max((uint32_t)exponent_for<CODE>(amax), was);
  if (tid == 0 && e != was) a.c.k_exp[ph] = (uint8_t)e;
  const float inv = pow2(254 - (int)e);
  odd = odd || e >= (uint32_t)Code<CODE>::kExpMax;  // there values may lie past the largest code

  auto put = [&](uint32_t i, const float *v) {
    const uint32_t j = i / per, u = i - j * per;
    uint8_t *to = codes + (size_t)j * D;
    if (vec) {
      const Groups g = groups_of<8>(t, u);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float *y = v + 8 * k;
        u32x2 w = {0, 0};
        if (odd) {
#pragma unroll
          for (int c = 0; c < 8; ++c) w[c / 4] |= encode<CODE>(y[c], inv) << (8 * (c % 4));
        } else {
          w = u32x2{encode4<CODE>(y, inv), encode4<CODE>(y + 4, inv)};
        }
        *(u32x2 *)(to + (k ? g.b : g.a)) = w;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        to[channel_of(t, 8 * u + k, 0)] = (uint8_t)encode<CODE>(v[2 * k], inv);
        to[channel_of(t, 8 * u + k, 1)] = (uint8_t)encode<CODE>(v[2 * k + 1], inv);
      }
    }
  };
#pragma unroll
  for (uint32_t k = 0; k < kKeep; ++k)
    if (tid + k * THREADS < count) put(tid + k * THREADS, held[k]);
  for (uint32_t i = tid + kKeep * THREADS; i < count; i += THREADS) {
    float v[16];
    load(i, v);
    put(i, v);
  }
  if (off && e > was) grow_page<CODE>(a.c.k + ph * P * D, false, off, D, P, was, e, tid, THREADS);
}

// A run of one row by a wave: a lane a pair or two.
template <int T, int CODE>
__device__ __forceinline__ void store_turned_one(const StoreArgs &a, const Turn &t, int32_t row, uint32_t h, uint32_t lane) {
  typedef typename Elem<T>::type Value;
  const uint32_t D = a.c.dim, P = a.c.page;
  const Value *x = (const Value *)a.x[0] + (int64_t)row * a.row[0] + (int64_t)h * a.head[0];
  const int64_t slot = a.slots[row];
  float v[2][2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint32_t p = lane + 64 * k;
    v[k][0] = v[k][1] = 0;
    if (p < D / 2) {
      v[k][0] = (float)x[channel_of(t, p, 0)];
      v[k][1] = (float)x[channel_of(t, p, 1)];
      if (p < t.half) turn_pair(turn_of(t, t.positions[row], p), v[k][0], v[k][1]);
    }
  }
  if (slot < 0 || (uint64_t)slot >= (uint64_t)a.c.n_pages << a.c.page_shift) return;
  const uint32_t page = (uint32_t)(slot >> a.c.page_shift), off = (uint32_t)slot & (P - 1);
  const size_t ph = (size_t)page * a.c.heads + h;
  uint8_t *codes = a.c.k + ph * P * D;
  const uint32_t was = off ? a.c.k_exp[ph] : 0;
  float amax = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float f = fabsf(v[k / 2][k % 2]);
    amax = fmaxf(amax, f < INFINITY ? f : 0.0f);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
  const uint32_t e = max((uint32_t)exponent_for<CODE>(amax), was);
  if (lane == 0 && e != was) a.c.k_exp[ph] = (uint8_t)e;
  const float inv = pow2(254 - (int)e);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t p = lane + 64 * (k / 2);
    if (p < D / 2) codes[(size_t)off * D + channel_of(t, p, k % 2)] = (uint8_t)encode<CODE>(v[k / 2][k % 2], inv);
  }
  if (off && e > was) grow_page<CODE>(codes, false, off, D, P, was, e, lane, 64);
}

// Workgroups: for each run, head and of keys and values one (or a wave, FEW); the rest turn queries.  Every
// function is inlined: as calls they took 199 registers, and 16384 tokens of 32 and 8 heads of 128 in bf16
// 202 us.  Now their 369 MB take 88 us, 4.2 TB/s, with 95 registers, which five waves a SIMD leave each; with 100, and so four
// waves, the call took 92.5 us instead of 89.3, and with the pairs' turns one half after the other, in 87 registers, 130.
template <int T, int CODE, bool FEW>
__global__ __launch_bounds__(256, FEW ? 4 : 5) void rotate_store_kernel(StoreArgs a, TurnRows q, Turn t, uint32_t max_runs, uint32_t head_blocks, bool turn_vec) {
  __shared__ CosSin table[kTurnTable];
  __shared__ float part[8];
  const uint32_t blocks = max_runs * head_blocks * 2;
  if (blockIdx.x >= blocks) {
    turn_rows<T>(q, t, blockIdx.x - blocks, table);
    return;
  }
  const uint32_t run = blockIdx.x / (2 * head_blocks), rest = blockIdx.x - run * 2 * head_blocks;
  const bool values = rest >= head_blocks;
  const uint32_t hb = rest - (values ? head_blocks : 0);
  if ((int32_t)run >= a.counts[1]) return;
  if (FEW) {
    const uint32_t h = hb * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int32_t row = a.runs[2 * (size_t)run], rows = a.runs[2 * (size_t)run + 1];
    if (h >= a.c.heads || row < 0 || (uint32_t)row >= a.n_rows) return;
    if (rows == 1) {
      if (values) store_one<T, CODE>(a, true, row, h, lane);
      else store_turned_one<T, CODE>(a, t, row, h, lane);
    } else if (values) {
      store_run<T, CODE, 64, true>(a, run, h, lane, nullptr, nullptr);
    } else {
      store_turned_run<T, CODE, 64>(a, t, turn_vec, run, h, lane, nullptr);
    }
  } else if (values) {
    store_run<T, CODE, 256, true>(a, run, hb, threadIdx.x, part, (uint32_t *)part + 4);
  } else {
    store_turned_run<T, CODE, 256>(a, t, turn_vec, run, hb, threadIdx.x, part);
  }
}

template <int T, int CODE>
void launch_rotate_store(const StoreArgs &a, const TurnRows &q, const Turn &t, uint32_t max_runs, hipStream_t stream) {
  const bool few = a.n_rows <= 2 * max_runs;  // as in uzip_kv_store
  const uint32_t head_blocks = few ? (a.c.heads + 3) / 4 : a.c.heads, grid = max_runs * head_blocks * 2 + turn_blocks(q);
  const bool vec = a.vec && t.even;
  if (few) rotate_store_kernel<T, CODE, true><<<grid, 256, 0, stream>>>(a, q, t, max_runs, head_blocks, vec);
  else rotate_store_kernel<T, CODE, false><<<grid, 256, 0, stream>>>(a, q, t, max_runs, head_blocks, vec);
}

}  // namespace
}  // namespace uzip_kv

using namespace uzip_kv;

extern "C" {

uzip_status uzip_kv_positions(const int32_t *d_lens, const int32_t *d_q_start, uint32_t n_reqs, uint32_t n_rows,
                              int32_t *d_positions, hipStream_t stream) {
  if (n_reqs > UZIP_KV_MAX_REQUESTS || n_rows > UZIP_KV_MAX_ROWS) return UZIP_EINVAL;
  if (n_rows == 0) return UZIP_OK;
  if (!d_positions || (n_reqs && (!d_lens || !d_q_start)) || !aligned(d_lens, 4) || !aligned(d_q_start, 4) || !aligned(d_positions, 4))
    return UZIP_EINVAL;
  if (const uzip_status s = device(nullptr); s != UZIP_OK) return s;
  positions_kernel<<<(n_rows + 255) / 256, 256, 0, stream>>>(d_lens, d_q_start, n_reqs, n_rows, d_positions);
  return hipGetLastError() == hipSuccess ? UZIP_OK : UZIP_EHIP;
}

uzip_status uzip_rotate(uzip_dtype dtype, const void *d_x, int64_t x_row, int64_t x_head, uint32_t n_rows,
                        uint32_t n_heads, uint32_t head_dim, const uzip_turn *turn, void *d_out, int64_t out_row,
                        int64_t out_head, hipStream_t stream) {
  if (!valid_type(dtype) || !valid_turn(turn) || head_dim > 1024 || turn->first + turn->rot > head_dim || n_rows > UZIP_KV_MAX_ROWS ||
      n_heads > 65535)
    return UZIP_EINVAL;
  if (n_rows == 0 || n_heads == 0) return UZIP_OK;
  TurnRows a{};
  if (!valid_places(turn) || !rows_to_turn(dtype, d_x, x_row, x_head, n_rows, n_heads, head_dim, turn, d_out, out_row, out_head, &a))
    return UZIP_EINVAL;
  if (const uzip_status s = device(nullptr); s != UZIP_OK) return s;
  const Turn t = turn_args(turn);
  const uint32_t grid = turn_blocks(a);
  switch (dtype) {
    case UZIP_BF16: rotate_kernel<UZIP_BF16><<<grid, kTurnThreads, 0, stream>>>(a, t); break;
    case UZIP_FP16: rotate_kernel<UZIP_FP16><<<grid, kTurnThreads, 0, stream>>>(a, t); break;
    default: rotate_kernel<UZIP_FP32><<<grid, kTurnThreads, 0, stream>>>(a, t); break;
  }
  return hipGetLastError() == hipSuccess ? UZIP_OK : UZIP_EHIP;
}

uzip_status uzip_kv_rotate_store(const uzip_kv_cache *cache, uzip_dtype dtype, const void *d_k, int64_t k_row,
                                 int64_t k_head, const void *d_v, int64_t v_row, int64_t v_head, uint32_t n_rows,
                                 const int64_t *d_slots, const int32_t *d_runs, const int32_t *d_counts,
                                 uint32_t max_runs, const uzip_turn *turn, const void *d_q, int64_t q_row,
                                 int64_t q_head, uint32_t n_q_heads, void *d_q_out, int64_t out_row,
                                 int64_t out_head, hipStream_t stream) {
  if (!valid_cache(cache) || !valid_type(dtype) || n_rows > UZIP_KV_MAX_ROWS || max_runs > UZIP_KV_MAX_ROWS || !valid_turn(turn) ||
      turn->inverse || turn->first + turn->rot > cache->head_dim)
    return UZIP_EINVAL;
  if (n_rows == 0) return UZIP_OK;
  if (!valid_rows(d_k, k_row, k_head, type_bytes(dtype)) || !valid_rows(d_v, v_row, v_head, type_bytes(dtype)) ||
      !d_slots || (max_runs && !d_runs) || !d_counts || !aligned(d_slots, 8) || !aligned(d_runs, 4) || !aligned(d_counts, 4) ||
      !valid_places(turn))
    return UZIP_EINVAL;
  TurnRows q{};
  if (n_q_heads && !rows_to_turn(dtype, d_q, q_row, q_head, n_rows, n_q_heads, cache->head_dim, turn, d_q_out, out_row, out_head, &q))
    return UZIP_EINVAL;
  if ((uint64_t)max_runs * cache->n_heads * 2 + turn_blocks(q) > INT32_MAX) return UZIP_EINVAL;
  if (max_runs == 0 && n_q_heads == 0) return UZIP_OK;
  if (const uzip_status s = device(nullptr); s != UZIP_OK) return s;
  StoreArgs a{{cache->k, cache->v, cache->k_exp, cache->v_exp, cache->n_pages, cache->n_heads, cache->head_dim,
               cache->page_tokens, (uint32_t)__builtin_ctz(cache->page_tokens)},
              {d_k, d_v}, {k_row, v_row}, {k_head, v_head}, d_slots, d_runs, d_counts, n_rows, false};
  const int64_t size = type_bytes(dtype);
  a.vec = aligned(d_k, 16) && aligned(d_v, 16);
  for (const int64_t s : {k_row, k_head, v_row, v_head}) a.vec = a.vec && s * size % 16 == 0;
  const Turn t = turn_args(turn);
  const bool e5 = cache->dtype == UZIP_E5M2;
  switch (dtype) {
    case UZIP_BF16: (e5 ? launch_rotate_store<UZIP_BF16, UZIP_E5M2> : launch_rotate_store<UZIP_BF16, UZIP_E4M3FN>)(a, q, t, max_runs, stream); break;
    case UZIP_FP16: (e5 ? launch_rotate_store<UZIP_FP16, UZIP_E5M2> : launch_rotate_store<UZIP_FP16, UZIP_E4M3FN>)(a, q, t, max_runs, stream); break;
    default: (e5 ? launch_rotate_store<UZIP_FP32, UZIP_E5M2> : launch_rotate_store<UZIP_FP32, UZIP_E4M3FN>)(a, q, t, max_runs, stream); break;
  }
  return hipGetLastError() == hipSuccess ? UZIP_OK : UZIP_EHIP;
}

}  // extern "C"
