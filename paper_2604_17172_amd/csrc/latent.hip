// latent.hip -- the latent cache: write of new tokens, and the entry points.
#include <algorithm>
#include <cmath>

#include "latent_host.h"
#include "rotary.h"

namespace uzip_kv {
namespace {

// ------------------------------------------------------------------ store
// A wave for each row: its latent (four or eight channels a lane), its rotary key (a pair to each of
// the first lanes), the largest of each by exchanges, the codes.  No row waits for another, since scales
// are a token's own.  16384 rows of 512 + 64 in bf16, 28 MB: 9.6 us, 2.9 TB/s; a wave's chain of loads, maxima and
// stores is the bound, not the bytes (5.6 us).
struct LatentStoreArgs {
  uint8_t *codes, *exps;
  const void *latent, *rot;
  int64_t latent_row, rot_row;
  const int64_t *slots;
  uint64_t n_slots;
  uint32_t n_rows, width;  // latent
  uint32_t blocks;         // workgroups for the rows; the others turn queries
  bool vec;
};

__device__ __forceinline__ float finite_or_zero(float x) {
  const float f = fabsf(x);
  return f < INFINITY ? f : 0.0f;
}
// The largest of a wave, in all lanes: within rows of 16 lanes, then the rows.  By cross-lane moves of the vector
// unit: the twelve exchanges of two such maxima over LDS took half of a store's time.
__device__ __forceinline__ float wave_max(float x) {
  auto moved = [](float y, auto control) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(y), decltype(control)::value, 0xf, 0xf, true));
  };
  x = fmaxf(x, moved(x, std::integral_constant<int, 0xB1>{}));   // lanes 1 0 3 2 of each four
  x = fmaxf(x, moved(x, std::integral_constant<int, 0x4E>{}));   // 2 3 0 1
  x = fmaxf(x, moved(x, std::integral_constant<int, 0x124>{}));  // row turned by 4
  x = fmaxf(x, moved(x, std::integral_constant<int, 0x128>{}));  // by 8
  const uint32_t w = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(w, w, false, false);
  return max_of_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

template <int T, int CODE>
__device__ void store_latent(const LatentStoreArgs &a, const Turn &t, uint32_t row, uint32_t lane) {
  typedef typename Elem<T>::type Value;
  const int64_t slot = a.slots[row];
  const uint32_t C = a.width, per = C / 64, R = 2 * t.half;
  const Value *x = (const Value *)a.latent + (int64_t)row * a.latent_row + lane * per;
  float v[8];
  if (per == 8 && a.vec) {
    Eight<T> e;
    e.load(x, true);
    e.get(v);
  } else {
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) v[j] = j < per ? (float)x[j] : 0.0f;
  }
  const Value *p = (const Value *)a.rot + (int64_t)row * a.rot_row;
  float ra = 0, rb = 0;
  const uint32_t ca = t.interleaved ? 2 * lane : lane, cb = t.interleaved ? 2 * lane + 1 : lane + t.half;
  if (lane < t.half) {
    ra = (float)p[ca];
    rb = (float)p[cb];
    turn_pair(turn_of(t, t.positions[row], lane), ra, rb);
  }
  if (slot < 0 || (uint64_t)slot >= a.n_slots) return;
  float most = 0;
  bool odd = false;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float f = finite_or_zero(v[j]);
    odd = odd || f != fabsf(v[j]);
    most = fmaxf(most, f);
  }
  const int ec = exponent_for<CODE>(wave_max(most));
  const int er = exponent_for<CODE>(wave_max(fmaxf(finite_or_zero(ra), finite_or_zero(rb))));
  const float inv = pow2(254 - ec), inv_r = pow2(254 - er);
  uint8_t *to = a.codes + (size_t)slot * (C + R);
  u32x2 w = {0, 0};
  if (odd || ec >= Code<CODE>::kExpMax) {  // there values may lie past the largest code
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j / 4] |= encode<CODE>(v[j], inv) << (8 * (j % 4));
  } else {
    w = u32x2{encode4<CODE>(v, inv), encode4<CODE>(v + 4, inv)};
  }
  if (per == 8) *(u32x2 *)(to + 8 * lane) = w;
  else *(uint32_t *)(to + 4 * lane) = w.x;
  if (lane < t.half) {
    const uint32_t ea = encode<CODE>(ra, inv_r), eb = encode<CODE>(rb, inv_r);
    if (t.interleaved) {
      *(uint16_t *)(to + C + ca) = (uint16_t)(ea | eb << 8);
    } else {
      to[C + ca] = (uint8_t)ea;
      to[C + cb] = (uint8_t)eb;
    }
  }
  if (lane == 0) *(uint16_t *)(a.exps + 2 * (size_t)slot) = (uint16_t)(ec | er << 8);
}

template <int T, int CODE>
__global__ __launch_bounds__(kTurnThreads) void latent_store_kernel(LatentStoreArgs a, TurnRows q, Turn t) {
  __shared__ CosSin table[kTurnTable];
  if (blockIdx.x >= a.blocks) {
    turn_rows<T>(q, t, blockIdx.x - a.blocks, table);
    return;
  }
  const uint32_t row = blockIdx.x * (kTurnThreads / 64) + (threadIdx.x >> 6);
  if (row < a.n_rows) store_latent<T, CODE>(a, t, row, threadIdx.x & 63);
}

bool attend_sizes(uint32_t n_rows, uint32_t n_heads, uint32_t n_reqs) {
  return n_heads > 0 && n_heads <= 1024 && n_rows <= UZIP_KV_MAX_ROWS && n_reqs <= UZIP_KV_MAX_REQUESTS &&
         (uint64_t)n_rows * n_heads <= UZIP_KV_MAX_ROW_HEADS;
}

}  // namespace
}  // namespace uzip_kv

using namespace uzip_kv;

extern "C" {

uzip_status uzip_latent_store(const uzip_latent_cache *cache, uzip_dtype dtype, const void *d_latent, int64_t latent_row,
                              const void *d_rot, int64_t rot_row, uint32_t n_rows, const int64_t *d_slots,
                              const uzip_turn *turn, const void *d_q, int64_t q_row, int64_t q_head, uint32_t n_q_heads,
                              void *d_q_out, int64_t out_row, int64_t out_head, hipStream_t stream) {
  if (!valid_latent_cache(cache) || !valid_type(dtype) || n_rows > UZIP_KV_MAX_ROWS || !valid_turn(turn) || turn->rot != cache->rot ||
      turn->first || turn->inverse)
    return UZIP_EINVAL;
  if (n_rows == 0) return UZIP_OK;
  const uint32_t bytes = type_bytes(dtype);
  if (!valid_rows(d_latent, latent_row, 0, bytes) || !valid_rows(d_rot, rot_row, 0, bytes) || !d_slots || !aligned(d_slots, 8) ||
      !valid_places(turn))
    return UZIP_EINVAL;
  TurnRows q{};
  if (n_q_heads && !rows_to_turn(dtype, d_q, q_row, q_head, n_rows, n_q_heads, cache->rot, turn, d_q_out, out_row, out_head, &q)) return UZIP_EINVAL;
  if (const uzip_status s = device(nullptr); s != UZIP_OK) return s;
  LatentStoreArgs a{cache->codes, cache->exps, d_latent, d_rot, latent_row, rot_row, d_slots, (uint64_t)cache->n_pages * cache->page_tokens,
                    n_rows, cache->latent, (n_rows + 3) / 4, aligned(d_latent, 16) && latent_row * bytes % 16 == 0};
  const Turn t = turn_args(turn);
  const uint32_t grid = a.blocks + turn_blocks(q);
  const bool e5 = cache->dtype == UZIP_E5M2;
  switch (dtype) {
    case UZIP_BF16:
      (e5 ? latent_store_kernel<UZIP_BF16, UZIP_E5M2> : latent_store_kernel<UZIP_BF16, UZIP_E4M3FN>)<<<grid, kTurnThreads, 0, stream>>>(a, q, t);
      break;
    case UZIP_FP16:
      (e5 ? latent_store_kernel<UZIP_FP16, UZIP_E5M2> : latent_store_kernel<UZIP_FP16, UZIP_E4M3FN>)<<<grid, kTurnThreads, 0, stream>>>(a, q, t);
      break;
    default:
      (e5 ? latent_store_kernel<UZIP_FP32, UZIP_E5M2> : latent_store_kernel<UZIP_FP32, UZIP_E4M3FN>)<<<grid, kTurnThreads, 0, stream>>>(a, q, t);
      break;
  }
  return hipGetLastError() == hipSuccess ? UZIP_OK : UZIP_EHIP;
}

size_t uzip_latent_attend_workspace(uint32_t latent, uint32_t n_rows, uint32_t n_heads, uint32_t n_reqs, uint32_t max_new) {
  if ((latent != 256 && latent != 512) || !attend_sizes(n_rows, n_heads, n_reqs)) return 0;
  return (size_t)2 * kLatentUnits * latent_rows(n_rows, n_heads, max_new) * (latent + 4) * sizeof(float) + kLatentUnits * sizeof(LatentCut);
}

uzip_status uzip_latent_attend(const uzip_latent_cache *cache, uzip_dtype dtype, const void *d_q, int64_t q_row,
                               int64_t q_head, uint32_t n_rows, uint32_t n_heads, const int32_t *d_table,
                               uint32_t max_pages, const int32_t *d_lens, const int32_t *d_q_start, uint32_t n_reqs,
                               uint32_t max_new, float scale, void *d_out, int64_t out_row, int64_t out_head,
                               float *d_lse, void *d_ws, size_t ws_bytes, hipStream_t stream) {
  if (!valid_latent_cache(cache) || (dtype != UZIP_BF16 && dtype != UZIP_FP16) || !attend_sizes(n_rows, n_heads, n_reqs))
    return UZIP_EINVAL;
  const uint32_t bytes = type_bytes(dtype);
  if (n_rows && (!valid_rows(d_q, q_row, q_head, bytes) || !valid_rows(d_out, out_row, out_head, bytes) || !d_q_start))
    return UZIP_EINVAL;
  if (n_rows && n_reqs && (!d_lens || (max_pages && !d_table))) return UZIP_EINVAL;
  if (!aligned(d_table, 4) || !aligned(d_lens, 4) || !aligned(d_q_start, 4) || !aligned(d_lse, 4) ||
      !aligned(d_ws, 16) || max_pages > INT32_MAX || !(scale - scale == 0))
    return UZIP_EINVAL;
  if (n_rows == 0) return UZIP_OK;
  if (!d_ws || ws_bytes < uzip_latent_attend_workspace(cache->latent, n_rows, n_heads, n_reqs, max_new)) return UZIP_ENOSPC;
  int cus = 0;
  if (const uzip_status s = device(&cus); s != UZIP_OK) return s;
  LatentCall call{};
  LatentArgs &a = call.a;
  a.codes = cache->codes;
  a.exps = cache->exps;
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
  a.n_pages = cache->n_pages;
  a.page_shift = (uint32_t)__builtin_ctz(cache->page_tokens);
  a.rot = cache->rot;
  a.n_rows = n_rows;
  a.heads = n_heads;
  a.max_pages = max_pages;
  a.n_reqs = n_reqs;
  a.scale_log2 = scale * 1.4426950408889634f;
  auto at_multiples = [&](const void *p, int64_t row, int64_t head, int64_t of) {
    return aligned(p, of) && row * bytes % of == 0 && head * bytes % of == 0;
  };
  a.q_vec = at_multiples(d_q, q_row, q_head, 16);
  a.out_vec = at_multiples(d_out, out_row, out_head, 8);
  call.units = std::min((uint32_t)std::max(cus, 1), kLatentUnits);
  call.rows = latent_rows(n_rows, n_heads, max_new);
  a.part_acc = (float *)d_ws;
  a.part_ml = a.part_acc + (size_t)2 * kLatentUnits * call.rows * cache->latent;
  a.cuts = (LatentCut *)(a.part_ml + (size_t)2 * kLatentUnits * call.rows * 4);
  call.type = dtype;
  call.code = cache->dtype;
  call.stream = stream;
  return cache->latent == 256 ? launch_latent<256>(call) : launch_latent<512>(call);
}

}  // extern "C"
