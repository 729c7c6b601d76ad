// expanded.h -- attention in the expanded form: keys and values of a head in 16 bits,
// one rotary key a token for all heads, ragged and causal.
//
//   s_t = scale (q . k_t + p . r_t)   out = sum_t e^(s_t) v_t / sum_t e^(s_t)
// in one pass over the tokens with a running maximum.  A workgroup takes 128 rows of one head, a
// wave 32 of them, over tiles of 64 tokens that all four stage into LDS.
#pragma once

#include <utility>

#include "latent.h"

namespace uzip_kv {

typedef short s16x4 __attribute__((ext_vector_type(4)));

struct ExpandedArgs {
  const void *q, *k, *rot, *v;
  void *out;
  float *lse;
  int64_t q_row, q_head, k_row, k_head, rot_row, v_row, v_head, out_row, out_head;
  const int32_t *q_start, *k_start;
  uint32_t n_rows, n_keys, heads, n_reqs;
  float scale_log2;
  bool direct;        // keys and values can go to LDS as they are
  bool q_vec, out_vec;
};

// Chunks of 16 bytes; chunk c of token t lies at c ^ spread<chunks in a row>(t).  Neither a read of one chunk
// of 16 tokens nor a transposing read of four tokens by four chunks meets a bank twice.
template <int CHUNKS>
__device__ __forceinline__ uint32_t spread(uint32_t t) {
  if constexpr (CHUNKS == 16) return ((t & 3) << 2) | ((t >> 2) & 3);
  else if constexpr (CHUNKS == 8) return ((t & 2) << 1) | ((t >> 2) & 3);
  else return (t >> 2) & 3;
}

struct ExpandedBlock {
  int32_t first, rows;  // the block's rows
  int32_t base;         // place of the first
  int32_t key0, keys;   // the request's keys
};

// Block `index` of the requests' blocks of ROWS rows, last blocks of a request first; found by one wave.
template <int ROWS>
__device__ bool find_expanded(const ExpandedArgs &a, uint32_t index, ExpandedBlock *out) {
  const uint32_t lane = threadIdx.x & 63, n = a.n_reqs + 1, each = (n + 63) / 64, lo = min(n, lane * each), hi = min(n, lo + each);
  auto rows_of = [&](uint32_t i, int32_t *first) {
    const int64_t all = a.n_rows;
    const int64_t from = min(max((int64_t)(a.n_reqs ? a.q_start[i] : 0), (int64_t)0), all);
    const int64_t to = i < a.n_reqs ? min(max((int64_t)a.q_start[i + 1], from), all) : all;
    *first = (int32_t)from;
    return (int32_t)(to - from);
  };
  uint32_t mine = 0;
  int32_t first;
  for (uint32_t i = lo; i < hi; ++i) mine += ((uint32_t)rows_of(i, &first) + ROWS - 1) / ROWS;
  uint32_t upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(upto, o);
    if ((int)lane >= o) upto += y;
  }
  ExpandedBlock b{};
  const bool here = index < upto && index >= upto - mine;
  if (here) {
    uint32_t at = upto - mine;
    for (uint32_t i = lo; i < hi; ++i) {
      const uint32_t rows = (uint32_t)rows_of(i, &first), blocks = (rows + ROWS - 1) / ROWS;
      if (index - at < blocks) {
        const uint32_t block = blocks - 1 - (index - at);
        int64_t k0 = 0, k1 = 0;
        if (i < a.n_reqs) {
          k0 = min(max((int64_t)a.k_start[i], (int64_t)0), (int64_t)a.n_keys);
          k1 = min(max((int64_t)a.k_start[i + 1], k0), (int64_t)a.n_keys);
        }
        b.key0 = (int32_t)k0;
        b.keys = (int32_t)(k1 - k0);
        b.first = first + (int32_t)(block * ROWS);
        b.rows = min((int32_t)ROWS, (int32_t)(rows - block * ROWS));
        b.base = b.keys - (int32_t)rows + (int32_t)(block * ROWS);
        break;
      }
      at += blocks;
    }
  }
  const uint64_t who = __ballot(here);
  if (!who) return false;
  const int from = __ffsll((unsigned long long)who) - 1;
  uint32_t words[sizeof(ExpandedBlock) / 4];
  __builtin_memcpy(words, &b, sizeof(b));
#pragma unroll
  for (uint32_t i = 0; i < sizeof(b) / 4; ++i) words[i] = __builtin_amdgcn_readlane(words[i], from);
  __builtin_memcpy(out, words, sizeof(b));
  return true;
}

template <int DN, int DR, int DV, int WAVES>
struct Expanded {
  static constexpr int kRows = 32 * WAVES, kThreads = 64 * WAVES;
  struct Tile {
    uint8_t k[kTile * DN * 2], rot[kTile * DR * 2], v[kTile * DV * 2];
  };
  struct Lds {
    Tile tile[2];
  };
};

template <int T, int DN, int DR, int DV, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES > 1 ? 2 : 1) void expanded_kernel(ExpandedArgs a) {
  typedef Expanded<DN, DR, DV, WAVES> L;
  typedef typename Elem<T>::type Value;
  typedef typename LatentType<T>::Eight Eight;
  constexpr int kSteps = (DN + DR) / 16, kBlocks = DV / 32;
  constexpr float kLag = 8;  // weights up to 2^8
  extern __shared__ __align__(16) uint8_t lds_bytes[];
  typename L::Lds &lds = *(typename L::Lds *)lds_bytes;
  __shared__ int32_t first_of[3][DV];  // the first token whose value is NaN, infinite, minus infinite
  __shared__ uint32_t trouble;
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, h = lane >> 5;
  const uint32_t head = blockIdx.x % a.heads;
  ExpandedBlock b;
  if (!find_expanded<L::kRows>(a, blockIdx.x / a.heads, &b)) return;

  const int32_t j = (int32_t)(32 * wave + col);
  const bool here = j < b.rows;
  const int32_t at = here ? b.base + j : -1, at_min = b.base + min((int32_t)(32 * wave), b.rows - 1);
  const int32_t seen = min(max(b.base + b.rows, 0), b.keys);
  const uint32_t rounds = ((uint32_t)seen + kTile - 1) / kTile;

  Eight query[kSteps];
  {
    const Value *src = (const Value *)a.q + (int64_t)(b.first + (here ? j : 0)) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const uint32_t d = 16 * s + 8 * h;
      if (a.q_vec) {
        query[s] = *(const Eight *)(src + d);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) query[s][e] = src[d + e];
      }
    }
  }

  // A kind of rows into LDS: `bytes` of a row, `row` bytes from one to the next in memory.
  auto stage = [&](auto width, const uint8_t *base, int64_t row, uint32_t t0, uint8_t *to) {
    const uint32_t to_at = lds_at(to);
    constexpr int kBytes = decltype(width)::value, kChunks = kBytes / 16, kPer = 1024 / kBytes, kLoads = kTile / kPer;
    const uint32_t most = (uint32_t)b.keys - 1 - t0;
#pragma unroll
    for (int i = 0; i < (kLoads + WAVES - 1) / WAVES; ++i) {
      const uint32_t k = i * WAVES + wave;
      if (kLoads % WAVES && k >= kLoads) break;
      const uint32_t t = k * kPer + lane / kChunks, chunk = (lane % kChunks) ^ spread<kChunks>(t);
      if (a.direct) {
        load_to_lds(base, min(t, most) * (uint32_t)row + chunk * 16, to_at + k * 1024);
      } else {
        const Value *from = (const Value *)(base + (int64_t)min(t, most) * row) + chunk * 8;
        Value x[8] __attribute__((aligned(16)));
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = from[e];
        *(u32x4 *)(to + k * 1024 + lane * 16) = *(u32x4 *)x;
      }
    }
  };
  const uint8_t *k_at = (const uint8_t *)a.k + 2 * ((int64_t)b.key0 * a.k_row + (int64_t)head * a.k_head);
  const uint8_t *r_at = (const uint8_t *)a.rot + 2 * ((int64_t)b.key0 * a.rot_row);
  const uint8_t *v_at = (const uint8_t *)a.v + 2 * ((int64_t)b.key0 * a.v_row + (int64_t)head * a.v_head);
  auto ask = [&](uint32_t i) {
    typename L::Tile &tile = lds.tile[i & 1];
    const uint32_t t0 = i * kTile;
    stage(std::integral_constant<int, DN * 2>{}, k_at + 2 * (int64_t)t0 * a.k_row, 2 * a.k_row, t0, tile.k);
    stage(std::integral_constant<int, DR * 2>{}, r_at + 2 * (int64_t)t0 * a.rot_row, 2 * a.rot_row, t0, tile.rot);
    stage(std::integral_constant<int, DV * 2>{}, v_at + 2 * (int64_t)t0 * a.v_row, 2 * a.v_row, t0, tile.v);
  };

  // where this lane reads
  const uint32_t k_off = col * DN * 2 + ((h ^ spread<DN / 8>(col)) << 4);
  const uint32_t r_off = col * DR * 2 + ((h ^ spread<DR / 8>(col)) << 4);
  const uint32_t v_tok = 4 * h + ((lane & 15) >> 2);
  const uint32_t v_off = v_tok * DV * 2 + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ spread<DV / 8>(v_tok)) << 4) + (lane & 1) * 8;

  for (int careful = 0;; careful = 1) {
    f32x16 acc[kBlocks];
#pragma unroll
    for (int n = 0; n < kBlocks; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[n][e] = 0;
    float m = -INFINITY, l = 0;
    if (threadIdx.x == 0) trouble = 0;
    if (careful)
      for (uint32_t i = threadIdx.x; i < 3 * DV; i += L::kThreads) (&first_of[0][0])[i] = INT32_MAX;
    if (rounds > 0) ask(0);
    for (uint32_t i = 0; i < rounds; ++i) {
      typename L::Tile &tile = lds.tile[i & 1];
      const int32_t t0 = (int32_t)(i * kTile);
      __builtin_amdgcn_s_waitcnt(0);  // this wave's part has arrived
      __syncthreads();
      if (careful) {  // values that are NaN or infinite are noted and left out
        for (uint32_t c = threadIdx.x; c < kTile * DV / 8; c += L::kThreads) {
          const uint32_t t = c / (DV / 8), channel = ((c % (DV / 8)) ^ spread<DV / 8>(t)) * 8;
          Value *x = (Value *)tile.v + c * 8;
#pragma unroll 1
          for (int e = 0; e < 8; ++e) {
            const float y = (float)x[e];
            if (y - y == 0) continue;
            if (t0 + (int32_t)t < b.keys) atomicMin(&first_of[y != y ? 0 : y > 0 ? 1 : 2][channel + e], t0 + (int32_t)t);
            x[e] = (Value)0.0f;
          }
        }
        __syncthreads();
      }
      if (i + 1 < rounds) ask(i + 1);
      f32x16 s[2];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[n][e] = 0;
#pragma unroll
      for (int k = 0; k < DN / 16; ++k)
#pragma unroll
        for (int n = 0; n < 2; ++n)
          s[n] = mfma16(*(const Eight *)(tile.k + (k_off ^ (k << 5)) + n * 32 * DN * 2), query[k], s[n]);
#pragma unroll
      for (int k = 0; k < DR / 16; ++k)
#pragma unroll
        for (int n = 0; n < 2; ++n)
          s[n] = mfma16(*(const Eight *)(tile.rot + (r_off ^ (k << 5)) + n * 32 * DR * 2), query[DN / 16 + k], s[n]);
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[n][e] *= a.scale_log2;
      if (t0 + kTile - 1 > at_min) {
        const int32_t upto = at - t0 - 4 * (int)h;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[n][e] = 32 * n + 8 * (e / 4) + e % 4 <= upto ? s[n][e] : -INFINITY;
      }
      float most = -INFINITY;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) most = fmaxf(most, s[n][e]);
      if (__any(most > m + kLag)) {
        most = max_of_halves(most);
        const float next = most > m + kLag ? most : m, f = next == m ? 1.0f : __builtin_amdgcn_exp2f(m - next);
        m = next;
        l *= f;
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[n][e] *= f;
      }
      const float ref = m == -INFINITY ? 0.0f : m;
      Eight w[4];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float y = __builtin_amdgcn_exp2f(s[n][e] - ref);
          l += y;
          w[2 * n + e / 8][e % 8] = (Value)y;
        }
#pragma unroll
      for (int n = 0; n < kBlocks; ++n)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          union {
            Eight e;
            s16x4 p[2];
          } v;
#pragma unroll
          for (int p = 0; p < 2; ++p)
            v.p[p] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4 *)(tile.v + (v_off ^ (n << 6) ^ (p << 5)) + (16 * k + 8 * p) * DV * 2));
          acc[n] = mfma16(v.e, w[k], acc[n]);
        }
    }
    l = sum_of_halves(l);
    if (!careful) {  // a sum that is not finite is computed again with care
      float odd = l * 0.0f;
#pragma unroll
      for (int n = 0; n < kBlocks; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) odd = __builtin_fmaf(acc[n][e], 0.0f, odd);
      __syncthreads();
      if (__any(odd != 0.0f) && lane == 0) trouble = 1;
      __syncthreads();
      if (trouble) continue;
    }
    if (here) {
      const float f = l > 0 ? 1.0f / l : l == 0 ? 0.0f : NAN;
      Value *out = (Value *)a.out + (int64_t)(b.first + j) * a.out_row + (int64_t)head * a.out_head;
#pragma unroll
      for (int n = 0; n < kBlocks; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const uint32_t d = 32 * n + 8 * g + 4 * h;
          Value y[4] __attribute__((aligned(8)));
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float x = acc[n][4 * g + k] * f;
            if (careful) {
              if (at >= first_of[0][d + k]) x = NAN;
              if (at >= first_of[1][d + k]) x += INFINITY;
              if (at >= first_of[2][d + k]) x -= INFINITY;
            }
            y[k] = (Value)x;
          }
          if (a.out_vec) {
            *(u32x2 *)(out + d) = *(u32x2 *)y;
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) out[d + k] = y[k];
          }
        }
      if (h == 0 && a.lse) a.lse[(size_t)(b.first + j) * a.heads + head] = l == 0 ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
    }
    break;
  }
}

}  // namespace uzip_kv
