// latent.h -- attention over the paged 8-bit latents, absorbed form: how a call is cut
// into pieces of work, and the kernels.
//
// A row q = (u, p) of a request sees tokens t of latents c and rotary keys r:
//   s_t = scale (u . c_t + p . r_t)   out = sum_t e^(s_t) c_t / sum_t e^(s_t)
// in one pass with a running maximum.  All heads share the tokens, so a request's rows are
// one list, row r = token r / heads, head r % heads, and a block of up to 128 of them
// reads each tile of 64 tokens once: a code is converted for the first product and taken as
// it is by the second.
//
// A token's scale 2^e belongs to its weight in the second product: with
//   g_t = s_t log2(e) + e_t,  w_t = 2^(g_t - m),  acc = sum w_t code_t,  l = sum w_t 2^-e_t
// out = acc / l, and the running maximum m is taken over g.
#pragma once

#include "kv_device.h"
#include "uzip_latent.h"

namespace uzip_kv {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

struct LatentArgs {
  const uint8_t *codes, *exps;
  const void *q;
  void *out;
  float *lse;
  int64_t q_row, q_head, out_row, out_head;
  const int32_t *table, *lens, *q_start;
  float *part_acc;  // [slot][row][latent]
  float *part_ml;   // [slot][row][2]
  uint32_t n_pages, page_shift, rot;
  uint32_t n_rows, heads, max_pages, n_reqs;
  uint32_t groups;    // workgroups that the work is shared by
  float scale_log2;   // scale log2 e
  bool q_vec, out_vec;
};

constexpr int kTile = 64;  // tokens

// ------------------------------------------------------------------ pieces of work
struct LatentRequest {
  int32_t first, rows, len, base;  // first row of the step's arrays, new tokens, tokens, place of the first new one
};

// Request i; the one past the last holds the rows of no request.
__device__ __forceinline__ LatentRequest latent_request(const LatentArgs &a, uint32_t i) {
  const int64_t n = a.n_rows;
  const int64_t lo = min(max((int64_t)(a.n_reqs ? a.q_start[i] : 0), (int64_t)0), n);
  const int64_t hi = i < a.n_reqs ? min(max((int64_t)a.q_start[i + 1], lo), n) : n;
  LatentRequest r;
  r.first = (int32_t)lo;
  r.rows = (int32_t)(hi - lo);
  const int64_t len = i < a.n_reqs ? min((int64_t)max(a.lens[i], 0), (int64_t)a.max_pages << a.page_shift) : 0;
  r.len = (int32_t)min(len, (int64_t)INT32_MAX - 2 * kTile);
  r.base = r.len - r.rows;
  return r;
}

// The work of a request's first b blocks of ROWS rows, in tiles: each block one for its beginning and end,
// and the tiles that its last row sees, which grow by ROWS / heads tokens from block to block.
// It only has to be the same everywhere; a block's real tiles are spread over its share.
template <int ROWS>
__device__ __forceinline__ uint64_t work_before(const LatentArgs &a, const LatentRequest &q, uint32_t b) {
  const int32_t seen = min(max(q.base + (int32_t)((min((uint32_t)q.rows * a.heads, (uint32_t)ROWS) - 1) / a.heads) + 1, 0), q.len);
  const uint64_t first = 1 + ((uint32_t)seen + kTile - 1) / kTile;
  uint64_t more = (uint64_t)b * (b - 1) / 2;
  if (b < 2) more = 0;
  return b * first + more * ROWS / (kTile * a.heads);
}
template <int ROWS>
__device__ __forceinline__ uint32_t blocks_of(const LatentArgs &a, const LatentRequest &q) {
  return ((uint32_t)q.rows * a.heads + ROWS - 1) / ROWS;
}

// Where a workgroup stands: a block of a request, and the work before it.
struct Place {
  LatentRequest q;
  uint32_t req, block, blocks;
  uint64_t before, size;  // of the block, in the call's work
};
__device__ __forceinline__ uint64_t wave_sum(uint64_t x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ uint64_t wave_before(uint64_t x) {  // sum over the lanes before this one
  uint64_t s = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = __shfl_up(s, o);
    if ((int)(threadIdx.x & 63) >= o) s += y;
  }
  return s - x;
}

template <int ROWS>
__device__ __forceinline__ void set_block(const LatentArgs &a, Place *p, uint64_t request_before, uint32_t block) {
  const uint64_t at = work_before<ROWS>(a, p->q, block);
  p->block = block;
  p->before = request_before + at;
  p->size = work_before<ROWS>(a, p->q, block + 1) - at;
}

// All work of the call, and which block the place x in it lies in (false: none).  By one wave, every
// lane a stretch of requests; `x_of` gives x from the sum.
template <int ROWS, class F>
__device__ bool find_block(const LatentArgs &a, const F &x_of, Place *out) {
  const uint32_t lane = threadIdx.x & 63, n = a.n_reqs + 1;
  const uint32_t each = (n + 63) / 64, lo = min(n, lane * each), hi = min(n, lo + each);
  uint64_t mine = 0;
  for (uint32_t i = lo; i < hi; ++i) {
    const LatentRequest q = latent_request(a, i);
    if (q.rows > 0) mine += work_before<ROWS>(a, q, blocks_of<ROWS>(a, q));
  }
  const uint64_t all = wave_sum(mine), before = wave_before(mine);
  uint64_t x;
  if (!x_of(all, &x) || x >= all) return false;
  Place p{};
  const bool here = x >= before && x - before < mine;
  if (here) {
    uint64_t at = before;
    for (uint32_t i = lo; i < hi; ++i) {
      p.q = latent_request(a, i);
      if (p.q.rows <= 0) continue;
      p.blocks = blocks_of<ROWS>(a, p.q);
      const uint64_t size = work_before<ROWS>(a, p.q, p.blocks);
      if (x - at < size) {
        p.req = i;
        uint32_t b = 0, top = p.blocks;  // the last block that begins at or before x
        while (top - b > 1) {
          const uint32_t mid = (b + top) / 2;
          if (at + work_before<ROWS>(a, p.q, mid) <= x) b = mid;
          else top = mid;
        }
        set_block<ROWS>(a, &p, at, b);
        break;
      }
      at += size;
    }
  }
  const int from = __ffsll((unsigned long long)__ballot(here)) - 1;
  uint32_t words[sizeof(Place) / 4];
  __builtin_memcpy(words, &p, sizeof(Place));
#pragma unroll
  for (uint32_t i = 0; i < sizeof(Place) / 4; ++i) words[i] = __builtin_amdgcn_readlane(words[i], from);
  __builtin_memcpy(out, words, sizeof(Place));
  return true;
}

// The block after p's, where there is one.
template <int ROWS>
__device__ __forceinline__ bool next_block(const LatentArgs &a, Place *p) {
  const uint64_t end = p->before + p->size;
  if (p->block + 1 < p->blocks) {
    set_block<ROWS>(a, p, end - work_before<ROWS>(a, p->q, p->block + 1), p->block + 1);
    return true;
  }
  for (uint32_t i = p->req + 1; i <= a.n_reqs; ++i) {
    p->q = latent_request(a, i);
    if (p->q.rows <= 0) continue;
    p->req = i;
    p->blocks = blocks_of<ROWS>(a, p->q);
    set_block<ROWS>(a, p, end, 0);
    return true;
  }
  return false;
}

// A workgroup's share of all work; shares are consecutive.
template <int MIN>
__device__ __forceinline__ uint64_t share_of(const LatentArgs &a, uint64_t all) {
  const uint64_t each = (all + a.groups - 1) / a.groups;
  return each > MIN ? each : MIN;
}

// Tiles of the block that the work from x0 to x1 (within the block's) stands for.
template <int ROWS>
__device__ __forceinline__ void tiles_of(const LatentArgs &a, const Place &p, uint64_t x0, uint64_t x1, uint32_t *t0, uint32_t *t1, uint32_t *all) {
  const uint32_t list = (uint32_t)p.q.rows * a.heads, r1 = min(list, (p.block + 1) * ROWS);
  const int32_t seen = min(max(p.q.base + (int32_t)((r1 - 1) / a.heads) + 1, 0), p.q.len);
  *all = ((uint32_t)seen + kTile - 1) / kTile;
  *t0 = (uint32_t)((x0 - p.before) * *all / p.size);
  *t1 = (uint32_t)((x1 - p.before) * *all / p.size);
}

// ------------------------------------------------------------------ the kernel
// One wave takes 32 rows.  Matrix instructions of 32 x 32: a lane holds, of the first operand, values of
// row lane % 32, of the second of column lane % 32; of the result, rows 8 (r / 4) + 4 (lane /
// 32) + r % 4 of column lane % 32.
//   S^T = K Q^T  in 16 bits: a lane ends up with 32 scores of one row
//   O^T = V^T P^T in 8 bits: the codes as they are; the weights in terms of four bits each,
//          of which the last is scaled by 2^-4 and so on.  The order of the tokens in the contraction is
//          the one in which the scores lie, so that no weight crosses lanes; V^T comes from
//          LDS by the transposing read, eight tokens of a channel to a lane.
// The first product is not taken in 8 bits: that instruction aligns eight products at a time to the
// largest and drops what lies 2^-13 below it (measured: 448 + 63 * 2^-6 gives 448.875), which scores,
// held in 32 bits, would lose; weights and codes have 8 and 4 bits, to which it is small.
template <int T>
struct LatentType {
  typedef bf16x8 Eight;
  static constexpr int kTerms = 2;  // of a weight: 8 bits, as many as the output has
};
template <>
struct LatentType<UZIP_FP16> {
  typedef f16x8 Eight;
  static constexpr int kTerms = 3;
};

// LDS of a tile.  Chunks of 16 codes; chunk c of token t lies at c ^ swizzle(t), so that both the rows
// of one chunk (the first product, 16 tokens at a time) and the eight tokens by two chunks of
// a transposing read fall on different banks.
template <int DC>
struct LatentTile {
  uint8_t latent[kTile * DC];
  uint8_t rot[kTile * 64];
  float scale_c[kTile], scale_r[kTile];  // on the codes of the first product
  float mul[kTile];                      // fp16: on the scores
  float e[kTile], inv[kTile];            // e_t, 2^-e_t
};
__device__ __forceinline__ uint32_t swizzle(uint32_t t) { return ((t & 3) << 1) | ((t >> 2) & 1) | (t & 8); }

template <int CODE, int T>
__device__ __forceinline__ typename LatentType<T>::Eight eight_codes(uint32_t lo, uint32_t hi, float scale) {
  union {
    typename LatentType<T>::Eight e;
    bf16x2 b[4];
    f16x2 h[4];
  } f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t w = i ? hi : lo;
    if constexpr (T == UZIP_FP16) {
      if constexpr (CODE == UZIP_E4M3FN) {
        f.h[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false);
        f.h[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true);
      } else {
        f.h[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w, scale, false);
        f.h[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w, scale, true);
      }
    } else {
      if constexpr (CODE == UZIP_E4M3FN) {
        f.b[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
        f.b[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
      } else {
        f.b[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, false);
        f.b[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, true);
      }
    }
  }
  return f.e;
}

__device__ __forceinline__ f32x16 mfma16(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma16(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }

// 16 bytes for each lane from base + offset on, into LDS side by side from `to` on.  Written out, so that the
// compiler does not know of it: else it has every later read of LDS wait until all have arrived.  The
// kernel waits itself, before the barrier that lets a tile be read.  (M0 holds where to; nothing else here uses it.)
__device__ __forceinline__ void load_to_lds(const uint8_t *base, uint32_t offset, const void *to) {
  const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)to);
  const uint32_t high = __builtin_amdgcn_readfirstlane((uint32_t)((uintptr_t)base >> 32)), low = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)base);
  const uint64_t from = (uint64_t)high << 32 | low;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(at), "v"(offset), "s"(from) : "memory");
}

// Bytes of four codes that are NaN or infinite: their sign bits.
template <int CODE>
__device__ __forceinline__ uint32_t not_numbers(uint32_t w) {
  return ((w & 0x7F7F7F7Fu) + (CODE == UZIP_E4M3FN ? 0x01010101u : 0x04040404u)) & 0x80808080u;
}

// RG groups of 32 rows, and two waves to each: in the first product each takes half of a tile's
// tokens, in the second half of the channels, so that 32 x DC sums fit its registers
// beside the queries.  A step of the loop is the scores of tile i, an exchange of their
// maxima, and then its weights, beside which the matrix units take the second product of tile i - 1.
template <int T, int CODE, int DC, int RG>
struct Latent {
  static constexpr int kRows = 32 * RG, kThreads = 128 * RG, kBlocks = DC / 64, kSteps = DC / 32, kBufs = 3;
  static constexpr int kMin = 2;       // the least share of a workgroup
  static constexpr float kLag = 3;     // weights up to 2^3: times 2^5 they are codes
  typedef LatentTile<DC> Tile;
  struct Lds {
    Tile tile[kBufs];
    i32x4 weights[RG][2][LatentType<T>::kTerms][64];  // of a wave's tokens, for the other
    float most[RG][2][32];
    float l[RG][2][32];
    uint32_t trouble;
    int32_t first_bad;
  };
};

template <int T, int CODE, int DC, int RG>
__global__ __launch_bounds__(128 * RG, DC == 256 ? 2 : 1) void latent_kernel(LatentArgs a) {
  typedef Latent<T, CODE, DC, RG> L;
  typedef typename Elem<T>::type Value;
  typedef typename LatentType<T>::Eight Eight;
  typedef typename L::Tile Tile;
  constexpr int TERMS = LatentType<T>::kTerms, kWaves = 2 * RG;
  extern __shared__ __align__(16) uint8_t lds_bytes[];
  typename L::Lds &lds = *(typename L::Lds *)lds_bytes;
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t rg = wave / 2, half = wave % 2, col = lane & 31, h = lane >> 5;

  uint64_t begin = 0, end = 0;
  Place place;
  if (!find_block<L::kRows>(a, [&](uint64_t all, uint64_t *x) {
        const uint64_t share = share_of<L::kMin>(a, all);
        begin = share * blockIdx.x;
        end = min(begin + share, all);
        *x = begin;
        return begin < all;
      }, &place))
    return;

  // what does not change from block to block
  const uint32_t row_bytes = DC + a.rot, rot_steps = a.rot / 32;
  // loads: 1 KiB at a time, 1024 / DC tokens of the latents, 16 of the rotary keys
  constexpr uint32_t kPer = 1024 / DC, kChunks = DC / 16, kLoads = kTile / kPer;
  const uint32_t load_tok = lane / kChunks, rot_tok = lane / 4;
  // the first product: token col of this wave's half, chunk 2 s + h
  const uint32_t k_off = (32 * half + col) * DC + ((h ^ swizzle(col & 15)) << 4);
  const uint32_t kr_off = (32 * half + col) * 64 + ((h ^ ((col >> 2) & 3)) << 4);
  // the second: eight tokens by 16 channels for 16 lanes, from this wave's first channel on
  const uint32_t j8 = (lane & 15) >> 1, v_tok = 8 * (j8 >> 2) + 4 * h + (j8 & 3);
  const uint32_t channel0 = half * (DC / 2);
  const uint32_t v_off = (v_tok * DC + ((((lane >> 4) & 1) ^ swizzle(v_tok)) << 4) + (lane & 1) * 8) ^ channel0;

  for (uint64_t x = begin; x < end;) {
    const uint64_t x1 = min(end, place.before + place.size);
    uint32_t tile0, tile1, tiles_all;
    tiles_of<L::kRows>(a, place, x, x1, &tile0, &tile1, &tiles_all);
    const LatentRequest &q = place.q;
    const bool whole = tile0 == 0 && tile1 == tiles_all;
    const uint32_t list = (uint32_t)q.rows * a.heads, r0 = place.block * L::kRows;
    const uint32_t r = r0 + 32 * rg + col;
    const bool here = r < list;
    const uint32_t tok = here ? r / a.heads : 0, head = here ? r - tok * a.heads : 0;
    const int32_t at = here ? q.base + (int32_t)tok : -1;       // the row's place
    const uint32_t w0 = min(r0 + 32 * rg, list - 1);
    const int32_t at_min = q.base + (int32_t)(w0 / a.heads);    // the first place of the wave's rows
    const int32_t *table = a.table + (size_t)place.req * a.max_pages;
    const uint32_t rounds = tile1 - tile0;

    if (rounds > 0 || whole) {
      Eight query[2 * L::kSteps], query_rot[4];
      {
        const Value *src = (const Value *)a.q + (int64_t)(q.first + (int32_t)tok) * a.q_row + (int64_t)head * a.q_head;
        auto get = [&](uint32_t d) {
          Eight e;
          if (!here) {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = (Value)0.0f;
          } else if (a.q_vec) {
            e = *(const Eight *)(src + d);
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = src[d + j];
          }
          return e;
        };
#pragma unroll
        for (int s = 0; s < 2 * L::kSteps; ++s) query[s] = get(32 * (s / 2) + 16 * h + 8 * (s % 2));
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          if (s < 2 || rot_steps > 1) query_rot[s] = get(DC + 32 * (s / 2) + 16 * h + 8 * (s % 2));
          else query_rot[s] = query_rot[0];
        }
      }
      for (int careful = 0;; careful = 1) {
        f32x16 acc[L::kBlocks];
#pragma unroll
        for (int b = 0; b < L::kBlocks; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[b][i] = 0;
        float m = -INFINITY, l = 0;
        if (threadIdx.x == 0) {
          lds.trouble = 0;
          lds.first_bad = INT32_MAX;
        }

        auto page_of = [&](uint32_t tile) {  // of the tile's token `lane`; -1 for none
          const int32_t t = (int32_t)(tile * kTile + lane);
          int32_t p = -1;
          if (tile < tile1 && t < q.len) p = table[(uint32_t)t >> a.page_shift];
          return (uint32_t)p < a.n_pages ? p : -1;
        };
        uint64_t valid_next = 0;
        uint32_t exps_next = 0;
        // asks for a tile of whose tokens the lanes have the pages
        auto ask = [&](uint32_t i, int32_t page) {
          Tile *to = &lds.tile[i % L::kBufs];
          valid_next = __ballot(page >= 0);
          if (valid_next == 0) return;
          const uint32_t safe = page < 0 ? 0 : (uint32_t)page, inside = (1u << a.page_shift) - 1;
          const uint32_t slot = (safe << a.page_shift) + (((tile0 + i) * kTile + lane) & inside);
#pragma unroll
          for (uint32_t j = 0; j < kLoads / kWaves; ++j) {
            const uint32_t k = j * kWaves + wave;  // this wave's
            const uint32_t first = __builtin_amdgcn_readlane(slot, k * kPer);
            const uint32_t chunk = (lane % kChunks) ^ swizzle((k * kPer + load_tok) & 15);
            load_to_lds(a.codes + (size_t)first * row_bytes, load_tok * row_bytes + chunk * 16, to->latent + k * 1024);
          }
#pragma unroll
          for (uint32_t j = 0; j < 4 / kWaves; ++j) {
            const uint32_t k = j * kWaves + wave;
            const uint32_t first = __builtin_amdgcn_readlane(slot, k * 16);
            const uint32_t chunk = ((lane & 3) ^ ((rot_tok >> 2) & 3)) & (a.rot / 16 - 1);
            load_to_lds(a.codes + (size_t)first * row_bytes, rot_tok * row_bytes + DC + chunk * 16, to->rot + k * 1024);
          }
          if (wave == 0) exps_next = *(const uint16_t *)(a.exps + 2 * (size_t)slot);
        };
        // waits for tile i, for all waves; what it needs beside the codes
        auto arrive = [&](uint32_t i, uint64_t valid) {
          Tile *tile = &lds.tile[i % L::kBufs];
          __builtin_amdgcn_s_waitcnt(0);  // this wave's part has arrived
          asm volatile("" ::: "memory");
          if (wave == 0) {
            const bool ok = valid >> lane & 1;
            const uint32_t ec = ok ? max(exps_next & 0xFF, 1u) : 127, er = ok ? max(exps_next >> 8 & 0xFF, 1u) : 127;
            if constexpr (T == UZIP_FP16) {  // fp16 holds codes times powers of two up to 1
              const uint32_t most = max(ec, er);
              tile->scale_c[lane] = pow2(max(127 + (int)ec - (int)most, 1));
              tile->scale_r[lane] = pow2(max(127 + (int)er - (int)most, 1));
              tile->mul[lane] = a.scale_log2 * pow2(most);
            } else {
              tile->scale_c[lane] = pow2(ec);
              tile->scale_r[lane] = pow2(er);
            }
            tile->e[lane] = (float)((int)ec - 127);
            tile->inv[lane] = pow2(254 - (int)ec);
          }
          if (~valid) {  // codes of places that are none count as zero
#pragma unroll 1
            for (uint32_t k = wave; k < kLoads; k += kWaves)
              if (!(valid >> (k * kPer + load_tok) & 1)) *(u32x4 *)(tile->latent + k * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
#pragma unroll 1
            for (uint32_t k = wave; k < 4; k += kWaves)
              if (!(valid >> (k * 16 + rot_tok) & 1)) *(u32x4 *)(tile->rot + k * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
          }
          __syncthreads();
          if (careful) {  // tokens that hold a NaN or an infinity are left out and noted
#pragma unroll 1
            for (uint32_t k = wave; k < kLoads; k += kWaves) {
              u32x4 *c = (u32x4 *)(tile->latent + k * 1024 + lane * 16);
              const bool bad = (not_numbers<CODE>(c->x) | not_numbers<CODE>(c->y) | not_numbers<CODE>(c->z) | not_numbers<CODE>(c->w)) != 0;
              const uint64_t bads = __ballot(bad) >> (load_tok * kChunks) & ((1ull << kChunks) - 1);
              if (bads) {
                *c = u32x4{0, 0, 0, 0};
                if (lane % kChunks == 0) atomicMin(&lds.first_bad, (int32_t)((tile0 + i) * kTile + k * kPer + load_tok));
              }
            }
            __syncthreads();
          }
        };
        // scores of this wave's 32 tokens of tile i, times log2(e), plus e_t; their largest
        auto score = [&](uint32_t i, uint64_t valid, f32x16 &s) {
          const Tile *tile = &lds.tile[i % L::kBufs];
          const int32_t t0 = (int32_t)((tile0 + i) * kTile);
          const float sc = tile->scale_c[32 * half + col], sr = tile->scale_r[32 * half + col];
          f32x16 s1;
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = s1[e] = 0;
#pragma unroll
          for (int k = 0; k < L::kSteps; ++k) {
            const u32x4 c = *(const u32x4 *)(tile->latent + (k_off ^ ((k & 7) << 5)) + (k >> 3) * 256);
            s = mfma16(eight_codes<CODE, T>(c.x, c.y, sc), query[2 * k], s);
            s1 = mfma16(eight_codes<CODE, T>(c.z, c.w, sc), query[2 * k + 1], s1);
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (k && rot_steps < 2) break;
            const u32x4 c = *(const u32x4 *)(tile->rot + (kr_off ^ (k << 5)));
            s = mfma16(eight_codes<CODE, T>(c.x, c.y, sr), query_rot[2 * k], s);
            s1 = mfma16(eight_codes<CODE, T>(c.z, c.w, sr), query_rot[2 * k + 1], s1);
          }
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const f32x4 e = *(const f32x4 *)(tile->e + 32 * half + 8 * g + 4 * h);
            f32x4 mul;
            if constexpr (T == UZIP_FP16) mul = *(const f32x4 *)(tile->mul + 32 * half + 8 * g + 4 * h);
#pragma unroll
            for (int k = 0; k < 4; ++k) s[4 * g + k] = __builtin_fmaf(s[4 * g + k] + s1[4 * g + k], T == UZIP_FP16 ? mul[k] : a.scale_log2, e[k]);
          }
          if (~valid || t0 + kTile - 1 > at_min) {
            const uint32_t mine = (uint32_t)(valid >> (32 * half + 4 * h));
            const int32_t upto = at - t0 - 32 * (int)half - 4 * (int)h;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int k = 8 * (e / 4) + e % 4;
              s[e] = (mine >> k & 1) && k <= upto ? s[e] : -INFINITY;
            }
          }
          float most = -INFINITY;
#pragma unroll
          for (int e = 0; e < 16; ++e) most = fmaxf(most, s[e]);
          most = fmaxf(most, other_half(most));
          if (h == 0) lds.most[rg][half][col] = most;
        };
        // The maxima of both halves are there: the weights, in this wave's registers and for the
        // other; the factor on the sums so far.
        auto weigh = [&](uint32_t i, const f32x16 &s, i32x4 *w) {
          const Tile *tile = &lds.tile[i % L::kBufs];
          const float most = fmaxf(lds.most[rg][0][col], lds.most[rg][1][col]);
          const float next = most > m + L::kLag ? most : m;
          const float f = next == m ? 1.0f : __builtin_amdgcn_exp2f(m - next);
          m = next;
          l *= f;
          const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const f32x4 inv = *(const f32x4 *)(tile->inv + 32 * half + 8 * g + 4 * h);
            float y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              y[k] = __builtin_amdgcn_exp2f(s[4 * g + k] - ref);
              l = __builtin_fmaf(y[k], inv[k], l);
              y[k] *= 32.0f;
            }
#pragma unroll
            for (int term = 0; term < TERMS; ++term) {
              int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
              c = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
              w[term][g] = c;
              if (term + 1 < TERMS) {
                const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
                y[0] = (y[0] - lo[0]) * 16.0f;
                y[1] = (y[1] - lo[1]) * 16.0f;
                y[2] = (y[2] - hi[0]) * 16.0f;
                y[3] = (y[3] - hi[1]) * 16.0f;
              }
            }
          }
          return f;
        };
        auto pass_on = [&](const i32x4 *w) {
#pragma unroll
          for (int term = 0; term < TERMS; ++term) lds.weights[rg][half][term][lane] = w[term];
        };
        auto take_over = [&](i32x4 *w) {
#pragma unroll
          for (int term = 0; term < TERMS; ++term) w[term] = lds.weights[rg][1 - half][term][lane];
        };
        // sums of tile i's latents with the weights of this wave's tokens and the other's
        auto add_up = [&](uint32_t i, const i32x4 *mine, const i32x4 *others) {
          const uint8_t *v = lds.tile[i % L::kBufs].latent;
          constexpr int kKind = CODE == UZIP_E4M3FN ? 0 : 1;
          i32x8 w[TERMS];
#pragma unroll
          for (int term = 0; term < TERMS; ++term)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              w[term][g] = half ? others[term][g] : mine[term][g];
              w[term][4 + g] = half ? mine[term][g] : others[term][g];
            }
#pragma unroll
          for (int b = 0; b < L::kBlocks; ++b) {
            i32x8 c;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const i32x2 p = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                  (__attribute__((address_space(3))) i32x2 *)(v + (v_off ^ ((b & 7) << 5)) + (b >> 3) * 256 + k * 16 * DC));
              c[2 * k] = p[0];
              c[2 * k + 1] = p[1];
            }
#pragma unroll
            for (int term = 0; term < TERMS; ++term)
              acc[b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(c, w[term], acc[b], kKind, 0, 0, 127, 0, 122 - 4 * term);
          }
        };

        if (rounds > 0) {
          i32x4 mine[TERMS], others[TERMS];
          ask(0, page_of(tile0));
          int32_t page_next = page_of(tile0 + 1);
          uint64_t valid = valid_next;
          arrive(0, valid);
          ask(1, page_next);
          page_next = page_of(tile0 + 2);
          f32x16 s;
          score(0, valid, s);
          __syncthreads();
          weigh(0, s, mine);
          pass_on(mine);
          for (uint32_t i = 1; i < rounds; ++i) {
            valid = valid_next;
            arrive(i, valid);
            ask(i + 1, page_next);
            page_next = page_of(tile0 + i + 2);
            take_over(others);
            score(i, valid, s);
            __syncthreads();
            i32x4 next[TERMS];
            const float f = weigh(i, s, next);
            add_up(i - 1, mine, others);
            if (__any(f != 1.0f)) {
#pragma unroll
              for (int b = 0; b < L::kBlocks; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[b][e] *= f;
            }
            pass_on(next);
#pragma unroll
            for (int term = 0; term < TERMS; ++term) mine[term] = next[term];
          }
          __syncthreads();
          take_over(others);
          add_up(rounds - 1, mine, others);
        }

        // the sums of a row's tokens from the halves of two waves
        l += other_half(l);
        if (h == 0) lds.l[rg][half][col] = l;
        float odd = l * 0.0f;
        if (!careful) {  // a sum that is not finite is computed again with care
#pragma unroll
          for (int b = 0; b < L::kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) odd = __builtin_fmaf(acc[b][e], 0.0f, odd);
          if (rounds == 0) __syncthreads();  // the mark is set after it was cleared
          if (__any(odd != 0.0f) && lane == 0) lds.trouble = 1;
        }
        __syncthreads();
        l = lds.l[rg][0][col] + lds.l[rg][1][col];
        const bool again = !careful && lds.trouble != 0;
        if (careful && at >= lds.first_bad) l = NAN;
        __syncthreads();
        if (again) continue;

        if (here) {
          if (whole) {
            const float f = l > 0 ? 1.0f / l : l == 0 ? 0.0f : NAN;
            Value *out = (Value *)a.out + (int64_t)(q.first + (int32_t)tok) * a.out_row + (int64_t)head * a.out_head + channel0;
#pragma unroll
            for (int b = 0; b < L::kBlocks; ++b)
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                Value y[4] __attribute__((aligned(8)));
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] = (Value)(acc[b][4 * g + k] * f);
                Value *to = out + 32 * b + 8 * g + 4 * h;
                if (a.out_vec) {
                  *(u32x2 *)to = *(u32x2 *)y;
                } else {
#pragma unroll
                  for (int k = 0; k < 4; ++k) to[k] = y[k];
                }
              }
            if (half == 0 && h == 0 && a.lse)
              a.lse[(size_t)(q.first + (int32_t)tok) * a.heads + head] = l == 0 ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
          } else {
            const size_t slot = 2 * (size_t)blockIdx.x + (begin > place.before ? 0 : 1), row = slot * L::kRows + 32 * rg + col;
#pragma unroll
            for (int b = 0; b < L::kBlocks; ++b)
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                f32x4 y;
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] = acc[b][4 * g + k];
                *(f32x4 *)(a.part_acc + row * DC + channel0 + 32 * b + 8 * g + 4 * h) = y;
              }
            if (half == 0 && h == 0) {
              a.part_ml[2 * row] = m;
              a.part_ml[2 * row + 1] = l;
            }
          }
        }
        break;
      }
    }
    x = x1;
    if (x < end && !next_block<L::kRows>(a, &place)) break;
  }
}

// The pieces of a block that several workgroups shared, one wave a row.  Workgroup (w, y): the block that
// the boundary between workgroups w and w + 1 cuts, if it is the first to cut it.
template <int T, int DC, int ROWS, int MIN>
__global__ __launch_bounds__(256) void latent_join_kernel(LatentArgs a) {
  typedef typename Elem<T>::type Value;
  uint64_t share = 0, x = 0, all_work = 0;
  Place p;
  if (!find_block<ROWS>(a, [&](uint64_t all, uint64_t *at) {
        share = share_of<MIN>(a, all);
        all_work = all;
        x = *at = share * (blockIdx.x + 1);
        return x < all;
      }, &p))
    return;
  if (p.before >= x || p.before < x - share) return;  // not cut there, or also before
  const uint32_t lane = threadIdx.x & 63, list = (uint32_t)p.q.rows * a.heads;
  const uint32_t i = blockIdx.y * 4 + (threadIdx.x >> 6), r = p.block * ROWS + i;
  if (r >= list) return;
  const uint32_t tok = r / a.heads, head = r - tok * a.heads;
  const uint32_t from = blockIdx.x, last = (uint32_t)((p.before + p.size - 1) / share);
  constexpr int N = DC / 64;
  float m = -INFINITY, l = 0, acc[N];
#pragma unroll
  for (int j = 0; j < N; ++j) acc[j] = 0;
  for (uint32_t w = from; w <= last; ++w) {
    const uint64_t x0 = max(share * w, p.before), x1 = min(min(share * (w + 1), p.before + p.size), all_work);
    uint32_t t0, t1, n;
    tiles_of<ROWS>(a, p, x0, x1, &t0, &t1, &n);
    if (t0 == t1 || (t0 == 0 && t1 == n)) {
      if (t0 != t1) return;  // one workgroup had all its tiles and wrote the result
      continue;
    }
    const size_t row = (2 * (size_t)w + (share * w > p.before ? 0 : 1)) * ROWS + i;
    const float pm = a.part_ml[2 * row], pl = a.part_ml[2 * row + 1];
    const float top = fmaxf(m, pm), f = m == top ? 1.0f : __builtin_amdgcn_exp2f(m - top), g = pm == top ? 1.0f : __builtin_amdgcn_exp2f(pm - top);
    const float *src = a.part_acc + row * DC + lane * N;
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      const f32x4 y = *(const f32x4 *)(src + j);
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[j + k] = acc[j + k] * f + y[k] * g;
    }
    l = l * f + pl * g;
    m = top;
  }
  const float f = l > 0 ? 1.0f / l : l == 0 ? 0.0f : NAN;
  Value *out = (Value *)a.out + (int64_t)(p.q.first + (int32_t)tok) * a.out_row + (int64_t)head * a.out_head + lane * N;
  Value y[N] __attribute__((aligned(16)));
#pragma unroll
  for (int j = 0; j < N; ++j) y[j] = (Value)(acc[j] * f);
  if (a.out_vec) {
#pragma unroll
    for (int j = 0; j < N; j += 4) *(u32x2 *)(out + j) = *(u32x2 *)(y + j);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) out[j] = y[j];
  }
  if (lane == 0 && a.lse) a.lse[(size_t)(p.q.first + (int32_t)tok) * a.heads + head] = l == 0 ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
}

}  // namespace uzip_kv
