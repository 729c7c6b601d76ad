// latent.h -- attention over the paged 8-bit latents, absorbed form: how a call is cut
// into pieces of work, and the kernels.
//
// A row q = (u, p) of a request sees tokens t of latents c and rotary keys r:
//   s_t = scale (u . c_t + p . r_t)   out = sum_t e^(s_t) c_t / sum_t e^(s_t)
// in one pass with a running maximum.  All heads share the tokens, so a request's rows are
// one list, row r = token r / heads, head r % heads, and a block of 32 or 64 of them
// reads each tile of 64 tokens once: a code is converted for the first product and taken as
// it is by the second.
//
// A token's scale 2^e belongs to its weight in the second product: with
//   g_t = s_t log2(e) + e_t,  w_t = 2^(g_t - m),  acc = sum w_t code_t,  l = sum w_t 2^-e_t
// out = acc / l, and the running maximum m is taken over g.  The weights of a tile count from the tile's own largest, 2^k of
// them from m as the matrix instruction's scale: of eight bits each, counted from m a long tail of small weights would end up as nothing
// beside one large one.  l holds its exponent apart, for the 2^-e_t of a row may lie 2^219 from one another.
#pragma once

#include <type_traits>
#include <utility>

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
  float *part_acc;  // [slot][32 rows][channels' half][32 channels][8 of them][lane][4]
  float *part_ml;   // [slot][row][4]: the power of two that the sums count from, l, l's power of two, none
  struct LatentCut *cuts;  // of each workgroup
  uint32_t n_pages, page_shift, rot;
  uint32_t n_rows, heads, max_pages, n_reqs;
  uint32_t groups;    // workgroups that the work is shared by
  uint32_t begin;     // what a block's beginning and end cost, in tiles
  FastDiv by_heads;
  double growth;      // by which a request's blocks grow from one to the next, in tiles
  float scale_log2;   // scale log2 e
  bool q_vec, out_vec;
};

constexpr int kTile = 64;  // tokens
constexpr int kAhead = 4;  // reads of the first product under way
// Sums of weights times codes are 2^-15 of what they stand for, so that the factor that makes them an output is a number of 32 bits
// wherever latents are: 2^(15 - 7) times a token's scale of up to 2^119, or a 2^29-th of 2^(15 - 7 - 4) times 2^-100.
constexpr int kDown = 15;
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

// The work of a request's first b blocks of ROWS rows, in tiles: each block a.begin for its beginning and end,
// and the tiles that its last row sees, which grow by ROWS / heads tokens from block to block.
// It only has to grow with b and be the same everywhere; a block's real tiles are spread over its share.  (Divisions of
// 64-bit numbers by such took 3 us of a workgroup's beginning: here and below they are of doubles, set right where
// the quotient has to be exact.)
template <int ROWS>
__device__ __forceinline__ uint64_t work_before(const LatentArgs &a, const LatentRequest &q, uint32_t b) {
  const int32_t seen = min(max(q.base + (int32_t)a.by_heads.div(min((uint32_t)q.rows * a.heads, (uint32_t)ROWS) - 1) + 1, 0), q.len);
  const uint64_t first = a.begin + ((uint32_t)seen + kTile - 1) / kTile;
  return b * first + (b < 2 ? 0 : (uint64_t)((double)((uint64_t)b * (b - 1) / 2) * a.growth));
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
// n / d, rounded down, both below 2^52
__device__ __forceinline__ uint64_t quotient(uint64_t n, uint64_t d) {
  uint64_t q = (uint64_t)((double)n / (double)d);
  if (q * d > n) --q;
  return q;
}
// The sum over the lanes up to and with this one: by moves between neighbouring lanes, then from rows of 16 lanes to the next.
__device__ __forceinline__ uint64_t wave_upto(uint64_t x) {
  auto add = [&](auto control, auto rows) {
    const uint32_t low = __builtin_amdgcn_update_dpp(0, (uint32_t)x, decltype(control)::value, decltype(rows)::value, 0xf, false);
    const uint32_t high = __builtin_amdgcn_update_dpp(0, (uint32_t)(x >> 32), decltype(control)::value, decltype(rows)::value, 0xf, false);
    x += (uint64_t)high << 32 | low;
  };
  typedef std::integral_constant<int, 0xf> Every;
  add(std::integral_constant<int, 0x111>{}, Every{});  // from the lane 1 before, of the row
  add(std::integral_constant<int, 0x112>{}, Every{});  // 2
  add(std::integral_constant<int, 0x114>{}, Every{});  // 4
  add(std::integral_constant<int, 0x118>{}, Every{});  // 8
  add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});  // lane 15 to row 1, 47 to row 3
  add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});  // lane 31 to rows 2 and 3
  return x;
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
  Place p{};
  for (uint32_t i = lo; i < hi; ++i) {
    p.q = latent_request(a, i);
    if (p.q.rows > 0) mine += work_before<ROWS>(a, p.q, blocks_of<ROWS>(a, p.q));
  }
  const uint64_t upto = wave_upto(mine), before = upto - mine;
  const uint64_t all = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(upto >> 32), 63) << 32 | (uint32_t)__builtin_amdgcn_readlane((uint32_t)upto, 63);
  uint64_t x;
  if (!x_of(all, &x) || x >= all) return false;
  const bool here = x >= before && x - before < mine;
  if (here) {
    uint64_t at = before;
    for (uint32_t i = lo; i < hi; ++i) {
      if (each > 1) p.q = latent_request(a, i);
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

// The same in all lanes, which the compiler is to know: it then holds it once for a wave.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) { return (uint64_t)uniform((uint32_t)(x >> 32)) << 32 | uniform((uint32_t)x); }
__device__ __forceinline__ void uniform(Place *p) {
  uint32_t words[sizeof(Place) / 4];
  __builtin_memcpy(words, p, sizeof(Place));
#pragma unroll
  for (uint32_t i = 0; i < sizeof(Place) / 4; ++i) words[i] = uniform(words[i]);
  __builtin_memcpy(p, words, sizeof(Place));
}

// f(0), f(1), ... f(N - 1), the arguments constants: what f indexes with them stays in registers.
template <int... I, class F>
__device__ __forceinline__ void times(std::integer_sequence<int, I...>, const F &f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void times(const F &f) {
  times(std::make_integer_sequence<int, N>{}, f);
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
__device__ __forceinline__ uint64_t share_of(const LatentArgs &a, uint64_t all) {
  const uint64_t each = quotient(all + a.groups - 1, a.groups);
  return each > 2 * a.begin ? each : 2 * a.begin;
}

// Tiles of the block that the work from x0 to x1 (within the block's) stands for.  A block's first a.begin are its
// beginning; where a share ends within them, the block is left to the next workgroup, whose share begins there.
template <int ROWS>
__device__ __forceinline__ void tiles_of(const LatentArgs &a, const Place &p, uint64_t x0, uint64_t x1, uint32_t *t0, uint32_t *t1) {
  const uint32_t list = (uint32_t)p.q.rows * a.heads, r1 = min(list, (p.block + 1) * ROWS);
  const int32_t seen = min(max(p.q.base + (int32_t)a.by_heads.div(r1 - 1) + 1, 0), p.q.len);
  const uint32_t all = ((uint32_t)seen + kTile - 1) / kTile;
  // rounded alike on both sides of a share's end; all of it gives `all` itself
  auto tiles = [&](uint64_t x) {
    const uint64_t done = x - p.before;
    return done <= a.begin ? 0u : done == p.size ? all : (uint32_t)((double)((done - a.begin) * all) / (double)(p.size - a.begin));
  };
  *t0 = tiles(x0);
  *t1 = x1 == p.before + p.size ? all : tiles(x1);
}
__device__ __forceinline__ bool leaves(const LatentArgs &a, const Place &p, uint64_t end) { return end < p.before + p.size && end - p.before <= a.begin; }

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
  float scale_c[kTile], scale_r[kTile];  // bf16: on the codes of the first product; fp16: on the products
  float e[kTile], inv[kTile];            // e_t, 2^-e_t
  uint64_t valid;                        // which tokens there are
  uint32_t far;                          // whether some e_t are far from others
  uint8_t fill[244];                     // the next tile begins at a multiple of 256 bytes
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

// A lane's value and that of the lane 32 away, in one order for both.
__device__ __forceinline__ f32x2 both_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f32x2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ float max_of_halves(float x) {
  const f32x2 r = both_halves(x);
  return fmaxf(r[0], r[1]);
}
__device__ __forceinline__ float sum_of_halves(float x) {
  const f32x2 r = both_halves(x);
  return r[0] + r[1];
}

// 16 bytes for each lane from base + offset on, to LDS side by side from byte `to` of it on; base and `to` are the same
// in all lanes.  Written out, so that the compiler does not know of it: else it has every later read of LDS
// wait until all have arrived.  The kernel waits itself, before the barrier that lets a tile be read.  (M0
// holds where to; nothing else here uses it.)
__device__ __forceinline__ void load_to_lds(const uint8_t *base, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(uniform(to)), "v"(offset), "s"(uniform((uint64_t)(uintptr_t)base)) : "memory");
}
// x 2^by; by may be infinite, or what is left of one infinity less another: then x is nothing.
__device__ __forceinline__ float times_pow2(float x, float by) { return __builtin_ldexpf(x, (int)__builtin_amdgcn_fmed3f(by, -500.0f, 500.0f)); }
// A sum and the power of two that it counts from, at first from none.
struct Sum {
  float x = 0, unit = -INFINITY;
  // where the sum stays in [1/2, 2^100), the unit stays; for sums of a wave's lanes
  __device__ __forceinline__ void add(float y, float y_unit) {
    const float next = x + times_pow2(y, y_unit - unit);
    if (__any(!(next < 0x1p100f))) {
      const float to = fmaxf(unit, y == 0 ? -INFINITY : y_unit + (float)__builtin_amdgcn_frexp_expf(y));
      x = times_pow2(x, unit - to) + times_pow2(y, y_unit - to);
      unit = to;
    } else {
      x = next;
    }
  }
  __device__ __forceinline__ void rebase(float to) {
    x = times_pow2(x, unit - to);
    unit = to;
  }
};
// The natural logarithm of x 2^unit, the same bits however the two are shared out: that depends on the wave's other rows.
__device__ __forceinline__ float log_of(float x, float unit) {
  const int e = __builtin_amdgcn_frexp_expf(x);
  return (unit + (float)e + __builtin_amdgcn_logf(__builtin_ldexpf(x, -e))) * 0.69314718055994530942f;
}
// x, from which nothing is computed before this place: what only a seldom taken branch needs would else be
// kept in registers through the loop around it.
__device__ __forceinline__ uint32_t only_here(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}
__device__ __forceinline__ uint32_t lds_at(const void *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }

// Bytes of four codes that are NaN or infinite: their sign bits.
template <int CODE>
__device__ __forceinline__ uint32_t not_numbers(uint32_t w) {
  return ((w & 0x7F7F7F7Fu) + (CODE == UZIP_E4M3FN ? 0x01010101u : 0x04040404u)) & 0x80808080u;
}

// RG groups of 32 rows, and four waves to each.  Two score: each takes half of a tile's tokens, with the queries in
// its registers, and makes their weights.  Two add: each takes half of the channels, with 32 x DC / 2 sums
// in its registers, and asks for the tiles.  Scoring and adding a tile are a round apart, so that a compute unit's
// matrix units have the products of the one beside the conversions and exponentials of the other; a wave that did both would
// need all 512 registers, and nothing would run beside it (32 requests of 1000 to 16383 tokens, 128 heads: 126 us, then 91; 94 with
// weights that keep their bits).
// Between the two barriers of a round the scores' maxima are exchanged.
// A round takes 1.7 us with 32 rows of 512, 1.9 with 64, 1.6 with 64 of 256 in fp16; of 512 with 64 rows that is 3800
// cycles, of which the matrix units work 2200: the rest is the wait of one kind of waves for the other, and the
// loads, which one wave's instructions ask for a kilobyte at a time.  64 requests of up to 8190 tokens of 512 + 64, 16
// heads: 43 us, 3.6 TB/s; 128 heads as above: 94 us, 825 TFLOP/s.
template <int T, int CODE, int DC, int RG>
struct Latent {
  static constexpr int kRows = 32 * RG, kThreads = 256 * RG, kBlocks = DC / 64, kSteps = DC / 32;
  static constexpr int kBufs = 3;      // tiles in LDS: one whose values are read, one whose keys are, one under way
  static constexpr float kTop = 7;     // a tile's largest weight is a code of 2^7 up to 2^8; less only where scores are past 2^24
  static constexpr float kLag = 4;     // how far a tile's may pass the reference of the sums
  typedef LatentTile<DC> Tile;
  struct Lds {
    Tile tile[kBufs];
    i32x4 weights[2][RG][2][LatentType<T>::kTerms][64];  // of two rounds: a half's tokens, as the lanes scored them
    f32x2 factor[2][RG][32];                             // on the sums before them; the weights' scale byte
    float most[RG][2][32];
    float m[RG][32];
    f32x2 l[RG][2][32];                                  // and its power of two
    uint32_t trouble;
    int32_t first_bad;
  };
  static_assert(sizeof(Lds) <= 160 * 1024, "a compute unit's LDS");
};

// A block that several workgroups share, from `from` to `last`: noted by the first of them.
struct LatentCut {
  uint32_t cut;           // 0: this workgroup is not the first of one
  int32_t first;          // row of the step's arrays of the request's first new token
  uint32_t r0, rows;      // of the request's list
  uint32_t from, last;
};

// The kernel's arguments, read once more: kept from its beginning to its end, those that only a block's beginning
// or end needs would take the registers of the loop.
__device__ __forceinline__ LatentArgs read_again() {
  auto p = (const __attribute__((address_space(4))) LatentArgs *)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  LatentArgs a;
  __builtin_memcpy(&a, (const LatentArgs *)p, sizeof(a));
  return a;
}

template <int T, int CODE, int DC, int RG>
__global__ __launch_bounds__(256 * RG, RG) void latent_kernel(LatentArgs args) {
  typedef Latent<T, CODE, DC, RG> L;
  typedef typename Elem<T>::type Value;
  typedef typename LatentType<T>::Eight Eight;
  typedef typename L::Tile Tile;
  typedef __attribute__((address_space(3))) i32x2 *LdsPair;
  typedef const __attribute__((address_space(3))) u32x4 *LdsFour;
  typedef const __attribute__((address_space(3))) f32x4 *LdsFloats;
  typedef const __attribute__((address_space(3))) float *LdsFloat;
  constexpr int TERMS = LatentType<T>::kTerms, kWaves = 2 * RG;  // of each kind
  extern __shared__ __align__(16) uint8_t lds_bytes[];
  typename L::Lds &lds = *(typename L::Lds *)lds_bytes;
  const uint32_t lane = threadIdx.x & 63, wave_of_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool adds = wave_of_all >= kWaves;
  const uint32_t wave = wave_of_all % kWaves, rg = wave / 2, half = wave % 2, col = lane & 31, h = lane >> 5;
  if (threadIdx.x == 0) args.cuts[blockIdx.x].cut = 0;
  uint64_t begin = 0, end = 0, share = 0;
  Place place;
  if (!find_block<L::kRows>(args, [&](uint64_t all, uint64_t *x) {
        share = uniform(share_of(args, all));
        begin = uniform(share * blockIdx.x);
        end = uniform((uint64_t)min(begin + share, all));
        *x = begin;
        return begin < all;
      }, &place))
    return;
  uniform(&place);
  if (begin - place.before <= args.begin) begin = place.before;

  // what does not change from block to block
  const uint32_t lds0 = lds_at(lds_bytes), tiles0 = lds0 + (uint32_t)offsetof(typename L::Lds, tile);
  const uint32_t row_bytes = DC + args.rot;
  // Loads are of 1 KiB at a time, 1024 / DC tokens of the latents or 16 of the rotary keys.
  constexpr uint32_t kPer = 1024 / DC, kChunks = DC / 16, kLoads = kTile / kPer;
  // Tiles lie at multiples of 256 bytes, so that the exclusive or of an address's swizzle may come last.
  static_assert(sizeof(Tile) % 256 == 0 && offsetof(typename L::Lds, tile) % 256 == 0 && offsetof(Tile, rot) % 256 == 0, "swizzled addresses");

  for (uint64_t x = begin; x < end && !leaves(args, place, end);) {
    const LatentArgs a = read_again();
    uniform(&place);
    const uint64_t x1 = min(end, place.before + place.size);
    uint32_t tile0, tile1;
    tiles_of<L::kRows>(a, place, x, x1, &tile0, &tile1);
    tile0 = uniform(tile0);
    tile1 = uniform(tile1);
    const LatentRequest &q = place.q;
    const bool whole = x == place.before && x1 == place.before + place.size;
    const uint32_t list = (uint32_t)q.rows * a.heads, r0 = place.block * L::kRows;
    const uint32_t rounds = tile1 - tile0;
    if (!whole && x == place.before && threadIdx.x == 0)
      a.cuts[blockIdx.x] = {1, q.first, r0, min(list - r0, (uint32_t)L::kRows), (uint32_t)blockIdx.x, (uint32_t)quotient(place.before + place.size - 1, share)};

    for (int careful = 0;; careful = 1) {
      bool again;
      if (threadIdx.x == 0) {
        lds.trouble = 0;
        lds.first_bad = INT32_MAX;
      }
      if (!adds) {
        // ---------------------------------------------------------------- scores
        const uint32_t r = r0 + 32 * rg + col;
        const bool here = r < list;
        const uint32_t tok = here ? a.by_heads.div(r) : 0, head = here ? r - tok * a.heads : 0;
        const int32_t at = here ? q.base + (int32_t)tok : -1;                                  // the row's place
        const int32_t at_min = q.base + (int32_t)a.by_heads.div(min(r0 + 32 * rg, list - 1));      // the first of the wave's rows
        const float scale_log2 = a.scale_log2;
        const bool two = a.rot > 32;
        Eight query[2 * L::kSteps + 4];
        {
          const Value *src = (const Value *)a.q + (int64_t)(q.first + (int32_t)tok) * a.q_row + (int64_t)head * a.q_head;
          const bool vec = a.q_vec;
#pragma unroll
          for (int s = 0; s < 2 * L::kSteps + 4; ++s) {
            const uint32_t d = 32 * (s / 2) + 16 * h + 8 * (s % 2);
            Eight e;
            if (!here || (s >= 2 * L::kSteps + 2 && !two)) {
#pragma unroll
              for (int j = 0; j < 8; ++j) e[j] = (Value)0.0f;
            } else if (vec) {
              e = *(const Eight *)(src + d);
            } else {
#pragma unroll
              for (int j = 0; j < 8; ++j) e[j] = src[d + j];
            }
            query[s] = e;
          }
        }
        // token col of this wave's half, chunk 2 k + h
        const uint32_t k_off = (32 * half + col) * DC + ((h ^ swizzle(col & 15)) << 4);
        const uint32_t r_off = (uint32_t)offsetof(Tile, rot) + (32 * half + col) * 64 + ((h ^ ((col >> 2) & 3)) << 4);
        float m = -INFINITY;  // a power of two, as are the tiles'
        Sum l;
#pragma unroll
        for (int term = 0; term < TERMS; ++term) lds.weights[1][rg][half][term][lane] = i32x4{0, 0, 0, 0};  // before the first
        lds.factor[1][rg][col] = f32x2{1, 0};
        for (uint32_t i = 0; i < rounds; ++i) {
          __syncthreads();  // tile i is there
          if (careful) __syncthreads();
          const uint32_t tile = tiles0 + i % L::kBufs * (uint32_t)sizeof(Tile);
          const uint32_t of_token = tile + 4 * (32 * half + col), of_four = tile + 4 * (32 * half + 4 * h);
          [[maybe_unused]] const float sc = *(LdsFloat)(uintptr_t)(of_token + offsetof(Tile, scale_c)), sr = *(LdsFloat)(uintptr_t)(of_token + offsetof(Tile, scale_r));
          const uint32_t k_at = tile + k_off, r_at = tile + r_off;
          // The order is written down, between barriers to the compiler's scheduler: reads some steps ahead.
          constexpr int kReads = L::kSteps + 2;
          auto chunk = [&](int k) {
            return k < L::kSteps ? *(LdsFour)(uintptr_t)((k_at ^ ((k & 7) << 5)) + (k >> 3) * 256) : *(LdsFour)(uintptr_t)(r_at ^ ((k - L::kSteps) << 5));
          };
          f32x16 s, of_rot;  // fp16: the latents' and the rotary keys' products apart
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = of_rot[e] = 0;
          u32x4 c[kAhead];
#pragma unroll
          for (int k = 0; k < kAhead; ++k) c[k] = chunk(k);
          __builtin_amdgcn_sched_barrier(0);
          times<kReads>([&](auto number) {
            constexpr int k = decltype(number)::value;
            const u32x4 now = c[k % kAhead];
            if constexpr (k + kAhead < kReads) c[k % kAhead] = chunk(k + kAhead);
            const float scale = T == UZIP_FP16 ? 1.0f : k < L::kSteps ? sc : sr;
            f32x16 &to = T == UZIP_FP16 && k >= L::kSteps ? of_rot : s;
            // (the last is of the rotary keys' second 32 channels: where there are none an infinity of the first would be times 0)
            if (k <= L::kSteps || two) {
              to = mfma16(eight_codes<CODE, T>(now.x, now.y, scale), query[2 * k], to);
              to = mfma16(eight_codes<CODE, T>(now.z, now.w, scale), query[2 * k + 1], to);
            }
            __builtin_amdgcn_sched_barrier(0);
          });
          // times log2(e), plus e_t; the largest
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const f32x4 e = *(LdsFloats)(uintptr_t)(of_four + offsetof(Tile, e) + 32 * g);
            if constexpr (T == UZIP_FP16) {
              const f32x4 by_c = *(LdsFloats)(uintptr_t)(of_four + offsetof(Tile, scale_c) + 32 * g);
              const f32x4 by_r = *(LdsFloats)(uintptr_t)(of_four + offsetof(Tile, scale_r) + 32 * g);
#pragma unroll
              for (int k = 0; k < 4; ++k) s[4 * g + k] = __builtin_fmaf(s[4 * g + k], by_c[k], __builtin_fmaf(of_rot[4 * g + k], by_r[k], e[k]));
            } else {
#pragma unroll
              for (int k = 0; k < 4; ++k) s[4 * g + k] = __builtin_fmaf(s[4 * g + k], scale_log2, e[k]);
            }
          }
          const int32_t t0 = (int32_t)((tile0 + i) * kTile);
          const uint64_t valid = lds.tile[i % L::kBufs].valid;
          const bool far = uniform(lds.tile[i % L::kBufs].far) != 0;
          if (~valid || t0 + kTile - 1 > at_min) {
            const uint32_t there = (uint32_t)(valid >> (32 * half + 4 * h));
            const int32_t upto = at - t0 - 32 * (int)half - 4 * (int)h;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int k = 8 * (e / 4) + e % 4;
              s[e] = (there >> k & 1) && k <= upto ? s[e] : -INFINITY;
            }
          }
          float most = -INFINITY;
#pragma unroll
          for (int e = 0; e < 16; ++e) most = fmaxf(most, s[e]);
          most = max_of_halves(most);
          if (h == 0) lds.most[rg][half][col] = most;
          __syncthreads();

          // the reference of this tile's weights and of the sums, the factor on the sums so far, the weights
          f32x4 scales[4];  // 2^-e_t; e_t where some are far from others
          const uint32_t at_scales = of_four + (far ? (uint32_t)offsetof(Tile, e) : (uint32_t)offsetof(Tile, inv));
#pragma unroll
          for (int g = 0; g < 4; ++g) scales[g] = *(LdsFloats)(uintptr_t)(at_scales + 32 * g);
          most = fmaxf(lds.most[rg][0][col], lds.most[rg][1][col]);
          const float ref = __builtin_floorf(most) - L::kTop;
          const float next = ref > m + L::kLag ? ref : m;
          if (half == 0 && h == 0)  // 2^(ref - m - kDown) as an exponent byte; what is below 2^-127 ends there
            lds.factor[i & 1][rg][col] = f32x2{next == m ? 1.0f : times_pow2(1.0f, m - next), __int_as_float(127 - kDown + (int)fmaxf(ref - next, kDown - 127.0f))};
          m = next;
          const float from = ref == -INFINITY ? 0.0f : ref;
          float sum = 0;  // of the divisor's terms
          if (far) {  // which are numbers where the weights may be none
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float x = s[e] - from;
              sum += __builtin_amdgcn_exp2f(x - scales[e / 4][e % 4]);
              s[e] = __builtin_amdgcn_exp2f(x);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              s[e] = __builtin_amdgcn_exp2f(s[e] - from);
              sum = __builtin_fmaf(s[e], scales[e / 4][e % 4], sum);
            }
          }
          i32x4 w[TERMS];
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            float y[4] = {s[4 * g], s[4 * g + 1], s[4 * g + 2], s[4 * g + 3]};
#pragma unroll
            for (int term = 0; term < TERMS; ++term) {
              int code = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
              code = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], code, true);
              w[term][g] = code;
              if (term + 1 < TERMS) {
                const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(code, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(code, true);
                y[0] = (y[0] - lo[0]) * 16.0f;
                y[1] = (y[1] - lo[1]) * 16.0f;
                y[2] = (y[2] - hi[0]) * 16.0f;
                y[3] = (y[3] - hi[1]) * 16.0f;
              }
            }
          }
#pragma unroll
          for (int term = 0; term < TERMS; ++term) lds.weights[i & 1][rg][half][term][lane] = w[term];
          l.add(sum, ref);
        }
        // the adding waves' last round
        __syncthreads();
        l.rebase(max_of_halves(l.unit));
        l.x = sum_of_halves(l.x);
        if (h == 0) {
          lds.l[rg][half][col] = f32x2{l.x, l.unit};
          lds.m[rg][col] = m;  // what the weights' sums count from
        }
        if (__any(l.x * 0.0f != 0.0f) && lane == 0) lds.trouble = 1;
        __syncthreads();
        again = !careful && lds.trouble != 0;
        __syncthreads();
      } else {
        // ---------------------------------------------------------------- sums
        f32x16 acc[L::kBlocks];
#pragma unroll
        for (int b = 0; b < L::kBlocks; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[b][e] = 0;
        const uint32_t channel0 = half * (DC / 2);
        // eight tokens by 16 channels for 16 lanes, from this wave's first channel on
        const uint32_t j8 = (lane & 15) >> 1, v_tok = 8 * (j8 >> 2) + 4 * h + (j8 & 3);
        const uint32_t v_off = (v_tok * DC + ((((lane >> 4) & 1) ^ swizzle(v_tok)) << 4) + (lane & 1) * 8) ^ channel0;
        // Where a lane's part of load k = j kWaves + wave lies from its 16 tokens' first code on: the same for every kPeriod-th j, for
        // swizzle() of a sum without carries is the exclusive or of its parts'.
        constexpr int kWaveTokens = kWaves * kPer, kPeriod = 16 / kWaveTokens;
        static_assert(16 % kWaveTokens == 0, "a round of loads lies in one page");
        uint32_t load_off[kPeriod];
#pragma unroll
        for (int j = 0; j < kPeriod; ++j) {
          const uint32_t t = j * kWaveTokens + wave * kPer + lane / kChunks;
          load_off[j] = t * row_bytes + (((lane % kChunks) ^ swizzle(t)) << 4);
        }
        const uint32_t rot_off = lane / 4 * row_bytes + DC + ((((lane & 3) ^ ((lane >> 4) & 3)) & (a.rot / 16 - 1)) << 4);
        const int32_t *table = a.table + (size_t)place.req * a.max_pages;

        auto page_of = [&](uint32_t i) {  // of tile i's token `lane`; -1 for none
          const int32_t t = (int32_t)((tile0 + i) * kTile + lane);
          int32_t p = -1;
          if (i < rounds && t < q.len) p = table[(uint32_t)t >> a.page_shift];
          return (uint32_t)p < a.n_pages ? p : -1;
        };
        // What the loads of a tile go by: where its tokens' codes lie, one to a lane, and which of them there are.
        struct Next {
          uint64_t at, valid;
          uint32_t exps;
        };
        auto next_of = [&](uint32_t i, int32_t page) {  // codes of some page where there is none
          const uint32_t slot = ((page < 0 ? 0 : (uint32_t)page) << a.page_shift) + (((tile0 + i) * kTile + lane) & ((1u << a.page_shift) - 1));
          return Next{(uint64_t)(uintptr_t)a.codes + (uint64_t)slot * row_bytes, (uint64_t)__ballot(page >= 0),
                      wave == 0 ? (uint32_t) * (const uint16_t *)(a.exps + 2 * (size_t)slot) : 0u};
        };
        // this wave's loads of tile i
        constexpr int kCodes = kLoads / kWaves;
        auto ask = [&](uint32_t i, const Next &n) {
          auto from = [&](uint32_t token) {
            const uint32_t low = __builtin_amdgcn_readlane((uint32_t)n.at, token), high = __builtin_amdgcn_readlane((uint32_t)(n.at >> 32), token);
            return (const uint8_t *)(uintptr_t)((uint64_t)high << 32 | low);
          };
          const uint32_t to = tiles0 + i % L::kBufs * (uint32_t)sizeof(Tile) + wave * 1024;
          times<kCodes>([&](auto number) {
            constexpr int j = decltype(number)::value;
            load_to_lds(from(j * kWaveTokens / 16 * 16), load_off[j % kPeriod], to + (uint32_t)offsetof(Tile, latent) + j * kWaves * 1024);
          });
          times<4 / kWaves>([&](auto number) {
            constexpr int j = decltype(number)::value;
            load_to_lds(from(16 * (j * kWaves + wave)), rot_off, to + (uint32_t)offsetof(Tile, rot) + j * kWaves * 1024);
          });
        };
        // what a tile needs beside the codes, from its tokens' exponents
        auto scales = [&](uint32_t i, const Next &n) {
          if (wave != 0) return;
          const uint32_t lane = only_here(threadIdx.x & 63);
          Tile *tile = &lds.tile[i % L::kBufs];
          const bool ok = n.valid >> lane & 1;
          const uint32_t ec = ok ? max(n.exps & 0xFF, 1u) : 127, er = ok ? max(n.exps >> 8 & 0xFF, 1u) : 127;
          // fp16 holds the codes themselves, but not codes of latents and rotary keys whose scales differ by 2^15 or more
          tile->scale_c[lane] = T == UZIP_FP16 ? a.scale_log2 * pow2(ec) : pow2(ec);
          tile->scale_r[lane] = T == UZIP_FP16 ? a.scale_log2 * pow2(er) : pow2(er);
          tile->e[lane] = (float)((int)ec - 127);
          tile->inv[lane] = pow2(254 - (int)ec);
          // weights of up to 2^-134 of the largest are numbers: enough for the divisor where no two e_t are more than 100 apart
          const int first = __builtin_amdgcn_readlane((int)ec, n.valid ? __ffsll((unsigned long long)n.valid) - 1 : 0);
          const bool far = __any(ok && abs((int)ec - first) > 50);
          if (lane == 0) {
            tile->valid = n.valid;
            tile->far = far;
          }
        };

        Next then{};  // of tile i + 1
        int32_t page_after = -1;
        uint64_t now_valid = 0;
        if (rounds > 0) {
          const Next now = next_of(0, page_of(0));
          now_valid = now.valid;
          ask(0, now);
          then = next_of(1, page_of(1));
          page_after = page_of(2);
          scales(0, now);
        }
        uint64_t valid = now_valid;
        for (uint32_t i = 0; i <= rounds; ++i) {
          __builtin_amdgcn_s_waitcnt(0);  // this wave's part of tile i has arrived
          asm volatile("" ::: "memory");
          if (~valid && i < rounds) {  // codes of places that are none count as zero
            Tile *tile = &lds.tile[i % L::kBufs];
            const uint32_t lane = only_here(threadIdx.x & 63), tok = lane / kChunks;
#pragma unroll 1
            for (uint32_t k = wave; k < kLoads; k += kWaves)
              if (!(valid >> (k * kPer + tok) & 1)) *(u32x4 *)(tile->latent + k * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
#pragma unroll 1
            for (uint32_t k = wave; k < 4; k += kWaves)
              if (!(valid >> (k * 16 + lane / 4) & 1)) *(u32x4 *)(tile->rot + k * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
          }
          __syncthreads();
          if (careful && i < rounds) {  // tokens that hold a NaN or an infinity are left out and noted
            Tile *tile = &lds.tile[i % L::kBufs];
            const uint32_t lane = only_here(threadIdx.x & 63), tok = lane / kChunks;
#pragma unroll 1
            for (uint32_t k = wave; k < kLoads; k += kWaves) {
              u32x4 *c = (u32x4 *)(tile->latent + k * 1024 + lane * 16);
              const bool bad = (not_numbers<CODE>(c->x) | not_numbers<CODE>(c->y) | not_numbers<CODE>(c->z) | not_numbers<CODE>(c->w)) != 0;
              const uint64_t bads = __ballot(bad) >> (tok * kChunks) & ((1ull << kChunks) - 1);
              if (bads) {
                *c = u32x4{0, 0, 0, 0};
                if (lane % kChunks == 0) atomicMin(&lds.first_bad, (int32_t)((tile0 + i) * kTile + k * kPer + tok));
              }
            }
            __syncthreads();
          }
          if (rounds == 0) break;
          if (i + 1 < rounds) {
            ask(i + 1, then);
            scales(i + 1, then);
          }
          valid = then.valid;
          then = next_of(i + 2, page_after);
          page_after = page_of(i + 3);

          // The products of tile i - 1; in the first round of tile 0 and weights that are 0.
          const uint32_t before = tiles0 + (i ? i - 1 : 0) % L::kBufs * (uint32_t)sizeof(Tile) + v_off;
          const f32x2 factor = lds.factor[(i + 1) & 1][rg][col];
          const float f = factor[0];
          const int scale = __float_as_int(factor[1]);
          constexpr int kTermScales = 0x777B7F;  // 2^0, 2^-4, 2^-8
          i32x8 w[TERMS], v[2];
#pragma unroll
          for (int term = 0; term < TERMS; ++term) {
            const i32x4 first = lds.weights[(i + 1) & 1][rg][0][term][lane], second = lds.weights[(i + 1) & 1][rg][1][term][lane];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              w[term][g] = first[g];
              w[term][4 + g] = second[g];
            }
          }
          if (__any(f != 1.0f)) {
#pragma unroll
            for (int b = 0; b < L::kBlocks; ++b)
#pragma unroll
              for (int e = 0; e < 16; ++e) acc[b][e] *= f;
          }
          auto values = [&](int b) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const i32x2 p = __builtin_amdgcn_ds_read_tr8_b64_v2i32((LdsPair)(uintptr_t)((before ^ ((b & 7) << 5)) + (b >> 3) * 256 + k * 16 * DC));
              v[b % 2][2 * k] = p[0];
              v[b % 2][2 * k + 1] = p[1];
            }
          };
          values(0);
#pragma unroll
          for (int b = 0; b < L::kBlocks; ++b) {
            if (b + 1 < L::kBlocks) values(b + 1);
            times<TERMS>([&](auto number) {
              constexpr int term = decltype(number)::value;
              acc[b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(v[b % 2], w[term], acc[b], CODE == UZIP_E4M3FN ? 0 : 1, 0, term, kTermScales, 0, scale);
            });
            if (b == L::kBlocks / 2 - 1 && i < rounds) __syncthreads();
          }
        }
        // a sum that is not finite is computed again with care
        float odd = 0;
        if (!careful) {
#pragma unroll
          for (int b = 0; b < L::kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) odd = __builtin_fmaf(acc[b][e], 0.0f, odd);
        }
        if (__any(odd != 0.0f) && lane == 0) lds.trouble = 1;
        __syncthreads();
        again = !careful && lds.trouble != 0;
        const uint32_t col = only_here(threadIdx.x & 31), h = only_here(threadIdx.x & 63) >> 5, r = r0 + 32 * rg + col;
        const uint32_t tok = a.by_heads.div(r), head = r - tok * a.heads;
        const f32x2 l0 = lds.l[rg][0][col], l1 = lds.l[rg][1][col];
        const float unit = fmaxf(l0[1], l1[1]), m = lds.m[rg][col];
        float l = times_pow2(l0[0], l0[1] - unit) + times_pow2(l1[0], l1[1] - unit);
        if (careful && q.base + (int32_t)tok >= lds.first_bad) l = NAN;
        __syncthreads();
        if (!again && r < list) {
          const LatentArgs a = read_again();
          if (whole) {
            const float f = times_pow2(l > 0 ? 1.0f / l : l == 0 ? 0.0f : NAN, m - unit + kDown);
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
              a.lse[(size_t)(q.first + (int32_t)tok) * a.heads + head] = l == 0 ? -INFINITY : log_of(l, unit);
          } else {
            const size_t slot = 2 * (size_t)blockIdx.x + (begin > place.before ? 0 : 1), row = slot * L::kRows + 32 * rg + col;
            f32x4 *part = (f32x4 *)a.part_acc + (((slot * RG + rg) * 2 + half) * L::kBlocks * 4) * 64 + 32 * h + col;  // as the lanes hold them
#pragma unroll
            for (int b = 0; b < L::kBlocks && rounds > 0; ++b)
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                f32x4 y;
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] = acc[b][4 * g + k];
                part[(4 * b + g) * 64] = y;
              }
            if (half == 0 && h == 0) *(f32x4 *)(a.part_ml + 4 * row) = f32x4{m, l, unit, 0};
          }
        }
      }
      if (!again) break;
    }
    x = x1;
    if (x < end && !next_block<L::kRows>(read_again(), &place)) break;
  }
}

// The pieces of a block that several workgroups shared.  Workgroup (w, y): 32 rows by 32 channels, the y-th such, of the block
// that workgroup w was the first of; a lane has what one of the adding waves' lanes had, so that pieces are read as they were
// written, 1024 bytes at a time (row by row, they were written 16 bytes at a time: 5.6 us of a workgroup's end, now 2.9).
template <int T, int DC, int RG>
__global__ __launch_bounds__(256) void latent_join_kernel(LatentArgs a) {
  typedef typename Elem<T>::type Value;
  constexpr int kBlocks = DC / 64, kRows = 32 * RG;
  const LatentCut c = a.cuts[blockIdx.x];
  const uint32_t lane = threadIdx.x & 63, col = lane & 31, h = lane >> 5, g = threadIdx.x >> 6;
  const uint32_t b = blockIdx.y % kBlocks, half = blockIdx.y / kBlocks % 2, rg = blockIdx.y / kBlocks / 2, i = 32 * rg + col;
  if (!c.cut || 32 * rg >= c.rows) return;
  // the piece of workgroup w: the second of its slots where the block begins within its share
  auto slot_of = [&](uint32_t w) { return 2 * (size_t)w + (w == c.from ? 1 : 0); };
  auto ml_of = [&](uint32_t w) { return *(const f32x4 *)(a.part_ml + 4 * (slot_of(w) * kRows + i)); };
  constexpr uint32_t kAtOnce = 4;  // pieces that are read side by side
  float m = -INFINITY;
  Sum sum;
  f32x4 acc = {0, 0, 0, 0};
  for (uint32_t w0 = c.from; w0 <= c.last; w0 += kAtOnce) {
    f32x4 ml[kAtOnce];
    f32x4 part[kAtOnce];
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      const uint32_t w = min(w0 + k, c.last);
      ml[k] = ml_of(w);
      part[k] = ((const f32x4 *)a.part_acc)[((((slot_of(w) * RG + rg) * 2 + half) * kBlocks + b) * 4 + g) * 64 + lane];
    }
    float top = m;
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) top = fmaxf(top, ml[k][0]);
    const float f = m == top ? 1.0f : times_pow2(1.0f, m - top);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] *= f;
    m = top;
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      if (w0 + k > c.last || ml[k][1] == 0) continue;  // a piece of no weight has no sums
      const float fk = ml[k][0] == top ? 1.0f : times_pow2(1.0f, ml[k][0] - top);
      sum.add(ml[k][1], ml[k][2]);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(part[k][e], fk, acc[e]);
    }
  }
  if (i >= c.rows) return;
  const uint32_t r = c.r0 + i, tok = a.by_heads.div(r), head = r - tok * a.heads;
  const float l = sum.x, f = times_pow2(l > 0 ? 1.0f / l : l == 0 ? 0.0f : NAN, m - sum.unit + kDown);
  Value *out = (Value *)a.out + (int64_t)(c.first + (int32_t)tok) * a.out_row + (int64_t)head * a.out_head + half * (DC / 2) + 32 * b + 8 * g + 4 * h;
  Value y[4] __attribute__((aligned(8)));
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (Value)(acc[e] * f);
  if (a.out_vec) {
    *(u32x2 *)out = *(u32x2 *)y;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = y[e];
  }
  if (blockIdx.y % (2 * kBlocks) == 0 && g == 0 && h == 0 && a.lse)
    a.lse[(size_t)(c.first + (int32_t)tok) * a.heads + head] = l == 0 ? -INFINITY : log_of(l, sum.unit);
}

}  // namespace uzip_kv
