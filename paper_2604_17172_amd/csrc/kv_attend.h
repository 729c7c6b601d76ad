// kv_attend.h -- attention of new tokens over the 8-bit pages: how a call is
// cut into pieces of work, and the kernels.
//
// For a row q at place p and the tokens t that it sees,
//   out = sum_t e^(s_t) v_t / sum_t e^(s_t),   s_t = scale q . k_t
// taken in one pass over the tokens: with a running maximum m,
//   l = sum 2^(s'_t - m), acc = sum 2^(s'_t - m) v_t   (s' = s log2 e)
// and a factor 2^(m - m') on both when m grows to m'.  Two pieces of one row,
// over different tokens, join the same way.
//
// A request's rows of one cache head -- new tokens times the query heads that
// share it -- are one list, row r = token r / group, head r % group; blocks of
// them read the same keys and values, so a group's heads cost one read.  The
// unit along the tokens is a step of 64.
#pragma once

#include <utility>

#include "kv_device.h"

namespace uzip_kv {

struct AttendArgs {
  Cache c;
  const void *q;
  void *out;
  float *lse;
  int64_t q_row, q_head, out_row, out_head;
  const int32_t *table, *lens, *q_start;
  float *part_acc;   // [row][dim]: acc of pieces that are joined, a row for each of their blocks' rows
  float *part_ml;    // [row][2]: their m and l
  uint32_t n_rows, n_q_heads, group, max_pages, n_reqs, window;
  uint32_t units;    // compute units
  float scale_log2;  // |scale| log2 e
  bool negate;       // scale < 0: the queries change sign instead
  bool q_vec, out_vec;  // rows start at multiples of 16 (q) and 4 elements (out), so loads and stores may be wide
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kMostUnits = 256;  // compute units that the workspace is sized for, whatever the device
constexpr int kStep = 64;      // tokens of a step
constexpr int kMinSteps = 8;   // steps of a piece: two for each of a workgroup's waves

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

// How far a score may pass the running maximum before that is taken anew: weights up
// to 2^8 cost no precision, and most steps need no exchange between lanes and no
// rescaling.  Such weights must not push the sum of weights times values out of range:
// 2^8, 2^31 tokens, codes below 2^16 and scales up to 2^72 stay below 2^127.  A step with a
// larger scale lets no score pass, so that each of its weights is at most 1.
__device__ __forceinline__ float lag_for(float value_scale) { return value_scale > 0x1p72f ? 0.0f : 8.0f; }

// Lists of more rows than this go to the many-rows kernel, in blocks of 128.  By few
// and by many rows, us, in bf16 (16 heads over 4):
//   16 requests of 4000 tokens, 72 rows: dim 64 32 and 36, 96 36 and 50, 128 55 and 52,
//   256 99 and 107; 32 of 96 rows: 128 98 and 69, 256 200 and 182; 16 of 160 rows: 64 44
//   and 55, 96 50 and 62, 192 84 and 132; 16 of 256: 64 51 and 57, 96 60 and 65, 192 107
//   and 136; but 4 of 60000 tokens, 200 rows: 96 174 and 166, 192 370 and 356.
// So few rows would still be faster up to 256 over some thousand tokens of dim 64, 96 and
// 192, and many rows from 72 on of dim 128; the lines are for long contexts.
// fp32 has no such kernel: its three terms make the matrix units the bound, which few
// rows reach as well.
constexpr uint32_t kManyRows = 128;
constexpr uint32_t many_from(uint32_t dim) { return dim % 128 ? 160 : 96; }

// ------------------------------------------------------------------ pieces of work
struct Request {
  int32_t first, rows, len, base;  // first row of the step's arrays, new tokens, tokens, place of the first new one
};

// Request i; the one past the last holds the rows of no request.
__device__ __forceinline__ Request request(const AttendArgs &a, uint32_t i) {
  const int64_t n = a.n_rows;
  const int64_t lo = min(max((int64_t)(i ? a.q_start[i] : (a.n_reqs ? a.q_start[0] : 0)), (int64_t)0), n);
  const int64_t hi = i < a.n_reqs ? min(max((int64_t)a.q_start[i + 1], lo), n) : n;
  Request r;
  r.first = (int32_t)lo;
  r.rows = (int32_t)(hi - lo);
  const int64_t len = i < a.n_reqs ? min((int64_t)max(a.lens[i], 0), (int64_t)a.max_pages << a.c.page_shift) : 0;
  r.len = (int32_t)min(len, (int64_t)INT32_MAX - 2 * kStep);
  r.base = r.len - r.rows;
  return r;
}

// Tokens [lo, hi) that rows r0 .. r1 - 1 of a request's list can see.
__device__ __forceinline__ void seen_range(const AttendArgs &a, const Request &q, uint32_t r0, uint32_t r1, int32_t *lo, int32_t *hi) {
  const int32_t p0 = q.base + (int32_t)(r0 / a.group), p1 = q.base + (int32_t)((r1 - 1) / a.group);
  *hi = min(max(p1 + 1, 0), q.len);
  *lo = a.window && (int64_t)p0 + 1 > a.window ? (int32_t)((int64_t)p0 + 1 - a.window) : 0;
}

// The tokens that the row at a place sees: first .. first + span.
struct Seen {
  int32_t first;
  uint32_t span;
};
__device__ __forceinline__ Seen seen_by(const AttendArgs &a, int32_t place) {
  if (place < 0) return {INT32_MAX, 0};  // none: no token is that far
  const int32_t first = a.window && (int64_t)place + 1 > a.window ? (int32_t)((int64_t)place + 1 - a.window) : 0;
  return {first, (uint32_t)(place - first)};
}
__device__ __forceinline__ bool sees(const Seen &s, int32_t t) { return (uint32_t)t - (uint32_t)s.first <= s.span; }

// The lists that one kernel takes: those of least to most rows, in blocks of rows.
struct Lists {
  uint32_t least, most;
  uint32_t rows, shift;  // rows = 2^shift
  uint32_t slots;        // first row of the workspace for their pieces
  bool many;             // the many-rows kernel's
  uint32_t per_unit;     // then: pieces for a compute unit
};

struct Piece {
  Request q;
  uint32_t req, head, block;     // which rows
  uint32_t split, splits;        // which part of their tokens
  size_t part;                   // row of the workspace of part 0's first row; the others follow, a block's rows apart
};

__device__ __forceinline__ uint32_t blocks_of(const AttendArgs &a, const Request &q, const Lists &l) {
  const uint32_t list = (uint32_t)q.rows * a.group;  // at most UZIP_KV_MAX_ROW_HEADS
  return list >= l.least && list <= l.most ? (list + l.rows - 1) >> l.shift : 0u;
}

// The most steps that a block of `rows` rows of the request can have.
__device__ __forceinline__ uint32_t steps_of(const AttendArgs &a, const Request &q, uint32_t rows) {
  uint32_t tokens = (uint32_t)q.len;
  if (a.window) tokens = min(tokens, min(a.window, (uint32_t)INT32_MAX) + rows + kStep);
  return (tokens + kStep - 1) / kStep;
}

__device__ __forceinline__ uint64_t wave_scan64(uint64_t x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = __shfl_up(x, o);
    if ((int)(threadIdx.x & 63) >= o) x += y;
  }
  return x;
}

// How many steps make a piece, from the steps and blocks of all lists.
//
// Many rows: two pieces for each compute unit, four of dim 64, whose workgroups are
// lighter (512 new tokens of dim 64 over 14000: 159 us, by two 180).
// Few rows: where there are fewer blocks than compute units, so that about one piece
// comes to each, and hardly ever a few more, which would be a second round (steps / S +
// blocks / 2 pieces come of S, more where the blocks are alike): one round of longer
// pieces beats two of shorter ones, a piece's beginning and end being a few us (a
// request of 100000 tokens, 8 heads: 50 us, with two to a unit 58; 8 requests of 2000 to
// 4000 tokens 22 and 23, by the rule that follows 26).  Where there are more, or at least
// half as many as units and long ones (18 requests of 7500 to 30000 tokens, 8 heads of
// 128, 144 blocks: 144 us, by the rule above 159; of dim 64 74 and 101; 20 of 1000 to 4000
// of dim 256 by that rule 52, by this one 54), pieces of no less than 32 steps and up to four
// to a unit, which even out requests of unlike lengths (64 requests of 1 to 8000 tokens:
// 112 us, with one to a unit 126).
constexpr uint32_t kFewPieces = 4, kLongPiece = 32;
constexpr uint32_t many_pieces(uint32_t dim) { return dim == 64 ? 4 : 2; }
__device__ __forceinline__ uint32_t piece_steps(const AttendArgs &a, const Lists &l, uint64_t steps, uint64_t blocks) {
  const bool many = l.many;
  const bool few_blocks = !many && blocks < a.units && (2 * blocks < a.units || steps < 2 * kLongPiece * blocks);
  const uint32_t pieces = many ? l.per_unit * a.units : few_blocks ? a.units - (uint32_t)blocks * 3 / 4 : kFewPieces * a.units;
  const uint32_t least = many || few_blocks ? kMinSteps : kLongPiece;
  if (steps <= (uint64_t)least * pieces) return least;
  return (uint32_t)min((steps + pieces - 1) / pieces, (uint64_t)INT32_MAX);
}

// Pieces and slots are added up in one word, pieces in the low bits.  Row starts that do
// not ascend make requests share rows, so that each may have all blocks; slots stay
// below twice the pieces that piece_steps aims at.
constexpr int kPieceBits = 40;
static_assert((UZIP_KV_MAX_REQUESTS + 1) * (UZIP_KV_MAX_ROW_HEADS / 16 + 1024ull) + 2 * kFewPieces * kMostUnits < 1ull << kPieceBits,
              "the pieces of all requests");
static_assert(2 * kFewPieces * kMostUnits < 1ull << (64 - kPieceBits) && many_pieces(64) <= kFewPieces, "their slots");

// Which piece of the lists is number `index`, found by the whole workgroup.  A block
// of n steps is split only where n > S = piece_steps, into ceil(n / S) < 2 n / S pieces:
// with at most k units of pieces' worth of steps, k = kFewPieces or many_pieces, there are at
// most k units + blocks pieces, k units split blocks and 2 k units slots of the
// workspace.  With JOIN the index counts the blocks that were split instead.  Every
// workgroup sums over the requests for itself: two scans.
template <int THREADS, bool JOIN>
__device__ bool find_piece(const AttendArgs &a, const Lists &lists, uint32_t index, Piece *out) {
  constexpr int kWaves = THREADS / 64;
  const uint32_t rows = lists.rows;
  __shared__ uint64_t part[3 * kWaves];
  __shared__ Piece found;
  const uint32_t tid = threadIdx.x, wave = tid >> 6, n = a.n_reqs + 1;  // with the rows of no request
  const uint32_t each = (n + THREADS - 1) / THREADS, lo = min(n, tid * each), hi = min(n, lo + each);
  // each thread's first request, most often its only one, is looked up once
  const Request first = lo < hi ? request(a, lo) : Request{};
  auto request_at = [&](uint32_t i) { return i == lo ? first : request(a, i); };
  uint64_t steps = 0, blocks = 0;
  for (uint32_t i = lo; i < hi; ++i) {
    const Request q = request_at(i);
    const uint64_t b = blocks_of(a, q, lists);
    blocks += b;
    steps += b * steps_of(a, q, rows);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    steps += __shfl_xor(steps, o);
    blocks += __shfl_xor(blocks, o);
  }
  if ((tid & 63) == 0) {
    part[wave] = steps;
    part[kWaves + wave] = blocks;
  }
  __syncthreads();
  steps = blocks = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    steps += part[w];
    blocks += part[kWaves + w];
  }
  steps *= a.c.heads;
  blocks *= a.c.heads;
  const uint32_t length = piece_steps(a, lists, steps, blocks);
  auto count = [&](const Request &q, uint32_t *splits) {
    const uint32_t b = blocks_of(a, q, lists);
    const uint32_t n = steps_of(a, q, rows);
    *splits = n > length ? (n + length - 1) / length : 1u;
    const uint64_t pieces = (uint64_t)b * a.c.heads * (JOIN ? (*splits > 1 ? 1u : 0u) : *splits);
    return pieces | (*splits > 1 ? (uint64_t)b * a.c.heads * *splits : 0) << kPieceBits;
  };
  uint64_t mine = 0;
  uint32_t splits;
  for (uint32_t i = lo; i < hi; ++i) mine += count(request_at(i), &splits);
  const uint64_t incl = wave_scan64(mine);
  if ((tid & 63) == 63) part[2 * kWaves + wave] = incl;
  __syncthreads();
  uint64_t at = incl - mine, total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < (int)wave) at += part[2 * kWaves + w];
    total += part[2 * kWaves + w];
  }
  constexpr uint64_t kPieces = (1ull << kPieceBits) - 1;
  if (index >= (total & kPieces)) return false;
  for (uint32_t i = lo; i < hi; ++i) {
    const Request q = request_at(i);
    const uint64_t c = count(q, &splits);
    const uint64_t before = at & kPieces;
    if (index >= before && index - before < (c & kPieces)) {
      const uint32_t rest = index - (uint32_t)before;
      Piece p;
      p.q = q;
      p.req = i;
      p.head = rest % a.c.heads;
      const uint32_t up = rest / a.c.heads;
      p.split = JOIN ? 0 : up % splits;
      p.splits = splits;
      p.block = JOIN ? up : up / splits;
      p.part = lists.slots + ((at >> kPieceBits) + (uint64_t)(p.block * a.c.heads + p.head) * splits) * rows;
      found = p;
    }
    at += c;
  }
  __syncthreads();
  if (JOIN) {
    *out = found;
    return true;
  }
  // The same in all lanes, which the compiler is to know: it then holds them once for a
  // wave, and few spill where the kernel holds a second computation of its piece (64
  // requests, dim 128 in blocks of 32: 73 us, else 97).
  uint32_t words[sizeof(Piece) / 4];
  __builtin_memcpy(words, &found, sizeof(Piece));
#pragma unroll
  for (uint32_t i = 0; i < sizeof(Piece) / 4; ++i) words[i] = __builtin_amdgcn_readfirstlane(words[i]);
  __builtin_memcpy(out, words, sizeof(Piece));
  return true;
}

// f(0), f(1), ... f(N - 1), the arguments constants: arrays that f indexes with them stay in registers.
template <int... I, class F>
__device__ __forceinline__ void static_for(std::integer_sequence<int, I...>, const F &f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(const F &f) {
  static_for(std::make_integer_sequence<int, N>{}, f);
}

// ------------------------------------------------------------------ fragments
// Matrix instructions of 16 x 16 x 32: a lane holds, of the first operand, eight
// values of row lane % 16; of the second, eight of column lane % 16; of the
// result, rows 4 (lane / 16) + 0..3 of column lane % 16.  Which place of the
// contraction a lane's values have is free as long as both operands agree.
//
// bf16: the query as it is, probabilities in one bf16 term, 8 bits, as many as the output
// has.  That takes the error against 64 bits from 1.6e-3, which rounding the output once
// costs, to 1.9e-3 (64 requests of up to 8191 tokens; a prompt of 8192 1.6e-3 and 2.0e-3).  A
// second term gives the 1.6e-3, and takes a third more where many rows share the
// keys: the prompt 862 us for 647, 64 requests of 32 rows 96 for 72; single tokens 116
// for 115.
template <int T>
struct Query {
  static constexpr int kTerms = 1, kProbs = 1;
};
template <>
struct Query<UZIP_FP16> {  // fp16 keys (codes are exact in it); probabilities need 16 bits: two terms
  static constexpr int kTerms = 1, kProbs = 2;
};
template <>
struct Query<UZIP_FP32> {  // 24 bits: three bf16 terms each
  static constexpr int kTerms = 3, kProbs = 3;
};

// An infinite value or a NaN is what it is for every row that sees it, however small
// its weight, and nothing for a row that does not.  Products do not give that: a weight
// of 0, or a later term of a probability, which may be 0 or negative, times it is no
// infinity, and a factor of 0 on a sum that holds it neither.  A piece is computed as if
// there were none; if its sums come out not finite, it is computed again with such
// codes left out, and they are added after that (with one such value in each request 64
// requests of up to 8191 tokens 155 us, else 116; a prompt of 8192 856, else 647).  A test of
// every step's codes instead costs all calls up to half (e5m2, dim 128 in blocks of 32: 111
// us, this 73; dim 192 61 and 47).
__device__ __forceinline__ float not_finite(float so_far, f32x4 x) {  // NaN from the first infinity or NaN on, else 0
#pragma unroll
  for (int j = 0; j < 4; ++j) so_far = __builtin_fmaf(x[j], 0.0f, so_far);
  return so_far;
}

// x * w, w >= 0, where an infinity stays one whatever w is.
__device__ __forceinline__ f32x4 weighed(f32x4 x, float w) {
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = fabsf(x[j]) == INFINITY ? x[j] : x[j] * w;
  return x;
}

union Frag {
  bf16x8 b;
  f16x8 h;
  bf16x2 b2[4];
  f16x2 h2[4];
  u32x4 u;
};

// Eight codes (two words) as a fragment, times 2^(e - 127) where scale = 2^(e - 127).
template <int CODE>
__device__ __forceinline__ Frag codes_bf16(uint32_t lo, uint32_t hi, float scale) {
  Frag f;
  if constexpr (CODE == UZIP_E4M3FN) {
    f.b2[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    f.b2[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    f.b2[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    f.b2[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  } else {
    f.b2[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, false);
    f.b2[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, true);
    f.b2[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, false);
    f.b2[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, true);
  }
  return f;
}
template <int CODE>
__device__ __forceinline__ Frag codes_f16(uint32_t lo, uint32_t hi) {
  Frag f;
  if constexpr (CODE == UZIP_E4M3FN) {
    f.h2[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false);
    f.h2[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    f.h2[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false);
    f.h2[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
  } else {
    f.h2[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(lo, 1.0f, false);
    f.h2[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(lo, 1.0f, true);
    f.h2[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(hi, 1.0f, false);
    f.h2[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(hi, 1.0f, true);
  }
  return f;
}

// Keys of a query's type: the scale goes onto the score instead.
template <int T, int CODE>
__device__ __forceinline__ Frag key_frag(uint32_t lo, uint32_t hi) {
  if constexpr (T == UZIP_FP16) return codes_f16<CODE>(lo, hi);
  else return codes_bf16<CODE>(lo, hi, 1.0f);
}

template <int T>
__device__ __forceinline__ f32x4 score_mfma(const Frag &k, const Frag *q, f32x4 c) {
  if constexpr (T == UZIP_FP16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(k.h, q[0].h, c, 0, 0, 0);
#pragma unroll
  for (int i = Query<T>::kTerms - 1; i >= 0; --i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.b, q[i].b, c, 0, 0, 0);
  return c;
}

// Eight values, or their negatives, as the query's fragments: fp32 in three bf16 terms, each the
// rounding of what the ones before left.
template <int T>
__device__ __forceinline__ void query_frag(const typename Elem<T>::type *x, bool wide, bool negate, Frag *f) {
  if constexpr (T == UZIP_FP32) {
    float v[8];
    if (wide) {
      *(float4 *)v = ((const float4 *)x)[0];
      *(float4 *)(v + 4) = ((const float4 *)x)[1];
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = x[j];
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        f[i].b[j] = (__bf16)v[j];
        v[j] -= (float)f[i].b[j];
      }
  } else if (wide) {
    f[0].u = *(const u32x4 *)x;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (T == UZIP_FP16) f[0].h[j] = x[j];
      else f[0].b[j] = x[j];
    }
  }
  if (negate) {
#pragma unroll
    for (int i = 0; i < Query<T>::kTerms; ++i) f[i].u = u32x4{f[i].u.x ^ 0x80008000u, f[i].u.y ^ 0x80008000u, f[i].u.z ^ 0x80008000u, f[i].u.w ^ 0x80008000u};
  }
}

// Words of eight codes that are NaN or infinite; the sign bits say where.
template <int CODE>
__device__ __forceinline__ uint32_t unbounded(uint32_t w) {
  return ((w & 0x7F7F7F7Fu) + (CODE == UZIP_E4M3FN ? 0x01010101u : 0x04040404u)) & 0x80808080u;
}

// Of four codes at tokens t .. t + 3, those with lo <= token < hi; zeros elsewhere.
__device__ __forceinline__ uint32_t keep_tokens(uint32_t w, int32_t t, int32_t lo, int32_t hi) {
  const int32_t below = min(max(lo - t, 0), 4), upto = min(max(hi - t, 0), 4);
  const uint32_t high = upto == 4 ? 0xFFFFFFFFu : (1u << (8 * upto)) - 1u;
  const uint32_t low = below == 4 ? 0xFFFFFFFFu : (1u << (8 * below)) - 1u;
  return w & high & ~low;
}

// Four results next to each other.
template <int T>
__device__ __forceinline__ void store4(typename Elem<T>::type *out, f32x4 x, bool wide) {
  typedef typename Elem<T>::type Value;
  Value o[4] __attribute__((aligned(16)));
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] = (Value)x[j];
  if (wide) {
    if constexpr (sizeof(Value) == 2) *(u32x2 *)out = *(u32x2 *)o;
    else *(u32x4 *)out = *(u32x4 *)o;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = o[j];
  }
}

// Zero for codes that are NaN or infinite.
template <int CODE>
__device__ __forceinline__ uint32_t bounded(uint32_t w) {
  return w & ~((unbounded<CODE>(w) >> 7) * 0xFFu);
}
template <int CODE>
__device__ __forceinline__ bool any_unbounded(u32x4 w) {
  return (unbounded<CODE>(w.x) | unbounded<CODE>(w.y) | unbounded<CODE>(w.z) | unbounded<CODE>(w.w)) != 0;
}
template <int CODE>
__device__ __forceinline__ u32x4 bounded(u32x4 w) {
  return u32x4{bounded<CODE>(w.x), bounded<CODE>(w.y), bounded<CODE>(w.z), bounded<CODE>(w.w)};
}

// 1 for each of the eight codes that is NaN (kind 0), infinite (1) or minus
// infinite (2), 0 for the others, as a fragment.
template <int CODE>
__device__ __forceinline__ Frag class_frag(uint32_t lo, uint32_t hi, int kind) {
  Frag f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float x = decode<CODE>(((j < 4 ? lo : hi) >> (8 * (j % 4))) & 0xFFu);
    f.b[j] = (__bf16)((kind == 0 ? x != x : x == (kind == 1 ? INFINITY : -INFINITY)) ? 1.0f : 0.0f);
  }
  return f;
}
__device__ __forceinline__ float class_value(int kind) { return kind == 0 ? NAN : kind == 1 ? INFINITY : -INFINITY; }

// ------------------------------------------------------------------ few rows
// One workgroup for up to 16 NM rows (NM 1 or 2) and a piece of their tokens, one
// wave a step of 64 tokens, everything from memory straight into registers:
//   S^T = K Q^T, four tiles of 16 tokens: row m of tile i is token 16 (m / 4) + 4
//   i + m % 4, so that a lane ends up with the scores of 16 tokens in a row for one
//   query -- which is just what it needs of the second product's
//   O^T = V^T P^T, whose first operand it loads as 16 bytes of a channel.
// No score or code crosses lanes; pages of 16 tokens and more never split a lane's
// load.  Each wave keeps its own maximum, sum and acc; they join at the end.
//
// Bound by the cache's bytes: the next step's keys are asked for when this one's
// scores are done, its values after this one's products, so that 16 KiB (dim 128) of
// each wave are under way.  4 requests of 120000 to 131072 tokens, 8 heads of 128: 1.03
// GB in 182 us, 5.6 TB/s (a copy of 1 GiB: 5.1 read and written); 64 of up to 8191 and
// 3 empty ones: 538 MB in 109 us, 4.9 TB/s.  The smallest call, 38 tokens: 7.1 us, of
// which 3 are any launch's and the rest a chain of lengths, table, codes and joins.
template <int D, int NM>
struct FewRows {
  static constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = 16 * NM;
  static constexpr int kPairs = D / 64, kOdd = (D / 32) % 2, kKeySteps = D / 32, kChannels = D / 16;
};

// Without LEAVE_OUT false where a NaN or an infinity was met: then nothing was written,
// and the piece is computed from its beginning with it, so that nothing is kept in
// registers for that (a loop around the steps alone: dim 256 102 us, this 73).
template <int T, int CODE, int D, int NM, bool LEAVE_OUT>
__device__ __forceinline__ bool few_rows_piece(const AttendArgs &a, const Lists &lists, uint32_t index,
                                               float (&join_acc)[2][16 * NM][D + 4],
                                               float (&join_ml)[FewRows<D, NM>::kWaves][16 * NM][2],
                                               uint32_t (&join_odd)[FewRows<D, NM>::kWaves]) {
  typedef FewRows<D, NM> F;
  typedef typename Elem<T>::type Value;
  constexpr int TERMS = Query<T>::kTerms, PROBS = Query<T>::kProbs;
  Piece pc;
  if (!find_piece<F::kThreads, false>(a, lists, index, &pc)) return true;
  const uint32_t lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
  // One number for a wave, which saves a few registers (16 requests of 4000 tokens, 72 rows:
  // dim 96 36 us, else 42, for a third workgroup fits a compute unit; 256 99 and 104; blocks of
  // 32, dim 128: 73 and 82), but not in blocks of 16 of dim 128 (64 requests: 106, without 104).
  constexpr bool kOneNumber = NM == 2 || D != 128;
  const uint32_t wave = kOneNumber ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : threadIdx.x >> 6;
  const uint32_t list = (uint32_t)pc.q.rows * a.group, r0 = pc.block * F::kRows, P = a.c.page;
  int32_t lo, hi;
  seen_range(a, pc.q, r0, min(list, r0 + F::kRows), &lo, &hi);
  const uint32_t step0 = (uint32_t)lo / kStep, steps = hi > lo ? ((uint32_t)hi + kStep - 1) / kStep - step0 : 0;
  const uint32_t share = (steps + pc.splits - 1) / pc.splits;
  const uint32_t begin = step0 + min(steps, pc.split * share), end = step0 + min(steps, (pc.split + 1) * share);

  // the rows' queries and places
  Frag q[NM][F::kKeySteps][TERMS];
  Seen seen[NM];
#pragma unroll
  for (int n = 0; n < NM; ++n) {
    const uint32_t r = r0 + 16 * n + col;
    const bool here = r < list;
    const uint32_t tok = here ? r / a.group : 0, head = pc.head * a.group + (here ? r % a.group : 0);
    seen[n] = seen_by(a, here ? pc.q.base + (int32_t)tok : -1);
    const Value *x = (const Value *)a.q + (int64_t)(pc.q.first + (int32_t)tok) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
    for (int s = 0; s < F::kKeySteps; ++s) {
      const uint32_t d = s < 2 * F::kPairs ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
      query_frag<T>(x + d, a.q_vec, a.negate, q[n][s]);
    }
  }
  // the first and the last place of the block's rows
  const int32_t p_min = pc.q.base + (int32_t)(r0 / a.group), p_max = pc.q.base + (int32_t)((min(list, r0 + F::kRows) - 1) / a.group);

  auto all_see = [&](int32_t t0) {
    return t0 + kStep - 1 <= p_min && (a.window == 0 || (int64_t)t0 > (int64_t)p_max - a.window);
  };

  f32x4 acc[NM][F::kChannels];
  float m[NM], l[NM];
#pragma unroll
  for (int n = 0; n < NM; ++n) {
    m[n] = -INFINITY;
    l[n] = 0;
#pragma unroll
    for (int c = 0; c < F::kChannels; ++c) acc[n][c] = f32x4{0, 0, 0, 0};
  }

  const int32_t *table = a.table + (size_t)pc.req * a.max_pages;
  const size_t page_bytes = (size_t)P * D;
  // page of the 16 tokens from t on; -1 past the tokens
  auto page_of = [&](int32_t t) { return t < hi ? table[(uint32_t)t >> a.c.page_shift] : -1; };
  const int32_t key_chunk = 16 * (int32_t)(col >> 2), value_chunk = 16 * (int32_t)g;
  u32x4 k16[4][F::kPairs > 0 ? F::kPairs : 1], v16[F::kChannels];
  u32x2 k8[4];
  uint32_t e_k, e_v;
  bool page_here;
  auto load_keys = [&](int32_t t0, int32_t page) {
    page = (uint32_t)page < a.c.n_pages ? page : 0;
    const uint8_t *row = a.c.k + ((size_t)page * a.c.heads + pc.head) * page_bytes +
                         (((uint32_t)(t0 + key_chunk) & (P - 1)) + (col & 3)) * D;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int s = 0; s < F::kPairs; ++s) k16[i][s] = *(const u32x4 *)(row + i * 4 * D + 64 * s + 16 * g);
      if (F::kOdd) k8[i] = *(const u32x2 *)(row + i * 4 * D + 64 * F::kPairs + 8 * g);
    }
  };
  auto load_values = [&](int32_t t0, int32_t page) {
    page_here = (uint32_t)page < a.c.n_pages;
    const size_t ph = (size_t)(page_here ? page : 0) * a.c.heads + pc.head;
    const uint8_t *at = a.c.v + ph * page_bytes + (size_t)col * P + ((uint32_t)(t0 + value_chunk) & (P - 1));
#pragma unroll
    for (int c = 0; c < F::kChannels; ++c) v16[c] = *(const u32x4 *)(at + (size_t)16 * c * P);
    e_k = a.c.k_exp[ph];
    e_v = a.c.v_exp[ph];
  };

  uint32_t step = begin + wave;
  int32_t key_page = -1, value_page = -1;
  if (step < end) {
    const int32_t t0 = (int32_t)(step * kStep);
    key_page = page_of(t0 + key_chunk);
    value_page = page_of(t0 + value_chunk);
    load_keys(t0, key_page);
    load_values(t0, value_page);
    if (step + F::kWaves < end) {
      key_page = page_of(t0 + F::kWaves * kStep + key_chunk);
      value_page = page_of(t0 + F::kWaves * kStep + value_chunk);
    }
  }
  for (; step < end; step += F::kWaves) {
    const int32_t t0 = (int32_t)(step * kStep), t_next = t0 + F::kWaves * kStep;
    const bool more = step + F::kWaves < end;
    f32x4 s[NM][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int n = 0; n < NM; ++n) s[n][i] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < F::kKeySteps; ++ks) {
        Frag k;
        if (ks < 2 * F::kPairs) {
          const u32x4 w = k16[i][ks / 2];
          k = ks % 2 ? key_frag<T, CODE>(w.z, w.w) : key_frag<T, CODE>(w.x, w.y);
        } else {
          k = key_frag<T, CODE>(k8[i].x, k8[i].y);
        }
#pragma unroll
        for (int n = 0; n < NM; ++n) s[n][i] = score_mfma<T>(k, q[n][ks], s[n][i]);
      }
    }
    const float ks_scale = pow2((int)e_k) * a.scale_log2, vs = page_here ? pow2((int)e_v) : 1.0f;
    const bool page_ok = page_here;
    if (more) load_keys(t_next, key_page);

    // scores, and what is not seen
    const bool whole = all_see(t0) && __all(page_ok);
    const int32_t t_lane = t0 + value_chunk;
    float c = ks_scale;  // what a score is still to be multiplied by
    if (!whole) {
#pragma unroll
      for (int n = 0; n < NM; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            s[n][i][j] = page_ok && sees(seen[n], t_lane + 4 * i + j) ? s[n][i][j] * c : -INFINITY;
      c = 1;
    }

    const float lag = lag_for(vs);
    Frag p[NM][2][PROBS];
#pragma unroll
    for (int n = 0; n < NM; ++n) {
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, s[n][i][j]);
      top *= c;
      if (__any(top > m[n] + lag)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m2 = fmaxf(m[n], top);
        const float shrink = m2 == -INFINITY ? 1.0f : exp2_fast(m[n] - m2);
        m[n] = m2;
        l[n] *= shrink;
#pragma unroll
        for (int c = 0; c < F::kChannels; ++c) acc[n][c] *= shrink;
      }
      const float base = m[n] == -INFINITY ? 0.0f : m[n];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float x = exp2_fast(__builtin_fmaf(s[n][i][j], c, -base));
          l[n] += x;
#pragma unroll
          for (int t = 0; t < PROBS; ++t) {
            p[n][i / 2][t].b[4 * (i % 2) + j] = (__bf16)x;
            if (t + 1 < PROBS) x -= (float)p[n][i / 2][t].b[4 * (i % 2) + j];
          }
        }
    }

    // codes that no row sees count as zero, for 0 times NaN is not 0
    if (!whole) {
#pragma unroll
      for (int c = 0; c < F::kChannels; ++c) {
        u32x4 w = v16[c];
        w.x = page_ok ? keep_tokens(w.x, t_lane, lo, hi) : 0u;
        w.y = page_ok ? keep_tokens(w.y, t_lane + 4, lo, hi) : 0u;
        w.z = page_ok ? keep_tokens(w.z, t_lane + 8, lo, hi) : 0u;
        w.w = page_ok ? keep_tokens(w.w, t_lane + 12, lo, hi) : 0u;
        v16[c] = w;
      }
    }
    if constexpr (LEAVE_OUT) {
#pragma unroll
      for (int c = 0; c < F::kChannels; ++c) v16[c] = bounded<CODE>(v16[c]);
    }

#pragma unroll
    for (int c = 0; c < F::kChannels; ++c) {
      const u32x4 w = v16[c];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const Frag v = u ? codes_bf16<CODE>(w.z, w.w, vs) : codes_bf16<CODE>(w.x, w.y, vs);
#pragma unroll
        for (int n = 0; n < NM; ++n)
#pragma unroll
          for (int t = PROBS - 1; t >= 0; --t)
            acc[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.b, p[n][u][t].b, acc[n][c], 0, 0, 0);
      }
    }
    if (more) {
      load_values(t_next, value_page);
      if (step + 2 * F::kWaves < end) {
        key_page = page_of(t_next + F::kWaves * kStep + key_chunk);
        value_page = page_of(t_next + F::kWaves * kStep + value_chunk);
      }
    }
  }

  if constexpr (LEAVE_OUT) {  // the rows that see such a value get it
#pragma unroll 1
    for (step = begin + wave; step < end; step += F::kWaves) {
      const int32_t t0 = (int32_t)(step * kStep), t_lane = t0 + value_chunk;
      load_values(t0, page_of(t_lane));
#pragma unroll
      for (int c = 0; c < F::kChannels; ++c) {
        if (!__any(any_unbounded<CODE>(v16[c]))) continue;
#pragma unroll 1
        for (int kind = 0; kind < 3; ++kind)
#pragma unroll
          for (int n = 0; n < NM; ++n) {
            f32x4 hits = {0, 0, 0, 0};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              Frag see;
#pragma unroll
              for (int j = 0; j < 8; ++j) see.b[j] = (__bf16)(page_here && sees(seen[n], t_lane + 8 * u + j) ? 1.0f : 0.0f);
              const Frag is = u ? class_frag<CODE>(v16[c].z, v16[c].w, kind) : class_frag<CODE>(v16[c].x, v16[c].y, kind);
              hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(is.b, see.b, hits, 0, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (hits[j] > 0) acc[n][c][j] += class_value(kind);
          }
      }
    }
  }

  // join the waves: common maximum, then acc in two rounds through LDS
#pragma unroll
  for (int n = 0; n < NM; ++n) {
    l[n] += __shfl_xor(l[n], 16);
    l[n] += __shfl_xor(l[n], 32);
    if (g == 0) {
      join_ml[wave][16 * n + col][0] = m[n];
      join_ml[wave][16 * n + col][1] = l[n];
    }
  }
  if constexpr (!LEAVE_OUT) {
    float sums = 0;
#pragma unroll
    for (int n = 0; n < NM; ++n)
#pragma unroll
      for (int c = 0; c < F::kChannels; ++c) sums = not_finite(sums, acc[n][c]);
    const bool odd = __any(sums != 0);
    if (lane == 0) join_odd[wave] = odd;
  }
  __syncthreads();
  if constexpr (!LEAVE_OUT) {
    uint32_t odd = 0;
#pragma unroll
    for (int w = 0; w < F::kWaves; ++w) odd |= join_odd[w];
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(odd), 0)) return false;
  }
#pragma unroll
  for (int n = 0; n < NM; ++n) {
    float top = -INFINITY, sum = 0;
#pragma unroll
    for (int w = 0; w < F::kWaves; ++w) top = fmaxf(top, join_ml[w][16 * n + col][0]);
#pragma unroll
    for (int w = 0; w < F::kWaves; ++w) {
      const float mw = join_ml[w][16 * n + col][0];
      sum += mw == top ? join_ml[w][16 * n + col][1] : join_ml[w][16 * n + col][1] * exp2_fast(mw - top);
    }
    const float shrink = m[n] == top ? 1.0f : exp2_fast(m[n] - top);
    m[n] = top;
    l[n] = sum;
#pragma unroll
    for (int c = 0; c < F::kChannels; ++c) acc[n][c] = LEAVE_OUT ? weighed(acc[n][c], shrink) : acc[n][c] * shrink;
  }
#pragma unroll
  for (int half = 2; half >= 1; half >>= 1) {
    if (wave >= (uint32_t)half && wave < 2u * half)
#pragma unroll
      for (int n = 0; n < NM; ++n)
#pragma unroll
        for (int c = 0; c < F::kChannels; ++c) *(f32x4 *)&join_acc[wave - half][16 * n + col][16 * c + 4 * g] = acc[n][c];
    __syncthreads();
    if (wave < (uint32_t)half)
#pragma unroll
      for (int n = 0; n < NM; ++n)
#pragma unroll
        for (int c = 0; c < F::kChannels; ++c) acc[n][c] += *(const f32x4 *)&join_acc[wave][16 * n + col][16 * c + 4 * g];
    __syncthreads();
  }
  if (wave != 0) return true;
#pragma unroll
  for (int n = 0; n < NM; ++n) {
    const uint32_t in = 16 * n + col, r = r0 + in;
    if (r >= list) continue;
    if (pc.splits > 1) {
      const size_t at = pc.part + (size_t)pc.split * F::kRows + in;
#pragma unroll
      for (int c = 0; c < F::kChannels; ++c) *(f32x4 *)(a.part_acc + at * D + 16 * c + 4 * g) = acc[n][c];
      if (g == 0) {
        a.part_ml[2 * at] = m[n];
        a.part_ml[2 * at + 1] = l[n];
      }
      continue;
    }
    const int64_t row = pc.q.first + (int64_t)(r / a.group), head = (int64_t)pc.head * a.group + r % a.group;
    Value *out = (Value *)a.out + row * a.out_row + head * a.out_head;
    const float inv = l[n] == 0 ? 0.0f : 1.0f / l[n];
#pragma unroll
    for (int c = 0; c < F::kChannels; ++c) store4<T>(out + 16 * c + 4 * g, acc[n][c] * inv, a.out_vec);
    if (a.lse && g == 0) a.lse[row * a.n_q_heads + head] = l[n] == 0 ? -INFINITY : (m[n] + log2_fast(l[n])) * 0.6931471805599453f;
  }
  return true;
}

template <int T, int CODE, int D, int NM>
__device__ __forceinline__ void few_rows(const AttendArgs &a, const Lists &lists, uint32_t index) {
  typedef FewRows<D, NM> F;
  __shared__ float join_acc[2][F::kRows][D + 4];
  __shared__ float join_ml[F::kWaves][F::kRows][2];
  __shared__ uint32_t join_odd[F::kWaves];  // a NaN or an infinity was met
  const bool done = few_rows_piece<T, CODE, D, NM, false>(a, lists, index, join_acc, join_ml, join_odd);
  if (__builtin_expect(!__builtin_amdgcn_readfirstlane(done), 0))
    few_rows_piece<T, CODE, D, NM, true>(a, lists, index, join_acc, join_ml, join_odd);
}

// ------------------------------------------------------------------ many rows
// One workgroup for 128 rows and a piece of their tokens, a wave 32 rows: the
// step's codes are staged in LDS and every wave reads them all.  As above, S^T = K
// Q^T and O^T = V^T P^T in matrix instructions of 32 x 32 x 16 (a lane holds, of the
// result, rows 8 (i / 4) + 4 (lane / 32) + i % 4 of column lane % 32): row m = 8 a + 4
// b + c of a tile of 32 keys is its token 16 b + 4 a + c, so a lane's 16 scores are of
// 16 tokens in a row and are its part of the second product's operand.
//
// LDS holds codes, not bf16: half the bytes to read, for one conversion per two
// codes and wave.  16-byte chunks are placed so that eight lanes next to each other
// read eight different places of 128 bytes.
//
// Bound by vector instructions: a wave's step has 32 matrix instructions and about 350
// others (128 conversions; for each of 32 scores a multiply-add, an exponential, an
// addition, half a maximum and half a rounding; the rest places and addresses).  Two
// waves of a SIMD hide a matrix instruction behind about six others, and these take
// 2 ns each.  A prompt of 8192 tokens, 32 heads over 8 of 128: 637 us, 864 TFLOP/s (a
// bf16 matrix product of 8192: 1230); counters at that: matrix units 39% busy, vector
// ALUs 64%.  Slower were: three waves to a SIMD (it spills), codes straight from memory
// to registers (980 us then, with LDS 890), barriers every second step (the same), scores
// of one tile during the softmax of another (740, 690 without).
template <int D>
struct ManyRows {
  static constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = kManyRows;
  static constexpr int kChunks = D / 16;              // of a key, and blocks of 16 channels
  static constexpr int kAll = kStep * kChunks, kLoads = (kAll + kThreads - 1) / kThreads;  // chunks of keys; of each thread; as many of values
  __device__ static __forceinline__ bool has(uint32_t n) { return kAll % kThreads == 0 || n < kAll; }
  static constexpr int kRing = 2, kPages = 4;         // steps in LDS: codes; their pages
  // Chunk c of token t of a step, and chunk c (16 tokens) of channel d, in units of 16 bytes.
  __device__ static __forceinline__ uint32_t key_at(uint32_t t, uint32_t c) {
    uint32_t turn;
    if constexpr (kChunks % 8 == 0) turn = (t & 3) | ((t >> 4) & 1) << 2;
    else if constexpr (kChunks % 4 == 0) turn = ((t >> 1) & 1) | ((t >> 4) & 1) << 1;
    else turn = (t >> 4) & 1;
    return t * kChunks + (c ^ turn);
  }
  __device__ static __forceinline__ uint32_t value_at(uint32_t d, uint32_t c) { return 4 * d + (c ^ ((d >> 1) & 3)); }
};

typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int T>
__device__ __forceinline__ f32x16 score_mfma32(const Frag &k, const Frag &q, f32x16 c) {
  if constexpr (T == UZIP_FP16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(k.h, q.h, c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.b, q.b, c, 0, 0, 0);
}

template <int T, int CODE, int D>
__device__ void many_rows(const AttendArgs &a, const Lists &lists, uint32_t index) {
  typedef ManyRows<D> F;
  typedef typename Elem<T>::type Value;
  constexpr int PROBS = Query<T>::kProbs, kTiles = kStep / 32, kChannels = D / 32, kKeySteps = D / 16;
  __shared__ u32x4 keys[F::kRing][F::kAll];
  __shared__ u32x4 values[F::kRing][F::kAll];
  __shared__ float key_scale[F::kRing][4], value_scale[F::kRing][4];  // of 16 tokens each; a key's is -1 where there is no page
  __shared__ int32_t step_page[F::kPages][4];        // pages of 16 tokens each
  __shared__ uint32_t odd;                           // a NaN or an infinity was met
  Piece pc;
  if (!find_piece<F::kThreads, false>(a, lists, index, &pc)) return;
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, half = lane >> 5;
  const uint32_t list = (uint32_t)pc.q.rows * a.group, P = a.c.page;
  // the blocks with the most tokens first: the last ones to run are short
  const uint32_t r0 = ((list + F::kRows - 1) / F::kRows - 1 - pc.block) * F::kRows;
  int32_t lo, hi;
  seen_range(a, pc.q, r0, min(list, r0 + F::kRows), &lo, &hi);
  const uint32_t step0 = (uint32_t)lo / kStep, steps = hi > lo ? ((uint32_t)hi + kStep - 1) / kStep - step0 : 0;
  const uint32_t share = (steps + pc.splits - 1) / pc.splits;
  const uint32_t begin = step0 + min(steps, pc.split * share), end = step0 + min(steps, (pc.split + 1) * share);

  // this wave's rows, and its first tile of a step's tokens
  const uint32_t w0 = r0 + 32 * wave, r = w0 + col;
  const bool here = r < list;
  const uint32_t tok = here ? r / a.group : 0, head = pc.head * a.group + (here ? r % a.group : 0);
  const Seen seen = seen_by(a, here ? pc.q.base + (int32_t)tok : -1);
  const uint32_t w1 = min(list, w0 + 32);
  const int32_t p_min = w0 < list ? pc.q.base + (int32_t)(w0 / a.group) : -1;
  const int32_t p_max = w0 < list ? pc.q.base + (int32_t)((w1 - 1) / a.group) : -1;
  Frag q[kKeySteps];
  {
    const Value *x = (const Value *)a.q + (int64_t)(pc.q.first + (int32_t)tok) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
    for (int s = 0; s < kKeySteps; ++s) query_frag<T>(x + 32 * (s / 2) + 16 * half + 8 * (s % 2), a.q_vec, a.negate, &q[s]);
  }
  f32x16 acc[kChannels];
  float m, l;

  // staging: thread's chunks n = tid + 256 i
  const int32_t *table = a.table + (size_t)pc.req * a.max_pages;
  const size_t page_bytes = (size_t)P * D;
  u32x4 stage_k[F::kLoads], stage_v[F::kLoads];
  uint32_t stage_exp = 0;
  bool exp_ok = true;
  const int32_t b_min = pc.q.base + (int32_t)(r0 / a.group), b_max = pc.q.base + (int32_t)((min(list, r0 + F::kRows) - 1) / a.group);
  auto all_see = [&](int32_t t0) {  // all rows of the block
    return t0 + kStep - 1 <= b_min && (a.window == 0 || (int64_t)t0 > (int64_t)b_max - a.window);
  };
  auto page_of = [&](int32_t t) { return t < hi ? table[(uint32_t)t >> a.c.page_shift] : -1; };
  // A step's pages are looked up a step before its codes are asked for, and those
  // are looked at only when they are put into LDS, after the products of another
  // step: nothing waits for memory that has not had a step's time.
  bool stage_ok = true;
  int32_t next_page = -1;
  auto load = [&](uint32_t step) {
    const int32_t t0 = (int32_t)(step * kStep);
    const int32_t *pages = step_page[step % F::kPages];
    const uint8_t *k_at[F::kLoads], *v_at[F::kLoads];
    if (P >= kStep) {  // one page: its address is the same in all lanes
      const int32_t page = __builtin_amdgcn_readfirstlane(pages[0]);
      stage_ok = (uint32_t)page < a.c.n_pages;
      const size_t at = ((size_t)(stage_ok ? page : 0) * a.c.heads + pc.head) * page_bytes;
      const uint32_t in = (uint32_t)t0 & (P - 1);
#pragma unroll
      for (int i = 0; i < F::kLoads; ++i) {
        const uint32_t n = tid + F::kThreads * i;
        k_at[i] = a.c.k + at + (size_t)in * D + 16 * n;
        v_at[i] = a.c.v + at + in + ((n / 4) * P + 16 * (n % 4));
      }
    } else {
      const int32_t value_page = pages[tid % 4];
      stage_ok = (uint32_t)value_page < a.c.n_pages;
      const uint8_t *v = a.c.v + ((size_t)(stage_ok ? value_page : 0) * a.c.heads + pc.head) * page_bytes + (16 * (tid % 4) & (P - 1));
#pragma unroll
      for (int i = 0; i < F::kLoads; ++i) {
        const uint32_t n = tid + F::kThreads * i, t = n / F::kChunks, c = n % F::kChunks;
        int32_t page = pages[F::has(n) ? t / 16 : 0];
        page = (uint32_t)page < a.c.n_pages ? page : 0;
        k_at[i] = a.c.k + ((size_t)page * a.c.heads + pc.head) * page_bytes + (t & (P - 1)) * D + 16 * c;
        v_at[i] = v + (n / 4) * P;
      }
    }
#pragma unroll
    for (int i = 0; i < F::kLoads; ++i)
      if (F::has(tid + F::kThreads * i)) {
        stage_k[i] = *(const u32x4 *)k_at[i];
        stage_v[i] = *(const u32x4 *)v_at[i];
      }
    if (tid < 8) {
      const int32_t page = pages[tid & 3];
      const bool ok = (uint32_t)page < a.c.n_pages;
      const size_t ph = (size_t)(ok ? page : 0) * a.c.heads + pc.head;
      stage_exp = (tid < 4 ? a.c.k_exp : a.c.v_exp)[ph];
      exp_ok = ok;
    }
    if (tid < 4) next_page = page_of(t0 + kStep + 16 * (int32_t)tid);
  };
  auto put_one = [&](auto leave_out, uint32_t b, int32_t t, bool edge, bool gaps, uint32_t n, const u32x4 &k, u32x4 w) {
    if (!F::has(n)) return;
    keys[b][F::key_at(n / F::kChunks, n % F::kChunks)] = k;
    if (edge || gaps) {  // codes that no row sees count as zero, for 0 times NaN is not 0
      w.x = stage_ok ? keep_tokens(w.x, t, lo, hi) : 0u;
      w.y = stage_ok ? keep_tokens(w.y, t + 4, lo, hi) : 0u;
      w.z = stage_ok ? keep_tokens(w.z, t + 8, lo, hi) : 0u;
      w.w = stage_ok ? keep_tokens(w.w, t + 12, lo, hi) : 0u;
    }
    if constexpr (leave_out) w = bounded<CODE>(w);
    values[b][F::value_at(n / 4, n % 4)] = w;
  };
  auto put = [&](auto leave_out, uint32_t step) {
    const uint32_t b = step % F::kRing;
    const int32_t t0 = (int32_t)(step * kStep), t = t0 + 16 * (int32_t)(tid % 4);
    const bool edge = !all_see(t0), gaps = !__all(stage_ok);
    static_for<F::kLoads>([&](auto i) { put_one(leave_out, b, t, edge, gaps, tid + F::kThreads * i, stage_k[i], stage_v[i]); });
    if (tid < 4) {
      key_scale[b][tid] = exp_ok ? pow2((int)stage_exp) : -1.0f;
      step_page[(step + 1) % F::kPages][tid] = next_page;
    } else if (tid < 8) {
      value_scale[b][tid - 4] = exp_ok ? pow2((int)stage_exp) : 1.0f;
    }
  };
  if (tid == 0) odd = 0;
  const uint32_t key_row = 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3);  // token of this lane's row
  auto sum_up = [&](auto leave_out) {  // m, l and acc over all steps, without codes that are not finite or with them
#pragma unroll
    for (int c = 0; c < kChannels; ++c) acc[c] = f32x16{};
    m = -INFINITY;
    l = 0;
    if (tid < 4) step_page[begin % F::kPages][tid] = page_of((int32_t)(begin * kStep) + 16 * (int32_t)tid);
    __syncthreads();
    if (begin < end) {
      load(begin);
      put(leave_out, begin);
    }
    __syncthreads();
    for (uint32_t step = begin; step < end; ++step) {
      const uint32_t b = step % F::kRing;
      const int32_t t0 = (int32_t)(step * kStep);
      if (step + 1 < end) load(step + 1);
      if (w0 < list && t0 <= p_max && (a.window == 0 || (int64_t)t0 + kStep - 1 > (int64_t)p_min - a.window)) {
        f32x16 s[kTiles];
        // The scores' products are issued before the other waves' softmax, which fills
        // the gaps between them (a prompt of 8192 takes 2% longer without).
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          s[i] = f32x16{};
#pragma unroll
          for (int c = 0; c < kChannels; ++c) {
            const u32x4 w = keys[b][F::key_at(32 * i + key_row, 2 * c + half)];
            s[i] = score_mfma32<T>(key_frag<T, CODE>(w.x, w.y), q[2 * c], s[i]);
            s[i] = score_mfma32<T>(key_frag<T, CODE>(w.z, w.w), q[2 * c + 1], s[i]);
          }
        }
        __builtin_amdgcn_s_setprio(0);
        static_assert(kTiles == 2, "two scales to a lane's part of a step");
        float ks[kTiles], vs[kTiles];  // ks: what a score is still to be multiplied by
        bool page_ok[kTiles], pages_ok = true;
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          const float x = key_scale[b][2 * i + half];
          page_ok[i] = x >= 0;
          pages_ok = pages_ok && page_ok[i];
          ks[i] = x * a.scale_log2;
          vs[i] = value_scale[b][2 * i + half];
        }
        const bool whole = t0 + kStep - 1 <= p_min && (a.window == 0 || (int64_t)t0 > (int64_t)p_max - a.window) && __all(pages_ok);
        if (!whole) {
#pragma unroll
          for (int i = 0; i < kTiles; ++i) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              s[i][j] = page_ok[i] && sees(seen, t0 + 32 * i + 16 * (int32_t)half + j) ? s[i][j] * ks[i] : -INFINITY;
            ks[i] = 1;
          }
        }
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          float t = s[i][0];
#pragma unroll
          for (int j = 1; j < 16; ++j) t = fmaxf(t, s[i][j]);
          top = fmaxf(top, t * ks[i]);
        }
        if (__any(top > m + lag_for(fmaxf(vs[0], vs[1])))) {
          top = fmaxf(top, __shfl_xor(top, 32));
          const float m2 = fmaxf(m, top);
          const float shrink = m2 == -INFINITY ? 1.0f : exp2_fast(m - m2);
          m = m2;
          l *= shrink;
#pragma unroll
          for (int c = 0; c < kChannels; ++c) acc[c] *= shrink;
        }
        const float base = m == -INFINITY ? 0.0f : m;
        Frag p[kTiles][2][PROBS];
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            float x = exp2_fast(__builtin_fmaf(s[i][j], ks[i], -base));
            l += x;
#pragma unroll
            for (int t = 0; t < PROBS; ++t) {
              p[i][j / 8][t].b[j % 8] = (__bf16)x;
              if (t + 1 < PROBS) x -= (float)p[i][j / 8][t].b[j % 8];
            }
          }
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
          for (int c = 0; c < kChannels; ++c) {
            const u32x4 w = values[b][F::value_at(32 * c + col, 2 * i + half)];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const Frag v = u ? codes_bf16<CODE>(w.z, w.w, vs[i]) : codes_bf16<CODE>(w.x, w.y, vs[i]);
#pragma unroll
              for (int t = PROBS - 1; t >= 0; --t)
                acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.b, p[i][u][t].b, acc[c], 0, 0, 0);
            }
          }
      }
      // the other slot was last read in the step before, which every wave has left
      if (step + 1 < end) put(leave_out, step + 1);
      __syncthreads();
    }
  };
  sum_up(std::false_type{});
  float sums = 0;
#pragma unroll
  for (int c = 0; c < kChannels; ++c)
#pragma unroll
    for (int j = 0; j < 16; ++j) sums = __builtin_fmaf(acc[c][j], 0.0f, sums);
  if (sums != 0) odd = 1;
  __syncthreads();
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(odd), 0)) {  // without it, and the rows that see such a value get it
    sum_up(std::true_type{});
#pragma unroll 1
    for (uint32_t step = begin; step < end; ++step) {
      const int32_t t0 = (int32_t)(step * kStep);
#pragma unroll
      for (int c = 0; c < kChannels; ++c)
#pragma unroll 1
        for (int i = 0; i < kTiles; ++i) {
          const int32_t t = t0 + 32 * i + 16 * (int32_t)half, page = page_of(t);
          const bool ok = (uint32_t)page < a.c.n_pages;
          const u32x4 w = *(const u32x4 *)(a.c.v + ((size_t)(ok ? page : 0) * a.c.heads + pc.head) * page_bytes +
                                           (size_t)(32 * c + col) * P + ((uint32_t)t & (P - 1)));
          if (!__any(any_unbounded<CODE>(w))) continue;
#pragma unroll 1
          for (int kind = 0; kind < 3; ++kind) {
            f32x16 hits = {};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              Frag see;
#pragma unroll
              for (int j = 0; j < 8; ++j) see.b[j] = (__bf16)(ok && sees(seen, t + 8 * u + j) ? 1.0f : 0.0f);
              const Frag is = u ? class_frag<CODE>(w.z, w.w, kind) : class_frag<CODE>(w.x, w.y, kind);
              hits = __builtin_amdgcn_mfma_f32_32x32x16_bf16(is.b, see.b, hits, 0, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (hits[j] > 0) acc[c][j] += class_value(kind);
          }
        }
    }
  }

  l += __shfl_xor(l, 32);
  if (!here) return;
  const uint32_t in = r - r0;
  const int64_t row = pc.q.first + (int64_t)tok;
  Value *out = (Value *)a.out + row * a.out_row + (int64_t)head * a.out_head;
  const size_t at = pc.part + (size_t)pc.split * F::kRows + in;
  const float inv = l == 0 ? 0.0f : 1.0f / l;
#pragma unroll
  for (int c = 0; c < kChannels; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t d = 32 * c + 8 * i + 4 * half;
      f32x4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = acc[c][4 * i + j];
      if (pc.splits > 1) *(f32x4 *)(a.part_acc + at * D + d) = x;
      else store4<T>(out + d, x * inv, a.out_vec);
    }
  if (half == 0) {
    if (pc.splits > 1) {
      a.part_ml[2 * at] = m;
      a.part_ml[2 * at + 1] = l;
    } else if (a.lse) {
      a.lse[row * a.n_q_heads + head] = l == 0 ? -INFINITY : (m + log2_fast(l)) * 0.6931471805599453f;
    }
  }
}

// ------------------------------------------------------------------ joining pieces
// Pieces' maxima, sums and accs of the blocks that were split.  A wave takes a row
// at a time: lanes in groups of dim / 4, four channels to a lane, each group every
// so many pieces; `part` tells which 16 rows of the block.  Bound by latency: 6 us where
// little was split, 8 for 32 blocks of 15 pieces, 14 for 144 blocks of 128 rows (a
// wave's four rows at once took 22: where a block has few rows it loads them again).
constexpr uint32_t kJoinRows = 16;
template <int T, int D>
__device__ void join_rows(const AttendArgs &a, const Lists &lists, bool last_first, uint32_t index, uint32_t part) {
  typedef typename Elem<T>::type Value;
  constexpr uint32_t kLanes = D / 4, kGroups = 64 / kLanes, kWaves = 4;
  static_assert((kGroups & (kGroups - 1)) == 0, "groups add up in halves");
  Piece pc;
  if (!find_piece<64 * kWaves, true>(a, lists, index, &pc)) return;
  const uint32_t lane = threadIdx.x & 63, group = lane / kLanes, d = 4 * (lane % kLanes), rows = lists.rows;
  const uint32_t list = (uint32_t)pc.q.rows * a.group;
  const uint32_t r0 = (last_first ? (list + rows - 1) / rows - 1 - pc.block : pc.block) * rows;
  const uint32_t end = min(min(rows, list - r0), (part + 1) * kJoinRows);
  for (uint32_t in = part * kJoinRows + (threadIdx.x >> 6); in < end; in += kWaves) {
    const uint32_t r = r0 + in;
    const float *ml = a.part_ml + 2 * (pc.part + in);
    const float *accs = a.part_acc + (pc.part + in) * D + d;
    float m = -INFINITY;
    for (uint32_t s = lane; s < pc.splits; s += 64) m = fmaxf(m, ml[2 * (size_t)s * rows]);
#pragma unroll
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    f32x4 acc = {0, 0, 0, 0};
    float l = 0;
    auto weight = [&](size_t at) {
      const float ms = ml[2 * at];
      return ms == m ? 1.0f : exp2_fast(ms - m);
    };
    if (group < kGroups) {
#pragma unroll 4
      for (uint32_t s = group; s < pc.splits; s += kGroups) {
        const size_t at = (size_t)s * rows;
        const float w = weight(at);
        l += w * ml[2 * at + 1];
        acc += w * *(const f32x4 *)(accs + at * D);
      }
    }
#pragma unroll
    for (uint32_t o = kGroups / 2; o; o >>= 1) {  // into the first group
      const int from = (int)(lane + o * kLanes) & 63;
      l += __shfl(l, from);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] += __shfl(acc[j], from);
    }
    if (__builtin_expect(__any(not_finite(0, acc) != 0), 0)) {  // a weight of 0 on an infinity, perhaps
      acc = f32x4{0, 0, 0, 0};
#pragma unroll 1
      for (uint32_t s = 0; s < pc.splits; ++s) {
        const size_t at = (size_t)s * rows;
        if (group == 0) acc += weighed(*(const f32x4 *)(accs + at * D), weight(at));
      }
    }
    if (group != 0) continue;
    const int64_t row = pc.q.first + (int64_t)(r / a.group), head = (int64_t)pc.head * a.group + r % a.group;
    const float inv = l == 0 ? 0.0f : 1.0f / l;
    store4<T>((Value *)a.out + row * a.out_row + head * a.out_head + d, acc * inv, a.out_vec);
    if (a.lse && d == 0) a.lse[row * a.n_q_heads + head] = l == 0 ? -INFINITY : (m + log2_fast(l)) * 0.6931471805599453f;
  }
}

// ------------------------------------------------------------------ kernels
// Blocks of 32 rows read a list's tokens once where blocks of 16 read them twice, the
// second time from a cache.  It pays where there are lists for every compute unit (64
// requests of up to 8000 tokens, 4 heads with 32 rows, bf16: dim 64 46 us, by blocks of 16
// 49; 128 72 and 87; 192 118 and 119) and not where the blocks of 16 are more work to
// share out (8 requests of 4000, 20 rows of dim 128: 35 and 25).  Not at all in fp32, dim
// 256, or fp16 of dim 128, where registers spill (as above, dim 128: 257 and 96 in fp32, 97
// and 87 in fp16; dim 256 in bf16 207 and 175).
constexpr bool has_two(uint32_t type, uint32_t dim) { return type != UZIP_FP32 && dim <= 192 && !(type == UZIP_FP16 && dim == 128); }
// Two workgroups to a compute unit where at most 6 registers spill for it (requests of 4000
// tokens: 64, 20 rows of dim 128 in blocks of 32, 59 us, one to a unit 71; 32, 20 rows of
// dim 192 48 and 62; but of dim 256 113 and 79).
template <int T, int D, int NM>
constexpr int kFewPerUnit = (D <= 128 || (D == 192 && NM == 1 && T != UZIP_FP32)) ? 2 : 1;
template <int T, int CODE, int D, int NM>
__global__ __launch_bounds__(256, (kFewPerUnit<T, D, NM>)) void few_rows_kernel(AttendArgs a, Lists few) {
  few_rows<T, CODE, D, NM>(a, few, blockIdx.x);
}
// Long lists and short ones in one launch: the first workgroups take the pieces of
// the long ones, and the short ones' fill the gaps as they end.
template <int T, int CODE, int D>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void all_rows_kernel(AttendArgs a, Lists many, uint32_t n_many, Lists few) {
  if (blockIdx.x < n_many) many_rows<T, CODE, D>(a, many, blockIdx.x);
  else few_rows<T, CODE, D, 1>(a, few, blockIdx.x - n_many);
}
template <int T, int D>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a, Lists many, uint32_t n_many, Lists few) {
  const uint32_t of_many = many.rows / kJoinRows, of_few = few.rows / kJoinRows, i = blockIdx.x - n_many * of_many;
  if (blockIdx.x < n_many * of_many) join_rows<T, D>(a, many, true, blockIdx.x / of_many, blockIdx.x % of_many);
  else join_rows<T, D>(a, few, false, i / of_few, i % of_few);
}

// ------------------------------------------------------------------ launches, by head_dim
struct AttendCall {
  AttendArgs a;
  uzip_dtype type, code;
  uint32_t max_new;
  hipStream_t stream;
};
// What a call launches and where its pieces go.
struct Layout {
  bool many;              // the kernel for both, with blocks of 16 rows for the short lists
  uint32_t few;           // blocks of 16 rows to a workgroup
  uint64_t rows_for_one;  // workspace rows for each compute unit
};
inline Layout layout(uzip_dtype type, uint32_t dim, uint32_t heads, uint32_t group, uint32_t n_reqs, uint32_t max_new) {
  const uint64_t list = (uint64_t)max_new * group;
  const bool many = type != UZIP_FP32 && list > many_from(dim);
  const bool two = !many && list > 16 && has_two(type, dim) && (uint64_t)n_reqs * heads >= kMostUnits;
  const uint32_t few = two ? 2 : 1;
  return {many, few, (many ? 2 * many_pieces(dim) * kManyRows : 0) + 2 * kFewPieces * 16ull * few};
}
template <int D>
uzip_status launch_attend(const AttendCall &call);

}  // namespace uzip_kv
