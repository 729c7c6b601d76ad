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

#include "kv_device.h"

namespace uzip_kv {

struct AttendArgs {
  Cache c;
  const void *q;
  void *out;
  float *lse;
  int64_t q_row, q_head, out_row, out_head;
  const int32_t *table, *lens, *q_start;
  float *part_acc;   // [slot][row of the block][dim]: acc of pieces that are joined
  float *part_ml;    // [slot][row of the block][2]: their m and l
  uint32_t n_rows, n_q_heads, group, max_pages, n_reqs, window;
  uint32_t target;   // pieces that fill the GPU
  float scale_log2;  // scale * log2 e
  bool q_vec, out_vec;  // rows start at multiples of 16 (q) and 4 elements (out), so loads and stores may be wide
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kStep = 64;      // tokens of a step
constexpr int kMinSteps = 4;   // steps of a piece, so each of a workgroup's waves has one

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

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

struct Piece {
  Request q;
  uint32_t req, head, block;     // which rows
  uint32_t split, splits, slot;  // which part of their tokens; the slot of part 0
};

__device__ __forceinline__ uint32_t blocks_of(const AttendArgs &a, const Request &q, uint32_t rows, int64_t least, int64_t most) {
  const int64_t list = (int64_t)q.rows * a.group;
  return list >= least && list <= most ? (uint32_t)((list + rows - 1) / rows) : 0u;
}

// The most steps that a block of `rows` rows of the request can have.
__device__ __forceinline__ uint32_t steps_of(const AttendArgs &a, const Request &q, uint32_t rows) {
  int64_t tokens = q.len;
  if (a.window) tokens = min(tokens, (int64_t)a.window + rows / a.group + 1 + kStep);
  return (uint32_t)((tokens + kStep - 1) / kStep);
}

__device__ __forceinline__ uint64_t wave_scan64(uint64_t x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = __shfl_up(x, o);
    if ((int)(threadIdx.x & 63) >= o) x += y;
  }
  return x;
}

// Which piece is number `index`, found by the whole workgroup.  Requests whose
// list has `least` to `most` rows take part, in blocks of `rows`.  All blocks'
// steps are shared out so that about `target` pieces of equal length come of
// them; a block shorter than that stays whole.  With JOIN the index counts the
// blocks that were split instead.  At most target + blocks pieces, at most
// target split blocks, and at most 2 target slots come of it: a block of n
// steps is split only where n > S, the steps of a piece, into ceil(n / S) <
// 2 n / S.  Every workgroup sums over the requests for itself: two scans.
template <int THREADS, bool JOIN>
__device__ bool find_piece(const AttendArgs &a, uint32_t rows, int64_t least, int64_t most, uint32_t index, Piece *out) {
  constexpr int kWaves = THREADS / 64;
  __shared__ uint64_t part[2 * kWaves];
  __shared__ Piece found;
  const uint32_t tid = threadIdx.x, wave = tid >> 6, n = a.n_reqs + 1;  // with the rows of no request
  const uint32_t each = (n + THREADS - 1) / THREADS, lo = min(n, tid * each), hi = min(n, lo + each);
  uint64_t steps = 0;
  for (uint32_t i = lo; i < hi; ++i) {
    const Request q = request(a, i);
    steps += (uint64_t)blocks_of(a, q, rows, least, most) * steps_of(a, q, rows);
  }
  steps = wave_scan64(steps);
  if ((tid & 63) == 63) part[wave] = steps;
  __syncthreads();
  uint64_t all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) all += part[w];
  all *= a.c.heads;
  const uint64_t length = max((all + a.target - 1) / a.target, (uint64_t)kMinSteps);  // S
  auto count = [&](const Request &q, uint32_t *splits) {
    const uint32_t b = blocks_of(a, q, rows, least, most);
    *splits = (uint32_t)max((steps_of(a, q, rows) + length - 1) / length, (uint64_t)1);
    const uint64_t pieces = (uint64_t)b * a.c.heads * (JOIN ? (*splits > 1 ? 1u : 0u) : *splits);
    return pieces | (*splits > 1 ? (uint64_t)b * a.c.heads * *splits : 0) << 32;  // pieces; slots
  };
  uint64_t mine = 0;
  uint32_t splits;
  for (uint32_t i = lo; i < hi; ++i) mine += count(request(a, i), &splits);
  const uint64_t incl = wave_scan64(mine);
  if ((tid & 63) == 63) part[kWaves + wave] = incl;
  __syncthreads();
  uint64_t at = incl - mine, total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < (int)wave) at += part[kWaves + w];
    total += part[kWaves + w];
  }
  if (index >= (uint32_t)total) return false;
  for (uint32_t i = lo; i < hi; ++i) {
    const Request q = request(a, i);
    const uint64_t c = count(q, &splits);
    const uint32_t rest = index - (uint32_t)at;
    if (index >= (uint32_t)at && rest < (uint32_t)c) {
      Piece p;
      p.q = q;
      p.req = i;
      p.head = rest % a.c.heads;
      const uint32_t up = rest / a.c.heads;
      p.split = JOIN ? 0 : up % splits;
      p.splits = splits;
      p.block = JOIN ? up : up / splits;
      p.slot = (uint32_t)(at >> 32) + (p.block * a.c.heads + p.head) * splits;
      found = p;
    }
    at += c;
  }
  __syncthreads();
  *out = found;
  return true;
}

// ------------------------------------------------------------------ fragments
// Matrix instructions of 16 x 16 x 32: a lane holds, of the first operand, eight
// values of row lane % 16; of the second, eight of column lane % 16; of the
// result, rows 4 (lane / 16) + 0..3 of column lane % 16.  Which place of the
// contraction a lane's values have is free as long as both operands agree.
template <int T>
struct Query {  // bf16: the query as it is, probabilities in one bf16 term
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

union Frag {
  bf16x8 b;
  f16x8 h;
  bf16x2 b2[4];
  f16x2 h2[4];
  uint4 u;
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

// Eight values as the query's fragments: fp32 in three bf16 terms, each the
// rounding of what the ones before left.
template <int T>
__device__ __forceinline__ void query_frag(const typename Elem<T>::type *x, bool wide, Frag *f) {
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
    f[0].u = *(const uint4 *)x;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (T == UZIP_FP16) f[0].h[j] = x[j];
      else f[0].b[j] = x[j];
    }
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

// ------------------------------------------------------------------ few rows
// One workgroup for up to 16 NM rows and a piece of their tokens, one wave a
// step of 64 tokens, everything from memory straight into registers:
//   S^T = K Q^T, four tiles of 16 tokens: row m of tile i is token 16 (m / 4) + 4
//   i + m % 4, so that a lane ends up with the scores of 16 tokens in a row for one
//   query -- which is just what it needs of the second product's
//   O^T = V^T P^T, whose first operand it loads as 16 bytes of a channel.
// No score or code crosses lanes; pages of 16 tokens and more never split a lane's
// load.  Each wave keeps its own maximum, sum and acc; they join at the end.
template <int D, int NM>
struct FewRows {
  static constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = 16 * NM;
  static constexpr int kPairs = D / 64, kOdd = (D / 32) % 2, kKeySteps = D / 32, kChannels = D / 16;
};

template <int T, int CODE, int D, int NM>
__global__ __launch_bounds__(256) void attend_few_kernel(AttendArgs a, int64_t least, int64_t most) {
  typedef FewRows<D, NM> F;
  typedef typename Elem<T>::type Value;
  constexpr int TERMS = Query<T>::kTerms, PROBS = Query<T>::kProbs;
  __shared__ float join_acc[2][F::kRows][D + 4];
  __shared__ float join_ml[F::kWaves][F::kRows][2];
  Piece pc;
  if (!find_piece<F::kThreads, false>(a, F::kRows, least, most, blockIdx.x, &pc)) return;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
  const uint32_t list = (uint32_t)pc.q.rows * a.group, r0 = pc.block * F::kRows, P = a.c.page;
  int32_t lo, hi;
  seen_range(a, pc.q, r0, min(list, r0 + F::kRows), &lo, &hi);
  const uint32_t step0 = (uint32_t)lo / kStep, steps = hi > lo ? ((uint32_t)hi + kStep - 1) / kStep - step0 : 0;
  const uint32_t share = (steps + pc.splits - 1) / pc.splits;
  const uint32_t begin = step0 + min(steps, pc.split * share), end = step0 + min(steps, (pc.split + 1) * share);

  // the rows' queries and places
  Frag q[NM][F::kKeySteps][TERMS];
  int32_t place[NM];
#pragma unroll
  for (int n = 0; n < NM; ++n) {
    const uint32_t r = r0 + 16 * n + col;
    const bool here = r < list;
    const uint32_t tok = here ? r / a.group : 0, head = pc.head * a.group + (here ? r % a.group : 0);
    place[n] = here ? pc.q.base + (int32_t)tok : -1;
    const Value *x = (const Value *)a.q + (int64_t)(pc.q.first + (int32_t)tok) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
    for (int s = 0; s < F::kKeySteps; ++s) {
      const uint32_t d = s < 2 * F::kPairs ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
      query_frag<T>(x + d, a.q_vec, q[n][s]);
    }
  }
  // the first and the last place of the block's rows
  const int32_t p_min = pc.q.base + (int32_t)(r0 / a.group), p_max = pc.q.base + (int32_t)((min(list, r0 + F::kRows) - 1) / a.group);

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
  uint4 k16[4][F::kPairs > 0 ? F::kPairs : 1], v16[F::kChannels];
  uint2 k8[4];
  uint32_t e_k, e_v;
  bool page_here;
  auto load_keys = [&](int32_t t0, int32_t page) {
    page = (uint32_t)page < a.c.n_pages ? page : 0;
    const uint8_t *row = a.c.k + ((size_t)page * a.c.heads + pc.head) * page_bytes +
                         (((uint32_t)(t0 + key_chunk) & (P - 1)) + (col & 3)) * D;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int s = 0; s < F::kPairs; ++s) k16[i][s] = *(const uint4 *)(row + i * 4 * D + 64 * s + 16 * g);
      if (F::kOdd) k8[i] = *(const uint2 *)(row + i * 4 * D + 64 * F::kPairs + 8 * g);
    }
  };
  auto load_values = [&](int32_t t0, int32_t page) {
    page_here = (uint32_t)page < a.c.n_pages;
    const size_t ph = (size_t)(page_here ? page : 0) * a.c.heads + pc.head;
    const uint8_t *at = a.c.v + ph * page_bytes + (size_t)col * P + ((uint32_t)(t0 + value_chunk) & (P - 1));
#pragma unroll
    for (int c = 0; c < F::kChannels; ++c) v16[c] = *(const uint4 *)(at + (size_t)16 * c * P);
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
          const uint4 w = k16[i][ks / 2];
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
    const bool whole = t0 >= lo && t0 + kStep - 1 <= p_min && (a.window == 0 || (int64_t)t0 > (int64_t)p_max - a.window) &&
                       __all(page_ok);
    const int32_t t_lane = t0 + value_chunk;
#pragma unroll
    for (int n = 0; n < NM; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float x = s[n][i][j] * ks_scale;
          if (!whole) {
            const int32_t t = t_lane + 4 * i + j;
            const bool seen = page_ok && t <= place[n] && (a.window == 0 || (int64_t)t > (int64_t)place[n] - a.window);
            x = seen ? x : -INFINITY;
          }
          s[n][i][j] = x;
        }

    // The maximum is taken anew only where a score passes the old one by more
    // than 8: powers of two up to 2^8 cost no precision, and most steps need
    // no exchange between lanes and no rescaling.
    Frag p[NM][2][PROBS];
#pragma unroll
    for (int n = 0; n < NM; ++n) {
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, s[n][i][j]);
      if (__any(top > m[n] + 8.0f)) {
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
          float x = exp2_fast(s[n][i][j] - base);
          l[n] += x;
#pragma unroll
          for (int t = 0; t < PROBS; ++t) {
            p[n][i / 2][t].b[4 * (i % 2) + j] = (__bf16)x;
            if (t + 1 < PROBS) x -= (float)p[n][i / 2][t].b[4 * (i % 2) + j];
          }
        }
    }

    // Codes that no row sees count as zero: 0 times NaN would not.  A NaN or an
    // infinity that some rows see and others do not is taken out of the product
    // and added to the rows that see it.
    if (!whole) {
      bool odd = false;
#pragma unroll
      for (int c = 0; c < F::kChannels; ++c) {
        uint32_t *w = (uint32_t *)&v16[c];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] = page_ok ? keep_tokens(w[i], t_lane + 4 * i, lo, hi) : 0u;
          odd = odd || unbounded<CODE>(w[i]) != 0;
        }
      }
      if (p_min != p_max && __any(odd)) {
#pragma unroll
        for (int c = 0; c < F::kChannels; ++c) {
          uint32_t *w = (uint32_t *)&v16[c];
#pragma unroll 1
          for (int kind = 0; kind < 3; ++kind) {  // NaN, infinity, -infinity
            const float value = kind == 0 ? NAN : kind == 1 ? INFINITY : -INFINITY;
#pragma unroll
            for (int n = 0; n < NM; ++n) {
              f32x4 hits = {0, 0, 0, 0};
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                Frag is, see;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                  const uint32_t code = (w[2 * u + j / 4] >> (8 * (j % 4))) & 0xFFu;
                  const float x = decode<CODE>(code);
                  is.b[j] = (__bf16)((kind == 0 ? x != x : x == value) ? 1.0f : 0.0f);
                  const int32_t t = t_lane + 8 * u + j;
                  see.b[j] = (__bf16)(page_ok && t <= place[n] && (a.window == 0 || (int64_t)t > (int64_t)place[n] - a.window) ? 1.0f : 0.0f);
                }
                hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(is.b, see.b, hits, 0, 0, 0);
              }
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (hits[j] > 0) acc[n][c][j] += value;
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t bad = unbounded<CODE>(w[i]) >> 7;
            w[i] &= ~(bad * 0xFFu);
          }
        }
      }
    }

#pragma unroll
    for (int c = 0; c < F::kChannels; ++c) {
      const uint4 w = v16[c];
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
  __syncthreads();
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
    for (int c = 0; c < F::kChannels; ++c) acc[n][c] *= shrink;
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
  if (wave != 0) return;
#pragma unroll
  for (int n = 0; n < NM; ++n) {
    const uint32_t in = 16 * n + col, r = r0 + in;
    if (r >= list) continue;
    if (pc.splits > 1) {
      const size_t at = (size_t)(pc.slot + pc.split) * F::kRows + in;
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
    for (int c = 0; c < F::kChannels; ++c) {
      Value o[4] __attribute__((aligned(4 * sizeof(Value))));
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = (Value)(acc[n][c][j] * inv);
      if (a.out_vec) {
        if constexpr (sizeof(Value) == 2) *(uint2 *)(out + 16 * c + 4 * g) = *(uint2 *)o;
        else *(uint4 *)(out + 16 * c + 4 * g) = *(uint4 *)o;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) out[16 * c + 4 * g + j] = o[j];
      }
    }
    if (a.lse && g == 0) a.lse[row * a.n_q_heads + head] = l[n] == 0 ? -INFINITY : (m[n] + log2_fast(l[n])) * 0.6931471805599453f;
  }
}

// ------------------------------------------------------------------ joining pieces
// One workgroup for each block that was split: the pieces' maxima, sums and accs.
template <int T, int D>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a, uint32_t rows, int64_t least, int64_t most) {
  typedef typename Elem<T>::type Value;
  Piece pc;
  if (!find_piece<256, true>(a, rows, least, most, blockIdx.x, &pc)) return;
  const uint32_t list = (uint32_t)pc.q.rows * a.group, r0 = pc.block * rows, n = min(rows, list - r0);
  constexpr uint32_t kLanes = D / 4;  // lanes of a row, four channels each
  for (uint32_t i = threadIdx.x; i < n * kLanes; i += 256) {
    const uint32_t in = i / kLanes, d = 4 * (i % kLanes), r = r0 + in;
    float m = -INFINITY;
    for (uint32_t s = 0; s < pc.splits; ++s) m = fmaxf(m, a.part_ml[2 * ((size_t)(pc.slot + s) * rows + in)]);
    f32x4 acc = {0, 0, 0, 0};
    float l = 0;
    for (uint32_t s = 0; s < pc.splits; ++s) {
      const size_t at = (size_t)(pc.slot + s) * rows + in;
      const float ms = a.part_ml[2 * at], w = ms == m ? 1.0f : exp2_fast(ms - m);
      l += w * a.part_ml[2 * at + 1];
      acc += w * *(const f32x4 *)(a.part_acc + at * D + d);
    }
    const int64_t row = pc.q.first + (int64_t)(r / a.group), head = (int64_t)pc.head * a.group + r % a.group;
    Value *out = (Value *)a.out + row * a.out_row + head * a.out_head + d;
    const float inv = l == 0 ? 0.0f : 1.0f / l;
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = (Value)(acc[j] * inv);
    if (a.lse && d == 0) a.lse[row * a.n_q_heads + head] = l == 0 ? -INFINITY : (m + log2_fast(l)) * 0.6931471805599453f;
  }
}

// ------------------------------------------------------------------ launches, by head_dim
struct AttendCall {
  AttendArgs a;
  uzip_dtype type, code;
  uint32_t max_new;
  hipStream_t stream;
};
// Rows of a block of the few-rows kernel for lists of `list` rows.
constexpr uint32_t few_blocks(uint32_t dim, uint64_t list) {
  const uint32_t most = dim <= 128 ? 4 : 2;  // LDS: 16 NM rows of dim fp32 values, twice, in 64 KiB
  return list <= 16 ? 1 : list <= 32 || most == 2 ? 2 : 4;
}
template <int D>
uzip_status launch_attend(const AttendCall &call);

}  // namespace uzip_kv
