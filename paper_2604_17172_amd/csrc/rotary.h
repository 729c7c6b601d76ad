// rotary.h -- rotary positions: the turn of a head's pairs of channels.
//
// A row at position p turns pair i of its rotary part by the angle p f_i:
//   a' = m (a cos - b sin)   b' = m (a sin + b cos)
// with frequencies f and a magnitude m that the caller gives.  The matrix is m times
// an orthogonal one, so the gradient is the same with the angle's sign changed.
#pragma once

#include "kv_host.h"
#include "kv_store.h"
#include "uzip_rotary.h"

namespace uzip_kv {

struct Turn {
  const int32_t *positions;
  const float *freq;   // [half]
  uint32_t half;       // pairs
  uint32_t first;      // channel where the rotary part begins
  bool interleaved;    // pairs (2 i, 2 i + 1), else (i, i + half)
  bool even;           // half and first are multiples of 8: no eight channels hold two kinds
  float m, m_low, sign;  // the magnitude and what 32 bits of it leave
};

struct CosSin {
  float c, s;
};

// The angle is taken in 64 bits: at position 2^20 a product in 32 bits is off by up to 2^-4.
// What is left of it after whole quarter turns, x and what 32 bits of x leave, goes to the two Taylor series up to
// x^10, |x| <= pi / 4: the first term left out is below 2e-9, a sine is off by 1.5 half steps at most, a cosine by 1.25.
__device__ __forceinline__ CosSin turn_of(const Turn &t, int32_t p, uint32_t pair) {
  const double quarters = (double)p * (double)t.freq[pair] * 0.63661977236758134308;  // 2 / pi
  const double n = __builtin_rint(quarters), angle = (quarters - n) * 1.57079632679489661923;
  const uint32_t q = (uint32_t)__builtin_bit_cast(uint64_t, n + 6755399441055744.0);  // n's last bits: 1.5 * 2^52 has a step of 1
  const float x = (float)angle, low = (float)(angle - (double)x), z = x * x, z_low = __builtin_fmaf(x, x, -z);
  const float h = __builtin_fmaf(z, -0.5f, 1.0f), h_low = __builtin_fmaf(z, -0.5f, 1.0f - h);  // 1 - z / 2 and what it leaves
  float s = __builtin_fmaf(z, 1.0f / 362880, -1.0f / 5040);
  s = __builtin_fmaf(z, s, 1.0f / 120);
  s = __builtin_fmaf(z, s, -1.0f / 6);
  s = __builtin_fmaf(x * z, s, __builtin_fmaf(x * z_low, -1.0f / 6, low * h));  // x + s
  float c = __builtin_fmaf(z, -1.0f / 3628800, 1.0f / 40320);
  c = __builtin_fmaf(z, c, -1.0f / 720);
  c = __builtin_fmaf(z, c, 1.0f / 24);
  c = __builtin_fmaf(z * z, c, h_low - __builtin_fmaf(0.5f, z_low, x * low));  // h + c
  s = __builtin_fmaf(t.m, x, __builtin_fmaf(t.m, s, t.m_low * x));
  c = __builtin_fmaf(t.m, h, __builtin_fmaf(t.m, c, t.m_low * h));
  const float cc = q & 1 ? s : c, ss = q & 1 ? c : s;
  // quarter turns: (c, s), (-s, c), (-c, -s), (s, -c)
  return {(q + 1) & 2 ? -cc : cc, (q & 2 ? -ss : ss) * t.sign};
}

__device__ __forceinline__ void turn_pair(const CosSin &r, float &a, float &b) {
  const float x = a, y = b;
  a = __builtin_fmaf(x, r.c, -(y * r.s));
  b = __builtin_fmaf(x, r.s, y * r.c);
}

// The channels of a head, `dim` of them, in pairs: pair p < half is pair p of the rotary part,
// the others are what lies before and after it, two by two.  `which` 0 or 1.
__device__ __forceinline__ uint32_t channel_of(const Turn &t, uint32_t p, uint32_t which) {
  if (p < t.half) return t.first + (t.interleaved ? 2 * p + which : p + which * t.half);
  const uint32_t r = 2 * (p - t.half) + which;
  return r < t.first ? r : r + 2 * t.half;
}

// A unit: pairs W u .. W u + W - 1.  Where half and first are multiples of W its channels are two
// groups of W; the first channel of each.
struct Groups {
  uint32_t a, b;
  bool turned;
};
template <int W>
__device__ __forceinline__ Groups groups_of(const Turn &t, uint32_t u) {
  if (W * u < t.half) {
    const uint32_t a = t.first + (t.interleaved ? 2 * W * u : W * u);
    return {a, t.interleaved ? a + W : a + t.half, true};
  }
  const uint32_t r = 2 * W * u - 2 * t.half;
  return {r < t.first ? r : r + 2 * t.half, r + W < t.first ? r + W : r + W + 2 * t.half, false};
}

// Turns a unit's values (two groups of W), rot(j) the turn of its pair j.  The two orders are two loops: as one
// with a choice inside, the values are reached through a chosen address and no longer stay in registers.
template <int W, class F>
__device__ __forceinline__ void turn_unit(const Turn &t, float *x, const F &rot) {
  if (t.interleaved) {
#pragma unroll
    for (int j = 0; j < W; ++j) turn_pair(rot(j), x[2 * j], x[2 * j + 1]);
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j) turn_pair(rot(j), x[j], x[j + W]);
  }
}

// W values that lie side by side, at a multiple of their bytes.
template <int T, int W>
struct Piece {
  typedef typename Elem<T>::type Value;
  typedef uint32_t Words __attribute__((ext_vector_type(W * sizeof(Value) / 4)));
  Words w;
  __device__ __forceinline__ void load(const Value *x) { w = *(const Words *)x; }
  __device__ __forceinline__ void store(Value *x) const { *(Words *)x = w; }
  __device__ __forceinline__ void get(float *x) const {
    Value v[W];
    __builtin_memcpy(v, &w, sizeof(w));
#pragma unroll
    for (int j = 0; j < W; ++j) x[j] = (float)v[j];
  }
  __device__ __forceinline__ void put(const float *x) {
    Value v[W];
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = (Value)x[j];
    __builtin_memcpy(&w, v, sizeof(w));
  }
};
template <int T>
struct Piece<T, 1> {
  typedef typename Elem<T>::type Value;
  Value w;
  __device__ __forceinline__ void load(const Value *x) { w = *x; }
  __device__ __forceinline__ void store(Value *x) const { *x = w; }
  __device__ __forceinline__ void get(float *x) const { *x = (float)w; }
  __device__ __forceinline__ void put(const float *x) { w = (Value)*x; }
};

// Rows of heads that are turned: [rows][heads][dim] at element strides.
struct TurnRows {
  const void *x;
  void *out;
  int64_t x_row, x_head, out_row, out_head;
  uint32_t n_rows, heads, dim;
  uint32_t block_rows;  // rows of a workgroup
  uint32_t width;       // pairs of a unit: what 16 bytes hold, 4, or 1
  uint32_t units;       // of a head, ceil(dim / 2 / width)
  FastDiv by_units, by_heads, by_half;
  bool in_place;        // out is x: what is not turned stays where it is
};

constexpr int kTurnThreads = 256;
constexpr uint32_t kTurnTable = 1024;  // turns that a workgroup holds, at most: 8 KiB

// One workgroup's rows.  The turns of a row are the same for all its heads: they are
// worked out once, into LDS, while the first values are on their way.  Bound by the rows' bytes: 16384 rows of
// 32 heads of 128 in bf16, 268 MB in 44 us, 6.1 TB/s.  Units of four pairs keep wide loads where the rotary part
// is no multiple of 8: 4099 rows of 11 heads of 104 in fp32, 40 of them turned, 37.5 MB in 8.5 us (pair by
// pair: 34.5 us).
template <int T, int W>
__device__ __forceinline__ void turn_units(const TurnRows &a, const Turn &t, uint32_t block, CosSin *table) {
  typedef typename Elem<T>::type Value;
  const uint32_t r0 = block * a.block_rows, rows = min(a.block_rows, a.n_rows - r0), tid = threadIdx.x;
  const uint32_t per_row = a.units * a.heads, count = rows * per_row;
  struct Unit {
    Piece<T, W> a, b;
    Groups g;
    Value *out;
    uint32_t turns;  // place of its first in the table
  };
  auto fetch = [&](uint32_t i) {
    const uint32_t rh = a.by_units.div(i), u = i - rh * a.units, r = a.by_heads.div(rh), h = rh - r * a.heads;
    Unit n;
    n.g = groups_of<W>(t, u);
    n.out = (Value *)a.out + (int64_t)(r0 + r) * a.out_row + (int64_t)h * a.out_head;
    n.turns = r * t.half + W * u;
    if (n.g.turned || !a.in_place) {
      const Value *x = (const Value *)a.x + (int64_t)(r0 + r) * a.x_row + (int64_t)h * a.x_head;
      n.a.load(x + n.g.a);
      if (n.g.b < a.dim) n.b.load(x + n.g.b);
    }
    return n;
  };
  Unit now;
  if (tid < count) now = fetch(tid);
  for (uint32_t i = tid; i < rows * t.half; i += kTurnThreads) {
    const uint32_t r = a.by_half.div(i);
    table[i] = turn_of(t, t.positions[r0 + r], i - r * t.half);
  }
  __syncthreads();
  for (uint32_t i = tid; i < count; i += kTurnThreads) {
    Unit next;
    if (i + kTurnThreads < count) next = fetch(i + kTurnThreads);
    if (now.g.turned) {
      float v[2 * W];
      now.a.get(v);
      now.b.get(v + W);
      turn_unit<W>(t, v, [&](int j) { return table[now.turns + j]; });
      now.a.put(v);
      now.b.put(v + W);
    }
    if (now.g.turned || !a.in_place) {
      now.a.store(now.out + now.g.a);
      if (now.g.b < a.dim) now.b.store(now.out + now.g.b);
    }
    now = next;
  }
}

template <int T>
__device__ __forceinline__ void turn_rows(const TurnRows &a, const Turn &t, uint32_t block, CosSin *table) {
  constexpr int kWide = 16 / sizeof(typename Elem<T>::type);
  if (a.width == kWide) turn_units<T, kWide>(a, t, block, table);
  else if (kWide != 4 && a.width == 4) turn_units<T, 4>(a, t, block, table);
  else turn_units<T, 1>(a, t, block, table);
}

// ------------------------------------------------------------------ host
inline bool valid_turn(const uzip_turn *t) {
  return t && t->rot >= 2 && t->rot <= 1024 && t->rot % 2 == 0 && t->first <= 1024 && t->interleaved <= 1 && t->inverse <= 1 &&
         (float)t->magnitude - (float)t->magnitude == 0;
}
inline bool valid_places(const uzip_turn *t) { return t->positions && t->freq && aligned(t->positions, 4) && aligned(t->freq, 4); }

inline Turn turn_args(const uzip_turn *t) {
  const uint32_t half = t->rot / 2;
  return {t->positions, t->freq, half, t->first, t->interleaved != 0, half % 8 == 0 && t->first % 8 == 0, (float)t->magnitude,
          (float)(t->magnitude - (double)(float)t->magnitude), t->inverse ? -1.0f : 1.0f};
}

// What a launch over rows of heads needs; false where they cannot be.
inline bool rows_to_turn(uzip_dtype dtype, const void *x, int64_t x_row, int64_t x_head, uint32_t n_rows, uint32_t heads, uint32_t dim,
                         const uzip_turn *t, void *out, int64_t out_row, int64_t out_head, TurnRows *a) {
  const uint32_t bytes = type_bytes(dtype);
  if (heads == 0 || heads > 65535 || dim > 1024 || t->first + t->rot > dim || !valid_rows(x, x_row, x_head, bytes) ||
      !valid_rows(out, out_row, out_head, bytes) || n_rows > UZIP_KV_MAX_ROWS || (uint64_t)n_rows * heads > UZIP_KV_MAX_ROW_HEADS)
    return false;
  const uint32_t half = t->rot / 2;
  auto fits = [&](uint32_t w) {
    const uint32_t size = w * bytes;
    return (half | t->first | dim) % w == 0 && aligned(x, size) && aligned(out, size) && ((x_row | x_head | out_row | out_head) & (w - 1)) == 0;
  };
  const uint32_t width = fits(16 / bytes) ? 16 / bytes : fits(4) ? 4 : 1;
  const uint32_t units = ((dim + 1) / 2 + width - 1) / width, per_row = units * heads;
  // Rows of a workgroup: four units to a thread, as long as there are rows for every compute unit and
  // the table holds their turns.
  uint32_t rows = 1;
  while (rows * per_row < 4 * kTurnThreads && 2 * rows * half <= kTurnTable && n_rows > 512 * rows) rows *= 2;
  *a = {x, out, x_row, x_head, out_row, out_head, n_rows, heads, dim, rows, width, units, FastDiv::of(units), FastDiv::of(heads),
        FastDiv::of(half), out == x && out_row == x_row && out_head == x_head};
  return true;
}
inline uint32_t turn_blocks(const TurnRows &a) { return a.block_rows ? (a.n_rows + a.block_rows - 1) / a.block_rows : 0; }

}  // namespace uzip_kv
