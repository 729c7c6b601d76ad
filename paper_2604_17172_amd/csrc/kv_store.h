// kv_store.h -- the write of one run of new tokens into an 8-bit page.
#pragma once

#include "kv_device.h"

namespace uzip_kv {

// ------------------------------------------------------------------ store
// For a run, a head, and keys or values: the largest finite magnitude, the page's
// exponent, the codes.  A thread takes eight channels of a token (keys) or of four
// tokens that lie in one word of a value page's channel (values: the page is
// transposed in registers); what it first loaded stays in registers until the exponent
// is known.  Bound by the rows' bytes, each read from memory once: 16384 tokens of 8
// heads of 128 in bf16, 101 MB in 20.9 us, 4.8 TB/s (value by value: 117 us).
struct StoreArgs {
  Cache c;
  const void *x[2];
  int64_t row[2], head[2];
  const int64_t *slots;
  const int32_t *runs, *counts;
  uint32_t n_rows;
  bool vec;  // rows start at multiples of 16 bytes
};

constexpr int kHeld = 4;  // pieces of eight values that a thread keeps

template <int T>
struct Eight {
  typedef typename Elem<T>::type Value;
  u32x4 w[sizeof(Value) / 2];
  __device__ __forceinline__ void load(const Value *x, bool vec) {
    if (vec) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(Value) / 2; ++i) w[i] = ((const u32x4 *)x)[i];
    } else {
      Value v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = x[j];
      __builtin_memcpy(w, v, sizeof(w));
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (int)sizeof(Value) / 2; ++i) w[i] = u32x4{0, 0, 0, 0};
  }
  __device__ __forceinline__ void get(float *x) const {
    Value v[8];
    __builtin_memcpy(v, w, sizeof(w));
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)v[j];
  }
};

// The codes of places 0 .. off - 1 again, where the page's scale grew.
template <int CODE>
__device__ __forceinline__ void grow_page(uint8_t *codes, bool values, uint32_t off, uint32_t D, uint32_t P, uint32_t was, uint32_t e,
                          uint32_t tid, uint32_t threads) {
  const float down = pow2(max(127 + (int)was - (int)e, 0));
  for (uint32_t i = tid; i < off * D; i += threads) {
    uint8_t &c = codes[values ? i / off * P + i % off : i];
    c = (uint8_t)recode<CODE>(c, down);
  }
}

template <int T, int CODE, int THREADS, bool VALUES>
__device__ __forceinline__ void store_run(const StoreArgs &a, uint32_t run, uint32_t h, uint32_t tid, float *part, uint32_t *odd_part) {
  typedef typename Elem<T>::type Value;
  const uint32_t D = a.c.dim, P = a.c.page, per = D / 8;
  const int32_t row = a.runs[2 * (size_t)run];
  int32_t n = a.runs[2 * (size_t)run + 1];
  if (row < 0 || n <= 0 || (uint32_t)row >= a.n_rows) return;
  const int64_t slot = a.slots[row];
  if (slot < 0 || (uint64_t)slot >= (uint64_t)a.c.n_pages << a.c.page_shift) return;
  const uint32_t page = (uint32_t)(slot >> a.c.page_shift), off = (uint32_t)slot & (P - 1);
  n = min((uint32_t)n, min(P - off, a.n_rows - (uint32_t)row));
  const uint32_t last = off + n;  // places off .. last - 1 of the page
  const int64_t stride = a.row[VALUES];
  // the row of place t of the page
  const Value *x = (const Value *)a.x[VALUES] + ((int64_t)row - off) * stride + (int64_t)h * a.head[VALUES];
  const size_t ph = (size_t)page * a.c.heads + h;
  uint8_t *codes = (VALUES ? a.c.v : a.c.k) + ph * P * D;
  uint8_t *exps = VALUES ? a.c.v_exp : a.c.k_exp;
  const uint32_t was = off ? exps[ph] : 0;

  // A piece: eight channels of one place; a unit: one piece (keys), or the four pieces of a word (values).
  constexpr uint32_t kUnit = VALUES ? 4 : 1;
  const uint32_t first = off / kUnit, count = ((last + kUnit - 1) / kUnit - first) * per;
  auto unit = [&](uint32_t i, uint32_t *t, uint32_t *d) {
    if (VALUES) {  // neighbours in a wave: 16 words of a channel (or what there are), so that stores join up
      const uint32_t words = (last + 3) / 4 - first;
      *t = 4 * (first + i % words);
      *d = 8 * (i / words);
    } else {
      *t = first + i / per;
      *d = 8 * (i % per);
    }
  };
  auto load = [&](uint32_t t, uint32_t d, Eight<T> *e) {
#pragma unroll
    for (uint32_t j = 0; j < kUnit; ++j) {
      if (t + j >= off && t + j < last) e[j].load(x + (int64_t)(t + j) * stride + d, a.vec);
      else e[j].zero();
    }
  };
  constexpr uint32_t kKeep = kHeld / kUnit;
  Eight<T> held[kHeld];
  float amax = 0;
  bool odd = false;
  auto scan = [&](const Eight<T> *e) {
#pragma unroll
    for (uint32_t j = 0; j < kUnit; ++j) {
      float v[8];
      e[j].get(v);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float f = fabsf(v[k]);
        const bool finite = f < INFINITY;
        odd = odd || !finite;
        amax = fmaxf(amax, finite ? f : 0.0f);
      }
    }
  };
#pragma unroll
  for (uint32_t k = 0; k < kKeep; ++k) {
    const uint32_t i = tid + k * THREADS;
    if (i < count) {
      uint32_t t, d;
      unit(i, &t, &d);
      load(t, d, held + k * kUnit);
    }
  }
#pragma unroll
  for (uint32_t k = 0; k < kKeep; ++k)
    if (tid + k * THREADS < count) scan(held + k * kUnit);
  for (uint32_t i = tid + kKeep * THREADS; i < count; i += THREADS) {
    uint32_t t, d;
    Eight<T> e[kUnit];
    unit(i, &t, &d);
    load(t, d, e);
    scan(e);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
  odd = __any(odd);
  if (THREADS > 64) {
    if ((tid & 63) == 0) {
      part[tid >> 6] = amax;
      odd_part[tid >> 6] = odd;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      amax = fmaxf(amax, part[w]);
      odd = odd || odd_part[w];
    }
  }
  const uint32_t e = max((uint32_t)exponent_for<CODE>(amax), was);
  if (tid == 0 && e != was) exps[ph] = (uint8_t)e;
  const float inv = pow2(254 - (int)e);
  odd = odd || e >= (uint32_t)Code<CODE>::kExpMax;  // there values may lie past the largest code

  auto put = [&](uint32_t t, uint32_t d, const Eight<T> *p) {
    float v[kUnit][8];
#pragma unroll
    for (uint32_t j = 0; j < kUnit; ++j) p[j].get(v[j]);
    if constexpr (VALUES) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float of[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) of[j] = v[j][k];
        uint32_t w = 0;
        if (odd) {
#pragma unroll
          for (int j = 0; j < 4; ++j) w |= encode<CODE>(of[j], inv) << (8 * j);
        } else {
          w = encode4<CODE>(of, inv);
        }
        uint8_t *at = codes + (size_t)(d + k) * P + t;
        if (t >= off && t + 4 <= last) {
          *(uint32_t *)at = w;
        } else {
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j)
            if (t + j >= off && t + j < last) at[j] = (uint8_t)(w >> (8 * j));
        }
      }
    } else {
      u32x2 w = {0, 0};
      if (odd) {
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k / 4] |= encode<CODE>(v[0][k], inv) << (8 * (k % 4));
      } else {
        w = u32x2{encode4<CODE>(v[0], inv), encode4<CODE>(v[0] + 4, inv)};
      }
      *(u32x2 *)(codes + (size_t)t * D + d) = w;
    }
  };
#pragma unroll
  for (uint32_t k = 0; k < kKeep; ++k) {
    const uint32_t i = tid + k * THREADS;
    if (i < count) {
      uint32_t t, d;
      unit(i, &t, &d);
      put(t, d, held + k * kUnit);
    }
  }
  for (uint32_t i = tid + kKeep * THREADS; i < count; i += THREADS) {
    uint32_t t, d;
    Eight<T> p[kUnit];
    unit(i, &t, &d);
    load(t, d, p);
    put(t, d, p);
  }
  if (off && e > was) grow_page<CODE>(codes, VALUES, off, D, P, was, e, tid, THREADS);
}

// A run of one row by a wave: every lane a channel or a few, nothing but the row
// number needed to ask for them.  64 rows of 8 heads: 4.0 us, by workgroups 6.5.
template <int T, int CODE>
__device__ __forceinline__ void store_one(const StoreArgs &a, bool values, int32_t row, uint32_t h, uint32_t lane) {
  typedef typename Elem<T>::type Value;
  const uint32_t D = a.c.dim, P = a.c.page;
  const Value *x = (const Value *)a.x[values] + (int64_t)row * a.row[values] + (int64_t)h * a.head[values];
  const int64_t slot = a.slots[row];
  float v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = lane + 64 * j < D ? (float)x[lane + 64 * j] : 0.0f;
  if (slot < 0 || (uint64_t)slot >= (uint64_t)a.c.n_pages << a.c.page_shift) return;
  const uint32_t page = (uint32_t)(slot >> a.c.page_shift), off = (uint32_t)slot & (P - 1);
  const size_t ph = (size_t)page * a.c.heads + h;
  uint8_t *codes = (values ? a.c.v : a.c.k) + ph * P * D, *exps = values ? a.c.v_exp : a.c.k_exp;
  const uint32_t was = off ? exps[ph] : 0;
  float amax = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float f = fabsf(v[j]);
    amax = fmaxf(amax, f < INFINITY ? f : 0.0f);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
  const uint32_t e = max((uint32_t)exponent_for<CODE>(amax), was);
  if (lane == 0 && e != was) exps[ph] = (uint8_t)e;
  const float inv = pow2(254 - (int)e);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t d = lane + 64 * j;
    if (d < D) codes[values ? d * P + off : off * D + d] = (uint8_t)encode<CODE>(v[j], inv);
  }
  if (off && e > was) grow_page<CODE>(codes, values, off, D, P, was, e, lane, 64);
}

}  // namespace uzip_kv
