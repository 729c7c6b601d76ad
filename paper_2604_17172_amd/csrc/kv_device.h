// kv_device.h -- device building blocks of the paged 8-bit key/value cache.
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "uzip_kv.h"

namespace uzip_kv {

// The cache as a kernel sees it.
struct Cache {
  uint8_t *k, *v, *k_exp, *v_exp;
  uint32_t n_pages, heads, dim, page, page_shift;
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ---- 8-bit codes ----
// E4M3: 1.75 * 2^8 is the largest value; E5M2: 1.75 * 2^15.  An exponent byte e
// scales a page by 2^(e - 127).  e >= 27 keeps every scaled code a normal
// number of bf16 and fp32, the upper limit keeps the largest finite.
template <int CODE>
struct Code;
template <>
struct Code<UZIP_E4M3FN> {
  static constexpr float kMax = 448.0f;
  static constexpr int kTop = 8, kExpMax = 246;
  static constexpr bool kInf = false;
};
template <>
struct Code<UZIP_E5M2> {
  static constexpr float kMax = 57344.0f;
  static constexpr int kTop = 15, kExpMax = 239;
  static constexpr bool kInf = true;
};
constexpr int kExpMin = 27;

// 2^(e - 127)
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)e << 23); }

// Least exponent byte whose scale brings amax (finite, >= 0) into the codes'
// range: the exponent field of amax less that of the largest code, one more
// where amax's fraction is past 1.75.
template <int CODE>
__device__ __forceinline__ int exponent_for(float amax) {
  const int up = (int)((__float_as_uint(amax) + 0x1FFFFFu) >> 23);
  return min(max(up - Code<CODE>::kTop, kExpMin), Code<CODE>::kExpMax);
}

// The code of x * inv (inv a power of two), rounded to nearest even.
template <int CODE>
__device__ __forceinline__ uint32_t encode(float x, float inv) {
  const uint32_t bits = __float_as_uint(x), sign = (bits >> 24) & 0x80u, mag = bits & 0x7FFFFFFFu;
  if (mag >= 0x7F800000u) return sign | (Code<CODE>::kInf && mag == 0x7F800000u ? 0x7Cu : 0x7Fu);
  const float y = fminf(fmaxf(x * inv, -Code<CODE>::kMax), Code<CODE>::kMax);
  const uint32_t c = CODE == UZIP_E4M3FN ? (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false)
                                         : (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(y, y, 0, false);
  return c & 0xFFu;
}

// Four codes of finite x * inv within the codes' range, x[0]'s in the low byte.
template <int CODE>
__device__ __forceinline__ uint32_t encode4(const float *x, float inv) {
  if constexpr (CODE == UZIP_E4M3FN) {
    const int c = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, c, true);
  } else {
    const int c = __builtin_amdgcn_cvt_pk_bf8_f32(x[0] * inv, x[1] * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(x[2] * inv, x[3] * inv, c, true);
  }
}

// The value of a code (byte 0 of c).
template <int CODE>
__device__ __forceinline__ float decode(uint32_t c) {
  return CODE == UZIP_E4M3FN ? __builtin_amdgcn_cvt_f32_fp8((int)c, 0) : __builtin_amdgcn_cvt_f32_bf8((int)c, 0);
}

// The code of a code's value times down (a power of two, at most 1): a page
// whose scale grew.  NaN and infinity stay what they are.
template <int CODE>
__device__ __forceinline__ uint32_t recode(uint32_t c, float down) {
  const uint32_t mag = c & 0x7Fu;
  if (mag >= (Code<CODE>::kInf ? 0x7Cu : 0x7Fu)) return (c & 0x80u) | (Code<CODE>::kInf && mag == 0x7Cu ? 0x7Cu : 0x7Fu);
  return encode<CODE>(decode<CODE>(c), down);
}

// ---- values of the model's types ----
template <int T>
struct Elem;
template <>
struct Elem<UZIP_BF16> {
  typedef __bf16 type;
};
template <>
struct Elem<UZIP_FP16> {
  typedef _Float16 type;
};
template <>
struct Elem<UZIP_FP32> {
  typedef float type;
};

// Division by a number known on the host, of n < 2^31.
struct FastDiv {
  uint32_t d, m, s;
  static FastDiv of(uint32_t d) {
    FastDiv f{d, 0, 0};
    while ((1ull << f.s) < d) ++f.s;
    f.m = (uint32_t)((((1ull << f.s) - d) << 32) / d + 1);
    return f;
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(n, m) + n) >> s; }
};

}  // namespace uzip_kv
