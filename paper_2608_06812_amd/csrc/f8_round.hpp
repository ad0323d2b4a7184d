// Scales and values of the 8-bit formats (device code; the definitions are
// beside ozfp4_quantize_f8 in ozfp4.h).
#pragma once

#include "f8.hpp"
#include "ozfp4.h"

namespace ozfp4 {

template <int kSrc> struct Source;
template <> struct Source<OZFP4_F32> { typedef float T; };
template <> struct Source<OZFP4_BF16> { typedef uint16_t T; };
template <> struct Source<OZFP4_F16> { typedef _Float16 T; };

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float widen(_Float16 v) { return (float)v; }

// |x| where it is finite, else 0
__device__ __forceinline__ float finite_abs(float x) {
  const float a = __builtin_fabsf(x);
  return a < __builtin_inff() ? a : 0.0f;
}

// A block's scale and what its elements need: S = m 2^e, m in [1, 2), and r,
// 1 / m to an ulp.
struct Scale {
  float m, r;
  int e;
};

// max(fl32(a / t), 2^-126). t = 1.75 2^e; with c = fl32(1 / t) and q = a c
// within an ulp, a - t q is exact (also where it is subnormal, for every q that
// the maximum leaves) and q + (a - t q) c rounds to the quotient rounded once
// (Markstein 1990): five instructions in place of a division's thirty.
template <int kFmt>
__device__ __forceinline__ float scale_f32(float a) {
  constexpr float top = kFmt == OZFP4_E4M3 ? 448.0f : 57344.0f, inv = 1.0f / top;
  const float q = a * inv, s = __builtin_fmaf(__builtin_fmaf(-top, q, a), inv, q);
  return a == 0.0f ? 1.0f : __builtin_fmaxf(s, 1.1754943508222875e-38f);
}

// Exponent E of the power-of-two scale: t = 1.75 2^8 or 1.75 2^15, so for a =
// f 2^e (f in [1, 2)) E = e - 8 (15), one more where f > 1.75. A subnormal a
// gives -126 like every a below 2^-118.
template <int kFmt>
__device__ __forceinline__ int scale_exp(float a) {
  const uint32_t b = __float_as_uint(a);
  const int e = (int)(b >> 23) - 127 - (kFmt == OZFP4_E4M3 ? 8 : 15) + ((b & 0x7fffff) > 0x600000);
  return a == 0.0f ? 0 : max(e, -126);
}

template <bool kPow2, int kFmt>
__device__ __forceinline__ Scale make_scale(float a) {
  Scale s;
  if constexpr (kPow2) {
    s.m = s.r = 1.0f;
    s.e = scale_exp<kFmt>(a);
  } else {
    const uint32_t b = __float_as_uint(scale_f32<kFmt>(a));
    s.e = (int)(b >> 23) - 127;
    s.m = __uint_as_float((b & 0x7fffff) | 0x3f800000);
    s.r = __builtin_amdgcn_rcpf(s.m);
  }
  return s;
}

template <bool kPow2, int kFmt>
__device__ __forceinline__ void store_scale(void* s, int64_t at, float a) {
  if constexpr (kPow2)
    static_cast<uint8_t*>(s)[at] = (uint8_t)(scale_exp<kFmt>(a) + 127);
  else
    static_cast<float*>(s)[at] = scale_f32<kFmt>(a);
}

// x / S as an FP32 value that rounds to the format as the exact quotient
// does. The FP32 quotient alone does not: a border between two 8-bit values
// is itself an FP32 value, and quotients within 2^-25 of it fall on it. So
// the quotient is rounded to odd: h is within an ulp of it, and the exact
// residual |x| - h S says whether it is above (then h is the quotient rounded
// down, else its lower neighbour is) and whether it is h (else the last bit
// is set, which no border has). Dividing x and S by 2^e first keeps the
// residuals away from underflow for every x that does not round to zero. NaN
// stays NaN; an infinity becomes NaN, unless kInf.
template <bool kPow2, bool kInf>
__device__ __forceinline__ float quotient(float x, const Scale& s) {
  const float y = __builtin_ldexpf(x, -s.e);
  if constexpr (kPow2) return y;
  const float a = __builtin_fabsf(y), q = a * s.r;
  const float h = __builtin_fmaf(__builtin_fmaf(-q, s.m, a), s.r, q);
  const uint32_t d = __float_as_uint(__builtin_fmaf(-h, s.m, a));
  const uint32_t b = (__float_as_uint(h) - (d >> 31)) | min(d, 1u);
  const float v = __builtin_copysignf(__uint_as_float(b), y);
  if constexpr (kInf) return __builtin_fabsf(x) < __builtin_inff() ? v : x;
  return v;
}

template <int kFmt>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  int v = 0;
  if constexpr (kFmt == OZFP4_E4M3) {
    v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, v, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
  } else {
    v = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, v, false);
    v = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, v, true);
  }
  return (uint32_t)v;
}

// Eight quotients as 8-bit values.
template <bool kPow2, bool kInf, int kFmt>
__device__ __forceinline__ uint2 pack8(const float (&x)[8], const Scale& s) {
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = quotient<kPow2, kInf>(x[j], s);
  return uint2{pack4<kFmt>(v[0], v[1], v[2], v[3]), pack4<kFmt>(v[4], v[5], v[6], v[7])};
}

// Eight neighbouring elements from src on, of which n exist (any alignment).
template <typename T>
__device__ __forceinline__ void load8(const T* src, int64_t n, float (&x)[8]) {
  if (n >= 8) {
    T v[8];
    __builtin_memcpy(v, src, sizeof(v));
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = widen(v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = 0.0f;
    if (n > 0) {   // eight loads at once, not one by one behind their conditions
      T v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = src[j < n ? j : n - 1];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = j < n ? widen(v[j]) : 0.0f;
    }
  }
}

}  // namespace ozfp4
