// The element formats that the row and matrix kernels share: conversion of 8 neighbouring values to and
// from MXFP4 and INT4 codes, and loads / stores of 8 values of an fp32, fp16 or bf16 array.
//
// MXFP4: 32 neighbouring values of a row are a block with one scale 2^(b - 127), stored as the byte b. With
// amax the block's largest magnitude, b - 127 = floor(log2(amax)) - 2, not below -127; since amax = 1.f * 2^(E - 127)
// has E in its exponent bits, b = max(E - 2, 0) for zero, subnormal and normal amax alike. A value x becomes the code of
// x / 2^(b-127) among 0, 0.5, 1, 1.5, 2, 3, 4, 6 (sign in bit 3), nearest, ties to the even code, magnitudes above 6
// to 6 (x / scale < 8). The division is by a power of two and exact, so the codes do not depend on how it is done. A
// block that holds a NaN or an infinity gets b = 255 and zero codes: all of it reads back as NaN.
#pragma once

#include "common.cuh"

namespace mfet {

constexpr int kMxBlock = 32;         // values per scale
constexpr uint32_t kMxNan = 255u;    // scale byte of a block with a value that is not finite

__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits) {
  const uint32_t e = amax_bits >> 23;  // amax_bits has no sign
  return e >= 255u ? kMxNan : (e > 2u ? e - 2u : 0u);
}
// 1 / 2^(b - 127) for b <= 252, as a normal number: 2^(127 - b)
__device__ __forceinline__ float mx_inv_scale(uint32_t b) { return __uint_as_float((254u - b) << 23); }
__device__ __forceinline__ float mx_scale(uint32_t b) {
  return __uint_as_float(b == 0u ? 0x00400000u : (b == kMxNan ? 0x7FC00000u : b << 23));
}

// codes of v[0..7] * inv, element j in bits 4j .. 4j+3
__device__ __forceinline__ uint32_t mx_encode8(const float* v, float inv) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(v[0] * inv), "f"(v[1] * inv), "f"(v[2] * inv), "f"(v[3] * inv), "f"(v[4] * inv), "f"(v[5] * inv),
        "f"(v[6] * inv), "f"(v[7] * inv));
  return r;
}

// v[j] = the value of code j of `codes`, times scale (exact: a code has two significant bits)
__device__ __forceinline__ void mx_decode8(uint32_t codes, float scale, float* v) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(codes));
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[j]));
    v[2 * j] = f.x * scale;
    v[2 * j + 1] = f.y * scale;
  }
}

template <int DT>
struct Elem;
template <>
struct Elem<MFET_F32> {
  using T = float;
  static __device__ __forceinline__ float to(T x) { return x; }
  static __device__ __forceinline__ T from(float x) { return x; }
};
template <>
struct Elem<MFET_F16> {
  using T = __half;
  static __device__ __forceinline__ float to(T x) { return __half2float(x); }
  static __device__ __forceinline__ T from(float x) { return __float2half_rn(x); }
};
template <>
struct Elem<MFET_BF16> {
  using T = __nv_bfloat16;
  static __device__ __forceinline__ float to(T x) { return __bfloat162float(x); }
  static __device__ __forceinline__ T from(float x) { return __float2bfloat16_rn(x); }
};

// Eight neighbouring values as they lie in memory: 16 bytes of a 16-bit type, 32 bytes of fp32.
template <int DT>
struct Raw8 {
  static constexpr int words = DT == MFET_F32 ? 2 : 1;
  uint4 w[words];
};

// The first `count` (<= 8) values at p, the rest 0. VEC: p is 16-byte aligned and full chunks are read in 16-byte pieces.
// The values are read once, so they are kept out of L1.
template <int DT, bool VEC>
__device__ __forceinline__ Raw8<DT> load8(const typename Elem<DT>::T* p, int count) {
  Raw8<DT> r;
  if (VEC && count == 8) {
#pragma unroll
    for (int i = 0; i < Raw8<DT>::words; ++i) r.w[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
    return r;
  }
  typename Elem<DT>::T t[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) t[j] = j < count ? p[j] : Elem<DT>::from(0.f);
  memcpy(&r, t, sizeof(t));
  return r;
}

template <int DT>
__device__ __forceinline__ void widen8(const Raw8<DT>& r, float* v) {
  typename Elem<DT>::T t[8];
  memcpy(t, &r, sizeof(t));
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = Elem<DT>::to(t[j]);
}

template <int DT, bool VEC>
__device__ __forceinline__ void store8(typename Elem<DT>::T* p, const float* v, int count) {
  typename Elem<DT>::T t[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) t[j] = Elem<DT>::from(v[j]);
  if (VEC && count == 8) {
    Raw8<DT> r;
    memcpy(&r, t, sizeof(t));
#pragma unroll
    for (int i = 0; i < Raw8<DT>::words; ++i) reinterpret_cast<uint4*>(p)[i] = r.w[i];
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < count) p[j] = t[j];
}

__device__ __forceinline__ uint32_t amax8(const float* v) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7FFFFFFFu);  // a NaN's bits are above infinity's
  return m;
}

}  // namespace mfet
