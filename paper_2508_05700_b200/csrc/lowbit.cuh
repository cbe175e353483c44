// The element formats that the row, matrix and clipping kernels share: MXFP4 scales and codes, and loads, conversions
// and stores of a few neighbouring values of an fp32, fp16 or bf16 array.
//
// MXFP4: 32 neighbouring values of a row are a block with one scale 2^(b - 127), stored as the byte b. With
// amax the block's largest magnitude, b - 127 = floor(log2(amax)) - 2, not below -127; since amax = 1.f * 2^(E - 127)
// has E in its exponent bits, b = max(E - 2, 0) for zero, subnormal and normal amax alike. A value x becomes the code of
// x / 2^(b-127) among 0, 0.5, 1, 1.5, 2, 3, 4, 6 (sign in bit 3), nearest, ties to the even code, magnitudes above 6
// to 6 (x / scale < 8). The division is by a power of two and exact, so the codes do not depend on how it is done. A
// block that holds a NaN or an infinity gets b = 255 and zero codes: all of it reads back as NaN.
#pragma once

#include "common.cuh"

#ifdef MFET_CHECKED
#include <cstdio>
#endif

namespace mfet {

// The bounds-checked build's test ahead of an access, for kernels without a handle's error word: what lies outside is printed, sets
// MFET_DEV_BOUNDS in the call's status word if it has one, and is skipped. The normal build has `true` in its place.
#ifdef MFET_CHECKED
static __device__ __noinline__ bool out_of_bounds(uint32_t* status, const char* where, int line) {
  printf("mfet: index out of bounds, %s:%d\n", where, line);
  if (status) atomicOr(status, (uint32_t)MFET_DEV_BOUNDS);
  return false;
}
#define MFET_INSIDE(status, cond) ((cond) || out_of_bounds((status), __FILE__, __LINE__))
#else
#define MFET_INSIDE(status, cond) true
#endif

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

// Ahead of the first access in every kernel of these calls, which are launched with launch_early: nothing is read or written before
// the stream's previous kernel has ended, and from then on the next such kernel may be set up. That hides 1 to 2 us of a launch
// between two calls and promises nothing that an ordinary launch does not: whoever is set up early finds all kernels ended but the one
// before it.
__device__ __forceinline__ void early_launch_wait() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
}

template <typename K, typename... Args>
cudaError_t launch_early(K kernel, unsigned blocks, unsigned threads, size_t smem, cudaStream_t s, Args... args) {
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int DT>
struct Elem;
template <>
struct Elem<MFET_F32> {
  using T = float;
  static __device__ __forceinline__ T from(float x) { return x; }
};
template <>
struct Elem<MFET_F16> {
  using T = __half;
  static __device__ __forceinline__ T from(float x) { return __float2half_rn(x); }
  static __device__ __forceinline__ float2 widen(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};
template <>
struct Elem<MFET_BF16> {
  using T = __nv_bfloat16;
  static __device__ __forceinline__ T from(float x) { return __float2bfloat16_rn(x); }
  static __device__ __forceinline__ float2 widen(uint32_t w) { return make_float2(bf16lo(w), bf16hi(w)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};

template <int DT>
__device__ __forceinline__ float to_float(typename Elem<DT>::T x) {
  if constexpr (DT == MFET_F32) return x;
  else if constexpr (DT == MFET_F16) return __half2float(x);
  else return __bfloat162float(x);
}

// E neighbouring values as they lie in memory
template <int DT, int E>
struct Raw {
  static constexpr int bytes = E * (int)sizeof(typename Elem<DT>::T);
  static constexpr int pieces = bytes / 16, per = 16 / (int)sizeof(typename Elem<DT>::T);
  uint4 w[pieces];
};

// 32 bytes, aligned to that: whole sectors in one instruction
__device__ __forceinline__ void load32(const void* p, uint4* a, uint4* b) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(a->x), "=r"(a->y), "=r"(a->z), "=r"(a->w), "=r"(b->x), "=r"(b->y), "=r"(b->z), "=r"(b->w)
               : "l"(p));
}
__device__ __forceinline__ void store32(void* p, const uint4& a, const uint4& b) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w),
               "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
               : "memory");
}

// The first `count` values at p, the rest 0. VEC: p is 16-byte aligned, and whole pieces of 16 bytes are read as such; wide: it is
// 32-byte aligned. The values are read once: they do not displace anything in the caches.
template <int DT, int E, bool VEC>
__device__ __forceinline__ Raw<DT, E> load_raw(const typename Elem<DT>::T* p, int count, bool wide = false) {
  using R = Raw<DT, E>;
  R r;
  if constexpr (VEC && R::pieces % 2 == 0) {
    if (wide && count == E) {
#pragma unroll
      for (int i = 0; i < R::pieces; i += 2) load32(reinterpret_cast<const char*>(p) + 16 * i, &r.w[i], &r.w[i + 1]);
      return r;
    }
  }
#pragma unroll
  for (int i = 0; i < R::pieces; ++i) {
    if (VEC && count >= (i + 1) * R::per) {
      r.w[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
    } else {
      typename Elem<DT>::T t[R::per];
#pragma unroll
      for (int j = 0; j < R::per; ++j) t[j] = i * R::per + j < count ? p[i * R::per + j] : Elem<DT>::from(0.f);
      memcpy(&r.w[i], t, 16);
    }
  }
  return r;
}

// The same for p at any address of its element type: the 16-byte pieces that hold the values are read whole and shifted into place.
// Only memory of the array [lo, hi) is read: a piece that reaches over its ends is read value by value.
template <int DT, int E>
__device__ __forceinline__ Raw<DT, E> load_shifted(const typename Elem<DT>::T* p, int count, const void* lo, const void* hi) {
  using R = Raw<DT, E>;
  using T = typename Elem<DT>::T;
  const uintptr_t at = reinterpret_cast<uintptr_t>(p), from = at & ~(uintptr_t)15;
  const uint32_t d = (uint32_t)(at & 15);
  uint32_t w[4 * (R::pieces + 1)];
#pragma unroll
  for (int i = 0; i <= R::pieces; ++i) {
    const uintptr_t a = from + 16 * i;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (a < at + count * sizeof(T)) {
      if (a >= reinterpret_cast<uintptr_t>(lo) && a + 16 <= reinterpret_cast<uintptr_t>(hi)) {
        v = __ldg(reinterpret_cast<const uint4*>(a));  // a neighbour reads most of it again
      } else {
        T t[R::per];
#pragma unroll
        for (int j = 0; j < R::per; ++j) {
          const T* e = reinterpret_cast<const T*>(a) + j;
          t[j] = e >= p && e < p + count ? *e : Elem<DT>::from(0.f);
        }
        memcpy(&v, t, 16);
      }
    }
    w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
  }
#pragma unroll
  for (int i = 0; i < 4 * R::pieces + 2; ++i) w[i] = (d & 8) ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < 4 * R::pieces + 1; ++i) w[i] = (d & 4) ? w[i + 1] : w[i];
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4 * R::pieces; ++i) w[i] = __byte_perm(w[i], w[i + 1], (d & 2) ? 0x5432 : 0x3210);
  }
  if (count < E) {  // what follows the values
#pragma unroll
    for (int i = 0; i < 4 * R::pieces; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = i < count ? w[i] : 0u;
      else w[i] = 2 * i + 1 < count ? w[i] : (2 * i < count ? w[i] & 0xFFFFu : 0u);
    }
  }
  R r;
#pragma unroll
  for (int i = 0; i < R::pieces; ++i) r.w[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  return r;
}

template <int DT, int E, bool VEC>
__device__ __forceinline__ Raw<DT, E> load_any(const typename Elem<DT>::T* p, int count, const void* lo, const void* hi, bool wide = false) {
  if constexpr (VEC) return load_raw<DT, E, true>(p, count, wide);
  else return load_shifted<DT, E>(p, count, lo, hi);
}

// the values of 16 bytes
template <int DT>
__device__ __forceinline__ void widen16(const uint4& w, float* v) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (DT == MFET_F32) {
      v[j] = __uint_as_float(x[j]);
    } else {
      const float2 f = Elem<DT>::widen(x[j]);
      v[2 * j] = f.x;
      v[2 * j + 1] = f.y;
    }
  }
}
template <int DT>
__device__ __forceinline__ uint4 narrow16(const float* v) {
  uint32_t x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (DT == MFET_F32) x[j] = __float_as_uint(v[j]);
    else x[j] = Elem<DT>::pack(v[2 * j], v[2 * j + 1]);
  }
  return make_uint4(x[0], x[1], x[2], x[3]);
}

template <int DT, int E>
__device__ __forceinline__ void widen_raw(const Raw<DT, E>& r, float* v) {
#pragma unroll
  for (int i = 0; i < Raw<DT, E>::pieces; ++i) widen16<DT>(r.w[i], v + i * Raw<DT, E>::per);
}

template <int DT, int E, bool VEC>
__device__ __forceinline__ void store_values(typename Elem<DT>::T* p, const float* v, int count, bool wide = false) {
  using R = Raw<DT, E>;
  if constexpr (VEC && R::pieces == 2) {
    if (wide && count == E) {
      store32(p, narrow16<DT>(v), narrow16<DT>(v + R::per));
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < R::pieces; ++i) {
    if (VEC && count >= (i + 1) * R::per) {
      reinterpret_cast<uint4*>(p)[i] = narrow16<DT>(v + i * R::per);
    } else {
#pragma unroll
      for (int j = 0; j < R::per; ++j)
        if (i * R::per + j < count) p[i * R::per + j] = Elem<DT>::from(v[i * R::per + j]);
    }
  }
}

// Bits of the largest magnitude as fp32; above infinity's when there is a NaN among the values. 16-bit values are
// compared as integers two at a time, which orders magnitudes, infinity and NaN alike.
template <int DT, int E>
__device__ __forceinline__ uint32_t amax_raw(const Raw<DT, E>& r) {
  if constexpr (DT == MFET_F32) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < Raw<DT, E>::pieces; ++i) {
      const uint32_t x[4] = {r.w[i].x, r.w[i].y, r.w[i].z, r.w[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(fabsf(__uint_as_float(x[j]))));
    }
    return __float_as_uint(m);
  } else {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < Raw<DT, E>::pieces; ++i) {
      const uint32_t x[4] = {r.w[i].x, r.w[i].y, r.w[i].z, r.w[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(x[j] & 0x7FFF7FFFu));
    }
    const float2 f = Elem<DT>::widen(max(m >> 16, m & 0xFFFFu));
    return __float_as_uint(f.x);
  }
}

}  // namespace mfet
