// What the tensor-core kernels share: barriers in shared memory with bounded waits, tiles that the copy engine moves,
// tensor memory, and the host's tensor maps.
#pragma once

#include <cuda.h>

#include <atomic>

#include "lowbit.cuh"

namespace mfet {

constexpr uint64_t kStallNs = 2000000000ull;  // the longest wait inside a kernel

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// True in one lane of a converged warp. Instructions of the tensor cores and the copy engine take their operands from uniform
// registers; under a branch on this the compiler knows that one lane runs and moves them there directly (under `lane == 0`
// each such instruction took 110 cycles to issue).
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\t"
               "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
               "selp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok)
               : "r"(bar), "r"(parity)
               : "memory");
  return ok != 0;
}
__device__ __forceinline__ uint64_t now_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// Waits for the phase `parity` of a barrier, two seconds at most; false: it did not come (or another role gave up). It polls (a
// suspended wait took longer to come back: 2 us of 47 for a 16384 x 2048 x 2048 product), and reads the clock rarely.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* dead) {
  uint64_t t0 = 0;
  for (uint32_t i = 1;; ++i) {
    if (bar_try(bar, parity)) return true;
    if ((i & 0xFFFF) == 0) {
      if (*dead) return false;
      const uint64_t t = now_ns();
      if (t0 == 0) t0 = t;
      if (t - t0 > kStallNs) {
        *dead = 1;
        return false;
      }
    }
  }
}

// The same for a role that may be late by a microsecond: its warp sleeps on the barrier instead of polling it, and what it does not issue is
// power that the tensor cores' clock gets.
__device__ __forceinline__ bool bar_sleep(uint32_t bar, uint32_t parity, volatile int* dead) {
  uint64_t t0 = 0;
  for (uint32_t i = 1;; ++i) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok)
                 : "r"(bar), "r"(parity)
                 : "memory");
    if (ok) return true;
    if ((i & 0xFF) == 0) {
      if (*dead) return false;
      const uint64_t t = now_ns();
      if (t0 == 0) t0 = t;
      if (t - t0 > kStallNs) {
        *dead = 1;
        return false;
      }
    }
  }
}

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(bar)
               : "memory");
}

__device__ __forceinline__ void bulk_store(const CUtensorMap* map, uint32_t src, int32_t x, int32_t y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src)
               : "memory");
}

__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"  // in one statement: nothing may use the registers before the wait
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr)
      : "memory");
}

// Two fp32 numbers in one instruction
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(r)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(r)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<uint64_t&>(r))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return r;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// ------------------------------------------------------------------ host side ----

inline bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
inline uint32_t size_of(uint32_t dtype) { return dtype == MFET_F32 ? 4 : 2; }

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// A function of the driver, by name; `found` keeps it
inline void* driver_function(const char* name, std::atomic<void*>* found) {
  void* f = found->load(std::memory_order_acquire);
  if (f) return f;
  cudaDriverEntryPointQueryResult r;
  if (cudaGetDriverEntryPoint(name, &f, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess) {
    cudaGetLastError();
    return nullptr;
  }
  found->store(f, std::memory_order_release);
  return f;
}

// The driver's function that describes a tile to the copy engine. It wants a context to be the calling thread's. A thread that makes its first call here
// may have none yet: it gets the one of its GPU. A context that the caller has made current, of whatever kind, stays.
inline EncodeTiled encode_tiled() {
  static std::atomic<void*> encode{nullptr}, get_current{nullptr};
  const auto current = reinterpret_cast<CUresult (*)(CUcontext*)>(driver_function("cuCtxGetCurrent", &get_current));
  CUcontext context = nullptr;
  if (!current) return nullptr;
  if (current(&context) != CUDA_SUCCESS || !context) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaSetDevice(dev) != cudaSuccess) {
      cudaGetLastError();
      return nullptr;
    }
  }
  return reinterpret_cast<EncodeTiled>(driver_function("cuTensorMapEncodeTiled", &encode));
}

// Lets a kernel use `bytes` of dynamic shared memory on the current GPU: always the same number for a kernel, so that no thread takes away
// what another one is about to launch with. ready: one bit per GPU where that is done.
template <typename K>
cudaError_t allow_smem(K kernel, uint32_t bytes, std::atomic<uint64_t>* ready) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (ready->load(std::memory_order_relaxed) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess) ready->fetch_or(bit, std::memory_order_relaxed);
  return e;
}

}  // namespace mfet
