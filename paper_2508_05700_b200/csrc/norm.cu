// Layer norm over the columns of a row, and its backward pass.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) r, y = xh w + b
//   t = dy w:  dx = r (t - mean(t) - xh mean(t xh)),  dw = sum over rows of dy xh,  db = sum over rows of dy
//
// Bound by memory: x is read once and kept in registers, the variance is taken of the differences d = x - mu (no cancellation for rows far
// from 0), and the backward pass computes mu and r from x again instead of reading them. Two rounds of sums a row: the mean,
// then the squares of d and, backward, t and t d with them (mean(t xh) is r mean(t d)). Everything is fp32 inside.
#include <type_traits>

#include "tensor.cuh"

using namespace mfet;

namespace mfet {
namespace {

constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kChunk = 8;             // neighbouring columns of a thread, for rows of more than
// Columns: the longest row that registers hold, of 16 warps. 1024 x 16384 to bf16: 30 us (bf16) and 35 (fp32) held, 46 and 55 by the kernel for longer rows;
// backward 68 and 70, 272 and 285.
constexpr int64_t kMostHeld = 16384;
constexpr int kLongThreads = 512;

struct NormParams {
  const void *x, *dy;  // dy: backward
  void* y;             // forward: y; backward: dx, of x's type
  const float *w, *b;
  float* partial;      // backward: the blocks' sums of dy xh and of dy; NULL: no sums wanted
  int64_t rows, cols, x_ld, y_ld, dy_ld;
  const void *x_end, *dy_end;
  float eps;
  uint32_t dy_dtype, y_dtype;
  bool x_vec, y_vec, dy_vec, w_vec, b_vec;  // rows start on 16-byte boundaries
};

template <int DT>
__device__ __forceinline__ Raw<DT, kChunk> chunk_in(const void* base, int64_t at, int count, bool vec, const void* end) {
  const typename Elem<DT>::T* p = reinterpret_cast<const typename Elem<DT>::T*>(base) + at;
  if (vec) return load_raw<DT, kChunk, true>(p, count);
  return load_shifted<DT, kChunk>(p, count, base, end);
}
// 8 values of a type that is only known here, widened
__device__ __forceinline__ void chunk_any(uint32_t dtype, const void* base, int64_t at, int count, bool vec, const void* end, float* v) {
  if (dtype == MFET_F32) widen_raw<MFET_F32, kChunk>(chunk_in<MFET_F32>(base, at, count, vec, end), v);
  else if (dtype == MFET_F16) widen_raw<MFET_F16, kChunk>(chunk_in<MFET_F16>(base, at, count, vec, end), v);
  else widen_raw<MFET_BF16, kChunk>(chunk_in<MFET_BF16>(base, at, count, vec, end), v);
}
template <int DT>
__device__ __forceinline__ void chunk_out(void* base, int64_t at, const float* v, int count, bool vec) {
  typename Elem<DT>::T* p = reinterpret_cast<typename Elem<DT>::T*>(base) + at;
  if (vec) store_values<DT, kChunk, true>(p, v, count);
  else store_values<DT, kChunk, false>(p, v, count);
}
__device__ __forceinline__ void chunk_put(uint32_t dtype, void* base, int64_t at, const float* v, int count, bool vec) {
  if (dtype == MFET_F32) chunk_out<MFET_F32>(base, at, v, count, vec);
  else if (dtype == MFET_F16) chunk_out<MFET_F16>(base, at, v, count, vec);
  else chunk_out<MFET_BF16>(base, at, v, count, vec);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kAll, v, d);
  return v;
}

// The sum over the threads of a block, the same in all of them. `turn` alternates: two sums in a row use different words.
__device__ __forceinline__ float block_sum(float v, float (*shared)[kLongThreads / 32], int* turn) {
  v = warp_sum(v);
  float* words = shared[*turn];
  *turn ^= 1;
  if ((threadIdx.x & 31) == 0) words[threadIdx.x >> 5] = v;
  __syncthreads();
  v = words[0];
#pragma unroll
  for (int i = 1; i < kLongThreads / 32; ++i) v += words[i];
  return v;
}

// 8 neighbouring weights of columns c and on; `none` where there are no weights or no columns
__device__ __forceinline__ void params8(const float* w, int64_t c, int64_t cols, bool vec, float none, float* v) {
  if (w && vec && c + kChunk <= cols) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(w + c)), b = __ldg(reinterpret_cast<const float4*>(w + c) + 1);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    return;
  }
#pragma unroll
  for (int j = 0; j < kChunk; ++j) v[j] = w && c + j < cols ? __ldg(w + c + j) : none;
}

// s / n, rounded like a quotient (one correction): the mean of equal values is that value
__device__ __forceinline__ float over(float s, float n, float inv_n) {
  const float q = s * inv_n;
  return fmaf(fmaf(-q, n, s), inv_n, q);
}

__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
// ... of which the first `bytes` are read and the others 0; from 0 bytes on nothing is
__device__ __forceinline__ void copy_part(uint32_t to, const void* from, int bytes) {
  const int n = bytes < 0 ? 0 : bytes > 16 ? 16 : bytes;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(n > 0 ? from : static_cast<const char*>(from) - 16), "r"(n) : "memory");
}
__device__ __forceinline__ void store16_shared(uint32_t to, const uint4& v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
template <typename T>
__device__ __forceinline__ void store_shared(uint32_t to, T v) {
  if constexpr (sizeof(T) == 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to), "r"(reinterpret_cast<const uint32_t&>(v)) : "memory");
  else asm volatile("st.shared.b16 [%0], %1;" ::"r"(to), "h"(reinterpret_cast<const uint16_t&>(v)) : "memory");
}
__device__ __forceinline__ uint32_t load4_shared(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint4 load16_shared(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}

// A row of results at any address: from shared memory, where it lies under the same address modulo 16, in whole units; the units at its ends
// value by value. (4 values a thread straight to memory: several times the transactions.)
__device__ __forceinline__ void row_out(uint8_t* to, const uint8_t* from, uint32_t head, uint32_t bytes, uint32_t size, int lane, int threads) {
  const uint32_t units = (head + bytes + 15) / 16;
  for (uint32_t u = lane; u < units; u += threads) {
    const uint32_t lo = max(16 * u, head), hi = min(16 * u + 16, head + bytes);
    if (hi - lo == 16) {
      *reinterpret_cast<uint4*>(to + 16 * u - head) = *reinterpret_cast<const uint4*>(from + 16 * u);
    } else if (size == 4) {
      for (uint32_t i = lo; i < hi; i += 4) *reinterpret_cast<uint32_t*>(to + i - head) = *reinterpret_cast<const uint32_t*>(from + i);
    } else {
      for (uint32_t i = lo; i < hi; i += 2) *reinterpret_cast<uint16_t*>(to + i - head) = *reinterpret_cast<const uint16_t*>(from + i);
    }
  }
}

// The block's sums for dw and db into its part of `partial`, as its threads hold them: word (which * NQ + i) * 4 + j of thread `lane` of a row is
// at that word times TPR plus lane (the kernel that adds up the blocks puts columns in order). Several groups leave theirs in shared memory
// (`sums`: 8 NQ words a thread) first, and each word is added up over them in their order.
template <int NQ, int GROUPS, int TPR>  // groups of a block and threads of a group
__device__ __forceinline__ void block_sums(const NormParams& p, float* sums, int group, int lane, const float2 (*dw)[2], const float2 (*db)[2]) {
  if (!p.partial) return;
  constexpr int kWords = 8 * NQ, kPitch = GROUPS * TPR;
  float* const to = p.partial + (int64_t)blockIdx.x * kWords * TPR + lane;
  auto word = [&](const float2 (*v)[2], int i, int j) { return j & 1 ? v[i][j >> 1].y : v[i][j >> 1].x; };
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (GROUPS > 1) {
        sums[(i * 4 + j) * kPitch + threadIdx.x] = word(dw, i, j);
        sums[((NQ + i) * 4 + j) * kPitch + threadIdx.x] = word(db, i, j);
      } else if (MFET_INSIDE(nullptr, lane < TPR)) {
        to[(i * 4 + j) * TPR] = word(dw, i, j);
        to[((NQ + i) * 4 + j) * TPR] = word(db, i, j);
      }
    }
  }
  if constexpr (GROUPS > 1) {
    __syncthreads();
    for (int e = group; e < kWords; e += GROUPS) {
      const float* from = sums + e * kPitch + lane;
      float v = from[0];
#pragma unroll
      for (int g = 1; g < GROUPS; ++g) v += from[g * TPR];
      if (MFET_INSIDE(nullptr, lane < TPR)) to[e * TPR] = v;
    }
  }
}

// ------------------------------------------------------------------ rows that registers hold ----

// Threads of a block of the kernel below. Backward one block per SM, as large as its registers let it be (some 160 with 32 columns a thread;
// at 128 it spilt: 37 us instead of 27 for 8192 x 896), since each leaves sums of all columns.
template <int NQ, int W, bool BACK>
constexpr int norm_threads = W == 16 ? 512 : !BACK || W == 8 ? 256 : NQ > 4 ? 384 : 512;

// What a block of it has in shared memory
template <int DT, int OT, int NQ, int W, bool BACK, bool ALIGNED>
struct NormShape {
  static constexpr int threads = norm_threads<NQ, W, BACK>, tpr = 32 * W, groups = threads / tpr;
  static constexpr int xs = (int)sizeof(typename Elem<DT>::T), os = (int)sizeof(typename Elem<OT>::T);
  static constexpr uint32_t pad = ALIGNED ? 0 : 16;
  static constexpr uint32_t x_bytes = NQ * tpr * 4 * xs + pad, dy_bytes = BACK ? NQ * tpr * 4 * os + pad : 0, stage = x_bytes + dy_bytes;  // a row
  static constexpr int stages = W == 16 && BACK && xs + os == 8 ? 1 : 2;  // rows of a group: computed and under way
  static constexpr uint32_t out_at = groups * stages * stage, out_bytes = ALIGNED || BACK ? 0 : NQ * tpr * 4 * os + pad;  // results (backward: over x)
  static constexpr uint32_t w_at = out_at + groups * out_bytes, w_bytes = W <= 8 ? NQ * tpr * 16 : 0;
  static constexpr uint32_t rows_end = w_at + w_bytes * (BACK ? 1 : 2), sums = BACK && groups > 1 ? threads * NQ * 32 : 0;
  static constexpr uint32_t smem = rows_end > sums ? rows_end : sums;
  static constexpr int per_sm = BACK || W == 16 ? 1 : smem <= 74 * 1024 ? 3 : smem <= 112 * 1024 ? 2 : 1;
  // quads that are full for all threads: no more are taken than rows of a size need (see columns_of)
  static constexpr int sure = W > 1 || NQ == 7 ? 4 : NQ == 8 ? (ALIGNED ? 7 : 4) : NQ == 4 ? (ALIGNED ? 2 : 1) : NQ / 2;
  template <int SIZE>
  static constexpr int pieces = (NQ * SIZE + 3) / 4 + (ALIGNED ? 0 : 1);  // that a thread fetches
  static_assert(smem <= 227 * 1024 - 1024, "shared memory of a block");
  static_assert(W == 1 || groups < 16, "named barriers");
};

// 4 values of a type in shared memory. ALIGNED: to all of their bytes; else to their type, `odd`: not to 4 bytes.
template <int DT, bool ALIGNED>
__device__ __forceinline__ void quad_in(uint32_t at, bool odd, float2* v) {
  if constexpr (DT == MFET_F32) {
    uint4 a;
    if constexpr (ALIGNED) a = load16_shared(at);
    else a = make_uint4(load4_shared(at), load4_shared(at + 4), load4_shared(at + 8), load4_shared(at + 12));
    v[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y));
    v[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
  } else {
    uint32_t a, b;
    if constexpr (ALIGNED) {
      asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(a), "=r"(b) : "r"(at) : "memory");
    } else {
      const uint32_t from = at & ~3u;
      a = load4_shared(from);
      b = load4_shared(from + 4);
      if (odd) {
        const uint32_t c = load4_shared(from + 8);
        a = __byte_perm(a, b, 0x5432);
        b = __byte_perm(b, c, 0x5432);
      }
    }
    v[0] = Elem<DT>::widen(a);
    v[1] = Elem<DT>::widen(b);
  }
}
__device__ __forceinline__ void keep(float2* v, int count) {  // the first `count` of 4 values, the others 0
  if (count < 1) v[0].x = 0.f;
  if (count < 2) v[0].y = 0.f;
  if (count < 3) v[1].x = 0.f;
  if (count < 4) v[1].y = 0.f;
}
template <int DT>
__device__ __forceinline__ void quad_out(typename Elem<DT>::T* to, const float2* v, int count) {
  if (count == 4) {
    if constexpr (DT == MFET_F32) *reinterpret_cast<float4*>(to) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
    else *reinterpret_cast<uint2*>(to) = make_uint2(Elem<DT>::pack(v[0].x, v[0].y), Elem<DT>::pack(v[1].x, v[1].y));
  } else {
    if (count > 0) to[0] = Elem<DT>::from(v[0].x);
    if (count > 1) to[1] = Elem<DT>::from(v[0].y);
    if (count > 2) to[2] = Elem<DT>::from(v[1].x);
  }
}
// ... to shared memory, at any address of the type
template <int DT>
__device__ __forceinline__ void quad_stage(uint32_t to, bool odd, const float2* v, int count) {
  constexpr int kSize = (int)sizeof(typename Elem<DT>::T);
  if (DT != MFET_F32 && !odd && count == 4) {
    if constexpr (DT != MFET_F32) {
      store_shared(to, Elem<DT>::pack(v[0].x, v[0].y));
      store_shared(to + 4, Elem<DT>::pack(v[1].x, v[1].y));
    }
    return;
  }
  if (count > 0) store_shared(to, Elem<DT>::from(v[0].x));
  if (count > 1) store_shared(to + kSize, Elem<DT>::from(v[0].y));
  if (count > 2) store_shared(to + 2 * kSize, Elem<DT>::from(v[1].x));
  if (count > 3) store_shared(to + 3 * kSize, Elem<DT>::from(v[1].y));
}

// W warps take a row of up to 1024 W columns (most instructions of a row do not depend on its columns: sums over lanes, barriers, addresses), a
// lane 4 neighbouring ones of every 128 W, so that every access of a warp is whole lines of memory and of shared memory (8 neighbouring ones:
// fp32 rows were fetched by halves of sectors, twice). The next row is under way to shared memory in pieces of 16 bytes; arithmetic
// goes two columns an instruction, and all distances are known to the compiler (with the threads of a row and of a block known at run
// time, 500 of a row's 1140 instructions formed addresses). Rows on 16-byte boundaries: columns behind the row's end are
// zeros with weight 0 and mean 0, so that nothing asks for them but the stores. Other rows are fetched in the pieces that hold them, read
// from shared memory where their values lie, and written from there.
// Backward with the sum of the blocks' parts, 8192 x 896, fp32 x, bf16 dy: a warp per row with its row in registers 56 us, 16 columns a thread
// 25, this 17.5 (the same inputs again and again, of which L2 holds a part; three sets of inputs in turn 21.2); 16384 x 2048 bf16 44, 201 MB at 4.6 TB/s.
template <int DT, int OT, int NQ, int W, bool BACK, bool ALIGNED>
__global__ void __launch_bounds__((norm_threads<NQ, W, BACK>), BACK || W == 16 ? 1 : 3) norm_kernel(const __grid_constant__ NormParams p) {
  using S = NormShape<DT, OT, NQ, W, BACK, ALIGNED>;
  constexpr int tpr = S::tpr, kXs = S::xs, kOs = S::os, kYs = BACK ? kXs : kOs, kType = BACK ? DT : OT;
  __shared__ float words[2][16][4];
  extern __shared__ __align__(16) uint8_t ring[];
  early_launch_wait();
  const int group = threadIdx.x / tpr, lane = threadIdx.x % tpr, warp0 = group * W;
  const uint32_t base = smem_addr(ring), mine = base + group * S::stages * S::stage;
  const uint32_t w_at = base + S::w_at + lane * 16, b_at = w_at + S::w_bytes;
  const bool ragged = p.cols % 4 != 0;
  const int cols = (int)p.cols;
  int count[NQ];  // columns of a quad
#pragma unroll
  for (int i = 0; i < NQ; ++i) count[i] = i < S::sure ? 4 : max(0, min(4, cols - (i * tpr + lane) * 4));
  const int64_t row0 = (int64_t)blockIdx.x * S::groups + group, step = (int64_t)gridDim.x * S::groups;
  // of the row that is computed; the one that is asked for next is `ahead` rows of this group further on
  const uint8_t* x_row = reinterpret_cast<const uint8_t*>(p.x) + row0 * p.x_ld * kXs;
  const uint8_t* dy_row = BACK ? reinterpret_cast<const uint8_t*>(p.dy) + row0 * p.dy_ld * kOs : nullptr;
  uint8_t* y_row = reinterpret_cast<uint8_t*>(p.y) + row0 * p.y_ld * kYs;
  const int64_t x_step = step * p.x_ld * kXs, dy_step = BACK ? step * p.dy_ld * kOs : 0, y_step = step * p.y_ld * kYs;
  int64_t left = row0 < p.rows ? (p.rows - row0 + step - 1) / step : 0;  // rows of this group
  auto meet = [&]() {
    if constexpr (W == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(tpr) : "memory");
  };
  if constexpr (ALIGNED) {  // zeros behind the rows' ends: nothing else is written there
    for (int at = lane * 16; at < (int)(S::stages * S::stage); at += tpr * 16) store16_shared(mine + at, make_uint4(0, 0, 0, 0));
    meet();
  }
  // the row at `row` into the pieces of 16 bytes from `to` on (from the piece that its first value is in)
  auto fetch = [&](uint32_t to, const uint8_t* row, const void* lo, int size, auto pieces) {
    const int head = ALIGNED ? 0 : (int)(reinterpret_cast<uintptr_t>(row) & 15), bytes = head + cols * size - lane * 16;
    const uint8_t* from = row - head + lane * 16;
#pragma unroll
    for (int k = 0; k < decltype(pieces)::value; ++k) {
      const int n = bytes - k * tpr * 16;
      const uint32_t at = to + (lane + k * tpr) * 16;
      if (!ALIGNED && k == 0 && lane == 0 && from < static_cast<const uint8_t*>(lo)) {  // the array begins inside this piece
        for (int e = head; e < 16 && e < n; e += size) {
          if (size == 4) store_shared(at + e, *reinterpret_cast<const uint32_t*>(from + e));
          else store_shared(at + e, *reinterpret_cast<const uint16_t*>(from + e));
        }
      } else if (n >= 16) {
        copy16(at, from + k * tpr * 16);
      } else if (n > 0) {
        copy_part(at, from + k * tpr * 16, n);
      }
    }
  };
  auto request = [&](uint32_t to, bool any, int64_t ahead) {
    if (any && MFET_INSIDE(nullptr, p.cols <= p.x_ld && p.cols <= NQ * tpr * 4)) {
      fetch(to, x_row + ahead * x_step, p.x, kXs, std::integral_constant<int, S::template pieces<kXs>>());
      if constexpr (BACK) fetch(to + S::x_bytes, dy_row + ahead * dy_step, p.dy, kOs, std::integral_constant<int, S::template pieces<kOs>>());
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  request(mine, left > 0, 0);
  // weight and bias as a group's threads read them; every group writes the same values
  auto param = [&](const float* v, float none, int i, float* a) {
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = j < count[i] ? (v ? __ldg(v + (i * tpr + lane) * 4 + j) : none) : 0.f;
  };
  if constexpr (W <= 8) {
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      float a[4];
      param(p.w, 1.f, i, a);
      store16_shared(w_at + i * tpr * 16, narrow16<MFET_F32>(a));
      if constexpr (!BACK) {
        param(p.b, 0.f, i, a);
        store16_shared(b_at + i * tpr * 16, narrow16<MFET_F32>(a));
      }
    }
  }
  auto weights = [&](uint32_t at, const float* from, float none, int i, float2* v) {
    if constexpr (W <= 8) {
      quad_in<MFET_F32, true>(at + i * tpr * 16, false, v);
    } else {  // no room for them
      float a[4];
      param(from, none, i, a);
      v[0] = make_float2(a[0], a[1]);
      v[1] = make_float2(a[2], a[3]);
    }
  };
  float2 dw[BACK ? NQ : 1][2], db[BACK ? NQ : 1][2];
#pragma unroll
  for (int i = 0; i < (BACK ? NQ : 0); ++i) dw[i][0] = dw[i][1] = db[i][0] = db[i][1] = both(0.f);
  int turn = 0;
  // the sums over a warp's lanes to the group, in all its threads: `v` of lanes 0, 16 and 8 is what the warp has of x, y and z
  auto joined = [&](float v, auto three) {
    constexpr bool kThree = decltype(three)::value;
    float3 r = make_float3(0.f, 0.f, 0.f);
    if constexpr (W == 1) {
      r.x = __shfl_sync(kAll, v, 0);
      if constexpr (kThree) r.y = __shfl_sync(kAll, v, 16), r.z = __shfl_sync(kAll, v, 8);
    } else {
      float(*at)[4] = words[turn] + warp0;
      turn ^= 1;
      const int l = lane & 31;
      if (l == 0) at[lane >> 5][0] = v;
      if constexpr (kThree) {
        if (l == 16) at[lane >> 5][1] = v;
        if (l == 8) at[lane >> 5][2] = v;
      }
      meet();
#pragma unroll
      for (int q = 0; q < W; ++q) {
        const float4 f = *reinterpret_cast<const float4*>(at[q]);
        r.x += f.x;
        if constexpr (kThree) r.y += f.y, r.z += f.z;
      }
    }
    return r;
  };
  const float n = (float)cols, inv_n = 1.f / n;
  uint32_t from = mine, to = mine + (S::stages - 1) * S::stage;
  __syncthreads();  // the weights
  for (; left > 0; --left) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    meet();  // this row has arrived for all, and the last one is done with
    if constexpr (S::stages == 2) request(to, left > 1, 1);
    const uint32_t x_head = ALIGNED ? 0 : (uint32_t)reinterpret_cast<uintptr_t>(x_row) & 15, dy_head = ALIGNED ? 0 : (uint32_t)reinterpret_cast<uintptr_t>(dy_row) & 15;
    const uint32_t x_at = from + x_head + lane * 4 * kXs, dy_at = from + S::x_bytes + dy_head + lane * 4 * kOs;
    const bool x_odd = x_head & 2, dy_odd = dy_head & 2;
    float2 v[NQ][2], s = both(0.f);
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      quad_in<DT, ALIGNED>(x_at + i * tpr * 4 * kXs, x_odd, v[i]);
      if (!ALIGNED && i >= S::sure) keep(v[i], count[i]);
      s = add2(s, add2(v[i][0], v[i][1]));
    }
    const float mu = over(joined(warp_sum(s.x + s.y), std::false_type()).x, n, inv_n);
    float2 s0 = both(0.f), s1 = both(0.f), s2 = both(0.f), t[2], w[2];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const float2 minus = both(i < S::sure || count[i] > 0 ? -mu : 0.f);
      v[i][0] = add2(v[i][0], minus);
      v[i][1] = add2(v[i][1], minus);
      if (i >= S::sure && ragged) keep(v[i], count[i]);  // the row may end inside this quad
      if constexpr (BACK) {
        quad_in<OT, ALIGNED>(dy_at + i * tpr * 4 * kOs, dy_odd, t);
        if (!ALIGNED && i >= S::sure) keep(t, count[i]);
        weights(w_at, p.w, 1.f, i, w);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        s0 = fma2(v[i][j], v[i][j], s0);
        if constexpr (BACK) {
          const float2 tw = mul2(t[j], w[j]);
          s1 = add2(s1, tw);
          s2 = fma2(tw, v[i][j], s2);
        }
      }
    }
    float3 q;
    if constexpr (BACK) {
      // three sums in six exchanges: half of the lanes go on with x and half with y, then half of each with z
      const int l = lane & 31;
      const float x = s0.x + s0.y, y = s1.x + s1.y;
      float z = s2.x + s2.y;
      float a = (l & 16 ? y : x) + __shfl_xor_sync(kAll, l & 16 ? x : y, 16);
      z += __shfl_xor_sync(kAll, z, 16);
      a = (l & 8 ? z : a) + __shfl_xor_sync(kAll, l & 8 ? a : z, 8);
#pragma unroll
      for (int d = 4; d > 0; d >>= 1) a += __shfl_xor_sync(kAll, a, d);
      q = joined(a, std::true_type());
    } else {
      q = joined(warp_sum(s0.x + s0.y), std::false_type());
    }
    const float r = rsqrtf(fmaf(q.x, inv_n, p.eps));
    const float2 rr = both(r), m0 = both(-(q.y * inv_n)), m1 = both(-(q.z * inv_n * r));
    const uint32_t y_head = (uint32_t)reinterpret_cast<uintptr_t>(y_row) & 15;
    // all have read this row's x by now: backward, the results take its place
    const uint32_t stage = BACK ? from - base : S::out_at + group * S::out_bytes;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      float2 b[2], o[2];
      weights(w_at, p.w, 1.f, i, w);
      if constexpr (BACK) {
        quad_in<OT, ALIGNED>(dy_at + i * tpr * 4 * kOs, dy_odd, t);
        if (!ALIGNED && i >= S::sure) keep(t, count[i]);
      } else {
        weights(b_at, p.b, 0.f, i, b);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float2 xh = mul2(v[i][j], rr);
        if constexpr (BACK) {
          db[i][j] = add2(db[i][j], t[j]);
          dw[i][j] = fma2(t[j], xh, dw[i][j]);
          // Short rows: t is rounded as in its mean, so that a row of one column has the gradient 0 (the two-number forms of product and
          // sum would be joined to one rounding; 16384 x 2048: 43.0 us, 41.6 without).
          float2 d;
          if constexpr (NQ == 1) d = add2(make_float2(__fmul_rn(t[j].x, w[j].x), __fmul_rn(t[j].y, w[j].y)), m0);
          else d = fma2(t[j], w[j], m0);
          o[j] = mul2(fma2(xh, m1, d), rr);
        } else {
          o[j] = fma2(xh, w[j], b[j]);
        }
      }
      const int c = (i * tpr + lane) * 4, live = i < S::sure ? 4 : count[i];
      if constexpr (!ALIGNED) quad_stage<kType>(base + stage + y_head + c * kYs, y_head & 2, o, live);
      else if (MFET_INSIDE(nullptr, c + live <= p.y_ld || live == 0)) quad_out<kType>(reinterpret_cast<typename Elem<kType>::T*>(y_row) + c, o, live);
    }
    if constexpr (!ALIGNED) {
      meet();
      if (MFET_INSIDE(nullptr, p.cols <= p.y_ld)) row_out(y_row, ring + stage, y_head, (uint32_t)(cols * kYs), kYs, lane, tpr);
    }
    if constexpr (S::stages == 1) {
      meet();
      request(from, left > 1, 1);
    }
    const uint32_t next = to;
    to = from;
    from = next;
    x_row += x_step;
    if constexpr (BACK) dy_row += dy_step;
    y_row += y_step;
  }
  if constexpr (BACK) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    block_sums<NQ, S::groups, tpr>(p, reinterpret_cast<float*>(ring), group, lane, dw, db);
  }
}

// Rows that registers do not hold: a block per row reads it once for each sum and once more for the result (from L2). BACK: the
// block's sums over its rows stay in its part of `partial`. Bound by latency, with one chunk of a thread under way at a time: 1024 x 20000 to bf16 takes
// 60 us (bf16) and 70 (fp32), floors 12.5 and 18.8; backward 322 and 339, where every row also goes through the block's sums in memory.
template <bool BACK>
__global__ void __launch_bounds__(kLongThreads) norm_long_kernel(const __grid_constant__ NormParams p, uint32_t x_dtype) {
  __shared__ float shared[2][kLongThreads / 32];
  early_launch_wait();
  int turn = 0;
  float* const to = BACK && p.partial ? p.partial + (int64_t)blockIdx.x * 2 * p.cols : nullptr;
  const float n = (float)p.cols;
  bool fresh = true;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, fresh = false) {
    auto each = [&](auto f) {
      for (int64_t c = (int64_t)threadIdx.x * kChunk; c < p.cols; c += (int64_t)kLongThreads * kChunk) {
        const int count = (int)min((int64_t)kChunk, p.cols - c);
        if (!MFET_INSIDE(nullptr, row < p.rows && c + count <= p.x_ld)) continue;
        float v[kChunk];
        chunk_any(x_dtype, p.x, row * p.x_ld + c, count, p.x_vec, p.x_end, v);
        f(c, count, v);
      }
    };
    auto grad = [&](int64_t c, int count, float* t) {
      if (MFET_INSIDE(nullptr, c + count <= p.dy_ld)) chunk_any(p.dy_dtype, p.dy, row * p.dy_ld + c, count, p.dy_vec, p.dy_end, t);
    };
    float s = 0.f;
    each([&](int64_t, int count, float* v) {
      for (int j = 0; j < count; ++j) s += v[j];
    });
    // A thread adds up so many values that the mean is off by more than its rounding (1.9 throughout 2^22 columns: by 1.5e-4). The mean of what is left
    // of the values puts that right.
    const float mu = block_sum(s, shared, &turn) / n;
    s = 0.f;
    float q = 0.f;
    each([&](int64_t, int count, float* v) {
      for (int j = 0; j < count; ++j) {
        const float d = v[j] - mu;
        q += d;
        s = fmaf(d, d, s);
      }
    });
    const float rest = block_sum(q, shared, &turn) / n, raw = block_sum(s, shared, &turn) / n - rest * rest;
    const float r = 1.f / sqrtf((raw < 0.f ? 0.f : raw) + p.eps);  // NaN stays NaN
    auto centred = [&](float v) { return (v - mu) - rest; };
    if constexpr (!BACK) {
      each([&](int64_t c, int count, float* v) {
        float w[kChunk], b[kChunk];
        params8(p.w, c, p.cols, p.w_vec, 1.f, w);
        params8(p.b, c, p.cols, p.b_vec, 0.f, b);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) v[j] = fmaf(centred(v[j]) * r, w[j], b[j]);
        if (MFET_INSIDE(nullptr, c + count <= p.y_ld)) chunk_put(p.y_dtype, p.y, row * p.y_ld + c, v, count, p.y_vec);
      });
    } else {
      float s0 = 0.f, s1 = 0.f;
      each([&](int64_t c, int count, float* v) {
        float w[kChunk], t[kChunk];
        grad(c, count, t);
        params8(p.w, c, p.cols, p.w_vec, 1.f, w);
        for (int j = 0; j < count; ++j) {
          const float xh = centred(v[j]) * r;
          if (to) {
            to[c + j] = fresh ? t[j] * xh : fmaf(t[j], xh, to[c + j]);
            to[p.cols + c + j] = fresh ? t[j] : to[p.cols + c + j] + t[j];
          }
          s0 = fmaf(t[j], w[j], s0);
          s1 = fmaf(t[j] * w[j], xh, s1);
        }
      });
      const float m0 = block_sum(s0, shared, &turn) / n, m1 = block_sum(s1, shared, &turn) / n;
      each([&](int64_t c, int count, float* v) {
        float w[kChunk], t[kChunk];
        grad(c, count, t);
        params8(p.w, c, p.cols, p.w_vec, 1.f, w);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) v[j] = r * (t[j] * w[j] - m0 - centred(v[j]) * r * m1);
        if (MFET_INSIDE(nullptr, c + count <= p.y_ld)) chunk_put(x_dtype, p.y, row * p.y_ld + c, v, count, p.y_vec);
      });
    }
  }
}

// The blocks' sums in their order: 32 threads for each word take every 32nd block.
constexpr int kSumWords = 8;
struct SumParams {
  const float* partial;
  float *dw, *db;
  int64_t cols;
  uint32_t blocks;
  int words, tpr, nq;  // words of a block; how they belong to columns (nq = 0: dw's columns, then db's)
};
__global__ void __launch_bounds__(32 * kSumWords) norm_sum_kernel(const __grid_constant__ SumParams p) {
  __shared__ float part[32][kSumWords + 1];
  early_launch_wait();
  const int word = threadIdx.x % kSumWords, seg = threadIdx.x / kSumWords;
  const int64_t at = (int64_t)blockIdx.x * kSumWords + word;
  float s = 0.f;
  if (at < p.words) {
#pragma unroll 4
    for (uint32_t b = seg; b < p.blocks; b += 32) s += p.partial[(int64_t)b * p.words + at];
  }
  part[seg][word] = s;
  __syncthreads();
  s = part[threadIdx.x & 31][threadIdx.x >> 5];  // a warp per word
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(kAll, s, d);
  const int64_t mine = (int64_t)blockIdx.x * kSumWords + (threadIdx.x >> 5);
  if ((threadIdx.x & 31) == 0 && mine < p.words) {
    int64_t c = mine;
    bool bias;
    if (p.nq) {
      const int e = (int)(mine / p.tpr), lane = (int)(mine - (int64_t)e * p.tpr), i = e / 4 % p.nq;
      bias = e / 4 >= p.nq;
      c = (int64_t)(i * p.tpr + lane) * 4 + e % 4;
    } else {
      bias = mine >= p.cols;
      c = bias ? mine - p.cols : mine;
    }
    float* to = bias ? p.db : p.dw;
    if (to && c < p.cols && MFET_INSIDE(nullptr, c >= 0)) to[c] = s;
  }
}

// ------------------------------------------------------------------ host side ----

bool on_16(const void* p, int64_t ld, uint32_t dtype) { return aligned(p, 16) && (uint64_t)ld * size_of(dtype) % 16 == 0; }
const void* end_of(const void* p, int64_t rows, int64_t cols, int64_t ld, uint32_t dtype) {
  return (const uint8_t*)p + ((rows - 1) * ld + cols) * size_of(dtype);
}
bool bad_matrix(int64_t rows, int64_t cols, int64_t ld, uint32_t dtype) {
  return dtype > MFET_BF16 || rows < 0 || rows >= (1ll << 31) || cols < 1 || cols >= (1ll << 30) || ld < cols || ld >= (1ll << 31);
}

// How a row is spread over threads: quads of each, warps of a row (0: the kernel for longer rows)
struct Columns {
  int nq, w;
};
Columns columns_of(int64_t cols, bool aligned_rows) {
  // The fewest quads and warps that hold a row, of those that there are; figures to bf16, of bf16 and of fp32 rows, backward in brackets:
  //   65536 x 128   one quad 14.4, 15.6 (23.6, 26.4), two 15.1, 20.9 (24.8, 27.5)
  //   32768 x 256   two 10.4, 14.0 (16.4, 20.6), four 15.1, 17.0 (23.1, 25.1)
  //   16384 x 512   four 11.2, 13.1 (15.9, 19.9), seven 12.7, 15.1 (22.8, 27.6)
  //   16384 x 640   seven 13.5, 16.0 (23.6, 31.1), eight 14.6, 17.6 (27.4, 38.3)
  //   8192 x 896    seven 10.7, 12.6 (16.3, 21.5), eight 11.3, 13.6 (18.8, 26.4), two warps 11.9, 13.9 (22.4, 24.5)
  //   8192 x 1024   eight 11.8, 14.3 (19.5, 27.8), two warps 12.1, 14.4 (22.5, 24.6)
  //   1024 x 8192   eight warps 12.1, 14.6 (22.5, 24.9), sixteen 22.6, 24.8 (58.5, 58.7)
  if (cols > kMostHeld) return {0, 0};
  // 6 quads in place of 8: 4099 x 1075, bf16 to fp16 at any address 11.4 us, 12.9; 8192 x 1280 of these types 12.4, 14.9, backward 20.4, 25.2
  for (int w = 2; w <= 16; w *= 2)
    if (cols > 512 * w && cols <= 1024 * w) return {w < 16 && cols <= 768 * w ? 6 : 8, w};
  if (cols <= 128) return {1, 1};
  if (cols <= 512) return {aligned_rows && cols <= 256 ? 2 : 4, 1};
  return {aligned_rows && cols <= 896 ? 7 : 8, 1};
}
// rows of a block at a time, backward
int groups_of(const Columns& c) { return c.w == 0 ? 1 : (c.w == 16 ? 512 : c.w == 8 ? 256 : c.nq > 4 ? 384 : 512) / (32 * c.w); }
int64_t back_blocks(int64_t rows, const Columns& c) {
  const int64_t want = (rows + groups_of(c) - 1) / groups_of(c), most = (int64_t)sm_count() * (c.w == 0 ? 2 : 1);
  return want < most ? want : most;
}
// sums that a block of the backward pass leaves
int64_t words_of(int64_t cols, const Columns& c) { return c.w ? 8ll * c.nq * 32 * c.w : 2 * cols; }

template <int DT, int OT, int NQ, int W, bool BACK, bool ALIGNED>
cudaError_t launch_norm(const NormParams& p, cudaStream_t s) {
  using S = NormShape<DT, OT, NQ, W, BACK, ALIGNED>;
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem(norm_kernel<DT, OT, NQ, W, BACK, ALIGNED>, S::smem, &ready);
  const int64_t want = (p.rows + S::groups - 1) / S::groups, most = (int64_t)sm_count() * S::per_sm;
  return e != cudaSuccess ? e : launch_early(norm_kernel<DT, OT, NQ, W, BACK, ALIGNED>, (unsigned)(want < most ? want : most), S::threads, S::smem, s, p);
}
template <int DT, int OT, bool BACK>
cudaError_t launch_types(const NormParams& p, bool aligned_rows, cudaStream_t s) {
  const Columns c = columns_of(p.cols, aligned_rows);
  if (aligned_rows) {
    switch (c.w * 16 + c.nq) {
      case 17: return launch_norm<DT, OT, 1, 1, BACK, true>(p, s);
      case 18: return launch_norm<DT, OT, 2, 1, BACK, true>(p, s);
      case 20: return launch_norm<DT, OT, 4, 1, BACK, true>(p, s);
      case 23: return launch_norm<DT, OT, 7, 1, BACK, true>(p, s);
      case 24: return launch_norm<DT, OT, 8, 1, BACK, true>(p, s);
      case 38: return launch_norm<DT, OT, 6, 2, BACK, true>(p, s);
      case 40: return launch_norm<DT, OT, 8, 2, BACK, true>(p, s);
      case 70: return launch_norm<DT, OT, 6, 4, BACK, true>(p, s);
      case 72: return launch_norm<DT, OT, 8, 4, BACK, true>(p, s);
      case 134: return launch_norm<DT, OT, 6, 8, BACK, true>(p, s);
      case 136: return launch_norm<DT, OT, 8, 8, BACK, true>(p, s);
      default: return launch_norm<DT, OT, 8, 16, BACK, true>(p, s);
    }
  }
  switch (c.w * 16 + c.nq) {
    case 17: return launch_norm<DT, OT, 1, 1, BACK, false>(p, s);
    case 20: return launch_norm<DT, OT, 4, 1, BACK, false>(p, s);
    case 24: return launch_norm<DT, OT, 8, 1, BACK, false>(p, s);
    case 38: return launch_norm<DT, OT, 6, 2, BACK, false>(p, s);
    case 40: return launch_norm<DT, OT, 8, 2, BACK, false>(p, s);
    case 70: return launch_norm<DT, OT, 6, 4, BACK, false>(p, s);
    case 72: return launch_norm<DT, OT, 8, 4, BACK, false>(p, s);
    case 134: return launch_norm<DT, OT, 6, 8, BACK, false>(p, s);
    case 136: return launch_norm<DT, OT, 8, 8, BACK, false>(p, s);
    default: return launch_norm<DT, OT, 8, 16, BACK, false>(p, s);
  }
}
template <int DT, bool BACK>
cudaError_t launch_dt(const NormParams& p, bool aligned_rows, cudaStream_t s) {
  switch (BACK ? p.dy_dtype : p.y_dtype) {
    case MFET_F32: return launch_types<DT, MFET_F32, BACK>(p, aligned_rows, s);
    case MFET_F16: return launch_types<DT, MFET_F16, BACK>(p, aligned_rows, s);
    default: return launch_types<DT, MFET_BF16, BACK>(p, aligned_rows, s);
  }
}
bool all_aligned(const NormParams& p) { return p.x_vec && p.y_vec && (!p.dy || p.dy_vec); }
template <bool BACK>
cudaError_t launch(NormParams& p, uint32_t x_dtype, cudaStream_t s) {
  p.w_vec = aligned(p.w, 16);
  p.b_vec = aligned(p.b, 16);
  if (p.cols > kMostHeld) {
    const int64_t most = (int64_t)sm_count() * 4;
    const int64_t blocks = BACK ? back_blocks(p.rows, columns_of(p.cols, false)) : p.rows < most ? p.rows : most;
    return launch_early(norm_long_kernel<BACK>, (unsigned)blocks, kLongThreads, 0, s, p, x_dtype);
  }
  const bool a = all_aligned(p);
  switch (x_dtype) {
    case MFET_F32: return launch_dt<MFET_F32, BACK>(p, a, s);
    case MFET_F16: return launch_dt<MFET_F16, BACK>(p, a, s);
    default: return launch_dt<MFET_BF16, BACK>(p, a, s);
  }
}

}  // namespace
}  // namespace mfet

extern "C" {

int mfet_layer_norm(const void* x, uint32_t x_dtype, int64_t x_ld, int64_t rows, int64_t cols, const float* weight, const float* bias,
                    float eps, void* y, uint32_t y_dtype, int64_t y_ld, mfet_stream_t stream) {
  if (bad_matrix(rows, cols, x_ld, x_dtype) || bad_matrix(rows, cols, y_ld, y_dtype) || !(eps >= 0.f)) return MFET_ERR_INVALID_ARG;
  if (rows == 0) return MFET_OK;
  if (!x || !y) return MFET_ERR_INVALID_ARG;
  if (!aligned(x, size_of(x_dtype)) || !aligned(y, size_of(y_dtype)) || !aligned(weight, 4) || !aligned(bias, 4)) return MFET_ERR_ALIGNMENT;
  NormParams p{};
  p.x = x;
  p.y = y;
  p.w = weight;
  p.b = bias;
  p.rows = rows;
  p.cols = cols;
  p.x_ld = x_ld;
  p.y_ld = y_ld;
  p.x_end = end_of(x, rows, cols, x_ld, x_dtype);
  p.eps = eps;
  p.y_dtype = y_dtype;
  p.x_vec = on_16(x, x_ld, x_dtype);
  p.y_vec = on_16(y, y_ld, y_dtype);
  return launch<false>(p, x_dtype, (cudaStream_t)stream) == cudaSuccess ? MFET_OK : MFET_ERR_CUDA;
}

uint64_t mfet_layer_norm_backward_bytes(int64_t rows, int64_t cols) {
  if (bad_matrix(rows, cols, cols, MFET_F32)) return 0;
  uint64_t most = 0;  // over the alignments that a call may have
  for (int a = 0; a < 2; ++a) {
    const Columns c = columns_of(cols, a);
    const uint64_t b = (uint64_t)back_blocks(rows, c) * words_of(cols, c) * 4;
    most = b > most ? b : most;
  }
  return most;
}

int mfet_layer_norm_backward(const void* x, uint32_t x_dtype, int64_t x_ld, int64_t rows, int64_t cols, const float* weight, float eps,
                             const void* dy, uint32_t dy_dtype, int64_t dy_ld, void* dx, int64_t dx_ld, float* dweight, float* dbias,
                             void* scratch, uint64_t scratch_bytes, mfet_stream_t stream) {
  if (bad_matrix(rows, cols, x_ld, x_dtype) || bad_matrix(rows, cols, dy_ld, dy_dtype) || dx_ld < cols || dx_ld >= (1ll << 31) || !(eps >= 0.f))
    return MFET_ERR_INVALID_ARG;
  if (rows > 0 && (!x || !dy || !dx)) return MFET_ERR_INVALID_ARG;
  if (!aligned(x, size_of(x_dtype)) || !aligned(dy, size_of(dy_dtype)) || !aligned(dx, size_of(x_dtype)) || !aligned(weight, 4) ||
      !aligned(dweight, 4) || !aligned(dbias, 4) || !aligned(scratch, 4))
    return MFET_ERR_ALIGNMENT;
  const bool sums = dweight || dbias;
  if (rows == 0) {  // sums over no rows
    if (dweight && cudaMemsetAsync(dweight, 0, cols * 4, (cudaStream_t)stream) != cudaSuccess) return MFET_ERR_CUDA;
    if (dbias && cudaMemsetAsync(dbias, 0, cols * 4, (cudaStream_t)stream) != cudaSuccess) return MFET_ERR_CUDA;
    return MFET_OK;
  }
  if (sums && (!scratch || scratch_bytes < mfet_layer_norm_backward_bytes(rows, cols))) return MFET_ERR_WORKSPACE;
  NormParams p{};
  p.x = x;
  p.dy = dy;
  p.y = dx;
  p.w = weight;
  p.partial = sums ? (float*)scratch : nullptr;
  p.rows = rows;
  p.cols = cols;
  p.x_ld = x_ld;
  p.y_ld = dx_ld;
  p.dy_ld = dy_ld;
  p.x_end = end_of(x, rows, cols, x_ld, x_dtype);
  p.dy_end = end_of(dy, rows, cols, dy_ld, dy_dtype);
  p.eps = eps;
  p.dy_dtype = dy_dtype;
  p.x_vec = on_16(x, x_ld, x_dtype);
  p.y_vec = on_16(dx, dx_ld, x_dtype);
  p.dy_vec = on_16(dy, dy_ld, dy_dtype);
  if (launch<true>(p, x_dtype, (cudaStream_t)stream) != cudaSuccess) return MFET_ERR_CUDA;
  if (!sums) return MFET_OK;
  const Columns c = columns_of(cols, all_aligned(p));
  const int64_t words = words_of(cols, c);
  const SumParams q{(const float*)scratch, dweight, dbias, cols, (uint32_t)back_blocks(rows, c), (int)words, 32 * c.w, c.nq};
  return launch_early(norm_sum_kernel, (unsigned)((words + kSumWords - 1) / kSumWords), 32 * kSumWords, 0, (cudaStream_t)stream, q) == cudaSuccess
             ? MFET_OK
             : MFET_ERR_CUDA;
}

}  // extern "C"
