// Layer norm over the columns of a row, and its backward pass.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) r, y = xh w + b
//   t = dy w:  dx = r (t - mean(t) - xh mean(t xh)),  dw = sum over rows of dy xh,  db = sum over rows of dy
//
// Both are bound by memory: x is read once and kept in registers, the variance is taken of the differences from the mean (no
// cancellation for rows far from 0), and the backward pass computes mu and r from x again instead of reading them. Everything is fp32 inside.
#include <type_traits>

#include "tensor.cuh"

using namespace mfet;

namespace mfet {
namespace {

constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kChunk = 8;            // neighbouring columns of a thread
constexpr int64_t kMostHeld = 16384; // columns of the longest row that is held in registers
constexpr int64_t kMostFast = 8192;   // ... by the kernel for rows on 16-byte boundaries, whose rows and weights are in shared memory
constexpr int kLongThreads = 512;

struct NormParams {
  const void *x, *dy;  // dy: backward
  void* y;             // forward: y; backward: dx, of x's type
  const float *w, *b;
  float* partial;      // backward: [blocks][2][cols] sums of dy xh, of dy; NULL: no sums wanted
  int64_t rows, cols, x_ld, y_ld, dy_ld;
  const void *x_end, *dy_end;
  float eps;
  uint32_t dy_dtype, y_dtype;
  bool x_vec, y_vec, dy_vec, w_vec, b_vec;  // rows start on 16-byte boundaries
  int tpr, groups;  // threads of a row; rows of a block at a time
  int stage_bytes;  // shared memory of a group for rows of results
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

// A row of results at an address that is not on 16 bytes: value by value to shared memory, under the same address modulo 16, and from there in
// whole units; the units at its ends value by value. (8 values a thread straight to memory: eight times the transactions.)
template <int DT>
__device__ __forceinline__ void values_to(uint8_t* row, int64_t c, const float* v, int count) {
  typename Elem<DT>::T* to = reinterpret_cast<typename Elem<DT>::T*>(row) + c;
#pragma unroll
  for (int j = 0; j < kChunk; ++j)
    if (j < count) to[j] = Elem<DT>::from(v[j]);
}
__device__ __forceinline__ void values_any(uint32_t dtype, uint8_t* row, int64_t c, const float* v, int count) {
  if (dtype == MFET_F32) values_to<MFET_F32>(row, c, v, count);
  else if (dtype == MFET_F16) values_to<MFET_F16>(row, c, v, count);
  else values_to<MFET_BF16>(row, c, v, count);
}
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

// s / n, rounded like a quotient (one correction): the mean of equal values is that value
__device__ __forceinline__ float over(float s, float n, float inv_n) {
  const float q = s * inv_n;
  return fmaf(fmaf(-q, n, s), inv_n, q);
}

// The block's sums for dw and db into its part of `partial`, as its threads hold them: word (which * chunks + i) * PER + j of thread `lane` of a row is
// at that word times tpr plus lane (the kernel that adds up the blocks puts columns in order). Several groups leave theirs in shared memory
// (`sums`: 2 PER NCH words a thread) first, and each word is added up over them in their order.
template <int NCH, int PER, int GROUPS, int TPR, typename W, typename B>  // groups of a block and threads of a group, 0: known at run time
__device__ __forceinline__ void block_sums(const NormParams& p, float* sums, int group, int lane, W dw, B db) {
  if (!p.partial) return;
  constexpr int kWords = 2 * NCH * PER;
  const int groups = GROUPS ? GROUPS : p.groups, tpr = TPR ? TPR : p.tpr;
  float* const to = p.partial + (int64_t)blockIdx.x * kWords * tpr + lane;
  if (groups > 1) {
    const int pitch = groups * tpr;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        sums[(i * PER + j) * pitch + threadIdx.x] = dw(i, j);
        sums[((NCH + i) * PER + j) * pitch + threadIdx.x] = db(i, j);
      }
    }
    __syncthreads();
    for (int e = group; e < kWords; e += groups) {
      const float* from = sums + e * pitch + lane;
      float v = from[0];
      for (int g = 1; g < groups; ++g) v += from[g * tpr];
      if (MFET_INSIDE(nullptr, lane < tpr)) to[e * tpr] = v;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if (!MFET_INSIDE(nullptr, lane < tpr)) continue;
      to[(i * PER + j) * tpr] = dw(i, j);
      to[((NCH + i) * PER + j) * tpr] = db(i, j);
    }
  }
}

// Rows that are held in registers, 8 * NCH columns a thread. As many threads as a row needs, counted up to a warp (p.tpr), are a group with its
// barrier; a block is p.groups of them, each with a row of its own at a time, so that enough rows are under way. Two rounds of sums a row:
// the mean, then of the differences d = x - mu their squares and, backward, t and t d together (mean(t xh) is r mean(t d)). The
// backward pass keeps its sums for dw and db in registers from row to row and joins them per block. 8192 x 896 fp32 x, bf16 dy: 56 us with a warp
// per row (28 columns a lane, 199 registers), 27.5 with 8 columns a thread (560 instructions per row and warp, most of them not per column).
template <int DT, int NCH, bool BACK, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS > 256 ? 1 : BACK ? 2 : 3) norm_kernel(const __grid_constant__ NormParams p) {
  constexpr int kValues = BACK ? 3 : 1;
  __shared__ float words[2][32 * kValues];  // of a round and the one after it: a word of each warp for each sum
  extern __shared__ __align__(16) uint8_t staged[];  // rows of results that do not start on 16 bytes; at the end: the groups' sums
  early_launch_wait();
  const int tpr = p.tpr, group = threadIdx.x / tpr, lane = threadIdx.x - group * tpr;
  const int warps = tpr >> 5, warp0 = group * warps;
  int turn = 0;
  auto meet = [&]() {
    if (warps == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(tpr) : "memory");
  };
  // sums of v[0 .. count) over the group, the same in all its threads
  auto total = [&](float* v, auto count) {
    constexpr int n = decltype(count)::value;
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = warp_sum(v[i]);
    if (warps == 1) return;
    float* at = words[turn] + warp0 * kValues;
    turn ^= 1;
    if ((lane & 31) == 0) {
#pragma unroll
      for (int i = 0; i < n; ++i) at[(lane >> 5) * kValues + i] = v[i];
    }
    meet();
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = at[i];
    for (int q = 1; q < warps; ++q) {
#pragma unroll
      for (int i = 0; i < n; ++i) v[i] += at[q * kValues + i];
    }
  };
  const float n = (float)p.cols, inv_n = 1.f / n;
  const uint32_t out_size = (BACK ? DT : p.y_dtype) == MFET_F32 ? 4 : 2;
  uint8_t* const stage = staged + group * p.stage_bytes;
  int count[NCH];
  float w[NCH][kChunk], b[BACK ? 1 : NCH][kChunk], dw[BACK ? NCH : 1][kChunk], db[BACK ? NCH : 1][kChunk];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int64_t c = (int64_t)(i * tpr + lane) * kChunk;
    count[i] = c < p.cols ? (int)min((int64_t)kChunk, p.cols - c) : 0;
    params8(p.w, c, p.cols, p.w_vec, 1.f, w[i]);
    if constexpr (!BACK) params8(p.b, c, p.cols, p.b_vec, 0.f, b[i]);
    if constexpr (BACK) {
#pragma unroll
      for (int j = 0; j < kChunk; ++j) dw[i][j] = db[i][j] = 0.f;
    }
  }
  for (int64_t row = (int64_t)blockIdx.x * p.groups + group; row < p.rows; row += (int64_t)gridDim.x * p.groups) {
    Raw<DT, kChunk> raw[NCH];
    float v[NCH][kChunk], t[BACK ? NCH : 1][kChunk];
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int64_t c = (int64_t)(i * tpr + lane) * kChunk;
      if (count[i] > 0 && MFET_INSIDE(nullptr, row < p.rows && c + count[i] <= p.x_ld)) raw[i] = chunk_in<DT>(p.x, row * p.x_ld + c, count[i], p.x_vec, p.x_end);
      else memset(&raw[i], 0, sizeof(raw[i]));
      if constexpr (BACK) {
        if (count[i] > 0 && MFET_INSIDE(nullptr, row < p.rows && c + count[i] <= p.dy_ld)) {
          chunk_any(p.dy_dtype, p.dy, row * p.dy_ld + c, count[i], p.dy_vec, p.dy_end, t[i]);
        } else {
#pragma unroll
          for (int j = 0; j < kChunk; ++j) t[i][j] = 0.f;
        }
      }
    }
    uint8_t* const y_row = reinterpret_cast<uint8_t*>(p.y) + row * p.y_ld * out_size;
    const uint32_t head = (uint32_t)reinterpret_cast<uintptr_t>(y_row) & 15u;
    float s[kValues];
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      widen_raw<DT, kChunk>(raw[i], v[i]);
#pragma unroll
      for (int j = 0; j < kChunk; ++j) s[0] += v[i][j];
    }
    total(s, std::integral_constant<int, 1>());
    const float mu = over(s[0], n, inv_n);
#pragma unroll
    for (int k = 0; k < kValues; ++k) s[k] = 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
#pragma unroll
      for (int j = 0; j < kChunk; ++j) {
        v[i][j] = j < count[i] ? v[i][j] - mu : 0.f;
        s[0] = fmaf(v[i][j], v[i][j], s[0]);
        if constexpr (BACK) {
          const float tw = t[i][j] * w[i][j];
          s[1] += tw;
          s[2] = fmaf(tw, v[i][j], s[2]);
        }
      }
    }
    total(s, std::integral_constant<int, kValues>());
    const float r = rsqrtf(fmaf(s[0], inv_n, p.eps));
    if constexpr (BACK) {
      const float m0 = s[1] * inv_n, m1 = s[2] * inv_n * r;
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
          const float xh = v[i][j] * r;
          db[i][j] += t[i][j];
          dw[i][j] = fmaf(t[i][j], xh, dw[i][j]);
          v[i][j] = r * (fmaf(t[i][j], w[i][j], -m0) - xh * m1);
        }
        const int64_t c = (int64_t)(i * tpr + lane) * kChunk;
        if (!p.y_vec) values_to<DT>(stage + head, c, v[i], count[i]);
        else if (count[i] > 0 && MFET_INSIDE(nullptr, row < p.rows && c + count[i] <= p.y_ld)) chunk_out<DT>(p.y, row * p.y_ld + c, v[i], count[i], true);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
#pragma unroll
        for (int j = 0; j < kChunk; ++j) v[i][j] = fmaf(v[i][j] * r, w[i][j], b[i][j]);
        const int64_t c = (int64_t)(i * tpr + lane) * kChunk;
        if (!p.y_vec) values_any(p.y_dtype, stage + head, c, v[i], count[i]);
        else if (count[i] > 0 && MFET_INSIDE(nullptr, row < p.rows && c + count[i] <= p.y_ld)) chunk_put(p.y_dtype, p.y, row * p.y_ld + c, v[i], count[i], true);
      }
    }
    if (!p.y_vec) {  // what the stage held before has left: two rounds of sums lie between
      meet();
      if (MFET_INSIDE(nullptr, row < p.rows && p.cols <= p.y_ld)) row_out(y_row, stage, head, (uint32_t)p.cols * out_size, out_size, lane, tpr);
      if (warps == 1) __syncwarp();
    }
  }
  if constexpr (BACK) {
    __syncthreads();
    block_sums<NCH, kChunk, 0, 0>(p, reinterpret_cast<float*>(staged), group, lane, [&](int i, int j) { return dw[i][j]; }, [&](int i, int j) { return db[i][j]; });
  }
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
__device__ __forceinline__ uint4 load16_shared(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}

// Threads of a block of the kernel below, and blocks that an SM has to hold. Backward one block, as large as its registers let it be (some 160 with
// 32 columns a thread; at 128 it spilt: 37 us instead of 27 for 8192 x 896), since each leaves sums of all columns.
template <int NQ, int W, bool BACK>
constexpr int fast_threads = !BACK || W == 8 ? 256 : NQ > 4 ? 384 : 512;
template <bool BACK>
constexpr int fast_blocks = BACK ? 1 : 3;

// 4 values of a type in shared memory
template <int DT>
__device__ __forceinline__ void quad_in(uint32_t at, float2* v) {
  if constexpr (DT == MFET_F32) {
    const uint4 a = load16_shared(at);
    v[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y));
    v[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
  } else {
    uint32_t a, b;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(a), "=r"(b) : "r"(at) : "memory");
    v[0] = Elem<DT>::widen(a);
    v[1] = Elem<DT>::widen(b);
  }
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

// The same where all rows start on 16-byte boundaries. A warp takes up to 1024 columns (most instructions of a row do not depend on its columns:
// sums over lanes, barriers, addresses), a lane 4 neighbouring ones of every 128, so that every access of a warp is whole lines of memory
// and of shared memory (8 neighbouring ones: fp32 rows were fetched by halves of sectors, twice). The next row is under way to shared
// memory in pieces of 16 bytes; arithmetic goes two columns an instruction, and all distances are known to the compiler (with
// the threads of a row and of a block known at run time, 500 of a row's 1140 instructions formed addresses). Columns
// behind the row's end are zeros with weight 0 and mean 0, so that nothing asks for them but the stores.
template <int DT, int OT, int NQ, int W, bool BACK>
__global__ void __launch_bounds__((fast_threads<NQ, W, BACK>), fast_blocks<BACK>) norm_fast_kernel(const __grid_constant__ NormParams p) {
  constexpr int kThreads = fast_threads<NQ, W, BACK>, tpr = 32 * W, kGroups = kThreads / tpr;
  constexpr int kXs = (int)sizeof(typename Elem<DT>::T), kOs = (int)sizeof(typename Elem<OT>::T);
  constexpr uint32_t kXb = NQ * tpr * 4 * kXs, kStage = kXb + (BACK ? NQ * tpr * 4 * kOs : 0);  // of a group: x (and dy) of a row
  constexpr int kXn = (NQ * kXs + 3) / 4, kOn = (NQ * kOs + 3) / 4;                            // pieces of 16 bytes that a thread fetches
  constexpr int kSure = W > 1 || NQ == 7 ? 4 : NQ == 8 ? 7 : NQ / 2;                           // quads that are full for all threads
  __shared__ float words[2][16][4];
  extern __shared__ __align__(16) uint8_t ring[];  // two rows of each group, weight and bias; at the end: the groups' sums
  early_launch_wait();
  const int group = threadIdx.x / tpr, lane = threadIdx.x % tpr, warp0 = group * W;
  const uint32_t mine = smem_addr(ring) + group * 2 * kStage;
  const uint32_t w_at = smem_addr(ring) + kGroups * 2 * kStage + lane * 16, b_at = w_at + NQ * tpr * 16;
  const bool ragged = p.cols % 4 != 0;
  int count[NQ];  // columns of a quad
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const int64_t c = (int64_t)(i * tpr + lane) * 4;
    count[i] = i < kSure ? 4 : c < p.cols ? (int)min((int64_t)4, p.cols - c) : 0;
  }
  const int64_t row0 = (int64_t)blockIdx.x * kGroups + group, step = (int64_t)gridDim.x * kGroups;
  const uint8_t* x_at = reinterpret_cast<const uint8_t*>(p.x) + row0 * p.x_ld * kXs + lane * 16;  // of the next row to be asked for
  const uint8_t* dy_at = reinterpret_cast<const uint8_t*>(p.dy) + row0 * p.dy_ld * kOs + lane * 16;
  uint8_t* y_at = reinterpret_cast<uint8_t*>(p.y) + (row0 * p.y_ld + lane * 4) * (BACK ? kXs : kOs);  // of the row that is computed
  const int64_t x_step = step * p.x_ld * kXs, dy_step = step * p.dy_ld * kOs, y_step = step * p.y_ld * (BACK ? kXs : kOs);
  int64_t left = row0 < p.rows ? (p.rows - row0 + step - 1) / step : 0, ask = left;  // rows of this group: to compute, to ask for
  const int x_bytes = (int)p.cols * kXs - lane * 16, dy_bytes = (int)p.cols * kOs - lane * 16;  // of a row from this thread's first piece on
  auto meet = [&]() {
    if constexpr (W == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(tpr) : "memory");
  };
  // zeros behind the rows' ends: nothing else is written there
  for (int at = lane * 16; at < (int)(2 * kStage); at += tpr * 16) store16_shared(mine + at, make_uint4(0, 0, 0, 0));
  meet();
  auto fetch = [&](uint32_t to, const uint8_t* from, int bytes, auto pieces) {
#pragma unroll
    for (int k = 0; k < decltype(pieces)::value; ++k) {
      const int n = bytes - k * tpr * 16;
      if (n >= 16) copy16(to + k * tpr * 16, from + k * tpr * 16);
      else if (n > 0) copy_part(to + k * tpr * 16, from + k * tpr * 16, n);
    }
  };
  auto request = [&](uint32_t to) {
    if (ask > 0 && MFET_INSIDE(nullptr, p.cols <= p.x_ld && p.cols <= NQ * tpr * 4)) {
      fetch(to + lane * 16, x_at, x_bytes, std::integral_constant<int, kXn>());
      if constexpr (BACK) fetch(to + kXb + lane * 16, dy_at, dy_bytes, std::integral_constant<int, kOn>());
      --ask;
      x_at += x_step;
      if constexpr (BACK) dy_at += dy_step;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  request(mine);
  // weight and bias as a group's threads read them; every group writes the same values
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const int64_t c = (int64_t)(i * tpr + lane) * 4;
    float a[4], b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      a[j] = j < count[i] ? (p.w ? __ldg(p.w + c + j) : 1.f) : 0.f;
      b[j] = j < count[i] && p.b ? __ldg(p.b + c + j) : 0.f;
    }
    store16_shared(w_at + i * tpr * 16, narrow16<MFET_F32>(a));
    if constexpr (!BACK) store16_shared(b_at + i * tpr * 16, narrow16<MFET_F32>(b));
  }
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
  const float n = (float)p.cols, inv_n = 1.f / n;
  uint32_t from = mine, to = mine + kStage;
  __syncthreads();  // the weights
  for (; left > 0; --left) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    meet();  // this row has arrived for all, and the last one is done with
    request(to);
    float2 v[NQ][2], s = both(0.f);
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      quad_in<DT>(from + (i * tpr + lane) * 4 * kXs, v[i]);
      s = add2(s, add2(v[i][0], v[i][1]));
    }
    const float mu = over(joined(warp_sum(s.x + s.y), std::false_type()).x, n, inv_n);
    float2 s0 = both(0.f), s1 = both(0.f), s2 = both(0.f), t[2], w[2];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const float2 minus = both(i < kSure || count[i] > 0 ? -mu : 0.f);
      v[i][0] = add2(v[i][0], minus);
      v[i][1] = add2(v[i][1], minus);
      if (i >= kSure && ragged && count[i] > 0) {  // the row may end inside this quad
        if (count[i] < 2) v[i][0].y = 0.f;
        if (count[i] < 3) v[i][1].x = 0.f;
        if (count[i] < 4) v[i][1].y = 0.f;
      }
      if constexpr (BACK) {
        quad_in<OT>(from + kXb + (i * tpr + lane) * 4 * kOs, t);
        quad_in<MFET_F32>(w_at + i * tpr * 16, w);
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
    const float2 rr = both(r), rm0 = both(-r * (q.y * inv_n)), rm1 = both(-r * (q.z * inv_n * r));
    constexpr int kType = BACK ? DT : OT;
    typename Elem<kType>::T* const out = reinterpret_cast<typename Elem<kType>::T*>(y_at);
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      float2 b[2], o[2];
      quad_in<MFET_F32>(w_at + i * tpr * 16, w);
      if constexpr (BACK) quad_in<OT>(from + kXb + (i * tpr + lane) * 4 * kOs, t);
      else quad_in<MFET_F32>(b_at + i * tpr * 16, b);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float2 xh = mul2(v[i][j], rr);
        if constexpr (BACK) {
          db[i][j] = add2(db[i][j], t[j]);
          dw[i][j] = fma2(t[j], xh, dw[i][j]);
          o[j] = fma2(xh, rm1, fma2(mul2(t[j], w[j]), rr, rm0));
        } else {
          o[j] = fma2(xh, w[j], b[j]);
        }
      }
      if (MFET_INSIDE(nullptr, (int64_t)(i * tpr + lane) * 4 + count[i] <= p.y_ld || count[i] == 0)) quad_out<kType>(out + i * tpr * 4, o, i < kSure ? 4 : count[i]);
    }
    const uint32_t next = to;
    to = from;
    from = next;
    y_at += y_step;
  }
  if constexpr (BACK) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    block_sums<NQ, 4, kGroups, tpr>(p, reinterpret_cast<float*>(ring), group, lane, [&](int i, int j) { return j & 1 ? dw[i][j >> 1].y : dw[i][j >> 1].x; },
                                    [&](int i, int j) { return j & 1 ? db[i][j >> 1].y : db[i][j >> 1].x; });
  }
}

// Rows that registers do not hold: a block per row reads it once for each sum and once more for the result (from L2). BACK: the
// block's sums over its rows stay in its part of `partial`.
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
    const float mu = block_sum(s, shared, &turn) / n;
    s = 0.f;
    each([&](int64_t, int count, float* v) {
      for (int j = 0; j < count; ++j) s = fmaf(v[j] - mu, v[j] - mu, s);
    });
    const float r = 1.f / sqrtf(block_sum(s, shared, &turn) / n + p.eps);
    if constexpr (!BACK) {
      each([&](int64_t c, int count, float* v) {
        float w[kChunk], b[kChunk];
        params8(p.w, c, p.cols, p.w_vec, 1.f, w);
        params8(p.b, c, p.cols, p.b_vec, 0.f, b);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) v[j] = fmaf((v[j] - mu) * r, w[j], b[j]);
        if (MFET_INSIDE(nullptr, c + count <= p.y_ld)) chunk_put(p.y_dtype, p.y, row * p.y_ld + c, v, count, p.y_vec);
      });
    } else {
      float s0 = 0.f, s1 = 0.f;
      each([&](int64_t c, int count, float* v) {
        float w[kChunk], t[kChunk];
        grad(c, count, t);
        params8(p.w, c, p.cols, p.w_vec, 1.f, w);
        for (int j = 0; j < count; ++j) {
          const float xh = (v[j] - mu) * r;
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
        for (int j = 0; j < kChunk; ++j) v[j] = r * (t[j] * w[j] - m0 - (v[j] - mu) * r * m1);
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
  int words, tpr, chunks, per;  // words of a block; how they belong to columns (chunks = 0: dw's columns, then db's)
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
    if (p.chunks) {
      const int e = (int)(mine / p.tpr), lane = (int)(mine - (int64_t)e * p.tpr), i = e / p.per % p.chunks;
      bias = e / p.per >= p.chunks;
      c = (int64_t)(i * p.tpr + lane) * p.per + e % p.per;
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

// How a row is spread over threads, and rows over blocks
struct Split {
  bool fast, held;          // which kernel
  int chunks, per, tpr, groups;  // chunks a thread, columns of a chunk, threads of a row, rows of a block
  int64_t at_once;          // blocks of the backward pass that the GPU holds
};
Split split_of(int64_t cols, bool fast, bool back) {
  Split s{};
  s.held = cols <= kMostHeld;
  s.fast = fast && cols <= kMostFast;
  if (s.fast) {
    s.tpr = cols <= 1024 ? 32 : cols <= 2048 ? 64 : cols <= 4096 ? 128 : 256;
    s.per = 4;
    s.chunks = s.tpr > 32 || cols > 896 ? 8 : cols > 512 ? 7 : cols > 256 ? 4 : cols > 128 ? 2 : 1;
    s.groups = (!back || s.tpr == 256 ? 256 : s.chunks > 4 ? 384 : 512) / s.tpr;  // as fast_threads
    s.at_once = sm_count();
  } else {
    s.per = kChunk;
    s.chunks = cols > 256 ? 2 : 1;
    const int64_t threads = (cols + kChunk * s.chunks - 1) / (kChunk * s.chunks);
    s.tpr = s.held ? (int)((threads + 31) / 32 * 32) : kLongThreads;
    s.groups = s.tpr > 128 ? 1 : 256 / s.tpr;
    s.at_once = (int64_t)sm_count() * (s.tpr > 256 ? 1 : 2);
  }
  return s;
}
// sums that a block of the backward pass leaves
int64_t words_of(int64_t cols, const Split& s) { return s.held ? 2ll * s.chunks * s.per * s.tpr : 2 * cols; }
int64_t blocks_of(int64_t rows, const Split& s) {
  const int64_t want = (rows + s.groups - 1) / s.groups;
  return want < s.at_once ? want : s.at_once;
}

template <int DT, int OT, int NQ, int W, bool BACK>
cudaError_t launch_fast(const NormParams& p, unsigned blocks, cudaStream_t s) {
  constexpr int threads = fast_threads<NQ, W, BACK>;
  constexpr uint32_t row = NQ * 4 * (uint32_t)(sizeof(typename Elem<DT>::T) + (BACK ? sizeof(typename Elem<OT>::T) : 0));  // of a thread
  constexpr uint32_t ring = threads * 2 * row + 32 * W * NQ * 16 * (BACK ? 1 : 2), sums = BACK ? threads * 2 * NQ * 16 : 0;
  constexpr uint32_t smem = ring > sums ? ring : sums;
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem(norm_fast_kernel<DT, OT, NQ, W, BACK>, smem, &ready);
  return e != cudaSuccess ? e : launch_early(norm_fast_kernel<DT, OT, NQ, W, BACK>, blocks, threads, smem, s, p);
}
template <int DT, int OT, bool BACK>
cudaError_t launch_fast(const NormParams& p, const Split& q, unsigned blocks, cudaStream_t s) {
  switch (q.tpr + q.chunks) {
    case 33: return launch_fast<DT, OT, 1, 1, BACK>(p, blocks, s);
    case 34: return launch_fast<DT, OT, 2, 1, BACK>(p, blocks, s);
    case 36: return launch_fast<DT, OT, 4, 1, BACK>(p, blocks, s);
    case 39: return launch_fast<DT, OT, 7, 1, BACK>(p, blocks, s);
    case 40: return launch_fast<DT, OT, 8, 1, BACK>(p, blocks, s);
    case 72: return launch_fast<DT, OT, 8, 2, BACK>(p, blocks, s);
    case 136: return launch_fast<DT, OT, 8, 4, BACK>(p, blocks, s);
    default: return launch_fast<DT, OT, 8, 8, BACK>(p, blocks, s);
  }
}

template <int DT, bool BACK>
cudaError_t launch_held(const NormParams& p, const Split& q, cudaStream_t s) {
  const unsigned threads = (unsigned)(q.tpr * q.groups);
  int64_t blocks = blocks_of(p.rows, q);
  if (!BACK && q.tpr <= 256) {  // no sums to join: as many blocks as fit
    const int64_t want = (p.rows + q.groups - 1) / q.groups, most = (int64_t)sm_count() * (768 / threads);
    blocks = want < most ? want : most;
  }
  if (q.fast) {
    switch (BACK ? p.dy_dtype : p.y_dtype) {
      case MFET_F32: return launch_fast<DT, MFET_F32, BACK>(p, q, (unsigned)blocks, s);
      case MFET_F16: return launch_fast<DT, MFET_F16, BACK>(p, q, (unsigned)blocks, s);
      default: return launch_fast<DT, MFET_BF16, BACK>(p, q, (unsigned)blocks, s);
    }
  }
  size_t stage = p.y_vec ? 0 : (size_t)p.stage_bytes * q.groups;
  if (BACK && q.groups > 1 && stage < (size_t)threads * 2 * kChunk * q.chunks * 4) stage = (size_t)threads * 2 * kChunk * q.chunks * 4;
  auto go = [&](auto kernel) { return launch_early(kernel, (unsigned)blocks, threads, stage, s, p); };
  if (q.chunks == 1) return go(norm_kernel<DT, 1, BACK, 256>);
  if (threads <= 256) return go(norm_kernel<DT, 2, BACK, 256>);
  if (threads <= 512) return go(norm_kernel<DT, 2, BACK, 512>);  // 32 KB of shared memory at most
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem(norm_kernel<DT, 2, BACK, 1024>, 4 * (uint32_t)kMostHeld + 32, &ready);
  return e != cudaSuccess ? e : go(norm_kernel<DT, 2, BACK, 1024>);
}
template <int DT>
cudaError_t launch_dt(const NormParams& p, const Split& q, bool back, cudaStream_t s) {
  return back ? launch_held<DT, true>(p, q, s) : launch_held<DT, false>(p, q, s);
}
Split how(const NormParams& p, bool back) {
  return split_of(p.cols, p.x_vec && p.y_vec && (!back || p.dy_vec), back);
}
cudaError_t launch(NormParams& p, uint32_t x_dtype, bool back, cudaStream_t s) {
  const Split q = how(p, back);
  p.tpr = q.tpr;
  p.groups = q.groups;
  p.stage_bytes = (int)((p.cols * (back ? size_of(x_dtype) : size_of(p.y_dtype)) + 31) / 16 * 16);
  p.w_vec = aligned(p.w, 16);
  p.b_vec = aligned(p.b, 16);
  if (p.cols > kMostHeld)
    return launch_early(back ? norm_long_kernel<true> : norm_long_kernel<false>, (unsigned)blocks_of(p.rows, q), kLongThreads, 0, s, p, x_dtype);
  switch (x_dtype) {
    case MFET_F32: return launch_dt<MFET_F32>(p, q, back, s);
    case MFET_F16: return launch_dt<MFET_F16>(p, q, back, s);
    default: return launch_dt<MFET_BF16>(p, q, back, s);
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
  return launch(p, x_dtype, false, (cudaStream_t)stream) == cudaSuccess ? MFET_OK : MFET_ERR_CUDA;
}

uint64_t mfet_layer_norm_backward_bytes(int64_t rows, int64_t cols) {
  if (bad_matrix(rows, cols, cols, MFET_F32)) return 0;
  uint64_t most = 0;  // over the alignments that a call may have
  for (int fast = 0; fast < 2; ++fast) {
    const Split s = split_of(cols, fast, true);
    const uint64_t b = (uint64_t)blocks_of(rows, s) * words_of(cols, s) * 4;
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
  if (launch(p, x_dtype, true, (cudaStream_t)stream) != cudaSuccess) return MFET_ERR_CUDA;
  if (!sums) return MFET_OK;
  const Split done = how(p, true);
  const int64_t words = words_of(cols, done);
  const SumParams q{(const float*)scratch, dweight, dbias, cols, (uint32_t)blocks_of(rows, done), (int)words, done.tpr, done.held ? done.chunks : 0, done.per};
  return launch_early(norm_sum_kernel, (unsigned)((words + kSumWords - 1) / kSumWords), 32 * kSumWords, 0, (cudaStream_t)stream, q) == cudaSuccess
             ? MFET_OK
             : MFET_ERR_CUDA;
}

}  // extern "C"
