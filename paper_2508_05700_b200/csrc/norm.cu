// Layer norm over the columns of a row, and its backward pass.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) r, y = xh w + b
//   t = dy w:  dx = r (t - mean(t) - xh mean(t xh)),  dw = sum over rows of dy xh,  db = sum over rows of dy
//
// Both are bound by memory: x is read once and kept in registers, the variance is taken of the differences from the mean (no
// cancellation for rows far from 0), and the backward pass computes mu and r from x again instead of reading them. Everything is fp32 inside.
#include "lowbit.cuh"

using namespace mfet;

namespace mfet {
namespace {

constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kChunk = 8;            // neighbouring columns of a thread
constexpr int64_t kMostHeld = 16384; // columns of the longest row that is held in registers
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
  bool x_vec, y_vec, dy_vec;  // rows start on 16-byte boundaries
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

// The sum over the TPR threads of a row, the same in all of them. `turn` alternates: two sums in a row use different words.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float (*shared)[2][TPR / 32], int* turn) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kAll, v, d);
  if constexpr (TPR > 32) {
    float* words = (*shared)[*turn];
    *turn ^= 1;
    if ((threadIdx.x & 31) == 0) words[threadIdx.x >> 5] = v;
    __syncthreads();
    v = words[0];
#pragma unroll
    for (int i = 1; i < TPR / 32; ++i) v += words[i];
  }
  return v;
}

// Threads of a block: a warp per row in blocks of 8, or a block per row
template <int TPR>
constexpr int block_threads = TPR == 32 ? 256 : TPR;

template <int DT, int NCH, int TPR>
struct Row {
  Raw<DT, kChunk> raw[NCH];
  float mu, r;

  __device__ __forceinline__ void load(const NormParams& p, int64_t row, int lane) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int64_t c = (int64_t)(i * TPR + lane) * kChunk;
      const int count = c < p.cols ? (int)min((int64_t)kChunk, p.cols - c) : 0;
      if (count > 0 && MFET_INSIDE(nullptr, row < p.rows && c + count <= p.x_ld)) raw[i] = chunk_in<DT>(p.x, row * p.x_ld + c, count, p.x_vec, p.x_end);
      else memset(&raw[i], 0, sizeof(raw[i]));
    }
  }
  // xh of the row (0 behind its end)
  __device__ __forceinline__ void normalise(const NormParams& p, int lane, float (*v)[kChunk], float (*shared)[2][TPR / 32], int* turn) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      widen_raw<DT, kChunk>(raw[i], v[i]);
#pragma unroll
      for (int j = 0; j < kChunk; ++j) s += v[i][j];
    }
    const float n = (float)p.cols;
    mu = row_sum<TPR>(s, shared, turn) / n;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int left = (int)min((int64_t)kChunk, p.cols - (int64_t)(i * TPR + lane) * kChunk);
#pragma unroll
      for (int j = 0; j < kChunk; ++j) {
        v[i][j] = j < left ? v[i][j] - mu : 0.f;
        s = fmaf(v[i][j], v[i][j], s);
      }
    }
    r = 1.f / sqrtf(row_sum<TPR>(s, shared, turn) / n + p.eps);
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int j = 0; j < kChunk; ++j) v[i][j] *= r;
  }
};

__device__ __forceinline__ void params8(const float* w, int64_t c, int64_t cols, float none, float* v) {
#pragma unroll
  for (int j = 0; j < kChunk; ++j) v[j] = w && c + j < cols ? __ldg(w + c + j) : none;
}

template <int DT, int NCH, int TPR>
__global__ void __launch_bounds__(block_threads<TPR>) norm_kernel(const __grid_constant__ NormParams p) {
  __shared__ float shared[2][TPR / 32];
  early_launch_wait();
  constexpr int kRows = block_threads<TPR> / TPR;
  const int lane = threadIdx.x % TPR;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; row < p.rows; row += (int64_t)gridDim.x * kRows) {
    Row<DT, NCH, TPR> x;
    float v[NCH][kChunk];
    x.load(p, row, lane);
    x.normalise(p, lane, v, &shared, &turn);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int64_t c = (int64_t)(i * TPR + lane) * kChunk;
      if (c >= p.cols) break;
      float w[kChunk], b[kChunk];
      params8(p.w, c, p.cols, 1.f, w);
      params8(p.b, c, p.cols, 0.f, b);
#pragma unroll
      for (int j = 0; j < kChunk; ++j) v[i][j] = fmaf(v[i][j], w[j], b[j]);
      const int count = (int)min((int64_t)kChunk, p.cols - c);
      if (MFET_INSIDE(nullptr, row < p.rows && c + count <= p.y_ld)) chunk_put(p.y_dtype, p.y, row * p.y_ld + c, v[i], count, p.y_vec);
    }
  }
}

template <int DT, int NCH, int TPR>
__global__ void __launch_bounds__(block_threads<TPR>) norm_back_kernel(const __grid_constant__ NormParams p) {
  __shared__ float shared[2][TPR / 32];
  constexpr int kRows = block_threads<TPR> / TPR;
  __shared__ float sums[kRows > 1 ? 32 * kChunk * NCH : 1];
  early_launch_wait();
  const int lane = threadIdx.x % TPR, mine = threadIdx.x / TPR;
  int turn = 0;
  float dw[NCH][kChunk], db[NCH][kChunk];
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int j = 0; j < kChunk; ++j) dw[i][j] = db[i][j] = 0.f;
  for (int64_t row = (int64_t)blockIdx.x * kRows + mine; row < p.rows; row += (int64_t)gridDim.x * kRows) {
    Row<DT, NCH, TPR> x;
    float v[NCH][kChunk], t[NCH][kChunk];
    x.load(p, row, lane);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int64_t c = (int64_t)(i * TPR + lane) * kChunk;
      const int count = c < p.cols ? (int)min((int64_t)kChunk, p.cols - c) : 0;
      if (count > 0 && MFET_INSIDE(nullptr, row < p.rows && c + count <= p.dy_ld)) {
        chunk_any(p.dy_dtype, p.dy, row * p.dy_ld + c, count, p.dy_vec, p.dy_end, t[i]);
      } else {
#pragma unroll
        for (int j = 0; j < kChunk; ++j) t[i][j] = 0.f;
      }
    }
    x.normalise(p, lane, v, &shared, &turn);
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int64_t c = (int64_t)(i * TPR + lane) * kChunk;
      float w[kChunk];
      params8(p.w, c, p.cols, 1.f, w);
#pragma unroll
      for (int j = 0; j < kChunk; ++j) {
        db[i][j] += t[i][j];
        dw[i][j] = fmaf(t[i][j], v[i][j], dw[i][j]);
        t[i][j] *= w[j];
        s0 += t[i][j];
        s1 = fmaf(t[i][j], v[i][j], s1);
      }
    }
    const float n = (float)p.cols;
    const float m0 = row_sum<TPR>(s0, &shared, &turn) / n, m1 = row_sum<TPR>(s1, &shared, &turn) / n;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int64_t c = (int64_t)(i * TPR + lane) * kChunk;
      if (c >= p.cols) break;
#pragma unroll
      for (int j = 0; j < kChunk; ++j) t[i][j] = x.r * (t[i][j] - m0 - v[i][j] * m1);
      const int count = (int)min((int64_t)kChunk, p.cols - c);
      if (MFET_INSIDE(nullptr, row < p.rows && c + count <= p.y_ld)) chunk_out<DT>(p.y, row * p.y_ld + c, t[i], count, p.y_vec);
    }
  }
  if (!p.partial) return;
  // the block's sums: its warps' one after the other
  float* const to = p.partial + (int64_t)blockIdx.x * 2 * p.cols;
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {
    if constexpr (kRows > 1) {
#pragma unroll 1
      for (int q = 0; q < kRows; ++q) {
        if (mine == q) {
#pragma unroll
          for (int i = 0; i < NCH; ++i)
#pragma unroll
            for (int j = 0; j < kChunk; ++j) {
              float* s = &sums[(i * kChunk + j) * 32 + lane];
              const float v = which ? db[i][j] : dw[i][j];
              *s = q ? *s + v : v;
            }
        }
        __syncthreads();
      }
      for (int64_t c = threadIdx.x; c < p.cols; c += block_threads<TPR>) {
        const int chunk = (int)(c / kChunk);
        if (MFET_INSIDE(nullptr, chunk / 32 < NCH)) to[which * p.cols + c] = sums[(chunk / 32 * kChunk + c % kChunk) * 32 + chunk % 32];
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int i = 0; i < NCH; ++i)
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
          const int64_t c = (int64_t)(i * TPR + lane) * kChunk + j;
          if (c < p.cols && MFET_INSIDE(nullptr, lane < TPR)) to[which * p.cols + c] = which ? db[i][j] : dw[i][j];
        }
    }
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
    const float mu = row_sum<kLongThreads>(s, &shared, &turn) / n;
    s = 0.f;
    each([&](int64_t, int count, float* v) {
      for (int j = 0; j < count; ++j) s = fmaf(v[j] - mu, v[j] - mu, s);
    });
    const float r = 1.f / sqrtf(row_sum<kLongThreads>(s, &shared, &turn) / n + p.eps);
    if constexpr (!BACK) {
      each([&](int64_t c, int count, float* v) {
        float w[kChunk], b[kChunk];
        params8(p.w, c, p.cols, 1.f, w);
        params8(p.b, c, p.cols, 0.f, b);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) v[j] = fmaf((v[j] - mu) * r, w[j], b[j]);
        if (MFET_INSIDE(nullptr, c + count <= p.y_ld)) chunk_put(p.y_dtype, p.y, row * p.y_ld + c, v, count, p.y_vec);
      });
    } else {
      float s0 = 0.f, s1 = 0.f;
      each([&](int64_t c, int count, float* v) {
        float w[kChunk], t[kChunk];
        grad(c, count, t);
        params8(p.w, c, p.cols, 1.f, w);
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
      const float m0 = row_sum<kLongThreads>(s0, &shared, &turn) / n, m1 = row_sum<kLongThreads>(s1, &shared, &turn) / n;
      each([&](int64_t c, int count, float* v) {
        float w[kChunk], t[kChunk];
        grad(c, count, t);
        params8(p.w, c, p.cols, 1.f, w);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) v[j] = r * (t[j] * w[j] - m0 - (v[j] - mu) * r * m1);
        if (MFET_INSIDE(nullptr, c + count <= p.y_ld)) chunk_put(x_dtype, p.y, row * p.y_ld + c, v, count, p.y_vec);
      });
    }
  }
}

// The blocks' sums in their order: 8 threads per column take every eighth block each.
constexpr int kSumCols = 32;
struct SumParams {
  const float* partial;
  float *dw, *db;
  int64_t cols;
  uint32_t blocks;
};
__global__ void __launch_bounds__(256) norm_sum_kernel(const __grid_constant__ SumParams p) {
  __shared__ float part[8][kSumCols];
  early_launch_wait();
  const int col = threadIdx.x % kSumCols, seg = threadIdx.x / kSumCols;
  const int64_t at = (int64_t)blockIdx.x * kSumCols + col;
  float s = 0.f;
  if (at < 2 * p.cols)
    for (uint32_t b = seg; b < p.blocks; b += 8) s += p.partial[b * 2 * p.cols + at];
  part[seg][col] = s;
  __syncthreads();
  if (seg == 0 && at < 2 * p.cols) {
    for (int i = 1; i < 8; ++i) s += part[i][col];
    float* to = at < p.cols ? p.dw : p.db;
    const int64_t c = at < p.cols ? at : at - p.cols;
    if (to && MFET_INSIDE(nullptr, c >= 0 && c < p.cols)) to[c] = s;
  }
}

// ------------------------------------------------------------------ host side ----

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
uint32_t size_of(uint32_t dtype) { return dtype == MFET_F32 ? 4 : 2; }
bool on_16(const void* p, int64_t ld, uint32_t dtype) { return aligned(p, 16) && (uint64_t)ld * size_of(dtype) % 16 == 0; }
const void* end_of(const void* p, int64_t rows, int64_t cols, int64_t ld, uint32_t dtype) {
  return (const uint8_t*)p + ((rows - 1) * ld + cols) * size_of(dtype);
}
bool bad_matrix(int64_t rows, int64_t cols, int64_t ld, uint32_t dtype) {
  return dtype > MFET_BF16 || rows < 0 || rows >= (1ll << 31) || cols < 1 || cols >= (1ll << 30) || ld < cols || ld >= (1ll << 31);
}

constexpr int kBackPerSm = 4;  // most blocks per SM of the backward pass: each has its own sums of all columns
// rows per block at a time
int64_t rows_at_once(int64_t cols) { return cols <= 1024 ? 8 : 1; }
int64_t back_blocks(int64_t rows, int64_t cols) {
  const int64_t want = (rows + rows_at_once(cols) - 1) / rows_at_once(cols), most = (int64_t)sm_count() * (cols <= 1024 ? 2 : kBackPerSm);
  return want < most ? want : most;
}

template <int DT, int NCH, int TPR>
cudaError_t launch_held(const NormParams& p, bool back, cudaStream_t s) {
  if (back) return launch_early(norm_back_kernel<DT, NCH, TPR>, (unsigned)back_blocks(p.rows, p.cols), block_threads<TPR>, 0, s, p);
  const int64_t per = block_threads<TPR> / TPR, want = (p.rows + per - 1) / per, most = (int64_t)sm_count() * (2048 / block_threads<TPR>);
  return launch_early(norm_kernel<DT, NCH, TPR>, (unsigned)(want < most ? want : most), block_threads<TPR>, 0, s, p);
}
template <int DT>
cudaError_t launch_dt(const NormParams& p, bool back, cudaStream_t s) {
  if (p.cols <= 256) return launch_held<DT, 1, 32>(p, back, s);
  if (p.cols <= 512) return launch_held<DT, 2, 32>(p, back, s);
  if (p.cols <= 1024) return launch_held<DT, 4, 32>(p, back, s);
  if (p.cols <= 2048) return launch_held<DT, 2, 128>(p, back, s);
  if (p.cols <= 4096) return launch_held<DT, 4, 128>(p, back, s);
  if (p.cols <= 8192) return launch_held<DT, 4, 256>(p, back, s);
  return launch_held<DT, 4, 512>(p, back, s);
}
cudaError_t launch(const NormParams& p, uint32_t x_dtype, bool back, cudaStream_t s) {
  if (p.cols > kMostHeld) {
    if (back) return launch_early(norm_long_kernel<true>, (unsigned)back_blocks(p.rows, p.cols), kLongThreads, 0, s, p, x_dtype);
    const int64_t most = (int64_t)sm_count() * 4;
    return launch_early(norm_long_kernel<false>, (unsigned)(p.rows < most ? p.rows : most), kLongThreads, 0, s, p, x_dtype);
  }
  switch (x_dtype) {
    case MFET_F32: return launch_dt<MFET_F32>(p, back, s);
    case MFET_F16: return launch_dt<MFET_F16>(p, back, s);
    default: return launch_dt<MFET_BF16>(p, back, s);
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
  return (uint64_t)back_blocks(rows, cols) * 2 * cols * 4;
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
  const SumParams q{(const float*)scratch, dweight, dbias, cols, (uint32_t)back_blocks(rows, cols)};
  return launch_early(norm_sum_kernel, (unsigned)((2 * cols + kSumCols - 1) / kSumCols), 256, 0, (cudaStream_t)stream, q) == cudaSuccess ? MFET_OK
                                                                                                                                    : MFET_ERR_CUDA;
}

}  // extern "C"
