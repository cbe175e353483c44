// A matrix orthogonalised by Newton-Schulz products: X = G / |G|, then per step, with A = X X^T over the shorter side,
//
//   X <- a X + (b A + c A A) X
//
// which takes every singular value s of X to a s + b s^3 + c s^5 and leaves the singular vectors. A step multiplies small singular
// values, and the errors in their directions, by a (3.4 in the usual schedule, some 480 in five steps): with operands of one 16-bit
// word the result is off by 1e-3 (fp16) to 1e-2 (bf16) of its size. So X, A and B = b A + c A A are held as the sum of two fp16 words
// (22 bits and more, under a power of two for each matrix that keeps its bound, known to the host, inside fp16's range), a product is three
// (high x high, high x low, low x high) in one fp32 accumulator, and the result is as near as one computed in fp32.
#include <cmath>

#include "gemm16.cuh"

using namespace mfet;
using namespace mfet::gemm16;

namespace mfet {
namespace {

constexpr int kSumThreads = 256;
constexpr int kMostParts = 512;  // blocks of the sum of squares
constexpr int kMostSteps = 64;

struct LoadParams {
  const uint8_t* g;
  int64_t rows, cols, ld;
  const void* end;
  bool vec;
  double* parts;       // sums of squares of the blocks
  uint32_t n_parts;
  __half *hi, *lo;     // [rows][up8(cols)]
  int64_t x_ld;
  double scale;        // 2^e of the words
};

template <int DT>
__device__ __forceinline__ void eight(const LoadParams& p, int64_t row, int64_t c, float* v) {
  using T = typename Elem<DT>::T;
  const int count = (int)min((int64_t)8, p.cols - c);
  const T* at = reinterpret_cast<const T*>(p.g) + row * p.ld + c;
  if (!MFET_INSIDE(nullptr, row < p.rows && count > 0 && c + count <= p.ld)) return;
  if (p.vec) widen_raw<DT, 8>(load_raw<DT, 8, true>(at, count), v);
  else widen_raw<DT, 8>(load_shifted<DT, 8>(at, count, p.g, p.end), v);
}

__device__ __forceinline__ double block_sum(double s, double* words) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(kAllLanes, s, d);
  if ((threadIdx.x & 31) == 0) words[threadIdx.x >> 5] = s;
  __syncthreads();
  s = 0.0;
  for (int i = 0; i < kSumThreads / 32; ++i) s += words[i];
  return s;
}

// squares in fp64: no overflow, whatever the scale of the gradients
template <int DT>
__global__ void __launch_bounds__(kSumThreads) squares_kernel(const __grid_constant__ LoadParams p) {
  __shared__ double words[kSumThreads / 32];
  early_launch_wait();
  const int64_t per_row = p.x_ld / 8, units = p.rows * per_row;
  double s = 0.0;
  for (int64_t u = (int64_t)blockIdx.x * kSumThreads + threadIdx.x; u < units; u += (int64_t)gridDim.x * kSumThreads) {
    const int64_t row = u / per_row;
    float v[8] = {};
    eight<DT>(p, row, (u - row * per_row) * 8, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fma((double)v[j], (double)v[j], s);
  }
  s = block_sum(s, words);
  if (threadIdx.x == 0 && MFET_INSIDE(nullptr, blockIdx.x < p.n_parts)) p.parts[blockIdx.x] = s;
}

// X = G / |G| in two words; 0 for G = 0, NaN throughout if G has a value that is not finite
template <int DT>
__global__ void __launch_bounds__(kSumThreads) scale_kernel(const __grid_constant__ LoadParams p) {
  __shared__ double words[kSumThreads / 32];
  early_launch_wait();
  double total = 0.0;
  for (uint32_t i = threadIdx.x; i < p.n_parts; i += kSumThreads) total += p.parts[i];
  total = block_sum(total, words);
  const double f = total > 0.0 ? (isinf(total) ? NAN : p.scale / sqrt(total)) : (total == 0.0 ? 0.0 : total);
  const int64_t per_row = p.x_ld / 8, units = p.rows * per_row;
  for (int64_t u = (int64_t)blockIdx.x * kSumThreads + threadIdx.x; u < units; u += (int64_t)gridDim.x * kSumThreads) {
    const int64_t row = u / per_row, c = (u - row * per_row) * 8;
    float v[8] = {}, lo[8];
    eight<DT>(p, row, c, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = (float)(v[j] * f);
      lo[j] = v[j] - __half2float(__float2half_rn(v[j]));
    }
    if (!MFET_INSIDE(nullptr, row < p.rows && c + 8 <= p.x_ld)) continue;
    *reinterpret_cast<uint4*>(p.hi + row * p.x_ld + c) = narrow16<MFET_F16>(v);
    *reinterpret_cast<uint4*>(p.lo + row * p.x_ld + c) = narrow16<MFET_F16>(lo);
  }
}

// ------------------------------------------------------------------ host side ----

struct Words {  // a matrix in two words: value = (hi + lo) * 2^-e
  Matrix hi, lo;
  int e = 0;
};

bool bad_sizes(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0 || rows >= (1ll << 31) || cols >= (1ll << 31)) return true;
  return (rows / 128 + 1) * (cols / 128 + 1) >= (1ll << 31);
}

uint64_t words_bytes(int64_t rows, int64_t cols) { return packed_bytes(rows, cols) * 2; }

Words words_at(uint8_t** to, int64_t rows, int64_t cols) {
  Words w;
  w.hi = {*to, cols, rows, up8(cols), true};
  w.lo = {*to + packed_bytes(rows, cols), cols, rows, up8(cols), true};
  *to += words_bytes(rows, cols);
  return w;
}

// 2^exponent_for(s) * s stays a factor of four or more below fp16's largest value
int exponent_for(double s) { return 14 - (int)std::ceil(std::log2(s > 1e-30 ? s : 1e-30)); }

// the largest |c0 t + c1 t^3 + c2 t^5| for t in [0, s]
double bound_of(double c0, double c1, double c2, double s) {
  auto at = [&](double t) { return std::fabs(((c2 * t * t + c1) * t * t + c0) * t); };
  double most = at(s);
  // where the slope c0 + 3 c1 q + 5 c2 q^2 vanishes, q = t^2
  const double qa = 5 * c2, qb = 3 * c1;
  double q[2];
  int n = 0;
  if (qa == 0.0) {
    if (qb != 0.0) q[n++] = -c0 / qb;
  } else {
    const double disc = qb * qb - 4 * qa * c0;
    if (disc >= 0.0) {
      q[n++] = (-qb + std::sqrt(disc)) / (2 * qa);
      q[n++] = (-qb - std::sqrt(disc)) / (2 * qa);
    }
  }
  for (int i = 0; i < n; ++i)
    if (q[i] > 0.0 && q[i] < s * s) most = std::fmax(most, at(std::sqrt(q[i])));
  return most;
}

constexpr float kUsual[3] = {3.4445f, -4.775f, 2.0315f};

template <int DT>
cudaError_t load(const LoadParams& p, unsigned blocks, cudaStream_t s) {
  const cudaError_t e = launch_early(squares_kernel<DT>, p.n_parts, kSumThreads, 0, s, p);
  return e != cudaSuccess ? e : launch_early(scale_kernel<DT>, blocks, kSumThreads, 0, s, p);
}

// the three products of two matrices in two words
void three(Problem* q, const Words& a, const Words& b, int64_t k) {
  q->a[0] = a.hi, q->a[1] = a.lo, q->n_a = 2;
  q->b[0] = b.hi, q->b[1] = b.lo, q->n_b = 2;
  q->segs = 3;
  q->p.seg_a = 0x100;  // high, high, low
  q->p.seg_b = 0x010;  // high, low, high
  q->k = k;
}

// v = alpha * C + beta * (A B), to be stored under 2^e
void combine(Problem* q, const Words* c, double alpha, double beta, int e_a, int e_b, int e) {
  if (c) {
    q->p.c0 = c->hi.p;
    q->p.c1 = c->lo.p;
    q->p.c_ld = c->hi.ld;
    q->p.c_vec = 1;
    q->p.alpha = (float)std::ldexp(alpha, e - c->e);
  }
  q->p.beta = (float)std::ldexp(beta, e - e_a - e_b);
}

void into(Problem* q, const Words& w) {
  q->out[0] = w.hi, q->out[1] = w.lo, q->n_out = 2;
  q->p.m = w.hi.outer;
  q->p.n = w.hi.inner;
}

}  // namespace
}  // namespace mfet

extern "C" {

uint64_t mfet_orthogonalize_bytes(int64_t rows, int64_t cols) {
  if (bad_sizes(rows, cols)) return 0;
  const int64_t d = rows < cols ? rows : cols;
  return kMostParts * 8 + 2 * words_bytes(rows, cols) + 2 * words_bytes(d, d);
}

int mfet_orthogonalize(const void* g, uint32_t dtype, int64_t ld, int64_t rows, int64_t cols, const float* coefficients, int32_t steps,
                       float scale, void* out, uint32_t out_dtype, int64_t out_ld, void* scratch, uint64_t scratch_bytes, uint32_t* status,
                       mfet_stream_t stream) {
  if (dtype > MFET_BF16 || out_dtype > MFET_BF16 || bad_sizes(rows, cols) || ld < cols || ld >= (1ll << 31) || out_ld < cols ||
      out_ld >= (1ll << 31) || steps < 1 || steps > kMostSteps || !std::isfinite(scale))
    return MFET_ERR_INVALID_ARG;
  // what bounds X's singular values before each step (1 at first: they are at most |G|), and B's largest magnitude
  double s[kMostSteps + 1], b_most[kMostSteps];
  s[0] = 1.0;
  for (int i = 0; i < steps; ++i) {
    const float* c = coefficients ? coefficients + 3 * i : kUsual;
    if (!std::isfinite(c[0]) || !std::isfinite(c[1]) || !std::isfinite(c[2])) return MFET_ERR_INVALID_ARG;
    s[i + 1] = bound_of(c[0], c[1], c[2], s[i]);
    const double q = s[i] * s[i];
    b_most[i] = std::fabs(c[1]) * q + std::fabs(c[2]) * q * q;
    if (s[i + 1] > 1048576.0 || b_most[i] > 1048576.0) return MFET_ERR_INVALID_ARG;
  }
  if (rows == 0 || cols == 0) return MFET_OK;
  if (!g || !out) return MFET_ERR_INVALID_ARG;
  if (!aligned(g, size_of(dtype)) || !aligned(out, size_of(out_dtype)) || !aligned(status, 4)) return MFET_ERR_ALIGNMENT;
  if (!scratch || scratch_bytes < mfet_orthogonalize_bytes(rows, cols)) return MFET_ERR_WORKSPACE;
  if (!aligned(scratch, 16)) return MFET_ERR_ALIGNMENT;
  const cudaStream_t st = (cudaStream_t)stream;
  const int64_t d = rows < cols ? rows : cols;
  uint8_t* to = (uint8_t*)scratch + kMostParts * 8;
  Words x[2] = {words_at(&to, rows, cols), words_at(&to, rows, cols)};
  Words a = words_at(&to, d, d), b = words_at(&to, d, d);

  x[0].e = exponent_for(s[0]);
  LoadParams p{};
  p.g = (const uint8_t*)g;
  p.rows = rows, p.cols = cols, p.ld = ld;
  p.end = p.g + ((rows - 1) * ld + cols) * size_of(dtype);
  p.vec = aligned(g, 16) && (uint64_t)ld * size_of(dtype) % 16 == 0;
  p.parts = (double*)scratch;
  p.hi = (__half*)x[0].hi.p, p.lo = (__half*)x[0].lo.p;
  p.x_ld = x[0].hi.ld;
  p.scale = std::ldexp(1.0, x[0].e);
  const int64_t want = (rows * (p.x_ld / 8) + kSumThreads - 1) / kSumThreads;
  p.n_parts = (uint32_t)(want < kMostParts ? want : kMostParts);
  const int64_t most = (int64_t)sm_count() * 8;
  const unsigned blocks = (unsigned)(want < most ? want : most);
  const cudaError_t e = dtype == MFET_F32   ? load<MFET_F32>(p, blocks, st)
                        : dtype == MFET_F16 ? load<MFET_F16>(p, blocks, st)
                                            : load<MFET_BF16>(p, blocks, st);
  if (e != cudaSuccess) return MFET_ERR_CUDA;

  const bool tall = rows > cols;
  for (int i = 0; i < steps; ++i) {
    const float* c = coefficients ? coefficients + 3 * i : kUsual;
    const Words& from = x[i & 1];
    Words& next = x[(i + 1) & 1];
    // A = X X^T, or X^T X
    a.e = exponent_for(s[i] * s[i]);
    Problem q;
    q.p.status = status;
    three(&q, from, from, tall ? rows : cols);
    q.p.a_mn = q.p.b_mn = tall;
    combine(&q, nullptr, 0.0, 1.0, from.e, from.e, a.e);
    into(&q, a);
    int rc = run<kPair, MFET_F16>(q, st);
    if (rc != MFET_OK) return rc;
    // B = b A + c A A, A being symmetric
    b.e = exponent_for(b_most[i]);
    q = Problem();
    q.p.status = status;
    three(&q, a, a, d);
    combine(&q, &a, c[1], c[2], a.e, a.e, b.e);
    into(&q, b);
    rc = run<kPair, MFET_F16>(q, st);
    if (rc != MFET_OK) return rc;
    // X = a X + B X, or a X + X B, B being symmetric
    q = Problem();
    q.p.status = status;
    if (tall) three(&q, from, b, d);
    else three(&q, b, from, d);
    q.p.b_mn = !tall;
    if (i + 1 < steps) {
      next.e = exponent_for(s[i + 1]);
      combine(&q, &from, c[0], 1.0, from.e, b.e, next.e);
      into(&q, next);
      rc = run<kPair, MFET_F16>(q, st);
    } else {
      combine(&q, &from, (double)c[0] * scale, scale, from.e, b.e, 0);
      q.out[0] = {out, cols, rows, out_ld};
      q.out_dtype = out_dtype;
      q.p.m = rows;
      q.p.n = cols;
      rc = out_dtype == MFET_F32   ? run<kPairOut, MFET_F32>(q, st)
           : out_dtype == MFET_F16 ? run<kPairOut, MFET_F16>(q, st)
                                   : run<kPairOut, MFET_BF16>(q, st);
    }
    if (rc != MFET_OK) return rc;
  }
  return MFET_OK;
}

}  // extern "C"
