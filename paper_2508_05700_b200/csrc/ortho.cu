// A matrix orthogonalised by Newton-Schulz products: X = G / |G|, then per step, with A = X X^T over the shorter side,
//
//   X <- a X + (b A + c A A) X
//
// which takes every singular value s of X to a s + b s^3 + c s^5 and leaves the singular vectors. A step multiplies small singular
// values, and the errors in their directions, by a (3.4 in the usual schedule, some 480 in five steps): with operands of one 16-bit
// word the result is off by 1e-3 (fp16) to 1e-2 (bf16) of its size. So X, A and B = b A + c A A are held as the sum of two fp16 words
// (22 bits and more, under a power of two for each matrix that keeps its bound, known to the host, inside fp16's range), a product is three
// (high x low, low x high, then high x high: the tensor cores truncate a sum after
// every 16 products, by a part of what it is by then) in fp32 accumulators of a part of the sum each, and the result is as near as one computed in fp32.
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

template <int THREADS>
__device__ __forceinline__ double block_sum(double s, double* words) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(kAllLanes, s, d);
  if ((threadIdx.x & 31) == 0) words[threadIdx.x >> 5] = s;
  __syncthreads();
  s = 0.0;
  for (int i = 0; i < THREADS / 32; ++i) s += words[i];
  return s;
}

// what G is multiplied by, from its sum of squares: 0 for 0, NaN if G has a value that is not finite
__device__ __forceinline__ double factor_of(double squares, double scale) {
  return squares > 0.0 ? (isinf(squares) ? NAN : scale / sqrt(squares)) : (squares == 0.0 ? 0.0 : squares);
}
__device__ __forceinline__ void cluster_or_block_sync(bool cluster) {
  __syncthreads();
  if (cluster) cluster_sync();
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
  s = block_sum<kSumThreads>(s, words);
  if (threadIdx.x == 0 && MFET_INSIDE(nullptr, blockIdx.x < p.n_parts)) p.parts[blockIdx.x] = s;
}

// X = G / |G| in two words; 0 for G = 0, NaN throughout if G has a value that is not finite
template <int DT>
__global__ void __launch_bounds__(kSumThreads) scale_kernel(const __grid_constant__ LoadParams p) {
  __shared__ double words[kSumThreads / 32];
  early_launch_wait();
  double total = 0.0;
  for (uint32_t i = threadIdx.x; i < p.n_parts; i += kSumThreads) total += p.parts[i];
  total = block_sum<kSumThreads>(total, words);
  const double f = factor_of(total, p.scale);
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

// ------------------------------------------------------------------ a short side of at most 128 ----

// All of the call in one launch: the long side in slices of up to 256 columns (of X with the short side as its rows), one per block of a
// cluster. A block has its slice of X in shared memory, in two words and in the order of the tensor cores: rows of 64 columns, 128 bytes with
// the 128-byte swizzle, are K-major for X X^T and, the other way round, MN-major for B X. A step: the slice's X X^T, summed over the cluster
// (each block adds up a share of the columns in the order of the slices, and all read the sums), B by every block for itself, and the slice of
// a X + B X over the old one. (With a on B's diagonal X is not read again, 3 us less, and errors are 1.4 times as large.) What costs is the
// chain: three products, each waited for, and three turns from tensor memory to shared memory.
// In five steps, here and as seventeen launches: 48 x 192 36 and 72 us, 128 x 128 42 and 76, 128 x 512 83 and 91, 128 x 2048 92 and 127. Beyond: 129 x 512
// 103, 129 x 2048 137 (a short side above 128 does not fit the tensor cores' 128 lanes), 128 x 4096 162 (eight blocks hold no longer side).
constexpr int kSmallThreads = 512;
constexpr int kSmallSide = 128, kSlice = 256, kMostSlices = 8;
constexpr uint32_t kBlock = 128 * 128;                    // 128 rows x 64 columns
constexpr uint32_t kXLo = kSlice / 64 * kBlock, kAHi = 2 * kXLo, kALo = kAHi + 2 * kBlock, kSmallBytes = kALo + 2 * kBlock;
constexpr uint32_t kSmallSmem = kSmallBytes + 1024;
static_assert(kALo - kAHi == 32768 && 2 * (kALo - kAHi) == 128 * 128 * 4, "partial sums in fp32 take the place of A");

struct SmallStep {
  float a_beta, b_alpha, b_beta, x_alpha, x_beta;
};
struct SmallParams {
  const uint8_t* g;
  void* out;
  int64_t ld, out_ld;
  int64_t long_side;
  int32_t d, slices, steps;
  uint32_t tall;       // the short side is the columns of g
  bool vec;            // rows of g start on 16-byte boundaries
  const void* end;     // of g
  uint32_t out_dtype;
  uint32_t* status;
  double scale;        // 2^e of X's words
  SmallStep step[kMostSteps];
};

// where 8 columns from c on of row r are in a matrix of blocks
__device__ __forceinline__ uint32_t words_offset(int r, int c) { return (uint32_t)(c >> 6) * kBlock + r * 128 + ((((c >> 3) & 7) ^ (r & 7)) << 4); }

// X[i][c .. c + 8) before it is scaled, 0 outside X. Its loads depend on nothing, so that a thread's can all be under way: outside X, and for
// a long side that 8 does not divide, they are of another element.
template <int DT>
__device__ __forceinline__ void eight_of(const SmallParams& p, int i, int64_t c, float* v) {
  using T = typename Elem<DT>::T;
  const T* g = reinterpret_cast<const T*>(p.g);
  const int64_t left = p.long_side - c;
  int count = i >= p.d || left <= 0 ? 0 : left < 8 ? (int)left : 8;
  const int64_t row = min(i, p.d - 1);
  if (!MFET_INSIDE(p.status, (p.tall ? row + 1 : count ? c + count : 0) <= p.ld)) count = 0;
  if (p.vec && !p.tall && p.long_side % 8 == 0) {
    widen_raw<DT, 8>(load_raw<DT, 8, true>(g + (count ? row * p.ld + c : 0), 8), v);
  } else if (p.tall) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = to_float<DT>(g[(c + j < p.long_side ? c + j : p.long_side - 1) * p.ld + row]);
  } else if (count) {
    widen_raw<DT, 8>(load_shifted<DT, 8>(g + row * p.ld + c, count, p.g, p.end), v);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = j < count ? v[j] : 0.f;
}

__device__ __forceinline__ void put_words(uint8_t* hi, uint8_t* lo, float* v) {  // 8 values, 16 bytes each
  const uint4 h = narrow16<MFET_F16>(v);
  float w[8];
  widen16<MFET_F16>(h, w);
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const float2 d = fma2(make_float2(w[j], w[j + 1]), both(-1.f), make_float2(v[j], v[j + 1]));
    w[j] = d.x, w[j + 1] = d.y;
  }
  *reinterpret_cast<uint4*>(hi) = h;
  *reinterpret_cast<uint4*>(lo) = narrow16<MFET_F16>(w);
}
__device__ __forceinline__ void get_words(const uint8_t* hi, const uint8_t* lo, float* v) {
  float r[8];
  widen16<MFET_F16>(*reinterpret_cast<const uint4*>(hi), v);
  widen16<MFET_F16>(*reinterpret_cast<const uint4*>(lo), r);
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const float2 a = add2(make_float2(v[j], v[j + 1]), make_float2(r[j], r[j + 1]));
    v[j] = a.x, v[j + 1] = a.y;
  }
}
// 8 values a * x + b * y into x
__device__ __forceinline__ void combine8(float* x, float a, const uint32_t* y, float b) {
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const float2 v = fma2(make_float2(__uint_as_float(y[j]), __uint_as_float(y[j + 1])), both(b), mul2(make_float2(x[j], x[j + 1]), both(a)));
    x[j] = v.x, x[j + 1] = v.y;
  }
}
__device__ __forceinline__ void mma_small(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t b_hi, uint32_t inst, uint32_t add) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
               "setp.ne.b32 p, %5, 0;\n\t"
               "mov.b64 a, {%1, %6};\n\t"
               "mov.b64 b, {%2, %3};\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n\t}" ::"r"(d),
               "r"(a_lo), "r"(b_lo), "r"(b_hi), "r"(inst), "r"(add), "n"(kDescHi)
               : "memory");
}

template <int DT>
__global__ void __launch_bounds__(kSmallThreads, 1) ortho_small_kernel(const __grid_constant__ SmallParams p) {
  extern __shared__ uint8_t raw_smem[];
  __shared__ __align__(8) uint64_t bar_words[2];
  __shared__ double sums[kSmallThreads / 32];
  __shared__ double total_of_block;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int dead;
  const uint32_t base = (smem_addr(raw_smem) + 1023) & ~1023u;
  uint8_t* const smem = raw_smem + (base - smem_addr(raw_smem));
  const uint32_t bar = smem_addr(bar_words), drained = bar + 8;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int slices = p.slices;
  const uint32_t rank = slices > 1 ? cluster_rank() : 0u;
  if (tid == 0) {
    bar_init(bar, 1);
    bar_init(drained, 1);
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&tmem_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  // accumulators of X X^T and A A: two of half of k each (what a sum loses to truncation grows with its length); of B X: two where they fit
  const uint32_t tmem = tmem_slot, acc_x = tmem + 128;
  constexpr uint32_t kSecondA = 384, kSecondX = 128;
  early_launch_wait();

  // this block's columns of X, in whole blocks of 64
  const int64_t all = (p.long_side + 63) / 64;
  const int64_t c0 = all * rank / slices * 64;
  const int width = (int)((all * (rank + 1) / slices) * 64 - c0);
  const int d16 = (p.d + 15) & ~15, half_d = (d16 / 16 + 1) / 2;  // instructions of the first sum over the short side
  const bool two_d = d16 > 16, two_x = two_d && width <= (int)128;

  // squares of the slice, then of all of G; 8 neighbouring columns of a row at a time
  double s = 0.0;
  const int units = 128 * (width / 8);
  const uint32_t per = (uint32_t)width / 8;
  auto place = [&](int u, int* i, int* c) {
    *i = p.tall ? u & 127 : (int)((uint32_t)u / per);
    *c = (p.tall ? u >> 7 : u - *i * (int)per) * 8;
  };
  constexpr int kUnits = 128 * (kSlice / 8) / kSmallThreads;  // of a thread, in registers until |G| is known
  float g[kUnits][8];
#pragma unroll
  for (int n = 0; n < kUnits; ++n) {
    const int u = tid + n * kSmallThreads;
    int i, c;
    place(u, &i, &c);
    eight_of<DT>(p, u < units ? i : 128, c0 + c, g[n]);
  }
  double s2 = 0.0;
#pragma unroll
  for (int n = 0; n < kUnits; ++n) {
    if (n * kSmallThreads >= units) break;
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      s = fma((double)g[n][j], (double)g[n][j], s);
      s2 = fma((double)g[n][j + 1], (double)g[n][j + 1], s2);
    }
  }
  s += s2;
  s = block_sum<kSmallThreads>(s, sums);
  if (slices > 1) {
    if (tid == 0) total_of_block = s;
    __syncthreads();
    cluster_sync();
    s = 0.0;
    for (int q = 0; q < slices; ++q) {
      double v;
      asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(peer_addr(smem_addr(&total_of_block), q)) : "memory");
      s += v;
    }
  }
  // The factor as a power of two, half of it before and half after, and a fraction in two words: fp32's range is enough for either half
  // where it may not be for the factor, and the result is off by an ulp at most. (Conversions to fp64 and back took 4 us.)
  int e = 0;
  const double f = frexp(factor_of(s, p.scale), &e);
  if (!(f > 0.0)) e = 0;
  const float f_hi = (float)f, f_lo = (float)(f - f_hi), before = ldexpf(1.f, e / 2), after = ldexpf(1.f, e - e / 2);
#pragma unroll
  for (int n = 0; n < kUnits; ++n) {
    const int u = tid + n * kSmallThreads;
    if (u >= units) break;
    int i, c;
    place(u, &i, &c);
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const float2 x = mul2(make_float2(g[n][j], g[n][j + 1]), both(before));
      const float2 y = mul2(fma2(x, both(f_hi), mul2(x, both(f_lo))), both(after));
      g[n][j] = y.x, g[n][j + 1] = y.y;
    }
    const uint32_t at = words_offset(i, c);
    put_words(smem + at, smem + kXLo + at, g[n]);
  }

  uint32_t phase = 0;
  // Every product that this warp waited for has ended. Where it has not, its operands may still be read: from then on the warp issues nothing and writes
  // no words, but comes to every barrier. (A warp that has seen the product end may go on: what it overwrites is no longer read.)
  bool ok = true;
  bool issues = false;  // this lane issues the products
  auto ready = [&]() {  // what this block's threads have written is there for the tensor cores
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  };
  auto done = [&]() {  // the products that one lane has issued
    ok = __all_sync(kAllLanes, ok && bar_wait(bar, phase, &dead));
    phase ^= 1;
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  };
  auto sums_of = [&](uint32_t at, uint32_t second, bool two, uint32_t* r) {
    tmem_load32(at, r);
    if (two) {
      uint32_t t[32];
      tmem_load32(at + second, t);
#pragma unroll
      for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) + __uint_as_float(t[j]));
    }
  };
  const uint32_t inst_a = (1u << 4) | ((uint32_t)(d16 >> 3) << 17) | (8u << 24);
  const uint32_t inst_x = (1u << 4) | (1u << 16) | ((uint32_t)(width >> 3) << 17) | (8u << 24);
  const uint32_t xs[2] = {base, base + kXLo}, as[2] = {base + kAHi, base + kALo};
  const int quarter = warp & 3, row = quarter * 32 + lane, turn = warp >> 2;  // four warps share the lanes of tensor memory
  const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
  cluster_or_block_sync(slices > 1);

#pragma unroll 1
  for (int step = 0; step < p.steps; ++step) {
    const SmallStep k = p.step[step];
    ready();
    // A = X X^T over the slice
    if (warp == 0 && ok) {
      if (elect_one()) {
        issues = true;
        for (int t = 0; t < 3; ++t) {  // high x low, low x high, high x high
          const uint32_t a = xs[t == 1], b = xs[t == 0];
          for (int q = 0; q < width / 16; ++q) {
            const uint32_t off = (uint32_t)(q >> 2) * kBlock + (q & 3) * 32, z = q >= width / 32;
            mma_small(tmem + z * kSecondA, desc_lo(a + off, 0), desc_lo(b + off, 0), kDescHi, inst_a, t || (q && q != width / 32));
          }
        }
        mma_commit(bar);
      }
      __syncwarp();
    }
    done();
    if (slices == 1) {
#pragma unroll 1
      for (int c = 32 * turn; ok && c < d16; c += 128) {
        uint32_t r[32];
        sums_of(tmem + lanes + c, kSecondA, true, r);
#pragma unroll
        for (int j = 0; j < 32; j += 8) {
          if (c + j >= d16) break;
          const uint32_t at = words_offset(row, c + j);
          float* const v = reinterpret_cast<float*>(r) + j;
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= k.a_beta;
          put_words(smem + kAHi + at, smem + kALo + at, v);
        }
      }
    } else {
      // the slice's sums, four columns of a row in 16 bytes, where A was
#pragma unroll 1
      for (int c = 32 * turn; ok && c < d16; c += 128) {
        uint32_t r[32];
        sums_of(tmem + lanes + c, kSecondA, true, r);
#pragma unroll
        for (int j = 0; j < 32; j += 4)
          *reinterpret_cast<uint4*>(smem + kAHi + (((c + j) >> 2) * 128 + row) * 16) = make_uint4(r[j], r[j + 1], r[j + 2], r[j + 3]);
      }
      cluster_sync();
      // Every block adds up each `slices`-th group of columns, four warps of a row in turn, and leaves the sums where its own part of
      // them was; then all read them there. (Words stored into all blocks, 8 bytes a row: 27000 cycles a step with 8 blocks.)
      constexpr int kMostGroups = 4;  // 32 groups, two blocks at least and four warps
#pragma unroll
      for (int q = 0; q < kMostGroups; ++q) {
        const int group = (int)rank + slices * (4 * q + turn);
        if (!ok || group * 4 >= d16) break;
        const uint32_t at = (group * 128 + row) * 16;
        float t[kMostSlices][4], v[4];
#pragma unroll
        for (int z = 0; z < kMostSlices; ++z)
          if (z < slices) peer_load(peer_addr(base + kAHi + at, z), t[z]);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = t[0][j];
#pragma unroll
        for (int z = 1; z < kMostSlices; ++z) {
          if (z >= slices) break;
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] += t[z][j];
        }
        *reinterpret_cast<float4*>(smem + kAHi + at) = make_float4(v[0] * k.a_beta, v[1] * k.a_beta, v[2] * k.a_beta, v[3] * k.a_beta);
      }
      cluster_sync();
      // two groups, 8 columns, a turn
      constexpr int kPairs = kMostGroups;  // 16 pairs of groups, four warps
      float v[kPairs][8];
#pragma unroll
      for (int q = 0; q < kPairs; ++q) {
        const int group = 2 * (4 * q + turn);
        if (group * 4 >= d16) break;
        const uint32_t at = base + kAHi + (group * 128 + row) * 16;
        peer_load(peer_addr(at, group & (slices - 1)), v[q]);
        peer_load(peer_addr(at + 2048, (group + 1) & (slices - 1)), v[q] + 4);
      }
      cluster_sync();  // all sums have been read: A goes to their place
#pragma unroll
      for (int q = 0; q < kPairs; ++q) {
        const int c = 8 * (4 * q + turn);
        if (!ok || c >= d16) break;
        const uint32_t at = words_offset(row, c);
        put_words(smem + kAHi + at, smem + kALo + at, v[q]);
      }
    }
    ready();
    // A A, A being symmetric
    if (warp == 0 && ok) {
      if (elect_one()) {
        issues = true;
        for (int t = 0; t < 3; ++t) {
          const uint32_t a = as[t == 1], b = as[t == 0];
          for (int q = 0; q < d16 / 16; ++q) {
            const uint32_t off = (uint32_t)(q >> 2) * kBlock + (q & 3) * 32, z = q >= half_d;
            mma_small(tmem + z * kSecondA, desc_lo(a + off, 0), desc_lo(b + off, 0), kDescHi, inst_a, t || (q && q != half_d));
          }
        }
        mma_commit(bar);
      }
      __syncwarp();
    }
    done();
    // B = b A + c A A over A
#pragma unroll 1
    for (int c = 32 * turn; ok && c < d16; c += 128) {
      uint32_t r[32];
      sums_of(tmem + lanes + c, kSecondA, two_d, r);
#pragma unroll
      for (int j = 0; j < 32; j += 8) {
        if (c + j >= d16) break;
        const uint32_t at = words_offset(row, c + j);
        float a[8];
        get_words(smem + kAHi + at, smem + kALo + at, a);
        combine8(a, k.b_alpha, r + j, k.b_beta);
        put_words(smem + kAHi + at, smem + kALo + at, a);
      }
    }
    ready();
    // B X
    if (warp == 0 && ok) {
      if (elect_one()) {
        issues = true;
        for (int t = 0; t < 3; ++t) {
          const uint32_t a = as[t == 1], b = xs[t == 0];
          for (int q = 0; q < d16 / 16; ++q) {
            const uint32_t b_lo = (((b + q * 2048) & 0x3FFFFu) >> 4) | ((kBlock >> 4) << 16), z = two_x && q >= half_d;
            mma_small(acc_x + z * kSecondX, desc_lo(a + (uint32_t)(q >> 2) * kBlock + (q & 3) * 32, 0), b_lo, kDescHi, inst_x,
                      t || (q && !(two_x && q == half_d)));
          }
        }
        mma_commit(bar);
      }
      __syncwarp();
    }
    done();
    const bool last = step + 1 == p.steps;
#pragma unroll 1
    for (int c = 32 * turn; ok && c < width; c += 128) {
      uint32_t r[32];
      sums_of(acc_x + lanes + c, kSecondX, two_x, r);
#pragma unroll
      for (int j = 0; j < 32; j += 8) {
        const uint32_t at = words_offset(row, c + j);
        float x[8];
        get_words(smem + at, smem + kXLo + at, x);
        combine8(x, k.x_alpha, r + j, k.x_beta);
        if (!last) {
          put_words(smem + at, smem + kXLo + at, x);
        } else {  // fp32, in the place of both words
          *reinterpret_cast<float4*>(smem + at) = make_float4(x[0], x[1], x[2], x[3]);
          *reinterpret_cast<float4*>(smem + kXLo + at) = make_float4(x[4], x[5], x[6], x[7]);
        }
      }
    }
  }
  // A warp writes a row of the result at a time. (From tensor memory, a lane with its own row: 8 us for 48 x 192.)
  __syncthreads();
  const int64_t left = p.long_side - c0;
  const int most = left < width ? (int)left : width, rows = p.tall ? most : p.d, cols = p.tall ? p.d : most;
  for (int i = warp; i < rows; i += kSmallThreads / 32) {
    const int64_t first = p.tall ? (c0 + i) * p.out_ld : i * p.out_ld + c0;
#pragma unroll 4
    for (int j = lane; j < cols; j += 32) {
      const int r = p.tall ? j : i, c = p.tall ? i : j;
      const float x = *reinterpret_cast<const float*>(smem + (c & 4 ? kXLo : 0u) + words_offset(r, c & ~7) + (c & 3) * 4);
      if (!MFET_INSIDE(p.status, (p.tall ? j : c0 + j) < p.out_ld)) continue;
      if (p.out_dtype == MFET_F32) reinterpret_cast<float*>(p.out)[first + j] = x;
      else if (p.out_dtype == MFET_F16) reinterpret_cast<__half*>(p.out)[first + j] = __float2half_rn(x);
      else reinterpret_cast<__nv_bfloat16*>(p.out)[first + j] = __float2bfloat16_rn(x);
    }
  }
  if (dead) {  // all threads have ended their last wait: what is waited for now, with the same limit, is the last product under way
    volatile int none = 0;
    if (issues) {
      mma_commit(drained);
      bar_wait(drained, 0, &none);
    }
    if (tid == 0 && p.status) atomicOr(p.status, (uint32_t)MFET_DEV_STALLED);
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  cluster_or_block_sync(slices > 1);
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
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
  // where the slope c0 + 3 c1 q + 5 c2 q^2 vanishes, q = t^2: h / (5 c2) and c0 / h. (The usual formula for the second subtracts two numbers that agree
  // where c2 is small, and finds q = 0.)
  const double qa = 5 * c2, qb = 3 * c1, disc = qb * qb - 4 * qa * c0;
  double q[2];
  int n = 0;
  if (disc >= 0.0) {
    const double h = -0.5 * (qb + std::copysign(std::sqrt(disc), qb));
    if (qa != 0.0) q[n++] = h / qa;
    if (h != 0.0) q[n++] = c0 / h;
  }
  for (int i = 0; i < n; ++i)
    if (q[i] > 0.0 && q[i] < s * s) most = std::fmax(most, at(std::sqrt(q[i])));
  return most;
}

constexpr float kUsual[3] = {3.4445f, -4.775f, 2.0315f};

template <int DT>
int launch_small(const SmallParams& p, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  if (allow_smem(ortho_small_kernel<DT>, kSmallSmem, &ready) != cudaSuccess) return MFET_ERR_CUDA;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.slices;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)p.slices);
  cfg.blockDim = dim3(kSmallThreads);
  cfg.dynamicSmemBytes = kSmallSmem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = p.slices > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, ortho_small_kernel<DT>, p) == cudaSuccess ? MFET_OK : MFET_ERR_CUDA;
}

template <int DT>
cudaError_t load(const LoadParams& p, unsigned blocks, cudaStream_t s) {
  const cudaError_t e = launch_early(squares_kernel<DT>, p.n_parts, kSumThreads, 0, s, p);
  return e != cudaSuccess ? e : launch_early(scale_kernel<DT>, blocks, kSumThreads, 0, s, p);
}

// Sums that are longer are taken in parts of few instructions each, which are added up outside the tensor cores: with fp32 results, and with 16-bit ones.
// Error of five steps to fp32 in one run of sums, in parts and of an iteration in fp32: 64 x 2^20 2.1e-4 of the result, 1.5e-6, 0.9e-6; 500 x 40000 5.4e-6,
// 3.3e-6, 2.5e-6; 2048 x 16384 1.3e-5, 2.2e-6, 3.1e-6. Time: 17.3 -> 21.4 ms, 1.21 -> 1.41, 3.53 -> 3.72 (a part's sums are read while the next part's
// products are under way, which takes longer than these do).
constexpr int64_t kLongSum = 4096, kLongSum16 = 65536;

// the three products of two matrices in two words
void three(Problem* q, const Words& a, const Words& b, int64_t k) {
  q->a[0] = a.hi, q->a[1] = a.lo, q->n_a = 2;
  q->b[0] = b.hi, q->b[1] = b.lo, q->n_b = 2;
  q->segs[0] = 3;
  q->p.part[0].seg_a = 0x010;  // high, low, high
  q->p.part[0].seg_b = 0x001;  // low, high, high
  q->k[0] = k;
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
  q->p.part[0].m = w.hi.outer;
  q->p.part[0].n = w.hi.inner;
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
  const int64_t d = rows < cols ? rows : cols, l = rows < cols ? cols : rows;
  const bool tall = rows > cols;
  if (d <= kSmallSide && l <= kSlice * kMostSlices) {
    SmallParams q{};
    q.g = (const uint8_t*)g;
    q.out = out;
    q.ld = ld, q.out_ld = out_ld;
    q.long_side = l;
    q.d = (int32_t)d;
    q.slices = l <= kSlice ? 1 : l <= 2 * kSlice ? 2 : l <= 4 * kSlice ? 4 : 8;
    q.steps = steps;
    q.tall = tall;
    q.vec = aligned(g, 16) && (uint64_t)ld * size_of(dtype) % 16 == 0;
    q.end = (const uint8_t*)g + ((rows - 1) * ld + cols) * size_of(dtype);
    q.out_dtype = out_dtype;
    q.status = status;
    int ex = exponent_for(s[0]);
    q.scale = std::ldexp(1.0, ex);
    for (int i = 0; i < steps; ++i) {
      const float* c = coefficients ? coefficients + 3 * i : kUsual;
      const int ea = exponent_for(s[i] * s[i]), eb = exponent_for(b_most[i]), next = exponent_for(s[i + 1]);
      const bool last = i + 1 == steps;
      // What the tensor cores' sums lose on average is put back (see launch in gemm16.cuh): sums of a slice, then of the short side, as of two sums each.
      // B X of slices wider than 128 columns is one sum, of which half stays: a step of fp32 at most, and a factor beside 1 comes in such steps only
      // (following the form changed 128 x 2048 by nothing and 48 x 192 from 1.3e-6 to 1.6e-6 of the result, which is one step in one coefficient).
      const double lost = 0.18 * 0x1p-23, of_l = 1.0 + lost * (double)(l / 32 / q.slices), of_d = 1.0 + lost * (double)(d / 32);
      q.step[i].a_beta = (float)std::ldexp(of_l, ea - 2 * ex);
      q.step[i].b_alpha = (float)std::ldexp((double)c[1], eb - ea);
      q.step[i].b_beta = (float)std::ldexp(of_d * c[2], eb - 2 * ea);
      q.step[i].x_alpha = (float)std::ldexp(last ? (double)c[0] * scale : (double)c[0], (last ? 0 : next) - ex);
      q.step[i].x_beta = (float)std::ldexp(of_d * (last ? (double)scale : 1.0), (last ? 0 : next) - eb - ex);
      ex = next;
    }
    return dtype == MFET_F32 ? launch_small<MFET_F32>(q, st) : dtype == MFET_F16 ? launch_small<MFET_F16>(q, st) : launch_small<MFET_BF16>(q, st);
  }
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

  const bool precise = out_dtype == MFET_F32;
  auto words_of = [&](const Problem& q) { return q.k[0] > (precise ? kLongSum : kLongSum16) ? run<kPairLong, MFET_F16>(q, st) : run<kPair, MFET_F16>(q, st); };
  for (int i = 0; i < steps; ++i) {
    const float* c = coefficients ? coefficients + 3 * i : kUsual;
    const Words& from = x[i & 1];
    Words& next = x[(i + 1) & 1];
    // A = X X^T, or X^T X
    a.e = exponent_for(s[i] * s[i]);
    Problem q;
    q.p.status = status;
    q.precise = precise;
    three(&q, from, from, tall ? rows : cols);
    q.p.part[0].a_mn = q.p.part[0].b_mn = tall;
    q.a_mn = q.b_mn = tall ? 3 : 0;
    q.p.sym = 1;
    combine(&q, nullptr, 0.0, 1.0, from.e, from.e, a.e);
    into(&q, a);
    int rc = words_of(q);
    if (rc != MFET_OK) return rc;
    // B = b A + c A A, A being symmetric
    b.e = exponent_for(b_most[i]);
    q = Problem();
    q.p.status = status;
    q.precise = precise;
    three(&q, a, a, d);
    q.p.sym = 1;
    combine(&q, &a, c[1], c[2], a.e, a.e, b.e);
    into(&q, b);
    rc = words_of(q);
    if (rc != MFET_OK) return rc;
    // X = a X + B X, or a X + X B, B being symmetric
    q = Problem();
    q.p.status = status;
    q.precise = precise;
    if (tall) three(&q, from, b, d);
    else three(&q, b, from, d);
    q.p.part[0].b_mn = !tall;
    q.b_mn = tall ? 0 : 3;
    if (i + 1 < steps) {
      next.e = exponent_for(s[i + 1]);
      combine(&q, &from, c[0], 1.0, from.e, b.e, next.e);
      into(&q, next);
      rc = words_of(q);
    } else {
      combine(&q, &from, (double)c[0] * scale, scale, from.e, b.e, 0);
      q.out[0] = {out, cols, rows, out_ld};
      q.out_dtype = out_dtype;
      q.p.part[0].m = rows;
      q.p.part[0].n = cols;
      rc = precise                 ? (d > kLongSum ? run<kPairOutLong, MFET_F32>(q, st) : run<kPairOut, MFET_F32>(q, st))
           : out_dtype == MFET_F16 ? run<kPairOut, MFET_F16>(q, st)
                                   : run<kPairOut, MFET_BF16>(q, st);
    }
    if (rc != MFET_OK) return rc;
  }
  return MFET_OK;
}

}  // extern "C"
