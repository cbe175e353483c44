// Global 2-norm of many gradient tensors, and the gradients scaled so that it is at most max_norm.
//
//   norm = sqrt(sum over all elements of g^2),  coef = norm > max_norm ? max_norm / norm : 1,  dst = round(g * coef)
//
// Two launches over the same pieces of 32 KB. The first adds up the squares in fp64 and leaves one sum per block. The second adds
// those sums up - every block the same ones in the same order, which costs less than another launch or a count of finished blocks -
// and scales. It walks the pieces from the last to the first, because the end of what the first launch has read is still in L2: all but
// the last 64 MB are read as what leaves it first (9 us less for 200 M bf16 values). Marking the last 64 MB to stay as well gained
// nothing more, and those lines stayed behind when nothing was scaled.
// Bound by DRAM, most of three passes, two of which the result needs: 33 M fp32 values in twelve lists 66 us (338 MB of traffic, 5.1 TB/s: 56 of
// the 132 MB of the second read come from L2), 200 M bf16 values in 300 tensors 218 us (1.16 GB, 5.3 TB/s: 45 MB come from L2); the norm of
// 200 M bf16 values alone 62 us (6.4 TB/s). Nothing depends on which block finishes when: equal inputs give equal bits.
#include <cmath>
#include <cstring>

#include "lowbit.cuh"

using namespace mfet;

namespace mfet {
namespace {

constexpr int kClipThreads = 256;
constexpr int kClipInFlight = 8;                                  // 16-byte loads that a thread requests together
constexpr int kPieceVecs = kClipThreads * kClipInFlight;          // 16-byte vectors per piece
constexpr int kClipBlocksPerSm = 4;
constexpr int kKeepPieces = 2048;                                 // 64 MB: what is still in L2 for the second launch

struct GradDev {
  const uint8_t* src;
  uint8_t* dst;           // nullptr: only counted
  const int64_t* n_rows;  // nullptr, or the number of rows on the device
  int64_t rows, cols, ld;
  int64_t pad;
  uint32_t dtype;
  uint32_t lead;          // elements between the 16-byte boundary before src and src; vectors are counted from that boundary
};
static_assert(sizeof(GradDev) == 64, "the capacities below count 64-byte entries");

// Tensors per launch: the entries are kernel parameters. The small block keeps the launch of a few tensors cheap:
// two tensors in two launches take a program 10.1 us with it, 13.2 with the large one.
constexpr int kFewTensors = 48, kManyTensors = 448;
template <int N>
struct GradParams {
  double* sums;       // all sums of the call
  float* norm;
  double max_norm;
  int64_t pieces;
  int32_t n;          // tensors of this launch
  int32_t first_sum;  // where this launch's blocks put theirs
  int32_t n_sums;     // sums of the call
  int32_t pad;
  GradDev t[N];
};
static_assert(sizeof(GradParams<kManyTensors>) <= 32000, "kernel parameters are limited to 32764 bytes");

// What a block works on: its share of the pieces that hold elements. The counts on the device are read once per block, the pieces of
// the tensors before each one are added up in shared memory, and the block goes along: no search per piece, and a list that is half
// empty spreads as evenly as a full one.
template <int N>
struct Share {
  int64_t live[N];    // elements
  int32_t first[N];   // pieces of the tensors before
  int32_t warp_sum[kClipThreads / 32];
  int32_t total;

  template <class P>
  __device__ __forceinline__ void fill(const P& p) {
    // Every thread has an entry of its own here. Constant loads would go through the entries one by one (20 us for 300 tensors):
    // behind this the compiler no longer knows where they are, and uses ordinary ones.
    const GradDev* entries = p.t;
    asm volatile("" : "+l"(entries));
    constexpr int kPer = (N + kClipThreads - 1) / kClipThreads;
    int32_t mine[kPer], sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = (int)threadIdx.x * kPer + j;
      mine[j] = 0;
      if (i < p.n && MFET_INSIDE(nullptr, i < N)) {
        const GradDev& t = entries[i];
        int64_t r = t.rows;
        if (t.n_rows) {
          const int64_t v = *t.n_rows;
          r = v < 0 ? 0 : (v < r ? v : r);
        }
        const int64_t e = r * t.cols, per = kPieceVecs * (t.dtype == MFET_F32 ? 4 : 8);
        live[i] = e;
        mine[j] = e > 0 ? (int32_t)((e + t.lead + per - 1) / per) : 0;
      }
      sum += mine[j];
    }
    int32_t before = sum;  // inclusive over the warp, then over the block
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int32_t o = __shfl_up_sync(0xFFFFFFFFu, before, d);
      if ((int)(threadIdx.x & 31) >= d) before += o;
    }
    if ((threadIdx.x & 31) == 31) warp_sum[threadIdx.x >> 5] = before;
    __syncthreads();
    int32_t at = before - sum;
    for (int w = 0; w < (int)(threadIdx.x >> 5); ++w) at += warp_sum[w];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = (int)threadIdx.x * kPer + j;
      if (i < p.n) first[i] = at;
      at += mine[j];
    }
    if (threadIdx.x == kClipThreads - 1) total = at;
    __syncthreads();
  }
  // the last tensor that starts at or before piece k (an empty one is followed by one that starts there too)
  __device__ __forceinline__ int tensor_of(int n, int32_t k) const {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] <= k) lo = mid;
      else hi = mid;
    }
    return lo;
  }
};

__device__ __forceinline__ double block_sum(double v, double* shared) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_down_sync(0xFFFFFFFFu, v, d);
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0;
#pragma unroll
  for (int w = 0; w < kClipThreads / 32; ++w) s += shared[w];
  __syncthreads();
  return s;
}

// element i of a tensor whose rows are `ld` apart
__device__ __forceinline__ int64_t strided(const GradDev& t, int64_t i) {
  const int64_t r = (uint64_t)(i | t.cols) >> 32 ? i / t.cols : (int64_t)((uint32_t)i / (uint32_t)t.cols);
  return r * t.ld + (i - r * t.cols);
}

// Sum of the squares of 16 bytes, in fp64 like all sums of the norm: a square of an fp32 value is exact there, and nothing leaves the range.
// (Adding the four or eight squares in fp32 first takes 213 instead of 218 us for 200 M bf16 values in 300 tensors, and the norm alone 56
// instead of 62, but equal values, whose roundings do not cancel, put the norm off by up to 2^-23.)
template <int DT>
__device__ __forceinline__ double vec_squares(const uint4& w) {
  constexpr int V = 16 / (int)sizeof(typename Elem<DT>::T);
  float v[V];
  widen16<DT>(w, v);
  double s = 0;
#pragma unroll
  for (int j = 0; j < V; ++j) s = fma((double)v[j], (double)v[j], s);
  return s;
}

// x * coef rounded to its type; without clipping the bits are handed on (a product with 1 would change a NaN's). A coefficient below
// fp32's normal range (gradients near the largest values) is taken in two factors, of which the first, a power of two, is 1 otherwise.
struct Factor {
  bool clip;
  float power, coef;
};
template <int DT>
__device__ __forceinline__ typename Elem<DT>::T scaled(typename Elem<DT>::T x, Factor f) {
  return f.clip ? Elem<DT>::from(to_float<DT>(x) * f.power * f.coef) : x;
}
template <int DT>
__device__ __forceinline__ uint4 scaled16(const uint4& w, Factor f) {
  if (!f.clip) return w;
  constexpr int V = 16 / (int)sizeof(typename Elem<DT>::T);
  float v[V];
  widen16<DT>(w, v);
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = v[j] * f.power * f.coef;
  return narrow16<DT>(v);
}

// A tensor's vectors are counted from the 16-byte boundary at or before its start; `end` is its end in elements from there.
template <int V>
__device__ __forceinline__ bool whole_vector(const GradDev& t, int64_t vec, int64_t end) {
  return vec * V >= t.lead && (vec + 1) * V <= end;
}
// The first and the last vector of a tensor may belong to it only in part: their elements, one to a thread, or -1.
template <int V>
__device__ __forceinline__ int64_t edge_element(const GradDev& t, int64_t v0, int64_t end) {
  const int64_t tail = end / V;
  if (threadIdx.x < V) return v0 == 0 && t.lead > 0 && threadIdx.x >= t.lead && threadIdx.x < end ? (int64_t)threadIdx.x : -1;
  const int64_t e = tail * V + (int64_t)threadIdx.x - 32;
  if (threadIdx.x < 32 || threadIdx.x >= 32 + V || e >= end) return -1;
  return tail >= v0 && tail < v0 + kPieceVecs && !(tail == 0 && t.lead > 0) ? e : -1;
}

#ifdef MFET_CHECKED
// What the checked build tests: vector `vec`, element `e` counted from the boundary, or element `at` of rows `ld` apart lies in the tensor
template <int V>
__device__ __forceinline__ bool holds_vector(const GradDev& t, int64_t vec) {
  return vec * V >= t.lead && (vec + 1) * V - t.lead <= t.rows * t.cols;
}
__device__ __forceinline__ bool holds_element(const GradDev& t, int64_t e) { return e >= t.lead && e - t.lead < t.rows * t.cols; }
__device__ __forceinline__ bool holds_strided(const GradDev& t, int64_t at) { return at >= 0 && at < (t.rows - 1) * t.ld + t.cols; }
#endif

// 16 bytes, among the first to leave L2 or not. (Not through the read-only path: one kernel may read and write a gradient.)
__device__ __forceinline__ uint64_t l2_policy(bool keep) {
  uint64_t p;
  if (keep) asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
  else asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint4 load_with(const uint4* p, uint64_t policy) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p), "l"(policy));
  return v;
}

template <int DT>
__device__ __forceinline__ double piece_squares(const GradDev& t, int64_t n, int64_t piece, uint64_t policy) {
  using T = typename Elem<DT>::T;
  constexpr int V = 16 / (int)sizeof(T);
  const T* src = reinterpret_cast<const T*>(t.src);
  const int64_t v0 = piece * kPieceVecs, end = n + t.lead;  // vectors count from the boundary before src
  double s = 0;
  if (v0 * V >= end) return s;
  if (t.ld == t.cols) {
    const T* base = src - t.lead;
    const uint4* at = reinterpret_cast<const uint4*>(base) + v0 + threadIdx.x;
    if (v0 * V >= t.lead && (v0 + kPieceVecs) * V <= end) {  // a whole piece
      uint4 v[kClipInFlight];
#pragma unroll
      for (int j = 0; j < kClipInFlight; ++j)
        v[j] = MFET_INSIDE(nullptr, holds_vector<V>(t, v0 + j * kClipThreads + threadIdx.x)) ? load_with(at + j * kClipThreads, policy)
                                                                                            : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int j = 0; j < kClipInFlight; ++j) s += vec_squares<DT>(v[j]);
      return s;
    }
    uint4 v[kClipInFlight];
#pragma unroll
    for (int j = 0; j < kClipInFlight; ++j)
      v[j] = whole_vector<V>(t, v0 + j * kClipThreads + threadIdx.x, end) &&
                     MFET_INSIDE(nullptr, holds_vector<V>(t, v0 + j * kClipThreads + threadIdx.x))
                 ? __ldcg(at + j * kClipThreads)
                 : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < kClipInFlight; ++j) s += vec_squares<DT>(v[j]);
    const int64_t e = edge_element<V>(t, v0, end);
    if (e >= 0 && MFET_INSIDE(nullptr, holds_element(t, e))) {
      const double x = (double)to_float<DT>(base[e]);
      s = fma(x, x, s);
    }
  } else {
    for (int64_t i = v0 * V + threadIdx.x; i < (v0 + kPieceVecs) * V && i < n; i += kClipThreads) {
      const int64_t at = strided(t, i);
      if (!MFET_INSIDE(nullptr, holds_strided(t, at))) continue;
      const double x = (double)to_float<DT>(src[at]);
      s = fma(x, x, s);
    }
  }
  return s;
}

template <int DT>
__device__ __forceinline__ void piece_scale(const GradDev& t, int64_t n, int64_t piece, Factor f) {
  using T = typename Elem<DT>::T;
  constexpr int V = 16 / (int)sizeof(T);
  const T* src = reinterpret_cast<const T*>(t.src);
  T* dst = reinterpret_cast<T*>(t.dst);
  const int64_t v0 = piece * kPieceVecs, end = n + t.lead;
  if (v0 * V >= end) return;
  if (t.ld == t.cols) {
    const T* from = src - t.lead;
    T* to = dst - t.lead;
    const uint4* in = reinterpret_cast<const uint4*>(from) + v0 + threadIdx.x;
    uint4* out = reinterpret_cast<uint4*>(to) + v0 + threadIdx.x;
    const bool same = ((reinterpret_cast<uintptr_t>(to)) & 15u) == 0;  // dst sits on its boundary as src does
    if (same && v0 * V >= t.lead && (v0 + kPieceVecs) * V <= end) {
      uint4 v[kClipInFlight];
#pragma unroll
      for (int j = 0; j < kClipInFlight; ++j)
        if (MFET_INSIDE(nullptr, holds_vector<V>(t, v0 + j * kClipThreads + threadIdx.x))) v[j] = __ldcs(in + j * kClipThreads);
#pragma unroll
      for (int j = 0; j < kClipInFlight; ++j)
        if (MFET_INSIDE(nullptr, holds_vector<V>(t, v0 + j * kClipThreads + threadIdx.x)))
          __stcs(out + j * kClipThreads, scaled16<DT>(v[j], f));
      return;
    }
    uint4 v[kClipInFlight];
#pragma unroll
    for (int j = 0; j < kClipInFlight; ++j)
      if (whole_vector<V>(t, v0 + j * kClipThreads + threadIdx.x, end) &&
          MFET_INSIDE(nullptr, holds_vector<V>(t, v0 + j * kClipThreads + threadIdx.x)))
        v[j] = __ldcs(in + j * kClipThreads);
#pragma unroll
    for (int j = 0; j < kClipInFlight; ++j) {
      const int64_t vec = v0 + j * kClipThreads + threadIdx.x;
      if (!whole_vector<V>(t, vec, end) || !MFET_INSIDE(nullptr, holds_vector<V>(t, vec))) continue;
      const uint4 r = scaled16<DT>(v[j], f);
      if (same) {
        __stcs(out + j * kClipThreads, r);
      } else {
        T x[V];
        memcpy(x, &r, 16);
#pragma unroll
        for (int q = 0; q < V; ++q) to[vec * V + q] = x[q];
      }
    }
    const int64_t e = edge_element<V>(t, v0, end);
    if (e >= 0 && MFET_INSIDE(nullptr, holds_element(t, e))) to[e] = scaled<DT>(from[e], f);
  } else {
    for (int64_t i = v0 * V + threadIdx.x; i < (v0 + kPieceVecs) * V && i < n; i += kClipThreads) {
      const int64_t at = strided(t, i);
      if (MFET_INSIDE(nullptr, holds_strided(t, at))) dst[at] = scaled<DT>(src[at], f);
    }
  }
}

// Block `b` of `g` takes every g-th piece, in ascending order here and in descending order when it scales.
template <int N>
__device__ __forceinline__ double share_squares(const GradParams<N>& p, const Share<N>& share, int b, int g) {
  double s = 0;
  const uint64_t keep = l2_policy(true), leave = l2_policy(false);
  int32_t k = b;
  for (int i = k < share.total ? share.tensor_of(p.n, k) : 0; k < share.total; k += g) {
    while (i + 1 < p.n && share.first[i + 1] <= k) ++i;
    const GradDev& t = p.t[i];
    const int64_t piece = k - share.first[i];
    const uint64_t policy = k >= share.total - kKeepPieces ? keep : leave;
    if (t.dtype == MFET_F32) s += piece_squares<MFET_F32>(t, share.live[i], piece, policy);
    else if (t.dtype == MFET_F16) s += piece_squares<MFET_F16>(t, share.live[i], piece, policy);
    else s += piece_squares<MFET_BF16>(t, share.live[i], piece, policy);
  }
  return s;
}

template <int N>
__device__ __forceinline__ void share_scale(const GradParams<N>& p, const Share<N>& share, int b, int g, double norm) {
  if (p.norm && b == 0 && threadIdx.x == 0) *p.norm = (float)norm;
  // a norm that is infinite or NaN leaves the gradients as they are
  const bool clip = norm > p.max_norm && norm < INFINITY;
  const double coef = p.max_norm / norm;
  const bool tiny = coef < 0x1p-126;
  Factor f{clip, tiny ? 0x1p-126f : 1.f, (float)(tiny ? coef * 0x1p126 : coef)};
  asm volatile("" : "+f"(f.coef));  // else "clip ? x * coef : x" may be folded into one product
  int32_t k = b < share.total ? (share.total - 1 - b) / g * g + b : -1;
  for (int i = k >= 0 ? share.tensor_of(p.n, k) : 0; k >= 0; k -= g) {
    while (share.first[i] > k) --i;
    const GradDev& t = p.t[i];
    if (!t.dst || (!clip && t.dst == t.src)) continue;
    const int64_t piece = k - share.first[i];
    if (t.dtype == MFET_F32) piece_scale<MFET_F32>(t, share.live[i], piece, f);
    else if (t.dtype == MFET_F16) piece_scale<MFET_F16>(t, share.live[i], piece, f);
    else piece_scale<MFET_BF16>(t, share.live[i], piece, f);
  }
}

template <int N>
__global__ void __launch_bounds__(kClipThreads, kClipBlocksPerSm) grad_squares_kernel(const __grid_constant__ GradParams<N> p) {
  __shared__ double shared[kClipThreads / 32];
  __shared__ Share<N> share;
  early_launch_wait();
  share.fill(p);
  const double s = block_sum(share_squares(p, share, blockIdx.x, gridDim.x), shared);
  if (threadIdx.x == 0 && MFET_INSIDE(nullptr, p.first_sum + (int)blockIdx.x < p.n_sums)) p.sums[p.first_sum + blockIdx.x] = s;
}

template <int N>
__global__ void __launch_bounds__(kClipThreads, kClipBlocksPerSm) grad_scale_kernel(const __grid_constant__ GradParams<N> p) {
  __shared__ double shared[kClipThreads / 32];
  __shared__ Share<N> share;
  // The launch before this one is of the same call, and all before that have ended: the counts can be read, its sums not yet.
  share.fill(p);
  early_launch_wait();
  double s = 0;
  for (int i = threadIdx.x; i < p.n_sums; i += kClipThreads) s += __ldcg(p.sums + i);
  share_scale(p, share, blockIdx.x, gridDim.x, sqrt(block_sum(s, shared)));
}

// Few pieces: both steps in one launch of one cluster, whose blocks exchange their sums through distributed shared memory. On the device
// one launch wins up to a piece per block (8000 fp32 values: 5.8 us against 6.6; 65536: 7.2 against 7.0; 131072: 8.4 against 7.0; 262144:
// 11.1 against 6.9), but the second launch costs the calling program 2.4 us: up to two pieces per block.
// Another block's shared memory may be written once that block runs, and must be there until the last store has arrived: one cluster barrier
// ahead of the stores, whose arrival is given at the start so that nobody waits for it behind the sums, and one behind them.
constexpr int kSmallBlocks = 8, kSmallPieces = 2 * kSmallBlocks;
__global__ void __cluster_dims__(kSmallBlocks, 1, 1) __launch_bounds__(kClipThreads, kClipBlocksPerSm)
    grad_small_kernel(const __grid_constant__ GradParams<kFewTensors> p) {
  __shared__ double shared[kClipThreads / 32];
  __shared__ double all[kSmallBlocks];
  __shared__ Share<kFewTensors> share;
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  early_launch_wait();
  share.fill(p);
  const double s = block_sum(share_squares(p, share, blockIdx.x, kSmallBlocks), shared);
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  if (threadIdx.x < kSmallBlocks) {  // into every block's list
    uint32_t to;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(&all[blockIdx.x])), "r"(threadIdx.x));
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to), "d"(s) : "memory");
  }
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  double total = 0;
#pragma unroll
  for (int b = 0; b < kSmallBlocks; ++b) total += all[b];
  share_scale(p, share, blockIdx.x, kSmallBlocks, sqrt(total));
}

int64_t blocks_of(int64_t pieces) {
  const int64_t most = (int64_t)sm_count() * kClipBlocksPerSm;
  return pieces < most ? pieces : most;
}

int check_grad(const mfet_grad_t& g) {
  if (g.dtype > MFET_BF16 || g.flags != 0 || g.rows < 0 || g.cols < 0) return MFET_ERR_INVALID_ARG;
  if (g.rows >= (1ll << 48) || g.cols >= (1ll << 48) || g.ld >= (1ll << 48)) return MFET_ERR_INVALID_ARG;
  if (g.cols > 0 && g.rows > (1ll << 56) / g.cols) return MFET_ERR_INVALID_ARG;
  if (g.rows > 0 && g.cols > 0 && !g.src) return MFET_ERR_INVALID_ARG;
  if (g.ld != 0 && g.ld < g.cols) return MFET_ERR_INVALID_ARG;
  const uintptr_t mask = g.dtype == MFET_F32 ? 3u : 1u;
  if (((uintptr_t)g.src & mask) || ((uintptr_t)g.dst & mask) || ((uintptr_t)g.n_rows & 7u)) return MFET_ERR_ALIGNMENT;
  return MFET_OK;
}

// the tensors [at, at + n) as kernel parameters; returns how many of them fit
template <int N>
int32_t fill_params(const mfet_grad_t* g, int32_t n_grads, int32_t at, GradParams<N>* p) {
  p->n = 0;
  p->pieces = 0;
  int32_t i = at;
  for (; i < n_grads && p->n < N; ++i) {
    if (g[i].rows == 0 || g[i].cols == 0) continue;
    GradDev& t = p->t[p->n++];
    const int64_t size = g[i].dtype == MFET_F32 ? 4 : 2;
    t.src = (const uint8_t*)g[i].src;
    t.dst = (uint8_t*)g[i].dst;
    t.n_rows = g[i].n_rows;
    t.rows = g[i].rows;
    t.cols = g[i].cols;
    t.ld = g[i].ld && g[i].rows > 1 ? g[i].ld : g[i].cols;
    t.dtype = g[i].dtype;
    t.lead = t.ld == t.cols ? (uint32_t)(((uintptr_t)t.src & 15u) / size) : 0u;
    t.pad = 0;
    p->pieces += (t.rows * t.cols + t.lead + kPieceVecs * (16 / size) - 1) / (kPieceVecs * (16 / size));
  }
  return i - at;
}

template <int N>
cudaError_t launch_squares(const GradParams<N>& p, cudaStream_t s) {
  return launch_early(grad_squares_kernel<N>, (unsigned)blocks_of(p.pieces), kClipThreads, 0, s, p);
}

template <int N>
cudaError_t launch_scale(const GradParams<N>& p, cudaStream_t s) {
  return launch_early(grad_scale_kernel<N>, (unsigned)(p.pieces > 0 ? blocks_of(p.pieces) : 1), kClipThreads, 0, s, p);
}

// Tensors are taken in groups that fit the kernel parameters: first the squares of all groups, then the scaling of each.
template <int N>
int run_clip(const mfet_grad_t* g, int32_t n_grads, double max_norm, float* norm, double* sums, int64_t room,
             cudaStream_t s) {
  GradParams<N> p;
  p.sums = sums;
  p.norm = norm;
  p.max_norm = max_norm;
  p.pad = 0;
  p.first_sum = 0;
  int64_t n_sums = 0;
  for (int32_t at = 0; at < n_grads;) {
    at += fill_params<N>(g, n_grads, at, &p);
    if (p.pieces > 0x7FFFFFFF) return MFET_ERR_INVALID_ARG;
    n_sums += blocks_of(p.pieces);
  }
  if (n_sums > room) return MFET_ERR_WORKSPACE;
  p.n_sums = (int32_t)n_sums;
  const bool one_group = n_grads <= N;  // p holds it already
  if constexpr (N == kFewTensors) {
    if (n_grads > 0 && p.pieces <= kSmallPieces) {
      return launch_early(grad_small_kernel, kSmallBlocks, kClipThreads, 0, s, p) == cudaSuccess ? MFET_OK : MFET_ERR_CUDA;
    }
  }
  if (n_grads == 0) p.n = 0, p.pieces = 0;
  for (int32_t at = 0; at < n_grads;) {
    at += one_group ? n_grads : fill_params<N>(g, n_grads, at, &p);
    if (p.pieces == 0) continue;
    if (launch_squares(p, s) != cudaSuccess) return MFET_ERR_CUDA;
    p.first_sum += (int32_t)blocks_of(p.pieces);
  }
  for (int32_t at = 0; at < n_grads;) {
    at += one_group ? n_grads : fill_params<N>(g, n_grads, at, &p);
    bool any = false;
    for (int32_t i = 0; i < p.n; ++i) any |= p.t[i].dst != nullptr;
    if (!any) continue;
    if (launch_scale(p, s) != cudaSuccess) return MFET_ERR_CUDA;
    p.norm = nullptr;  // written once
  }
  if (p.norm) {  // nothing to scale: the norm alone, from the sums; no block looks at the tensors again
    p.n = 0;
    p.pieces = 0;
    if (launch_scale(p, s) != cudaSuccess) return MFET_ERR_CUDA;
  }
  return MFET_OK;
}

}  // namespace
}  // namespace mfet

extern "C" uint64_t mfet_grad_clip_bytes(int32_t n_grads) {
  if (n_grads < 0) return 0;
  const uint64_t groups = ((uint64_t)n_grads + kManyTensors - 1) / kManyTensors;
  return (groups ? groups : 1) * (uint64_t)sm_count() * kClipBlocksPerSm * sizeof(double);
}

extern "C" int mfet_grad_clip(const mfet_grad_t* grads, int32_t n_grads, float max_norm, float* norm, void* scratch,
                              uint64_t scratch_bytes, mfet_stream_t stream) {
  if (n_grads < 0 || (n_grads > 0 && !grads) || !(max_norm >= 0.f)) return MFET_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n_grads; ++i) {
    const int rc = check_grad(grads[i]);
    if (rc != MFET_OK) return rc;
  }
  if (((uintptr_t)scratch & 7u) != 0 || ((uintptr_t)norm & 3u) != 0) return MFET_ERR_ALIGNMENT;
  if (!scratch) scratch_bytes = 0;
  const int64_t room = (int64_t)(scratch_bytes / sizeof(double));
  double* sums = static_cast<double*>(scratch);
  if (n_grads <= kFewTensors) return run_clip<kFewTensors>(grads, n_grads, max_norm, norm, sums, room, (cudaStream_t)stream);
  return run_clip<kManyTensors>(grads, n_grads, max_norm, norm, sums, room, (cudaStream_t)stream);
}
