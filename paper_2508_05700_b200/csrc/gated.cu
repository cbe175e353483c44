// The gated linear block h = act(x Wg^T) * (x Wu^T) and its backward pass, 16-bit operands and fp32 sums.
//
// Forward, a few rows: a warp per unit (gated_few_kernel). More: one product whose columns are pairs of a gate and an up unit, the activation and the product of the two on the accumulators.
// Backward: the same product again (neither G nor U is kept between the passes; computing them costs less memory traffic than storing and
// reading them would where k is below some 1500, and no training memory), with the gradient of h beside it:
//   dG = dh * U * act'(G), dU = dh * act(G), rounded to the operands' type (the tensor cores take nothing wider), then
//   dx = dG Wg + dU Wu in one product of two segments, dWg = dG^T x and dWu = dU^T x in one launch.
#include "gemm16.cuh"

using namespace mfet;
using namespace mfet::gemm16;

namespace mfet {
namespace {

bool bad_sizes(int64_t m, int64_t n, int64_t k) {
  if (m < 0 || m >= (1ll << 31) || n < 0 || n >= (1ll << 31) || k < 1 || k >= (1ll << 30)) return true;
  // tiles are counted in 32 bits
  const int64_t a = m / 128 + 1, b = n / 64 + 1, c = k / 128 + 1;
  return a * b >= (1ll << 31) || a * c >= (1ll << 31) || 2 * b * c >= (1ll << 31);
}
bool bad_ld(int64_t ld, int64_t cols) { return ld < cols || ld >= (1ll << 31); }

struct Call {
  const void *x, *wg, *wu, *dh;
  void *h, *dx, *dwg, *dwu;
  int64_t x_ld, wg_ld, wu_ld, dh_ld, h_ld, dx_ld, dwg_ld, dwu_ld;
  int64_t m, n, k;
  uint32_t dtype, act;
  uint8_t* scratch;
  uint64_t scratch_bytes;
  uint32_t* status;
  cudaStream_t stream;
};

uint64_t grad_bytes(int64_t m, int64_t n) { return packed_bytes(m, n); }

// ------------------------------------------------------------------ a few rows, forward ----

constexpr int kFewThreads = 256;
constexpr int kFewMost = 8;                // rows of x
constexpr uint32_t kFewSmem = 96 * 1024;   // all of x in fp32 has to fit this
// The most work in multiply-adds, m counted up to a power of two: 2^25, 2^24 for 5 rows and more. (us here and on the tensor cores: 1 x 896 x 1024 3.2
// and 7.3; at the limit 4 x 2048 x 4096 13.9 and 15.0, 8 x 896 x 1024 5.3 and 7.3; beyond it 8 x 2048 x 2048 15.0 and 11.9.)
constexpr int64_t kFewWork = 1ll << 25;

struct FewParams {
  const uint8_t *x, *wg, *wu;
  uint8_t* h;
  int64_t x_ld, wg_ld, wu_ld, h_ld, n;
  const void *x_end, *wg_end, *wu_end;
  int32_t m, k;
  uint32_t act;
};

template <int DT>
__device__ __forceinline__ float gate_any(uint32_t act, float g) {
  const float2 v = make_float2(g, g);
  switch (act) {
    case MFET_ACT_RELU: return gate2<MFET_ACT_RELU, false>(v, nullptr).x;
    case MFET_ACT_SILU: return gate2<MFET_ACT_SILU, false>(v, nullptr).x;
    case MFET_ACT_GELU: return gate2<MFET_ACT_GELU, false>(v, nullptr).x;
    case MFET_ACT_SIGMOID: return gate2<MFET_ACT_SIGMOID, false>(v, nullptr).x;
    default: return g;
  }
}

// A warp per unit: its lanes read 8 values of the gate's and of the up row at a time (512 bytes of each a warp), the next ones while these are
// multiplied with the same columns of all MT rows of x, which the block has in shared memory in fp32. Bound by reading the weights (and
// by the launch): 1 x 896 x 1024, 3.7 MB of weights, 3.2 us, 7.3 on the tensor cores, whose tiles are 128 rows high.
template <int DT, int MT, bool VEC>
__global__ void __launch_bounds__(kFewThreads) gated_few_kernel(const __grid_constant__ FewParams p) {
  using T = typename Elem<DT>::T;
  extern __shared__ float4 sx[];  // [MT][2][chunks]: the halves of 8 values of a row
  early_launch_wait();
  const int lane = threadIdx.x & 31, chunks = (p.k + 255) / 256 * 32;
  const int64_t first = (int64_t)blockIdx.x * (kFewThreads / 32) + (threadIdx.x >> 5), step = (int64_t)gridDim.x * (kFewThreads / 32);
  struct Pair {
    Raw<DT, 8> g, u;
  };
  auto fetch = [&](int64_t j, int c, Pair* w) {  // chunk c of unit j; zeros behind the ends
    const int count = j < p.n ? min(8, p.k - c * 8) : 0;
    if (count > 0 && MFET_INSIDE(nullptr, c * 8 + count <= p.wg_ld && c * 8 + count <= p.wu_ld)) {
      w->g = load_any<DT, 8, VEC>(reinterpret_cast<const T*>(p.wg) + j * p.wg_ld + c * 8, count, p.wg, p.wg_end);
      w->u = load_any<DT, 8, VEC>(reinterpret_cast<const T*>(p.wu) + j * p.wu_ld + c * 8, count, p.wu, p.wu_end);
    } else {
      memset(w, 0, sizeof(*w));
    }
  };
  Pair next[2];  // the first weights do not depend on x: they are under way while it is staged
  fetch(first, lane, &next[0]);
  fetch(first, lane + 32, &next[1]);
  for (int i = threadIdx.x; i < MT * chunks; i += kFewThreads) {
    const int row = i / chunks, c = i - row * chunks;
    float v[8];
    const int count = row < p.m ? min(8, p.k - c * 8) : 0;
    if (count > 0 && MFET_INSIDE(nullptr, c * 8 + count <= p.x_ld))
      widen_raw<DT, 8>(load_any<DT, 8, VEC>(reinterpret_cast<const T*>(p.x) + row * p.x_ld + c * 8, count, p.x, p.x_end), v);
    else memset(v, 0, sizeof(v));
    sx[(row * 2) * chunks + c] = make_float4(v[0], v[1], v[2], v[3]);
    sx[(row * 2 + 1) * chunks + c] = make_float4(v[4], v[5], v[6], v[7]);
  }
  __syncthreads();
  for (int64_t j = first; j < p.n; j += step) {
    float2 g[MT], u[MT];
#pragma unroll
    for (int r = 0; r < MT; ++r) g[r] = u[r] = both(0.f);
    for (int c0 = lane; c0 < chunks; c0 += 64) {
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int c = c0 + 32 * z;
        if (c >= chunks) break;  // the same for the whole warp
        float wg[8], wu[8];
        widen_raw<DT, 8>(next[z].g, wg);
        widen_raw<DT, 8>(next[z].u, wu);
        if (c + 64 < chunks) fetch(j, c + 64, &next[z]);
        else fetch(j + step, lane + 32 * z, &next[z]);
#pragma unroll
        for (int r = 0; r < MT; ++r) {
          const float4 a = sx[(r * 2) * chunks + c], b = sx[(r * 2 + 1) * chunks + c];
          const float2 x[4] = {make_float2(a.x, a.y), make_float2(a.z, a.w), make_float2(b.x, b.y), make_float2(b.z, b.w)};
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            g[r] = fma2(x[q], make_float2(wg[2 * q], wg[2 * q + 1]), g[r]);
            u[r] = fma2(x[q], make_float2(wu[2 * q], wu[2 * q + 1]), u[r]);
          }
        }
      }
    }
    float mine_g = 0.f, mine_u = 0.f;
#pragma unroll
    for (int r = 0; r < MT; ++r) {
      float a = g[r].x + g[r].y, b = u[r].x + u[r].y;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        a += __shfl_xor_sync(kAllLanes, a, d);
        b += __shfl_xor_sync(kAllLanes, b, d);
      }
      if (lane == r) mine_g = a, mine_u = b;
    }
    if (lane < p.m && MFET_INSIDE(nullptr, j < p.h_ld))
      reinterpret_cast<T*>(p.h)[lane * p.h_ld + j] = Elem<DT>::from(gate_any<DT>(p.act, mine_g) * mine_u);
  }
}

uint32_t few_rows(int64_t m) { return m == 1 ? 1 : m == 2 ? 2 : m <= 4 ? 4 : 8; }
uint32_t few_smem(int64_t m, int64_t k) { return (uint32_t)((k + 255) / 256 * 32 * few_rows(m) * 32); }
bool few(int64_t m, int64_t n, int64_t k) {
  return m <= kFewMost && k <= kFewSmem / 4 && few_smem(m, k) <= kFewSmem && (int64_t)few_rows(m) * n <= (m <= 4 ? kFewWork : kFewWork / 2) / k;
}

template <int DT, int MT>
int launch_few(const FewParams& p, bool vec, cudaStream_t s) {
  static std::atomic<uint64_t> ready[2];
  const auto kernel = vec ? gated_few_kernel<DT, MT, true> : gated_few_kernel<DT, MT, false>;
  if (allow_smem(kernel, kFewSmem, &ready[vec]) != cudaSuccess) return MFET_ERR_CUDA;
  const int64_t want = (p.n + kFewThreads / 32 - 1) / (kFewThreads / 32), most = (int64_t)sm_count() * 4;
  return launch_early(kernel, (unsigned)(want < most ? want : most), kFewThreads, few_smem(MT, p.k), s, p) == cudaSuccess ? MFET_OK : MFET_ERR_CUDA;
}
template <int DT>
int launch_few(const FewParams& p, bool vec, cudaStream_t s) {
  switch (few_rows(p.m)) {
    case 1: return launch_few<DT, 1>(p, vec, s);
    case 2: return launch_few<DT, 2>(p, vec, s);
    case 4: return launch_few<DT, 4>(p, vec, s);
    default: return launch_few<DT, 8>(p, vec, s);
  }
}

// ------------------------------------------------------------------ products ----

template <int MODE>
int gates(const Call& c, const Matrix& x, const Matrix& wg, const Matrix& wu, const Matrix* out, int n_out, const Matrix* dh) {
  Problem q;
  q.dtype = q.out_dtype = c.dtype;
  q.a[0] = x;
  q.b[0] = wg;
  q.b[1] = wu;
  q.n_b = 2;
  q.n_out = n_out;
  for (int i = 0; i < n_out; ++i) q.out[i] = out[i];
  q.k[0] = c.k;
  q.p.part[0].m = c.m;
  q.p.part[0].n = c.n;
  q.p.act = c.act;
  q.p.status = c.status;
  if (dh) {
    q.p.c0 = dh->p;
    q.p.c_ld = dh->ld;
    q.p.c_vec = on_16(*dh, c.dtype);
  }
  return c.dtype == MFET_F16 ? run<MODE, MFET_F16>(q, c.stream) : run<MODE, MFET_BF16>(q, c.stream);
}

template <int MODE>
int out_product(Problem& q, const Call& c) {
  q.dtype = q.out_dtype = c.dtype;
  q.p.status = c.status;
  return c.dtype == MFET_F16 ? run<MODE, MFET_F16>(q, c.stream) : run<MODE, MFET_BF16>(q, c.stream);
}

// The weights' gradients are sums over the rows. The tensor cores truncate a sum once in 16 of them, by up to 2^-22 of what it holds (its 16 products
// included), so that beyond some rows it loses more than its rounding to 16 bits does: fp16 products of one sign were off by 2.1e-4 of their sum for
// 2^17 rows, 1.7e-3 for 2^20 and 6.6e-3 for 2^22 (half a step of fp16 is 4.9e-4), 64 x 64 weights in four parts of the rows. Sums over more than
// kLongRows are taken in parts of kPartRows, which are added up in fp32, to nearest: 131072 x 1024 x 896 1134 -> 1157 us, 2^20 x 64 x 64 1232 -> 1240;
// with both products in one launch 131072 x 1024 x 2048 2271 -> 2279, 66000 x 100 x 5000 770 -> 845 (922 in two launches).
constexpr int64_t kLongRows = 1ll << 16, kPartRows = 1ll << 14;

// Both products of the backward pass in one launch, where that takes less time than one after the other: blocks that have no tile of one left
// go on with the other (the backward pass of 8192 x 896 x 1024: 80 us, 84 in two launches). 1: it does not.
template <int TWO, int OF_W, int DT>
int out_products_dt(const Problem& both, const Problem& of_x, const Problem& of_w, cudaStream_t s) {
  return cost_two<TWO, DT>(both) < least_cost<kOut, DT>(of_x) + least_cost<OF_W, DT>(of_w) ? launch<2, 256, TWO, DT>(both, 1, s) : 1;
}
template <int TWO, int OF_W>
int out_products(Problem* both, Problem* of_x, Problem* of_w, const Call& c) {
  for (Problem* q : {both, of_x, of_w}) {
    q->dtype = q->out_dtype = c.dtype;
    q->p.status = c.status;
  }
  return c.dtype == MFET_F16 ? out_products_dt<TWO, OF_W, MFET_F16>(*both, *of_x, *of_w, c.stream)
                             : out_products_dt<TWO, OF_W, MFET_BF16>(*both, *of_x, *of_w, c.stream);
}

// scratch for operands whose rows do not start on 16-byte boundaries, as they are
uint64_t packing(const Matrix* x, int count) {
  uint64_t b = 0;
  for (int i = 0; i < count; ++i)
    if (!on_16(x[i], MFET_F16)) b += packed_bytes(x[i].outer, x[i].inner);
  return b;
}

}  // namespace
}  // namespace mfet

extern "C" {

uint64_t mfet_gated_linear_bytes(int64_t m, int64_t n, int64_t k) {
  if (bad_sizes(m, n, k)) return 0;
  return packed_bytes(m, k) + 2 * packed_bytes(n, k);
}

int mfet_gated_linear(const void* x, uint32_t dtype, int64_t x_ld, int64_t m, const void* w_gate, int64_t wg_ld, const void* w_up,
                      int64_t wu_ld, int64_t n, int64_t k, uint32_t act, void* h, int64_t h_ld, void* scratch, uint64_t scratch_bytes,
                      uint32_t* status, mfet_stream_t stream) {
  if ((dtype != MFET_F16 && dtype != MFET_BF16) || act > MFET_ACT_SIGMOID || bad_sizes(m, n, k) || bad_ld(x_ld, k) || bad_ld(wg_ld, k) ||
      bad_ld(wu_ld, k) || bad_ld(h_ld, n))
    return MFET_ERR_INVALID_ARG;
  if (m == 0 || n == 0) return MFET_OK;
  if (!x || !w_gate || !w_up || !h) return MFET_ERR_INVALID_ARG;
  if (!aligned(x, 2) || !aligned(w_gate, 2) || !aligned(w_up, 2) || !aligned(h, 2) || !aligned(status, 4)) return MFET_ERR_ALIGNMENT;
  Call c{};
  c.m = m, c.n = n, c.k = k;
  c.dtype = dtype, c.act = act;
  c.status = status;
  c.stream = (cudaStream_t)stream;
  Matrix in[3] = {{x, k, m, x_ld}, {w_gate, k, n, wg_ld}, {w_up, k, n, wu_ld}};
  const uint64_t need = packing(in, 3);
  if (need && (!scratch || scratch_bytes < need)) return MFET_ERR_WORKSPACE;
  if (need && !aligned(scratch, 16)) return MFET_ERR_ALIGNMENT;
  if (few(m, n, k)) {
    const bool vec = on_16(in[0], dtype) && on_16(in[1], dtype) && on_16(in[2], dtype);
    auto end = [](const Matrix& a) { return (const uint8_t*)a.p + ((a.outer - 1) * a.ld + a.inner) * 2; };
    const FewParams p{(const uint8_t*)x, (const uint8_t*)w_gate, (const uint8_t*)w_up, (uint8_t*)h, x_ld, wg_ld, wu_ld, h_ld, n,
                      end(in[0]), end(in[1]), end(in[2]), (int32_t)m, (int32_t)k, act};
    return dtype == MFET_F16 ? launch_few<MFET_F16>(p, vec, c.stream) : launch_few<MFET_BF16>(p, vec, c.stream);
  }
  if (packed(in, 3, (uint8_t*)scratch, c.stream) != cudaSuccess) return MFET_ERR_CUDA;
  const Matrix out{h, n, m, h_ld};
  return gates<kGated>(c, in[0], in[1], in[2], &out, 1, nullptr);
}

uint64_t mfet_gated_linear_backward_bytes(int64_t m, int64_t n, int64_t k) {
  if (bad_sizes(m, n, k)) return 0;
  return packed_bytes(m, k) + 2 * packed_bytes(n, k) + packed_bytes(m, n) + 2 * grad_bytes(m, n);
}

int mfet_gated_linear_backward(const void* x, uint32_t dtype, int64_t x_ld, int64_t m, const void* w_gate, int64_t wg_ld, const void* w_up,
                               int64_t wu_ld, int64_t n, int64_t k, uint32_t act, const void* dh, int64_t dh_ld, void* dx, int64_t dx_ld,
                               void* dw_gate, int64_t dwg_ld, void* dw_up, int64_t dwu_ld, void* scratch, uint64_t scratch_bytes,
                               uint32_t* status, mfet_stream_t stream) {
  if ((dtype != MFET_F16 && dtype != MFET_BF16) || act > MFET_ACT_SIGMOID || bad_sizes(m, n, k) || bad_ld(x_ld, k) || bad_ld(wg_ld, k) ||
      bad_ld(wu_ld, k) || bad_ld(dh_ld, n) || (dx && bad_ld(dx_ld, k)) || !dw_gate != !dw_up || (dw_gate && (bad_ld(dwg_ld, k) || bad_ld(dwu_ld, k))))
    return MFET_ERR_INVALID_ARG;
  if (!aligned(x, 2) || !aligned(w_gate, 2) || !aligned(w_up, 2) || !aligned(dh, 2) || !aligned(dx, 2) || !aligned(dw_gate, 2) ||
      !aligned(dw_up, 2) || !aligned(status, 4))
    return MFET_ERR_ALIGNMENT;
  Call c{};
  c.m = m, c.n = n, c.k = k;
  c.dtype = dtype, c.act = act;
  c.status = status;
  c.stream = (cudaStream_t)stream;
  if (m == 0 || n == 0) {  // sums over nothing
    if (n > 0 && dw_gate)
      if (cudaMemset2DAsync(dw_gate, dwg_ld * 2, 0, k * 2, n, c.stream) != cudaSuccess ||
          cudaMemset2DAsync(dw_up, dwu_ld * 2, 0, k * 2, n, c.stream) != cudaSuccess)
        return MFET_ERR_CUDA;
    if (m > 0 && dx)
      if (cudaMemset2DAsync(dx, dx_ld * 2, 0, k * 2, m, c.stream) != cudaSuccess) return MFET_ERR_CUDA;
    return MFET_OK;
  }
  if (!x || !w_gate || !w_up || !dh) return MFET_ERR_INVALID_ARG;
  if (!dx && !dw_gate) return MFET_OK;
  Matrix in[4] = {{x, k, m, x_ld}, {w_gate, k, n, wg_ld}, {w_up, k, n, wu_ld}, {dh, n, m, dh_ld}};
  if (!scratch || scratch_bytes < packing(in, 4) + 2 * grad_bytes(m, n)) return MFET_ERR_WORKSPACE;
  if (!aligned(scratch, 16)) return MFET_ERR_ALIGNMENT;
  uint8_t* to = (uint8_t*)scratch;
  Matrix g[2];
  for (Matrix& i : g) {
    i = {to, n, m, up8(n), true};
    to += grad_bytes(m, n);
  }
  if (packed(in, 4, to, c.stream) != cudaSuccess) return MFET_ERR_CUDA;
  int rc = gates<kGatedBack>(c, in[0], in[1], in[2], g, 2, &in[3]);
  if (rc != MFET_OK) return rc;
  Problem of_x, of_w, both;
  if (dx) {  // dG Wg + dU Wu
    Problem& q = of_x;
    q.a[0] = g[0], q.a[1] = g[1], q.n_a = 2;
    q.b[0] = in[1], q.b[1] = in[2], q.n_b = 2, q.b_mn = 3;
    q.out[0] = {dx, k, m, dx_ld};
    q.k[0] = n, q.segs[0] = 2;
    q.p.part[0].seg_a = q.p.part[0].seg_b = 0x10;
    q.p.part[0].b_mn = 1;
    q.p.part[0].m = m, q.p.part[0].n = k;
  }
  if (dw_gate) {  // dG^T x, dU^T x
    Problem& q = of_w;
    q.a[0] = g[0], q.a[1] = g[1], q.n_a = 2, q.a_mn = 3;
    q.b[0] = in[0], q.b_mn = 1;
    q.out[0] = {dw_gate, k, n, dwg_ld};
    q.out[1] = {dw_up, k, n, dwu_ld};
    q.n_out = q.results[0] = 2;
    q.k[0] = m;
    q.p.part[0].a_mn = q.p.part[0].b_mn = 1;
    q.p.part[0].m = n, q.p.part[0].n = k;
  }
  const bool long_sum = m > kLongRows;
  of_w.p.part_kb = kPartRows / kSlab;
  if (dx && dw_gate && (!long_sum || n <= kPartRows)) {
    both = of_w;
    both.a[2] = g[0], both.a[3] = g[1], both.n_a = 4;
    both.b[1] = in[1], both.b[2] = in[2], both.n_b = 3, both.b_mn = 7;
    both.out[2] = of_x.out[0], both.n_out = 3;
    both.k[1] = n, both.segs[1] = 2, both.results[1] = 1;
    both.p.part[1] = of_x.p.part[0];
    both.p.part[1].seg_a = 0x32, both.p.part[1].seg_b = 0x21, both.p.part[1].out = 2;
    rc = long_sum ? out_products<kOutTwoLong, kOutLong>(&both, &of_x, &of_w, c) : out_products<kOutTwo, kOut>(&both, &of_x, &of_w, c);
    if (rc <= 0) return rc;
  }
  rc = dx ? out_product<kOut>(of_x, c) : MFET_OK;
  if (rc == MFET_OK && dw_gate) rc = long_sum ? out_product<kOutLong>(of_w, c) : out_product<kOut>(of_w, c);
  return rc;
}

}  // extern "C"
