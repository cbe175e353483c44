// The gated linear block h = act(x Wg^T) * (x Wu^T) and its backward pass, 16-bit operands and fp32 sums.
//
// Forward: one product whose columns are pairs of a gate and an up unit, the activation and the product of the two on the accumulators.
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

int out_product(Problem& q, const Call& c) {
  q.dtype = q.out_dtype = c.dtype;
  q.p.status = c.status;
  return c.dtype == MFET_F16 ? run<kOut, MFET_F16>(q, c.stream) : run<kOut, MFET_BF16>(q, c.stream);
}

// Both products of the backward pass in one launch, where that takes less time than one after the other: blocks that have no tile of one left
// go on with the other (8192 x 896 x 1024: 48 us, 58 in two launches). 1: it does not.
template <int DT>
int out_products_dt(const Problem& both, const Problem& of_x, const Problem& of_w, cudaStream_t s) {
  return cost_two<DT>(both) < least_cost<kOut, DT>(of_x) + least_cost<kOut, DT>(of_w) ? launch<2, 256, kOutTwo, DT>(both, 1, s) : 1;
}
int out_products(Problem* both, Problem* of_x, Problem* of_w, const Call& c) {
  for (Problem* q : {both, of_x, of_w}) {
    q->dtype = q->out_dtype = c.dtype;
    q->p.status = c.status;
  }
  return c.dtype == MFET_F16 ? out_products_dt<MFET_F16>(*both, *of_x, *of_w, c.stream) : out_products_dt<MFET_BF16>(*both, *of_x, *of_w, c.stream);
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
  if (dx && dw_gate) {
    both = of_w;
    both.a[2] = g[0], both.a[3] = g[1], both.n_a = 4;
    both.b[1] = in[1], both.b[2] = in[2], both.n_b = 3, both.b_mn = 7;
    both.out[2] = of_x.out[0], both.n_out = 3;
    both.k[1] = n, both.segs[1] = 2, both.results[1] = 1;
    both.p.part[1] = of_x.p.part[0];
    both.p.part[1].seg_a = 0x32, both.p.part[1].seg_b = 0x21, both.p.part[1].out = 2;
    rc = out_products(&both, &of_x, &of_w, c);
    if (rc <= 0) return rc;
  }
  rc = dx ? out_product(of_x, c) : MFET_OK;
  if (rc == MFET_OK && dw_gate) rc = out_product(of_w, c);
  return rc;
}

}  // extern "C"
