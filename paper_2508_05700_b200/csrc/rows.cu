// Rows of values written into a table in its own format (quantised as they are written), and rows read back.
//
// Both kernels move each byte once; a lane owns 8 neighbouring values of a row, the lanes of a row are the
// power of two that covers it (4 .. 32; wider rows take several rounds of a whole warp), and a warp keeps kRowsInFlight
// rows per lane group in flight, because the table rows are scattered and a warp has to cover their latency.
#include <cstring>

#include "lowbit.cuh"

using namespace mfet;

namespace mfet {
namespace {

constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kRowsThreads = 256;
constexpr int kRowsInFlight = 4;

struct RowsParams {
  uint8_t* table;
  uint64_t rows, stride;
  const int64_t* list;   // nullptr: row i
  int64_t n;
  const int64_t* n_dev;  // nullptr, or the number of entries on the device (at most n are used)
  uint8_t* mem;          // values in (write) or out (read)
  int64_t ld;            // elements between the rows of mem
  uint32_t* status;
  uint32_t dim, row_bytes, lanes_log2, rounds;
};

__device__ __forceinline__ int64_t live_count(const RowsParams& p) {
  if (!p.n_dev) return p.n;
  const int64_t v = *p.n_dev;
  return v < 0 ? 0 : (v < p.n ? v : p.n);
}

// Table row of list entry i; -1: no row (beyond the list, a negative entry, or one past the table, which is reported)
__device__ __forceinline__ int64_t entry(const RowsParams& p, int64_t i, int64_t n) {
  if (i >= n) return -1;
  int64_t r = p.list ? p.list[i] : i;
  if (r >= 0 && (uint64_t)r >= p.rows) {
    if (p.status) atomicOr(p.status, (uint32_t)MFET_DEV_ROW_RANGE);
    r = -1;
  }
  return r < 0 ? -1 : r;
}

// code of x in an INT4 row: clamp(rint((x - bias) / scale), 0, 15) with the quotient rounded once in double precision, as
// the synthetic generator has it. The fp32 estimate's error is below 2e-5 (a quotient up to 15 and a bit, three fp32
// roundings), so only a quotient within 1e-4 of a half-way point needs the double-precision one.
__device__ __forceinline__ uint32_t int4_code(float x, float scale, float bias, float inv) {
  float q = (x - bias) * inv;
  const float f = q - floorf(q);
  if (!(fabsf(f - 0.5f) > 1e-4f) || !(fabsf(q) < 32.f)) q = (float)rint(((double)x - (double)bias) / (double)scale);
  return (uint32_t)(int)fminf(15.f, fmaxf(0.f, rintf(q)));
}

template <int TD, int SD, bool VEC>
__global__ void __launch_bounds__(kRowsThreads) rows_write_kernel(const __grid_constant__ RowsParams p) {
  using S = typename Elem<SD>::T;
  const int64_t n = live_count(p);
  const int lane = threadIdx.x & 31;
  const int lanes = 1 << p.lanes_log2, per_warp = 32 >> p.lanes_log2;
  const int sub = lane & (lanes - 1), group = lane >> p.lanes_log2;
  const int64_t warp = ((int64_t)blockIdx.x * kRowsThreads + threadIdx.x) >> 5;
  const int64_t step = (int64_t)gridDim.x * (kRowsThreads / 32) * per_warp * kRowsInFlight;
  for (int64_t w0 = warp * per_warp * kRowsInFlight; w0 < n; w0 += step) {
    int64_t row[kRowsInFlight];
    const S* src[kRowsInFlight];
#pragma unroll
    for (int u = 0; u < kRowsInFlight; ++u) {
      const int64_t i = w0 + u * per_warp + group;
      row[u] = entry(p, i, n);
      src[u] = reinterpret_cast<const S*>(p.mem) + i * p.ld;
    }
    float lo[kRowsInFlight], hi[kRowsInFlight];  // INT4: the whole row's smallest and largest value
    if constexpr (TD == MFET_INT4) {
#pragma unroll
      for (int u = 0; u < kRowsInFlight; ++u) lo[u] = INFINITY, hi[u] = -INFINITY;
      for (uint32_t rd = 0; rd < p.rounds; ++rd) {
        const uint32_t c = rd * 32 + sub;
        Raw8<SD> raw[kRowsInFlight];
#pragma unroll
        for (int u = 0; u < kRowsInFlight; ++u)
          if (row[u] >= 0 && c * 8 < p.dim) raw[u] = load8<SD, VEC>(src[u] + c * 8, 8);
#pragma unroll
        for (int u = 0; u < kRowsInFlight; ++u)
          if (row[u] >= 0 && c * 8 < p.dim) {
            float v[8];
            widen8<SD>(raw[u], v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              // a NaN has to reach the row's scale: fminf would drop it
              lo[u] = v[j] != v[j] ? v[j] : (lo[u] != lo[u] ? lo[u] : fminf(lo[u], v[j]));
              hi[u] = fmaxf(hi[u], v[j]);
            }
          }
      }
#pragma unroll
      for (int u = 0; u < kRowsInFlight; ++u)
        for (int d = 1; d < lanes; d <<= 1) {
          const float l = __shfl_xor_sync(kAll, lo[u], d), h = __shfl_xor_sync(kAll, hi[u], d);
          lo[u] = (l != l || lo[u] != lo[u]) ? NAN : fminf(lo[u], l);
          hi[u] = fmaxf(hi[u], h);
        }
    }
    for (uint32_t rd = 0; rd < p.rounds; ++rd) {
      const uint32_t c = rd * 32 + sub;
      const int count = c * 8 < p.dim ? (int)min(8u, p.dim - c * 8) : 0;
      Raw8<SD> raw[kRowsInFlight];
#pragma unroll
      for (int u = 0; u < kRowsInFlight; ++u)
        if (row[u] >= 0 && count > 0) raw[u] = load8<SD, VEC>(src[u] + c * 8, count);
#pragma unroll
      for (int u = 0; u < kRowsInFlight; ++u) {
        const bool live = row[u] >= 0 && count > 0;
        uint8_t* out = p.table + (uint64_t)(row[u] >= 0 ? row[u] : 0) * p.stride;
        float v[8] = {};
        if (live) widen8<SD>(raw[u], v);
        if constexpr (TD == MFET_MXFP4) {
          uint32_t m = amax8(v);  // 0 where the row has ended: a short last block counts what it has
          m = max(m, __shfl_xor_sync(kAll, m, 1));
          m = max(m, __shfl_xor_sync(kAll, m, 2));
          const uint32_t b = mx_scale_byte(m);
          if (live) *reinterpret_cast<uint32_t*>(out + c * 4) = b == kMxNan ? 0u : mx_encode8(v, mx_inv_scale(b));
          // the scale bytes and the padding behind them, as words: this round's blocks are 4 lanes apart
          const int first = lane - sub;
          const uint32_t tail = (p.row_bytes - p.dim / 2) / 4, w = rd * 2 + sub;
          const uint32_t blocks = (p.dim + kMxBlock - 1) / kMxBlock;
          uint32_t word = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t s = __shfl_sync(kAll, b, first + ((4 * sub + j) * 4 & (lanes - 1)));
            if (4 * w + j < blocks) word |= s << (8 * j);
          }
          const bool last = rd + 1 == p.rounds;
          if (row[u] >= 0 && w < tail && (last || sub < 2)) *reinterpret_cast<uint32_t*>(out + p.dim / 2 + 4 * w) = word;
        } else if constexpr (TD == MFET_INT4) {
          const __half sh = __float2half_rn(__fdiv_rn(__fsub_rn(hi[u], lo[u]), 15.0f)), bh = __float2half_rn(lo[u]);
          const float scale = __half2float(sh), bias = __half2float(bh);
          const bool fine = isfinite(scale) && isfinite(bias);
          uint32_t word = 0;
          if (fine && scale > 0.f) {
            const float inv = __fdiv_rn(1.f, scale);
#pragma unroll
            for (int j = 0; j < 8; ++j) word |= int4_code(v[j], scale, bias, inv) << (4 * j);
          }
          if (live) *reinterpret_cast<uint32_t*>(out + c * 4) = word;
          const uint32_t tail = (p.row_bytes - p.dim / 2) / 4, w = rd * 32 + sub;
          // scale and bias, then zeros up to the row's end (at most 16 bytes: one round writes them all)
          if (row[u] >= 0 && rd == 0 && w < tail)
            *reinterpret_cast<uint32_t*>(out + p.dim / 2 + 4 * w) =
                w > 0 ? 0u
                      : (fine ? (uint32_t)__half_as_ushort(sh) | ((uint32_t)__half_as_ushort(bh) << 16) : 0x7E007E00u);
        } else {
          if (live) store8<TD, true>(reinterpret_cast<typename Elem<TD>::T*>(out) + c * 8, v, count);
        }
      }
    }
  }
}

template <int TD, int DD, bool VEC>
__global__ void __launch_bounds__(kRowsThreads) rows_read_kernel(const __grid_constant__ RowsParams p) {
  using D = typename Elem<DD>::T;
  const int64_t n = live_count(p);
  const int lane = threadIdx.x & 31;
  const int lanes = 1 << p.lanes_log2, per_warp = 32 >> p.lanes_log2;
  const int sub = lane & (lanes - 1), group = lane >> p.lanes_log2;
  const int64_t warp = ((int64_t)blockIdx.x * kRowsThreads + threadIdx.x) >> 5;
  const int64_t step = (int64_t)gridDim.x * (kRowsThreads / 32) * per_warp * kRowsInFlight;
  constexpr bool kCodes = TD == MFET_MXFP4 || TD == MFET_INT4;
  constexpr int kTable = kCodes ? MFET_F32 : TD;  // element type of a row that is stored plainly
  for (int64_t w0 = warp * per_warp * kRowsInFlight; w0 < n; w0 += step) {
    int64_t row[kRowsInFlight];
#pragma unroll
    for (int u = 0; u < kRowsInFlight; ++u) row[u] = entry(p, w0 + u * per_warp + group, n);
    for (uint32_t rd = 0; rd < p.rounds; ++rd) {
      const uint32_t c = rd * 32 + sub;
      const int count = c * 8 < p.dim ? (int)min(8u, p.dim - c * 8) : 0;
      uint32_t codes[kRowsInFlight], meta[kRowsInFlight];
      Raw8<kTable> raw[kRowsInFlight];
#pragma unroll
      for (int u = 0; u < kRowsInFlight; ++u) {
        codes[u] = meta[u] = 0;
        if (row[u] >= 0 && count > 0) {
          const uint8_t* at = p.table + (uint64_t)row[u] * p.stride;
          if constexpr (kCodes) {
            codes[u] = *reinterpret_cast<const uint32_t*>(at + c * 4);
            meta[u] = TD == MFET_MXFP4 ? (uint32_t)at[p.dim / 2 + c / 4] : *reinterpret_cast<const uint32_t*>(at + p.dim / 2);
          } else {
            raw[u] = load8<kTable, true>(reinterpret_cast<const typename Elem<kTable>::T*>(at) + c * 8, count);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < kRowsInFlight; ++u) {
        const int64_t i = w0 + u * per_warp + group;
        if (i >= n || count == 0) continue;
        float v[8] = {};
        if (row[u] >= 0) {
          if constexpr (TD == MFET_MXFP4) {
            mx_decode8(codes[u], mx_scale(meta[u]), v);
          } else if constexpr (TD == MFET_INT4) {
            const float2 sb = __half22float2(*reinterpret_cast<const __half2*>(&meta[u]));
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = fmaf((float)((codes[u] >> (4 * j)) & 15u), sb.x, sb.y);
          } else {
            widen8<kTable>(raw[u], v);
          }
        }
        store8<DD, VEC>(reinterpret_cast<D*>(p.mem) + i * p.ld + c * 8, v, count);
      }
    }
  }
}

// the narrowest lane group that covers a row, and how many rounds a wider row takes
void lanes_of(uint32_t dim, RowsParams* p) {
  const uint32_t chunks = (dim + 31) / 32 * 4;  // whole blocks of 32 values
  uint32_t l = 2;
  while ((1u << l) < chunks && l < 5) ++l;
  p->lanes_log2 = l;
  p->rounds = (chunks + (1u << l) - 1) >> l;
}

int check(const mfet_table_desc_t* d, const int64_t* list, int64_t n, const void* mem, uint32_t mem_dtype, int64_t ld,
          RowsParams* p) {
  if (!d || !d->data || d->rows == 0 || d->rows >= (1ULL << 63) || d->dim == 0 || d->flags != 0) return MFET_ERR_INVALID_ARG;
  if (d->dtype > MFET_MXFP4 || d->location != MFET_LOC_DEVICE || mem_dtype > MFET_BF16) return MFET_ERR_INVALID_ARG;
  if (n < 0 || n >= (1ll << 56) || (n > 0 && !mem)) return MFET_ERR_INVALID_ARG;
  if (d->dtype >= MFET_INT4 && d->dim % 8u != 0) return MFET_ERR_UNSUPPORTED_DIM;
  const uint64_t rb = mfet_row_bytes(d->dim, d->dtype);
  if (rb == 0 || rb % 16 != 0 || rb > 0x7FFFFFFFull) return MFET_ERR_UNSUPPORTED_DIM;
  const uint64_t stride = d->row_stride_bytes ? d->row_stride_bytes : rb;
  if (stride < rb || d->rows > 0xFFFFFFFFFFFFFFFFULL / stride) return MFET_ERR_INVALID_ARG;
  if (stride % 16 != 0 || ((uintptr_t)d->data & 15u) != 0) return MFET_ERR_ALIGNMENT;
  if (ld < (int64_t)d->dim || ld >= (1ll << 40)) return MFET_ERR_INVALID_ARG;
  if (((uintptr_t)mem & (mem_dtype == MFET_F32 ? 3u : 1u)) != 0) return MFET_ERR_ALIGNMENT;
  std::memset(p, 0, sizeof(*p));
  p->table = static_cast<uint8_t*>(d->data);
  p->rows = d->rows;
  p->stride = stride;
  p->list = list;
  p->n = n;
  p->mem = static_cast<uint8_t*>(const_cast<void*>(mem));
  p->ld = ld;
  p->dim = d->dim;
  p->row_bytes = (uint32_t)rb;
  lanes_of(d->dim, p);
  return MFET_OK;
}

// 16-byte pieces of the value rows can be used when every row starts on a 16-byte boundary
bool vectors(const RowsParams& p, uint32_t dtype) {
  return (reinterpret_cast<uintptr_t>(p.mem) & 15u) == 0 && (p.ld * (dtype == MFET_F32 ? 4 : 2)) % 16 == 0;
}

unsigned blocks_for(const RowsParams& p) {
  const int64_t per_block = (int64_t)(kRowsThreads >> p.lanes_log2) * kRowsInFlight;
  const int64_t want = (p.n + per_block - 1) / per_block, most = (int64_t)sm_count() * 16;
  return (unsigned)(want < most ? want : most);
}

template <int TD, int MD>
cudaError_t launch_one(const RowsParams& p, bool write, cudaStream_t s) {
  const unsigned b = blocks_for(p);
  const bool vec = vectors(p, MD);
  if (write) {
    if (vec) rows_write_kernel<TD, MD, true><<<b, kRowsThreads, 0, s>>>(p);
    else rows_write_kernel<TD, MD, false><<<b, kRowsThreads, 0, s>>>(p);
  } else {
    if (vec) rows_read_kernel<TD, MD, true><<<b, kRowsThreads, 0, s>>>(p);
    else rows_read_kernel<TD, MD, false><<<b, kRowsThreads, 0, s>>>(p);
  }
  return cudaGetLastError();
}

template <int TD>
cudaError_t launch_td(const RowsParams& p, uint32_t mem_dtype, bool write, cudaStream_t s) {
  switch (mem_dtype) {
    case MFET_F32: return launch_one<TD, MFET_F32>(p, write, s);
    case MFET_F16: return launch_one<TD, MFET_F16>(p, write, s);
    default: return launch_one<TD, MFET_BF16>(p, write, s);
  }
}

int run_rows(const mfet_table_desc_t* d, const int64_t* list, int64_t n, const int64_t* n_dev, const void* mem,
             uint32_t mem_dtype, int64_t ld, uint32_t* status, bool write, mfet_stream_t stream) {
  RowsParams p;
  const int rc = check(d, list, n, mem, mem_dtype, ld, &p);
  if (rc != MFET_OK) return rc;
  if (n == 0) return MFET_OK;
  p.n_dev = n_dev;
  p.status = status;
  cudaStream_t s = (cudaStream_t)stream;
  cudaError_t e;
  switch (d->dtype) {
    case MFET_F32: e = launch_td<MFET_F32>(p, mem_dtype, write, s); break;
    case MFET_F16: e = launch_td<MFET_F16>(p, mem_dtype, write, s); break;
    case MFET_BF16: e = launch_td<MFET_BF16>(p, mem_dtype, write, s); break;
    case MFET_INT4: e = launch_td<MFET_INT4>(p, mem_dtype, write, s); break;
    default: e = launch_td<MFET_MXFP4>(p, mem_dtype, write, s); break;
  }
  return e == cudaSuccess ? MFET_OK : MFET_ERR_CUDA;
}

}  // namespace
}  // namespace mfet

extern "C" int mfet_rows_write(const mfet_table_desc_t* table, const int64_t* rows, int64_t n, const int64_t* n_dev,
                               const void* values, uint32_t dtype, int64_t ld, uint32_t* status, mfet_stream_t stream) {
  return run_rows(table, rows, n, n_dev, values, dtype, ld, status, true, stream);
}

extern "C" int mfet_rows_read(const mfet_table_desc_t* table, const int64_t* rows, int64_t n, const int64_t* n_dev,
                              void* values, uint32_t dtype, int64_t ld, uint32_t* status, mfet_stream_t stream) {
  return run_rows(table, rows, n, n_dev, values, dtype, ld, status, false, stream);
}
