// Rows of values written into a table in its own format (quantised as they are written), and rows read back.
//
// Both kernels move each byte once. A lane owns 32 bytes of a row of values (8 fp32 or 16 16-bit values), the lanes of a row are the
// power of two that covers it (wider rows take several rounds of a whole warp), and a lane group works on kRowsInFlight rows at a
// time, the list entries of the next ones under way: the table rows are scattered, and what the kernels wait for is their
// latency. 2 M rows of 64 bf16 values into an 8 M-row MXFP4 table and 4 M rows read from it: 338 us for 1.52 GB of DRAM traffic (4.5 TB/s; the
// read alone 5.2): a 48-byte row costs 128 to 160 bytes of DRAM reads. 37 k rows of 128 fp32 values written and 74 k read:
// 19 us, a few dependent loads per launch. More rows in flight or more blocks changed that by 4 % at most, and a whole block of 32 values
// per lane made it slower (404 instead of 358 us, 30 instead of 19.5).
#include <cstring>

#include "lowbit.cuh"

using namespace mfet;

namespace mfet {
namespace {

constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kRowsThreads = 256;
constexpr int kRowsInFlight = 2;   // rows that a lane group writes at a time
constexpr int kRowsReadAhead = 4;  // ... and reads: a row of codes takes fewer registers
constexpr int kRowsBlocksPerSm = 4;

struct RowsParams {
  uint8_t* table;
  uint64_t rows, stride;
  const int64_t* list;   // nullptr: row i
  int64_t n;
  const int64_t* n_dev;  // nullptr, or the number of entries on the device (at most n are used)
  uint8_t* mem;          // values in (write) or out (read)
  const uint8_t* mem_end;
  int64_t ld;            // elements between the rows of mem
  uint32_t* status;
  uint32_t dim, row_bytes, lanes_log2, rounds;
  bool wide;             // every row of mem starts on a 32-byte boundary
};

__device__ __forceinline__ int64_t live_count(const RowsParams& p) {
  if (!p.n_dev) return p.n;
  const int64_t v = *p.n_dev;
  return v < 0 ? 0 : (v < p.n ? v : p.n);
}

// Entry i of the list; -1 beyond its end
__device__ __forceinline__ int64_t entry(const RowsParams& p, int64_t i, int64_t n) {
  return i < n && MFET_INSIDE(p.status, i >= 0 && i < p.n) ? (p.list ? __ldg(reinterpret_cast<const long long*>(p.list) + i) : i) : -1;
}
#ifdef MFET_CHECKED
// What the checked build tests: `count` values from column `at` of value row i, or bytes [from, to) of a table row
__device__ __forceinline__ bool holds_values(const RowsParams& p, int64_t i, uint32_t at, int count) {
  return i >= 0 && i < p.n && (uint64_t)at + count <= p.dim;
}
__device__ __forceinline__ bool holds_bytes(const RowsParams& p, int64_t r, uint64_t from, uint64_t to) {
  return (uint64_t)r < p.rows && from <= to && to <= p.row_bytes;
}
#endif
// The table row that an entry names, or -1: a negative entry, or one past the table, which is reported
__device__ __forceinline__ int64_t checked(const RowsParams& p, int64_t r) {
  if (r < 0) return -1;
  if ((uint64_t)r < p.rows) return r;
  if (p.status) atomicOr(p.status, (uint32_t)MFET_DEV_ROW_RANGE);
  return -1;
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
__global__ void __launch_bounds__(kRowsThreads, kRowsBlocksPerSm) rows_write_kernel(const __grid_constant__ RowsParams p) {
  using S = typename Elem<SD>::T;
  constexpr int E = 32 / (int)sizeof(S), LPB = kMxBlock / E;  // values per lane, lanes per block of 32
  constexpr int U = kRowsInFlight;
  early_launch_wait();
  const int64_t n = live_count(p);
  const int lane = threadIdx.x & 31;
  const int lanes = 1 << p.lanes_log2, per_warp = 32 >> p.lanes_log2;
  const int sub = lane & (lanes - 1), group = lane >> p.lanes_log2;
  const int64_t step = (int64_t)gridDim.x * (kRowsThreads / 32) * per_warp * U;
  const uint32_t rounds = p.rounds;
  int64_t w0 = (((int64_t)blockIdx.x * kRowsThreads + threadIdx.x) >> 5) * per_warp * U;
  int64_t next[U];
#pragma unroll
  for (int u = 0; u < U; ++u) next[u] = entry(p, w0 + u * per_warp + group, n);
  for (; w0 < n; w0 += step) {
    int64_t row[U];
    const S* src[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = w0 + u * per_warp + group;
      row[u] = next[u];
      next[u] = entry(p, i + step, n);
      src[u] = reinterpret_cast<const S*>(p.mem) + (i < n ? i : 0) * p.ld;
    }
    float lo[U], hi[U];  // INT4: the whole row's smallest and largest value
    if constexpr (TD == MFET_INT4) {
#pragma unroll
      for (int u = 0; u < U; ++u) lo[u] = INFINITY, hi[u] = -INFINITY;
      for (uint32_t rd = 0; rd < rounds; ++rd) {
        const uint32_t at = (rd * 32 + sub) * E;
        const int count = at < p.dim ? (int)min((uint32_t)E, p.dim - at) : 0;
        Raw<SD, E> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (count > 0 && MFET_INSIDE(p.status, holds_values(p, (src[u] - reinterpret_cast<const S*>(p.mem)) / p.ld, at, count)))
            raw[u] = load_any<SD, E, VEC>(src[u] + at, count, p.mem, p.mem_end, p.wide);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (count > 0) {
            float v[E];
            widen_raw<SD, E>(raw[u], v);
#pragma unroll
            for (int j = 0; j < E; ++j)
              if (j < count) {
                // a NaN has to reach the row's scale: fminf would drop it
                lo[u] = v[j] != v[j] ? v[j] : (lo[u] != lo[u] ? lo[u] : fminf(lo[u], v[j]));
                hi[u] = fmaxf(hi[u], v[j]);
              }
          }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        for (int d = 1; d < lanes; d <<= 1) {
          const float l = __shfl_xor_sync(kAll, lo[u], d), h = __shfl_xor_sync(kAll, hi[u], d);
          lo[u] = (l != l || lo[u] != lo[u]) ? NAN : fminf(lo[u], l);
          hi[u] = fmaxf(hi[u], h);
        }
    }
    for (uint32_t rd = 0; rd < rounds; ++rd) {
      const uint32_t c = rd * 32 + sub, at = c * E;
      const int count = at < p.dim ? (int)min((uint32_t)E, p.dim - at) : 0;
      Raw<SD, E> raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (count > 0 && MFET_INSIDE(p.status, holds_values(p, (src[u] - reinterpret_cast<const S*>(p.mem)) / p.ld, at, count)))
          raw[u] = load_any<SD, E, VEC>(src[u] + at, count, p.mem, p.mem_end, p.wide);  // does not wait for the list entry
        else memset(&raw[u], 0, sizeof(raw[u]));
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t r = checked(p, row[u]);
        const bool ok = r >= 0;
        uint8_t* out = p.table + (uint64_t)(ok ? r : 0) * p.stride;
        if constexpr (TD == MFET_MXFP4) {
          uint32_t m = amax_raw<SD, E>(raw[u]);  // 0 where the row has ended: a short last block counts what it has
#pragma unroll
          for (int d = 1; d < LPB; d <<= 1) m = max(m, __shfl_xor_sync(kAll, m, d));
          const uint32_t b = mx_scale_byte(m);
          // the scale bytes of four neighbouring blocks as one word
          uint32_t word = b << (8 * ((sub / LPB) & 3));
          if (lanes > LPB) word |= __shfl_xor_sync(kAll, word, LPB);
          if (lanes > 2 * LPB) word |= __shfl_xor_sync(kAll, word, 2 * LPB);
          float v[E];
          widen_raw<SD, E>(raw[u], v);
          const float inv = b == kMxNan ? 0.f : mx_inv_scale(b);
          if (ok && count > 0 && MFET_INSIDE(p.status, holds_bytes(p, r, at / 2, (at + count) / 2))) {
            uint32_t codes[E / 8];
#pragma unroll
            for (int j = 0; j < E / 8; ++j) codes[j] = b == kMxNan ? 0u : mx_encode8(v + 8 * j, inv);
            uint32_t* dst = reinterpret_cast<uint32_t*>(out + at / 2);
            if (E == 16 && count == 16) *reinterpret_cast<uint2*>(dst) = make_uint2(codes[0], codes[E / 8 - 1]);
            else *dst = codes[0];
          }
          if (ok) {
            uint32_t* tail = reinterpret_cast<uint32_t*>(out + p.dim / 2);
            const uint32_t tail_words = (p.row_bytes - p.dim / 2) / 4, data_words = (p.dim + 127) / 128;
            const uint32_t w = c / (4 * LPB);
            if (c % (4 * LPB) == 0 && w < data_words && MFET_INSIDE(p.status, w < tail_words && r < (int64_t)p.rows)) tail[w] = word;
            if (rd + 1 == rounds)
              for (uint32_t x = data_words + sub; x < tail_words; x += lanes) tail[x] = 0u;  // the padding
          }
        } else if constexpr (TD == MFET_INT4) {
          float v[E];
          widen_raw<SD, E>(raw[u], v);
          const __half sh = __float2half_rn(__fdiv_rn(__fsub_rn(hi[u], lo[u]), 15.0f)), bh = __float2half_rn(lo[u]);
          const float scale = __half2float(sh), bias = __half2float(bh);
          const bool fine = isfinite(scale) && isfinite(bias);
          const float inv = __fdiv_rn(1.f, scale);
#pragma unroll
          for (int q = 0; q < E / 8; ++q) {
            uint32_t word = 0;
            if (fine && scale > 0.f) {
#pragma unroll
              for (int j = 0; j < 8; ++j) word |= int4_code(v[8 * q + j], scale, bias, inv) << (4 * j);
            }
            if (ok && count >= 8 * (q + 1) && MFET_INSIDE(p.status, holds_bytes(p, r, at / 2 + 4 * q, at / 2 + 4 * q + 4)))
              reinterpret_cast<uint32_t*>(out + at / 2)[q] = word;
          }
          // scale and bias, then zeros up to the row's end
          if (ok && rd == 0)
            for (uint32_t x = sub; x < (p.row_bytes - p.dim / 2) / 4; x += lanes)
              reinterpret_cast<uint32_t*>(out + p.dim / 2)[x] =
                  x > 0 ? 0u : (fine ? (uint32_t)__half_as_ushort(sh) | ((uint32_t)__half_as_ushort(bh) << 16) : 0x7E007E00u);
        } else {
          float v[E];
          widen_raw<SD, E>(raw[u], v);
          if (ok && count > 0 && MFET_INSIDE(p.status, holds_bytes(p, r, 0, (uint64_t)(at + count) * sizeof(typename Elem<TD>::T))))
            store_values<TD, E, true>(reinterpret_cast<typename Elem<TD>::T*>(out) + at, v, count);
        }
      }
    }
  }
}

template <int TD, int DD, bool VEC>
__global__ void __launch_bounds__(kRowsThreads, kRowsBlocksPerSm) rows_read_kernel(const __grid_constant__ RowsParams p) {
  using D = typename Elem<DD>::T;
  constexpr int E = 32 / (int)sizeof(D), LPB = kMxBlock / E;
  constexpr int U = kRowsReadAhead;
  early_launch_wait();
  const int64_t n = live_count(p);
  const int lane = threadIdx.x & 31;
  const int lanes = 1 << p.lanes_log2, per_warp = 32 >> p.lanes_log2;
  const int sub = lane & (lanes - 1), group = lane >> p.lanes_log2;
  const int64_t step = (int64_t)gridDim.x * (kRowsThreads / 32) * per_warp * U;
  const uint32_t rounds = p.rounds;
  constexpr bool kCodes = TD == MFET_MXFP4 || TD == MFET_INT4;
  constexpr int kTable = kCodes ? MFET_F32 : TD;  // element type of a row that is stored plainly
  int64_t w0 = (((int64_t)blockIdx.x * kRowsThreads + threadIdx.x) >> 5) * per_warp * U;
  int64_t next[U];
#pragma unroll
  for (int u = 0; u < U; ++u) next[u] = entry(p, w0 + u * per_warp + group, n);
  for (; w0 < n; w0 += step) {
    int64_t row[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      row[u] = checked(p, next[u]);
      next[u] = entry(p, w0 + step + u * per_warp + group, n);
    }
    for (uint32_t rd = 0; rd < rounds; ++rd) {
      const uint32_t c = rd * 32 + sub, at = c * E;
      const int count = at < p.dim ? (int)min((uint32_t)E, p.dim - at) : 0;
      uint32_t codes[U][E / 8], meta[U];
      Raw<kTable, E> raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int j = 0; j < E / 8; ++j) codes[u][j] = 0;
        meta[u] = 0;
        if (row[u] >= 0 && count > 0 &&
            MFET_INSIDE(p.status, kCodes ? holds_bytes(p, row[u], at / 2, at / 2 + E / 2) &&
                                               holds_bytes(p, row[u], p.dim / 2, p.dim / 2 + (TD == MFET_MXFP4 ? c / LPB + 1 : 4))
                                         : holds_bytes(p, row[u], 0, (uint64_t)(at + count) * sizeof(typename Elem<kTable>::T)))) {
          const uint8_t* from = p.table + (uint64_t)row[u] * p.stride;
          if constexpr (kCodes) {
            // 16 codes are read together; behind the last 8 of a row lie its scales, which are not used as codes
            if constexpr (E == 16) {
              const uint2 two = *reinterpret_cast<const uint2*>(from + at / 2);
              codes[u][0] = two.x;
              codes[u][E / 8 - 1] = two.y;
            } else {
              codes[u][0] = *reinterpret_cast<const uint32_t*>(from + at / 2);
            }
            meta[u] = TD == MFET_MXFP4 ? (uint32_t)from[p.dim / 2 + c / LPB] : *reinterpret_cast<const uint32_t*>(from + p.dim / 2);
          } else {
            raw[u] = load_raw<kTable, E, true>(reinterpret_cast<const typename Elem<kTable>::T*>(from) + at, count);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t i = w0 + u * per_warp + group;
        if (i >= n || count == 0) continue;
        float v[E] = {};
        if (row[u] >= 0) {
          if constexpr (TD == MFET_MXFP4) {
            const float scale = mx_scale(meta[u]);
#pragma unroll
            for (int j = 0; j < E / 8; ++j) mx_decode8(codes[u][j], scale, v + 8 * j);
          } else if constexpr (TD == MFET_INT4) {
            const float2 sb = __half22float2(*reinterpret_cast<const __half2*>(&meta[u]));
#pragma unroll
            for (int j = 0; j < E; ++j) v[j] = fmaf((float)((codes[u][j / 8] >> (4 * (j % 8))) & 15u), sb.x, sb.y);
          } else {
            widen_raw<kTable, E>(raw[u], v);
          }
        }
        if (!MFET_INSIDE(p.status, holds_values(p, i, at, count))) continue;
        store_values<DD, E, VEC>(reinterpret_cast<D*>(p.mem) + i * p.ld + at, v, count, p.wide);
      }
    }
  }
}

// the narrowest lane group that covers a row (32 bytes of values per lane, whole blocks of 32 values), and how many rounds
// a wider row takes
void lanes_of(uint32_t dim, uint32_t mem_dtype, RowsParams* p) {
  const uint32_t per_block = mem_dtype == MFET_F32 ? 4 : 2, chunks = (dim + 31) / 32 * per_block;
  uint32_t l = per_block == 4 ? 2 : 1;
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
  p->mem_end = n > 0 ? p->mem + ((n - 1) * ld + d->dim) * (mem_dtype == MFET_F32 ? 4 : 2) : p->mem;
  p->dim = d->dim;
  p->row_bytes = (uint32_t)rb;
  p->wide = (reinterpret_cast<uintptr_t>(mem) & 31u) == 0 && (ld * (mem_dtype == MFET_F32 ? 4 : 2)) % 32 == 0;
  lanes_of(d->dim, mem_dtype, p);
  return MFET_OK;
}

// 16-byte pieces of the value rows can be used when every row starts on a 16-byte boundary
bool vectors(const RowsParams& p, uint32_t dtype) {
  return (reinterpret_cast<uintptr_t>(p.mem) & 15u) == 0 && (p.ld * (dtype == MFET_F32 ? 4 : 2)) % 16 == 0;
}

unsigned blocks_for(const RowsParams& p) {
  const int64_t per_block = (int64_t)(kRowsThreads >> p.lanes_log2) * kRowsInFlight;
  const int64_t want = (p.n + per_block - 1) / per_block, most = (int64_t)sm_count() * kRowsBlocksPerSm;
  return (unsigned)(want < most ? want : most);
}

template <int TD, int MD, bool VEC>
cudaError_t launch_as(const RowsParams& p, bool write, cudaStream_t s) {
  return launch_early(write ? rows_write_kernel<TD, MD, VEC> : rows_read_kernel<TD, MD, VEC>, blocks_for(p), kRowsThreads, 0, s, p);
}

template <int TD, int MD>
cudaError_t launch_one(const RowsParams& p, bool write, cudaStream_t s) {
  return vectors(p, MD) ? launch_as<TD, MD, true>(p, write, s) : launch_as<TD, MD, false>(p, write, s);
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
  if (((uintptr_t)list & 7u) || ((uintptr_t)n_dev & 7u) || ((uintptr_t)status & 3u)) return MFET_ERR_ALIGNMENT;
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
