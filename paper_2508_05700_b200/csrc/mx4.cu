// MXFP4 matrices: quantisation of a matrix into an operand, and the product of two operands,
//
//   y[i, j] = act(sum over k of a[i, k] * w[j, k] + bias[j])
//
// An operand of r rows and k columns is its codes, row by row (16 bytes per block of 32 values, the last block filled up
// with zeros), and its scale bytes in tiles of 128 rows x 4 blocks = 512 bytes, tile by tile along a row of tiles: byte
// (r % 32) * 16 + (r % 128) / 32 * 4 + block % 4 of a tile. That is the order in which the tensor cores read
// scales, so a tile goes from global to shared to tensor memory as it lies. Codes and scales are defined in lowbit.cuh.
//
// Two kernels for the product. A few rows (mx4_few_kernel): the weights are read once and nothing else costs bandwidth,
// so a warp per output column and integer dot products suffice, and x is quantised in the same launch. More rows
// (mx4_gemm_kernel): block-scaled 5th-generation tensor-core instructions.
#include <cstring>

#include "tensor.cuh"

using namespace mfet;

namespace mfet {
namespace {

constexpr unsigned kAll = 0xFFFFFFFFu;

// ------------------------------------------------------------------ quantisation ----

constexpr int kQuantThreads = 256;

struct QuantParams {
  const uint8_t* x;
  int64_t ld;
  int64_t units;     // rows * 4 * groups
  const void* x_end;
  uint32_t k, blocks, groups;  // values, blocks of 32, groups of 4 blocks per row
  bool wide;         // every row of x starts on a 32-byte boundary
  uint8_t* codes;
  uint8_t* scales;
};

// A lane takes a block of 32 values: no exchange for its scale, and 16 bytes of codes in one store. Four lanes write their scale
// bytes as one word (a row's blocks are counted up to a multiple of four). Bound by reading x; with fewer values per lane the
// instructions around them were the limit (16384 x 2048 bf16: 16 us = 5.3 TB/s read and written, 19 with 16 values per lane; 8192 x 896
// fp32: 6.5 us = 5.2 TB/s). Rows that do not start on 16 bytes are read in shifted pieces: 500 x 1075 bf16 2.5 us, 6.3 value by value.
template <int DT, bool VEC>
__global__ void __launch_bounds__(kQuantThreads, 4) mx4_quantize_kernel(const __grid_constant__ QuantParams p) {
  using T = typename Elem<DT>::T;
  constexpr int U = VEC && DT != MFET_F32 ? 2 : 1;  // blocks that a lane requests together
  early_launch_wait();
  const int lane = threadIdx.x & 31;
  const uint32_t per_row = p.groups * 4;
  const int64_t step = (int64_t)gridDim.x * kQuantThreads * U;
  for (int64_t u0 = ((int64_t)blockIdx.x * kQuantThreads + (threadIdx.x & ~31u)) * U; u0 < p.units; u0 += step) {
    Raw<DT, 32> raw[U];
    int64_t row[U];
    uint32_t c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = u0 + 32 * u + lane;
      row[u] = (uint64_t)i >> 32 ? i / per_row : (int64_t)((uint32_t)i / per_row);
      c[u] = (uint32_t)(i - row[u] * per_row);
      const uint32_t at = c[u] * 32;
      const int count = i < p.units && at < p.k ? (int)min(32u, p.k - at) : 0;
      if (count > 0 && MFET_INSIDE(nullptr, row[u] * per_row + c[u] < p.units && at + count <= p.k))
        raw[u] = load_any<DT, 32, VEC>(reinterpret_cast<const T*>(p.x) + row[u] * p.ld + at, count, p.x, p.x_end, p.wide);
      else memset(&raw[u], 0, sizeof(raw[u]));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u0 + 32 * u >= p.units) break;  // the same for the whole warp
      const uint32_t e = mx_scale_byte(amax_raw<DT, 32>(raw[u]));
      uint32_t word = e << (8 * (lane & 3));
      word |= __shfl_xor_sync(kAll, word, 1);
      word |= __shfl_xor_sync(kAll, word, 2);
      const float inv = mx_inv_scale(e == kMxNan ? 0u : e);
      uint32_t codes[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v[8];
#pragma unroll
        for (int h = 0; h < 8 / Raw<DT, 32>::per; ++h) widen16<DT>(raw[u].w[q * (8 / Raw<DT, 32>::per) + h], v + h * Raw<DT, 32>::per);
        codes[q] = mx_encode8(v, inv);
      }
      if (e == kMxNan) codes[0] = codes[1] = codes[2] = codes[3] = 0u;
      if (u0 + 32 * u + lane < p.units) {
        if (c[u] < p.blocks && MFET_INSIDE(nullptr, row[u] * per_row < p.units))
          *reinterpret_cast<uint4*>(p.codes + (row[u] * p.blocks + c[u]) * 16) = make_uint4(codes[0], codes[1], codes[2], codes[3]);
        if ((lane & 3) == 0 && MFET_INSIDE(nullptr, row[u] * per_row < p.units && (c[u] >> 2) < p.groups))
          *reinterpret_cast<uint32_t*>(p.scales + ((row[u] >> 7) * p.groups + (c[u] >> 2)) * 512 + (row[u] & 31) * 16 +
                                       ((row[u] & 127) >> 5) * 4) = word;
      }
    }
  }
}

// ------------------------------------------------------------------ epilogue ----

struct OutParams {
  uint8_t* y;
  int64_t ld;
  const float* bias;
  uint32_t dtype;
  uint32_t relu;
};

__device__ __forceinline__ float activate(float v, float bias, uint32_t relu) {
  v += bias;
  if (relu) asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(v));  // a NaN stays one
  return v;
}

__device__ __forceinline__ void put(const OutParams& o, int64_t i, int64_t j, float v) {
  const int64_t at = i * o.ld + j;
  if (o.dtype == MFET_F32) reinterpret_cast<float*>(o.y)[at] = v;
  else if (o.dtype == MFET_F16) reinterpret_cast<__half*>(o.y)[at] = __float2half_rn(v);
  else reinterpret_cast<__nv_bfloat16*>(o.y)[at] = __float2bfloat16_rn(v);
}

// ------------------------------------------------------------------ a few rows ----

constexpr int kFewThreads = 256;
constexpr int kFewMost = 8;  // rows of x
// The most work, in multiply-adds, with the rows counted up to a power of two. The integer products grow with it and the two-launch form
// hardly does; a second launch costs a calling program 2.4 us besides its time on the device. On the device: 1 x 896 x 1024 2.5 us here
// against 4.8; at 2^24 7 x 2048 x 1000 6.9 against 7.6, 2 x 2048 x 4096 5.2 against 6.3; at the limit 4 x 2048 x 4096 6.8 against 6.6,
// 1 x 2048 x 16384 9.4 against 8.3, 8 x 2048 x 2048 8.8 against 6.3 (with the launch about even); beyond it 4 x 2048 x 8192 (2^26) 9.8
// against 8.2 and 8 x 2048 x 8192 17.5 against 8.3.
constexpr int64_t kFewWork = 1ll << 25;
constexpr uint32_t kFewSmem = 96 * 1024;  // the quantised x has to fit this (k up to 10,000 for 8 rows)

struct FewParams {
  const uint8_t* x;
  int64_t ld;
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t n;
  uint32_t k, blocks, groups;
  int32_t m;
  uint32_t x_dtype, vec;
  const void* x_end;
  OutParams out;
};

// twice the values of codes 0..3 of `codes`' low half, as signed bytes. A code's low three bits pick the magnitude
// 0,1,2,3,4,6,8,12; prmt reads the code's sign bit as "replicate the sign of the picked byte", which is 0 for these tables,
// so `pos` holds the non-negative codes and `neg` the magnitudes of the others.
__device__ __forceinline__ uint32_t pick4(uint32_t codes) {
  uint32_t r;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(0x03020100u), "r"(0x0C080604u), "r"(codes));  // reads 16 bits of codes
  return r;
}
__device__ __forceinline__ uint32_t twice4(uint32_t codes) {
  const uint32_t pos = pick4(codes), neg = pick4(codes ^ 0x8888u);
  return ((pos | 0x80808080u) - neg) ^ 0x80808080u;  // no borrow crosses a byte
}

// The block's copy of x: a block's 32 signed bytes go to two arrays of 16-byte halves, so that neighbouring lanes' reads of
// neighbouring blocks hit neighbouring banks. `padded` blocks per row, a multiple of 32. kFewInFlight loads are under way at a time:
// this phase is nothing but their latency.
constexpr int kFewInFlight = 4;
template <int DT, bool VEC>
__device__ __forceinline__ void few_stage(const FewParams& p, int mt, int4* sx, float* ss, uint32_t padded) {
  using T = typename Elem<DT>::T;
  constexpr int U = VEC ? kFewInFlight : 2;
  const uint32_t units = (uint32_t)mt * padded * 4;  // chunks of 8 values: whole warps
  for (uint32_t i0 = threadIdx.x; i0 < units; i0 += kFewThreads * U) {
    Raw<DT, 8> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t i = i0 + u * kFewThreads, row = i / (padded * 4), c = i - row * padded * 4;
      const int count = i < units && (int)row < p.m && c * 8 < p.k ? (int)min(8u, p.k - c * 8) : 0;
      if (count > 0 && MFET_INSIDE(nullptr, (int)row < p.m && c * 8 + count <= p.k))
        raw[u] = load_any<DT, 8, VEC>(reinterpret_cast<const T*>(p.x) + (int64_t)row * p.ld + c * 8, count, p.x, p.x_end);
      else memset(&raw[u], 0, sizeof(raw[u]));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t i = i0 + u * kFewThreads, row = i / (padded * 4), c = i - row * padded * 4;
      if (i >= units) break;  // the same for a whole warp
      float v[8];
      widen_raw<DT, 8>(raw[u], v);
      uint32_t m = amax_raw<DT, 8>(raw[u]);
      m = max(m, __shfl_xor_sync(kAll, m, 1));
      m = max(m, __shfl_xor_sync(kAll, m, 2));
      const uint32_t s = mx_scale_byte(m);
      const uint32_t codes = s == kMxNan ? 0u : mx_encode8(v, mx_inv_scale(s));
      if (!MFET_INSIDE(nullptr, (int)row < mt && (c >> 2) < padded)) continue;
      uint2* dst = reinterpret_cast<uint2*>(sx + (row * 2 + ((c >> 1) & 1)) * padded + (c >> 2)) + (c & 1);
      *dst = make_uint2(twice4(codes), twice4(codes >> 16));
      if ((c & 3) == 0) ss[row * padded + (c >> 2)] = mx_scale(s);
    }
  }
}
template <int DT>
__device__ __forceinline__ void few_stage(const FewParams& p, int mt, int4* sx, float* ss, uint32_t padded) {
  if (p.vec) few_stage<DT, true>(p, mt, sx, ss, padded);
  else few_stage<DT, false>(p, mt, sx, ss, padded);
}

// A warp per output column: lane b takes block b, b + 32, ... of the column's weights (16 bytes each, 512 bytes per warp and
// load) against the same block of all MT rows of x from shared memory: 8 integer dot products of 4 values per
// row and block, exact, then the two scales and an fp32 addition. Latency: 2.5 us for 1 x 896 x 1024 (0.5 MB of weights, 0.1 us of
// bandwidth), of which a launch is most; 6.9 us for 7 x 2048 x 1000, where every block quantises all of x for itself.
template <int MT>
__global__ void __launch_bounds__(kFewThreads) mx4_few_kernel(const __grid_constant__ FewParams p) {
  extern __shared__ int4 sx[];  // [MT][2][padded] 16-byte halves, then [MT][padded] scales
  const uint32_t padded = (p.blocks + 31) & ~31u;
  float* ss = reinterpret_cast<float*>(sx + (size_t)MT * 2 * padded);
  const int lane = threadIdx.x & 31;
  const int64_t first = (int64_t)blockIdx.x * (kFewThreads / 32) + (threadIdx.x >> 5);
  const int64_t step = (int64_t)gridDim.x * (kFewThreads / 32);
  auto weights = [&](int64_t j, uint32_t b, uint4* w, uint32_t* s) {
    const bool in = j < p.n && b < p.blocks && MFET_INSIDE(nullptr, j >= 0 && (b >> 2) < p.groups);
    *w = in ? __ldg(reinterpret_cast<const uint4*>(p.codes + (j * p.blocks + b) * 16)) : make_uint4(0, 0, 0, 0);
    *s = in ? (uint32_t)__ldg(p.scales + ((j >> 7) * p.groups + (b >> 2)) * 512 + (j & 31) * 16 + ((j & 127) >> 5) * 4 + (b & 3))
            : 0u;
  };
  early_launch_wait();
  // the first weights do not depend on x: they are under way while x is quantised
  uint4 w;
  uint32_t s;
  weights(first, lane, &w, &s);
  if (p.x_dtype == MFET_F32) few_stage<MFET_F32>(p, MT, sx, ss, padded);
  else if (p.x_dtype == MFET_F16) few_stage<MFET_F16>(p, MT, sx, ss, padded);
  else few_stage<MFET_BF16>(p, MT, sx, ss, padded);
  __syncthreads();
  for (int64_t j = first; j < p.n; j += step) {
    float acc[MT];
#pragma unroll
    for (int r = 0; r < MT; ++r) acc[r] = 0.f;
    for (uint32_t b = lane; b < padded; b += 32) {
      const uint4 wn = w;
      // Both factors of the integer product are doubled. It goes up to 4608: under the largest weights' scales (2^116 and above) it is held
      // 2^12 smaller until x's scale is in, else it would leave fp32's range where the product of all three does not.
      const bool large = s > 242u;
      const float sw = mx_scale(s) * (large ? 0x1p-14f : 0x1p-2f), back = large ? 0x1p12f : 1.f;
      // the next block's weights, or the next column's first ones
      if (b + 32 < padded) weights(j, b + 32, &w, &s);
      else weights(j + step, lane, &w, &s);
      const uint32_t c[4] = {wn.x, wn.y, wn.z, wn.w};
      uint32_t v[8];
#pragma unroll
      for (int q = 0; q < 4; ++q) v[2 * q] = twice4(c[q]), v[2 * q + 1] = twice4(c[q] >> 16);
#pragma unroll
      for (int r = 0; r < MT; ++r) {
        const int4 x0 = sx[(r * 2) * padded + b], x1 = sx[(r * 2 + 1) * padded + b];
        int d = __dp4a((int)v[0], x0.x, 0);
        d = __dp4a((int)v[1], x0.y, d);
        d = __dp4a((int)v[2], x0.z, d);
        d = __dp4a((int)v[3], x0.w, d);
        d = __dp4a((int)v[4], x1.x, d);
        d = __dp4a((int)v[5], x1.y, d);
        d = __dp4a((int)v[6], x1.z, d);
        d = __dp4a((int)v[7], x1.w, d);
        acc[r] = fmaf((float)d * sw * ss[r * padded + b], back, acc[r]);
      }
    }
#pragma unroll
    for (int r = 0; r < MT; ++r) {
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) acc[r] += __shfl_xor_sync(kAll, acc[r], d);
    }
    float mine = acc[0];
#pragma unroll
    for (int r = 1; r < MT; ++r)
      if (lane == r) mine = acc[r];
    if (lane < p.m && MFET_INSIDE(nullptr, j >= 0 && j < p.n && j < p.out.ld)) put(p.out, lane, j, activate(mine, p.out.bias ? p.out.bias[j] : 0.f, p.out.relu));
  }
}

// ------------------------------------------------------------------ tensor cores ----

constexpr int kGemmThreads = 320;  // warp 0 loads, warp 1 issues the products, warps 2..9 write results
constexpr int kTileM = 128;        // rows of x per tile: lanes of tensor memory
constexpr int kSlab = 256;         // k per stage: 128 bytes of codes per row, four instructions of k = 64

template <int TN, int DT>  // output columns per tile: 64 or 128; type of y
struct GemmShape {
  static constexpr uint32_t a_bytes = kTileM * 128, b_bytes = TN * 128, s_bytes = 1024;  // a stage: k = 256; two tiles of scales each
  static constexpr uint32_t b_at = a_bytes, scale_at = a_bytes + b_bytes, stage_bytes = scale_at + 2 * s_bytes;
  static constexpr int stages = TN == 64 ? 6 : 5;
  // Results leave in pieces of 32 rows x 32 columns (wider ones of 16-bit values were slower: 46 instead of 41 us for 16384 x 2048 x 2048)
  static constexpr int piece_row = 32 * (int)sizeof(typename Elem<DT>::T);  // 64 or 128 bytes
  static constexpr int pieces = 4096 / (32 * piece_row);                    // that a warp has room for
  static constexpr uint32_t out_at = stage_bytes * stages;
  static constexpr uint32_t bias_at = out_at + 8 * 4096;
  static constexpr uint32_t smem = bias_at + 8 * (TN / 2) * 4 + 1024;  // + room to align to 1024
  // Tensor memory: two accumulators, then two sets of scales (copies and products run in the order of their issue, so a set may be
  // overwritten by the copies of the stage after the next)
  static constexpr uint32_t acc_cols = TN, scale_col = 2 * TN;
  static_assert(scale_col + 2 * 16 <= 512, "tensor memory has 512 columns");
  static_assert(smem <= 227 * 1024 - 256, "shared memory of a block");
  // 64 columns: an odd tile starts in the middle of a tile of scales, two of its four columns further on
  static __device__ __forceinline__ uint32_t half_shift(uint32_t tn) { return TN % 128 ? (tn & 1) * 2 : 0; }
  // the 16 bytes `q` of row `row` of a piece, where the bulk copy's swizzle expects them: no bank conflicts among eight rows
  static __device__ __forceinline__ int at(int row, int q) {
    return row * piece_row + ((piece_row == 128 ? q ^ (row & 7) : q ^ ((row >> 1) & 3)) << 4);
  }
};

struct GemmParams {
  const uint8_t* a_scales;  // x
  const uint8_t* b_scales;  // weights
  int64_t m, n;
  uint32_t k, groups, stages_k;  // stages_k: stages that cover k
  uint32_t n_tiles;
  uint32_t bulk_y;          // every row of y starts on a 16-byte boundary
  uint32_t whole_y;         // ... and ends on one: bulk copies write whole units of 16 bytes, also where a row ends inside one
  int64_t tiles;
  uint32_t* status;
  OutParams out;
};

// The tiles of a block, one after the other: column tiles run fastest
struct TileWalk {
  int64_t t;
  uint32_t tm, tn, n_tiles, dm, dn;
  __device__ __forceinline__ explicit TileWalk(uint32_t n_tiles_) : t(blockIdx.x), n_tiles(n_tiles_) {
    tm = blockIdx.x / n_tiles;
    tn = blockIdx.x - tm * n_tiles;
    dm = gridDim.x / n_tiles;
    dn = gridDim.x - dm * n_tiles;
  }
  __device__ __forceinline__ void next() {
    t += gridDim.x;
    tm += dm;
    tn += dn;
    if (tn >= n_tiles) tn -= n_tiles, ++tm;
  }
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}

// Shared-memory matrix descriptors; the low word holds the address, the high word is constant.
// Codes: K-major rows of 128 bytes with the 128-byte swizzle, groups of 8 rows 1024 bytes apart.
constexpr uint32_t kTileDescHi = 64u | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t tile_desc_lo(uint32_t addr) { return (addr >> 4) | (1u << 16); }
// Scales: 32 rows of 16 bytes without a swizzle, groups of 8 rows 128 bytes apart.
constexpr uint32_t kScaleDescHi = 8u | (1u << 14);
__device__ __forceinline__ uint32_t scale_desc_lo(uint32_t addr) { return (addr >> 4) | (8u << 16); }
// Instruction descriptor: both operands E2M1, K-major, scales UE8M0, fp32 accumulator; `id`: which two of a row's four scale
// bytes (0 or 2) this instruction's two blocks use
template <int TN>
__device__ __forceinline__ uint32_t inst_desc(uint32_t id) {
  return (id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TN >> 3) << 17) | (1u << 23) | ((uint32_t)(kTileM >> 7) << 27) | (id << 29);
}

__device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t desc_lo) {
  asm volatile("{\n\t.reg .b64 d;\n\t"
               "mov.b64 d, {%1, %2};\n\t"
               "tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], d;\n\t}" ::"r"(tmem),
               "r"(desc_lo), "n"(kScaleDescHi)
               : "memory");
}
__device__ __forceinline__ void mma_mx4(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t inst, uint32_t sa, uint32_t sb, uint32_t add) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
               "setp.ne.b32 p, %6, 0;\n\t"
               "mov.b64 a, {%1, %7};\n\t"
               "mov.b64 b, {%2, %7};\n\t"
               "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], a, b, %3, [%4], [%5], p;\n\t}" ::"r"(d),
               "r"(a_lo), "r"(b_lo), "r"(inst), "r"(sa), "r"(sb), "r"(add), "n"(kTileDescHi)
               : "memory");
}
// One block per SM walks over the tiles (128 rows of x times TN output columns); output columns run fastest, so that the blocks
// at work share the rows of x in L2. 8192 x 896 x 1024 to bf16 takes 10 us (1.5 PFLOP/s), 16384 x 2048 x 2048 41 us (3.4 PFLOP/s; without its loads 29,
// without its stores 36: it is bound by what loads, stores and scales share, not by the tensor cores, which are busy 44 % of the time).
// Stages go through a ring of shared memory, scales from there to tensor memory ahead
// of the products that use them; two accumulators in tensor memory, so that a tile is written while the next one is computed. A
// lane of tensor memory is a row of x: each of the eight writing warps takes its 32 rows and half of the columns, adds the bias, rounds,
// and leaves 32 columns at a time in shared memory (swizzled: no bank conflicts), from where a bulk
// copy writes them and clips what lies beyond y. (Stores straight from the registers touch a line per lane, and the barriers of
// the other roles wait behind them: 43 us instead of 41 for 16384 x 2048 x 2048.) A y whose rows do not start on 16 bytes is written by
// plain stores from there.
template <int TN, int DT>
__global__ void __launch_bounds__(kGemmThreads, 1) mx4_gemm_kernel(const __grid_constant__ CUtensorMap a_map,
                                                                  const __grid_constant__ CUtensorMap b_map,
                                                                  const __grid_constant__ CUtensorMap y_map,
                                                                  const __grid_constant__ GemmParams p) {
  using G = GemmShape<TN, DT>;
  using T = typename Elem<DT>::T;
  extern __shared__ uint8_t raw_smem[];
  __shared__ __align__(8) uint64_t bars[2 * G::stages + 5];
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int dead;
  const uint32_t base = (smem_addr(raw_smem) + 1023) & ~1023u;
  uint8_t* const smem = raw_smem + (base - smem_addr(raw_smem));
  const uint32_t bar0 = smem_addr(bars);
  auto full = [&](int s) { return bar0 + 8 * s; };
  auto empty = [&](int s) { return bar0 + 8 * (G::stages + s); };
  auto acc_full = [&](int a) { return bar0 + 8 * (2 * G::stages + a); };
  auto acc_empty = [&](int a) { return bar0 + 8 * (2 * G::stages + 2 + a); };
  const uint32_t drained = bar0 + 8 * (2 * G::stages + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < G::stages; ++s) bar_init(full(s), 1), bar_init(empty(s), 1);
    for (int a = 0; a < 2; ++a) bar_init(acc_full(a), 1), bar_init(acc_empty(a), 8);
    bar_init(drained, 1);
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&tmem_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;

  // The barriers and the tensor memory are set up by now. This kernel does not let the next one in early: blocks that wait beside it
  // made it slower (8192 x 896 x 1024 with its quantisation: 21 instead of 17 us).
  asm volatile("griddepcontrol.wait;" ::: "memory");

  uint64_t filled = 0;  // stages that this lane has asked for
  bool issues = false;  // this lane issues the products
  if (warp == 0) {
    // One lane runs this role from end to end: what it does per stage is on the critical path of a product with many tiles.
    if (elect_one()) {
      uint32_t st = 0, phase = 1;  // an empty barrier's phase before the first is taken as complete
      bool ok = true;
      for (TileWalk w(p.n_tiles); ok && w.t < p.tiles; w.next()) {
        const int32_t ya = (int32_t)(w.tm * kTileM), yb = (int32_t)(w.tn * TN);
        const uint8_t* sa = p.a_scales + (size_t)w.tm * p.groups * 512;
        const uint8_t* sb = p.b_scales + (size_t)((uint32_t)yb >> 7) * p.groups * 512;
        for (uint32_t s = 0; s < p.stages_k; ++s) {
          if (!(ok = bar_wait(empty(st), phase, &dead))) break;
          // the scale tiles that are read here; codes outside their operand read as 0
          if (!MFET_INSIDE(p.status, 2 * s < p.groups && (int64_t)w.tm * kTileM < p.m && (int64_t)yb < p.n)) {
            ok = false;
            dead = 1;
            break;
          }
          const uint32_t at = base + st * G::stage_bytes, bar = full(st);
          const uint32_t sc = min(2u, p.groups - 2 * s) * 512;  // scale bytes per operand
          bar_expect(bar, G::a_bytes + G::b_bytes + 2 * sc);
          tma_load(at, &a_map, (int32_t)(s * 128), ya, bar);
          tma_load(at + G::b_at, &b_map, (int32_t)(s * 128), yb, bar);
          bulk_load(at + G::scale_at, sa + (size_t)s * 1024, sc, bar);
          bulk_load(at + G::scale_at + G::s_bytes, sb + (size_t)s * 1024, sc, bar);
          ++filled;
          if (++st == (uint32_t)G::stages) st = 0, phase ^= 1;
        }
      }
    }
  } else if (warp == 1) {
    // One lane runs this role from end to end. The tensor cores' queue is short, so what the lane does between the instructions of two
    // stages has to be short too: stage and phase are counted along, and the next stage's barrier is asked between this one's instructions.
    if (elect_one()) {
      issues = true;
      uint32_t st = 0, phase = 0, done = 0, set = 0;
      bool ok = true, ready = false;
      for (TileWalk w(p.n_tiles); ok && w.t < p.tiles; w.next(), ++done) {
        const int acc = done & 1;
        if (done >= 2 && !(ok = bar_wait(acc_empty(acc), (done / 2 - 1) & 1, &dead))) break;
        const uint32_t d = tmem + acc * G::acc_cols;
        const uint32_t half = G::half_shift(w.tn);
        for (uint32_t s = 0; s < p.stages_k; ++s) {
          if (!ready && !(ok = bar_wait(full(st), phase, &dead))) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t at = base + st * G::stage_bytes;
          const uint32_t this_empty = empty(st);
          const uint32_t sf = tmem + G::scale_col + 16 * (set ^= 1);
          const uint32_t a_lo = tile_desc_lo(at), b_lo = tile_desc_lo(at + G::b_at), sc_lo = scale_desc_lo(at + G::scale_at);
          if (++st == (uint32_t)G::stages) st = 0, phase ^= 1;
          // the scales of k = 128 (x, then weights), and instruction j of the stage
          auto scales = [&](int g) {
            copy_scales(sf + 8 * g, sc_lo + 32 * g);
            copy_scales(sf + 8 * g + 4, sc_lo + (G::s_bytes >> 4) + 32 * g);
          };
          auto product = [&](int j) {
            mma_mx4(d, a_lo + 2 * j, b_lo + 2 * j, inst_desc<TN>((j & 1) * 2), sf + 8 * (j >> 1), sf + 8 * (j >> 1) + 4 + half, s | j);
          };
          const uint32_t left = p.k - s * kSlab;
          if (left > 192u) {
            scales(0);
            scales(1);
            product(0);
            product(1);
            ready = bar_try(full(st), phase);
            product(2);
            product(3);
          } else {
            const int steps = (int)((left + 63) / 64);
            for (int g = 0; 2 * g < steps; ++g) scales(g);
            for (int j = 0; j < steps; ++j) product(j);
            ready = bar_try(full(st), phase);
          }
          mma_commit(this_empty);
          if (s + 1 == p.stages_k) mma_commit(acc_full(acc));
        }
      }
    }
  } else {
    const int quarter = warp & 3;                // the 32 lanes of tensor memory that this warp may read
    const int c0 = warp < 6 ? 0 : TN / 2;        // two warps share them, each takes half of the columns
    uint8_t* const out_ptr = smem + G::out_at + (warp - 2) * 4096;
    const uint32_t out_at = base + G::out_at + (warp - 2) * 4096;
    float* const bias = reinterpret_cast<float*>(smem + G::bias_at) + (warp - 2) * (TN / 2);
    uint32_t done = 0, turn = 0;
    for (TileWalk w(p.n_tiles); w.t < p.tiles; w.next(), ++done) {
      const int acc = done & 1;
      const int64_t i0 = (int64_t)w.tm * kTileM + quarter * 32, j0 = (int64_t)w.tn * TN + c0;
      for (int c = lane; c < TN / 2; c += 32) bias[c] = p.out.bias && j0 + c < p.n ? p.out.bias[j0 + c] : 0.f;
      __syncwarp();
      const bool ok = bar_wait(acc_full(acc), (done / 2) & 1, &dead);
      if (!__all_sync(kAll, ok)) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
      for (int c = 0; c < TN / 2; c += 32) {
        uint32_t r[32];
        tmem_load32(tmem + acc * G::acc_cols + c0 + c + ((uint32_t)(quarter * 32) << 16), r);
        if (c + 32 >= TN / 2) {  // the accumulator is read: the next tile but one may overwrite it
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) bar_arrive(acc_empty(acc));
        }
        float v[32];
#pragma unroll
        for (int q = 0; q < 32; q += 4) {
          const float4 b4 = *reinterpret_cast<const float4*>(bias + c + q);
          v[q] = activate(__uint_as_float(r[q]), b4.x, p.out.relu);
          v[q + 1] = activate(__uint_as_float(r[q + 1]), b4.y, p.out.relu);
          v[q + 2] = activate(__uint_as_float(r[q + 2]), b4.z, p.out.relu);
          v[q + 3] = activate(__uint_as_float(r[q + 3]), b4.w, p.out.relu);
        }
        constexpr int kPer = 16 / (int)sizeof(T);  // values per 16 bytes
        const uint32_t piece = (turn++ % G::pieces) * (32 * G::piece_row);
        uint8_t* const to = out_ptr + piece;
        if (p.bulk_y) {  // what this piece's memory held before has left
          asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(G::pieces - 1) : "memory");
          __syncwarp();
        }
#pragma unroll
        for (int q = 0; q < 32; q += kPer) *reinterpret_cast<uint4*>(to + G::at(lane, q / kPer)) = narrow16<DT>(v + q);
        const int64_t j1 = j0 + c;
        if (p.bulk_y && (p.whole_y || j1 + 32 <= p.n)) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (i0 < p.m && j1 < p.n && elect_one()) bulk_store(&y_map, out_at + piece, (int32_t)j1, (int32_t)i0);
          __syncwarp();
        } else {
          __syncwarp();
          T* y = reinterpret_cast<T*>(p.out.y) + i0 * p.out.ld + j1 + lane;
#pragma unroll 8
          for (int i = 0; i < 32; ++i) {  // a warp writes a row's 32 columns
            const T x = *reinterpret_cast<const T*>(to + G::at(i, lane / kPer) + lane % kPer * sizeof(T));
            if (i0 + i < p.m && j1 + lane < p.n && MFET_INSIDE(p.status, i0 >= 0 && j1 >= 0 && j1 + lane < p.out.ld)) y[i * p.out.ld] = x;
          }
          __syncwarp();
        }
        if (p.bulk_y) asm volatile("cp.async.bulk.commit_group;" ::: "memory");  // one per piece, which the wait above counts on
      }
    }
    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // shared memory outlives the copies that read it
  }
  __syncwarp();  // the one lane that loaded or issued rejoins its warp
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  // Without a stall every copy and product has been waited for by the role that needed it. After one, whoever was ahead of the role that
  // gave up has left some under way: all roles have ended here, so what is waited for now (with the same limit) is the last of them.
  if (dead) {
    volatile int none = 0;
    const uint64_t from = filled > G::stages ? filled - G::stages : 0;
    for (uint64_t i = from; i < filled; ++i) bar_wait(full(i % G::stages), (i / G::stages) & 1, &none);
    if (issues) {
      mma_commit(drained);
      bar_wait(drained, 0, &none);
    }
    if (threadIdx.x == 0 && p.status) atomicOr(p.status, (uint32_t)MFET_DEV_STALLED);
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  }
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// ------------------------------------------------------------------ host side ----

struct Dims {
  uint32_t blocks, groups;
};
Dims dims_of(int64_t k) { return {(uint32_t)((k + 31) / 32), (uint32_t)((k + 127) / 128)}; }

bool bad_size(int64_t rows, int64_t k) { return rows < 0 || rows >= (1ll << 31) || k < 1 || k >= (1ll << 30); }

uint64_t code_bytes(int64_t rows, int64_t k) { return (uint64_t)rows * dims_of(k).blocks * 16; }
uint64_t scale_bytes(int64_t rows, int64_t k) { return (uint64_t)((rows + 127) / 128) * dims_of(k).groups * 512; }

template <int DT>
cudaError_t launch_quantize(const QuantParams& p, bool vec, cudaStream_t s) {
  const int64_t want = (p.units + kQuantThreads - 1) / kQuantThreads, most = (int64_t)sm_count() * 16;
  const unsigned b = (unsigned)(want < most ? want : most);
  return launch_early(vec ? mx4_quantize_kernel<DT, true> : mx4_quantize_kernel<DT, false>, b, kQuantThreads, 0, s, p);
}

int quantize(const void* x, uint32_t dtype, int64_t rows, int64_t k, int64_t ld, void* codes, void* scales, cudaStream_t s) {
  const Dims d = dims_of(k);
  QuantParams p{(const uint8_t*)x, ld, rows * 4 * (int64_t)d.groups, (const uint8_t*)x + ((rows - 1) * ld + k) * size_of(dtype),
                (uint32_t)k, d.blocks, d.groups, aligned(x, 32) && (uint64_t)ld * size_of(dtype) % 32 == 0, (uint8_t*)codes,
                (uint8_t*)scales};
  const bool vec = aligned(x, 16) && (uint64_t)ld * size_of(dtype) % 16 == 0;
  cudaError_t e;
  switch (dtype) {
    case MFET_F32: e = launch_quantize<MFET_F32>(p, vec, s); break;
    case MFET_F16: e = launch_quantize<MFET_F16>(p, vec, s); break;
    default: e = launch_quantize<MFET_BF16>(p, vec, s); break;
  }
  return e == cudaSuccess ? MFET_OK : MFET_ERR_CUDA;
}

// codes [rows, blocks * 16 bytes] read in boxes of `box` rows x 128 bytes; what lies outside reads as code 0
bool code_map(CUtensorMap* map, const void* codes, int64_t rows, uint32_t blocks, uint32_t box) {
  const EncodeTiled f = encode_tiled();
  if (!f) return false;
  const cuuint64_t size[2] = {(cuuint64_t)blocks * 16, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)blocks * 16};
  const cuuint32_t boxes[2] = {128, box}, ones[2] = {1, 1};
  return f(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(codes), size, stride, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// y [m, n] written in boxes of 32 rows x `row` bytes (64 or 128)
bool out_map(CUtensorMap* map, const OutParams& o, int64_t m, int64_t n, uint32_t row) {
  const EncodeTiled f = encode_tiled();
  if (!f) return false;
  const uint32_t size = size_of(o.dtype);
  const cuuint64_t dims[2] = {(cuuint64_t)n, (cuuint64_t)m}, stride[1] = {(cuuint64_t)o.ld * size};
  const cuuint32_t boxes[2] = {row / size, 32}, ones[2] = {1, 1};
  const CUtensorMapDataType t = o.dtype == MFET_F32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                : o.dtype == MFET_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                      : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  return f(map, t, 2, o.y, dims, stride, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, row == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
           CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int TN, int DT>
int gemm(const void* xc, const void* xs, int64_t m, const void* wc, const void* ws, int64_t n, int64_t k, const OutParams& out,
         uint32_t* status, cudaStream_t s) {
  const Dims d = dims_of(k);
  CUtensorMap a, b, y;
  if (!code_map(&a, xc, m, d.blocks, kTileM) || !code_map(&b, wc, n, d.blocks, TN)) return MFET_ERR_CUDA;
  GemmParams p;
  p.a_scales = (const uint8_t*)xs;
  p.b_scales = (const uint8_t*)ws;
  p.m = m;
  p.n = n;
  p.k = (uint32_t)k;
  p.groups = d.groups;
  p.stages_k = (uint32_t)((k + kSlab - 1) / kSlab);
  p.n_tiles = (uint32_t)((n + TN - 1) / TN);
  p.tiles = (m + kTileM - 1) / kTileM * p.n_tiles;
  p.status = status;
  p.out = out;
  p.bulk_y = aligned(out.y, 16) && (uint64_t)out.ld * size_of(out.dtype) % 16 == 0;
  p.whole_y = n * size_of(out.dtype) % 16 == 0;
  if (!p.bulk_y) y = a;  // not used
  else if (!out_map(&y, out, m, n, GemmShape<TN, DT>::piece_row)) return MFET_ERR_CUDA;
  static std::atomic<uint64_t> ready{0};
  if (allow_smem(mx4_gemm_kernel<TN, DT>, GemmShape<TN, DT>::smem, &ready) != cudaSuccess) return MFET_ERR_CUDA;
  const unsigned blocks = (unsigned)(p.tiles < sm_count() ? p.tiles : sm_count());
  return launch_early(mx4_gemm_kernel<TN, DT>, blocks, kGemmThreads, GemmShape<TN, DT>::smem, s, a, b, y, p) == cudaSuccess ? MFET_OK
                                                                                                                        : MFET_ERR_CUDA;
}

template <int DT>
int product_dt(const void* xc, const void* xs, int64_t m, const void* wc, const void* ws, int64_t n, int64_t k, const OutParams& out,
               uint32_t* status, cudaStream_t s) {
  // Tiles of 128 columns when there is one for three quarters of the SMs, else of 64: twice the blocks. With quantisation, k = 896, n = 1024:
  // 64 tiles of 128 (m = 1024) 6.4 us against 6.0 with 64 columns, 128 tiles 7.3 against 8.0, 512 tiles 17.1 against 19.9.
  if ((m + kTileM - 1) / kTileM * ((n + 127) / 128) * 4 >= sm_count() * 3)
    return gemm<128, DT>(xc, xs, m, wc, ws, n, k, out, status, s);
  return gemm<64, DT>(xc, xs, m, wc, ws, n, k, out, status, s);
}

int product(const void* xc, const void* xs, int64_t m, const void* wc, const void* ws, int64_t n, int64_t k, const OutParams& out,
            uint32_t* status, cudaStream_t s) {
  switch (out.dtype) {
    case MFET_F32: return product_dt<MFET_F32>(xc, xs, m, wc, ws, n, k, out, status, s);
    case MFET_F16: return product_dt<MFET_F16>(xc, xs, m, wc, ws, n, k, out, status, s);
    default: return product_dt<MFET_BF16>(xc, xs, m, wc, ws, n, k, out, status, s);
  }
}

template <int MT>
cudaError_t launch_few(const FewParams& p, cudaStream_t s) {
  const size_t padded = (p.blocks + 31) & ~31u;
  const size_t smem = MT * padded * (32 + 4);
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem(mx4_few_kernel<MT>, kFewSmem, &ready);
  if (e != cudaSuccess) return e;
  const int64_t want = (p.n + kFewThreads / 32 - 1) / (kFewThreads / 32), most = (int64_t)sm_count() * 4;
  return launch_early(mx4_few_kernel<MT>, (unsigned)(want < most ? want : most), kFewThreads, smem, s, p);
}

int check_out(int64_t m, int64_t n, const float* bias, uint32_t act, const void* y, uint32_t dtype, int64_t ld) {
  if (dtype > MFET_BF16 || act > MFET_ACT_RELU || ld < n || ld >= (1ll << 31) || (m > 0 && n > 0 && !y)) return MFET_ERR_INVALID_ARG;
  if (!aligned(y, size_of(dtype)) || !aligned(bias, 4)) return MFET_ERR_ALIGNMENT;
  return MFET_OK;
}

}  // namespace
}  // namespace mfet

extern "C" {

uint64_t mfet_mx4_code_bytes(int64_t rows, int64_t k) { return bad_size(rows, k) ? 0 : code_bytes(rows, k); }
uint64_t mfet_mx4_scale_bytes(int64_t rows, int64_t k) { return bad_size(rows, k) ? 0 : scale_bytes(rows, k); }

int mfet_mx4_quantize(const void* x, uint32_t dtype, int64_t ld, int64_t rows, int64_t k, void* codes, void* scales,
                      mfet_stream_t stream) {
  if (dtype > MFET_BF16 || bad_size(rows, k) || ld < k || ld >= (1ll << 31)) return MFET_ERR_INVALID_ARG;
  if (rows == 0) return MFET_OK;
  if (!x || !codes || !scales) return MFET_ERR_INVALID_ARG;
  if (!aligned(x, size_of(dtype)) || !aligned(codes, 16) || !aligned(scales, 16)) return MFET_ERR_ALIGNMENT;
  return quantize(x, dtype, rows, k, ld, codes, scales, (cudaStream_t)stream);
}

int mfet_mx4_matmul(const void* a_codes, const void* a_scales, int64_t m, const void* w_codes, const void* w_scales, int64_t n,
                    int64_t k, const float* bias, uint32_t act, void* y, uint32_t y_dtype, int64_t y_ld, uint32_t* status,
                    mfet_stream_t stream) {
  if (bad_size(m, k) || bad_size(n, k)) return MFET_ERR_INVALID_ARG;
  const int rc = check_out(m, n, bias, act, y, y_dtype, y_ld);
  if (rc != MFET_OK) return rc;
  if (m == 0 || n == 0) return MFET_OK;
  if (!a_codes || !a_scales || !w_codes || !w_scales) return MFET_ERR_INVALID_ARG;
  if (!aligned(a_codes, 16) || !aligned(a_scales, 16) || !aligned(w_codes, 16) || !aligned(w_scales, 16) ||
      !aligned(status, 4))
    return MFET_ERR_ALIGNMENT;
  const OutParams out{(uint8_t*)y, y_ld, bias, y_dtype, act == MFET_ACT_RELU};
  return product(a_codes, a_scales, m, w_codes, w_scales, n, k, out, status, (cudaStream_t)stream);
}

uint64_t mfet_mx4_linear_bytes(int64_t m, int64_t k) {
  if (bad_size(m, k)) return 0;
  return scale_bytes(m, k) + code_bytes(m, k);
}

int mfet_mx4_linear(const void* x, uint32_t x_dtype, int64_t x_ld, int64_t m, const void* w_codes, const void* w_scales, int64_t n,
                    int64_t k, const float* bias, uint32_t act, void* y, uint32_t y_dtype, int64_t y_ld, void* scratch,
                    uint64_t scratch_bytes, uint32_t* status, mfet_stream_t stream) {
  if (x_dtype > MFET_BF16 || bad_size(m, k) || bad_size(n, k) || x_ld < k || x_ld >= (1ll << 31)) return MFET_ERR_INVALID_ARG;
  int rc = check_out(m, n, bias, act, y, y_dtype, y_ld);
  if (rc != MFET_OK) return rc;
  if (m == 0 || n == 0) return MFET_OK;
  if (!x || !w_codes || !w_scales) return MFET_ERR_INVALID_ARG;
  if (!aligned(x, size_of(x_dtype)) || !aligned(w_codes, 16) || !aligned(w_scales, 16) || !aligned(status, 4)) return MFET_ERR_ALIGNMENT;
  const OutParams out{(uint8_t*)y, y_ld, bias, y_dtype, act == MFET_ACT_RELU};
  const Dims d = dims_of(k);
  cudaStream_t s = (cudaStream_t)stream;
  // a few rows and little work
  const uint32_t mt = m == 1 ? 1 : m == 2 ? 2 : m <= 4 ? 4 : 8;
  if (m <= kFewMost && mt * n <= kFewWork / k && (uint64_t)mt * ((d.blocks + 31) & ~31u) * 36 <= kFewSmem) {
    FewParams p{(const uint8_t*)x, x_ld, (const uint8_t*)w_codes, (const uint8_t*)w_scales, n, (uint32_t)k, d.blocks, d.groups,
                (int32_t)m, x_dtype, aligned(x, 16) && (uint64_t)x_ld * size_of(x_dtype) % 16 == 0,
                (const uint8_t*)x + ((m - 1) * x_ld + k) * size_of(x_dtype), out};
    const cudaError_t e = mt == 1 ? launch_few<1>(p, s) : mt == 2 ? launch_few<2>(p, s) : mt == 4 ? launch_few<4>(p, s) : launch_few<8>(p, s);
    return e == cudaSuccess ? MFET_OK : MFET_ERR_CUDA;
  }
  if (!scratch || scratch_bytes < scale_bytes(m, k) + code_bytes(m, k)) return MFET_ERR_WORKSPACE;
  if (!aligned(scratch, 16)) return MFET_ERR_ALIGNMENT;
  uint8_t* scales = (uint8_t*)scratch;
  uint8_t* codes = scales + scale_bytes(m, k);
  rc = quantize(x, x_dtype, m, k, x_ld, codes, scales, s);
  if (rc != MFET_OK) return rc;
  return product(codes, scales, m, w_codes, w_scales, n, k, out, status, s);
}

}  // extern "C"
