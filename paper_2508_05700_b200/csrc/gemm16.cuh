// Products of 16-bit matrices on the tensor cores, with what follows them done on the accumulators:
//
//   acc[i, j] = sum over segments s, sum over k of A_s[i, k] * B_s[j, k]      (fp32)
//
// An operand lies K-major (rows of neighbouring k: x and W in x W^T) or MN-major (k runs over its rows: dG and x in dG^T x); the tensor
// cores read both, so nothing is transposed in memory. Segments add up products of several pairs of matrices in one accumulator
// (dG Wg + dU Wu; the three products of numbers held in two words).
//
// A tile is computed by one block, or by a pair of blocks that shares its operands (CTAS = 2: each loads its 128 rows of A and half of
// B, one issues the instructions of both; a pair reads 64 bytes per SM and cycle at full rate where a block alone would need 96).
// Copies of tiles go through a ring of shared memory; two accumulators in tensor memory, so that one tile is written while the next
// one is computed. With few tiles, `split` blocks (pairs) of a cluster take a part of k each, leave their sums in shared memory, and
// each adds up its share of the columns over all of them, in the order of k: the result does not depend on who is first. The tensor cores truncate a
// running sum; long ones are taken in parts, in the two accumulators in turn, that the writing warps add up in registers (the modes *Long).
#pragma once

#include <cstring>
#include <type_traits>

#include "tensor.cuh"

namespace mfet {
namespace gemm16 {

constexpr int kThreads = 320;  // warp 0 loads, warp 1 issues the products, warps 2..9 write results
constexpr int kSlab = 64;      // k per stage: 128 bytes of a K-major row
constexpr unsigned kAllLanes = 0xFFFFFFFFu;

enum Mode {
  kGated,      // columns are units: h = act(g) * u
  kGatedBack,  // ... with the gradient of h: dG and dU
  kOut,        // the accumulator, rounded
  kOutTwo,     // ... of two products of different operands in one launch
  kPair,       // v = alpha * C + beta * acc in two fp16 words
  kPairOut,    // the same, rounded to the type of the result
  kOutLong,    // kOut of a long sum: the tensor cores add up parts of k, registers the parts
  kOutTwoLong, // kOutTwo, of which the first product's sum is long and the second's is one part
  kPairLong,   // kPair and kPairOut of a long sum
  kPairOutLong
};
template <int MODE>
constexpr bool is_long = MODE >= kOutLong;
template <int MODE>
constexpr bool is_two = MODE == kOutTwo || MODE == kOutTwoLong;
template <int MODE>
constexpr bool is_pair = MODE == kPair || MODE == kPairLong;
template <int MODE>
constexpr bool is_pair_out = MODE == kPairOut || MODE == kPairOutLong;

template <int CTAS, int TN, int MODE, int DT>
struct Shape {
  static constexpr bool dual = MODE == kGated || MODE == kGatedBack;  // half of the columns of B come from a second matrix
  static constexpr int outs = MODE == kGatedBack || is_pair<MODE> ? 2 : 1;
  static constexpr int b_rows = TN / CTAS;
  static constexpr bool precise = is_pair<MODE> || is_pair_out<MODE>;  // two words each; several sums of a part of k each (Params::sums)
  // With few columns the loads' latency is what a block of k takes: both words of both operands come together, and serve the three products
  static constexpr bool fused = precise && TN == 64;
  static constexpr uint32_t a_bytes = 128 * 128, b_bytes = b_rows * 128, stage_bytes = (a_bytes + b_bytes) * (fused ? 2 : 1);
  // Results leave in pieces of 32 rows x 32 columns; a warp has room for two of each output, or for the one that it has of a tile of 64 columns
  static constexpr int turns = TN == 64 ? 1 : 2;
  static constexpr int piece_row = 32 * (int)sizeof(typename Elem<DT>::T);
  static constexpr uint32_t piece = 32 * piece_row;
  static constexpr uint32_t warp_out = turns * outs * piece;
  static constexpr int stages = (int)((226u * 1024 - 1024 - 8 * warp_out) / stage_bytes);
  static constexpr uint32_t out_at = stages * stage_bytes;
  static constexpr uint32_t smem = out_at + 8 * warp_out + 1024;  // + room to align to 1024
  static constexpr int width = dual ? TN / 2 : TN;                // output columns of a tile
  static constexpr uint32_t tmem_cols = precise ? 512 : 2 * TN;
  static_assert(tmem_cols <= 512 && stages >= 4, "tensor memory, stages");
  static_assert((uint32_t)stages * stage_bytes >= 128u * TN * 4, "the ring holds a tile of sums");
  // the 16 bytes `q` of row `row` of a piece, where the bulk copy's swizzle expects them
  static __device__ __forceinline__ int at(int row, int q) {
    return row * piece_row + ((piece_row == 128 ? q ^ (row & 7) : q ^ ((row >> 1) & 3)) << 4);
  }
};

struct Maps {
  CUtensorMap a[4], b[3], out[3];
};

// A product: one result, or two of different A (z = 0, 1)
struct Part {
  int64_t m, n;             // rows and columns of the result (units, where dual)
  uint32_t m_tiles, n_tiles;
  uint32_t kb, segs, iters; // blocks of k per segment; of all segments
  uint32_t tail;            // instructions (k = 16) in the last block of a segment
  uint32_t a_mn, b_mn;      // MN-major operands
  uint32_t inst;            // instruction descriptor
  uint32_t seg_a, seg_b;    // operand of segment s: bits 4s.. (A: of the first result)
  uint32_t out;             // its first output
};

struct Params {
  Part part[2];
  uint32_t tiles, tiles0;   // of all results; of the first product's
  uint32_t heavy, later;    // two products: see Walk
  uint32_t band;            // tiles of rows that are walked through together, so that the blocks at work share operands in L2
  uint32_t split;
  uint32_t sums, buffers;   // accumulators of a tile, each of its part of k; tiles that are in tensor memory at a time
  uint32_t part_kb;         // long sums: blocks of k in a part
  uint32_t sym;             // the result is symmetric: tiles on and below the diagonal alone, each written to both of its places
  uint32_t act;
  uint32_t bulk;            // bit o: rows of output o start on 16-byte boundaries; bit 4 + o: ... and may be written up to one (bulk copies
                            // write whole units of 16 bytes, also where a row ends inside one)
  void* out[3];
  int64_t out_ld[3];
  const void* c0;           // kGatedBack: gradient of h; kPair*: high words of C, or NULL
  const void* c1;           // low words of C
  int64_t c_ld;
  uint32_t c_vec;           // rows of c0 start on 16-byte boundaries
  float alpha, beta;        // alpha has C's scale in it, beta the product's; both the result's
  uint32_t* status;
};
static_assert(sizeof(Maps) + sizeof(Params) <= 4000, "the kernel's parameter space");

// ------------------------------------------------------------------ instructions ----

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// the address of the same place in the shared memory of block `rank` of the cluster
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void peer_load(uint32_t addr, float* v) {
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void peer_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// a tile into this block's memory; the barrier may be the pair's other block's
template <int CTAS>
__device__ __forceinline__ void tile_load(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint32_t bar) {
  if constexpr (CTAS == 1) {
    tma_load(dst, map, x, y, bar);
  } else {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
  }
}

// Shared-memory matrix descriptors, 128-byte swizzle. K-major: groups of 8 rows 1024 bytes apart. MN-major: boxes of 64 elements x 64 k,
// 8192 bytes apart, groups of 8 k 1024 bytes apart. (In a cluster an address in shared memory has the block's rank above its 18 bits.)
constexpr uint32_t kDescHi = 64u | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t mn) { return ((addr & 0x3FFFFu) >> 4) | ((mn ? 512u : 1u) << 16); }

template <int CTAS>
__device__ __forceinline__ void mma16(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t inst, uint32_t add) {
  if constexpr (CTAS == 1)
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "mov.b64 a, {%1, %5};\n\t"
                 "mov.b64 b, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d),
                 "r"(a_lo), "r"(b_lo), "r"(inst), "r"(add), "n"(kDescHi)
                 : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "mov.b64 a, {%1, %5};\n\t"
                 "mov.b64 b, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d),
                 "r"(a_lo), "r"(b_lo), "r"(inst), "r"(add), "n"(kDescHi)
                 : "memory");
}
// arrives at the barrier (of both blocks of a pair) when the products issued so far are done
template <int CTAS>
__device__ __forceinline__ void commit(uint32_t bar, uint32_t mask) {
  if constexpr (CTAS == 1)
    mma_commit(bar);
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"((uint16_t)mask)
                 : "memory");
}

// 16 columns of two and of four sums, `apart` columns from one to the next: while products are under way a load takes 0.4 us to come back
__device__ __forceinline__ void tmem_load16x2(uint32_t addr, uint32_t apart, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%32];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%33];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
        "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr), "r"(addr + apart)
      : "memory");
}
__device__ __forceinline__ void tmem_load16x4(uint32_t addr, uint32_t apart, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%64];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%65];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47}, [%66];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%67];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
        "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]), "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]),
        "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]),
        "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]),
        "=r"(r[54]), "=r"(r[55]), "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]),
        "=r"(r[63])
      : "r"(addr), "r"(addr + apart), "r"(addr + 2 * apart), "r"(addr + 3 * apart)
      : "memory");
}

// ------------------------------------------------------------------ activations ----

// erfc(z), called: 32 copies of it in a row would not fit the instruction cache
static __device__ __noinline__ float erfc_of(float z) { return erfcf(z); }

// 1 / (1 + e^-g), and e^-g: two instructions of the special functions, whose results are off by 2^-22; e^-g beyond fp32 gives 0
__device__ __forceinline__ float2 sigmoid2(float2 g, float2* e) {
  const float2 t = mul2(g, both(-1.4426950408889634f));
  float2 s;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e->x) : "f"(t.x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e->y) : "f"(t.y));
  const float2 d = add2(*e, both(1.f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s.x) : "f"(d.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s.y) : "f"(d.y));
  return s;
}

// act(g) of two gates, and its derivative. What the functions are off by (2^-17 of themselves where e^-g is large, 2^-21 in the middle) is far
// below a 16-bit result's rounding.
template <int ACT, bool SLOPE>
__device__ __forceinline__ float2 gate2(float2 g, float2* slope) {
  if constexpr (ACT == MFET_ACT_RELU) {
    float2 r = g;
    asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(r.x));
    asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(r.y));
    if (SLOPE) *slope = make_float2(g.x > 0.f ? 1.f : 0.f, g.y > 0.f ? 1.f : 0.f);
    return r;
  } else if constexpr (ACT == MFET_ACT_SILU) {
    float2 e;
    const float2 s = sigmoid2(g, &e);
    // 1 - s may cancel here: where it does, it stands beside 1
    if (SLOPE) *slope = mul2(s, fma2(g, fma2(s, both(-1.f), both(1.f)), both(1.f)));
    return mul2(g, s);
  } else if constexpr (ACT == MFET_ACT_SIGMOID) {
    float2 e;
    const float2 s = sigmoid2(g, &e);
    if (SLOPE) {  // s (1 - s), with 1 - s as e^-g s where it would cancel (from g = 12 on it was off by 1 %, from 17 on 0)
      const float2 c = fma2(s, both(-1.f), both(1.f)), d = mul2(e, s);
      *slope = mul2(s, make_float2(g.x > 0.f ? d.x : c.x, g.y > 0.f ? d.y : c.y));
    }
    return s;
  } else if constexpr (ACT == MFET_ACT_GELU) {
    const float2 z = mul2(g, both(-0.70710678118654752f));
    const float2 c = mul2(make_float2(erfc_of(z.x), erfc_of(z.y)), both(0.5f));  // no cancellation for negative g
    if (SLOPE) {
      const float2 d = make_float2(__expf(-0.5f * g.x * g.x), __expf(-0.5f * g.y * g.y));
      *slope = fma2(mul2(g, both(0.3989422804014327f)), d, c);
    }
    return mul2(g, c);
  } else {
    if (SLOPE) *slope = both(1.f);
    return g;
  }
}

// 32 gates `v` and up units `u` to results, two an instruction: h in v; or, with the gradient x of h beside them, dG in v and dU in u. (One
// at a time: 87 cycles a gate and SM quarter, backward, as much as the products take.)
template <int ACT, bool BACK>
__device__ __forceinline__ void gates32(float* v, float* u, const float* x) {
#pragma unroll
  for (int j = 0; j < 32; j += 2) {
    const float2 g = make_float2(v[j], v[j + 1]), w = make_float2(u[j], u[j + 1]);
    if constexpr (BACK) {
      float2 slope;
      const float2 a = gate2<ACT, true>(g, &slope), d = make_float2(x[j], x[j + 1]);
      const float2 dg = mul2(mul2(d, w), slope), du = mul2(d, a);
      v[j] = dg.x, v[j + 1] = dg.y;
      u[j] = du.x, u[j + 1] = du.y;
    } else {
      const float2 h = mul2(gate2<ACT, false>(g, nullptr), w);
      v[j] = h.x, v[j + 1] = h.y;
    }
  }
}
template <bool BACK>
__device__ __forceinline__ void gates32(uint32_t act, float* v, float* u, const float* x) {
  switch (act) {  // once per 32 columns: a choice per value made the code outgrow the instruction cache (8192 x 896 x 1024 backward: 71 us)
    case MFET_ACT_RELU: return gates32<MFET_ACT_RELU, BACK>(v, u, x);
    case MFET_ACT_SILU: return gates32<MFET_ACT_SILU, BACK>(v, u, x);
    case MFET_ACT_GELU: return gates32<MFET_ACT_GELU, BACK>(v, u, x);
    case MFET_ACT_SIGMOID: return gates32<MFET_ACT_SIGMOID, BACK>(v, u, x);
    default: return gates32<MFET_ACT_NONE, BACK>(v, u, x);
  }
}

// ------------------------------------------------------------------ the kernel ----

struct Tile {
  uint32_t z, tm, tn, part;
};
template <bool TWO>
__device__ __forceinline__ Tile tile_at(const Params& p, uint32_t t) {
  if (p.sym) {  // row by row: r (r + 1) / 2 tiles lie ahead of row r
    uint32_t r = (uint32_t)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while ((uint64_t)r * (r + 1) / 2 > t) --r;
    while ((uint64_t)(r + 1) * (r + 2) / 2 <= t) ++r;
    return {0, r, t - r * (r + 1) / 2, 0};
  }
  const uint32_t part = TWO && t >= p.tiles0 ? 1 : 0;
  if (part) t -= p.tiles0;
  const Part& q = p.part[part];
  const uint32_t per = q.m_tiles * q.n_tiles, z = t / per, r = t - z * per;
  const uint32_t band = r / (p.band * q.n_tiles), in = r - band * p.band * q.n_tiles;
  const uint32_t rows = min(p.band, q.m_tiles - band * p.band);
  const uint32_t tn = in / rows;
  return {z, band * p.band + (in - tn * rows), tn, part};
}

// The tiles of a block (pair), one after the other: each `step`-th. TWO: the first product's tiles are the longer ones and go first, the blocks
// below `heavy` get one more of them than the others; the second's fill up round by round, and in the first `later` rounds the heavy
// blocks are still busy and take none.
template <bool TWO>
struct Walk {
  const Params& p;
  uint32_t first, step, own;
  __device__ __forceinline__ Walk(const Params& p_, uint32_t first_, uint32_t step_) : p(p_), first(first_), step(step_) {
    own = TWO ? p.tiles0 / step + (first < p.heavy) : 0;
  }
  // tile k, or one beyond the last
  __device__ __forceinline__ uint32_t operator()(uint32_t k) const {
    if (!TWO || k < own) return first + k * step;
    const bool heavy = first < p.heavy;
    const uint32_t light = step - p.heavy, round = k - own + (heavy ? p.later : 0), place = heavy ? light + first : first - p.heavy;
    return p.tiles0 + (round < p.later ? round * light + place : p.later * light + (round - p.later) * step + place);
  }
};

// 32 neighbouring 16-bit values of a row on its way to registers, 0 behind its end. vec: rows start on 16-byte boundaries.
struct Row32 {
  uint4 w[4];
};
__device__ __forceinline__ void fetch_row32(const void* base, int64_t at, int64_t left, uint32_t vec, Row32* r) {
  const uint16_t* p = reinterpret_cast<const uint16_t*>(base) + at;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (vec && left >= 8 * q + 8) {
      r->w[q] = *reinterpret_cast<const uint4*>(p + 8 * q);
    } else {
      uint32_t v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 8 * q + j < left ? p[8 * q + j] : 0;
      r->w[q] = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
    }
  }
}

template <int CTAS, int TN, int MODE, int DT>
__global__ void __launch_bounds__(kThreads, 1) gemm16_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Params p) {
  using G = Shape<CTAS, TN, MODE, DT>;
  using T = typename Elem<DT>::T;
  extern __shared__ uint8_t raw_smem[];
  __shared__ __align__(8) uint64_t bars[2 * G::stages + 5];
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int dead;
  const uint32_t base = (smem_addr(raw_smem) + 1023) & ~1023u;  // the same in all blocks
  uint8_t* const smem = raw_smem + (base - smem_addr(raw_smem));
  const uint32_t bar0 = smem_addr(bars);
  auto full = [&](int s) { return bar0 + 8 * s; };
  auto empty = [&](int s) { return bar0 + 8 * (G::stages + s); };
  auto acc_full = [&](int a) { return bar0 + 8 * (2 * G::stages + a); };
  auto acc_empty = [&](int a) { return bar0 + 8 * (2 * G::stages + 2 + a); };
  const uint32_t drained = bar0 + 8 * (2 * G::stages + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool clustered = CTAS * p.split > 1;
  const uint32_t rank = clustered ? cluster_rank() : 0u;
  const uint32_t part = rank / CTAS, half = rank % CTAS, leader = rank - half;
  const uint32_t pair_mask = (CTAS == 2 ? 3u : 1u) << leader;

  if (threadIdx.x == 64) {
    prefetch_map(&maps.a[p.part[0].seg_a & 15u]);
    prefetch_map(&maps.b[p.part[0].seg_b & 15u]);
    if (G::dual || (p.part[0].seg_b >> 4)) prefetch_map(&maps.b[1]);
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < G::stages; ++s) bar_init(full(s), 1), bar_init(empty(s), 1);
    for (int a = 0; a < 2; ++a) bar_init(acc_full(a), 1), bar_init(acc_empty(a), 8 * CTAS);
    bar_init(drained, 1);
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    if constexpr (CTAS == 1) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_slot)), "n"(G::tmem_cols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_slot)), "n"(G::tmem_cols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (clustered) cluster_sync();  // the barriers of the other blocks exist, and so do the blocks
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  early_launch_wait();

  const uint32_t members = CTAS * p.split;
  constexpr bool kTwo = is_two<MODE>, kLong = is_long<MODE>;
  const uint32_t first = blockIdx.x / members;
  const Walk<kTwo> walk(p, first, gridDim.x / members);
  auto share_begin = [&](const Part& q) { return (uint32_t)((uint64_t)q.kb * part / p.split); };  // this block's share of k, in each segment
  auto share_end = [&](const Part& q) { return (uint32_t)((uint64_t)q.kb * (part + 1) / p.split); };
  // sums of a tile that are each of a part of `len` blocks of k (one more holds the products with low words, where they come together)
  auto sums_for = [&](uint32_t len) { return G::precise ? min(p.sums - (G::fused ? 1u : 0u), len) : 1u; };

  uint64_t filled = 0;  // stages that this lane has asked for
  bool issues = false;  // this lane issues the products
  if (warp == 0) {
    if (elect_one()) {
      uint32_t st = 0, phase = 1;  // an empty barrier's phase before the first is taken as complete
      bool ok = true;
      uint32_t turn = 0;
      for (uint32_t t = walk(0); ok && t < p.tiles; t = walk(++turn)) {
        const Tile w = tile_at<kTwo>(p, t);
        const Part& q = p.part[kTwo ? w.part : 0];
        const uint32_t k0 = share_begin(q), k1 = share_end(q);
        const int32_t row = (int32_t)((w.tm * CTAS + half) * 128);
        uint32_t seg = 0, kk = k0, from = k0, to = kLong ? min(k0 + p.part_kb, k1) : k1;  // of a part
        for (uint32_t i = (k1 - k0) * (G::fused ? 1 : q.segs); i > 0; --i) {
          if (!(ok = bar_sleep(empty(st), phase, &dead))) break;
          // tiles and blocks of k outside their matrix read as 0
          if (!MFET_INSIDE(p.status, seg < 3 && w.z < 2 && (int64_t)row < q.m + 128 && w.tn < q.n_tiles)) {
            ok = false;
            dead = 1;
            break;
          }
          const uint32_t at = base + st * G::stage_bytes;
          const uint32_t bar = CTAS == 1 ? full(st) : peer_addr(full(st), leader);
          if (half == 0) bar_expect(full(st), CTAS * G::stage_bytes);
          const int32_t k = (int32_t)(kk * kSlab);
          auto load_a = [&](const CUtensorMap* a, uint32_t to) {
            if (q.a_mn) {
              tile_load<CTAS>(to, a, row, k, bar);
              tile_load<CTAS>(to + 8192, a, row + 64, k, bar);
            } else {
              tile_load<CTAS>(to, a, k, row, bar);
            }
          };
          auto load_b = [&](const CUtensorMap* b, uint32_t to) {
            const int32_t col = (int32_t)(w.tn * TN + half * G::b_rows);
            if (q.b_mn) {
#pragma unroll
              for (int j = 0; j < G::b_rows / 64; ++j) tile_load<CTAS>(to + 8192 * j, b, col + 64 * j, k, bar);
            } else {
              tile_load<CTAS>(to, b, k, col, bar);
            }
          };
          if constexpr (G::fused) {
            load_a(&maps.a[0], at);
            load_a(&maps.a[1], at + G::a_bytes);
            load_b(&maps.b[0], at + 2 * G::a_bytes);
            load_b(&maps.b[1], at + 2 * G::a_bytes + G::b_bytes);
          } else {
            load_a(&maps.a[((q.seg_a >> (4 * seg)) & 15u) + w.z], at);
            if constexpr (G::dual) {
              const int32_t unit = (int32_t)(w.tn * G::width);
              if constexpr (CTAS == 2) {
                tile_load<CTAS>(at + G::a_bytes, &maps.b[half], k, unit, bar);
              } else {
                tile_load<CTAS>(at + G::a_bytes, &maps.b[0], k, unit, bar);
                tile_load<CTAS>(at + G::a_bytes + G::b_bytes / 2, &maps.b[1], k, unit, bar);
              }
            } else {
              load_b(&maps.b[(q.seg_b >> (4 * seg)) & 15u], at + G::a_bytes);
            }
          }
          ++filled;
          if (++st == (uint32_t)G::stages) st = 0, phase ^= 1;
          if (++kk == to) {
            kk = from, ++seg;
            if (kLong && seg == (G::fused ? 1 : q.segs)) seg = 0, kk = from = to, to = min(to + p.part_kb, k1);
          }
        }
      }
    }
  } else if (warp == 1) {
    if (half == 0 && elect_one()) {
      issues = true;
      uint32_t st = 0, phase = 0, done = 0, unit = 0;  // unit: accumulators used so far, one a tile (a part)
      bool ok = true, ready = false;
      for (uint32_t t = walk(0); ok && t < p.tiles; t = walk(++done)) {
        const Part& q = p.part[kTwo && t >= p.tiles0 ? 1 : 0];
        const uint32_t a_step = q.a_mn ? 128u : 2u, b_step = q.b_mn ? 128u : 2u, end = share_end(q);
        uint32_t k0 = share_begin(q);
        do {
          const uint32_t k1 = kLong ? min(k0 + p.part_kb, end) : end;
          const uint32_t acc = unit % p.buffers;
          if (unit >= p.buffers && !(ok = bar_wait(acc_empty(acc), (unit / p.buffers - 1) & 1, &dead))) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t len = k1 - k0, sums = sums_for(len);
          uint32_t kk = k0, left = len * (G::fused ? 1 : q.segs), sum = 0, fresh = 1, of_sum = 0;  // fresh: nothing has been added to this sum yet
          for (uint32_t i = 0; left > 0; ++i) {
            if (!ready && !(ok = bar_wait(full(st), phase, &dead))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t at = base + st * G::stage_bytes;
            const uint32_t this_empty = empty(st);
            const uint32_t a_lo = desc_lo(at, q.a_mn), b_lo = desc_lo(at + (G::fused ? 2 : 1) * G::a_bytes, q.b_mn);
            const uint32_t first_sum = tmem + acc * (G::precise ? p.sums : 1u) * TN, d = first_sum + sum * TN, add = !fresh;
            const bool last = kk + 1 == q.kb;
            if (++st == (uint32_t)G::stages) st = 0, phase ^= 1;
            if constexpr (G::fused) {  // high x low, low x high to a sum of their own, high x high to this part's
              const uint32_t steps = last ? q.tail : 4u, low = first_sum + sums * TN, a2 = a_lo + (G::a_bytes >> 4), b2 = b_lo + (G::b_bytes >> 4);
              for (uint32_t j = 0; j < steps; ++j) mma16<CTAS>(low, a_lo + j * a_step, b2 + j * b_step, q.inst, i | j);
              for (uint32_t j = 0; j < steps; ++j) mma16<CTAS>(low, a2 + j * a_step, b_lo + j * b_step, q.inst, 1);
              ready = bar_try(full(st), phase);
              for (uint32_t j = 0; j < steps; ++j) mma16<CTAS>(d, a_lo + j * a_step, b_lo + j * b_step, q.inst, add | j);
            } else if (!last || q.tail == 4) {
              mma16<CTAS>(d, a_lo, b_lo, q.inst, add);
              mma16<CTAS>(d, a_lo + a_step, b_lo + b_step, q.inst, 1);
              ready = bar_try(full(st), phase);
              mma16<CTAS>(d, a_lo + 2 * a_step, b_lo + 2 * b_step, q.inst, 1);
              mma16<CTAS>(d, a_lo + 3 * a_step, b_lo + 3 * b_step, q.inst, 1);
            } else {
              for (uint32_t j = 0; j < q.tail; ++j) mma16<CTAS>(d, a_lo + j * a_step, b_lo + j * b_step, q.inst, add | j);
              ready = bar_try(full(st), phase);
            }
            commit<CTAS>(this_empty, pair_mask);
            if (--left == 0) commit<CTAS>(acc_full(acc), pair_mask);
            fresh = 0;
            ++kk;
            if constexpr (G::precise) {
              of_sum += sums;  // block kk - k0 belongs to sum (kk - k0) * sums / len
              if (of_sum >= len) of_sum -= len, ++sum, fresh = i + 1 < len;
            }
            if (kk == k1) kk = k0, sum = 0, of_sum = 0;
          }
          k0 = k1;
          ++unit;
        } while (kLong && ok && k0 < end);
      }
    }
  }
  const int quarter = warp & 3;            // the 32 lanes of tensor memory that this warp may read
  const int second = warp >= 6 ? 1 : 0;    // two warps share them and take every other 32 columns
  uint8_t* const out_ptr = smem + G::out_at + (warp - 2) * G::warp_out;
  const uint32_t out_at = base + G::out_at + (warp - 2) * G::warp_out;
  uint32_t turn = 0;
  const Part* q = &p.part[0];  // of the tile that is written
  // 32 columns `v` of this lane's row, from column j1 on, to output o of the result (i0: the warp's first row)
  auto put = [&](float* v, int o, int64_t i0, int64_t j1) {
    constexpr int kPer = 16 / (int)sizeof(T);  // values per 16 bytes
    const uint32_t piece = (turn * G::outs + (G::outs == 2 ? o : 0)) * G::piece;
    uint8_t* const to = out_ptr + piece;
#pragma unroll
    for (int c = 0; c < 32; c += kPer) *reinterpret_cast<uint4*>(to + G::at(lane, c / kPer)) = narrow16<DT>(v + c);
    if (((p.bulk >> o) & 1) && (j1 + 32 <= q->n || ((p.bulk >> o) & 16))) {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (i0 < q->m && j1 < q->n && elect_one()) bulk_store(&maps.out[o], out_at + piece, (int32_t)j1, (int32_t)i0);
      __syncwarp();
    } else {
      __syncwarp();
      const int64_t ld = p.out_ld[o];
      T* y = reinterpret_cast<T*>(p.out[o]) + i0 * ld + j1 + lane;
      const int rows = j1 + lane < q->n && MFET_INSIDE(p.status, i0 >= 0 && j1 >= 0 && j1 + lane < ld) ? (int)(q->m - i0 < 32 ? q->m - i0 : 32) : 0;
#pragma unroll
      for (int i = 0; i < 32; ++i, y += ld) {  // a warp writes a row's 32 columns
        const T x = *reinterpret_cast<const T*>(to + G::at(i, lane / kPer) + lane % kPer * sizeof(T));
        if (i < rows) *y = x;
      }
      __syncwarp();
    }
  };
  // the same with rows and columns exchanged (of a symmetric result, which has bulk copies)
  auto put_mirror = [&](const float* v, int o, int64_t i0, int64_t j1) {
    if constexpr (is_pair<MODE>) {
      const uint32_t piece = (turn * G::outs + o) * G::piece;
#pragma unroll
      for (int j = 0; j < 32; ++j) *reinterpret_cast<T*>(out_ptr + piece + G::at(j, lane >> 3) + (lane & 7) * sizeof(T)) = Elem<DT>::from(v[j]);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (i0 < q->m && j1 < q->n && elect_one()) bulk_store(&maps.out[o], out_at + piece, (int32_t)i0, (int32_t)j1);
      __syncwarp();
    }
  };
  auto put_begin = [&]() {  // what the memory of the pieces held before has left
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(G::turns - 1) : "memory");
    __syncwarp();
  };
  auto put_end = [&]() {
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    if (G::turns == 2) turn ^= 1;
  };
  // what becomes of 32 columns of the accumulator (and of the same units' other half, where dual): x is what c0 (c1) held there
  auto finish = [&](float* v, float* u, float* x, int z, int64_t i0, int64_t j1, bool mirror) {
    put_begin();
    if constexpr (MODE == kGated) {
      gates32<false>(p.act, v, u, x);
      put(v, 0, i0, j1);
    } else if constexpr (MODE == kGatedBack) {
      gates32<true>(p.act, v, u, x);
      put(v, 0, i0, j1);
      put(u, 1, i0, j1);
    } else if constexpr (!G::precise) {
      put(v, (int)q->out + z, i0, j1);
    } else {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = fmaf(v[j], p.beta, x[j] * p.alpha);
      if constexpr (is_pair<MODE>) {
#pragma unroll
        for (int j = 0; j < 32; ++j) x[j] = v[j] - __half2float(__float2half_rn(v[j]));
        put(v, 0, i0, j1);
        put(x, 1, i0, j1);
        if (mirror) {
          put_end();
          put_begin();
          put_mirror(v, 0, i0, j1);
          put_mirror(x, 1, i0, j1);
        }
      } else {
        put(v, 0, i0, j1);
      }
    }
    put_end();
  };
  // What stands beside 32 columns of row i: asked for a chunk ahead (waiting for it took longer than all else that is done with a chunk: 4.4 us
  // a tile of 128 x 64 units, backward, where its products take 2.2)
  constexpr bool kBeside = MODE == kGatedBack || G::precise;
  constexpr int kBesides = G::precise ? 2 : 1;
  auto ask = [&](Row32* r, int64_t i, int64_t j1) {
    if constexpr (kBeside) {
      if (i < q->m && j1 < q->n && p.c0 && MFET_INSIDE(p.status, j1 >= 0 && i >= 0)) {
        fetch_row32(p.c0, i * p.c_ld + j1, q->n - j1, p.c_vec, r);
        if constexpr (kBesides == 2) fetch_row32(p.c1, i * p.c_ld + j1, q->n - j1, p.c_vec, r + 1);
      } else {
        memset(r, 0, kBesides * sizeof(Row32));
      }
    }
  };
  auto got = [&](const Row32* r, float* x) {
    if constexpr (kBeside) {
      constexpr int kType = MODE == kGatedBack ? DT : MFET_F16;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        widen16<kType>(r->w[q], x + 8 * q);
        if constexpr (kBesides == 2) {
          float lo[8];
          widen16<kType>(r[1].w[q], lo);
#pragma unroll
          for (int j = 0; j < 8; ++j) x[8 * q + j] += lo[j];
        }
      }
    }
  };
  if (warp >= 2) {
    uint32_t done = 0;
    Row32 next[kBesides];
    const uint32_t sums = sums_for(share_end(p.part[0]) - share_begin(p.part[0])) + (G::fused ? 1 : 0);
    auto sums_of = [&](uint32_t at, uint32_t* r) {  // 32 columns of a tile: its sums in their order
      tmem_load32(at, r);
      if constexpr (G::precise) {
        for (uint32_t z = 1; z < sums; ++z) {
          uint32_t t[32];
          tmem_load32(at + z * TN, t);
#pragma unroll
          for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) + __uint_as_float(t[j]));
        }
      }
    };
    auto row_of = [&](const Tile& w) { return (int64_t)(w.tm * CTAS + half) * 128 + quarter * 32; };
    if (p.split == 1 && first < p.tiles) {
      const Tile w = tile_at<false>(p, first);
      ask(next, row_of(w) + lane, (int64_t)w.tn * G::width + 32 * second);
    }
    uint32_t unit = 0;
    for (uint32_t t = walk(0); t < p.tiles; t = walk(++done)) {
      const Tile w = tile_at<kTwo>(p, t);
      if constexpr (kTwo) q = &p.part[w.part];
      const uint32_t len = share_end(*q) - share_begin(*q), parts = kLong ? (len + p.part_kb - 1) / p.part_kb : 1;
      if (kLong && parts > 1) {  // a tile's parts in their order, added up in registers while the next one is computed
        constexpr int kChunks = G::width / 64;
        // (64 columns leave room for fp64, whose additions cost nothing beside the products: the longest sums are the narrowest ones)
        std::conditional_t<G::fused, double, float> v[kChunks][32];
        bool ok = true;
        for (uint32_t n = 0; n < parts; ++n, ++unit) {
          const uint32_t acc = unit % p.buffers;
          ok = __all_sync(kAllLanes, bar_sleep(acc_full(acc), (unit / p.buffers) & 1, &dead));
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
          for (int c = 0; c < kChunks; ++c) {
            const uint32_t from = tmem + acc * (G::precise ? p.sums : 1u) * TN + ((uint32_t)(quarter * 32) << 16) + 32 * second + 64 * c;
            if constexpr (G::precise) {
              constexpr int kSums = G::fused ? 4 : 2;  // Params::sums; the last part may have fewer
              const uint32_t sums = sums_for(min(p.part_kb, len - n * p.part_kb)) + (G::fused ? 1 : 0);
#pragma unroll
              for (int h = 0; h < 32; h += 16) {
                uint32_t r[16 * kSums];
                if constexpr (G::fused) tmem_load16x4(from + h, TN, r);
                else tmem_load16x2(from + h, TN, r);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                  float t = __uint_as_float(r[j]);
#pragma unroll
                  for (int z = 1; z < kSums; ++z) t += z < sums ? __uint_as_float(r[16 * z + j]) : 0.f;
                  v[c][h + j] = n ? v[c][h + j] + t : t;
                }
              }
            } else {
              uint32_t r[32];
              tmem_load32(from, r);
#pragma unroll
              for (int j = 0; j < 32; ++j) v[c][j] = n ? v[c][j] + __uint_as_float(r[j]) : __uint_as_float(r[j]);
            }
          }
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            if constexpr (CTAS == 1) bar_arrive(acc_empty(acc));
            else peer_arrive(peer_addr(acc_empty(acc), leader));
          }
        }
        if (!ok) break;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          const int c0 = 32 * second + 64 * c;
          float r[32], x[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) r[j] = (float)v[c][j];
          if (p.split > 1) {
#pragma unroll
            for (int j = 0; j < 32; j += 4)
              *reinterpret_cast<float4*>(smem + (((c0 + j) >> 2) * 128 + quarter * 32 + lane) * 16) = make_float4(r[j], r[j + 1], r[j + 2], r[j + 3]);
          } else {
            const int64_t i0 = row_of(w), j1 = (int64_t)w.tn * G::width + c0;
            ask(next, i0 + lane, j1);
            got(next, x);
            finish(r, nullptr, x, (int)w.z, i0, j1, p.sym && w.tm != w.tn);
          }
        }
        if (p.split > 1) break;
        continue;
      }
      const uint32_t acc = unit % p.buffers;
      const int64_t i0 = row_of(w), j0 = (int64_t)w.tn * G::width;
      const uint32_t from = tmem + acc * (G::precise ? p.sums : 1u) * TN + ((uint32_t)(quarter * 32) << 16);
      const bool ok = bar_sleep(acc_full(acc), (unit / p.buffers) & 1, &dead);
      ++unit;
      if (!__all_sync(kAllLanes, ok)) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      if (p.split > 1) {  // one tile per block: its sums go to shared memory, where the ring was
#pragma unroll 1
        for (int c = 32 * second; c < TN; c += 64) {
          uint32_t r[32];
          sums_of(from + c, r);
#pragma unroll
          for (int j = 0; j < 32; j += 4)
            *reinterpret_cast<uint4*>(smem + (((c + j) >> 2) * 128 + quarter * 32 + lane) * 16) = make_uint4(r[j], r[j + 1], r[j + 2], r[j + 3]);
        }
        break;
      }
#pragma unroll 1
      for (int c = 32 * second; c < G::width; c += 64) {
        uint32_t r[32], r2[32];
        float x[32];
        sums_of(from + c, r);
        if constexpr (G::dual) tmem_load32(from + G::width + c, r2);
        got(next, x);
        if (c + 64 < G::width) {
          ask(next, i0 + lane, j0 + c + 64);
        } else {  // the accumulator is read: the next tile but one may overwrite it
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            if constexpr (CTAS == 1) bar_arrive(acc_empty(acc));
            else peer_arrive(peer_addr(acc_empty(acc), leader));
          }
          if (kBeside && walk(done + 1) < p.tiles) {
            const Tile v = tile_at<false>(p, walk(done + 1));
            ask(next, row_of(v) + lane, (int64_t)v.tn * G::width + 32 * second);
          }
        }
        finish(reinterpret_cast<float*>(r), reinterpret_cast<float*>(r2), x, (int)w.z, i0, j0 + c, p.sym && w.tm != w.tn);
      }
    }
  }
  __syncwarp();  // the one lane that loaded or issued rejoins its warp
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (clustered) cluster_sync();  // of a split: all sums are in shared memory
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (p.split > 1) {
    if (warp >= 2 && !dead && first < p.tiles) {
      const Tile w = tile_at<kTwo>(p, first);
      const int64_t i0 = (int64_t)(w.tm * CTAS + half) * 128 + quarter * 32, j0 = (int64_t)w.tn * G::width;
      const int share = G::width / (int)p.split;
#pragma unroll 1
      for (int c = (int)part * share + 32 * second; c < (int)(part + 1) * share; c += 64) {
        float x[32], v[32], u[32], t[32];
        // the sums of one part after the other: of columns `from` on, four columns of a row in 16 bytes
        auto fetch = [&](float* to, uint32_t s, int from) {
          const uint32_t src = peer_addr(base + ((from >> 2) * 128 + quarter * 32 + lane) * 16, s * CTAS + half);
#pragma unroll
          for (int j = 0; j < 32; j += 4) peer_load(src + j * 512, to + j);
        };
        Row32 beside[kBesides];
        ask(beside, i0 + lane, j0 + c);
        fetch(v, 0, c);
        if constexpr (G::dual) fetch(u, 0, G::width + c);
        for (uint32_t s = 1; s < p.split; ++s) {
          fetch(t, s, c);
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] += t[j];
          if constexpr (G::dual) {
            fetch(t, s, G::width + c);
#pragma unroll
            for (int j = 0; j < 32; ++j) u[j] += t[j];
          }
        }
        got(beside, x);
        finish(v, u, x, (int)w.z, i0, j0 + c, p.sym && w.tm != w.tn);
      }
    }
    __syncwarp();
    cluster_sync();  // nobody's shared memory goes while another block reads it
  }
  if (warp >= 2) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // shared memory outlives the copies that read it
  // Without a stall every copy and product has been waited for by the role that needed it. After one, whoever was ahead of the role that
  // gave up has left some under way: all roles have ended here, so what is waited for now (with the same limit) is the last of them.
  if (dead) {
    volatile int none = 0;
    if (half == 0) {
      const uint64_t from = filled > G::stages ? filled - G::stages : 0;
      for (uint64_t i = from; i < filled; ++i) bar_wait(full(i % G::stages), (i / G::stages) & 1, &none);
    }
    if (issues) {
      commit<CTAS>(drained, pair_mask);
      bar_wait(drained, 0, &none);
    }
    if (threadIdx.x == 0 && p.status) atomicOr(p.status, (uint32_t)MFET_DEV_STALLED);
  }
  __syncthreads();
  if (clustered) cluster_sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 1) {
    if constexpr (CTAS == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(G::tmem_cols));
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(G::tmem_cols));
  }
}

// ------------------------------------------------------------------ host side ----

// `outer` rows of `inner` neighbouring 16-bit values, `ld` apart
struct Matrix {
  const void* p;
  int64_t inner, outer, ld;
  bool spare = false;  // what lies between its rows is the library's own
};

inline bool tile_map(CUtensorMap* map, const Matrix& x, uint32_t dtype, uint32_t rows, uint32_t cols, CUtensorMapSwizzle swizzle, bool load) {
  const EncodeTiled f = encode_tiled();
  if (!f) return false;
  const uint32_t size = size_of(dtype);
  const int64_t ld = x.outer == 1 ? (x.inner * size + 15) / 16 * 16 / size : x.ld;  // of one row: not used
  const cuuint64_t dims[2] = {(cuuint64_t)x.inner, (cuuint64_t)x.outer}, stride[1] = {(cuuint64_t)ld * size};
  const cuuint32_t box[2] = {cols, rows}, ones[2] = {1, 1};
  const CUtensorMapDataType t = dtype == MFET_F32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                : dtype == MFET_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                    : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  return f(map, t, 2, const_cast<void*>(x.p), dims, stride, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
           load ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// may a bulk copy write (or read) its rows?
inline bool on_16(const Matrix& x, uint32_t dtype) {
  return aligned(x.p, 16) && (x.outer == 1 || (uint64_t)x.ld * size_of(dtype) % 16 == 0);
}

struct Problem {
  uint32_t dtype = MFET_F16;  // of the operands
  Matrix a[4] = {}, b[3] = {}, out[3] = {};
  int n_a = 1, n_b = 1, n_out = 1;
  uint32_t a_mn = 0, b_mn = 0;            // bit i: a[i] (b[i]) is MN-major
  int64_t k[2] = {0, 0};                  // of one segment, of each product
  int segs[2] = {1, 1}, results[2] = {1, 0};  // results of the second product: 0 where there is one product alone
  uint32_t out_dtype = MFET_F16;
  bool precise = false;                   // the two-word modes: for a result in fp32
  Params p = {};                          // sizes, majors and segments' operands of the products, epilogue
};

inline int64_t tiles_of(const Problem& q, int part, int64_t rows, int64_t cols) {
  const int64_t r = (q.p.part[part].m + rows - 1) / rows, c = (q.p.part[part].n + cols - 1) / cols;
  return q.p.sym ? r * (r + 1) / 2 : r * c * q.results[part];
}
inline int64_t iters_of(const Problem& q, int part) { return (q.k[part] + kSlab - 1) / kSlab * q.segs[part]; }

// rounds of the second product's tiles in which blocks with one more tile of the first take none
inline uint32_t rounds_later(uint32_t first, uint32_t second) { return (first + second / 2) / second; }

// Clusters of 1, 2, 4 or 8 blocks that the current GPU runs at a time (148 SMs are not 18 clusters of 8: parts of the chip have odd numbers
// of them; one cluster too many doubled a product's time).
template <auto Kernel>  // each kernel has its own answers
int64_t clusters_at_once(uint32_t members, uint32_t smem) {
  if (members == 1) return sm_count();
  static std::atomic<int> known[64][4];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return sm_count() / (members + 1);
  std::atomic<int>& k = known[dev][members == 2 ? 1 : members == 4 ? 2 : 3];
  n = k.load(std::memory_order_relaxed);
  if (n > 0) return n;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = members;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(members * (unsigned)sm_count());
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&n, Kernel, &cfg) != cudaSuccess || n < 1) {
    cudaGetLastError();
    return sm_count() / (members + 1);  // not remembered: asked again next time
  }
  k.store(n, std::memory_order_relaxed);
  return n;
}

template <int CTAS, int TN, int MODE, int DT>
int launch(const Problem& q, uint32_t split, cudaStream_t s) {
  using G = Shape<CTAS, TN, MODE, DT>;
  Maps maps;
  memset(&maps, 0, sizeof(maps));
  Params p = q.p;
  const CUtensorMapSwizzle sw = CU_TENSOR_MAP_SWIZZLE_128B;
  for (int i = 0; i < q.n_a; ++i)
    if (!tile_map(&maps.a[i], q.a[i], q.dtype, (q.a_mn >> i) & 1 ? 64 : 128, 64, sw, true)) return MFET_ERR_CUDA;
  for (int i = 0; i < q.n_b; ++i)
    if (!tile_map(&maps.b[i], q.b[i], q.dtype, (q.b_mn >> i) & 1 ? 64 : G::dual ? TN / 2 : G::b_rows, 64, sw, true)) return MFET_ERR_CUDA;
  p.bulk = 0;
  for (int i = 0; i < q.n_out; ++i) {
    p.out[i] = const_cast<void*>(q.out[i].p);
    p.out_ld[i] = q.out[i].ld;
    if (!on_16(q.out[i], q.out_dtype)) continue;
    p.bulk |= (q.out[i].spare || q.out[i].inner * size_of(q.out_dtype) % 16 == 0 ? 17u : 1u) << i;
    if (!tile_map(&maps.out[i], q.out[i], q.out_dtype, 32, 32, G::piece_row == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, false))
      return MFET_ERR_CUDA;
  }
  const uint32_t fmt = q.dtype == MFET_BF16 ? 1u : 0u;
  constexpr bool kTwo = is_two<MODE>;
  for (int i = 0; i < (kTwo ? 2 : 1); ++i) {
    Part& x = p.part[i];
    x.m_tiles = (uint32_t)((x.m + CTAS * 128 - 1) / (CTAS * 128));
    x.n_tiles = (uint32_t)((x.n + G::width - 1) / G::width);
    x.kb = (uint32_t)((q.k[i] + kSlab - 1) / kSlab);
    x.segs = (uint32_t)q.segs[i];
    x.iters = x.kb * x.segs;
    x.tail = (uint32_t)((q.k[i] - (int64_t)(x.kb - 1) * kSlab + 15) / 16);
    x.inst = (1u << 4) | (fmt << 7) | (fmt << 10) | (x.a_mn << 15) | (x.b_mn << 16) | ((uint32_t)(TN >> 3) << 17) | ((uint32_t)(CTAS * 128 >> 4) << 24);
    p.tiles += (uint32_t)tiles_of(q, i, CTAS * 128, G::width);
    if (i == 0) p.tiles0 = p.tiles;
  }
  p.band = 8;
  p.split = split;
  static std::atomic<uint64_t> ready{0};
  if (allow_smem(gemm16_kernel<CTAS, TN, MODE, DT>, G::smem, &ready) != cudaSuccess) return MFET_ERR_CUDA;
  const uint32_t members = CTAS * split, at_once = (uint32_t)clusters_at_once<gemm16_kernel<CTAS, TN, MODE, DT>>(members, G::smem);
  const uint32_t clusters = split > 1 || p.tiles < at_once ? p.tiles : at_once;
  p.sums = 1;
  p.buffers = 2;
  if (G::precise) {
    // The tensor cores truncate a sum at every instruction, and the products that an instruction adds to it beside each other. A sum of n instructions
    // ends up short by 0.27 n 2^-23 of its value where signs are random, 0.33 to 0.43 in updates that many samples share, 0.45 to 0.75 where all
    // terms have one sign (A X of 1024 x 896 to 2300 x 3000). Several sums of a part of k each, added up in fp32, lose as many times less; 0.25 of
    // it is put back. (2300 x 3000, error of one step 1.14e-6 of the result with 0.18, 0.76e-6 with 0.25, 0.57e-6 with 0.3, in fp32 0.38e-6; of five,
    // where large singular values end beside each other, 2.30, 2.47, 2.58 and 2.71e-6.) Results in fp32 are worth waiting with the next tile until
    // one is written.
    const bool one_tile = clusters == p.tiles;
    p.buffers = !is_long<MODE> && (one_tile || q.precise) ? 1 : 2;
    p.sums = 512 / TN / p.buffers;
    double len = (double)p.part[0].kb / split, most = p.sums - (G::fused ? 1 : 0), of = len < most ? len : most;
    if (is_long<MODE>) {  // two blocks of k a sum, and the next part's sums while these are added up
      p.part_kb = 2 * (uint32_t)most;
      len = 2 * (of = most);
    }
    p.beta = (float)(p.beta * (1.0 + 0.25 * 0x1p-23 * 4.0 * len / of));
  }
  if (kTwo) {
    p.heavy = p.tiles0 % clusters;
    p.later = p.heavy ? rounds_later(p.part[0].iters, p.part[1].iters) : 0;
  }
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = members;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(clusters * members);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = G::smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = members > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, gemm16_kernel<CTAS, TN, MODE, DT>, maps, p) == cudaSuccess ? MFET_OK : MFET_ERR_CUDA;
}

// The form for a problem: the least of the microseconds that were measured for each. A launch with a tile's start and end 6.9 for pairs, 4.2
// for blocks of 128 columns, 3.5 for 64; 64 of k 0.325 for 256 x 256 by a pair, 0.25 for 128 x 128 by a block and 0.2 for 64 columns (its loads
// bound it), 0.135 in each segment where three segments' tiles come together; joining two parts 3, four 6.
// Forward, k = 896, n = 1024: m = 1024 blocks 7.9, pairs 11.4; 8192 blocks 30.4, pairs 25.2. Backward 16384 x 2048 x 4096 1187 by pairs, 1803 by
// blocks. Orthogonalising 512 x 512: 125 with 64 columns, 183 with 128; 2048 x 2048: 538 by pairs, 920 by blocks, 966 with 64 columns.
template <int CTAS, int TN, int MODE, int DT>
double cost(const Problem& q, uint32_t split) {
  using G = Shape<CTAS, TN, MODE, DT>;
  const int64_t kb = (q.k[0] + kSlab - 1) / kSlab;
  if (split > 1 && (split * CTAS > 8 || split * 32 > (uint32_t)G::width || (int64_t)split > kb)) return 1e300;
  const int64_t tiles = tiles_of(q, 0, CTAS * 128, G::width);
  static std::atomic<uint64_t> ready{0};
  if (allow_smem(gemm16_kernel<CTAS, TN, MODE, DT>, G::smem, &ready) != cudaSuccess) return 1e300;
  const int64_t at_once = clusters_at_once<gemm16_kernel<CTAS, TN, MODE, DT>>(CTAS * split, G::smem), waves = (tiles + at_once - 1) / at_once;
  if (split > 1 && waves > 1) return 1e300;
  if (q.p.sym && CTAS * 128 != TN) return 1e300;  // tiles are exchanged with their mirror images
  return (CTAS == 2 ? 6.9 : TN == 128 ? 4.2 : 3.5) + (double)waves * ((kb + split - 1) / split) * q.segs[0] * (CTAS == 2 ? 0.325 : TN == 128 ? 0.25 : G::fused ? 0.135 : 0.2) + (split == 1 ? 0.0 : split == 2 ? 3.0 : 6.0);
}

// Two products in one launch, by pairs: the microseconds of it, as above
template <int MODE, int DT>
double cost_two(const Problem& q) {
  using G = Shape<2, 256, MODE, DT>;
  static std::atomic<uint64_t> ready{0};
  if (allow_smem(gemm16_kernel<2, 256, MODE, DT>, G::smem, &ready) != cudaSuccess) return 1e300;
  const int64_t pairs = clusters_at_once<gemm16_kernel<2, 256, MODE, DT>>(2, G::smem);
  const int64_t t0 = tiles_of(q, 0, 256, 256), t1 = tiles_of(q, 1, 256, 256), a = iters_of(q, 0), b = iters_of(q, 1);
  if (t0 + t1 < pairs || t0 + t1 >= (1ll << 31)) return 1e300;
  const int64_t heavy = t0 % pairs, light = pairs - heavy, later = heavy ? rounds_later((uint32_t)a, (uint32_t)b) : 0;
  const int64_t rest = t1 - later * light > 0 ? t1 - later * light : 0, rounds = (rest + pairs - 1) / pairs;  // that all take part in
  const int64_t of_light = t0 / pairs * a + (rest ? later + rounds : (t1 + light - 1) / light) * b;
  const int64_t of_heavy = heavy ? (t0 / pairs + 1) * a + (rest > light ? rounds : rounds > 0 ? rounds - 1 : 0) * b : 0;
  return 6.9 + 0.325 * (double)(of_light > of_heavy ? of_light : of_heavy);
}

// A symmetric result is computed by half where that saves a wave of tiles: writing a tile twice takes 0.8 (orthogonalising 256 x 256 with tiles of
// 128 columns, one wave either way: 138 by half, 123 without; 4096 x 2048: 833 by half, 985 without).
//
// Pairs have tensor memory for two sums of a tile, blocks for four. Where the result is fp32, pairs are left out if one would be of more than
// kSumOfPairs instructions, since truncation's scatter shows: 2048 x 2048 in five steps 5.5e-6 of the result and 538 us with pairs, 2.6e-6 and 610
// without (an iteration in fp32: 3.0e-6); 2048 x 4096 5.3e-6 and 867, 1.7e-6 and 1034; 1300 x 1200, 42 instructions, 1.6e-6 with pairs.
constexpr int kSumOfPairs = 44;
struct Choice {
  double cost;
  int form;  // 0: pairs, 1: blocks, 2: blocks of 64 columns
  uint32_t split, sym;
};
template <int MODE>
constexpr bool has_pairs = !(Shape<2, 256, MODE, MFET_F16>::precise && is_long<MODE>);  // no room for several sums and the next part's
template <int MODE, int DT>
Choice choose(const Problem& q) {
  Choice c{1e300, has_pairs<MODE> ? 0 : 1, 1, 0};
  for (uint32_t sym = 0; sym <= q.p.sym; ++sym) {
    Problem r = q;
    r.p.sym = sym;
    for (uint32_t part = 1; part <= 4; part *= 2) {
      if constexpr (has_pairs<MODE>) {
        const double pair = cost<2, 256, MODE, DT>(r, part) + 0.8 * sym;
        if (pair < c.cost && !(q.precise && (q.k[0] + kSlab - 1) / kSlab * 2 / part > kSumOfPairs)) c = {pair, 0, part, sym};
      }
      const double block = cost<1, 128, MODE, DT>(r, part) + 0.8 * sym;
      if (block < c.cost) c = {block, 1, part, sym};
      if constexpr (!Shape<1, 128, MODE, DT>::dual) {
        const double narrow = cost<1, 64, MODE, DT>(r, part);
        if (narrow < c.cost) c = {narrow, 2, part, sym};
      }
    }
  }
  return c;
}
template <int MODE, int DT>
double least_cost(const Problem& q) {
  return choose<MODE, DT>(q).cost;
}
template <int MODE, int DT>
int run(Problem q, cudaStream_t s) {
  const Choice c = choose<MODE, DT>(q);
  q.p.sym = c.sym;
  if constexpr (!Shape<1, 128, MODE, DT>::dual)
    if (c.form == 2) return launch<1, 64, MODE, DT>(q, c.split, s);
  if constexpr (has_pairs<MODE>)
    if (c.form == 0) return launch<2, 256, MODE, DT>(q, c.split, s);
  return launch<1, 128, MODE, DT>(q, c.split, s);
}

// ------------------------------------------------------------------ rows that no bulk copy can read ----

struct Pack {
  const uint16_t* src;
  uint8_t* dst;
  int64_t rows, cols, src_ld, dst_ld;
  int64_t first;  // of the units of all matrices
};
struct PackParams {
  Pack of[4];
  int64_t units;
};

// 16-bit rows at any address into rows on 16-byte boundaries, of up to four matrices in one launch: 8 values a thread
static __global__ void __launch_bounds__(256) pack_kernel(const __grid_constant__ PackParams p) {
  early_launch_wait();
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < p.units; u += (int64_t)gridDim.x * 256) {
    int z = 0;
    while (z < 3 && u >= p.of[z + 1].first) ++z;
    const Pack& x = p.of[z];
    const int64_t per_row = x.dst_ld / 8, v = u - x.first;
    const int64_t row = (uint64_t)v >> 32 ? v / per_row : (int64_t)((uint32_t)v / (uint32_t)per_row), c = (v - row * per_row) * 8;
    const int count = (int)(x.cols - c < 8 ? x.cols - c : 8);
    if (!MFET_INSIDE(nullptr, row < x.rows && count > 0 && c + 8 <= x.dst_ld)) continue;
    const void* end = x.src + (x.rows - 1) * x.src_ld + x.cols;
    const Raw<MFET_F16, 8> r = load_shifted<MFET_F16, 8>(reinterpret_cast<const __half*>(x.src + row * x.src_ld + c), count, x.src, end);
    *reinterpret_cast<uint4*>(x.dst + (row * x.dst_ld + c) * 2) = r.w[0];
  }
}

inline int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }
inline uint64_t packed_bytes(int64_t rows, int64_t cols) { return ((uint64_t)rows * up8(cols) * 2 + 15) / 16 * 16; }

// Those of `n` (at most four) matrices whose rows do not start on 16-byte boundaries are copied to `to`, and their entries become the copies'.
inline cudaError_t packed(Matrix* x, int n, uint8_t* to, cudaStream_t s) {
  PackParams p{};
  int k = 0;
  for (int i = 0; i < n; ++i) {
    if (on_16(x[i], MFET_F16)) continue;
    p.of[k++] = {(const uint16_t*)x[i].p, to, x[i].outer, x[i].inner, x[i].ld, up8(x[i].inner), p.units};
    p.units += x[i].outer * (up8(x[i].inner) / 8);
    x[i].p = to;
    x[i].ld = up8(x[i].inner);
    to += packed_bytes(x[i].outer, x[i].inner);
  }
  if (k == 0) return cudaSuccess;
  for (; k < 4; ++k) p.of[k].first = p.units;
  const int64_t want = (p.units + 255) / 256, most = (int64_t)sm_count() * 16;
  return launch_early(pack_kernel, (unsigned)(want < most ? want : most), 256, 0, s, p);
}

}  // namespace gemm16
}  // namespace mfet
