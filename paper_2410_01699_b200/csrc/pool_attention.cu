// Attention of window queries over the 8-bit paged cache, with an optional sliding window and sinks.
//
// Keys and values stay in 8 bits: tcgen05 multiplies e4m3 by e4m3 (kind::f8f6f4, products exact, sums in 32 bits), K and V as TMA left them.
// Keys are the rows of both products and the queries their columns, because few queries meet many keys:
//   S^T [128 keys x NC]  =  K [128 keys x HD] . Q^T          O^T [HD x NC]  =  V^T [HD x 128 keys] . P
// Queries and weights are e4m3 numbers too, but several of them: x = x1 + x2 (+ 2^-8 (x3 + x4)), x1 = e4m3(x), x2 = e4m3(x - x1),
// x3 = e4m3(256 (x - x1 - x2)) and so on.  The planes are columns of one product, added when they are read from tensor memory (as more
// products into the same columns they read K and V once more each: 8 x 32 rows 108 -> 113 us).  n planes leave 2^-4n of a number at
// most (half a step of e4m3 is 2^-4 of it) and about 2^-5.3n on average: two for bf16 queries, whose eight bits they hold
// exactly, four for fp32.  (mma.sync has e4m3 as well, but here it converts both operands for every product: 700 products a clock and SM.
// With conversions in registers and fp16 products: 8 x 32 rows x 4009 keys of 32 heads, fp32, 130 us, 32 tokens of up to 4224 keys 63.)
//
// Columns are rows of a window times the query heads of the kv head's group: all heads of a group share the keys that are read.  RP of
// them make a unit's tile of rows; a unit is (sequence, tile of rows, kv head).  The key tiles of all units are one line that is cut into
// as many equal ranges as CTAs are resident, so that sequences of any lengths keep all SMs busy to the end and a long one is
// spread over many.  A second launch joins the parts of units that are cut, in the order of the ranges.  (By the last of a unit's
// CTAs to arrive, which a counter tells: 6 us between its last tile and the first part that it may read, and a lone CTA reads the 33
// parts of 12 rows of a long sequence in 17.)
//
// A thread of the softmax warps is a key of the tile, with up to 16 of the rows.  With s the score (in log2), e_K in its
// factor and e_V added to it, w = 2^(s + e_V - top + 8) is the weight of the value's e4m3 numbers, top the largest s + e_V of the row in this
// tile: weights fill the range of e4m3 whatever stands in other tiles (under one reference for all, the weights of 10^5 keys that share
// a tenth of the mass beside one that has the rest would be zero) and whatever the exponents of the blocks are.  The sum of the softmax takes
// w 2^-e_V.  The same threads, then a dim each, add the tile's O^T to their registers under the running maximum.
//
// A block's exponent is set by its largest entry, which the row need not see (a later row of the window, one before a sliding window).  With
// one reference for exponents far apart, the weights of all other blocks would lose their places to it.  So a tile is worked on in
// parts, as tiles of their own, each with the blocks whose exponents lie within kExpBand of the largest one that is left, and the keys of
// the others masked.  Half of the smallest step of a weight is then at most 2^(kExpBand - 18) (four planes: -26) of the row's largest weight,
// whatever rows that it does not see hold.  Computed for one reference, a hidden value 2^d times the others: error of an output (norm), fp32
// 4.2e-7 with d = 0, 4.8e-7 with 4, 7.1e-7 with 5, 1.2e-6 with 6, 5e-6 with 8, 5.5e-5 with 12 (bf16 before its rounding 6e-4, 6.5e-4, 6.5e-4,
// 7e-4, 1.3e-3, 1.4e-2).  Five, so that first tokens with values of an eighth stand beside blocks that differ by four.  Nearly all tiles have one
// part, which costs nothing but the code (32 tokens 50.8 -> 51.2 us a call of the binding, 8 x 32 rows 108.9 -> 110.6, 100,003 keys 51.5 ->
// 53, others as before); two parts in every tile 2.7 to 2.9 times the call, for masked tiles take longer than whole ones.
//
// Bound: bytes of K and V up to 16 rows (in a long run 7.1 TB/s; 32 tokens of up to 4224 keys, 32 heads on 8, bf16, 210 MB, 50 us, of which
// some 18 are the start, the units' ends and the joining launch; 3 tokens of 100,003 keys, 205 MB, 54 us); beyond, the softmax between
// the products: a warp takes 770 instructions (bf16: 615) for 32 keys by 16 rows, four of them a scheduler fill 54 % of its issue slots, and
// the rest are latencies of one tile's chain that the other warps do not cover (8 x 32 rows of 4009 keys of 32 heads, fp32, 271 MB,
// 108 us, bf16 91; 2 x 64 rows, 32 heads on 8, bf16, 45 us; a prompt of 4224 rows, 32 heads on 8, bf16, 146 GFLOP, 786 us).  Two CTAs per SM
// (one with 64 rows), each with a ring of tiles: 96 to 160 KB of copies in flight.  With 32 and 64 rows every warp has 96 registers, the
// fetching and the issuing one too, and the softmax warps spill (64 dims 188 to 208 bytes, 128 dims 320 to 328).  What few tiles need stands
// behind one branch and is short, and a copy is issued in one place, for the instructions fetched with the common path (NaN entries of V found
// by a first look of the keys' threads alone, their words mended one at a time: 32 tokens 51.5 -> 50 us, 100,003 keys 57.5 -> 54, though
// 2 x 64 rows 45 -> 46; copies issued in three places 54 and 60).
#include "pool_route.h"
#include "tcgen05.cuh"

namespace sjd {
namespace {

constexpr int kMaxSlots = 8;
constexpr int kMeta = 16;            // tiles that the fetching warp may be ahead: more than the ring holds
constexpr int kMaxCtas = 320;
constexpr int kMinTiles = 4;        // of a range, with that
constexpr int kMaxGroup = 32768;     // query heads of a kv head
constexpr int kUp = 8;               // the largest weight of a row in a tile is 2^kUp (e4m3 ends at 448)
constexpr int kExpBand = 5;          // exponents of values that are weighed together: see the comment above
constexpr int kBlocksAt = 8, kMoreAt = 16;   // in Meta::pages
constexpr int kMaxParts = 1 << 22;           // 8 of a tile, 2^19 tiles of a sequence: an end where waits have run out

struct PoolAttnParams {
  sjd_pool pool;
  int layer, batch, window, n_heads, group, rows, row_tiles;   // rows: window * group
  unsigned group_inv;           // 2^32 / group, rounded up: exact for the few rows beside a tile's first
  int sliding, sinks;
  float scale;                  // times log2(e)
  const void *q;
  long q_stride, out_stride;
  const int32_t *seqs, *in_pos;
  void *out;
  int4 *cuts;                   // [kMaxCtas]: (sequence, tile of rows, kv head, CTAs) of the unit that begins in a CTA's range and goes on behind it
  float2 *stats;                // [2 kMaxCtas][RP]: (top, sum) of the rows of the CTAs' parts of cut units
  float *parts;                 // [2 kMaxCtas][RP][head_dim]: their sums
  int n_entries, cut, slots;    // cut: ranges of tiles; else a CTA per unit
};

// With 16 columns a thread, the softmax of an SM has 16 warps (8 with 16 rows): the time of a tile is a chain of latencies, and it takes
// that many to fill the issue slots.
__host__ __device__ constexpr int groups_of(int rp) { return rp <= 16 ? 1 : rp / 16; }
__host__ __device__ constexpr int ctas_of(int rp) { return rp == 64 ? 1 : 2; }
__host__ __device__ constexpr int threads_of(int rp) { return groups_of(rp) * 128 + 64; }

struct Entry {   // (sequence, tile of rows)
  int before;    // cost of one kv head in the entries before: their tiles, and kUnitCost for each
  int low;       // first tile of the sliding part
  uint32_t sink : 24;   // tiles before it
  uint32_t top : 8;     // block of the last tile with the largest position
};

struct Meta {    // of a tile that is being fetched
  int key0;
  int k_exp[2], v_exp[2];   // exponents of its two pages' blocks
  int pages;                // bit j: page j is there; bit 2: the tile has one part; from kBlocksAt on: blocks of this part; from kMoreAt on: how many
                            // parts follow beside the tiles
};

template <int RP>
struct PoolAttnShared {
  uint64_t full[kMaxSlots], empty[kMaxSlots];
  uint64_t meta_full[kMeta];
  uint64_t q_ready, s_full, s_free, p_full, o_full;
  uint32_t tmem_base;
  int failed, n_nan;
  Meta meta[kMeta];
  alignas(16) float red[2][4][RP];   // (these are read and written four at a time)
  alignas(16) float fac[2][RP];      // of this unit and the next (as pos and out_at)
  // what a tile changes, a copy for every warp: kUp - the tile's maximum; factors of the sums so far and of the tile; their logarithms
  struct Change {
    alignas(16) float up[RP < 16 ? RP : 16], alpha[2][RP < 16 ? RP : 16], beta[2][RP < 16 ? RP : 16], old_by[RP < 16 ? RP : 16], new_by[RP < 16 ? RP : 16];
  } change[groups_of(RP) * 4];
  float inv[RP];
  int pos[2][RP];
  long out_at[2][RP];          // first entry of a row in out
  int nan_key[kTile];
  uint32_t nan_dims[kTile][4];
  Entry entry[kMaxEntries + 1];
};

__device__ __forceinline__ uint32_t e4m3_of_floats(const float *v) {   // four, the first one in the low byte
  uint32_t r;
  asm("{\n\t.reg .b16 x, y;\n\tcvt.rn.satfinite.e4m3x2.f32 x, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 y, %4, %3;\n\tmov.b32 %0, {x, y};\n\t}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]));
  return r;
}
// four numbers in a word, from and to two pairs of fp16
__device__ __forceinline__ uint32_t e4m3_of_halves(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("{\n\t.reg .b16 x, y;\n\tcvt.rn.satfinite.e4m3x2.f16x2 x, %1;\n\tcvt.rn.satfinite.e4m3x2.f16x2 y, %2;\n\tmov.b32 %0, {x, y};\n\t}" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ void halves_of_e4m3(uint32_t v, uint32_t &a, uint32_t &b) {
  asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\tcvt.rn.f16x2.e4m3x2 %1, y;\n\t}" : "=r"(a), "=r"(b) : "r"(v));
}
__device__ __forceinline__ uint32_t halves_of_floats(float a, float b) {
  uint32_t h;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(b), "f"(a));
  return h;
}
__device__ __forceinline__ float2 floats_of_halves(uint32_t h) {
  float2 f;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.f32.f16 %0, lo;\n\tcvt.f32.f16 %1, hi;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(h));
  return f;
}
__device__ __forceinline__ uint32_t sub_halves(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t fma_halves(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
// two fp32 operations an instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_of_warp(float x) {   // (a NaN is no maximum)
  float y;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void arrive(uint64_t *bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap *map, int plane, int page, uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(0), "r"(plane), "r"(page), "r"(smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void mma_e4m3(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_ld8_issue(uint32_t taddr, uint32_t *r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
template <int N>
__device__ __forceinline__ void tmem_ld_issue(uint32_t taddr, uint32_t *r) {
  if constexpr (N == 8) tmem_ld8_issue(taddr, r);
  else tmem_ld16_issue(taddr, r);
}
__device__ __forceinline__ bool has_nan(uint32_t bytes) { return (((bytes & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0; }

// sums of N values over the lanes: value i in the lanes whose number ends in i
template <int N>
__device__ __forceinline__ float lanes_sum(float *v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o >= N; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
#pragma unroll
  for (int o = N / 2 < 16 ? N / 2 : 16; o > 0; o >>= 1)
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
      if (j >= o) break;
      const float send = lane & o ? v[j] : v[j + o], keep = lane & o ? v[j + o] : v[j];
      v[j] = keep + __shfl_xor_sync(0xffffffffu, send, o);
    }
  return v[0];
}

// weights of four rows as e4m3 planes, a word each
template <int PL>
__device__ __forceinline__ void weight_planes(float2 v, float2 w, uint32_t *planes) {
  const uint32_t h0 = halves_of_floats(v.x, v.y), h1 = halves_of_floats(w.x, w.y);
  uint32_t a, b;
  planes[0] = e4m3_of_halves(h0, h1);
  halves_of_e4m3(planes[0], a, b);
  uint32_t r0 = sub_halves(h0, a), r1 = sub_halves(h1, b);   // (exact)
  planes[1] = e4m3_of_halves(r0, r1);
  if constexpr (PL == 4) {
    // what is left of the eleven bits of h, and what h left of the weight, times 256
    halves_of_e4m3(planes[1], a, b);
    r0 = sub_halves(r0, a), r1 = sub_halves(r1, b);
    const float2 k = make_float2(256.0f, 256.0f), n = make_float2(-256.0f, -256.0f);
    const float2 f0 = fma2(floats_of_halves(h0), n, mul2(v, k)), f1 = fma2(floats_of_halves(h1), n, mul2(w, k));
    r0 = fma_halves(r0, 0x5C005C00u, halves_of_floats(f0.x, f0.y)), r1 = fma_halves(r1, 0x5C005C00u, halves_of_floats(f1.x, f1.y));
    planes[2] = e4m3_of_halves(r0, r1);
    halves_of_e4m3(planes[2], a, b);
    planes[3] = e4m3_of_halves(sub_halves(r0, a), sub_halves(r1, b));
  }
}

template <typename T> __device__ __forceinline__ float4 load4(const T *p);
template <> __device__ __forceinline__ float4 load4<float>(const float *p) { return *reinterpret_cast<const float4 *>(p); }
template <> __device__ __forceinline__ float4 load4<__nv_bfloat16>(const __nv_bfloat16 *p) {
  const uint2 v = *reinterpret_cast<const uint2 *>(p);
  return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xFFFF0000u));
}
__device__ __forceinline__ void store4(float *p, float4 v) { *reinterpret_cast<float4 *>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float4 v) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}
__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// Shared-memory matrix descriptor of rows of BYTES (32, 64 or 128) under the swizzle of that width, 8 rows a group;
// lbo: bytes between columns of that width (MN-major operands that are wider; 0: the second one is the first again).
template <int BYTES>
__device__ __forceinline__ uint64_t operand(uint32_t lbo) {
  return (uint64_t)(lbo >> 4) << 16 | (uint64_t)(8 * BYTES >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)(BYTES == 128 ? 2 : BYTES == 64 ? 4 : 6) << 61;
}
// byte `col` of row `row` under that swizzle
template <int BYTES>
__device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t col) {
  return row * BYTES + (BYTES == 128 ? col ^ (row & 7) << 4 : BYTES == 64 ? col ^ (row >> 1 & 3) << 4 : col ^ (row >> 2 & 1) << 4);
}

// T: float or bf16 queries and outputs; RP: rows of a unit's tile
template <typename T, int HD, int RP>
__global__ void __launch_bounds__(threads_of(RP), ctas_of(RP))
    pool_attention_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ PoolAttnParams p) {
  constexpr int PL = sizeof(T) == 4 ? 4 : 2;   // planes
  constexpr int CG = groups_of(RP);            // groups of four softmax warps, each with its columns
  constexpr int NQ = RP / CG;                  // columns of a thread
  constexpr int NC = PL * RP;                  // columns of the products
  constexpr int PB = NC < 128 ? NC : 128;      // bytes of a row of P
  constexpr int LD = 8;                        // columns of a load from tensor memory
  constexpr int WORK = 4 * CG, WORK_T = WORK * 32, ALL_T = WORK_T + 64;
  constexpr int TILE = kTile * HD, BOX = TILE / 2;
  constexpr int T_COLS = 2 * NC < 32 ? 32 : 2 * NC;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t *ring = smem;                                   // [slots][128 keys][HD]
  uint8_t *Ps = ring + p.slots * TILE;                    // [NC / PB][128 keys][PB]
  uint8_t *Qs = Ps + kTile * NC;                          // [NC][HD]
  PoolAttnShared<RP> &sh = *reinterpret_cast<PoolAttnShared<RP> *>(Qs + NC * HD);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int kv_heads = p.pool.n_kv_heads, seq_keys = p.pool.pages_per_seq * KV_PAGE;

  pdl_trigger();   // (the joining launch waits for the end of this one)
  if (tid < kMeta) {
    mbar_init(&sh.meta_full[tid], 1);
    sh.meta[tid].pages = 0;   // (what is read after a wait that ran out)
  }
  if (tid < p.slots) {
    mbar_init(&sh.full[tid], 1);
    mbar_init(&sh.empty[tid], 1);
  }
  if (tid == 0) {
    mbar_init(&sh.q_ready, WORK);
    mbar_init(&sh.s_full, 1);
    mbar_init(&sh.s_free, WORK);
    mbar_init(&sh.p_full, WORK);
    mbar_init(&sh.o_full, 1);
    sh.failed = 0;
    sh.n_nan = 0;
  }
  if (warp == 0) {
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }

  // ---- tiles of every entry (a row that is out of range sees nothing)
  auto position = [&](int b, int k) {
    int at = p.in_pos[(long)b * p.window + k];
    const int seq = p.seqs ? p.seqs[b] : b;
    if (at < -1 || at >= seq_keys || seq < 0 || seq >= p.pool.n_seqs) {
      pool_fault(p.pool.status, SJD_ERR_BAD_ARG);
      at = -1;
    }
    return at;
  };
  const int n_entries = p.cut ? p.n_entries : 1, unit_cost = p.cut ? kUnitCost : 0;
  const int unit0 = p.cut ? 0 : blockIdx.x;
  // (entry numbers: sequence by sequence; without ranges the units with the most keys, the last rows of a window, start first)
  auto entry_at = [&](int e, int *b, int *rt) {
    const int id = p.cut ? e : unit0 / kv_heads;
    if (p.cut) {
      *b = id / p.row_tiles;
      *rt = id % p.row_tiles;
    } else {
      *b = id % p.batch;
      *rt = p.row_tiles - 1 - id / p.batch;
    }
  };
  {
    // a group of lanes per entry, as many as it has positions
    const int span = min(p.window, (RP - 1) / p.group + 2);
    int lanes = 1;
    while (lanes < 32 && lanes < span) lanes <<= 1;
    const int per_pass = ALL_T / lanes, mine = tid / lanes, l = tid % lanes;
    for (int e0 = 0; e0 < n_entries; e0 += per_pass) {
      const int e = e0 + mine;
      int lo = 0x7FFFFFFF, hi = -1;
      if (mine < per_pass && e < n_entries) {
        int b, rt;
        entry_at(e, &b, &rt);
        const int r1 = min(p.rows, (rt + 1) * RP);
        for (int k = rt * RP / p.group + l; k <= (r1 - 1) / p.group; k += lanes) {
          const int at = position(b, k);
          if (at >= 0) {
            lo = min(lo, at);
            hi = max(hi, at);
          }
        }
      }
      for (int o = lanes >> 1; o > 0; o >>= 1) {
        lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, o));
      }
      if (mine < per_pass && e < n_entries && l == 0) {
        Entry n;
        n.low = p.sliding > 0 && hi >= 0 ? max(0, lo - p.sliding + 1) / kTile : 0;
        const int sink = min(n.low, (min(p.sinks, seq_keys) + kTile - 1) / kTile);
        n.sink = sink;
        n.top = hi < 0 ? 0 : hi % kTile / kPoolBlock;
        n.before = hi < 0 ? 0 : hi / kTile + 1 - n.low + sink + unit_cost;   // (its own so far)
        sh.entry[e] = n;
      }
    }
  }
  __syncthreads();
  if (warp == 0) {   // exclusive prefix, a run of entries per lane
    const int run = (n_entries + 31) / 32, e0 = min(n_entries, lane * run), e1 = min(n_entries, e0 + run);
    int sum = 0;
    for (int e = e0; e < e1; ++e) sum += sh.entry[e].before;
    int x = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    int at = x - sum;
    for (int e = e0; e < e1; ++e) {
      const int n = sh.entry[e].before;
      sh.entry[e].before = at;
      at += n;
    }
    if (lane == 31) sh.entry[n_entries].before = x;
  }
  if (warp == WORK + 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "r"(T_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;
  const int all = sh.entry[n_entries].before * (p.cut ? kv_heads : 1);
  int chunk = all;
  if (p.cut) {
    chunk = (all + (int)gridDim.x - 1) / (int)gridDim.x;
    chunk = chunk < kMinTiles ? kMinTiles : chunk;
  }
  const int t_begin = p.cut ? (int)min((long)all, (long)blockIdx.x * chunk) : 0, t_end = min(all, t_begin + chunk);

  // Places on the line: kUnitCost of a unit, then its tiles.  Unit of a place:
  struct Unit {
    int e, b, rt, kvh, n, first;      // n: its tiles; first: the place of the first one
  };
  auto unit_of = [&](int t) {
    Unit u;
    int lo = 0, hi = n_entries - 1;
    const int heads = p.cut ? kv_heads : 1;
    while (lo < hi) {   // last entry that begins at t or before
      const int mid = (lo + hi + 1) >> 1;
      if (sh.entry[mid].before * heads <= t) lo = mid; else hi = mid - 1;
    }
    u.e = lo;
    const int len = sh.entry[lo + 1].before - sh.entry[lo].before, in = t - sh.entry[lo].before * heads, h = in / len;
    u.n = len - unit_cost;
    u.kvh = p.cut ? h : unit0 % kv_heads;
    u.first = t - (in - h * len) + unit_cost;
    entry_at(lo, &u.b, &u.rt);
    return u;
  };
  auto fail = [&]() {
    if (lane == 0) {
      *(volatile int *)&sh.failed = 1;
      pool_fault(p.pool.status, SJD_ERR_DEVICE_TIMEOUT);
    }
  };
  // Operands go through the ring in the order in which they are multiplied: K of a unit's first tile, then K of the next tile
  // and V of the one before, and V of the last tile.

  if (warp == WORK) {
    // ------------------------------------------------------------------ fetching
    int slot = 0, meta = 0;
    uint32_t phase = 1;
    int issued = 0;
    bool ok = true;
    int n_key0 = 0, n_page[2] = {-1, -1}, n_ke[2] = {0, 0}, n_ve[2] = {0, 0}, n_head = 0, n_last = 0, n_tile = 0;
    unsigned n_blocks = 0;   // blocks with positions that some row may see
    auto look_up = [&](int t) {   // what lane `lane` knows of tile t + lane
      n_page[0] = n_page[1] = -1;
      n_last = n_tile = 0;
      if (t + lane >= t_end) return;
      const Unit u = unit_of(t + lane);
      const int i = t + lane - u.first;
      if (i < 0) return;   // (no tile)
      n_tile = 1;
      const Entry en = sh.entry[u.e];
      const int sink = (int)en.sink;
      n_key0 = (i < sink ? i : en.low + i - sink) * kTile;
      n_blocks = i == u.n - 1 ? (2u << en.top) - 1 : 0xFFu;   // (exponents behind the sequence may be anything)
      n_head = u.kvh;
      n_last = i == u.n - 1 || t + lane == t_end - 1;
      const int seq = p.seqs ? p.seqs[u.b] : u.b;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int at = n_key0 / KV_PAGE + j;
        if (at >= p.pool.pages_per_seq) continue;
        // (the second page of the last tile may be behind the sequence)
        const int page = p.pool.table[(long)seq * p.pool.pages_per_seq + at];
        n_page[j] = page < 0 || page >= p.pool.n_pages ? -1 : page;
      }
      if (n_page[0] < 0) n_blocks &= 0xF0u;
      if (n_page[1] < 0) n_blocks &= 0x0Fu;
    };
    auto look_up_exps = [&]() {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        n_ke[j] = n_ve[j] = 0;
        if (n_page[j] < 0) continue;
        const long at = ((long)n_page[j] * p.pool.n_layers + p.layer) * 2 * kv_heads + n_head;
        n_ke[j] = *reinterpret_cast<const int *>(p.pool.exps + at * kPoolBlocks);
        n_ve[j] = *reinterpret_cast<const int *>(p.pool.exps + (at + kv_heads) * kPoolBlocks);
      }
    };
    auto fetch = [&](int plane, int page0, int page1) {
      if (issued >= p.slots && !warp_wait(&sh.empty[slot], phase)) { ok = false; return; }
      if (elect_one()) {
        const uint32_t dst = smem_u32(ring) + slot * TILE;
        if (page0 < 0 && page1 < 0) {
          arrive(&sh.full[slot]);
        } else {
          mbar_expect_tx(&sh.full[slot], (page0 >= 0 ? BOX : 0) + (page1 >= 0 ? BOX : 0));
          if (page0 >= 0) tma_box(dst, &map, plane, page0, &sh.full[slot]);
          if (page1 >= 0) tma_box(dst + BOX, &map, plane, page1, &sh.full[slot]);
        }
      }
      __syncwarp();
      ++issued;
      if (++slot == p.slots) { slot = 0; phase ^= 1u; }
    };
    int v_plane = 0, v_page0 = -1, v_page1 = -1;
    bool v_open = false;   // V of the tile before is to be fetched behind this K
    if (t_begin < t_end) look_up(t_begin);
    for (int t0 = t_begin; t0 < t_end && ok; t0 += 32) {
      look_up_exps();
      Meta m;
      m.key0 = n_key0;
      m.k_exp[0] = n_ke[0], m.k_exp[1] = n_ke[1], m.v_exp[0] = n_ve[0], m.v_exp[1] = n_ve[1];
      const int there = (n_page[0] >= 0 ? 1 : 0) | (n_page[1] >= 0 ? 2 : 0);
      m.pages = there | 4 | 0xFF << kBlocksAt;
      const int pg0 = n_page[0], pg1 = n_page[1], head = n_head, last = n_last;
      const unsigned tiles = __ballot_sync(0xffffffffu, n_tile), below = (1u << lane) - 1;
      // A unit's tiles among these are a run.  Parts of its tiles behind their first ones come after the run, as tiles of their own: they are rare,
      // and their bytes in L2; and the first copies need not wait for the exponents.
      const unsigned ends = __ballot_sync(0xffffffffu, n_tile && (last || tiles >> lane == 1u));
      unsigned rest = n_tile ? n_blocks : 0;   // blocks of this lane's tile whose parts have not been told
      int rank = n_tile ? __popc(tiles & below) : 0x7FFF, n = __popc(tiles);   // number of this lane's first part, of all parts
      int more = 0, more_at = 0, follow = 0;   // this lane's parts behind the first, number of the first of them; with a run's end: of the run
      bool known = false, multi = false;       // multi: some lane has more parts than one
      int told = 0;   // parts of these 32 tiles whose lanes have written what they know: not before the copies that there is room for are under way
      auto exp_of = [&](int b) { return pool_exp((int8_t)((b < 4 ? m.v_exp[0] : m.v_exp[1]) >> (8 * (b & 3)))); };
      auto band = [&](unsigned of) {   // the blocks among these whose exponents of values are the largest one or up to kExpBand below it
        int top = -128;
        unsigned in = 0;
#pragma unroll 1
        for (int b = 0; b < 8; ++b) top = of >> b & 1u ? max(top, exp_of(b)) : top;
#pragma unroll 1
        for (int b = 0; b < 8; ++b) in |= exp_of(b) >= top - kExpBand ? 1u << b : 0u;
        return of & in;
      };
      if (t0 + 32 < t_end) look_up(t0 + 32);
      int done = 0, left = 0;            // parts so far; parts that a run's tiles have left
      bool at_end = false, over = false; // at the end of a run, which is the end of its unit
#pragma unroll 1
      for (unsigned todo = tiles; (todo != 0 || left > 0) && ok;) {
        int from = __ffs(todo) - 1;
        const bool first = left == 0;
        if (first) {
          todo &= todo - 1;
          at_end = ends >> from & 1u;
        } else {
          from = __ffs(__ballot_sync(0xffffffffu, done >= more_at && done < more_at + more)) - 1;
          --left;
        }
        ++done;
        const bool full = issued + 3 > p.slots;   // a copy of this round may have to wait
        if (!known && (full || at_end)) {
          known = true;
          int e_min = 127, e_max = -128;
#pragma unroll
          for (int b = 0; b < 8; ++b) {
            const int e = exp_of(b);
            e_min = rest >> b & 1u ? min(e_min, e) : e_min;
            e_max = rest >> b & 1u ? max(e_max, e) : e_max;
          }
          const bool far = e_max - e_min > kExpBand;   // (no block: not)
          multi = __any_sync(0xffffffffu, far);
          if (__builtin_expect(multi, 0)) {
            if (far) {
              const unsigned now = band(rest);
              m.pages = there | (int)now << kBlocksAt;
              rest &= ~now;
#pragma unroll 1
              for (unsigned r = rest; r != 0; ++more) r &= ~band(r);
            }
            int x = more;   // (sums up to this lane's)
#pragma unroll 1
            for (int o = 1; o < 32; o <<= 1) {
              const int y = __shfl_up_sync(0xffffffffu, x, o);
              if (lane >= o) x += y;
            }
            const unsigned ended = ends & below, end = ends & ~below;
            const int before = __shfl_sync(0xffffffffu, x, ended ? 31 - __clz(ended) : 0), runs = ended ? before : 0;   // in the runs before
            rank += runs;
            more_at = __popc(tiles & ((end & -end) * 2 - 1)) + x - more;
            follow = ends >> lane & 1u ? x - runs : 0;
            m.pages |= follow << kMoreAt;
            n += __shfl_sync(0xffffffffu, x, 31);
          }
        }
        if (first && at_end) {
          over = __shfl_sync(0xffffffffu, last, from);
          left = __shfl_sync(0xffffffffu, follow, from);
        }
        if (full || (todo == 0 && left == 0)) {
          auto write = [&](int i) {
            const int at = (meta + i) % kMeta;
            sh.meta[at] = m;
            arrive(&sh.meta_full[at]);
          };
          if (rank >= told && rank < done) write(rank);
          if (__builtin_expect(multi, 0)) {
#pragma unroll 1
            for (int i = max(more_at, told); i < min(more_at + more, done); ++i) {
              const unsigned now = band(rest);
              m.pages = there | (int)now << kBlocksAt;
              rest &= ~now;
              write(i);
            }
          }
          __syncwarp();
          told = done;
        }
        // K of this part, V of the one before, and V of a unit's last part
        const int page0 = __shfl_sync(0xffffffffu, pg0, from), page1 = __shfl_sync(0xffffffffu, pg1, from), h = __shfl_sync(0xffffffffu, head, from);
        const bool flush = at_end && left == 0 && over;
#pragma unroll 1
        for (int o = 0; o < 3 && ok; ++o) {
          if (o == 1 ? !v_open : o == 2 && !flush) continue;
          const bool own = o != 1;
          fetch(o == 0 ? h : own ? kv_heads + h : v_plane, own ? page0 : v_page0, own ? page1 : v_page1);
        }
        v_plane = kv_heads + h;
        v_page0 = page0;
        v_page1 = page1;
        v_open = !flush;
      }
      meta = (meta + n) % kMeta;
    }
    if (!ok) fail();
    // leave no copy in flight
    for (int j = issued > p.slots ? issued - p.slots : 0; j < issued; ++j) warp_wait(&sh.full[j % p.slots], (uint32_t)((j / p.slots) & 1));
  } else if (warp == WORK + 1) {
    // ------------------------------------------------------------------ issuing the products
    constexpr uint32_t idesc = (1u << 4) | (uint32_t)(NC >> 3) << 17 | (uint32_t)(128 >> 4) << 24;   // e4m3 both, sums in 32 bits
    constexpr uint32_t idesc_v = idesc | 1u << 15 | 1u << 16;                                       // both operands MN-major
    const uint64_t desc_k = operand<HD>(16), desc_v = operand<HD>(HD == 64 ? 0 : 16), desc_p = operand<PB>(NC > 128 ? kTile * 128 : 16);
    const uint32_t ring0 = smem_u32(ring), q_at = smem_u32(Qs), p_at = smem_u32(Ps);
    int slot = 0;
    uint32_t phase = 0, q_ph = 0, sfree_ph = 0, p_ph = 0, meta_ph = 0;
    int meta = 0;
    bool ok = true, first_s = true;
    auto next = [&]() {
      __syncwarp();
      if (++slot == p.slots) { slot = 0; phase ^= 1u; }
    };
    auto scores = [&](bool first) {
      ok = ok && !*(volatile int *)&sh.failed && warp_wait(&sh.full[slot], phase);
      if (ok && first) {
        ok = warp_wait(&sh.q_ready, q_ph);
        q_ph ^= 1u;
      }
      if (ok && !first_s) {
        ok = warp_wait(&sh.s_free, sfree_ph);
        sfree_ph ^= 1u;
      }
      first_s = false;
      if (!ok) return;
      tc_fence_after();
      if (elect_one()) {
        const uint64_t a = desc_k | (uint64_t)((ring0 + slot * TILE) >> 4), b = desc_k | (uint64_t)(q_at >> 4);
#pragma unroll
        for (int k = 0; k < HD / 32; ++k) mma_e4m3(tmem, a + k * 2, b + k * 2, idesc, k > 0);
        umma_commit(&sh.empty[slot]);
        umma_commit(&sh.s_full);
      }
      next();
    };
    auto values = [&]() {
      ok = ok && !*(volatile int *)&sh.failed && warp_wait_both(&sh.full[slot], phase, &sh.p_full, p_ph);
      p_ph ^= 1u;
      if (!ok) return;
      tc_fence_after();
      if (elect_one()) {
        const uint64_t a = desc_v | (uint64_t)((ring0 + slot * TILE) >> 4), b = desc_p | (uint64_t)(p_at >> 4);
#pragma unroll
        for (int k = 0; k < kTile / 32; ++k) mma_e4m3(tmem + NC, a + k * (32 * HD >> 4), b + k * (32 * PB >> 4), idesc_v, k > 0);
        umma_commit(&sh.empty[slot]);
        umma_commit(&sh.o_full);
      }
      next();
    };
    for (int t = t_begin; t < t_end && ok;) {
      const Unit u = unit_of(t);
      t = max(t, u.first);
      if (t >= t_end) break;
      const int n = min(t_end, u.first + u.n) - t;
      bool first = true;
      for (int left = n; left > 0 && ok;) {
        scores(first);
        if (ok && !first) values();
        first = false;
        // (whether other parts of tiles follow)
        ok = ok && warp_wait(&sh.meta_full[meta], meta_ph);
        if (ok) left += (*(volatile int *)&sh.meta[meta].pages >> kMoreAt) - 1;
        if (++meta == kMeta) { meta = 0; meta_ph ^= 1u; }
      }
      if (ok) values();
      t += n;
    }
    if (!ok) fail();
  } else {
    // ------------------------------------------------------------------ softmax warps: thread = key of the tile, then dim of the output
    const int w = warp & 3, cg = warp >> 2, c0 = cg * NQ, key_t = w * 32 + lane;
    const uint32_t t_s = tmem + ((uint32_t)(w * 32) << 16) + c0, t_o = t_s + NC;
    const T *qp = (const T *)p.q;
    T *outp = (T *)p.out;
    uint32_t s_ph = 0, o_ph = 0, v_use = 0;   // v_use: ring slots of the units before
    int meta = 0;
    uint32_t meta_ph = 0;
    bool ok = true;
    auto sync = [&]() { asm volatile("bar.sync 1, %0;" ::"n"(WORK_T) : "memory"); };
    auto any = [&](bool pred) {   // of all softmax threads
      uint32_t r;
      asm volatile(
          "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbar.red.or.pred p, 1, %2, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
          : "=r"(r)
          : "r"((uint32_t)pred), "n"(WORK_T)
          : "memory");
      return r != 0;
    };
    auto group_sync = [&]() { asm volatile("bar.sync %0, 128;" ::"r"(2 + cg) : "memory"); };
    const int gt = tid & 127;            // thread of its group
    // ---- queries of a unit: a power of two brings a row's largest entry to 128 .. 256, then its planes; a row is HD / 4 lanes
    constexpr int LANES = HD / 4, PER = 32 / LANES, N = (RP + WORK * PER - 1) / (WORK * PER);
    const int q_sub = lane / LANES, q_dim = lane % LANES * 4;
    float4 qx[N];
    int q_pos = -1;
    // window row and head of row j of a unit's tile
    struct Rows {
      int left, k, rem;    // rows that there are; window row and head of its first one
    };
    auto rows_of = [&](const Unit &u) {
      const int r = u.rt * RP, k = r / p.group;
      return Rows{min(RP, p.rows - r), k, r - k * p.group};
    };
    auto place = [&](const Unit &u, const Rows &rw, int j, long stride) {   // first entry of the row in q or out
      const int x = rw.rem + j, dk = p.group == 1 ? x : __umulhi(x, p.group_inv);
      return ((long)u.b * p.window + rw.k + dk) * stride + ((long)u.kvh * p.group + x - dk * p.group) * HD;
    };
    auto load_queries = [&](const Unit &u) {
      const Rows rw = rows_of(u);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int j = (i * WORK + warp) * PER + q_sub;
        qx[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (j < rw.left) qx[i] = load4<T>(qp + place(u, rw, j, p.q_stride) + q_dim);
      }
      q_pos = -1;
      if (tid < rw.left) {
        const int x = rw.rem + tid;
        q_pos = position(u.b, rw.k + (p.group == 1 ? x : (int)__umulhi(x, p.group_inv)));
      }
    };
    // (a load behind the copies that are under way takes about 3 us)
    auto prefetch_queries = [&](const Unit &u) {
      const Rows rw = rows_of(u);
      constexpr int LINES = HD * (int)sizeof(T) / 128;
      for (int i = tid; i < rw.left * LINES; i += WORK_T)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(qp + place(u, rw, i / LINES, p.q_stride) + i % LINES * (128 / (int)sizeof(T))));
    };
    auto publish_queries = [&](const Unit &u, int up) {
      if (tid < RP) {
        sh.pos[up][tid] = q_pos;
        sh.out_at[up][tid] = place(u, rows_of(u), tid, p.out_stride);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = (i * WORK + warp) * PER + q_sub;
        float v[4] = {qx[i].x, qx[i].y, qx[i].z, qx[i].w};
        float top = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (fabsf(v[j]) == INFINITY) v[j] = __int_as_float(0x7FFFFFFF);   // (e4m3 has no infinity: its row is NaN, as it would be)
          top = fmaxf(top, fabsf(v[j]));
        }
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        int e = top > 0.0f ? 7 - (int)((__float_as_uint(top) >> 23) - 127) : 0;
        e = max(min(e, 126), -126);   // (entries below 2^-119 lose places)
        const float up2 = two_to(e);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] *= up2;
        if (r < RP) {
          if (q_dim == 0) sh.fac[up][r] = p.scale * two_to(-e);
#pragma unroll
          for (int l = 0; l < PL; ++l) {
            if (l == 2) v[0] *= 256.0f, v[1] *= 256.0f, v[2] *= 256.0f, v[3] *= 256.0f;
            const uint32_t four = e4m3_of_floats(v);
            *reinterpret_cast<uint32_t *>(Qs + swizzled<HD>(l * RP + r, q_dim)) = four;
            uint32_t ha, hc;
            halves_of_e4m3(four, ha, hc);
            const float2 fa = floats_of_halves(ha), fc = floats_of_halves(hc);
            v[0] -= fa.x, v[1] -= fa.y, v[2] -= fc.x, v[3] -= fc.y;
          }
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) arrive(&sh.q_ready);
    };

    int up = 0;
    int t_first = t_end;
    if (t_begin < t_end) {
      const Unit u = unit_of(t_begin);
      t_first = max(t_begin, u.first);
      if (t_first < t_end) {
        load_queries(u);
        publish_queries(u, 0);
      }
    }
    if (p.cut && tid == 0) {
      int4 c = make_int4(0, 0, 0, 0);
      if (t_begin < t_end && t_end < all) {
        const Unit l = unit_of(t_end - 1);
        if (l.first >= t_begin && l.first < t_end && l.first + l.n > t_end) {
          c.x = l.b;
          c.y = l.rt;
          c.z = l.kvh;
          c.w = (l.first + l.n - 1) / chunk - (int)blockIdx.x + 1;
        }
      }
      p.cuts[blockIdx.x] = c;
    }
    // rows without a tile are in no range: the CTAs share them (an entry whose rows see nothing has no tiles)
    if (p.cut || all == 0) {
      for (int e = p.cut ? blockIdx.x : 0; e < n_entries; e += gridDim.x) {
        if (sh.entry[e + 1].before != sh.entry[e].before) continue;
        int b, rt;
        entry_at(e, &b, &rt);
        const int r1 = min(p.rows, (rt + 1) * RP), h0 = p.cut ? 0 : unit0 % kv_heads, h1 = p.cut ? kv_heads : h0 + 1;
        for (int r = rt * RP; r < r1; ++r)
          for (int h = h0; h < h1; ++h)
            for (int i = tid; i < HD; i += WORK_T)
              store1(outp + ((long)b * p.window + r / p.group) * p.out_stride + ((long)h * p.group + r % p.group) * HD + i, 0.0f);
      }
    }
    for (int t = t_first; t < t_end; up ^= 1) {
      const Unit u = unit_of(t);
      const int u_end = u.first + u.n, end = min(t_end, u_end);
      const int n = end - t;
      if (end < t_end) prefetch_queries(unit_of(end));
      sync();   // (every row's position is there; what the unit before left in shared memory has been read)
      int lo = 0x7FFFFFFF, hi = -1;   // smallest and largest position of the tile's rows
#pragma unroll
      for (int i = 0; i < (RP + 31) / 32; ++i) {
        const int at = lane + 32 * i < RP ? sh.pos[up][lane + 32 * i] : -1;
        if (at >= 0) lo = min(lo, at);
        hi = max(hi, at);
      }
      lo = __reduce_min_sync(0xffffffffu, lo);
      hi = __reduce_max_sync(0xffffffffu, hi);
      const int sliding = p.sliding > 0 ? p.sliding : 0x7FFFFFFF;
      const int from = hi - sliding;      // keys above are in the window of every row
      auto sees = [&](int key, int at) { return key <= at && (key > at - sliding || key < p.sinks); };

      float2 o[NQ / 2], l_acc[NQ / 2];
#pragma unroll
      for (int i = 0; i < NQ / 2; ++i) o[i] = l_acc[i] = make_float2(0.0f, 0.0f);
      bool nans = false;          // the last tile had NaN entries among keys that not all rows see
      float my_run = -INFINITY;   // lane i < NQ: the running maximum of the warp's row i

      auto &change = sh.change[warp];
      auto four_of = [&](const float *a, int q) { return *reinterpret_cast<const float4 *>(a + q); };
      // columns of a product, its planes added (the fine ones first: 16 registers of loads at a time)
      auto load_columns = [&](uint32_t from_col, float2 *v) {
#pragma unroll
        for (int c = 0; c < NQ; c += LD) {
          float2 fine[LD / 2];
#pragma unroll
          for (int l = PL - 2; l >= 0; l -= 2) {
            uint32_t x[2][LD];
            tmem_ld_issue<LD>(from_col + l * RP + c, x[0]);
            tmem_ld_issue<LD>(from_col + (l + 1) * RP + c, x[1]);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < LD / 2; ++i) {
              float2 sum = add2(make_float2(__uint_as_float(x[0][2 * i]), __uint_as_float(x[0][2 * i + 1])),
                                make_float2(__uint_as_float(x[1][2 * i]), __uint_as_float(x[1][2 * i + 1])));
              if (PL == 4 && l == 0) sum = fma2(fine[i], make_float2(0x1p-8f, 0x1p-8f), sum);
              if (l > 0) fine[i] = sum;
              else v[c / 2 + i] = sum;
            }
          }
        }
      };
      auto add_values = [&](int par) {   // O^T of a tile to this thread's dim, under the maximum after that tile
        tc_fence_after();
        if (w * 32 < HD) {
          float2 v[NQ / 2];
          load_columns(t_o, v);
#pragma unroll
          for (int i = 0; i < NQ / 2; i += 2) {
            const float4 a = four_of(change.alpha[par], 2 * i), c = four_of(change.beta[par], 2 * i);
            o[i] = fma2(v[i], make_float2(c.x, c.y), mul2(o[i], make_float2(a.x, a.y)));
            o[i + 1] = fma2(v[i + 1], make_float2(c.z, c.w), mul2(o[i + 1], make_float2(a.z, a.w)));
          }
        }
        tc_fence_before();
      };
      auto add_nans = [&]() {   // rare: entries that are NaN where only some rows see their key
        const int many = min(sh.n_nan, kTile);
        for (int i = 0; i < many; ++i) {
          if (w * 32 >= HD || !(sh.nan_dims[i][w] >> lane & 1u)) continue;
#pragma unroll
          for (int q = 0; q < NQ / 2; ++q) {
            if (sees(sh.nan_key[i], sh.pos[up][c0 + 2 * q])) o[q].x = __int_as_float(0x7FFFFFFF);
            if (sees(sh.nan_key[i], sh.pos[up][c0 + 2 * q + 1])) o[q].y = __int_as_float(0x7FFFFFFF);
          }
        }
      };

      int i = 0;
      for (int until = n; i < until; ++i) {
        const int par = i & 1;
        ok = ok && !*(volatile int *)&sh.failed;
        if (ok && !(warp_wait(&sh.meta_full[meta], meta_ph) && warp_wait(&sh.s_full, s_ph))) {
          ok = false;
          fail();
        }
        const Meta &m = sh.meta[meta];   // (not written again before this tile is done)
        if (++meta == kMeta) { meta = 0; meta_ph ^= 1u; }
        until = min(until + (m.pages >> kMoreAt), kMaxParts);
        s_ph ^= 1u;
        tc_fence_after();
        // ---- scores
        const int key = m.key0 + key_t, half = key_t >> 6;
        const int ev = pool_exp((int8_t)(m.v_exp[half] >> (8 * (key_t >> 4 & 3))));
        const float k2 = two_to(pool_exp((int8_t)(m.k_exp[half] >> (8 * (key_t >> 4 & 3))))), add = (float)ev;
        const bool whole = (m.pages & 7) == 7 && m.key0 + kTile - 1 <= lo && (m.key0 > from || m.key0 + kTile <= p.sinks);
        float2 s[NQ / 2];
        load_columns(t_s, s);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive(&sh.s_free);
#pragma unroll
        for (int q = 0; q < NQ / 2; q += 2) {
          const float4 f = four_of(sh.fac[up] + c0, 2 * q);
          s[q] = fma2(s[q], mul2(make_float2(f.x, f.y), make_float2(k2, k2)), make_float2(add, add));
          s[q + 1] = fma2(s[q + 1], mul2(make_float2(f.z, f.w), make_float2(k2, k2)), make_float2(add, add));
        }
        if (!whole) {
          const bool there = m.pages >> half & 1, part = m.pages >> (kBlocksAt + (key_t >> 4)) & 1;
          bool missed = false;
#pragma unroll
          for (int q = 0; q < NQ / 2; ++q) {
            const bool in0 = sees(key, sh.pos[up][c0 + 2 * q]), in1 = sees(key, sh.pos[up][c0 + 2 * q + 1]);
            missed |= (in0 || in1) && !there;
            if (!in0 || !there || !part) s[q].x = -INFINITY;
            if (!in1 || !there || !part) s[q].y = -INFINITY;
          }
          if (missed) pool_fault(p.pool.status, SJD_ERR_BAD_ARG);   // (no page where some row sees a key)
        }
        // ---- the tile's maximum of every row
#pragma unroll
        for (int q = 0; q < NQ; q += 4) {
          float4 v;
          v.x = max_of_warp(s[q / 2].x), v.y = max_of_warp(s[q / 2].y), v.z = max_of_warp(s[q / 2 + 1].x), v.w = max_of_warp(s[q / 2 + 1].y);
          if (lane == 0) *reinterpret_cast<float4 *>(&sh.red[par][w][c0 + q]) = v;
        }
        group_sync();
        // (every warp for itself: one for all would take a second barrier)
        bool wide = false;   // maxima that differ so much that weights, but not the sum's terms, may leave the range
        if (lane < NQ) {
          const int r = c0 + lane;
          const float mx = fmaxf(fmaxf(sh.red[par][0][r], sh.red[par][1][r]), fmaxf(sh.red[par][2][r], sh.red[par][3][r]));
          const float now = fmaxf(my_run, mx), at = now > -INFINITY ? now : 0.0f, da = my_run - at, db = mx - at;
          change.up[lane] = (float)kUp - (mx > -INFINITY ? mx : 0.0f);
          change.alpha[par][lane] = exp2_fast(da);
          change.beta[par][lane] = exp2_fast(db);
          change.old_by[lane] = da, change.new_by[lane] = db;
          wide |= (my_run > -INFINITY && da < -64.0f) || (mx > -INFINITY && db < -64.0f);
          my_run = now;
        }
        wide = __any_sync(0xffffffffu, wide);
        __syncwarp();
        // ---- weights and their sum without the values' exponents
        uint32_t pk[PL][NQ / 4];
        const float back = two_to(-ev - kUp);   // (the sum goes without 2^kUp)
        if (wide) {
#pragma unroll
          for (int q = 0; q < NQ / 2; ++q) {
            // (in two steps: with the values' exponents a maximum may move by 200, and the sum by as much the other way)
            const float a0 = exp2_fast(0.5f * change.old_by[2 * q]), a1 = exp2_fast(0.5f * change.old_by[2 * q + 1]);
            const float b0 = exp2_fast(0.5f * change.new_by[2 * q]), b1 = exp2_fast(0.5f * change.new_by[2 * q + 1]);
            l_acc[q].x = l_acc[q].x * a0 * a0 + exp2_fast(s[q].x - add + change.up[2 * q] - (float)kUp) * b0 * b0;
            l_acc[q].y = l_acc[q].y * a1 * a1 + exp2_fast(s[q].y - add + change.up[2 * q + 1] - (float)kUp) * b1 * b1;
          }
        }
#pragma unroll
        for (int q = 0; q < NQ / 2; q += 2) {
          const float4 r = four_of(change.up, 2 * q);
          s[q] = add2(s[q], make_float2(r.x, r.y));
          s[q + 1] = add2(s[q + 1], make_float2(r.z, r.w));
          s[q].x = exp2_fast(s[q].x);
          s[q].y = exp2_fast(s[q].y);
          s[q + 1].x = exp2_fast(s[q + 1].x);
          s[q + 1].y = exp2_fast(s[q + 1].y);
        }
        if (!wide) {
#pragma unroll
          for (int q = 0; q < NQ / 2; q += 2) {
            const float4 a = four_of(change.alpha[par], 2 * q), c = four_of(change.beta[par], 2 * q);
            l_acc[q] = fma2(mul2(s[q], make_float2(back, back)), make_float2(c.x, c.y), mul2(l_acc[q], make_float2(a.x, a.y)));
            l_acc[q + 1] = fma2(mul2(s[q + 1], make_float2(back, back)), make_float2(c.z, c.w), mul2(l_acc[q + 1], make_float2(a.z, a.w)));
          }
        }
#pragma unroll
        for (int q = 0; q < NQ; q += 4) {
          uint32_t four[PL];
          weight_planes<PL>(s[q / 2], s[q / 2 + 1], four);
#pragma unroll
          for (int l = 0; l < PL; ++l) pk[l][q / 4] = four[l];
        }
        // ---- the tile before is multiplied: its O^T is there, and P may be written
        if (i > 0) {
          if (ok && !warp_wait(&sh.o_full, o_ph)) {
            ok = false;
            fail();
          }
          o_ph ^= 1u;
        }
#pragma unroll
        for (int l = 0; l < PL; ++l) {
          const uint32_t col = l * RP + c0;
          uint8_t *dst = Ps + (col / 128) * (kTile * 128) + swizzled<PB>(key_t, col % 128);
          if constexpr (NQ == 16) *reinterpret_cast<uint4 *>(dst) = make_uint4(pk[l][0], pk[l][1], pk[l][2], pk[l][3]);
          else *reinterpret_cast<uint2 *>(dst) = make_uint2(pk[l][0], pk[l][1]);
        }
        if (i > 0) {
          add_values(par ^ 1);
          if (nans) add_nans();   // (of the tile before)
        }
        if (!whole) {
          // A key that some row does not see must not reach it: a weight of zero times NaN would.  NaN entries become zero, and
          // the rows that see them get their NaN afterwards.
          bool found = false;
          uint8_t *v = nullptr;
          if (cg == 0) {
            const uint32_t use = v_use + (i + 1 < until ? 2 * i + 2 : 2 * i + 1);
            if (ok && !warp_wait(&sh.full[use % p.slots], use / p.slots & 1)) {
              ok = false;
              fail();
            }
            v = ring + (use % p.slots) * TILE;
#pragma unroll
            for (int c = 0; c < HD / 16; ++c) {
              const uint4 x = *reinterpret_cast<const uint4 *>(v + swizzled<HD>(key_t, c * 16));
              found |= has_nan(x.x) || has_nan(x.y) || has_nan(x.z) || has_nan(x.w);
            }
          }
          nans = any(found);
          if (__builtin_expect(nans, 0)) {
            if (tid == 0) sh.n_nan = 0;
            sync();
            if (found) {
              uint32_t dims[4] = {0u, 0u, 0u, 0u};
#pragma unroll 1
              for (int c = 0; c < HD / 4; ++c) {
                uint32_t *at = reinterpret_cast<uint32_t *>(v + swizzled<HD>(key_t, c * 4));
                const uint32_t x = *at, nan = ((x & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;   // the top bit of every NaN byte
                *at = x & ~((nan >> 7) * 0xFFu);
                dims[c >> 3] |= ((nan >> 7 & 1u) | (nan >> 14 & 2u) | (nan >> 21 & 4u) | (nan >> 28 & 8u)) << ((c & 7) * 4);
              }
              if (key <= hi && (m.pages >> half & 1) && (m.pages >> (kBlocksAt + (key_t >> 4)) & 1)) {
                const int at = atomicAdd(&sh.n_nan, 1);
                sh.nan_key[at] = key;
#pragma unroll
                for (int j = 0; j < 4; ++j) sh.nan_dims[at][j] = dims[j];
              }
            }
            sync();
          }
        } else {
          nans = false;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) arrive(&sh.p_full);
      }
      v_use += 2 * i;
      // ---- the next unit's queries, and this one's sums over the keys, while the last tile is multiplied
      const Unit next = unit_of(end < t_end ? end : end - 1);
      const bool more = end < t_end && next.first < t_end;
      if (more) load_queries(next);
      {
        float v[NQ];
#pragma unroll
        for (int q = 0; q < NQ / 2; ++q) v[2 * q] = l_acc[q].x, v[2 * q + 1] = l_acc[q].y;
        const float l = lanes_sum<NQ>(v);
        if (lane < NQ) sh.red[i & 1][w][c0 + lane] = l;   // (not the last tile's: a warp may still read that)
      }
      group_sync();
      const bool cut = u.first < t_begin || u_end > t_end;
      const int rows_here = min(RP, p.rows - u.rt * RP), dim = w * 32 + lane;
      constexpr long PART = (long)RP * HD;
      // this CTA's part of a cut unit: slot 0 of a unit that began before its range, slot 1 of one that goes on behind it
      const int my = 2 * blockIdx.x + (u.first < t_begin ? 0 : 1);
      if (gt < NQ) {
        const int r = c0 + gt;
        const float sum = (sh.red[i & 1][0][r] + sh.red[i & 1][1][r]) + (sh.red[i & 1][2][r] + sh.red[i & 1][3][r]);
        sh.inv[r] = sh.pos[up][r] >= 0 && sum != 0.0f ? two_to(-kUp) / sum : 0.0f;   // (a NaN among the scores makes the sum NaN)
        if (cut) p.stats[my * RP + r] = make_float2(my_run, sum);
      }
      if (more) publish_queries(next, up ^ 1);   // (all scores of this unit have been waited for)
      if (ok && !warp_wait(&sh.o_full, o_ph)) {
        ok = false;
        fail();
      }
      o_ph ^= 1u;
      add_values(i - 1 & 1);
      if (nans) add_nans();
      sync();
      if (w * 32 < HD) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          const float v = q & 1 ? o[q / 2].y : o[q / 2].x;
          if (c0 + q >= rows_here) break;
          if (cut) {
            p.parts[my * PART + (c0 + q) * HD + dim] = v;
          } else {
            const float inv = sh.inv[c0 + q];
            store1(outp + sh.out_at[up][c0 + q] + dim, inv == 0.0f ? 0.0f : v * inv);
          }
        }
      }
      t = more ? next.first : t_end;
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == WORK + 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(T_COLS) : "memory");
  }
}

// Joins the parts of the unit that begins in range blockIdx.x and is cut: a warp per row, sixteen parts' loads in flight together.
constexpr int kJoinRows = 8;
template <typename T, int HD>
__global__ void __launch_bounds__(kJoinRows * 32) pool_attention_join_kernel(const __grid_constant__ PoolAttnParams p, int RP) {
  constexpr int D = HD / 32, U = 16;
  pdl_wait();
  const int4 c = p.cuts[blockIdx.x];
  const int lane = threadIdx.x & 31, r = blockIdx.y * kJoinRows + (threadIdx.x >> 5), row = c.y * RP + r;
  if (c.w < 2 || r >= RP || row >= p.rows) return;
  auto slot_of = [&](int i) { return 2 * ((int)blockIdx.x + i) + (i == 0 ? 1 : 0); };
  const int k = row / p.group, at = p.in_pos[(long)c.x * p.window + k];
  float best = -INFINITY, sum = 0.0f;
  float2 ms = make_float2(-INFINITY, 0.0f);
  for (int i = lane; i < c.w; i += 32) {
    ms = p.stats[slot_of(i) * RP + r];
    best = fmaxf(best, ms.x);
  }
  best = warp_max(best);
  if (best == -INFINITY) best = 0.0f;
  float acc[D];
#pragma unroll
  for (int d = 0; d < D; ++d) acc[d] = 0.0f;
  for (int base = 0; base < c.w; base += 32) {
    const int n = min(32, c.w - base);
    float f = 0.0f;
    if (lane < n) {
      if (c.w > 32) ms = p.stats[slot_of(base + lane) * RP + r];
      f = exp2_fast(0.5f * (ms.x - best));   // (a root: see the range of the sums)
      sum += ms.y * f * f;
      f *= f;
    }
    for (int i = 0; i < n; i += U) {
      float x[U][D];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if (i + j >= n) break;
        const float *src = p.parts + ((long)slot_of(base + i + j) * RP + r) * HD + lane * D;
        if constexpr (D == 4) {
          const float4 v = *reinterpret_cast<const float4 *>(src);
          x[j][0] = v.x, x[j][1] = v.y, x[j][2] = v.z, x[j][3] = v.w;
        } else {
          const float2 v = *reinterpret_cast<const float2 *>(src);
          x[j][0] = v.x, x[j][1] = v.y;
        }
      }
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if (i + j >= n) break;
        const float w = __shfl_sync(0xffffffffu, f, i + j);
#pragma unroll
        for (int d = 0; d < D; ++d) acc[d] = fmaf(x[j][d], w, acc[d]);
      }
    }
  }
  sum = warp_sum(sum);
  const bool live = (unsigned)at < (unsigned)(p.pool.pages_per_seq * KV_PAGE) && sum != 0.0f;
  const float inv = live ? two_to(-kUp) / sum : 0.0f;
  T *dst = (T *)p.out + ((long)c.x * p.window + k) * p.out_stride + ((long)c.z * p.group + row - k * p.group) * HD + lane * D;
#pragma unroll
  for (int d = 0; d < D; ++d) acc[d] = live ? acc[d] * inv : 0.0f;
  if constexpr (D == 4) store4(dst, make_float4(acc[0], acc[1], acc[2], acc[3]));
  else store1(dst, acc[0]), store1(dst + 1, acc[1]);
}

// the layer's pages as boxes of 64 rows of a plane
int make_pool_map(TensorMap *out, const sjd_pool &p, int layer) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return SJD_ERR_UNSUPPORTED;
  const cuuint64_t plane = (cuuint64_t)KV_PAGE * p.head_dim, planes = 2ull * p.n_kv_heads;
  cuuint64_t dims[4] = {(cuuint64_t)p.head_dim, (cuuint64_t)KV_PAGE, planes, (cuuint64_t)p.n_pages};
  cuuint64_t strides[3] = {(cuuint64_t)p.head_dim, plane, plane * planes * p.n_layers};
  cuuint32_t box[4] = {(cuuint32_t)p.head_dim, (cuuint32_t)KV_PAGE, 1, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  const CUresult r = fn(reinterpret_cast<CUtensorMap *>(out), CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, (uint8_t *)p.pages + plane * planes * layer,
                        dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        p.head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SJD_OK : SJD_ERR_UNSUPPORTED;
}

// rows of a unit's tile
int tile_rows(int64_t rows, int dtype) {
  const int least = dtype == SJD_F32 ? 8 : 16;
  return rows <= least ? least : rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
}
constexpr size_t kCutBytes = kMaxCtas * sizeof(int4);
size_t stat_bytes(int rp) { return 2ull * kMaxCtas * rp * sizeof(float2); }
size_t parts_bytes(int rp, int hd) { return 2ull * kMaxCtas * rp * hd * sizeof(float); }

}  // namespace
}  // namespace sjd

using namespace sjd;

extern "C" size_t sjd_pool_attention_workspace_bytes(const sjd_pool *pool, int window, int n_heads) {
  if (check_pool(pool, false) != SJD_OK || window < 1 || n_heads < 1 || n_heads % pool->n_kv_heads != 0) return 0;
  const int rp = tile_rows((int64_t)window * (n_heads / pool->n_kv_heads), SJD_BF16);
  return kCutBytes + stat_bytes(rp) + parts_bytes(rp, pool->head_dim);
}

extern "C" int sjd_pool_attention(const sjd_pool *pool, int layer, int batch, int window, int n_heads, int dtype, const void *q,
                                  int64_t q_stride, const int32_t *seqs, const int32_t *in_pos, int sliding, int sinks, float scale,
                                  void *out, int64_t out_stride, void *ws, size_t ws_bytes, void *cuda_stream) {
  int rc = check_pool(pool, false);
  if (rc != SJD_OK) return rc;
  if (dtype != SJD_F32 && dtype != SJD_BF16) return SJD_ERR_UNSUPPORTED;
  if (layer < 0 || layer >= pool->n_layers || batch < 1 || window < 1 || n_heads < 1 || !q || !in_pos || !out || !ws) return SJD_ERR_BAD_ARG;
  if (n_heads % pool->n_kv_heads != 0 || sliding < 0 || sinks < 0 || !(scale >= 0.0f) || scale > 1e30f) return SJD_ERR_BAD_ARG;
  const int64_t row = (int64_t)n_heads * pool->head_dim;
  if (q_stride < row || out_stride < row || ((q_stride | out_stride) & 3)) return SJD_ERR_BAD_ARG;
  if ((((uintptr_t)q | (uintptr_t)out) & (dtype == SJD_F32 ? 15 : 7)) != 0 || ((uintptr_t)ws & 255u) != 0) return SJD_ERR_BAD_ARG;
  const int group = n_heads / pool->n_kv_heads;
  const int64_t rows = (int64_t)window * group;
  // (kMaxGroup: up to there products with group_inv are quotients by the group)
  if (group > kMaxGroup || (int64_t)batch * window > 0x7FFFFFFF || rows > 0x7FFFFFFF) return SJD_ERR_CAPACITY;
  if (ws_bytes < sjd_pool_attention_workspace_bytes(pool, window, n_heads)) return SJD_ERR_CAPACITY;
  int dev = 0, cc_major = 0, sms = 0;
  SJD_CUDA(cudaGetDevice(&dev));
  SJD_CUDA(cudaDeviceGetAttribute(&cc_major, cudaDevAttrComputeCapabilityMajor, dev));
  SJD_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  if (cc_major != 10) return SJD_ERR_UNSUPPORTED;
  TensorMap map;
  rc = make_pool_map(&map, *pool, layer);
  if (rc != SJD_OK) return rc;
  const int rp = tile_rows(rows, dtype), hd = pool->head_dim;
  PoolAttnParams p;
  memset(&p, 0, sizeof(p));
  p.pool = *pool;
  p.layer = layer;
  p.batch = batch;
  p.window = window;
  p.n_heads = n_heads;
  p.group = group;
  p.group_inv = (unsigned)((0x100000000ull + group - 1) / group);   // (not used with 1)
  p.rows = (int)rows;
  p.row_tiles = (int)((rows + rp - 1) / rp);
  p.sliding = sliding;
  p.sinks = sliding > 0 ? sinks : 0;
  p.scale = (scale > 0.0f ? scale : 1.0f / sqrtf((float)hd)) * 1.4426950408889634f;
  p.q = q;
  p.q_stride = q_stride;
  p.out_stride = out_stride;
  p.seqs = seqs;
  p.in_pos = in_pos;
  p.out = out;
  p.cuts = (int4 *)ws;
  p.stats = (float2 *)((char *)ws + kCutBytes);
  p.parts = (float *)((char *)ws + kCutBytes + stat_bytes(rp));
  const int64_t entries = (int64_t)batch * p.row_tiles, units = entries * pool->n_kv_heads;
  if (units > 0x7FFFFFFF) return SJD_ERR_CAPACITY;
  p.cut = pool_equal_ranges(entries, pool->n_kv_heads, (int64_t)batch * window, pool->pages_per_seq, window, sliding, sinks, sms);
  p.n_entries = (int)entries;
  const CUtensorMap &m = reinterpret_cast<const CUtensorMap &>(map);
  auto launch = [&](auto kernel, auto join, int RP, int PL, size_t shared) -> int {
    const int per_sm = ctas_of(RP), tile = kTile * hd, fixed = PL * RP * (kTile + hd) + (int)shared;
    p.slots = (232448 / per_sm - 1024 - fixed) / tile;   // (1 KB of an SM's shared memory goes to every CTA)
    p.slots = p.slots > kMaxSlots ? kMaxSlots : p.slots;
    const size_t smem = (size_t)fixed + (size_t)p.slots * tile;
    const int r = allow_smem(kernel, smem);   // (the size follows from the kernel's types and sizes)
    if (r != SJD_OK) return r;
    const int ctas = sms * per_sm < kMaxCtas ? sms * per_sm : kMaxCtas;
    SJD_CUDA(launch_kernel(kernel, dim3(p.cut ? (unsigned)ctas : (unsigned)units), dim3(threads_of(RP)), smem, (cudaStream_t)cuda_stream, m, p));
    SJD_CHECK_LAUNCH();
    if (!p.cut) return SJD_OK;
    g_pdl = true;   // (waits for the launch before it itself)
    const cudaError_t e = launch_kernel(join, dim3((unsigned)ctas, (unsigned)((RP + kJoinRows - 1) / kJoinRows)), dim3(kJoinRows * 32), 0,
                                        (cudaStream_t)cuda_stream, p, RP);
    g_pdl = false;
    SJD_CUDA(e);
    SJD_CHECK_LAUNCH();
    return SJD_OK;
  };
#define SJD_PICK(T, PL, HD, RP) launch(pool_attention_kernel<T, HD, RP>, pool_attention_join_kernel<T, HD>, RP, PL, sizeof(PoolAttnShared<RP>))
#define SJD_PICK_ROWS(T, PL, RP) (hd == 128 ? SJD_PICK(T, PL, 128, RP) : SJD_PICK(T, PL, 64, RP))
  if (dtype == SJD_F32)
    return rp == 8 ? SJD_PICK_ROWS(float, 4, 8) : rp == 16 ? SJD_PICK_ROWS(float, 4, 16) : rp == 32 ? SJD_PICK_ROWS(float, 4, 32) : SJD_PICK_ROWS(float, 4, 64);
  return rp == 16 ? SJD_PICK_ROWS(__nv_bfloat16, 2, 16) : rp == 32 ? SJD_PICK_ROWS(__nv_bfloat16, 2, 32) : SJD_PICK_ROWS(__nv_bfloat16, 2, 64);
#undef SJD_PICK
#undef SJD_PICK_ROWS
}
