// Attention over the 8-bit paged cache for sequences that share pages: the pages that all tables of a group begin with are attended once,
// with the rows of all its sequences.
//
// Queries are the rows of both products (128 of a stream), keys and dims the columns:
//   S [128 rows x 128 keys]  =  Q . K^T          O [128 rows x HD]  +=  P . V          (tcgen05, sums in 32 bits in tensor memory)
// Keys stay e4m3, as TMA left them; a query is two e4m3 numbers, x1 = e4m3(x) and x2 = e4m3(x - x1) of its entries times a power of two, which hold
// the eight bits of bf16, and both meet the keys in one sum; a block's exponent is a factor of 16 columns of scores.  Values become bf16, entry times
// 2^exponent, which holds it exactly (four bits and any exponent; with exponents left to the weights, as sjd_pool_attention has them, a block's largest
// entry would take places from other blocks' weights): four warps turn a tile for all rows that meet it.  P goes to the second product
// through tensor memory, in the columns of the scores that it was.
// The rows of all sequences of a call follow one another (per kv head), 256 are a unit.  A unit's keys are segments: a group's common pages,
// seen by all of its rows among the unit's, and every sequence's own pages, seen by its rows; the weights of the other rows are zeros.  So a
// unit begins and ends once for many sequences, however short what is theirs alone.
// Two streams of four softmax warps, a row a thread, have 128 rows each: a tile of keys is for both streams, or (a sequence's own) for the one that
// has the rows, and those of the two streams take turns, so that one stream's softmax runs under the other's products.  A unit of up to
// 128 rows gives both streams the same rows and every other tile.
// A weight is taken under a reference that follows the row's maximum only when that has grown by 2^8 (the sums in tensor memory
// then need no factor in nearly all tiles), and rounded to bf16, by up to 2^-8 of itself.
//
// Three launches: a plan (positions, what tables share, the line of units), the tiles, the joining of parts.  The line of all units' tiles is cut into
// equal ranges, a CTA each; a unit that is within one is written by its CTA, the parts of the others are joined in the order of the ranges.
//
// What bounds it (32 heads of 128): the softmax.  A tile of 128 keys for both streams takes 3.0 us (2.9 before a row's factor could change, which is 1 to 2 % of a call),
// where its exponentials alone would take 1.07 by their rate.
// Left out one at a time, the exponentials take 0.8 us with them, half of the maxima 0.2, the turning of the values 0.13, the second numbers of the
// queries 0.04; without a softmax at all the two products and their barriers take 1.8.  Two softmax warps share a scheduler, 43 % of its slots are used.
// Slower: 16 softmax warps with 88 registers; 64 scores at once (by 0.2 us a tile); one pass under the reference that there is, with the maxima behind it (by 0.6 to
// 0.8: more of a row is held at a time, and what is laid aside is far away, for shared memory leaves the cache little room).  Around the tiles 40 to 45 us
// stay the same for any lengths: the plan 7 to 12, queries and first copies 7 to 8, parts 3 to 4, the longest range 6 to 10 beyond the mean, the joining
// launch 11 to 13.
#include "pool_route.h"
#include "tcgen05.cuh"

namespace sjd {
namespace {

constexpr int kKeys = 128;              // of a tile
constexpr int kTileRows = 256;          // of a unit
// Places on the line: of a unit's begin and end, of a tile for both streams, of one for one of them (about 1 us each: 10, 3.1 and 2.0 to 2.3 measured)
constexpr int kUnit = 10, kBoth = 3, kSingle = 2;
constexpr int kLeast = 2;               // common pages that are worth a tile of their own
constexpr int kMaxCtas = 192;
constexpr int kMaxSeqs = SJD_POOL_MAX_LIST;
constexpr int kSegs = 128;              // segments of a unit that are kept there
constexpr int kInfo = 8;                // tiles whose notes are kept: more than copies are ahead of weights (five would do by tests/test_pool_shared_barriers.py)
constexpr int kKStages = 3;
constexpr int kConv = 128, kSoft = 256, kThreads = kSoft + kConv + 96;
constexpr int kPlanThreads = 1024;
constexpr int kCosts = 1024;            // units of a kv head whose places the plan keeps in shared memory
constexpr float kGrow = 8.0f;           // log2 of what a maximum may grow before its reference follows
constexpr float kLeastFactor = 1.1754944e-38f;   // 2^-126
constexpr float kCoarse = 67108864.0f;  // 2^26

struct Segment {       // keys k0 .. k1 - 1 of a sequence's table, for rows ra .. rb - 1 of a unit
  int seq, k0, k1, ra, rb, base;   // base: tiles of the unit's segments for the same streams before it
};
struct Entry {         // 256 rows of a kv head
  int segs;            // first of its segments: those for both streams, for the first, for the second
  int n_segs[3], tiles[3];
  int rows;
};
struct Begin {         // the unit in which a CTA begins
  int e, h, first;     // first: place of its first tile, counted from where the CTA begins
  Entry en;
};
struct SharedParams {
  sjd_pool pool;
  int layer, batch, window, n_heads, group, rows, n_entries, n_groups;   // rows: window * group
  float scale;         // times log2(e)
  const __nv_bfloat16 *q;
  long q_stride, out_stride;
  const int32_t *seqs, *in_pos, *group_begin;
  __nv_bfloat16 *out;
  long *all;           // places of the call
  int *before;         // [n_entries + 1]: places of a kv head in the units before
  Entry *entry;        // [n_entries]
  Segment *segs;
  Begin *begin;        // [ctas]
  float2 *stats;       // (reference, sum) of a row's part
  float *parts;        // [HD / 4][rows of the part][4]
  int ctas;
};

__device__ __forceinline__ int padded(int rows) { return (rows + 7) & ~7; }
__device__ __forceinline__ bool one_stream(int rows) { return rows <= 128; }

__device__ __forceinline__ int row_position(const SharedParams &p, int b, int k, bool tell) {
  int at = p.in_pos[(long)b * p.window + k];
  const int seq = p.seqs ? p.seqs[b] : b;
  if (at < -1 || at >= p.pool.pages_per_seq * KV_PAGE || seq < 0 || seq >= p.pool.n_seqs) {
    if (tell) pool_fault(p.pool.status, SJD_ERR_BAD_ARG);
    at = -1;
  }
  return at;
}

__device__ __forceinline__ int tiles_of(const Entry &en) { return en.tiles[0] + en.tiles[1] + en.tiles[2]; }
__device__ __forceinline__ int places_of(const Entry &en) { return kBoth * en.tiles[0] + kSingle * (en.tiles[1] + en.tiles[2]); }
// tiles of a unit that begin before place t
template <typename Place>
__device__ __forceinline__ int tiles_before(const Entry &en, Place first, Place t) {
  const Place in = t - first;
  if (in <= 0) return 0;
  if (in >= places_of(en)) return tiles_of(en);
  const int n = (int)in;
  return n <= kBoth * en.tiles[0] ? (n + kBoth - 1) / kBoth : en.tiles[0] + (n - kBoth * en.tiles[0] + kSingle - 1) / kSingle;
}
__device__ __forceinline__ long range_of(long all, int ctas) {
  const long least = 2 * kUnit, chunk = (all + ctas - 1) / ctas;
  return chunk < least ? least : chunk;
}

// ---------------------------------------------------------------------------------------------------------------- plan
__global__ void __launch_bounds__(kPlanThreads) shared_plan_kernel(const __grid_constant__ SharedParams p) {
  __shared__ int lo[kMaxSeqs], hi[kMaxSeqs], group_of[kMaxSeqs], seq_of[kMaxSeqs];              // by sequence of the call
  __shared__ int share[kMaxSeqs], leader[kMaxSeqs], live[kMaxSeqs], begin[kMaxSeqs + 1];         // by group
  __shared__ int bad, sums[32], costs[kCosts];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = kPlanThreads / 32;
  pdl_wait();
  pdl_trigger();
  const int groups = p.group_begin ? p.n_groups : 1;
  if (tid == 0) bad = 0;
  for (int g = tid; g <= groups; g += kPlanThreads) {
    begin[g] = p.group_begin ? p.group_begin[g] : g * p.batch;
    if (g < groups) share[g] = leader[g] = 0x7FFFFFFF, live[g] = 0;
  }
  // positions of every sequence, a group of lanes each
  int lanes = 1;
  while (lanes < 32 && lanes < p.window) lanes <<= 1;
  for (int b0 = 0; b0 < p.batch; b0 += kPlanThreads / lanes) {
    const int b = b0 + tid / lanes;
    int l = 0x7FFFFFFF, h = -1;
    if (b < p.batch)
      for (int k = tid % lanes; k < p.window; k += lanes) {
        const int at = row_position(p, b, k, true);
        if (at >= 0) l = min(l, at), h = max(h, at);
      }
    for (int o = lanes >> 1; o > 0; o >>= 1) {
      l = min(l, __shfl_xor_sync(0xffffffffu, l, o));
      h = max(h, __shfl_xor_sync(0xffffffffu, h, o));
    }
    if (b < p.batch && tid % lanes == 0) lo[b] = l, hi[b] = h, seq_of[b] = p.seqs ? p.seqs[b] : b;
  }
  __syncthreads();
  // groups: ranges of sequences that follow one another
  for (int g = tid; g < groups; g += kPlanThreads)
    if (begin[g] < 0 || begin[g + 1] < begin[g] || begin[g + 1] > p.batch || (g == 0 && begin[g] != 0) || (g == groups - 1 && begin[g + 1] != p.batch)) bad = 1;
  __syncthreads();
  if (bad && tid == 0) pool_fault(p.pool.status, SJD_ERR_BAD_ARG);   // (every sequence for itself)
  if (!bad) {
    for (int b = tid; b < p.batch; b += kPlanThreads) {
      int l = 0, h = groups - 1;   // last group that begins at b or before
      while (l < h) {
        const int mid = (l + h + 1) >> 1;
        if (begin[mid] <= b) l = mid; else h = mid - 1;
      }
      group_of[b] = l;
      if (hi[b] < 0) continue;
      atomicMin(&share[l], (lo[b] + 1) / KV_PAGE);
      atomicMin(&leader[l], b);
      atomicAdd(&live[l], 1);
    }
    __syncthreads();
    for (int g = tid; g < groups; g += kPlanThreads)
      if (live[g] < 2) share[g] = 0;
    __syncthreads();
    // pages that the tables of a group begin with: up to the first that differs or is absent
    for (int b = warp; b < p.batch; b += warps) {
      const int g = group_of[b];
      if (hi[b] < 0) continue;
      const int *ta = p.pool.table + (long)seq_of[leader[g]] * p.pool.pages_per_seq, *tb = p.pool.table + (long)seq_of[b] * p.pool.pages_per_seq;
      constexpr int U = 8;
      for (int at = 0;; at += 32 * U) {
        // (other warps lower it meanwhile: one lane looks, and all go by what it saw)
        const int end = __shfl_sync(0xffffffffu, lane == 0 ? *(volatile int *)&share[g] : 0, 0);
        if (at >= end) break;
        int x[U], y[U], least = 0x7FFFFFFF;
#pragma unroll
        for (int j = 0; j < U; ++j) {
          const int i = at + 32 * j + lane;
          x[j] = y[j] = 0;
          if (i < end) x[j] = ta[i], y[j] = tb[i];
        }
#pragma unroll
        for (int j = U - 1; j >= 0; --j)
          if (x[j] != y[j] || x[j] < 0 || x[j] >= p.pool.n_pages) least = at + 32 * j + lane;
        least = __reduce_min_sync(0xffffffffu, least);
        if (least == 0x7FFFFFFF) continue;
        if (lane == 0) atomicMin(&share[g], least);
        break;
      }
    }
    __syncthreads();
    for (int g = tid; g < groups; g += kPlanThreads)
      if (share[g] < kLeast) share[g] = 0;
    __syncthreads();
  }
  // ---- units: their segments, a warp each
  const int all_rows = p.batch * p.rows;
  for (int e = warp; e < p.n_entries; e += warps) {
    const int r0 = e * kTileRows, rows = min(kTileRows, all_rows - r0), b0 = r0 / p.rows, b1 = (r0 + rows - 1) / p.rows;
    const int g0 = bad ? 0 : group_of[b0], n_groups = bad ? 0 : group_of[b1] - g0 + 1, n = n_groups + b1 - b0 + 1;
    int hi0 = -1;   // of the unit's rows of its first sequence, if that has more than a unit's
    if (p.rows > kTileRows) {
      for (int k = (r0 - b0 * p.rows) / p.group + lane; k <= min(p.rows - 1, r0 + rows - 1 - b0 * p.rows) / p.group; k += 32)
        hi0 = max(hi0, row_position(p, b0, k, false));
      hi0 = __reduce_max_sync(0xffffffffu, hi0);
    }
    Entry en;
    en.rows = rows;
    en.segs = b0 + 2 * e + (bad ? 0 : g0);   // (a unit's sequences and groups are those from its first on to the next unit's first, and one each beside)
    int made = 0;
#pragma unroll
    for (int c = 0; c < 3; ++c) {   // for both streams, the first, the second
      en.n_segs[c] = en.tiles[c] = 0;
      if (one_stream(rows) && c != 1) continue;
      for (int i0 = 0; i0 < n; i0 += 32) {
        const int i = i0 + lane;
        Segment s;
        s.k0 = s.k1 = s.ra = s.rb = s.seq = 0;
        if (i < n_groups) {
          const int g = g0 + i;
          if (live[g] > 0) s.seq = seq_of[leader[g]], s.k1 = share[g] * KV_PAGE;
          s.ra = max(0, begin[g] * p.rows - r0), s.rb = min(rows, begin[g + 1] * p.rows - r0);
        } else if (i < n) {
          const int b = b0 + i - n_groups;
          s.seq = seq_of[b], s.k0 = bad ? 0 : share[group_of[b]] * KV_PAGE, s.k1 = (b == b0 && p.rows > kTileRows ? hi0 : hi[b]) + 1;
          if (hi[b] < 0) s.k0 = s.k1 = 0;
          s.ra = max(0, b * p.rows - r0), s.rb = min(rows, (b + 1) * p.rows - r0);
        }
        const int cls = one_stream(rows) || s.rb <= 128 ? 1 : s.ra >= 128 ? 2 : 0;
        const int tiles = s.k1 > s.k0 && s.rb > s.ra && cls == c ? (s.k1 - s.k0 + kKeys - 1) / kKeys : 0;
        int x = tiles;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += y;
        }
        const unsigned have = __ballot_sync(0xffffffffu, tiles > 0);
        s.base = en.tiles[c] + x - tiles;
        if (tiles > 0) p.segs[en.segs + made + __popc(have & ((1u << lane) - 1))] = s;
        made += __popc(have);
        en.n_segs[c] += __popc(have);
        en.tiles[c] += __shfl_sync(0xffffffffu, x, 31);
      }
    }
    if (lane == 0) {
      p.entry[e] = en;
      const int cost = places_of(en);
      (p.n_entries <= kCosts ? costs[e] : p.before[e + 1]) = cost > 0 ? cost + kUnit : 0;   // (its own so far)
    }
  }
  __syncthreads();
  // places on the line, sums over the units before
  const int run = (p.n_entries + kPlanThreads - 1) / kPlanThreads, e0 = min(p.n_entries, tid * run), e1 = min(p.n_entries, e0 + run);
  int cost = 0;
  auto cost_of = [&](int e) { return p.n_entries <= kCosts ? costs[e] : p.before[e + 1]; };
  for (int e = e0; e < e1; ++e) cost += cost_of(e);
  int x = cost;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) sums[warp] = x;
  __syncthreads();
  for (int w = 0; w < warp; ++w) x += sums[w];
  int at = x - cost;
  for (int e = e0; e < e1; ++e) {
    at += cost_of(e);
    p.before[e + 1] = at;
  }
  if (tid == 0) p.before[0] = 0;
  __syncthreads();
  // where every CTA begins
  const long all = (long)p.before[p.n_entries] * p.pool.n_kv_heads, chunk = range_of(all, p.ctas);
  for (int c = tid; c < p.ctas; c += kPlanThreads) {
    const long t = c * chunk;
    Begin b;
    b.e = b.h = b.first = 0;
    if (t < all) {
      int lo = 0, hi = p.n_entries - 1;
      while (lo < hi) {   // last unit that begins at t or before
        const int mid = (lo + hi + 1) >> 1;
        if ((long)p.before[mid] * p.pool.n_kv_heads <= t) lo = mid; else hi = mid - 1;
      }
      const int b0 = p.before[lo], cost = p.before[lo + 1] - b0;
      b.e = lo;
      b.h = (int)((t - (long)b0 * p.pool.n_kv_heads) / cost);
      b.first = (int)((long)b0 * p.pool.n_kv_heads + (long)b.h * cost + kUnit - t);
    }
    b.en = p.entry[b.e];
    p.begin[c] = b;
  }
  if (tid == 0) *p.all = all;
}

// ---------------------------------------------------------------------------------------------------------------- units
// which streams tile i of a unit is for (0, 1, 2: both); `from`: the first tile of the CTA.  The tiles of the two streams take turns.
__device__ __forceinline__ int stream_of(const Entry &en, int i, int from) {
  if (one_stream(en.rows)) return (i - from) & 1;
  const int j = i - en.tiles[0];
  if (j < 0) return 2;
  return j < 2 * min(en.tiles[1], en.tiles[2]) ? j & 1 : en.tiles[1] > en.tiles[2] ? 0 : 1;
}
// first row of a part: of the unit's first tiles, or of those that CTA c goes on with
__device__ __forceinline__ long part_row(const SharedParams &p, int e, int h, bool begins, int c) {
  return begins ? ((long)e * p.pool.n_kv_heads + h) * kTileRows : ((long)p.n_entries * p.pool.n_kv_heads + c) * kTileRows;
}

// ---------------------------------------------------------------------------------------------------------------- tiles
// two fp32 operations an instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t *r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, "
      "%22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t *r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t *r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t *r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// the first operand in tensor memory
__device__ __forceinline__ void umma_bf16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
__device__ __forceinline__ void arrive(uint64_t *bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ float max3(uint32_t a, uint32_t b, uint32_t c) {   // (a NaN is no maximum)
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)), "f"(__uint_as_float(c)));
  return d;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float power_near(float v) {   // a power of two, 2/3 to 4/3 of v (normal and positive)
  return __uint_as_float((__float_as_uint(v) + 0x400000u) & 0x7F800000u);
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Two e4m3 bytes, in the high bytes of the halves of t, as bf16 times 2^-120: their bits moved into place (a subnormal number stays one).
__device__ __forceinline__ uint32_t bf16_bits_of_e4m3(uint32_t t) { return (t & 0x80008000u) | (t >> 4 & 0x07F007F0u); }
__device__ __forceinline__ uint32_t pair_of(float v) { return bf16_pair(v, v); }

struct alignas(16) Info {   // of a tile
  int key0, k1, ra, rb;
  int there;                // bit j: page j of the tile is there
  int v_exp[2];             // exponents of its pages' blocks of values; some are above 0
  int large;
  float k_up[8];            // 2^exponent of its blocks of keys
  uint32_t v_up[8];         // and of values, times 2^120, twice in bf16 (exponents up to 0)
};
// pairs of fp16, and four e4m3 numbers in a word
__device__ __forceinline__ uint32_t halves_of_floats(float a, float b) {
  uint32_t h;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(b), "f"(a));
  return h;
}
__device__ __forceinline__ uint32_t e4m3_of_halves(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("{\n\t.reg .b16 x, y;\n\tcvt.rn.satfinite.e4m3x2.f16x2 x, %1;\n\tcvt.rn.satfinite.e4m3x2.f16x2 y, %2;\n\tmov.b32 %0, {x, y};\n\t}" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ void halves_of_e4m3(uint32_t v, uint32_t &a, uint32_t &b) {
  asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\tcvt.rn.f16x2.e4m3x2 %1, y;\n\t}" : "=r"(a), "=r"(b) : "r"(v));
}
__device__ __forceinline__ uint32_t sub_halves(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ void umma_e4m3(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
// 64 rows of a plane of a page, swizzled; and a plane of a page as it lies
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap *map, int plane, int page, uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(0), "r"(plane), "r"(page), "r"(smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void copy_plane(uint32_t dst, const void *src, uint32_t bytes, uint64_t *bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
// K-major operand of rows of BYTES (64 or 128) under the swizzle of that width
template <int BYTES>
__device__ __forceinline__ uint64_t rows_desc() {
  return (uint64_t)1 << 16 | (uint64_t)(8 * BYTES >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)(BYTES == 128 ? 2 : 4) << 61;
}
template <int BYTES>
__device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t col) {
  return row * BYTES + (BYTES == 128 ? col ^ (row & 7) << 4 : col ^ (row >> 1 & 3) << 4);
}

template <int HD>
struct SharedSmem {
  uint64_t k_full[kKStages], k_empty[kKStages], raw_full[2], raw_empty[2], v_full[2][2], v_empty[2][2], s_full[2][2], p_ready[2][2], o_done[2][2], q_ready, q_seen;
  uint32_t tmem_base;
  Info info[kInfo];
  alignas(4) uint8_t nan_warps[2][2][kConv / 32];      // of half a tile: some entry of V that a warp turned was NaN
  alignas(16) uint16_t nan_dims[2][kKeys][HD / 16];    // which, if so
  float2 stat[2][128];                         // of both streams' rows
  uint32_t nan_row[2][128][HD / 32];
  float factor[2][128];                        // of the scores of a row: the scale, and what its query was multiplied by
  Segment segs[kSegs];
  Begin begin;                                 // where this CTA begins
};

template <int HD>
__global__ void __launch_bounds__(kThreads, 1) shared_tiles_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ SharedParams p) {
  constexpr int OP = 128 * HD;              // bytes of 128 rows of e4m3
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  // queries [stream][plane], keys [stage], values as they come [stage]; values in bf16 [stage][HD / 64][128 rows][128 bytes], 128-byte swizzle
  uint8_t *Qs = smem, *Ks = Qs + 4 * OP, *Rs = Ks + kKStages * OP, *Vs = Rs + 2 * OP;
  SharedSmem<HD> &sh = *reinterpret_cast<SharedSmem<HD> *>(Vs + 4 * OP);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, kv_heads = p.pool.n_kv_heads;
  constexpr int ISSUE = (kSoft + kConv) / 32, COPY = ISSUE + 2;   // (a warp issues the products of a stream)
  if (tid == 0) {
    for (int i = 0; i < kKStages; ++i) {
      mbar_init(&sh.k_full[i], 1);
      mbar_init(&sh.k_empty[i], 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.raw_full[i], 1);
      mbar_init(&sh.raw_empty[i], kConv / 32);
      for (int h = 0; h < 2; ++h) {
        mbar_init(&sh.v_full[i][h], kConv / 32);
        mbar_init(&sh.v_empty[i][h], 2);
        mbar_init(&sh.s_full[i][h], 1);
        mbar_init(&sh.p_ready[i][h], 4);
        mbar_init(&sh.o_done[i][h], 1);
      }
    }
    mbar_init(&sh.q_ready, kSoft / 32);
    mbar_init(&sh.q_seen, 2);
    tma_prefetch_desc(&map);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == ISSUE) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  const long all = *p.all;
  if (tid < (int)(sizeof(Begin) / 4)) reinterpret_cast<int *>(&sh.begin)[tid] = reinterpret_cast<const int *>(p.begin + blockIdx.x)[tid];
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_trigger();   // (not before the allocation: a CTA of a later kernel that holds tensor memory waits for this one)
  const uint32_t tmem = sh.tmem_base;
  const long chunk = range_of(all, gridDim.x);
  const int places = (int)max(0l, min(chunk, all - blockIdx.x * chunk));   // of this CTA
  auto fail = [&]() {
    if (lane == 0) pool_fault(p.pool.status, SJD_ERR_DEVICE_TIMEOUT);
  };
  // This CTA's units that have tiles in its range, one after the other: tiles i0 .. i1 - 1 of one.
  struct Span {
    int e, h, next;    // next: the place behind it (-1: before the first)
    Entry en;
    int i0, i1;
  };
  auto next_span = [&](Span &s) {
    for (;;) {
      int first;
      if (s.next < 0) {
        if (places == 0) return false;
        s.e = sh.begin.e, s.h = sh.begin.h, s.en = sh.begin.en, first = sh.begin.first;
      } else {
        if (s.next >= places) return false;
        if (++s.h == kv_heads) {
          s.h = 0;
          do s.en = p.entry[++s.e];
          while (tiles_of(s.en) == 0);   // (there is one: the line goes on)
        }
        first = s.next + kUnit;
      }
      s.i0 = tiles_before(s.en, first, 0);
      s.i1 = tiles_before(s.en, first, places);
      s.next = first + places_of(s.en);
      if (s.i1 > s.i0) return true;
    }
  };

  if (warp == COPY) {
    // ------------------------------------------------------------------ copies: what 32 tiles are is looked up together, a lane each
    const long plane = (long)KV_PAGE * HD, head_planes = 2l * kv_heads, page_planes = head_planes * p.pool.n_layers;
    struct Batch {
      int n, h;                                   // tiles, kv head
      int key0, k1, ra, rb, page[2], k_exp[2], v_exp[2];   // of this lane's
    };
    Span s;
    s.next = -1;
    bool more = false, kept = false;
    int i = 0;
    auto begin_span = [&]() {
      more = next_span(s);
      if (!more) return;
      i = s.i0;
      const int n = s.en.n_segs[0] + s.en.n_segs[1] + s.en.n_segs[2];
      kept = n <= kSegs;
      __syncwarp();
      if (kept)
        for (int j = lane; j < n * (int)(sizeof(Segment) / 4); j += 32) reinterpret_cast<int *>(sh.segs)[j] = reinterpret_cast<const int *>(p.segs + s.en.segs)[j];
      __syncwarp();
    };
    auto look_up = [&](Batch &b) {
      b.n = 0;
      if (!more) return;
      b.n = min(32, s.i1 - i);
      b.h = s.h;
      const int x = min(i + lane, s.i1 - 1);
      // its kind, its number among that kind's, its segment: the last of them that begins there or before
      const int st = stream_of(s.en, x, s.i0), kind = one_stream(s.en.rows) ? 1 : st == 2 ? 0 : st + 1;
      int j = x;
      if (kind > 0) {
        const int turns = min(s.en.tiles[1], s.en.tiles[2]);
        j = x - s.en.tiles[0];
        j = j < 2 * turns ? j >> 1 : j - turns;
      }
      const int from = kind == 0 ? 0 : kind == 1 ? s.en.n_segs[0] : s.en.n_segs[0] + s.en.n_segs[1];
      int lo = from, hi = from + (kind == 0 ? s.en.n_segs[0] : kind == 1 ? s.en.n_segs[1] : s.en.n_segs[2]) - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((kept ? sh.segs[mid].base : p.segs[s.en.segs + mid].base) <= j) lo = mid; else hi = mid - 1;
      }
      const Segment g = kept ? sh.segs[lo] : p.segs[s.en.segs + lo];
      b.key0 = g.k0 + (j - g.base) * kKeys;
      b.k1 = g.k1, b.ra = g.ra, b.rb = g.rb;
#pragma unroll
      for (int k = 0; k < 2; ++k)
        b.page[k] = b.key0 + k * KV_PAGE < g.k1 ? p.pool.table[(long)g.seq * p.pool.pages_per_seq + b.key0 / KV_PAGE + k] : -1;
      i += b.n;
      if (i == s.i1) begin_span();
    };
    auto look_up_exps = [&](Batch &b) {
      if (b.n == 0) return;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        b.k_exp[k] = b.v_exp[k] = 0;
        if ((unsigned)b.page[k] >= (unsigned)p.pool.n_pages) b.page[k] = -1;
        if (b.page[k] < 0) continue;
        const long at = (long)b.page[k] * page_planes + head_planes * p.layer + b.h;
        b.k_exp[k] = *reinterpret_cast<const int *>(p.pool.exps + at * kPoolBlocks);
        b.v_exp[k] = *reinterpret_cast<const int *>(p.pool.exps + (at + kv_heads) * kPoolBlocks);
      }
    };
    Batch now, next;
    begin_span();
    look_up(now);
    look_up_exps(now);
    bool ok = true;
    uint32_t made = 0;
    int stage = 0;
    uint32_t ph = 1;
    while (now.n > 0 && ok) {
      look_up(next);
#pragma unroll 1
      for (int k = 0; k < now.n && ok; ++k, ++made) {
        if (k == now.n / 2) look_up_exps(next);
        const int page0 = __shfl_sync(0xffffffffu, now.page[0], k), page1 = __shfl_sync(0xffffffffu, now.page[1], k);
        const int boxes = (page0 >= 0) + (page1 >= 0);
        ok = made < kKStages || warp_wait(&sh.k_empty[stage], ph);
        if (!ok) break;
        if (lane == k) {   // (its notes are read by those who wait for the copies)
          Info f;
          f.key0 = now.key0, f.k1 = now.k1, f.ra = now.ra, f.rb = now.rb;
          f.v_exp[0] = now.v_exp[0], f.v_exp[1] = now.v_exp[1], f.large = 0;
          f.there = (page0 >= 0 ? 1 : 0) | (page1 >= 0 ? 2 : 0);
#pragma unroll
          for (int b = 0; b < 8; ++b) {
            const int e = pool_exp((int8_t)((b < 4 ? now.v_exp[0] : now.v_exp[1]) >> (8 * (b & 3))));
            f.k_up[b] = two_to(pool_exp((int8_t)((b < 4 ? now.k_exp[0] : now.k_exp[1]) >> (8 * (b & 3)))));
            f.v_up[b] = pair_of(two_to(min(e, 0) + 120));
            f.large |= e > 0;
          }
          sh.info[made % kInfo] = f;
          __threadfence_block();
        }
        __syncwarp();
        if (elect_one()) {
          const uint32_t dst = smem_u32(Ks) + stage * OP;
          if (boxes > 0) mbar_expect_tx(&sh.k_full[stage], boxes * (OP / 2)); else arrive(&sh.k_full[stage]);
          if (page0 >= 0) copy_box(dst, &map, now.h, page0, &sh.k_full[stage]);
          if (page1 >= 0) copy_box(dst + OP / 2, &map, now.h, page1, &sh.k_full[stage]);
        }
        __syncwarp();
        const int raw = made & 1;
        ok = made < 2 || warp_wait(&sh.raw_empty[raw], (made >> 1 & 1) ^ 1u);
        if (!ok) break;
        if (elect_one()) {
          const uint32_t dst = smem_u32(Rs) + raw * OP;
          const uint8_t *from = (const uint8_t *)p.pool.pages + (head_planes * p.layer + kv_heads + now.h) * plane;
          if (boxes > 0) mbar_expect_tx(&sh.raw_full[raw], boxes * (OP / 2)); else arrive(&sh.raw_full[raw]);
          if (page0 >= 0) copy_plane(dst, from + page0 * page_planes * plane, OP / 2, &sh.raw_full[raw]);
          if (page1 >= 0) copy_plane(dst + OP / 2, from + page1 * page_planes * plane, OP / 2, &sh.raw_full[raw]);
        }
        __syncwarp();
        if (++stage == kKStages) { stage = 0; ph ^= 1u; }
      }
      now = next;
    }
    if (!ok) fail();
    // leave no copy in flight
    for (uint32_t j = made > kKStages ? made - kKStages : 0; j < made; ++j) warp_wait(&sh.k_full[j % kKStages], j / kKStages & 1);
    for (uint32_t j = made > 2 ? made - 2 : 0; j < made; ++j) warp_wait(&sh.raw_full[j & 1], j >> 1 & 1);
  } else if (warp >= kSoft / 32 && warp < ISSUE) {
    // ------------------------------------------------------------------ values: e4m3 to bf16
    constexpr int SEG = HD / 16, ROWS = kConv / SEG, N = kKeys / ROWS;   // lanes of a row, rows at a time, 16-byte loads of a thread
    const int ct = tid - kSoft, seg = ct % SEG, row0 = ct / SEG, cw = ct >> 5;
    // (ROWS is a multiple of 8: a thread's rows have one swizzle)
    const uint32_t at0 = (uint32_t)(seg >> 2) * (128 * 128) + row0 * 128 + ((((seg & 3) * 2) ^ (row0 & 7)) << 4);
    long tiles = 0;
    {
      Span s;
      s.next = -1;
      while (next_span(s)) tiles += s.i1 - s.i0;
    }
    bool ok = true;
    for (uint32_t made = 0; made < tiles && ok; ++made) {
      const int stage = made & 1;
      ok = warp_wait(&sh.raw_full[stage], made >> 1 & 1);
      if (!ok) break;
      const Info &f = sh.info[made % kInfo];
      const uint8_t *from = Rs + stage * OP + row0 * HD + seg * 16;
      uint8_t *to = Vs + stage * 2 * OP + at0;
      const int left = f.k1 - f.key0 - row0, there = f.there, large = f.large;   // left: rows of this thread that there are
      // (a half as soon as the products with the one there are done)
#pragma unroll 1
      for (int h = 0; h < 2 && ok; ++h) {
        ok = made < 2 || warp_wait(&sh.v_empty[stage][h], (made >> 1 & 1) ^ 1u);
        if (!ok) break;
        uint32_t nan = 0;
        // two loads at a time: as many independent numbers as it takes, and a loop that is short to fetch
#pragma unroll 1
        for (int n0 = h * (N / 2); n0 < (h + 1) * (N / 2); n0 += 2) {
          uint4 x[2];
          uint32_t out[2][8], up[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int n = n0 + j;
            x[j] = *reinterpret_cast<const uint4 *>(from + n * ROWS * HD);
            if (!(there >> (n / (N / 2)) & 1) || n * ROWS >= left) x[j] = make_uint4(0, 0, 0, 0);
            up[j] = f.v_up[(row0 + n * ROWS) >> 4];
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
            uint32_t any = 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              out[j][2 * c] = mul_bf16x2(bf16_bits_of_e4m3(__byte_perm(w[c], 0, 0x1404)), up[j]);
              out[j][2 * c + 1] = mul_bf16x2(bf16_bits_of_e4m3(__byte_perm(w[c], 0, 0x3424)), up[j]);
              any |= (w[c] & 0x7F7F7F7Fu) + 0x01010101u;
            }
            nan |= any & 0x80808080u;
          }
          if (__builtin_expect(large, 0)) {   // (exponents above 0 in a second step)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const int block = (row0 + (n0 + j) * ROWS) >> 4;
              const uint32_t over = pair_of(two_to(max(pool_exp((int8_t)((block < 4 ? f.v_exp[0] : f.v_exp[1]) >> (8 * (block & 3)))), 0)));
#pragma unroll
              for (int c = 0; c < 8; ++c) out[j][c] = mul_bf16x2(out[j][c], over);
            }
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint8_t *dst = to + (n0 + j) * ROWS * 128;
            *reinterpret_cast<uint4 *>(dst) = make_uint4(out[j][0], out[j][1], out[j][2], out[j][3]);
            *reinterpret_cast<uint4 *>((uint8_t *)((uintptr_t)dst ^ 16)) = make_uint4(out[j][4], out[j][5], out[j][6], out[j][7]);
          }
        }
        const bool found = __any_sync(0xffffffffu, nan != 0);
        if (__builtin_expect(found, 0)) {   // NaN entries become zeros, and are told
#pragma unroll 1
          for (int n = h * (N / 2); n < (h + 1) * (N / 2); ++n) {
            uint32_t dims = 0;
            uint16_t *dst = reinterpret_cast<uint16_t *>(to + n * ROWS * 128);
            const bool row = (there >> (n / (N / 2)) & 1) && n * ROWS < left;
#pragma unroll 1
            for (int c = 0; c < 16; ++c) {
              if (!row || (from[n * ROWS * HD + c] & 0x7F) != 0x7F) continue;
              dims |= 1u << c;
              *reinterpret_cast<uint16_t *>((uintptr_t)(dst + (c & 7)) ^ (c < 8 ? 0 : 16)) = 0;
            }
            sh.nan_dims[stage][row0 + n * ROWS][seg] = (uint16_t)dims;
          }
        }
        if (lane == 0) sh.nan_warps[stage][h][cw] = found;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          if (h == 1) arrive(&sh.raw_empty[stage]);
          arrive(&sh.v_full[stage][h]);
        }
      }
    }
    if (!ok) fail();
  } else if (warp == ISSUE || warp == ISSUE + 1) {
    // ------------------------------------------------------------------ products of a stream; of tiles that are the other's alone it only lets go
    constexpr uint32_t idesc_s = (1u << 4) | (uint32_t)(kKeys / 2 >> 3) << 17 | (uint32_t)(128 >> 4) << 24;   // e4m3 both
    constexpr uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | 1u << 16 | (uint32_t)(HD >> 3) << 17 | (uint32_t)(128 >> 4) << 24;   // V: dims follow one another
    const int st = warp - ISSUE;
    const uint64_t desc_k = rows_desc<HD>() | (uint64_t)(smem_u32(Ks) >> 4);
    const uint64_t desc_v = (uint64_t)(128 * 128 >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61 | (uint64_t)(smem_u32(Vs) >> 4);
    const uint32_t t_s = tmem + st * 128, t_o = tmem + 256 + st * 128;
    Span s;
    s.next = -1;
    bool ok = true;
    uint32_t q_ph = 0, p_ph = 0;
    int k_stage = 0, v_stage = 0;
    uint32_t k_ph = 0, v_ph = 0;
    while (ok && next_span(s)) {
      ok = warp_wait(&sh.q_ready, q_ph);
      q_ph ^= 1u;
      if (lane == 0) arrive(&sh.q_seen);
      const uint64_t desc_q = rows_desc<HD>() | (uint64_t)((smem_u32(Qs) + (one_stream(s.en.rows) ? 0 : st * 2 * OP)) >> 4);
      // Scores of the halves of the own tiles before `end`, each when the weights in its columns have been multiplied.  (No further than two tiles ahead
      // of the values: what the copies wait for is let go of there.  Three meet parities that have come round: tests/test_pool_shared_barriers.py.)
      int i = s.i0;
      bool half = false, open0 = false, open1 = false;   // the first half of tile i has its scores; weights that have not been multiplied
      auto products = [&](int h) {
        const uint64_t b = desc_k + k_stage * (OP >> 4) + h * (OP / 2 >> 4);
#pragma unroll
        for (int k = 0; k < HD / 32; ++k) umma_e4m3(t_s + h * 64, desc_q + k * 2, b + k * 2, idesc_s, k > 0);
#pragma unroll
        for (int k = 0; k < HD / 32; ++k) umma_e4m3(t_s + h * 64, desc_q + (OP >> 4) + k * 2, b + k * 2, idesc_s, true);
        umma_commit(&sh.s_full[st][h]);
      };
      auto scores = [&](int end) {
        for (; i < min(end, s.i1); ++i) {
          const int c = stream_of(s.en, i, s.i0);
          const bool own = c == 2 || c == st;
          if (!half) {
            if (own && open0) return;
            ok = warp_wait(&sh.k_full[k_stage], k_ph);
            if (!ok) return;
            tc_fence_after();
            if (elect_one()) {
              if (own) products(0);
              else arrive(&sh.k_empty[k_stage]);
            }
            __syncwarp();
            if (own) half = open0 = true;
          }
          if (own) {
            if (open1) return;
            if (elect_one()) {
              products(1);
              umma_commit(&sh.k_empty[k_stage]);
            }
            __syncwarp();
            open1 = true;
            half = false;
          }
          if (++k_stage == kKStages) { k_stage = 0; k_ph ^= 1u; }
        }
      };
      scores(s.i0 + 2);
      bool begun = false;
      for (int j = s.i0; j < s.i1 && ok; ++j) {
        const int c = stream_of(s.en, j, s.i0);
        const bool own = c == 2 || c == st;
        if (own) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (ok) ok = warp_wait_both(&sh.p_ready[st][h], p_ph, &sh.v_full[v_stage][h], v_ph);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
              const uint64_t b = desc_v + v_stage * (2 * OP >> 4) + h * (64 * 128 >> 4);
#pragma unroll
              for (int k = 0; k < kKeys / 32; ++k) umma_bf16_ts(t_o, t_s + h * 64 + (k >> 1) * 32 + (k & 1) * 8, b + k * (16 * 128 >> 4), idesc_o, begun || h > 0 || k > 0);
              umma_commit(&sh.o_done[st][h]);
              umma_commit(&sh.v_empty[v_stage][h]);
            }
            __syncwarp();
            (h == 0 ? open0 : open1) = false;
            if (h == 0) scores(j + 3);
          }
          begun = true;
          p_ph ^= 1u;
        } else {
          ok = warp_wait_both(&sh.v_full[v_stage][0], v_ph, &sh.v_full[v_stage][1], v_ph);
          if (ok && elect_one()) arrive(&sh.v_empty[v_stage][0]), arrive(&sh.v_empty[v_stage][1]);
          __syncwarp();
        }
        if (ok) scores(j + 3);
        v_stage ^= 1;
        v_ph ^= v_stage == 0;
      }
    }
    if (!ok) fail();
  } else {
    // ------------------------------------------------------------------ softmax warps: a row a thread
    const int st = warp >> 2, quarter = warp & 3, r_in = quarter * 32 + lane;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16, t_s = tmem + lanes + st * 128, t_o = tmem + lanes + 256;
    auto sync = [&]() { asm volatile("bar.sync 1, %0;" ::"n"(kSoft) : "memory"); };
    Span s;
    s.next = -1;
    bool ok = true;
    uint32_t tile0 = 0, done = 0, q_ph = 1;   // done: this stream's tiles so far
    while (next_span(s)) {
      tile0 -= s.i0;
      const int rows = s.en.rows, row_first = s.e * kTileRows;
      const bool alone = one_stream(rows);
      const int r = r_in + (alone ? 0 : st * 128);
      int pos = -1;   // of this thread's row
      // (a stream without tiles in the unit before may not have looked for its queries yet, and would miss them behind the next ones)
      if (ok && !warp_wait(&sh.q_seen, q_ph)) {
        ok = false;
        fail();
      }
      q_ph ^= 1u;
      // ---- queries of the unit's rows: a power of two brings a row's largest entry to 128 .. 256, then its two numbers; a row is HD / 8 lanes
      {
        constexpr int LANES = HD / 8, PER = 32 / LANES, U = 4, STEP = kSoft / 32 * PER;   // lanes of a row, rows of a warp's load, loads under way, rows between them
        const int sub = lane / LANES, dim = lane % LANES * 8;
        const __nv_bfloat16 *q = p.q + (long)s.h * p.group * HD + dim;
        auto load = [&](int r0, uint2 (&x)[U][2]) {
#pragma unroll
          for (int j = 0; j < U; ++j) {
            const int y = row_first + min(r0 + j * STEP + sub, rows - 1), m = y / p.group;
            const uint2 *from = reinterpret_cast<const uint2 *>(q + (long)m * p.q_stride + (y - m * p.group) * HD);
            x[j][0] = from[0], x[j][1] = from[1];
          }
        };
        uint2 x[U][2], next[U][2];
        load(warp * PER, x);
#pragma unroll 1
        for (int r0 = warp * PER; r0 < rows; r0 += STEP * U) {
          load(r0 + STEP * U, next);   // (behind the last: the last row)
          // (each step for all of the rows: it takes that many to hide its latency)
          float v[U][8], top[U], up[U];
          int e[U];
#pragma unroll
          for (int j = 0; j < U; ++j) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              v[j][4 * c] = __uint_as_float(x[j][c].x << 16), v[j][4 * c + 1] = __uint_as_float(x[j][c].x & 0xFFFF0000u);
              v[j][4 * c + 2] = __uint_as_float(x[j][c].y << 16), v[j][4 * c + 3] = __uint_as_float(x[j][c].y & 0xFFFF0000u);
            }
            top[j] = fmaxf(fmaxf(fmaxf(fabsf(v[j][0]), fabsf(v[j][1])), fmaxf(fabsf(v[j][2]), fabsf(v[j][3]))),
                           fmaxf(fmaxf(fabsf(v[j][4]), fabsf(v[j][5])), fmaxf(fabsf(v[j][6]), fabsf(v[j][7]))));
            x[j][0] = next[j][0], x[j][1] = next[j][1];
          }
#pragma unroll
          for (int o = LANES / 2; o > 0; o >>= 1) {
            float other[U];
#pragma unroll
            for (int j = 0; j < U; ++j) other[j] = __shfl_xor_sync(0xffffffffu, top[j], o);
#pragma unroll
            for (int j = 0; j < U; ++j) top[j] = fmaxf(top[j], other[j]);
          }
          uint32_t h[U][4], first[U][2];   // (fp16 holds eight bits of what is 2^-10 or more)
#pragma unroll
          for (int j = 0; j < U; ++j) {
            e[j] = top[j] > 0.0f ? 7 - (int)((__float_as_uint(top[j]) >> 23) - 127) : 0;
            e[j] = max(min(e[j], 126), -126);   // (entries below 2^-119 lose places)
            up[j] = top[j] == INFINITY ? __int_as_float(0x7FFFFFFF) : two_to(e[j]);   // (e4m3 has no infinity: its row is NaN, as it would be)
          }
#pragma unroll
          for (int j = 0; j < U; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) h[j][c] = halves_of_floats(v[j][2 * c] * up[j], v[j][2 * c + 1] * up[j]);
#pragma unroll
          for (int j = 0; j < U; ++j)
#pragma unroll
            for (int c = 0; c < 2; ++c) first[j][c] = e4m3_of_halves(h[j][2 * c], h[j][2 * c + 1]);
#pragma unroll
          for (int j = 0; j < U; ++j) {
            const int y = r0 + j * STEP + sub;
            uint32_t second[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              uint32_t a, b;
              halves_of_e4m3(first[j][c], a, b);
              second[c] = e4m3_of_halves(sub_halves(h[j][2 * c], a), sub_halves(h[j][2 * c + 1], b));
            }
            if (y < rows) {
              uint8_t *to = Qs + (y >> 7) * 2 * OP + swizzled<HD>(y & 127, dim);   // (eight bytes stay together)
              *reinterpret_cast<uint2 *>(to) = make_uint2(first[j][0], first[j][1]);
              *reinterpret_cast<uint2 *>(to + OP) = make_uint2(second[0], second[1]);
              if (dim == 0) sh.factor[y >> 7][y & 127] = p.scale * two_to(-e[j]);
            }
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) arrive(&sh.q_ready);
        if (r < rows) {
          const int m = (row_first + r) / p.group, b = m / p.window;
          pos = row_position(p, b, m - b * p.window, false);
        }
        sync();   // (the factors are there)
      }
      float factor = r < rows ? sh.factor[r >> 7][r & 127] : 0.0f;
      const bool warp_rows = quarter * 32 + (alone ? 0 : st * 128) < rows;   // this warp has any
      float m_ref = -INFINITY, l = 0.0f;
      bool nans = false;   // the row has seen some: sh.nan_row says which dims
      int mine = 0;
      for (int i = s.i0; i < s.i1; ++i) {
        const int c = stream_of(s.en, i, s.i0);
        if (c != 2 && c != st) continue;
        const uint32_t use = tile0 + i, stage = use & 1;
        const Info &f = sh.info[use % kInfo];
        int limit = 0, there = 0, key0 = 0;
        // (the halves take turns: while one is worked on, the other's weights are multiplied and its next scores come)
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          if (ok && !warp_wait(&sh.s_full[st][h], done & 1)) {
            ok = false;
            fail();
          }
          tc_fence_after();
          if (h == 0) {
            const int4 a = *reinterpret_cast<const int4 *>(&f);
            key0 = a.x, there = f.there;
            limit = r >= a.z && r < a.w ? min(pos, a.y - 1) : -1;   // the last key that this row sees
            ++mine;
          }
          const uint32_t t_h = t_s + h * 64;
          int n_seen = min(max(limit - (key0 + h * 64) + 1, 0), 64);   // of the 64 keys (no row: any number)
          if (!(there >> h & 1)) {
            if (n_seen > 0) pool_fault(p.pool.status, SJD_ERR_BAD_ARG);   // (no page where the row sees a key)
            n_seen = 0;
          }
          if (__any_sync(0xffffffffu, n_seen > 0)) {
            // 32 scores at a time, the first of them twice: more do not fit beside the rest of the registers, and what the compiler lays aside is far away (shared
            // memory leaves the cache little room: with 64 at once, 136 bytes laid aside, a tile of two streams took 0.2 us more)
            const bool all = __all_sync(0xffffffffu, n_seen == 64 || r >= rows);
            uint32_t x[32];
            auto load = [&](int k) { tmem_ld32(t_h + k * 32, x); };
            auto hide = [&](int k) {   // scores of keys that the row does not see
              const int n = n_seen - 32 * k;
              const uint32_t bits = n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1;
#pragma unroll
              for (int j = 0; j < 32; ++j) x[j] = bits >> j & 1u ? x[j] : 0xFF800000u;
            };
            load(0);
            const float4 up = *reinterpret_cast<const float4 *>(&f.k_up[h * 4]);
            // of 16 columns; never zero: masked scores stay infinite (others, up to 2^24, are nothing with a factor this small)
            float by[4] = {fmaxf(factor * up.x, kLeastFactor), fmaxf(factor * up.y, kLeastFactor), fmaxf(factor * up.z, kLeastFactor), fmaxf(factor * up.w, kLeastFactor)};
            float top = -INFINITY;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              tmem_ld_wait();
              if (!all) hide(k);
              float tops[2];
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                const uint32_t *v = x + 16 * c;
                const float a = max3(v[0], v[1], v[2]), b = max3(v[3], v[4], v[5]), d = max3(v[6], v[7], v[8]), e = max3(v[9], v[10], v[11]), g = max3(v[12], v[13], v[14]);
                tops[c] = max3(__float_as_uint(max3(__float_as_uint(a), __float_as_uint(b), __float_as_uint(d))), __float_as_uint(fmaxf(e, g)), v[15]) * by[2 * k + c];
              }
              if (k == 0) load(1);
              top = max3(__float_as_uint(top), __float_as_uint(tops[0]), __float_as_uint(tops[1]));
            }
            // Where a score has outgrown the reference, that, O and the sum follow.
            const bool need = r < rows && (top > m_ref + kGrow || (m_ref == -INFINITY && top > -INFINITY));
            if (__builtin_expect(__any_sync(0xffffffffu, need), 0)) {
              // A weight's argument is the exact product less the reference, a rounded one, which is off from its own exact one by 4 at 2^26 and beyond what an exponential
              // holds at 2^31. While it is 2^26 or more, or as far below zero, the row's factor is a power of two: products are exact then. (Its scores are off by 2^7 and more
              // as they are, and smaller differences, in which alone a factor of 2/3 to 4/3 could show, mean nothing.)
              const float asked = need ? sh.factor[r >> 7][r & 127] : factor, use = need && fabsf(top) >= kCoarse ? power_near(asked) : asked;
              const bool other = factor != use;
              if (__builtin_expect(__any_sync(0xffffffffu, other), 0)) {
                if (other) m_ref *= use / factor, factor = use, top = -INFINITY;
#pragma unroll 1
                for (int c = 0; c < 8; ++c) {
                  uint32_t v[8];
                  tmem_ld8(t_h + c * 8, v);
                  tmem_ld_wait();
#pragma unroll
                  for (int j = 0; j < 8; ++j)
                    if (other && c * 8 + j < n_seen) top = fmaxf(top, __uint_as_float(v[j]) * fmaxf(factor * f.k_up[h * 4 + c / 2], kLeastFactor));
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) by[c] = fmaxf(factor * f.k_up[h * 4 + c], kLeastFactor);
              }
              const float g = need ? exp2_fast(m_ref - top) : 1.0f;
              m_ref = need ? top : m_ref;
              l *= g;
              if (mine > 1 || h > 0) {   // O has been written
                // (the scores have waited for the products of their half of the tile before; those of the half before this one may be under way)
                if (ok && !warp_wait(&sh.o_done[st][h ^ 1], (done - 1 + h) & 1)) {
                  ok = false;
                  fail();
                }
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < HD / 8; ++c) {
                  uint32_t v[8];
                  tmem_ld8(t_o + st * 128 + c * 8, v);
                  tmem_ld_wait();
#pragma unroll
                  for (int j = 0; j < 8; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * g);
                  tmem_st8(t_o + st * 128 + c * 8, v);
                }
              }
            }
            const float ref = m_ref == -INFINITY ? 0.0f : m_ref;
            float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
            for (int k = 1; k >= 0; --k) {   // (the second 32 scores are still here)
              if (k == 0) {
                load(0);
                tmem_ld_wait();
                if (!all) hide(0);
              }
#pragma unroll
              for (int c = 0; c < 2; ++c) {   // 16 at a time, and each operation for all of them: it takes that many to hide its latency
                float2 y[8];
                uint32_t w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                  y[j] = fma2(make_float2(__uint_as_float(x[16 * c + 2 * j]), __uint_as_float(x[16 * c + 2 * j + 1])), make_float2(by[2 * k + c], by[2 * k + c]), make_float2(-ref, -ref));
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j].x = exp2_fast(y[j].x), y[j].y = exp2_fast(y[j].y);
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = bf16_pair(y[j].x, y[j].y);
                tmem_st8(t_h + k * 32 + c * 8, w);   // (over their own scores)
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = add2(y[j], y[j + 4]);
#pragma unroll
                for (int j = 0; j < 2; ++j) sum[j] = add2(sum[j], add2(y[j], y[j + 2]));
              }
            }
            l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
            tmem_st_wait();
          } else if (warp_rows) {   // (a warp without rows that see them: no weights)
            uint32_t w[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) w[k] = 0;
            tmem_st16(t_h, w);
            tmem_st16(t_h + 32, w);
            tmem_st_wait();
          }
          tc_fence_before();
          // NaN entries of V, which are zeros there, and the rows that see them
          if (ok && !warp_wait(&sh.v_full[stage][h], use >> 1 & 1)) {
            ok = false;
            fail();
          }
          if (__builtin_expect(*reinterpret_cast<const uint32_t *>(sh.nan_warps[stage][h]) != 0, 0)) {
            constexpr int ROWS = kConv / (HD / 16), WARP = 32 / (HD / 16);
#pragma unroll 1
            for (int k = h * 64; k < h * 64 + 64; ++k) {
              if (!sh.nan_warps[stage][h][k % ROWS / WARP] || key0 + k > limit) continue;
#pragma unroll
              for (int j = 0; j < HD / 32; ++j) sh.nan_row[st][r_in][j] = (nans ? sh.nan_row[st][r_in][j] : 0u) | *reinterpret_cast<const uint32_t *>(&sh.nan_dims[stage][k][2 * j]);
              nans = true;
            }
          }
          __syncwarp();
          if (lane == 0) arrive(&sh.p_ready[st][h]);
        }
        ++done;
      }
      // ---- what this CTA has of the unit: references, sums and O
      if (mine > 0) {
        if (ok && !warp_wait_both(&sh.o_done[st][0], (done - 1) & 1, &sh.o_done[st][1], (done - 1) & 1)) {
          ok = false;
          fail();
        }
        tc_fence_after();
      }
      if (const float asked = r < rows ? sh.factor[r >> 7][r & 127] : 0.0f; factor != asked) m_ref *= asked / factor;   // (in the unit that all parts have)
      const bool complete = s.i0 == 0 && s.i1 == tiles_of(s.en);
      const long row = part_row(p, s.e, s.h, s.i0 == 0, blockIdx.x);
      const int stride = padded(rows);
      float4 *parts = reinterpret_cast<float4 *>(p.parts + row * HD) + r;   // [HD / 4][padded rows]
      __nv_bfloat16 *out = p.out;
      if (r < rows) {
        const int m = (row_first + r) / p.group;
        out += (long)m * p.out_stride + ((long)s.h * p.group + (row_first + r - m * p.group)) * HD;
      }
      // 32 dims of this row, times f (the whole unit: outputs)
      auto store = [&](int k, const float *v, float f) {
        if (r >= rows) return;
        if (complete) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            *reinterpret_cast<uint2 *>(out + k * 32 + j * 4) = f == 0.0f ? make_uint2(0u, 0u) : make_uint2(bf16_pair(v[4 * j] * f, v[4 * j + 1] * f), bf16_pair(v[4 * j + 2] * f, v[4 * j + 3] * f));
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) parts[(k * 8 + j) * stride] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        }
      };
      float2 a = make_float2(m_ref, l), b = make_float2(-INFINITY, 0.0f);
      bool second = false;
      if (alone) {   // both streams have sums of the same rows: each joins half of the dims
        sh.stat[st][r_in] = a;
        if (!nans) {
#pragma unroll
          for (int j = 0; j < HD / 32; ++j) sh.nan_row[st][r_in][j] = 0;
        }
        tc_fence_before();
        sync();
        tc_fence_after();   // (the other stream's products, which its warps have waited for)
        second = s.i1 - s.i0 > 1;
        a = sh.stat[0][r_in];
        if (second) b = sh.stat[1][r_in];
        nans = true;
      }
      if (warp_rows) {
        const float best = fmaxf(a.x, b.x), f0 = a.x == -INFINITY ? (a.y == 0.0f ? 0.0f : 1.0f) : exp2_fast(a.x - best);   // (scores that are all NaN leave no maximum)
        const float f1 = b.x == -INFINITY ? (b.y == 0.0f ? 0.0f : 1.0f) : exp2_fast(b.x - best), sum = a.y * f0 + b.y * f1, inv = sum != 0.0f ? 1.0f / sum : 0.0f;
        if (r < rows && !complete && (!alone || st == 0)) p.stats[row + r] = make_float2(best, sum);
        const int k0 = alone ? st * (HD / 64) : 0, k1 = alone ? k0 + HD / 64 : HD / 32, o0 = alone ? 0 : st * 128;
#pragma unroll 1
        for (int k = k0; k < k1; ++k) {
          float v[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = 0.0f;
          if (mine > 0 || alone) {
            uint32_t x[32], y[32];
            tmem_ld32(t_o + o0 + k * 32, x);
            if (second) tmem_ld32(t_o + 128 + k * 32, y);
            tmem_ld_wait();
            uint32_t bad = 0;
            if (nans) bad = alone ? sh.nan_row[0][r_in][k] | (second ? sh.nan_row[1][r_in][k] : 0u) : sh.nan_row[st][r_in][k];
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              v[j] = __uint_as_float(x[j]) * f0;
              if (second) v[j] = fmaf(__uint_as_float(y[j]), f1, v[j]);
              if (bad >> j & 1u) v[j] = __int_as_float(0x7FFFFFFF);
            }
          }
          store(k, v, inv);
        }
      }
      tc_fence_before();
      sync();   // (queries, statistics and sums may be written again)
      tc_fence_after();
      tile0 += s.i1;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == ISSUE) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// ---------------------------------------------------------------------------------------------------------------- joining
// Eight rows of a unit that is cut a block: lane = row + 8 * (dims / 4 % 4), every kJoinWarps-th of the parts a warp.  96 registers of a thread for 128 dims, 72 for 64.  (Two
// parts' loads at a time: a call of 64 units 61.2 us against 58.7, one of 8 units of 19 parts each the same; with 2 warps the latter takes 105 instead of 98, with 8 the former 68.)
constexpr int kJoinWarps = 4;
template <int HD>
__global__ void __launch_bounds__(kJoinWarps * 32) shared_join_kernel(const __grid_constant__ SharedParams p) {
  constexpr int D = HD / 16;
  __shared__ float4 of_warp[kJoinWarps - 1][D][32];
  __shared__ float2 stat_of_warp[kJoinWarps - 1][32];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, kv_heads = p.pool.n_kv_heads, all_rows = p.batch * p.rows;
  const int h = (int)(blockIdx.x % kv_heads), r0 = (int)(blockIdx.x / kv_heads) * 8, r = min(r0 + (lane & 7), all_rows - 1), d0 = lane >> 3;
  const int e = r0 / kTileRows, in = r - e * kTileRows;   // (the eight rows are of one unit)
  const int b0 = p.before[e], cost = p.before[e + 1] - b0;
  const long chunk = range_of(*p.all, p.ctas);
  float4 acc[D];
#pragma unroll
  for (int i = 0; i < D; ++i) acc[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float ref = -INFINITY, sum = 0.0f;
  auto add = [&](float2 s, const float4 (&x)[D]) {   // (scores that are all NaN leave no maximum, but a sum)
    const float now = fmaxf(ref, s.x), f = ref == -INFINITY ? (sum == 0.0f ? 0.0f : 1.0f) : exp2_fast(ref - now), g = s.x == -INFINITY ? (s.y == 0.0f ? 0.0f : 1.0f) : exp2_fast(s.x - now);
    ref = now;
    sum = sum * f + s.y * g;
#pragma unroll
    for (int i = 0; i < D; ++i) {
      acc[i].x = fmaf(x[i].x, g, acc[i].x * f), acc[i].y = fmaf(x[i].y, g, acc[i].y * f);
      acc[i].z = fmaf(x[i].z, g, acc[i].z * f), acc[i].w = fmaf(x[i].w, g, acc[i].w * f);
    }
  };
  int warps = 1;
  if (cost > 0) {
    const Entry en = p.entry[e];
    const long first = (long)b0 * kv_heads + (long)h * cost + kUnit;
    const int n = tiles_of(en), c0 = (int)(first / chunk), c1 = (int)((first + cost - kUnit - 1) / chunk), stride = padded(en.rows);
    if (tiles_before(en, first, c0 * chunk) == 0 && tiles_before(en, first, (c0 + 1) * chunk) == n) return;   // (written by its CTA)
    warps = min(kJoinWarps, c1 - c0 + 1);
    for (int c = c0 + warp; c <= c1; c += kJoinWarps) {
      const int i0 = tiles_before(en, first, c * chunk), i1 = tiles_before(en, first, (c + 1) * chunk);
      if (i0 == i1) continue;
      const long row = part_row(p, e, h, i0 == 0, c);
      const float4 *from = reinterpret_cast<const float4 *>(p.parts + row * HD) + in;
      const float2 s = p.stats[row + in];
      float4 x[D];
#pragma unroll
      for (int i = 0; i < D; ++i) x[i] = from[(d0 + 4 * i) * stride];
      add(s, x);
    }
  }
  if (warp > 0) {
    stat_of_warp[warp - 1][lane] = make_float2(ref, sum);
#pragma unroll
    for (int i = 0; i < D; ++i) of_warp[warp - 1][i][lane] = acc[i];
  }
  __syncthreads();
  if (warp > 0 || r0 + (lane & 7) >= all_rows) return;
  for (int w = 1; w < warps; ++w) {
    float4 x[D];
#pragma unroll
    for (int i = 0; i < D; ++i) x[i] = of_warp[w - 1][i][lane];
    add(stat_of_warp[w - 1][lane], x);
  }
  const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
  const int m = r / p.group;
  __nv_bfloat16 *out = p.out + (long)m * p.out_stride + ((long)h * p.group + r - m * p.group) * HD;
#pragma unroll
  for (int i = 0; i < D; ++i) {
    const uint2 v = inv == 0.0f ? make_uint2(0u, 0u) : make_uint2(bf16_pair(acc[i].x * inv, acc[i].y * inv), bf16_pair(acc[i].z * inv, acc[i].w * inv));
    *reinterpret_cast<uint2 *>(out + (d0 + 4 * i) * 4) = v;
  }
}

// ---------------------------------------------------------------------------------------------------------------- host
struct SharedLayout {
  int64_t entries, rows;          // units of a kv head; rows of parts
  size_t before, entry, segs, begin, stats, parts, bytes;
};
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
SharedLayout layout_of(const sjd_pool &pool, int64_t batch, int64_t window, int64_t n_heads) {
  SharedLayout l;
  const int64_t rows = batch * window * (n_heads / pool.n_kv_heads);
  l.entries = (rows + kTileRows - 1) / kTileRows;
  l.rows = (l.entries * pool.n_kv_heads + kMaxCtas) * kTileRows;
  l.before = 256;
  l.entry = l.before + up256((l.entries + 1) * sizeof(int));
  l.segs = l.entry + up256(l.entries * sizeof(Entry));
  l.begin = l.segs + up256((2 * batch + 2 * l.entries) * sizeof(Segment));
  l.stats = l.begin + up256(kMaxCtas * sizeof(Begin));
  l.parts = l.stats + up256(l.rows * sizeof(float2));
  l.bytes = l.parts + up256((size_t)l.rows * pool.head_dim * sizeof(float));
  const size_t alone = sjd_pool_attention_workspace_bytes(&pool, (int)window, (int)n_heads);   // (calls that are left to it)
  if (l.bytes < alone) l.bytes = alone;
  return l;
}

}  // namespace
}  // namespace sjd

using namespace sjd;

extern "C" size_t sjd_pool_attention_shared_workspace_bytes(const sjd_pool *pool, int batch, int window, int n_heads) {
  if (check_pool(pool, false) != SJD_OK || batch < 1 || batch > kMaxSeqs || window < 1 || n_heads < 1 || n_heads % pool->n_kv_heads != 0) return 0;
  if ((int64_t)batch * window * n_heads > 1ll << 30) return 0;
  return layout_of(*pool, batch, window, n_heads).bytes;
}

extern "C" int sjd_pool_attention_shared(const sjd_pool *pool, int layer, int batch, int window, int n_heads, int dtype, const void *q,
                                         int64_t q_stride, const int32_t *seqs, const int32_t *in_pos, int n_groups,
                                         const int32_t *group_begin, float scale, void *out, int64_t out_stride, void *ws, size_t ws_bytes,
                                         void *cuda_stream) {
  const int rc = check_pool(pool, false);
  if (rc != SJD_OK) return rc;
  if (dtype != SJD_BF16) return SJD_ERR_UNSUPPORTED;
  if (layer < 0 || layer >= pool->n_layers || batch < 1 || window < 1 || n_heads < 1 || !q || !in_pos || !out || !ws) return SJD_ERR_BAD_ARG;
  if (n_heads % pool->n_kv_heads != 0 || (group_begin && n_groups < 1) || !(scale >= 0.0f) || scale > 1e30f) return SJD_ERR_BAD_ARG;
  const int64_t row = (int64_t)n_heads * pool->head_dim;
  if (q_stride < row || out_stride < row || ((q_stride | out_stride) & 3)) return SJD_ERR_BAD_ARG;
  if ((((uintptr_t)q | (uintptr_t)out) & 7u) != 0 || ((uintptr_t)ws & 255u) != 0) return SJD_ERR_BAD_ARG;
  if ((((uintptr_t)seqs | (uintptr_t)in_pos | (uintptr_t)group_begin) & 3u) != 0) return SJD_ERR_BAD_ARG;
  if (batch > kMaxSeqs || (group_begin && n_groups > batch) || (int64_t)batch * window * n_heads > 1ll << 30) return SJD_ERR_CAPACITY;
  const SharedLayout l = layout_of(*pool, batch, window, n_heads);
  if (ws_bytes < l.bytes) return SJD_ERR_CAPACITY;
  // (places of a kv head are counted in 32 bits: a sequence's keys count in each of the units that it has rows in;
  const int64_t most = ((int64_t)pool->pages_per_seq + 1) / 2 + 1;
  // and those of a CTA)
  const int64_t line = kBoth * most * (2 * (int64_t)batch + 2 * l.entries) + kUnit * l.entries;
  if (line >= 1ll << 30 || line * pool->n_kv_heads / 64 >= 1ll << 30) return SJD_ERR_CAPACITY;
  int dev = 0, cc_major = 0, sms = 0;
  SJD_CUDA(cudaGetDevice(&dev));
  SJD_CUDA(cudaDeviceGetAttribute(&cc_major, cudaDevAttrComputeCapabilityMajor, dev));
  SJD_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  if (cc_major != 10) return SJD_ERR_UNSUPPORTED;
  if (pool_each_for_itself(batch, window, pool->n_kv_heads, (int64_t)window * (n_heads / pool->n_kv_heads), pool->pages_per_seq, batch == 1 || (group_begin && n_groups == batch), sms))
    return sjd_pool_attention(pool, layer, batch, window, n_heads, dtype, q, q_stride, seqs, in_pos, 0, 0, scale, out, out_stride, ws, ws_bytes, cuda_stream);
  const int hd = pool->head_dim;
  SharedParams p;
  memset(&p, 0, sizeof(p));
  p.pool = *pool;
  p.layer = layer, p.batch = batch, p.window = window, p.n_heads = n_heads, p.group = n_heads / pool->n_kv_heads;
  p.rows = window * p.group, p.n_entries = (int)l.entries, p.n_groups = n_groups;
  p.scale = (scale > 0.0f ? scale : 1.0f / sqrtf((float)hd)) * 1.4426950408889634f;
  p.q = (const __nv_bfloat16 *)q, p.q_stride = q_stride, p.out = (__nv_bfloat16 *)out, p.out_stride = out_stride;
  p.seqs = seqs, p.in_pos = in_pos, p.group_begin = group_begin;
  char *at = (char *)ws;
  p.all = (long *)at, p.before = (int *)(at + l.before), p.begin = (Begin *)(at + l.begin), p.entry = (Entry *)(at + l.entry), p.segs = (Segment *)(at + l.segs);
  p.stats = (float2 *)(at + l.stats), p.parts = (float *)(at + l.parts);
  p.ctas = sms < kMaxCtas ? sms : kMaxCtas;
  TensorMap tm;
  const int made = make_pool_map(&tm, *pool, layer);
  if (made != SJD_OK) return made;
  const CUtensorMap &map = reinterpret_cast<const CUtensorMap &>(tm);
  const size_t smem = 1024 + (4ull + kKStages + 2 + 4) * 128 * hd + (hd == 128 ? sizeof(SharedSmem<128>) : sizeof(SharedSmem<64>));
  auto tiles = hd == 128 ? shared_tiles_kernel<128> : shared_tiles_kernel<64>;
  auto join = hd == 128 ? shared_join_kernel<128> : shared_join_kernel<64>;
  const int r = allow_smem(tiles, smem);   // (the size follows from the kernel's type)
  if (r != SJD_OK) return r;
  auto launch = [&](auto kernel, unsigned blocks, int threads, size_t shared, const auto &...args) -> int {
    g_pdl = true;   // (each waits for the launch before it itself)
    const cudaError_t e = launch_kernel(kernel, dim3(blocks), dim3(threads), shared, (cudaStream_t)cuda_stream, args...);
    g_pdl = false;
    SJD_CUDA(e);
    SJD_CHECK_LAUNCH();
    return SJD_OK;
  };
  int s = launch(shared_plan_kernel, 1, kPlanThreads, 0, p);
  if (s == SJD_OK) s = launch(tiles, (unsigned)p.ctas, kThreads, smem, map, p);
  if (s == SJD_OK) s = launch(join, (unsigned)(((int64_t)batch * p.rows + 7) / 8 * pool->n_kv_heads), kJoinWarps * 32, 0, p);
  return s;
}
