// Attention over the 8-bit paged cache for sequences that share pages: the pages that all tables of a group begin with are attended once,
// with the rows of all its sequences, the rest of each sequence with its own rows, and the parts are joined.
//
// Queries are the rows of both products (128 of a stream), keys and dims the columns:
//   S [128 rows x 128 keys]  =  Q . K^T          O [128 rows x HD]  +=  P . V          (tcgen05, bf16, sums in 32 bits in tensor memory)
// A shared prefix meets many rows, so that the products and exponentials of a tile decide and its keys may be prepared once for all of them: eight
// warps turn e4m3 entries times 2^exponent into bf16, which holds them exactly (four bits and any exponent), as they lay them out for
// the tensor cores.  P goes to the second product through tensor memory, in the columns of the scores that it was.
// Two streams of four softmax warps, a row a thread: units of more than 128 rows give them 128 rows each of every tile of keys, others every
// other tile of keys with the same rows, so that one stream's softmax runs under the other's products either way.
// A weight is taken under a reference that follows the row's maximum only when that has grown by 2^8 (the sums in tensor memory
// then need no factor in nearly all tiles), and rounded to bf16, by up to 2^-8 of itself.
//
// Three launches: a plan (positions, what tables share, the line of units), the tiles, the joining of parts.  A unit is (group or sequence,
// up to 256 rows, kv head); the line of all units' tiles is cut into equal ranges, a CTA each.
#include "tcgen05.cuh"

namespace sjd {
namespace {

constexpr int kKeys = 128;              // of a tile
constexpr int kTileRows = 256;          // of a unit
constexpr int kUnit = 4;                // what a unit's begin and end take, in tiles of one stream
constexpr int kLeast = 2;               // pages that are worth a unit of their own
constexpr int kMaxCtas = 192;
constexpr int kMaxSeqs = SJD_POOL_MAX_LIST;
constexpr int kBefore = 2048;           // entries whose places are kept in shared memory
constexpr int kInfo = 4;                // tiles whose notes are kept
constexpr int kConv = 256, kSoft = 256, kThreads = kSoft + kConv + 32;
constexpr int kPlanThreads = 1024;
constexpr float kGrow = 8.0f;           // log2 of what a maximum may grow before its reference follows

struct Entry {   // (group or sequence, tile of rows)
  int b0, r0, rows;    // first sequence of its rows; row of the first one, counted from there; how many
  int seq;             // whose table (-1: none)
  int k0, k1;          // keys
  int row_base;        // rows of the parts of a kv head in the entries before
  int prefix;          // keys are before every row's position
};
struct Plan {          // in the workspace
  int n_entries, all, rows;   // places and rows of the parts of a kv head
};

struct SharedParams {
  sjd_pool pool;
  int layer, batch, window, n_heads, group, rows, row_tiles, n_groups;   // rows: window * group
  float scale;         // times log2(e)
  const __nv_bfloat16 *q;
  long q_stride, out_stride;
  const int32_t *seqs, *in_pos, *group_begin;
  __nv_bfloat16 *out;
  int by_eight;        // queries start on 16 bytes
  Plan *plan;
  int *before;         // [max entries + 1]: places of a kv head in the entries before
  Entry *entry;        // [max entries]
  int *group_of;       // [batch]
  int *prefix_of;      // [batch]: first entry of a group's shared keys, -1: none
  float2 *stats;       // (reference, sum) of a row's parts
  float *parts;        // [HD / 4][rows of the part][4]
  int max_entries, ctas;
};

__device__ __forceinline__ int padded(int rows) { return (rows + 7) & ~7; }
// places of a tile: both streams work on it, or one does
__device__ __forceinline__ int weight_of(int rows) { return rows > 128 ? 2 : 1; }

__device__ __forceinline__ int row_position(const SharedParams &p, int b, int k, bool tell) {
  int at = p.in_pos[(long)b * p.window + k];
  const int seq = p.seqs ? p.seqs[b] : b;
  if (at < -1 || at >= p.pool.pages_per_seq * KV_PAGE || seq < 0 || seq >= p.pool.n_seqs) {
    if (tell) pool_fault(p.pool.status, SJD_ERR_BAD_ARG);
    at = -1;
  }
  return at;
}

// ---------------------------------------------------------------------------------------------------------------- plan
__global__ void __launch_bounds__(kPlanThreads) shared_plan_kernel(const __grid_constant__ SharedParams p) {
  __shared__ int lo[kMaxSeqs], hi[kMaxSeqs], share[kMaxSeqs], leader[kMaxSeqs], first[kMaxSeqs + 1];   // by sequence, and by group
  __shared__ int bad, sums[2][32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = kPlanThreads / 32;
  pdl_wait();
  pdl_trigger();
  if (tid == 0) bad = 0;
  for (int b = tid; b < p.batch; b += kPlanThreads) lo[b] = 0x7FFFFFFF, hi[b] = -1;
  __syncthreads();
  // positions of every (sequence, tile of rows)
  const int own = p.batch * p.row_tiles;
  for (int e = warp; e < own; e += warps) {
    const int b = e / p.row_tiles, r0 = (e - b * p.row_tiles) * kTileRows, r1 = min(p.rows, r0 + kTileRows);
    int l = 0x7FFFFFFF, h = -1;
    for (int k = r0 / p.group + lane; k <= (r1 - 1) / p.group; k += 32) {
      const int at = row_position(p, b, k, true);
      if (at >= 0) l = min(l, at), h = max(h, at);
    }
    l = __reduce_min_sync(0xffffffffu, l);
    h = __reduce_max_sync(0xffffffffu, h);
    if (lane == 0) {
      if (h >= 0) atomicMin(&lo[b], l), atomicMax(&hi[b], h);
      Entry n;
      n.b0 = b, n.r0 = r0, n.rows = r1 - r0, n.seq = h < 0 ? -1 : p.seqs ? p.seqs[b] : b, n.k0 = 0, n.k1 = h + 1, n.row_base = 0, n.prefix = 0;
      p.entry[e] = n;
    }
  }
  // groups: ranges of sequences that follow one another
  const int groups = p.group_begin ? p.n_groups : 1;
  auto begin_of = [&](int g) { return p.group_begin ? p.group_begin[g] : g * p.batch; };
  for (int g = tid; g < groups; g += kPlanThreads) {
    const int b0 = begin_of(g), b1 = begin_of(g + 1);
    if (b0 < 0 || b1 < b0 || b1 > p.batch || (g == 0 && b0 != 0) || (g == groups - 1 && b1 != p.batch)) bad = 1;
  }
  __syncthreads();
  if (bad) {
    if (tid == 0) pool_fault(p.pool.status, SJD_ERR_BAD_ARG);
    for (int b = tid; b < p.batch; b += kPlanThreads) p.prefix_of[b] = -1;   // (every sequence for itself)
  } else {
    for (int g = tid; g < groups; g += kPlanThreads) {
      const int b0 = begin_of(g), b1 = begin_of(g + 1);
      int pages = 0x7FFFFFFF, lead = -1, live = 0;
      for (int b = b0; b < b1; ++b) {
        p.group_of[b] = g;
        if (hi[b] < 0) continue;
        pages = min(pages, (lo[b] + 1) / KV_PAGE);
        if (lead < 0) lead = b;
        ++live;
      }
      share[g] = live > 1 ? pages : 0;
      leader[g] = lead;
    }
    __syncthreads();
    // pages that the tables of a group begin with: up to the first that differs or is absent
    for (int b = warp; b < p.batch; b += warps) {
      const int g = p.group_of[b];
      if (hi[b] < 0) continue;
      const int sa = p.seqs ? p.seqs[leader[g]] : leader[g], sb = p.seqs ? p.seqs[b] : b;
      const int *ta = p.pool.table + (long)sa * p.pool.pages_per_seq, *tb = p.pool.table + (long)sb * p.pool.pages_per_seq;
      constexpr int U = 8;
      for (int at = 0; at < *(volatile int *)&share[g]; at += 32 * U) {
        int x[U], y[U], least = 0x7FFFFFFF;
#pragma unroll
        for (int j = 0; j < U; ++j) {
          const int i = at + 32 * j + lane;
          x[j] = i < share[g] ? ta[i] : -1;
          y[j] = i < share[g] ? tb[i] : -1;
        }
#pragma unroll
        for (int j = U - 1; j >= 0; --j)
          if (x[j] != y[j] || x[j] < 0 || x[j] >= p.pool.n_pages) least = at + 32 * j + lane;
        least = __reduce_min_sync(0xffffffffu, least);
        if (lane == 0) atomicMin(&share[g], least);
        if (least != 0x7FFFFFFF) break;
      }
    }
    __syncthreads();
    // entries of the groups' rows behind those of the sequences
    if (warp == 0) {
      int at = 0;
      for (int g0 = 0; g0 < groups; g0 += 32) {
        const int g = g0 + lane;
        int n = 0;
        if (g < groups) {
          if (share[g] < kLeast) share[g] = 0;
          if (share[g] > 0) n = (int)(((long)(begin_of(g + 1) - begin_of(g)) * p.rows + kTileRows - 1) / kTileRows);
        }
        int x = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += y;
        }
        if (g < groups) first[g] = at + x - n;
        at += __shfl_sync(0xffffffffu, x, 31);
      }
      if (lane == 0) first[groups] = at;
    }
    __syncthreads();
    for (int g = warp; g < groups; g += warps) {
      const int b0 = begin_of(g), all = (begin_of(g + 1) - b0) * p.rows;
      for (int i = lane; i < first[g + 1] - first[g]; i += 32) {
        Entry n;
        n.b0 = b0, n.r0 = i * kTileRows, n.rows = min(all - n.r0, kTileRows), n.seq = p.seqs ? p.seqs[leader[g]] : leader[g];
        n.k0 = 0, n.k1 = share[g] * KV_PAGE, n.row_base = 0, n.prefix = 1;
        p.entry[own + first[g] + i] = n;
      }
    }
    for (int b = tid; b < p.batch; b += kPlanThreads) {
      const int g = p.group_of[b];
      p.prefix_of[b] = share[g] > 0 ? own + first[g] : -1;
      p.group_of[b] = begin_of(g);   // (from here on: its first sequence)
      lo[b] = share[g] * KV_PAGE;    // (and: its first own key)
    }
  }
  __syncthreads();
  // places on the line and rows of the parts, sums over the entries before
  const int n = own + (bad ? 0 : first[groups]), run = (n + kPlanThreads - 1) / kPlanThreads, e0 = min(n, tid * run), e1 = min(n, e0 + run);
  int cost = 0, rows = 0;
  auto cost_of = [&](const Entry &en) { return en.seq < 0 || en.k1 <= en.k0 ? 0 : (en.k1 - en.k0 + kKeys - 1) / kKeys * weight_of(en.rows) + kUnit; };
  for (int e = e0; e < e1; ++e) {
    if (e < own && !bad) p.entry[e].k0 = lo[p.entry[e].b0];
    const Entry en = p.entry[e];
    const int c = cost_of(en);
    cost += c;
    rows += c > 0 ? padded(en.rows) : 0;
  }
  int x = cost, y = rows;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int a = __shfl_up_sync(0xffffffffu, x, o), c = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) x += a, y += c;
  }
  if (lane == 31) sums[0][warp] = x, sums[1][warp] = y;
  __syncthreads();
  for (int w = 0; w < warp; ++w) x += sums[0][w], y += sums[1][w];
  int at = x - cost, row = y - rows;
  for (int e = e0; e < e1; ++e) {
    const Entry en = p.entry[e];
    const int c = cost_of(en);
    p.before[e] = at;
    p.entry[e].row_base = row;
    at += c;
    row += c > 0 ? padded(en.rows) : 0;
  }
  if (tid == kPlanThreads - 1) {
    p.before[n] = x;
    p.plan->n_entries = n;
    p.plan->all = x;
    p.plan->rows = y;
  }
}

// ---------------------------------------------------------------------------------------------------------------- units
struct Unit {
  int e, h, n, w;      // entry, kv head, tiles, places of a tile
  long first;          // place of the first tile
};
// the unit that place t is in
template <typename Before>
__device__ __forceinline__ Unit unit_at(const SharedParams &p, const Before &before, int n_entries, long t) {
  int lo = 0, hi = n_entries - 1;
  const int heads = p.pool.n_kv_heads;
  while (lo < hi) {   // last entry that begins at t or before
    const int mid = (lo + hi + 1) >> 1;
    if ((long)before(mid) * heads <= t) lo = mid; else hi = mid - 1;
  }
  Unit u;
  u.e = lo;
  const int b = before(lo), cost = before(lo + 1) - b;
  const long in = t - (long)b * heads;
  u.h = (int)(in / cost);
  u.w = weight_of(p.entry[lo].rows);
  u.n = (cost - kUnit) / u.w;
  u.first = (long)b * heads + (long)u.h * cost + kUnit;
  return u;
}
// tiles of a unit that begin before place t
__device__ __forceinline__ int tiles_before(const Unit &u, long t) {
  const long n = t <= u.first ? 0 : (t - u.first + u.w - 1) / u.w;
  return n < u.n ? (int)n : u.n;
}
__device__ __forceinline__ long range_of(const Plan &plan, int kv_heads, int ctas) {
  const long all = (long)plan.all * kv_heads, least = 2 * kUnit;
  const long chunk = (all + ctas - 1) / ctas;
  return chunk < least ? least : chunk;
}
// first row of a part: of the unit's first tiles, or of those that CTA c finds begun
__device__ __forceinline__ long part_row(const SharedParams &p, const Plan &plan, const Entry &en, int h, bool begins, int c) {
  return begins ? (long)en.row_base * p.pool.n_kv_heads + (long)h * padded(en.rows) : (long)plan.rows * p.pool.n_kv_heads + (long)c * kTileRows;
}

// ---------------------------------------------------------------------------------------------------------------- tiles
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
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ bool has_nan(uint32_t bytes) { return (((bytes & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0; }
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Two e4m3 bytes, in the high bytes of the halves of t, as bf16: their bits moved into place are the numbers times 2^-120 (a
// subnormal one stays one), and up (and more, where that is not 1) bring them up by 2^120 and the exponent.  Exact.
__device__ __forceinline__ uint32_t bf16_of_e4m3(uint32_t t, uint32_t up, uint32_t more, bool twice) {
  const uint32_t bits = (t & 0x80008000u) | (t >> 4 & 0x07F007F0u);
  const uint32_t v = mul_bf16x2(bits, up);
  return twice ? mul_bf16x2(v, more) : v;
}
__device__ __forceinline__ uint32_t pair_of(float v) { return bf16_pair(v, v); }

template <int HD>
struct SharedSmem {
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_ready[2], o_full[2], q_ready;
  uint32_t tmem_base;
  int failed;
  int there[kInfo];                            // bit j: page j of the tile is there
  uint32_t nan_warps[kInfo][kConv / 32];       // some entry of V that a warp turned was NaN
  uint16_t nan_dims[kInfo][kKeys][HD / 16];    // which, if so
  float2 stat[2][128];                         // of both streams' rows
  uint32_t nan_row[2][128][HD / 32];
  int before[kBefore];
};

template <int HD>
__global__ void __launch_bounds__(kThreads, 1) shared_tiles_kernel(const __grid_constant__ SharedParams p) {
  constexpr int OP = 128 * HD * 2;          // bytes of an operand: [HD / 64][128 rows][128 bytes], 128-byte swizzle
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t *Qs = smem, *Ks = smem + 2 * OP, *Vs = smem + 4 * OP;
  SharedSmem<HD> &sh = *reinterpret_cast<SharedSmem<HD> *>(smem + 6 * OP);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, kv_heads = p.pool.n_kv_heads;
  constexpr int ISSUE = (kSoft + kConv) / 32;
  pdl_trigger();
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.k_full[i], kConv / 32);
      mbar_init(&sh.k_empty[i], 1);
      mbar_init(&sh.v_full[i], kConv / 32);
      mbar_init(&sh.v_empty[i], 1);
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.p_ready[i], 4);
      mbar_init(&sh.o_full[i], 1);
    }
    mbar_init(&sh.q_ready, kSoft / 32);
    sh.failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == ISSUE) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  const Plan plan = *p.plan;
  const int n_entries = plan.n_entries;
  const bool near = n_entries < kBefore;
  if (near)
    for (int i = tid; i <= n_entries; i += kThreads) sh.before[i] = p.before[i];
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;
  auto before = [&](int e) { return near ? sh.before[e] : p.before[e]; };
  const long all = (long)plan.all * kv_heads, chunk = range_of(plan, kv_heads, gridDim.x);
  const long t_begin = min(all, blockIdx.x * chunk), t_end = min(all, t_begin + chunk);
  auto fail = [&]() {
    if (lane == 0) {
      *(volatile int *)&sh.failed = 1;
      pool_fault(p.pool.status, SJD_ERR_DEVICE_TIMEOUT);
    }
  };
  // this CTA's next unit with tiles from place t on: tiles i0 .. i1 - 1 of it; false: no more
  struct Span {
    Unit u;
    Entry en;
    int i0, i1;
  };
  auto next_span = [&](long &t, Span &s) {
    while (t < t_end) {
      s.u = unit_at(p, before, n_entries, t);
      s.i0 = tiles_before(s.u, t_begin);
      s.i1 = tiles_before(s.u, t_end);
      t = s.u.first + (long)s.u.n * s.u.w;
      if (s.i1 > s.i0) {
        s.en = p.entry[s.u.e];
        return true;
      }
    }
    return false;
  };

  if (warp >= kSoft / 32 && warp < ISSUE) {
    // ------------------------------------------------------------------ keys and values: e4m3 to bf16
    constexpr int SEG = HD / 16, ROWS = kConv / SEG, N = kKeys / ROWS;   // lanes of a row, rows at a time, 16-byte loads of a thread
    const int ct = tid - kSoft, seg = ct % SEG, row0 = ct / SEG, cw = ct >> 5;
    const uint32_t at0 = (uint32_t)(seg >> 2) * (128 * 128) + row0 * 128, unit0 = (seg & 3) * 2;   // (ROWS is a multiple of 8: the swizzle is the same)
    const long plane = (long)KV_PAGE * HD, head_planes = 2l * kv_heads, page_planes = head_planes * p.pool.n_layers;
    struct Raw {
      uint4 k[N], v[N];
      int k_exp[2], v_exp[2], there, left;   // left: keys of the tile
    };
    long t = t_begin;
    Span s;
    bool more = next_span(t, s);
    int i = more ? s.i0 : 0;
    auto load = [&](Raw &r) {   // the next tile's bytes; false: none left
      if (!more) return false;
      const int key0 = s.en.k0 + i * kKeys;
      r.left = s.en.k1 - key0;
      r.there = 0;
      int page[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int at = key0 / KV_PAGE + j;
        page[j] = j * KV_PAGE < r.left && at < p.pool.pages_per_seq ? p.pool.table[(long)s.en.seq * p.pool.pages_per_seq + at] : -1;
        if (page[j] >= p.pool.n_pages) page[j] = -1;
        if (page[j] >= 0) r.there |= 1 << j;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        r.k_exp[j] = r.v_exp[j] = 0;
        if (page[j] < 0) continue;
        const long at = (long)page[j] * page_planes + head_planes * p.layer + s.u.h;
        r.k_exp[j] = *reinterpret_cast<const int *>(p.pool.exps + at * kPoolBlocks);
        r.v_exp[j] = *reinterpret_cast<const int *>(p.pool.exps + (at + kv_heads) * kPoolBlocks);
        const uint8_t *base = (const uint8_t *)p.pool.pages + at * plane + seg * 16;
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const int row = row0 + n * ROWS;
          if (row >> 6 != j) continue;
          r.k[n] = *reinterpret_cast<const uint4 *>(base + (row & 63) * HD);
          r.v[n] = *reinterpret_cast<const uint4 *>(base + (row & 63) * HD + plane * kv_heads);
        }
      }
      if (++i == s.i1) {
        more = next_span(t, s);
        i = s.i0;
      }
      return true;
    };
    uint32_t made = 0;
    bool ok = true;
    // one operand of a tile; nan: told of NaN entries, which become zeros (null: they become NaN)
    auto turn = [&](const Raw &r, const uint4 (&x)[N], const int (&exps)[2], uint8_t *to, uint32_t *dims) {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int row = row0 + n * ROWS, j = row >> 6;
        uint32_t out[8];
        if (row < r.left && (r.there >> j & 1)) {
          const int e = pool_exp((int8_t)(exps[j] >> (8 * (row >> 4 & 3))));
          const uint32_t up = pair_of(two_to(min(e, 0) + 120)), over = pair_of(two_to(max(e, 0)));
          const uint32_t w[4] = {x[n].x, x[n].y, x[n].z, x[n].w};
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            out[2 * c] = bf16_of_e4m3(__byte_perm(w[c], 0, 0x1404), up, over, e > 0);
            out[2 * c + 1] = bf16_of_e4m3(__byte_perm(w[c], 0, 0x3424), up, over, e > 0);
          }
          if (__builtin_expect(has_nan(w[0]) || has_nan(w[1]) || has_nan(w[2]) || has_nan(w[3]), 0)) {
#pragma unroll
            for (int c = 0; c < 16; ++c) {
              if ((w[c >> 2] >> (8 * (c & 3)) & 0x7Fu) != 0x7Fu) continue;
              const uint32_t half = 0xFFFFu << (16 * (c & 1));
              out[c >> 1] = dims ? out[c >> 1] & ~half : out[c >> 1] | half;
              if (dims) dims[n] |= 1u << c;
            }
          }
        } else {
#pragma unroll
          for (int c = 0; c < 8; ++c) out[c] = 0;
        }
        uint8_t *dst = to + at0 + n * ROWS * 128;
        *reinterpret_cast<uint4 *>(dst + ((unit0 ^ (row & 7)) << 4)) = make_uint4(out[0], out[1], out[2], out[3]);
        *reinterpret_cast<uint4 *>(dst + (((unit0 + 1) ^ (row & 7)) << 4)) = make_uint4(out[4], out[5], out[6], out[7]);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
    };
    auto make = [&](const Raw &r) {
      const int stage = made & 1, slot = made % kInfo;
      const uint32_t ph = (made >> 1 & 1) ^ 1u;
      ok = ok && !*(volatile int *)&sh.failed && (made < 2 || warp_wait(&sh.k_empty[stage], ph));
      if (!ok) return;
      if (ct == 0) sh.there[slot] = r.there;
      turn(r, r.k, r.k_exp, Ks + stage * OP, nullptr);
      if (lane == 0) arrive(&sh.k_full[stage]);
      ok = made < 2 || warp_wait(&sh.v_empty[stage], ph);
      if (!ok) return;
      uint32_t dims[N];
#pragma unroll
      for (int n = 0; n < N; ++n) dims[n] = 0;
      turn(r, r.v, r.v_exp, Vs + stage * OP, dims);
      uint32_t any = 0;
#pragma unroll
      for (int n = 0; n < N; ++n) any |= dims[n];
      any = __any_sync(0xffffffffu, any != 0);
      if (__builtin_expect(any, 0)) {
#pragma unroll
        for (int n = 0; n < N; ++n) sh.nan_dims[slot][row0 + n * ROWS][seg] = (uint16_t)dims[n];
      }
      if (lane == 0) sh.nan_warps[slot][cw] = any;
      __syncwarp();
      if (lane == 0) arrive(&sh.v_full[stage]);
      ++made;
    };
    // two tiles' bytes in registers: one is turned while the other is on its way
    Raw a, b;
    bool have_a = load(a), have_b = false;
    while (have_a && ok) {
      have_b = load(b);
      make(a);
      if (!have_b || !ok) break;
      have_a = load(a);
      make(b);
    }
    if (!ok) fail();
  } else if (warp == ISSUE) {
    // ------------------------------------------------------------------ products
    constexpr uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | (uint32_t)(kKeys >> 3) << 17 | (uint32_t)(128 >> 4) << 24;
    constexpr uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | 1u << 16 | (uint32_t)(HD >> 3) << 17 | (uint32_t)(128 >> 4) << 24;   // V: dims follow one another
    const uint64_t desc = umma_desc_sw128(0);
    const uint64_t desc_v = (uint64_t)(128 * 128 >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
    const uint32_t q_at = smem_u32(Qs), k_at = smem_u32(Ks), v_at = smem_u32(Vs);
    long t = t_begin;
    Span s;
    bool ok = true;
    uint32_t q_ph = 0, p_ph[2] = {0, 0}, tile0 = 0;   // tile0: tiles of the units before
    while (ok && next_span(t, s)) {
      const int n = s.i1 - s.i0, both = s.u.w == 2, jobs = both ? 2 * n : n;
      ok = warp_wait(&sh.q_ready, q_ph);
      q_ph ^= 1u;
      auto scores = [&](int j) {
        const int st = j & 1, tile = both ? j >> 1 : j;
        const uint32_t use = tile0 + tile, stage = use & 1;
        ok = ok && !*(volatile int *)&sh.failed && warp_wait(&sh.k_full[stage], use >> 1 & 1);
        if (!ok) return;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t a = desc | (uint64_t)((q_at + (both ? st * OP : 0)) >> 4), b = desc | (uint64_t)((k_at + stage * OP) >> 4);
#pragma unroll
          for (int k = 0; k < HD / 16; ++k) umma_bf16(tmem + st * 128, a + (k >> 2) * (128 * 128 >> 4) + (k & 3) * 2, b + (k >> 2) * (128 * 128 >> 4) + (k & 3) * 2, idesc_s, k > 0);
          umma_commit(&sh.s_full[st]);
          if (!both || st == 1) umma_commit(&sh.k_empty[stage]);
        }
        __syncwarp();
      };
      scores(0);
      if (jobs > 1) scores(1);
      for (int j = 0; j < jobs && ok; ++j) {
        const int st = j & 1, tile = both ? j >> 1 : j;
        const uint32_t use = tile0 + tile, stage = use & 1;
        ok = !*(volatile int *)&sh.failed && warp_wait_both(&sh.p_ready[st], p_ph[st], &sh.v_full[stage], use >> 1 & 1);
        p_ph[st] ^= 1u;
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t b = desc_v | (uint64_t)((v_at + stage * OP) >> 4);
#pragma unroll
          for (int k = 0; k < kKeys / 16; ++k) umma_bf16_ts(tmem + 256 + st * 128, tmem + st * 128 + k * 8, b + k * (16 * 128 >> 4), idesc_o, j >= 2 || k > 0);
          if (!both || st == 1) umma_commit(&sh.v_empty[stage]);
          if (j + 2 >= jobs) umma_commit(&sh.o_full[st]);
        }
        __syncwarp();
        if (j + 2 < jobs) scores(j + 2);
      }
      tile0 += n;
    }
    if (!ok) fail();
  } else {
    // ------------------------------------------------------------------ softmax warps: a row a thread
    const int st = warp >> 2, quarter = warp & 3, r_in = quarter * 32 + lane;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16, t_s = tmem + lanes + st * 128, t_o = tmem + lanes + 256;
    auto sync = [&]() { asm volatile("bar.sync 1, %0;" ::"n"(kSoft) : "memory"); };
    long t = t_begin;
    Span s;
    bool ok = true;
    uint32_t s_ph = 0, o_ph = 0, tile0 = 0;
    while (next_span(t, s)) {
      const int n = s.i1 - s.i0, both = s.u.w == 2, mine = both ? n : (n + 1 - st) / 2, rows = s.en.rows;
      // ---- queries of the unit's rows
      {
        const int per_lane = p.by_eight ? 8 : 4, row_lanes = HD / per_lane, each = 32 / row_lanes;   // rows of a warp's load
        const int sub = lane / row_lanes, dim = lane % row_lanes * per_lane;
        const int count = both ? 256 : 128;
        auto source = [&](int r) {
          const int x = s.en.r0 + r, m = x / p.group;
          return p.q + ((long)s.en.b0 * p.window + m) * p.q_stride + ((long)s.u.h * p.group + (x - m * p.group)) * HD + dim;
        };
        auto place = [&](int r) {
          return Qs + (r >> 7) * OP + (dim >> 6) * (128 * 128) + (r & 127) * 128 + ((((dim & 63) >> 3) ^ (r & 7)) << 4) + (dim & 7) * 2;
        };
        constexpr int U = 8;
        for (int r0 = warp * each; r0 < min(count, rows); r0 += kSoft / 32 * each * U) {
          uint4 v[U];
#pragma unroll
          for (int j = 0; j < U; ++j) {
            const int r = r0 + j * (kSoft / 32) * each + sub;
            v[j] = make_uint4(0, 0, 0, 0);
            if (r >= rows) continue;
            if (p.by_eight) {
              v[j] = *reinterpret_cast<const uint4 *>(source(r));
            } else {
              const uint2 x = *reinterpret_cast<const uint2 *>(source(r));
              v[j].x = x.x, v[j].y = x.y;
            }
          }
#pragma unroll
          for (int j = 0; j < U; ++j) {
            const int r = r0 + j * (kSoft / 32) * each + sub;
            if (r >= rows) continue;
            if (p.by_eight) *reinterpret_cast<uint4 *>(place(r)) = v[j];
            else *reinterpret_cast<uint2 *>(place(r)) = make_uint2(v[j].x, v[j].y);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) arrive(&sh.q_ready);
      }
      const int r = r_in + (both ? st * 128 : 0);
      const bool warp_live = quarter * 32 + (both ? st * 128 : 0) < rows;
      int limit = 0x3FFFFFFF;   // the last key that this thread's row sees (no row: any)
      if (r < rows) {
        const int m = (s.en.r0 + r) / p.group, b = s.en.b0 + m / p.window;
        const int at = row_position(p, b, m % p.window, false);
        limit = at < 0 ? -1 : s.en.prefix ? s.en.k1 - 1 : min(at, s.en.k1 - 1);
      }
      const int least = __reduce_min_sync(0xffffffffu, limit);
      float m_ref = -INFINITY, l = 0.0f;
      uint32_t nan[HD / 32];
#pragma unroll
      for (int j = 0; j < HD / 32; ++j) nan[j] = 0;
      auto note_nans = [&](int tile) {   // entries of V that are NaN, of a tile whose second product is done
        const uint32_t slot = (tile0 + tile) % kInfo;
        uint32_t any = 0;
#pragma unroll
        for (int w = 0; w < kConv / 32; ++w) any |= sh.nan_warps[slot][w];
        if (__builtin_expect(any, 0)) {
          constexpr int ROWS = kConv / (HD / 16), WARP = 32 / (HD / 16);
          const int key0 = s.en.k0 + (s.i0 + tile) * kKeys;
#pragma unroll 1
          for (int k = 0; k < kKeys; ++k) {
            if (!sh.nan_warps[slot][k % ROWS / WARP] || key0 + k > limit) continue;
#pragma unroll
            for (int j = 0; j < HD / 32; ++j) nan[j] |= *reinterpret_cast<const uint32_t *>(&sh.nan_dims[slot][k][2 * j]);
          }
        }
      };
      for (int j = 0; j < mine; ++j) {
        const int tile = both ? j : 2 * j + st, key0 = s.en.k0 + (s.i0 + tile) * kKeys;
        ok = ok && !*(volatile int *)&sh.failed;
        if (ok && !warp_wait(&sh.s_full[st], s_ph)) {
          ok = false;
          fail();
        }
        s_ph ^= 1u;
        if (!warp_live) {   // (what its rows of P hold does not matter)
          __syncwarp();
          if (lane == 0) arrive(&sh.p_ready[st]);
          continue;
        }
        tc_fence_after();
        if (j > 0) note_nans(both ? tile - 1 : tile - 2);
        const int there = sh.there[(tile0 + tile) % kInfo];
        const bool whole = key0 + kKeys - 1 <= least && there == 3;
        // which of 32 keys this row sees
        auto seen = [&](int c) {
          const int n_seen = limit - (key0 + c * 32) + 1;
          const uint32_t bits = n_seen >= 32 ? 0xFFFFFFFFu : n_seen <= 0 ? 0u : (1u << n_seen) - 1;
          return there >> (c >> 1) & 1 ? bits : 0u;
        };
        float top = -INFINITY;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t v[32];
          tmem_ld32(t_s + c * 32, v);
          tmem_ld_wait();
          if (!whole) {
            const uint32_t bits = seen(c);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = bits >> i & 1u ? v[i] : 0xFF800000u;
          }
          float a[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < 32; ++i) a[i & 3] = fmaxf(a[i & 3], __uint_as_float(v[i]));
          top = fmaxf(top, fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])));
        }
        if (!whole && there != 3 && r < rows) {   // (no page where the row sees a key)
          const int miss = there & 1 ? key0 + KV_PAGE : key0;
          if (limit >= miss) pool_fault(p.pool.status, SJD_ERR_BAD_ARG);
        }
        top *= p.scale;
        if (j == 0) {
          m_ref = top;
        } else if (__any_sync(0xffffffffu, top > m_ref + kGrow)) {
          const float now = fmaxf(m_ref, top), f = now == -INFINITY ? 1.0f : exp2_fast(m_ref - now);
          m_ref = now;
          l *= f;
#pragma unroll 1
          for (int c = 0; c < HD / 32; ++c) {
            uint32_t v[32];
            tmem_ld32(t_o + st * 128 + c * 32, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
            tmem_st16(t_o + st * 128 + c * 32, v);
            tmem_st16(t_o + st * 128 + c * 32 + 16, v + 16);
          }
          tmem_st_wait();
        }
        const float ref = m_ref == -INFINITY ? 0.0f : m_ref;
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t v[32], w[16];
          tmem_ld32(t_s + c * 32, v);
          tmem_ld_wait();
          if (!whole) {
            const uint32_t bits = seen(c);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = bits >> i & 1u ? v[i] : 0xFF800000u;
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float x = exp2_fast(fmaf(__uint_as_float(v[2 * i]), p.scale, -ref)), y = exp2_fast(fmaf(__uint_as_float(v[2 * i + 1]), p.scale, -ref));
            sum[i & 3] += x + y;
            w[i] = bf16_pair(x, y);
          }
          tmem_st16(t_s + c * 16, w);   // (over scores that have been read)
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive(&sh.p_ready[st]);
      }
      // ---- this unit's part: references, sums and O
      if (mine > 0) {
        if (ok && !warp_wait(&sh.o_full[st], o_ph)) {
          ok = false;
          fail();
        }
        o_ph ^= 1u;
        tc_fence_after();
        if (warp_live) note_nans(both ? mine - 1 : 2 * (mine - 1) + st);
      }
      const long row = part_row(p, plan, s.en, s.u.h, s.i0 == 0, blockIdx.x);
      const int stride = padded(rows);
      float4 *parts = reinterpret_cast<float4 *>(p.parts + row * HD) + r;   // [HD / 4][padded rows]
      if (both) {
        if (warp_live) {
#pragma unroll 1
          for (int c = 0; c < HD / 32; ++c) {
            uint32_t v[32];
            tmem_ld32(t_o + st * 128 + c * 32, v);
            tmem_ld_wait();
            uint32_t bad = nan[0];
#pragma unroll
            for (int j = 1; j < HD / 32; ++j) bad = c == j ? nan[j] : bad;
            if (__builtin_expect(bad != 0, 0)) {
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = bad >> i & 1u ? 0x7FFFFFFFu : v[i];
            }
            if (r < rows) {
#pragma unroll
              for (int i = 0; i < 8; ++i)
                parts[(c * 8 + i) * stride] = make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
            }
          }
          if (r < rows) p.stats[row + r] = make_float2(m_ref, l);
        }
      } else {
        // both streams have sums of the same rows: each joins half of the dims
        sh.stat[st][r_in] = make_float2(m_ref, l);
#pragma unroll
        for (int j = 0; j < HD / 32; ++j) sh.nan_row[st][r_in][j] = nan[j];
        sync();
        if (warp_live) {
          const float2 a = sh.stat[0][r_in], b = n > 1 ? sh.stat[1][r_in] : make_float2(-INFINITY, 0.0f);
          const float best = fmaxf(a.x, b.x), f0 = a.x == -INFINITY ? 0.0f : exp2_fast(a.x - best), f1 = b.x == -INFINITY ? 0.0f : exp2_fast(b.x - best);
#pragma unroll 1
          for (int c = st * (HD / 64); c < (st + 1) * (HD / 64); ++c) {
            uint32_t v[32], w[32];
            tmem_ld32(t_o + c * 32, v);
            if (n > 1) tmem_ld32(t_o + 128 + c * 32, w);
            tmem_ld_wait();
            const uint32_t bad = sh.nan_row[0][r_in][c] | (n > 1 ? sh.nan_row[1][r_in][c] : 0u);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              float x = __uint_as_float(v[i]) * f0;
              if (n > 1) x = fmaf(__uint_as_float(w[i]), f1, x);
              v[i] = bad >> i & 1u ? 0x7FFFFFFFu : __float_as_uint(x);
            }
            if (r < rows) {
#pragma unroll
              for (int i = 0; i < 8; ++i)
                parts[(c * 8 + i) * stride] = make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
            }
          }
          if (st == 0 && r < rows) p.stats[row + r] = make_float2(best, a.y * f0 + b.y * f1);
        }
      }
      tc_fence_before();
      sync();   // (queries, statistics and sums may be written again)
      tc_fence_after();
      tile0 += n;
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
// Eight rows of a sequence and kv head a warp: lane = row + 8 * (dims / 4 % 4).  Parts in the order of their keys.
constexpr int kJoinWarps = 4;
template <int HD>
__global__ void __launch_bounds__(kJoinWarps * 32) shared_join_kernel(const __grid_constant__ SharedParams p) {
  constexpr int D = HD / 16;
  pdl_wait();
  pdl_trigger();
  const Plan plan = *p.plan;
  const int lane = threadIdx.x & 31, kv_heads = p.pool.n_kv_heads, eights = (p.rows + 7) / 8;
  const long job = (long)blockIdx.x * kJoinWarps + (threadIdx.x >> 5);
  if (job >= (long)p.batch * eights * kv_heads) return;
  const int h = (int)(job % kv_heads), b = (int)(job / kv_heads / eights), r = (int)(job / kv_heads % eights) * 8 + (lane & 7), d0 = lane >> 3;
  if (r >= p.rows) return;
  const int k = r / p.group;
  const bool live = row_position(p, b, k, false) >= 0;
  const long chunk = range_of(plan, kv_heads, p.ctas);
  float4 acc[D];
#pragma unroll
  for (int i = 0; i < D; ++i) acc[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float ref = -INFINITY, sum = 0.0f;
  auto add_unit = [&](int e, int in) {   // the parts of row `in` of an entry's rows
    const int cost = p.before[e + 1] - p.before[e];
    if (cost == 0) return;
    const Entry en = p.entry[e];
    Unit u;
    u.e = e, u.h = h, u.w = weight_of(en.rows), u.n = (cost - kUnit) / u.w, u.first = (long)p.before[e] * kv_heads + (long)h * cost + kUnit;
    const int c1 = (int)((u.first + (long)(u.n - 1) * u.w) / chunk);
    for (int c = (int)(u.first / chunk); c <= c1; ++c) {
      const int i0 = tiles_before(u, c * chunk), i1 = tiles_before(u, (c + 1) * chunk);
      if (i0 == i1) continue;
      const long row = part_row(p, plan, en, h, i0 == 0, c);
      const float2 s = p.stats[row + in];
      const float4 *from = reinterpret_cast<const float4 *>(p.parts + row * HD) + in;
      float4 x[D];
#pragma unroll
      for (int i = 0; i < D; ++i) x[i] = from[(d0 + 4 * i) * padded(en.rows)];
      const float now = fmaxf(ref, s.x), f = ref == -INFINITY ? 0.0f : exp2_fast(ref - now), g = s.x == -INFINITY ? 0.0f : exp2_fast(s.x - now);
      ref = now;
      sum = sum * f + s.y * g;
#pragma unroll
      for (int i = 0; i < D; ++i) {
        acc[i].x = fmaf(x[i].x, g, acc[i].x * f), acc[i].y = fmaf(x[i].y, g, acc[i].y * f);
        acc[i].z = fmaf(x[i].z, g, acc[i].z * f), acc[i].w = fmaf(x[i].w, g, acc[i].w * f);
      }
    }
  };
  if (live) {
    const int e = p.prefix_of[b];
    if (e >= 0) {
      const int in = (b - p.group_of[b]) * p.rows + r;
      add_unit(e + in / kTileRows, in % kTileRows);
    }
    add_unit(b * p.row_tiles + r / kTileRows, r % kTileRows);
  }
  const float inv = live && sum != 0.0f ? 1.0f / sum : 0.0f;
  __nv_bfloat16 *out = p.out + ((long)b * p.window + k) * p.out_stride + ((long)h * p.group + r - k * p.group) * HD;
#pragma unroll
  for (int i = 0; i < D; ++i) {
    const uint2 v = inv == 0.0f ? make_uint2(0u, 0u) : make_uint2(bf16_pair(acc[i].x * inv, acc[i].y * inv), bf16_pair(acc[i].z * inv, acc[i].w * inv));
    *reinterpret_cast<uint2 *>(out + (d0 + 4 * i) * 4) = v;
  }
}

// ---------------------------------------------------------------------------------------------------------------- host
struct SharedLayout {
  int64_t entries, rows;          // most entries; most rows of parts
  size_t before, entry, group_of, prefix_of, stats, parts, bytes;
};
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
SharedLayout layout_of(const sjd_pool &pool, int64_t batch, int64_t window, int64_t n_heads) {
  SharedLayout l;
  const int64_t rows = window * (n_heads / pool.n_kv_heads), own = batch * ((rows + kTileRows - 1) / kTileRows);
  l.entries = own + (batch * rows + kTileRows - 1) / kTileRows + batch;
  l.rows = pool.n_kv_heads * (2 * batch * rows + 8 * l.entries) + (int64_t)kMaxCtas * kTileRows;
  l.before = 256;
  l.entry = l.before + up256((l.entries + 1) * sizeof(int));
  l.group_of = l.entry + up256(l.entries * sizeof(Entry));
  l.prefix_of = l.group_of + up256(batch * sizeof(int));
  l.stats = l.prefix_of + up256(batch * sizeof(int));
  l.parts = l.stats + up256(l.rows * sizeof(float2));
  l.bytes = l.parts + up256((size_t)l.rows * pool.head_dim * sizeof(float));
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
  // (places of a kv head are counted in 32 bits)
  if (l.entries * (((int64_t)pool->pages_per_seq + 1) + kUnit) >= 1ll << 31) return SJD_ERR_CAPACITY;
  int dev = 0, cc_major = 0, sms = 0;
  SJD_CUDA(cudaGetDevice(&dev));
  SJD_CUDA(cudaDeviceGetAttribute(&cc_major, cudaDevAttrComputeCapabilityMajor, dev));
  SJD_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  if (cc_major != 10) return SJD_ERR_UNSUPPORTED;
  const int hd = pool->head_dim;
  SharedParams p;
  memset(&p, 0, sizeof(p));
  p.pool = *pool;
  p.layer = layer, p.batch = batch, p.window = window, p.n_heads = n_heads, p.group = n_heads / pool->n_kv_heads;
  p.rows = window * p.group, p.row_tiles = (p.rows + kTileRows - 1) / kTileRows, p.n_groups = n_groups;
  p.scale = (scale > 0.0f ? scale : 1.0f / sqrtf((float)hd)) * 1.4426950408889634f;
  p.q = (const __nv_bfloat16 *)q, p.q_stride = q_stride, p.out = (__nv_bfloat16 *)out, p.out_stride = out_stride;
  p.by_eight = ((uintptr_t)q & 15u) == 0 && (q_stride & 7) == 0;
  p.seqs = seqs, p.in_pos = in_pos, p.group_begin = group_begin;
  char *at = (char *)ws;
  p.plan = (Plan *)at, p.before = (int *)(at + l.before), p.entry = (Entry *)(at + l.entry), p.group_of = (int *)(at + l.group_of);
  p.prefix_of = (int *)(at + l.prefix_of), p.stats = (float2 *)(at + l.stats), p.parts = (float *)(at + l.parts);
  p.max_entries = (int)l.entries;
  p.ctas = sms < kMaxCtas ? sms : kMaxCtas;
  const size_t smem = 1024 + 6ull * 128 * hd * 2 + (hd == 128 ? sizeof(SharedSmem<128>) : sizeof(SharedSmem<64>));
  auto tiles = hd == 128 ? shared_tiles_kernel<128> : shared_tiles_kernel<64>;
  auto join = hd == 128 ? shared_join_kernel<128> : shared_join_kernel<64>;
  const int r = allow_smem(tiles, smem);   // (the size follows from the kernel's type)
  if (r != SJD_OK) return r;
  auto launch = [&](auto kernel, unsigned blocks, int threads, size_t shared) -> int {
    g_pdl = true;   // (each waits for the launch before it itself)
    const cudaError_t e = launch_kernel(kernel, dim3(blocks), dim3(threads), shared, (cudaStream_t)cuda_stream, p);
    g_pdl = false;
    SJD_CUDA(e);
    SJD_CHECK_LAUNCH();
    return SJD_OK;
  };
  int s = launch(shared_plan_kernel, 1, kPlanThreads, 0);
  if (s == SJD_OK) s = launch(tiles, (unsigned)p.ctas, kThreads, smem);
  if (s == SJD_OK) s = launch(join, (unsigned)(((int64_t)batch * ((p.rows + 7) / 8) * pool->n_kv_heads + kJoinWarps - 1) / kJoinWarps), kJoinWarps * 32, 0);
  return s;
}
