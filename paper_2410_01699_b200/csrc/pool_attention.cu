// Attention of window queries over the 8-bit paged cache, with an optional sliding window and sinks.
//
// Keys and values stay in 8 bits up to the registers of the warp that multiplies them, where they become fp16 (which holds every e4m3
// number) for mma.sync m16n8k16.  bf16 queries are fp16 after a power of two that brings a row's largest entry to 2^7 .. 2^8 (what that
// leaves out is below 2^-32 of it), fp32 queries and their weights are two fp16 numbers, the second what the first leaves (2^-22).
// (mma.sync takes e4m3 as well, but on this device it then converts both operands for every product: 700 products a clock and SM where
// operands change, against 1016 with fp16.)
//
// Rows are (window row, query head of the kv head's group): all heads of a group share the keys that are read.
//   S [16 rows x 8 keys]   = Q K^T           a word of a key is what a thread holds of one step of 16 dims
//   O [16 rows x 8 dims]  += P V             values of 2 keys x 4 dims are paired by byte permutes
// The order of dims in the first product and of keys in the second is free as long as both operands use the same; it is chosen so that
// the 16-byte loads of both meet no bank twice (see key_of).
//
// Exponents: with s the score (in log2), e_K in its factor and e_V added to it, w = 2^(s + e_V - top) is the weight of a value's e4m3
// number, top the largest s + e_V of the row so far, so that weights and products stay near 1 whatever the exponents of the
// blocks; the sum of the softmax takes w 2^-e_V, which stays within 2^+-100 of the top as well.
//
// A CTA has eight warps that work and one that fetches.  A tile is 32 keys (TMA, K and V of one page half); RG warps share a tile's keys
// (16 rows each), 8 / RG tiles are in work at a time, each with its own running maximum, and are joined at the end of a unit through
// shared memory.  A unit is (sequence, tile of rows, kv head).  The tiles of all units are one line that is cut into as many equal
// ranges as there are SMs (one CTA each): sequences of any lengths keep all SMs busy to the end, and a long one is spread over
// many.  A unit that is cut is joined by the last of its CTAs to arrive (in the order of its ranges: results do not hang on who that is).
// Bound: bytes of K and V up to 32 rows (fp32: 16), the tensor cores' fp16 rate beyond.
#include "tcgen05.cuh"

namespace sjd {
namespace {

constexpr int kTile = 32;            // keys
constexpr int kWorkWarps = 8;
constexpr int kThreads = (kWorkWarps + 4) * 32;   // the working warps, and a warpgroup of which one warp fetches
constexpr int kMaxEntries = 1024;    // (sequence, tile of rows) pairs of a call whose tiles are cut into equal ranges
constexpr int kMaxSlots = 24;
constexpr int kMaxCtas = 160;
constexpr int kSmem = 232448;
// Weights are 2^kUp at the row's maximum so far, which is renewed when a score passes it by more than kSlack: fp16 holds what is
// between 2^15 and 2^-24, 2^-37 of the maximum's weight.
constexpr int kUp = 13;
constexpr float kSlack = 2.0f;

struct PoolAttnParams {
  sjd_pool pool;
  int layer, batch, window, n_heads, group, rows, row_tiles;   // rows: window * group
  int sliding, sinks;
  float scale;                  // times log2(e)
  const void *q;
  long q_stride, out_stride;
  const int32_t *seqs, *in_pos;
  void *out;
  int *tickets;                 // [kMaxCtas], zero between calls
  float *parts;                 // [2 kMaxCtas][16 RG rows][head_dim], then (top, sum) of each
  int n_entries, cut, slots;    // cut: ranges of tiles; else a CTA per unit
};

struct Entry {   // (sequence, tile of rows)
  int before;    // tiles of one kv head in the entries before
  int low;       // first tile of the sliding part
  int sink;      // tiles before it
};

__device__ __forceinline__ int key_of(int c) { return c ^ ((c & 1) << 2); }   // key of column c of 8

__device__ __forceinline__ void mma_f16(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// two e4m3 numbers of a word (exact: fp16 holds all of them)
__device__ __forceinline__ void halves_of_e4m3(uint32_t w, uint32_t &lo, uint32_t &hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
}
__device__ __forceinline__ uint32_t halves_of_floats(float a, float b) {   // a in the low half
  uint32_t h;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(b), "f"(a));
  return h;
}
__device__ __forceinline__ float2 floats_of_halves(uint32_t h) {
  float2 f;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.f32.f16 %0, lo;\n\tcvt.f32.f16 %1, hi;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(h));
  return f;
}
// a, b as fp16 planes: the number and, of two, what is left of it
template <int PL>
__device__ __forceinline__ void split_halves(float a, float b, uint32_t *planes) {
  planes[0] = halves_of_floats(a, b);
  if constexpr (PL == 2) {
    const float2 f = floats_of_halves(planes[0]);
    planes[1] = halves_of_floats(a - f.x, b - f.y);
  }
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void arrive(uint64_t *bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap *map, int row, int plane, int page, uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(map), "r"(0), "r"(row), "r"(plane), "r"(page), "r"(smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void work_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kWorkWarps * 32) : "memory"); }
__device__ __forceinline__ bool has_nan(uint32_t bytes) { return (((bytes & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0; }

template <typename T> __device__ __forceinline__ void load16(const T *p, float *x);   // 16 entries
template <> __device__ __forceinline__ void load16<float>(const float *p, float *x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = *reinterpret_cast<const float4 *>(p + 4 * i);
    x[4 * i] = v.x, x[4 * i + 1] = v.y, x[4 * i + 2] = v.z, x[4 * i + 3] = v.w;
  }
}
template <> __device__ __forceinline__ void load16<__nv_bfloat16>(const __nv_bfloat16 *p, float *x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint2 v = *reinterpret_cast<const uint2 *>(p + 4 * i);
    x[4 * i] = __uint_as_float(v.x << 16), x[4 * i + 1] = __uint_as_float(v.x & 0xFFFF0000u);
    x[4 * i + 2] = __uint_as_float(v.y << 16), x[4 * i + 3] = __uint_as_float(v.y & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void store4(float *p, float4 v) { *reinterpret_cast<float4 *>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float4 v) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}

template <int HD>
struct AttnShared {
  uint64_t full[kMaxSlots], empty[kMaxSlots];
  int key0[kMaxSlots];                 // first key of the tile in a slot, -1: it has no page
  int k_exp[kMaxSlots], v_exp[kMaxSlots];   // exponents of the page's four blocks
  float top[kWorkWarps][16], sum[kWorkWarps][16];
  float factor[kWorkWarps][16];
  int scan[32];
  int failed, last;
  Entry entry[kMaxEntries + 1];
};

// T: float or bf16 queries and outputs; RG: warps of 16 rows that share a tile
template <typename T, int HD, int RG>
__global__ void __launch_bounds__(kThreads, 1) pool_attention_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ PoolAttnParams p) {
  constexpr int PL = sizeof(T) == 4 ? 2 : 1;   // planes
  constexpr int KG = kWorkWarps / RG;          // tiles in work at a time
  constexpr int KS = HD / 16;                  // steps of the first product
  constexpr int NT = HD / 8;                   // column tiles of the second
  constexpr int BOX = kTile * HD;              // bytes of K or V of a tile
  constexpr int ROWS = 16 * RG;
  constexpr int CW = HD / 8;                   // bytes of a value row that a thread takes
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t *ring = smem;                                                            // [slots][K | V]
  float *join = reinterpret_cast<float *>(ring + p.slots * 2 * BOX);               // [8 warps][16][HD]
  AttnShared<HD> &sh = *reinterpret_cast<AttnShared<HD> *>(join + kWorkWarps * 16 * HD);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int kv_heads = p.pool.n_kv_heads, seq_keys = p.pool.pages_per_seq * KV_PAGE;

  if (tid < p.slots) {
    mbar_init(&sh.full[tid], 1);
    mbar_init(&sh.empty[tid], RG);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (tid == 0) sh.failed = 0;

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
  const int n_entries = p.cut ? p.n_entries : 1;
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
    const int span = min(p.window, (ROWS - 1) / p.group + 2);
    int lanes = 1;
    while (lanes < 32 && lanes < span) lanes <<= 1;
    const int per_pass = kThreads / lanes, mine = tid / lanes, l = tid % lanes;
    for (int e0 = 0; e0 < n_entries; e0 += per_pass) {
      const int e = e0 + mine;
      int lo = 0x7FFFFFFF, hi = -1;
      if (e < n_entries) {
        int b, rt;
        entry_at(e, &b, &rt);
        const int r1 = min(p.rows, (rt + 1) * ROWS);
        for (int k = rt * ROWS / p.group + l; k <= (r1 - 1) / p.group; k += lanes) {
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
      if (e < n_entries && l == 0) {
        Entry n;
        n.low = p.sliding > 0 && hi >= 0 ? max(0, lo - p.sliding + 1) / kTile : 0;
        n.sink = min(n.low, (min(p.sinks, seq_keys) + kTile - 1) / kTile);
        n.before = hi < 0 ? 0 : hi / kTile + 1 - n.low + n.sink;   // (its own tiles so far)
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
  __syncthreads();
  const long all = (long)sh.entry[n_entries].before * (p.cut ? kv_heads : 1);
  // a range has enough tiles for all warps of a CTA
  long chunk = all;
  if (p.cut) {
    chunk = (all + gridDim.x - 1) / gridDim.x;
    chunk = chunk < 2 * KG ? 2 * KG : chunk;
  }
  const long t_begin = p.cut ? blockIdx.x * chunk : 0, t_end = min(all, t_begin + chunk);

  // unit of a tile: its entry, kv head, first tile
  struct Unit {
    int e, kvh, n;      // n: its tiles
    long first;
  };
  auto unit_of = [&](long t) {
    Unit u;
    int lo = 0, hi = n_entries - 1;
    const int heads = p.cut ? kv_heads : 1;
    while (lo < hi) {   // last entry that begins at t or before
      const int mid = (lo + hi + 1) >> 1;
      if ((long)sh.entry[mid].before * heads <= t) lo = mid; else hi = mid - 1;
    }
    u.e = lo;
    u.n = sh.entry[lo + 1].before - sh.entry[lo].before;
    const long in = t - (long)sh.entry[lo].before * heads;
    const int h = (int)(in / u.n);
    u.kvh = p.cut ? h : unit0 % kv_heads;
    u.first = t - (in - (long)h * u.n);
    return u;
  };

  if (warp >= kWorkWarps) {
    // 384 x 168 registers at the launch: 128 x 40 + 256 x 232
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp > kWorkWarps) return;
    // ------------------------------------------------------------------ fetching: tiles in order into the ring
    int slot = 0;
    uint32_t phase = 1;
    long issued = 0;
    bool ok = true;
    int n_key0 = -1, n_page = -1, n_kexp = 0, n_vexp = 0, n_plane = 0;
    auto look_up = [&](long t) {   // what lane `lane` knows of tile t + lane
      n_key0 = n_page = -1;
      n_kexp = n_vexp = n_plane = 0;
      if (t + lane >= t_end) return;
      const Unit u = unit_of(t + lane);
      const int i = (int)(t + lane - u.first);
      const Entry en = sh.entry[u.e];
      int b, rt;
      entry_at(u.e, &b, &rt);
      n_key0 = (i < en.sink ? i : en.low + i - en.sink) * kTile;
      const int seq = p.seqs ? p.seqs[b] : b;
      n_page = p.pool.table[(long)seq * p.pool.pages_per_seq + n_key0 / KV_PAGE];
      if (n_page < 0 || n_page >= p.pool.n_pages) {
        pool_fault(p.pool.status, SJD_ERR_BAD_ARG);
        n_page = -1;
        return;
      }
      n_plane = u.kvh;
      const long at = ((long)n_page * p.pool.n_layers + p.layer) * 2 * kv_heads + u.kvh;
      n_kexp = *reinterpret_cast<const int *>(p.pool.exps + at * kPoolBlocks);
      n_vexp = *reinterpret_cast<const int *>(p.pool.exps + (at + kv_heads) * kPoolBlocks);
    };
    if (t_begin < t_end) look_up(t_begin);
    for (long t0 = t_begin; t0 < t_end && ok; t0 += 32) {
      const int key0 = n_key0, page = n_page, kexp = n_kexp, vexp = n_vexp, plane = n_plane;
      if (t0 + 32 < t_end) look_up(t0 + 32);
      const int n = (int)min(32L, t_end - t0);
      for (int i = 0; i < n; ++i) {
        const int key = __shfl_sync(0xffffffffu, key0, i), pg = __shfl_sync(0xffffffffu, page, i), pl = __shfl_sync(0xffffffffu, plane, i);
        const int ke = __shfl_sync(0xffffffffu, kexp, i), ve = __shfl_sync(0xffffffffu, vexp, i);
        if (issued >= p.slots && !warp_wait(&sh.empty[slot], phase)) { ok = false; break; }
        if (elect_one()) {
          sh.key0[slot] = pg < 0 ? -1 : key;
          sh.k_exp[slot] = ke;
          sh.v_exp[slot] = ve;
          const uint32_t dst = smem_u32(ring) + slot * 2 * BOX;
          if (pg < 0) {
            arrive(&sh.full[slot]);
          } else {
            mbar_expect_tx(&sh.full[slot], 2 * BOX);
            tma_box(dst, &map, key % KV_PAGE, pl, pg, &sh.full[slot]);
            tma_box(dst + BOX, &map, key % KV_PAGE, kv_heads + pl, pg, &sh.full[slot]);
          }
        }
        __syncwarp();
        ++issued;
        if (++slot == p.slots) { slot = 0; phase ^= 1u; }
      }
    }
    if (!ok && lane == 0) {
      *(volatile int *)&sh.failed = 1;
      pool_fault(p.pool.status, SJD_ERR_DEVICE_TIMEOUT);
    }
    // leave no copy in flight
    for (long j = issued > p.slots ? issued - p.slots : 0; j < issued; ++j) warp_wait(&sh.full[j % p.slots], (uint32_t)((j / p.slots) & 1));
    return;
  }

  // -------------------------------------------------------------------- working warps
  asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
  const int kg = warp / RG, rg = warp % RG;
  const int g = lane >> 2, t4 = lane & 3;
  const T *qp = (const T *)p.q;
  T *outp = (T *)p.out;
  long mine = t_begin + kg;   // this warp's next tile, its slot in the ring and the parity of the slot's round
  int slot = kg;
  uint32_t phase = 0;
  bool ok = true;
  // rows without a tile are in no range: the CTAs share them (an entry whose rows see nothing has no tiles)
  if (p.cut || all == 0) {
    for (int e = p.cut ? blockIdx.x : 0; e < n_entries; e += gridDim.x) {
      if (sh.entry[e + 1].before != sh.entry[e].before) continue;
      int b, rt;
      entry_at(e, &b, &rt);
      const int r1 = min(p.rows, (rt + 1) * ROWS);
      for (int i = tid; i < (r1 - rt * ROWS) * (HD / 4); i += kWorkWarps * 32) {
        const int r = rt * ROWS + i / (HD / 4), dim = i % (HD / 4) * 4;
        for (int h = p.cut ? 0 : unit0 % kv_heads; h < (p.cut ? kv_heads : unit0 % kv_heads + 1); ++h)
          store4(outp + ((long)b * p.window + r / p.group) * p.out_stride + ((long)h * p.group + r % p.group) * HD + dim, make_float4(0.0f, 0.0f, 0.0f, 0.0f));
      }
    }
  }

  for (long t = t_begin; t < t_end;) {
    const Unit u = unit_of(t);
    const long u_end = u.first + u.n, end = min(t_end, u_end);
    int b, rt;
    entry_at(u.e, &b, &rt);
    // ---- this thread's rows: g and g + 8 of its warp's 16
    int pos[2];
    float factor[2];
    uint32_t qa[PL][KS][4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = rt * ROWS + rg * 16 + g + 8 * j;
      const bool have = r < p.rows;
      pos[j] = -1;
      float x[HD / 4];
#pragma unroll
      for (int i = 0; i < HD / 4; ++i) x[i] = 0.0f;
      if (have) {
        const int k = r / p.group, h = u.kvh * p.group + r % p.group;
        pos[j] = position(b, k);
        const T *src = qp + ((long)b * p.window + k) * p.q_stride + (long)h * HD;
#pragma unroll
        for (int c = 0; c < HD / 64; ++c) load16<T>(src + 16 * (t4 + 4 * c), x + 16 * c);
      }
      float top = 0.0f;
#pragma unroll
      for (int i = 0; i < HD / 4; ++i) {
        if (fabsf(x[i]) == INFINITY) x[i] = __int_as_float(0x7FFFFFFF);   // (e4m3 has no infinity: its row is NaN, as it would be)
        top = fmaxf(top, fabsf(x[i]));
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // a power of two that brings the largest entry to 128 .. 256
      int e = top > 0.0f ? 7 - (int)((__float_as_uint(top) >> 23) - 127) : 0;
      e = min(e, 126);   // (entries below 2^-119 lose places)
      const float up = two_to(max(e, -126));
      factor[j] = p.scale * two_to(-max(e, -126));
#pragma unroll
      for (int i = 0; i < HD / 4; i += 2) {   // step i / 4 of the product: its words j (k = 2 t4, ..) and j + 2 (k = 2 t4 + 8, ..)
        uint32_t w[PL];
        split_halves<PL>(x[i] * up, x[i + 1] * up, w);
#pragma unroll
        for (int l = 0; l < PL; ++l) qa[l][i / 4][i % 4 + j] = w[l];
      }
    }
    int lo = min(pos[0] >= 0 ? pos[0] : 0x7FFFFFFF, pos[1] >= 0 ? pos[1] : 0x7FFFFFFF), hi = max(pos[0], pos[1]);
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    const int sliding = p.sliding > 0 ? p.sliding : 0x7FFFFFFF;
    // keys above `from` are in the window of every row, those up to `until` in none's
    const int from = hi - sliding, until = lo == 0x7FFFFFFF ? 0x7FFFFFFF : lo - sliding;

    float o[NT][4], run[2] = {-INFINITY, -INFINITY}, total[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;

    auto next = [&]() {
      mine += KG;
      slot += KG;
      if (slot >= p.slots) { slot -= p.slots; phase ^= 1u; }
    };
    for (; mine < end; next()) {
      ok = ok && !*(volatile int *)&sh.failed;
      if (ok && !warp_wait(&sh.full[slot], phase)) {
        ok = false;
        if (lane == 0) {
          *(volatile int *)&sh.failed = 1;
          pool_fault(p.pool.status, SJD_ERR_DEVICE_TIMEOUT);
        }
      }
      if (!ok) continue;
      const int key0 = sh.key0[slot];
      const bool seen = key0 >= 0 && key0 <= hi && (key0 + kTile - 1 > until || key0 < p.sinks);
      if (seen) {
        const bool whole = key0 + kTile - 1 <= lo && (key0 > from || key0 + kTile <= p.sinks);
        const uint8_t *ks = ring + slot * 2 * BOX, *vs = ks + BOX;
        const int half = key0 % KV_PAGE / kTile * 16;   // the tile's two blocks of the page's four
        const int kw = sh.k_exp[slot] >> half, vw = sh.v_exp[slot] >> half;
        // ---- scores
        float s[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.0f;
        {
          uint4 kb[4][HD / 64];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = i * 8 + key_of(g);
#pragma unroll
            for (int c = 0; c < HD / 64; ++c) {
              const int piece = HD == 128 ? (t4 + 4 * c) ^ (key & 7) : t4 ^ (key >> 1 & 3);
              kb[i][c] = *reinterpret_cast<const uint4 *>(ks + key * HD + piece * 16);
            }
          }
#pragma unroll
          for (int c = 0; c < HD / 64; ++c)
#pragma unroll
            for (int w = 0; w < 4; ++w)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t word = w == 0 ? kb[i][c].x : w == 1 ? kb[i][c].y : w == 2 ? kb[i][c].z : kb[i][c].w;
                uint32_t b0, b1;
                halves_of_e4m3(word, b0, b1);
#pragma unroll
                for (int l = PL - 1; l >= 0; --l) mma_f16(s[i], qa[l][4 * c + w], b0, b1);
              }
        }
        float top[2] = {-INFINITY, -INFINITY};
        int ev[2];
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
          const float k2 = two_to(pool_exp((int8_t)(kw >> (8 * blk))));
          ev[blk] = pool_exp((int8_t)(vw >> (8 * blk)));
          const float f0 = factor[0] * k2, f1 = factor[1] * k2, add = (float)ev[blk];
#pragma unroll
          for (int i = 2 * blk; i < 2 * blk + 2; ++i) {
            s[i][0] = fmaf(s[i][0], f0, add);
            s[i][1] = fmaf(s[i][1], f0, add);
            s[i][2] = fmaf(s[i][2], f1, add);
            s[i][3] = fmaf(s[i][3], f1, add);
          }
        }
        if (!whole) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const int key = key0 + i * 8 + key_of(2 * t4 + (c & 1)), at = pos[c >> 1];
              if (!(key <= at && (key > at - sliding || key < p.sinks))) s[i][c] = -INFINITY;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          top[0] = fmaxf(top[0], fmaxf(s[i][0], s[i][1]));
          top[1] = fmaxf(top[1], fmaxf(s[i][2], s[i][3]));
        }
        bool renew = false, far = false;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], 1));
          top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], 2));
          renew |= top[j] > run[j] + kSlack;
          far |= top[j] > -INFINITY && run[j] - top[j] > 64.0f;
        }
        if (__any_sync(0xffffffffu, renew)) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            if (!(top[j] > run[j])) continue;
            // (by way of the root: with the values' exponents a maximum may move by 200, and the sum by as much the other way)
            const float d = exp2_fast(0.5f * (run[j] - top[j]));
            total[j] = total[j] * d * d;
            const float decay = d * d;
#pragma unroll
            for (int i = 0; i < NT; ++i) o[i][2 * j] *= decay, o[i][2 * j + 1] *= decay;
            run[j] = top[j];
          }
        }
        // ---- weights, and their sum without the values' exponents
        uint32_t pa[2][PL][4];
        float ref[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) ref[j] = run[j] > -INFINITY ? run[j] : 0.0f;
        {
          float sum[2] = {0.0f, 0.0f};
#pragma unroll
          for (int blk = 0; blk < 2; ++blk) {
            const float back = two_to(-ev[blk] - kUp);
            float part[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const float a = exp2_fast(s[2 * blk + i][2 * j] - ref[j] + kUp), c = exp2_fast(s[2 * blk + i][2 * j + 1] - ref[j] + kUp);
                part[j] += a + c;
                uint32_t w[PL];
                split_halves<PL>(a, c, w);
#pragma unroll
                for (int l = 0; l < PL; ++l) pa[blk][l][2 * i + j] = w[l];
              }
            sum[0] = fmaf(part[0], back, sum[0]);
            sum[1] = fmaf(part[1], back, sum[1]);
          }
          // rare: values' exponents that differ so much that weights, but not the sum's terms, have left the range
          if (__any_sync(0xffffffffu, far) || abs(ev[0] - ev[1]) > 64) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              sum[j] = 0.0f;
#pragma unroll
              for (int i = 0; i < 4; ++i) sum[j] += exp2_fast(s[i][2 * j] - ev[i >> 1] - ref[j]) + exp2_fast(s[i][2 * j + 1] - ev[i >> 1] - ref[j]);
            }
          }
          total[0] += sum[0];
          total[1] += sum[1];
        }
        // ---- values: this thread's eight keys (four for each half of the product's step), CW dims of each
        uint32_t vb[8][CW / 4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int key = i * 8 + key_of(2 * t4 + c);
            uint32_t *to = vb[2 * i + c];
            if constexpr (HD == 128) {
              const uint4 v = *reinterpret_cast<const uint4 *>(vs + key * HD + ((g ^ (key & 7)) << 4));
              to[0] = v.x, to[1] = v.y, to[2] = v.z, to[3] = v.w;
            } else {
              const uint2 v = *reinterpret_cast<const uint2 *>(vs + key * HD + (((g >> 1) ^ (key >> 1 & 3)) << 4) + (g & 1) * 8);
              to[0] = v.x, to[1] = v.y;
            }
          }
        bool odd = false;
        if (!whole) {   // some row does not see some key: what stands there must not reach it, a NaN times a weight of zero would
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int c = 0; c < CW / 4; ++c) odd |= has_nan(vb[i][c]);
          odd = __any_sync(0xffffffffu, odd);
          if (odd) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int c = 0; c < CW / 4; ++c) {
                const uint32_t n = ((vb[i][c] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;   // the top bit of every NaN byte
                vb[i][c] &= ~((n >> 7) * 0xFFu);
              }
          }
        }
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
          for (int c = 0; c < CW / 4; ++c) {
            // bytes of two keys x four dims -> pairs of keys for each dim
            uint32_t b0[4], b1[4];
            const uint32_t *v = &vb[4 * blk][c];
            constexpr int W = CW / 4;
            halves_of_e4m3(__byte_perm(v[0], v[W], 0x5140), b0[0], b0[1]);
            halves_of_e4m3(__byte_perm(v[0], v[W], 0x7362), b0[2], b0[3]);
            halves_of_e4m3(__byte_perm(v[2 * W], v[3 * W], 0x5140), b1[0], b1[1]);
            halves_of_e4m3(__byte_perm(v[2 * W], v[3 * W], 0x7362), b1[2], b1[3]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int l = PL - 1; l >= 0; --l) mma_f16(o[4 * c + i], pa[blk][l], b0[i], b1[i]);
          }
        if (odd) {   // rare: a row that sees a NaN gets it
#pragma unroll 1
          for (int key = 0; key < kTile; ++key) {
            bool sees[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) sees[j] = key0 + key <= pos[j] && (key0 + key > pos[j] - sliding || key0 + key < p.sinks);
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                const int dim = (2 * t4 + c) * CW + i;
                const int piece = HD == 128 ? (dim >> 4) ^ (key & 7) : (dim >> 4) ^ (key >> 1 & 3);
                if ((vs[key * HD + piece * 16 + (dim & 15)] & 0x7F) == 0x7F) {
                  if (sees[0]) o[i][c] = __int_as_float(0x7FFFFFFF);
                  if (sees[1]) o[i][2 + c] = __int_as_float(0x7FFFFFFF);
                }
              }
          }
        }
      }
      __syncwarp();
      if (lane == 0) arrive(&sh.empty[slot]);
    }

    t = end;
    // ---- join the warps that share rows
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      total[j] += __shfl_xor_sync(0xffffffffu, total[j], 1);
      total[j] += __shfl_xor_sync(0xffffffffu, total[j], 2);
    }
    work_sync();   // (the unit before has been read)
    if (t4 == 0) {
      sh.top[warp][g] = run[0];
      sh.top[warp][g + 8] = run[1];
      sh.sum[warp][g] = total[0];
      sh.sum[warp][g + 8] = total[1];
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int row = g + 8 * j;
      float *dst = join + (warp * 16 + row) * HD;
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < NT; i += 4) {
          const int at = ((2 * t4 + c) * CW + i) / 4;   // of HD / 4 groups of four
          const int where = HD == 128 ? at ^ (at >> 3 & 3) ^ ((row & 1) << 2) : at ^ (at >> 2 & 3) ^ ((row & 1) << 2);
          *reinterpret_cast<float4 *>(dst + where * 4) = make_float4(o[i][2 * j + c], o[i + 1][2 * j + c], o[i + 2][2 * j + c], o[i + 3][2 * j + c]);
        }
    }
    work_sync();
    if (tid < ROWS) {   // factor of every warp's part of row tid; the row's maximum and sum in place of warp (row group)'s
      const int w0 = tid / 16, r = tid % 16;
      float best = -INFINITY;
      for (int i = 0; i < KG; ++i) best = fmaxf(best, sh.top[i * RG + w0][r]);
      const float ref = best > -INFINITY ? best : 0.0f;
      float sum = 0.0f;
      for (int i = 0; i < KG; ++i) {
        const float f = exp2_fast(0.5f * (sh.top[i * RG + w0][r] - ref));
        sh.factor[i * RG + w0][r] = f * f;
        sum += sh.sum[i * RG + w0][r] * f * f;
      }
      sh.top[w0][r] = best;
      sh.sum[w0][r] = sum;
    }
    work_sync();
    const bool cut = u.first < t_begin || u_end > t_end;
    const int c0 = cut ? (int)(u.first / chunk) : 0, c1 = cut ? (int)((u_end - 1) / chunk) : 0;
    auto joined = [&](int r, int at) {   // group `at` of four dims of row r
      float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      const int w0 = r / 16, row = r % 16;
      const int where = HD == 128 ? at ^ (at >> 3 & 3) ^ ((row & 1) << 2) : at ^ (at >> 2 & 3) ^ ((row & 1) << 2);
#pragma unroll
      for (int i = 0; i < KG; ++i) {
        const float f = sh.factor[i * RG + w0][row];
        const float4 x = *reinterpret_cast<const float4 *>(join + ((i * RG + w0) * 16 + row) * HD + where * 4);
        v.x = fmaf(x.x, f, v.x), v.y = fmaf(x.y, f, v.y), v.z = fmaf(x.z, f, v.z), v.w = fmaf(x.w, f, v.w);
      }
      return v;
    };
    auto store_row = [&](int r, int at, float4 v, float sum) {
      const int row = rt * ROWS + r;
      const int k = row / p.group;
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum * two_to(-kUp);   // (weights carry 2^kUp, their sum does not)
      const bool live = (unsigned)p.in_pos[(long)b * p.window + k] < (unsigned)seq_keys && sum != 0.0f;   // (a NaN among the scores makes the sum NaN)
      v = live ? make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      store4(outp + ((long)b * p.window + k) * p.out_stride + ((long)u.kvh * p.group + row % p.group) * HD + at * 4, v);
    };
    const int rows_here = min(ROWS, p.rows - rt * ROWS);
    constexpr int G4 = HD / 4;
    if (!cut) {
      for (int i = tid; i < rows_here * G4; i += kWorkWarps * 32) store_row(i / G4, i % G4, joined(i / G4, i % G4), sh.sum[i / G4 / 16][i / G4 % 16]);
    } else {
      // this CTA's part: slot 0 of a unit that began before its range, slot 1 of one that goes on behind it
      constexpr long PART = (long)ROWS * HD;
      float *stats = p.parts + 2L * kMaxCtas * PART;
      const int my = 2 * blockIdx.x + (u.first < t_begin ? 0 : 1);
      for (int i = tid; i < rows_here * G4; i += kWorkWarps * 32) __stcg(reinterpret_cast<float4 *>(p.parts + my * PART) + i, joined(i / G4, i % G4));
      if (tid < rows_here) __stcg(reinterpret_cast<float2 *>(stats) + my * ROWS + tid, make_float2(sh.top[tid / 16][tid % 16], sh.sum[tid / 16][tid % 16]));
      __threadfence();
      work_sync();
      if (tid == 0) sh.last = atomicAdd(&p.tickets[c0], 1) == c1 - c0;
      work_sync();
      if (sh.last) {
        __threadfence();
        for (int i = tid; i < rows_here * G4; i += kWorkWarps * 32) {
          const int r = i / G4;
          float best = -INFINITY, sum = 0.0f;
          float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          for (int c = c0; c <= c1; ++c) {
            const int from_slot = 2 * c + (c == c0 ? 1 : 0);
            const float2 ms = __ldcg(reinterpret_cast<const float2 *>(stats) + from_slot * ROWS + r);
            const float4 x = __ldcg(reinterpret_cast<const float4 *>(p.parts + from_slot * PART) + i);
            const float now = fmaxf(best, ms.x), ref = now > -INFINITY ? now : 0.0f;
            const float k2 = exp2_fast(0.5f * (best - ref)), t2 = exp2_fast(0.5f * (ms.x - ref)), keep = k2 * k2, take = t2 * t2;
            best = now;
            sum = sum * k2 * k2 + ms.y * t2 * t2;
            v.x = v.x * keep + x.x * take, v.y = v.y * keep + x.y * take, v.z = v.z * keep + x.z * take, v.w = v.w * keep + x.w * take;
          }
          store_row(r, i % G4, v, sum);
        }
        if (tid == 0) p.tickets[c0] = 0;
      }
    }
  }
}

// the layer's pages as boxes of 32 rows of a plane
int make_pool_map(TensorMap *out, const sjd_pool &p, int layer) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return SJD_ERR_UNSUPPORTED;
  const cuuint64_t plane = (cuuint64_t)KV_PAGE * p.head_dim, planes = 2ull * p.n_kv_heads;
  cuuint64_t dims[4] = {(cuuint64_t)p.head_dim, (cuuint64_t)KV_PAGE, planes, (cuuint64_t)p.n_pages};
  cuuint64_t strides[3] = {(cuuint64_t)p.head_dim, plane, plane * planes * p.n_layers};
  cuuint32_t box[4] = {(cuuint32_t)p.head_dim, (cuuint32_t)kTile, 1, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  const CUresult r = fn(reinterpret_cast<CUtensorMap *>(out), CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, (uint8_t *)p.pages + plane * planes * layer,
                        dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        p.head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SJD_OK : SJD_ERR_UNSUPPORTED;
}

int row_groups(int rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : rows <= 64 ? 4 : 8; }
size_t parts_bytes(int rg, int hd) { return 2ull * kMaxCtas * 16 * rg * (hd + 2) * 4; }

}  // namespace
}  // namespace sjd

using namespace sjd;

extern "C" size_t sjd_pool_attention_workspace_bytes(const sjd_pool *pool, int window, int n_heads) {
  if (check_pool(pool, false) != SJD_OK || window < 1 || n_heads < 1 || n_heads % pool->n_kv_heads != 0) return 0;
  const int64_t rows = (int64_t)window * (n_heads / pool->n_kv_heads);
  return 1024 + parts_bytes(row_groups(rows > 128 ? 128 : (int)rows), pool->head_dim);
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
  if ((int64_t)batch * window > 0x7FFFFFFF || rows > 0x7FFFFFFF) return SJD_ERR_CAPACITY;
  if (ws_bytes < sjd_pool_attention_workspace_bytes(pool, window, n_heads)) return SJD_ERR_CAPACITY;
  int dev = 0, cc_major = 0, sms = 0;
  SJD_CUDA(cudaGetDevice(&dev));
  SJD_CUDA(cudaDeviceGetAttribute(&cc_major, cudaDevAttrComputeCapabilityMajor, dev));
  SJD_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  if (cc_major != 10) return SJD_ERR_UNSUPPORTED;
  TensorMap map;
  rc = make_pool_map(&map, *pool, layer);
  if (rc != SJD_OK) return rc;
  const int rg = row_groups(rows > 128 ? 128 : (int)rows), hd = pool->head_dim;
  PoolAttnParams p;
  memset(&p, 0, sizeof(p));
  p.pool = *pool;
  p.layer = layer;
  p.batch = batch;
  p.window = window;
  p.n_heads = n_heads;
  p.group = group;
  p.rows = (int)rows;
  p.row_tiles = (int)((rows + 16 * rg - 1) / (16 * rg));
  p.sliding = sliding;
  p.sinks = sliding > 0 ? sinks : 0;
  p.scale = (scale > 0.0f ? scale : 1.0f / sqrtf((float)hd)) * 1.4426950408889634f;
  p.q = q;
  p.q_stride = q_stride;
  p.out_stride = out_stride;
  p.seqs = seqs;
  p.in_pos = in_pos;
  p.out = out;
  p.tickets = (int *)ws;
  p.parts = (float *)((char *)ws + 1024);
  const int64_t entries = (int64_t)batch * p.row_tiles, units = entries * pool->n_kv_heads;
  if (units > 0x7FFFFFFF) return SJD_ERR_CAPACITY;
  // Equal ranges, unless the CTAs would have to look at too many positions to find them: then there are units enough
  p.cut = entries <= kMaxEntries && (int64_t)batch * window <= 8192;
  p.n_entries = (int)entries;
  const int box = kTile * hd, fixed = kWorkWarps * 16 * hd * 4 + (int)sizeof(AttnShared<128>);
  p.slots = (kSmem - 1024 - fixed) / (2 * box);
  p.slots = p.slots > kMaxSlots ? kMaxSlots : p.slots;
  const size_t smem = (size_t)fixed + (size_t)p.slots * 2 * box;
  const unsigned grid = p.cut ? (unsigned)(sms < kMaxCtas ? sms : kMaxCtas) : (unsigned)units;
  const CUtensorMap &m = reinterpret_cast<const CUtensorMap &>(map);
  auto launch = [&](auto kernel) -> int {
    const int r = allow_smem(kernel, smem);   // (the size follows from the kernel's head_dim)
    if (r != SJD_OK) return r;
    SJD_CUDA(launch_kernel(kernel, dim3(grid), dim3(kThreads), smem, (cudaStream_t)cuda_stream, m, p));
    SJD_CHECK_LAUNCH();
    return SJD_OK;
  };
#define SJD_PICK(T, HD) \
  (rg == 1 ? launch(pool_attention_kernel<T, HD, 1>) : rg == 2 ? launch(pool_attention_kernel<T, HD, 2>) \
   : rg == 4 ? launch(pool_attention_kernel<T, HD, 4>) : launch(pool_attention_kernel<T, HD, 8>))
  if (dtype == SJD_F32) return hd == 128 ? SJD_PICK(float, 128) : SJD_PICK(float, 64);
  return hd == 128 ? SJD_PICK(__nv_bfloat16, 128) : SJD_PICK(__nv_bfloat16, 64);
#undef SJD_PICK
}
