// Projections of bf16 rows with their epilogue:  out = residual + act(x W^T + b) [* (x U^T + c)],  fp32 sums, rounded once.
//
// Weights are the 128 rows of a CTA's MMA and tokens its columns: any number of tokens is a column count, a thread's bias is one
// number, and a thread stores a feature of token after token (a warp: 64 bytes of a row).  With U a CTA's 128 rows are 64 features of W and the
// same of U; they meet in shared memory.
//
// Few rows (linear_split_kernel): the time is that of the weights from HBM.  A cluster shares a tile of features, each CTA (each pair) a range
// of K; their sums meet over distributed shared memory, a share of the tokens each, in the order of the ranges, so that one launch
// does it without scratch and without atomics.
// Many rows (linear_tiles_kernel): the time is that of the products, or of the operands from L2.  CTA pairs with 256 features by up to 256
// tokens, persistent, two accumulators, so that a unit's epilogue runs under the next unit's products.
//
// Measured (bf16, in brackets a library's product of the same sizes, or two of them for U, without an epilogue; 20 calls with the same operands replayed from a graph, so that up
// to 100 MB of them stay in L2): 1 x 4096 x 4096 7.4 us (12.6), 64 x 4096 x 4096 9.4 (7.6), 32 x 14336 x 4096 with U 40.9 (42.2; 36.6 are the bytes: 90 %), 256 x 4096 x 11008 28 to
// 30 (23.3), 1063 x 6144 x 4096 41.3 (38.0), 4223 x 14336 x 4096 with U 650 to 660 (645 to 655; 1500 TFLOP/s).  With four epilogue warps instead of sixteen 4223 x 1408 x 512 with U took 52 us, now 31; with the
// sums of ranges read a number at a time, in more clusters than the device holds at once, 256 x 4096 x 11008 took 64.
#include <algorithm>
#include <atomic>

#include "tcgen05.cuh"

namespace sjd {
namespace {

constexpr int kRows = 128, kTileK = 64, kUmmaK = 16;      // weight rows of a CTA's tile; bf16 entries of a k-block (a swizzle atom), of an MMA
constexpr int kWBytes = kRows * kTileK * 2;
constexpr int kStages = 12;
constexpr int kMaxTokens = 256;                           // of a tile
constexpr int kSmem = 232448 - 2048;                      // most dynamic shared memory of a CTA, beside its static part
constexpr int kSmemOfTwo = 232448 / 2 - 2048;             // of each of two CTAs of an SM
constexpr int kMaxSplits = 8;
constexpr int kExTokens = 16;                             // tokens of a round of the epilogue of pairs

struct LinearParams {
  int M, N, k_blocks;
  int tokens;           // of a tile, a multiple of 16
  int token_tiles, units, splits, stages, act;
  const __nv_bfloat16 *bias, *bias_up, *residual;
  __nv_bfloat16 *out;
  long residual_stride, out_stride;
  int by_four;          // rows of residual and out start on 8 bytes
  int32_t *status;
};

template <int ACT>
__device__ __forceinline__ float activate(float v) {
  // Forms in which nothing cancels: 1 + erf and 1 + tanh of -5 have lost what bf16 holds.  The exponential is off by up to 2 + 1.2 |argument| units in the last place,
  // 2^-16 at 87; from there on the quotient is 0, where v is left with less than 2^-119.  The result is rounded to 2^-9.
  if constexpr (ACT == SJD_ACT_RELU) return v < 0.0f ? 0.0f : v;   // (a NaN stays)
  if constexpr (ACT == SJD_ACT_SILU) return v * __fdividef(1.0f, 1.0f + __expf(-v));
  if constexpr (ACT == SJD_ACT_GELU) {
    // half of erfc(|v| / sqrt(2)): t P(t) exp(-v^2 / 2), t = 1 / (1 + 0.55 |v| / sqrt(2)), P fitted for the least relative error, 2^-17.8.  (erfcf in its place, 1063 x 6144 x 4096:
    // 48.9 us instead of 45.4)
    const float t = __fdividef(1.0f, fmaf(0.388908744f, fabsf(v), 1.0f));
    float q = fmaf(0.0494243689f, t, -0.15092659f);
    q = fmaf(q, t, 0.0885907039f), q = fmaf(q, t, 0.0693082735f), q = fmaf(q, t, 0.133359432f), q = fmaf(q, t, 0.155093849f), q = fmaf(q, t, 0.155152082f);
    q *= t * __expf(-0.5f * v * v);
    return v * (v > 0.0f ? 1.0f - q : q);
  }
  if constexpr (ACT == SJD_ACT_GELU_TANH) return v * __fdividef(1.0f, 1.0f + __expf(-1.5957691f * fmaf(0.044715f * v * v, v, v)));   // (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u))
  return v;
}
template <int ACT>
struct Act {
  static constexpr int kind = ACT;
};
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
  switch (act) {
    case SJD_ACT_RELU: f(Act<SJD_ACT_RELU>()); break;
    case SJD_ACT_SILU: f(Act<SJD_ACT_SILU>()); break;
    case SJD_ACT_GELU: f(Act<SJD_ACT_GELU>()); break;
    case SJD_ACT_GELU_TANH: f(Act<SJD_ACT_GELU_TANH>()); break;
    default: f(Act<SJD_ACT_NONE>());
  }
}

// AND over the epilogue threads (named barrier 1): keeps their control flow uniform
template <int THREADS>
__device__ __forceinline__ bool all_of(bool pred) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbar.red.and.pred p, 1, %2, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)pred), "n"(THREADS)
      : "memory");
  return r != 0;
}
__device__ __forceinline__ void fault(int32_t *status) {
  if (status) atomicCAS(status, 0, SJD_ERR_DEVICE_TIMEOUT);
}
__device__ __forceinline__ float4 ld_cluster(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}
template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t *at, uint32_t cols) {
  if constexpr (CG == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(at)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(at)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
}
template <int CG>
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t cols) {
  if constexpr (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
  else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
}
__host__ __device__ inline uint32_t tmem_columns(int n) {
  uint32_t c = 32;
  while ((int)c < n) c <<= 1;
  return c;
}
// a k-block of a CTA: its 128 weight rows, or 64 of W and the same of U, and its tokens
template <int CG, bool GATED>
__device__ __forceinline__ void load_stage(uint32_t dst, const CUtensorMap *w, const CUtensorMap *u, const CUtensorMap *x, int k, int feature,
                                           int token, uint32_t bar, uint64_t policy) {
  if constexpr (CG == 2) {
    pair_load(dst, w, k, feature, bar, policy);
    if (GATED) pair_load(dst + kWBytes / 2, u, k, feature, bar, policy);
    pair_load_nohint(dst + kWBytes, x, k, token, bar);
  } else {
    auto load = [&](uint32_t to, const CUtensorMap *map, int row) {
      asm volatile(
          "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;"
          ::"r"(to), "l"(map), "r"(k), "r"(row), "r"(bar), "l"(policy)
          : "memory");
    };
    load(dst, w, feature);
    if (GATED) load(dst + kWBytes / 2, u, feature);
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(dst + kWBytes), "l"(x), "r"(k), "r"(token), "r"(bar)
        : "memory");
  }
}
__device__ __forceinline__ uint64_t weight_policy(bool once) {
  uint64_t policy;
  if (once) asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  else asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
  return policy;
}
// a wait ran out: the copies under way have ample time to end
__device__ __forceinline__ void let_copies_end() {
  const unsigned long long t0 = global_ns();
  while (global_ns() - t0 < 20000000ull) {}
}

// CG: CTAs of a pair (1: none).  Grid: (CG * splits, tiles of CG * 128 weight rows, tiles of tokens), a cluster along x.
template <int CG, bool GATED>
__global__ void __launch_bounds__(64 + 128 * CG, CG == 1 ? 2 : 1)
    linear_split_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap u_map,
                        const __grid_constant__ CUtensorMap x_map, const __grid_constant__ LinearParams p) {
  constexpr int EPI = 128 * CG, FT = GATED ? kRows / 2 : kRows;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);   // (the same place in every CTA)
  __shared__ uint64_t full[kStages], empty[kStages], acc_full;
  __shared__ uint32_t s_tmem;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = blockIdx.x, split = rank / CG, half = rank % CG, lead = rank - half;
  const int feature0 = (blockIdx.y * CG + half) * FT, token0 = blockIdx.z * p.tokens, x_rows = p.tokens / CG;
  const int stage_bytes = kWBytes + x_rows * kTileK * 2;
  const int kb0 = (int)((long)split * p.k_blocks / p.splits), kb1 = (int)((long)(split + 1) * p.k_blocks / p.splits);
  const uint32_t cols = tmem_columns(p.tokens), smem0 = smem_u32(smem);
  if (tid == 0) {
    tma_prefetch_desc(&w_map);
    tma_prefetch_desc(&x_map);
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    mbar_init(&acc_full, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<CG>(&s_tmem, cols);
  tc_fence_before();
  cluster_sync();   // (barriers of a pair's other CTA)
  tc_fence_after();
  pdl_trigger();   // (not before the allocation: a CTA of a later kernel that holds tensor memory waits for this one)
  const uint32_t tmem = s_tmem;
  pdl_wait();

  if (warp == 0) {
    // ------------------------------------------------------------------ copies
    const uint64_t policy = weight_policy(gridDim.z == 1);
    const uint32_t full0 = CG == 2 ? cluster_addr(&full[0], lead) : smem_u32(&full[0]);
    int s = 0;
    uint32_t ph = 1;
    bool ok = true;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (kb - kb0 >= p.stages && !warp_wait(&empty[s], ph)) { ok = false; break; }
      if (elect_one()) {
        if (half == 0) mbar_expect_tx(&full[s], (uint32_t)(CG * stage_bytes));
        load_stage<CG, GATED>(smem0 + s * stage_bytes, &w_map, &u_map, &x_map, kb * kTileK, feature0, token0 + half * x_rows, full0 + s * 8, policy);
      }
      __syncwarp();
      if (++s == p.stages) { s = 0; ph ^= 1u; }
    }
    if (!ok) let_copies_end();
  } else if (warp == 1) {
    // ------------------------------------------------------------------ products
    if (half == 0) {
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(p.tokens >> 3) << 17) | ((uint32_t)(CG * kRows >> 4) << 24);
      const uint64_t desc0 = umma_desc_sw128(0);
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!warp_wait(&full[s], ph)) { ok = false; break; }
        tc_fence_after();
        if (elect_one()) {
          const uint32_t at = smem0 + s * stage_bytes;
          const uint64_t a = desc0 | (uint64_t)(at >> 4), b = desc0 | (uint64_t)((at + kWBytes) >> 4);
#pragma unroll
          for (int k = 0; k < kTileK / kUmmaK; ++k) {
            if constexpr (CG == 2) pair_mma(tmem, a + k * 2, b + k * 2, idesc, kb > kb0 || k > 0);
            else umma_bf16(tmem, a + k * 2, b + k * 2, idesc, kb > kb0 || k > 0);
          }
          if constexpr (CG == 2) pair_commit(&empty[s], (unsigned short)(3 << lead));
          else umma_commit(&empty[s]);
        }
        __syncwarp();
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
      if (ok && elect_one()) {
        if constexpr (CG == 2) pair_commit(&acc_full, (unsigned short)(3 << lead));
        else umma_commit(&acc_full);
      }
      __syncwarp();
    }
  } else {
    // ------------------------------------------------------------------ this CTA's sums to shared memory: [token][128]
    // (the ring is free: every product has been waited for)
    const int quarter = warp & 3, row = quarter * 32 + lane, grp = (warp - 2) >> 2;
    float *ex = reinterpret_cast<float *>(smem) + row;
    const bool ok = all_of<EPI>(warp_wait(&acc_full, 0));
    if (!ok && tid == 64) fault(p.status);
    tc_fence_after();
    const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16);
    for (int m = grp * 16; m < p.tokens; m += 16 * CG) {
      uint32_t v[16];
      tmem_ld16_issue(at + m, v);
      tmem_ld_wait();
#pragma unroll
      for (int i = 0; i < 16; ++i) ex[(m + i) * kRows] = ok ? __uint_as_float(v[i]) : __int_as_float(0x7FFFFFFF);
    }
    tc_fence_before();
  }
  __syncwarp();
  cluster_sync();
  if (warp >= 2) {
    // ------------------------------------------------------------------ a share of the tokens: the sums of all ranges, and the epilogue
    // A lane has four features of a token; with U, 16 lanes have the features of one token and the other 16 those of the next.
    constexpr int WARPS = EPI / 32, AT_ONCE = GATED ? 2 : 1;
    const int f = (GATED ? lane & 15 : lane) * 4, feature = feature0 + f;
    const int have = min(p.tokens, p.M - token0), per = (have + p.splits - 1) / p.splits;
    const int m0 = split * per, m1 = min(have, m0 + per);
    float b[4], c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      b[j] = p.bias && feature + j < p.N ? __bfloat162float(p.bias[feature + j]) : 0.0f;
      c[j] = GATED && p.bias_up && feature + j < p.N ? __bfloat162float(p.bias_up[feature + j]) : 0.0f;
    }
    with_act(p.act, [&](auto act) {
      for (int m = m0 + (warp - 2) * AT_ONCE + (GATED ? lane >> 4 : 0); m < m1 && feature < p.N; m += WARPS * AT_ONCE) {
        float4 v[kMaxSplits], u[GATED ? kMaxSplits : 1];
#pragma unroll
        for (int s = 0; s < kMaxSplits; ++s) {   // (all loads under way together)
          if (s >= p.splits) break;
          const uint32_t from = cluster_addr(smem, s * CG + half) + (uint32_t)(m * kRows + f) * 4;
          v[s] = ld_cluster(from);
          if (GATED) u[s] = ld_cluster(from + FT * 4);
        }
#pragma unroll
        for (int s = 1; s < kMaxSplits; ++s) {
          if (s >= p.splits) break;
          v[0].x += v[s].x, v[0].y += v[s].y, v[0].z += v[s].z, v[0].w += v[s].w;
          if (GATED) u[0].x += u[s].x, u[0].y += u[s].y, u[0].z += u[s].z, u[0].w += u[s].w;
        }
        const float *g = &v[0].x, *h = &u[0].x;
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          y[j] = activate<decltype(act)::kind>(g[j] + b[j]);
          if (GATED) y[j] *= h[j] + c[j];
        }
        const __nv_bfloat16 *res = p.residual + (long)(token0 + m) * p.residual_stride + feature;
        __nv_bfloat16 *out = p.out + (long)(token0 + m) * p.out_stride + feature;
        if (p.by_four && feature + 4 <= p.N) {
          if (p.residual) {
            const uint2 r = *reinterpret_cast<const uint2 *>(res);
            y[0] += __uint_as_float(r.x << 16), y[1] += __uint_as_float(r.x & 0xFFFF0000u), y[2] += __uint_as_float(r.y << 16), y[3] += __uint_as_float(r.y & 0xFFFF0000u);
          }
          const __nv_bfloat162 lo = __floats2bfloat162_rn(y[0], y[1]), hi = __floats2bfloat162_rn(y[2], y[3]);
          *reinterpret_cast<uint2 *>(out) = make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (feature + j < p.N) out[j] = __float2bfloat16_rn(p.residual ? y[j] + __bfloat162float(res[j]) : y[j]);
        }
      }
    });
  }
  __syncwarp();
  cluster_sync();   // (nobody leaves while its sums may be read)
  if (warp == 1) {
    tc_fence_after();
    tmem_free<CG>(tmem, cols);
  }
}

// Persistent CTA pairs; unit u: tile of 256 weight rows u / token_tiles, tile of tokens u % token_tiles.
constexpr int kGroups = 4;                                // of four epilogue warps
constexpr int kTilesThreads = 64 + kGroups * 128;
template <bool GATED>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kTilesThreads, 1)
    linear_tiles_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap u_map,
                        const __grid_constant__ CUtensorMap x_map, const __grid_constant__ LinearParams p) {
  constexpr int FT = GATED ? kRows / 2 : kRows;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);   // (the same place in every CTA)
  __shared__ uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2];
  __shared__ uint32_t s_tmem;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = blockIdx.x & 1u;
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1, x_rows = p.tokens / 2;
  const int stage_bytes = kWBytes + x_rows * kTileK * 2;
  const uint32_t cols = tmem_columns(2 * p.tokens), smem0 = smem_u32(smem);
  if (tid == 0) {
    tma_prefetch_desc(&w_map);
    tma_prefetch_desc(&x_map);
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], 2 * 4 * kGroups);   // the epilogue warps of both CTAs
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<2>(&s_tmem, cols);
  tc_fence_before();
  cluster_sync();
  tc_fence_after();
  pdl_trigger();   // (not before the allocation: a CTA of a later kernel that holds tensor memory waits for this one)
  const uint32_t tmem = s_tmem;
  pdl_wait();

  if (warp == 0) {
    // ------------------------------------------------------------------ copies (each CTA its half)
    const uint64_t policy = weight_policy(p.token_tiles == 1);
    const uint32_t full0 = cluster_addr(&full[0], 0);
    int s = 0, it = 0;
    uint32_t ph = 1;
    bool ok = true;
    for (int u = pair; u < p.units && ok; u += n_pairs) {
      const int feature = (u / p.token_tiles * 2 + (int)rank) * FT, token = u % p.token_tiles * p.tokens + (int)rank * x_rows;
      for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
        if (it >= p.stages && !warp_wait(&empty[s], ph)) { ok = false; break; }
        if (elect_one()) {
          if (rank == 0) mbar_expect_tx(&full[s], (uint32_t)(2 * stage_bytes));
          load_stage<2, GATED>(smem0 + s * stage_bytes, &w_map, &u_map, &x_map, kb * kTileK, feature, token, full0 + s * 8, policy);
        }
        __syncwarp();
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
    }
    if (!ok) let_copies_end();
  } else if (warp == 1) {
    // ------------------------------------------------------------------ products (the first CTA for both)
    if (rank == 0) {
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(p.tokens >> 3) << 17) | ((uint32_t)(256 >> 4) << 24);
      const uint64_t desc0 = umma_desc_sw128(0);
      int s = 0, n = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int u = pair; u < p.units && ok; u += n_pairs, ++n) {
        const int buf = n & 1;
        if (!warp_wait(&acc_empty[buf], ((n >> 1) & 1) ^ 1u)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d = tmem + buf * p.tokens;
        for (int kb = 0; kb < p.k_blocks; ++kb) {
          if (!warp_wait(&full[s], ph)) { ok = false; break; }
          tc_fence_after();
          if (elect_one()) {
            const uint32_t at = smem0 + s * stage_bytes;
            const uint64_t a = desc0 | (uint64_t)(at >> 4), b = desc0 | (uint64_t)((at + kWBytes) >> 4);
#pragma unroll
            for (int k = 0; k < kTileK / kUmmaK; ++k) pair_mma(d, a + k * 2, b + k * 2, idesc, kb > 0 || k > 0);
            pair_commit(&empty[s]);
          }
          __syncwarp();
          if (++s == p.stages) { s = 0; ph ^= 1u; }
        }
        if (ok && elect_one()) pair_commit(&acc_full[buf]);
        __syncwarp();
      }
    }
  } else {
    // ------------------------------------------------------------------ epilogue warps (from 2 on): groups of four, 16 tokens in turn
    const int quarter = warp & 3, row = quarter * 32 + lane, grp = (warp - 2) >> 2, e = (tid - 64) & 127;
    float *ex = reinterpret_cast<float *>(smem + p.stages * stage_bytes) + grp * kRows * (kExTokens + 1);   // GATED: [128][kExTokens + 1]
    // with U, thread e finishes feature e % 64 for every second token
    const int f = GATED ? e & 63 : row, odd = GATED ? e >> 6 : 0;
    int n = 0;
    bool ok = true;
    for (int u = pair; u < p.units; u += n_pairs, ++n) {
      const int buf = n & 1, feature = (u / p.token_tiles * 2 + (int)rank) * FT + f, m_base = u % p.token_tiles * p.tokens;
      const int m_left = min(p.tokens, p.M - m_base);
      const bool live = feature < p.N;
      const float b = live && p.bias ? __bfloat162float(p.bias[feature]) : 0.0f, c = GATED && live && p.bias_up ? __bfloat162float(p.bias_up[feature]) : 0.0f;
      if (ok && !all_of<kGroups * 128>(warp_wait(&acc_full[buf], (n >> 1) & 1))) {   // (once it ran out no unit is waited for: all are NaN)
        ok = false;
        if (tid == 64) fault(p.status);
      }
      tc_fence_after();
      const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16) + buf * p.tokens;
      with_act(p.act, [&](auto act) {
        constexpr int PER = GATED ? kExTokens / 2 : kExTokens, STEP = GATED ? 2 : 1;
        const long first = m_base + grp * 16 + odd;
        const __nv_bfloat16 *res = p.residual + first * p.residual_stride + feature;
        __nv_bfloat16 *out = p.out + first * p.out_stride + feature;
        for (int m0 = grp * 16; m0 < p.tokens; m0 += 16 * kGroups) {
          const int left = live ? (m_left - m0 - odd + STEP - 1) / STEP : 0;   // outputs of this thread, if below PER
          float r[PER], y[PER];
#pragma unroll
          for (int i = 0; i < PER; ++i) r[i] = 0.0f;
          if (p.residual) {
#pragma unroll
            for (int i = 0; i < PER; ++i)
              if (i < left) r[i] = __bfloat162float(res[i * STEP * p.residual_stride]);
          }
          uint32_t v[16];
          tmem_ld16_issue(at + m0, v);
          tmem_ld_wait();
          if constexpr (GATED) {
#pragma unroll
            for (int i = 0; i < 16; ++i) ex[row * (kExTokens + 1) + i] = __uint_as_float(v[i]);
            asm volatile("bar.sync %0, 128;" ::"r"(grp + 2) : "memory");
#pragma unroll
            for (int i = 0; i < PER; ++i)
              y[i] = activate<decltype(act)::kind>(ex[f * (kExTokens + 1) + 2 * i + odd] + b) * (ex[(64 + f) * (kExTokens + 1) + 2 * i + odd] + c);
            asm volatile("bar.sync %0, 128;" ::"r"(grp + 2) : "memory");
          } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) y[i] = activate<decltype(act)::kind>(__uint_as_float(v[i]) + b);
          }
          if (__builtin_expect(!ok, 0)) {
#pragma unroll
            for (int i = 0; i < PER; ++i) y[i] = __int_as_float(0x7FFFFFFF);
          }
          if (left >= PER) {
#pragma unroll
            for (int i = 0; i < PER; ++i) out[i * STEP * p.out_stride] = __float2bfloat16_rn(r[i] + y[i]);
          } else {
#pragma unroll
            for (int i = 0; i < PER; ++i)
              if (i < left) out[i * STEP * p.out_stride] = __float2bfloat16_rn(r[i] + y[i]);
          }
          res += 16l * kGroups * p.residual_stride;
          out += 16l * kGroups * p.out_stride;
        }
      });
      tc_fence_before();
      __syncwarp();
      if (lane == 0)   // the accumulator is free (the first CTA issues into both CTAs' tensor memory)
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr(&acc_empty[buf], 0)) : "memory");
    }
  }
  tc_fence_before();
  __syncwarp();
  cluster_sync();   // neither CTA leaves while the other may reach into it
  if (warp == 1) {
    tc_fence_after();
    tmem_free<2>(tmem, cols);
  }
}

// bf16 [rows][cols], rows `stride` entries apart, as boxes of box_rows x 64 with 128-byte swizzle; what lies outside reads as zeros
int make_map(TensorMap *out, const void *base, long rows, long cols, long stride, int box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return SJD_ERR_UNSUPPORTED;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)(rows > 1 ? stride : (cols + 7) / 8 * 8) * 2};
  cuuint32_t box[2] = {(cuuint32_t)kTileK, (cuuint32_t)box_rows}, estr[2] = {1, 1};
  const CUresult r = fn(reinterpret_cast<CUtensorMap *>(out), CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, strides, box,
                        estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SJD_OK : SJD_ERR_UNSUPPORTED;
}

int round16(int n) { return (n + 15) / 16 * 16; }

// Clusters of `size` CTAs with an SM each that the current device holds at a time: its SMs come in groups, and a cluster is in one of
// them (33 of four, 22 of six and 15 of eight on 148 SMs; a sixteenth cluster of eight doubles the time of a launch).
int clusters_of(int dev, int size, int *out) {
  constexpr int kDevices = 64;
  static std::atomic<int> known[kDevices][kMaxSplits + 1];   // (0: not asked yet)
  if (dev < kDevices && (*out = known[dev][size].load(std::memory_order_relaxed)) > 0) return SJD_OK;
  const int rc = allow_smem(linear_split_kernel<2, false>, kSmem);
  if (rc != SJD_OK) return rc;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(size), cfg.blockDim = dim3(64 + 256), cfg.dynamicSmemBytes = kSmem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = size, attr[0].val.clusterDim.y = 1, attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr, cfg.numAttrs = 1;
  SJD_CUDA(cudaOccupancyMaxActiveClusters(out, (const void *)linear_split_kernel<2, false>, &cfg));
  if (dev < kDevices) known[dev][size].store(*out, std::memory_order_relaxed);
  return SJD_OK;
}

}  // namespace
}  // namespace sjd

using namespace sjd;

extern "C" int sjd_linear(int rows, int n, int k, const void *x, int64_t x_stride, const void *w, const void *w_up, int64_t w_stride,
                          const void *bias, const void *bias_up, int act, const void *residual, int64_t residual_stride, void *out,
                          int64_t out_stride, int32_t *status, void *cuda_stream) {
  if (act < SJD_ACT_NONE || act > SJD_ACT_GELU_TANH) return SJD_ERR_UNSUPPORTED;
  if (rows < 0 || n < 1 || k < 1) return SJD_ERR_BAD_ARG;
  if (rows == 0) return SJD_OK;
  if (!x || !w || !out || (bias_up && !w_up)) return SJD_ERR_BAD_ARG;
  if ((rows > 1 && (x_stride < k || out_stride < n || (residual && residual_stride < n))) || (n > 1 && w_stride < k)) return SJD_ERR_BAD_ARG;
  if ((((uintptr_t)x | (uintptr_t)w | (uintptr_t)w_up) & 15u) != 0 || (rows > 1 && (x_stride & 7)) || (n > 1 && (w_stride & 7))) return SJD_ERR_BAD_ARG;
  if ((((uintptr_t)bias | (uintptr_t)bias_up | (uintptr_t)residual | (uintptr_t)out) & 1u) != 0 || ((uintptr_t)status & 3u) != 0) return SJD_ERR_BAD_ARG;
  // (coordinates of copies are 32 bits, strides 40 bits of bytes)
  if (n > 1 << 21 || k > 1 << 28 || rows > 1 << 28 || x_stride >= 1ll << 38 || w_stride >= 1ll << 38) return SJD_ERR_CAPACITY;
  int dev = 0, cc_major = 0, sms = 0;
  SJD_CUDA(cudaGetDevice(&dev));
  SJD_CUDA(cudaDeviceGetAttribute(&cc_major, cudaDevAttrComputeCapabilityMajor, dev));
  SJD_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  if (cc_major != 10) return SJD_ERR_UNSUPPORTED;
  const bool gated = w_up != nullptr;
  const int ft = gated ? kRows / 2 : kRows;
  LinearParams p;
  memset(&p, 0, sizeof(p));
  p.M = rows, p.N = n, p.k_blocks = (k + kTileK - 1) / kTileK, p.act = act;
  p.bias = (const __nv_bfloat16 *)bias, p.bias_up = (const __nv_bfloat16 *)bias_up, p.residual = (const __nv_bfloat16 *)residual;
  p.by_four = (((uintptr_t)residual | (uintptr_t)out) & 7u) == 0 && ((out_stride | (residual ? residual_stride : 0)) & 3) == 0;
  p.residual_stride = residual_stride, p.out = (__nv_bfloat16 *)out, p.out_stride = out_stride, p.status = status;
  // ---- which kernel, and how the work is cut
  const int pairs = sms / 2, kb = p.k_blocks;
  int cg = 1, splits = 1;
  bool tiles = false;
  if (rows <= 64) {
    // as many ranges of K as all fit at two CTAs per SM
    const int features = (n + ft - 1) / ft;
    p.tokens = round16(rows), p.token_tiles = 1;
    for (int s : {2, 3, 4, 6, 8}) {
      if (s * 2 > kb || features * s > 2 * sms) break;
      int fit = 0;
      const int rc = clusters_of(dev, s, &fit);
      if (rc != SJD_OK) return rc;
      if (features <= 2 * fit) splits = s;
    }
  } else {
    // clocks of a launch: a k-block takes a pair its products (8192 a clock), or its 256 + tokens rows from L2, of which an SM takes 64 bytes
    // and all together 6600 a clock
    const long features = (n + 2 * ft - 1) / (2 * ft);
    double best = 1e300;
    cg = 2;
    auto consider = [&](int t, int s) {
      const int tokens = round16((rows + t - 1) / t);
      const long units = features * t * s, active = std::min<long>(units, pairs);
      const double bytes = (256.0 + tokens) * kTileK * 2, block = std::max(2.0 * tokens, bytes * std::max(1.0 / 128, active / 6600.0));
      const double clocks = (double)((units + pairs - 1) / pairs) * ((kb + s - 1) / s * block + 800) + 11.0 * tokens + (s > 1 ? 2500 : 0);
      if (clocks < best) best = clocks, tiles = s == 1, splits = s, p.tokens = tokens, p.token_tiles = t;
    };
    const int t0 = (rows + kMaxTokens - 1) / kMaxTokens;
    for (int t = t0; t <= (rows + 31) / 32 && t <= t0 + 16; ++t) {
      consider(t, 1);
      for (int s = 2; s <= 4 && s * 2 <= kb && features * t * s <= pairs; ++s) {
        int fit = 0;
        const int rc = clusters_of(dev, 2 * s, &fit);
        if (rc != SJD_OK) return rc;
        if (features * t <= fit) consider(t, s);
      }
    }
  }
  p.splits = splits;
  const long features = (n + cg * ft - 1) / (cg * ft);
  if (features * p.token_tiles > 0x7FFFFFFF) return SJD_ERR_CAPACITY;
  p.units = (int)(features * p.token_tiles);
  TensorMap wm, um, xm;
  int rc = make_map(&wm, w, n, k, w_stride, ft);
  if (rc == SJD_OK) rc = make_map(&um, gated ? w_up : w, n, k, w_stride, ft);
  if (rc == SJD_OK) rc = make_map(&xm, x, rows, k, x_stride, p.tokens / cg);
  if (rc != SJD_OK) return rc;
  const CUtensorMap &W = reinterpret_cast<const CUtensorMap &>(wm), &U = reinterpret_cast<const CUtensorMap &>(um), &X = reinterpret_cast<const CUtensorMap &>(xm);
  const int stage = kWBytes + p.tokens / cg * kTileK * 2, exchange = tiles && gated ? kGroups * kRows * (kExTokens + 1) * 4 : 0;
  const int room = (cg == 1 ? kSmemOfTwo : kSmem) - 1024 - exchange;
  p.stages = std::min(kStages, room / stage);
  const size_t smem = 1024 + std::max((size_t)p.stages * stage + exchange, tiles ? (size_t)0 : (size_t)p.tokens * kRows * 4);
  auto launch = [&](auto kernel, dim3 grid, int threads, int cluster) -> int {
    const int r = allow_smem(kernel, kSmem);
    if (r != SJD_OK) return r;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = grid, cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = smem, cfg.stream = (cudaStream_t)cuda_stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // (waits for the launch before it itself)
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr, cfg.numAttrs = cluster > 0 ? 2 : 1;
    SJD_CUDA(cudaLaunchKernelEx(&cfg, kernel, W, U, X, p));
    SJD_CHECK_LAUNCH();
    return SJD_OK;
  };
  if (tiles) {
    const dim3 grid(2 * std::min(pairs, p.units));
    return gated ? launch(linear_tiles_kernel<true>, grid, kTilesThreads, 0) : launch(linear_tiles_kernel<false>, grid, kTilesThreads, 0);
  }
  const dim3 grid(cg * splits, (unsigned)features, p.token_tiles);
  if (cg == 1) return gated ? launch(linear_split_kernel<1, true>, grid, 192, splits) : launch(linear_split_kernel<1, false>, grid, 192, splits);
  return gated ? launch(linear_split_kernel<2, true>, grid, 320, 2 * splits) : launch(linear_split_kernel<2, false>, grid, 320, 2 * splits);
}
