// Rotary step with several axes and append to the 8-bit paged cache.
//
// A block of threads owns a block of 16 positions of a sequence and some heads, a warp one head (of the queries, keys or values) at a time:
// it loads the head's rows, rotates them, reduces the largest entry, and stores 16 x head_dim bytes under one power-of-two scale.  Rows that
// were in the block before are read, scaled to what they stand for, and take part; nothing outside the block's rows up to the last
// new one is touched, so no two warps meet.  A lane holds pairs (i, i + head_dim / 2) of all rows, so that the rotation needs no exchange.
//   (a, b) -> (a c - b s, b c + a s), angle = position * theta^(-2 f / rot)
// Angles are products in 64 bits (a position of 10^6 times a frequency in 32 bits is off by 0.06), their cosine and sine are rounded to
// 32 bits once and shared by the heads of a block of threads through shared memory.  Products and sums are single 32-bit operations
// (no fused multiply-add), so that an entry next to a rounding border falls on the side that the formula says.
// Rounding: q to its own type, k and v to e4m3 (half a step is 2^-4 of an entry) under a scale that lets the largest entry reach
// 224 to 448; the scale itself is exact.
// Bound: bytes, one pass over q, k, v.
#include "common.cuh"

namespace sjd {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kAppendWarps = kAppendThreads / 32;

struct AppendParams {
  sjd_pool pool;
  int layer, window, n_heads, batch;
  const void *q, *k, *v;
  long q_stride, k_stride, v_stride, out_stride;
  const int32_t *seqs, *in_pos, *axis_pos;
  void *q_out;
  int n_axes, rotate;
  int blocks_per_seq;   // blocks of 16 positions that a window can touch
  int heads_per_block;  // of the n_heads + 2 n_kv_heads heads, in turns of a warp each
  double turns[64];     // frequency of a pair over pi
  uint8_t axis[64];
};

// two neighbouring entries as floats
template <typename T> struct Pair;
template <> struct Pair<float> {
  typedef float2 raw;
  static __device__ __forceinline__ float2 get(raw r) { return r; }
  static __device__ __forceinline__ raw put(float a, float b) { return make_float2(a, b); }
};
template <> struct Pair<__nv_bfloat16> {
  typedef __nv_bfloat162 raw;
  static __device__ __forceinline__ float2 get(raw r) { return __bfloat1622float2(r); }
  static __device__ __forceinline__ raw put(float a, float b) { return __floats2bfloat162_rn(a, b); }
};

__device__ __forceinline__ uint16_t to_e4m3x2(float a, float b) {   // a in the low byte; NaN stays NaN, the rest saturates
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ float2 from_e4m3x2(uint16_t v) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(v));
  float2 f;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.f32.f16 %0, lo;\n\tcvt.f32.f16 %1, hi;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(h));
  return f;
}
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.0f;   // (NaN too)
}
__device__ __forceinline__ float scaled(float x, float s) { return fabsf(x) < INFINITY ? x * s : __int_as_float(0x7FFFFFFF); }

template <typename T, int HD>
__global__ void __launch_bounds__(kAppendThreads) pool_append_kernel(const AppendParams p) {
  constexpr int HALF = HD / 2;
  constexpr int LANES = HD / 4;              // lanes of a row: two pairs each
  constexpr int STEP = 32 / LANES;           // rows a warp works on at once
  constexpr int N = kPoolBlock / STEP;       // rows of a lane
  __shared__ float2 turn[kPoolBlock][HALF];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b = blockIdx.x / p.blocks_per_seq, j = blockIdx.x - b * p.blocks_per_seq;
  const int32_t *pos = p.in_pos + (long)b * p.window;
  const int start = pos[0];
  if (start >= p.pool.pages_per_seq * KV_PAGE) {   // (at most 2^26: the sums below stay in 32 bits)
    if (tid == 0) pool_fault(p.pool.status, SJD_ERR_BAD_ARG);
    return;
  }
  const int base = (start < 0 ? 0 : start / kPoolBlock * kPoolBlock) + j * kPoolBlock;
  // rows of the window in this block: k0 .. k1 - 1, of which the first n_new are active
  const int k0 = start < 0 ? j * kPoolBlock : max(0, base - start), k1 = min(p.window, start < 0 ? k0 + kPoolBlock : base + kPoolBlock - start);
  if (k0 >= k1) return;
  bool bad = false;
  int active = 0;
  if (tid < k1 - k0) {
    const int at = pos[k0 + tid];
    active = at >= 0;
    bad = at < -1 || (active && (start < 0 || at != start + k0 + tid));
    if (active && k0 + tid > 0 && pos[k0 + tid - 1] < 0) bad = true;   // a hole before an active row
  }
  int seq = p.seqs ? p.seqs[b] : b;
  if (seq < 0 || seq >= p.pool.n_seqs) bad = true;
  for (int i = tid; p.seqs && i < p.batch; i += kAppendThreads) bad |= i != b && p.seqs[i] == seq;
  const int n_new = __syncthreads_count(active);
  if (n_new > 0 && (long)base + kPoolBlock > (long)p.pool.pages_per_seq * KV_PAGE) bad = true;
  bad = __syncthreads_or(bad);
  int page = -1;
  if (!bad && n_new > 0) {
    page = p.pool.table[(long)seq * p.pool.pages_per_seq + base / KV_PAGE];
    bad = page < 0 || page >= p.pool.n_pages;
  }
  if (bad) {
    if (tid == 0) pool_fault(p.pool.status, SJD_ERR_BAD_ARG);
    return;
  }
  if (n_new == 0) return;
  const long m0 = (long)b * p.window + k0;      // first new row
  const int row0 = start + k0 - base;           // its place in the block; rows before it are kept

  const int h_begin = blockIdx.y * p.heads_per_block, h_all = p.n_heads + 2 * p.pool.n_kv_heads;
  const int h_end = min(h_all, h_begin + p.heads_per_block);
  if (p.rotate && h_begin < p.n_heads + p.pool.n_kv_heads) {
    for (int i = tid; i < n_new * HALF; i += kAppendThreads) {
      const int r = i / HALF, f = i % HALF;
      const int at = p.axis_pos ? p.axis_pos[(m0 + r) * p.n_axes + p.axis[f]] : start + k0 + r;
      double s, c;
      sincospi((double)at * p.turns[f], &s, &c);
      turn[r][f] = make_float2((float)c, (float)s);
    }
    __syncthreads();
  }

  typedef typename Pair<T>::raw raw;
  const int sub = lane / LANES, d = (lane % LANES) * 2;   // lane's row of a step, its first pair
  for (int h = h_begin + warp; h < h_end; h += kAppendWarps) {
    const bool is_q = h < p.n_heads, is_k = !is_q && h < p.n_heads + p.pool.n_kv_heads;
    const int kh = is_q ? h : is_k ? h - p.n_heads : h - p.n_heads - p.pool.n_kv_heads;
    const long stride = is_q ? p.q_stride : is_k ? p.k_stride : p.v_stride;
    const T *src = (const T *)(is_q ? p.q : is_k ? p.k : p.v) + m0 * stride + (long)kh * HD + d;
    raw ra[N], rb[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = i * STEP + sub;
      if (r < n_new) {
        ra[i] = *reinterpret_cast<const raw *>(src + r * stride);
        rb[i] = *reinterpret_cast<const raw *>(src + r * stride + HALF);
      }
    }
    float2 a[N], c[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = i * STEP + sub;
      a[i] = c[i] = make_float2(0.0f, 0.0f);
      if (r >= n_new) continue;
      const float2 x = Pair<T>::get(ra[i]), y = Pair<T>::get(rb[i]);
      if (p.rotate && (is_q || is_k)) {
        const float2 t0 = turn[r][d], t1 = turn[r][d + 1];
        a[i].x = __fsub_rn(__fmul_rn(x.x, t0.x), __fmul_rn(y.x, t0.y));
        a[i].y = __fsub_rn(__fmul_rn(x.y, t1.x), __fmul_rn(y.y, t1.y));
        c[i].x = __fadd_rn(__fmul_rn(y.x, t0.x), __fmul_rn(x.x, t0.y));
        c[i].y = __fadd_rn(__fmul_rn(y.y, t1.x), __fmul_rn(x.y, t1.y));
      } else {
        a[i] = x;
        c[i] = y;
      }
    }
    if (is_q) {
      T *dst = (T *)p.q_out + m0 * p.out_stride + (long)kh * HD + d;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = i * STEP + sub;
        if (r >= n_new) continue;
        *reinterpret_cast<raw *>(dst + r * p.out_stride) = Pair<T>::put(a[i].x, a[i].y);
        *reinterpret_cast<raw *>(dst + r * p.out_stride + HALF) = Pair<T>::put(c[i].x, c[i].y);
      }
      continue;
    }
    const long plane = (((long)page * p.pool.n_layers + p.layer) * 2 + (is_k ? 0 : 1)) * p.pool.n_kv_heads + kh;
    uint8_t *bytes = (uint8_t *)p.pool.pages + (plane * KV_PAGE + base % KV_PAGE) * HD + d;
    int8_t *exp_at = p.pool.exps + plane * kPoolBlocks + base % KV_PAGE / kPoolBlock;
    // rows that stay: at most 15, only in the window's first block
    float2 ka[N], kc[N];
    float top = 0.0f;
    if (row0 > 0) {
      const float s = two_to(pool_exp(*exp_at));
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = i * STEP + sub;
        ka[i] = kc[i] = make_float2(0.0f, 0.0f);
        if (r >= row0) continue;
        ka[i] = from_e4m3x2(*reinterpret_cast<const uint16_t *>(bytes + r * HD));
        kc[i] = from_e4m3x2(*reinterpret_cast<const uint16_t *>(bytes + r * HD + HALF));
        ka[i].x *= s, ka[i].y *= s, kc[i].x *= s, kc[i].y *= s;
        top = fmaxf(top, fmaxf(fmaxf(finite_abs(ka[i].x), finite_abs(ka[i].y)), fmaxf(finite_abs(kc[i].x), finite_abs(kc[i].y))));
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      top = fmaxf(top, fmaxf(fmaxf(finite_abs(a[i].x), finite_abs(a[i].y)), fmaxf(finite_abs(c[i].x), finite_abs(c[i].y))));
    top = warp_max(top);
    // top = f 2^e, 1/2 <= f < 1: the smallest power of two that brings it to 448 = 7/8 2^9 at most
    int e = 0;
    if (top > 0.0f) {
      const float f = frexpf(top, &e);
      e = pool_exp(e - 9 + (f > 0.875f));
    }
    const float inv = two_to(-e);
    auto put = [&](int r, float2 x, float2 y) {
      *reinterpret_cast<uint16_t *>(bytes + r * HD) = to_e4m3x2(scaled(x.x, inv), scaled(x.y, inv));
      *reinterpret_cast<uint16_t *>(bytes + r * HD + HALF) = to_e4m3x2(scaled(y.x, inv), scaled(y.y, inv));
    };
    if (row0 > 0) {
      __syncwarp();   // (every lane has read the exponent)
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i * STEP + sub < row0) put(i * STEP + sub, ka[i], kc[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i * STEP + sub < n_new) put(row0 + i * STEP + sub, a[i], c[i]);
    if (lane == 0) *exp_at = (int8_t)e;
  }
}

}  // namespace
}  // namespace sjd

using namespace sjd;

extern "C" int sjd_pool_append(const sjd_pool *pool, int layer, int batch, int window, int n_heads, int dtype, const void *q,
                               int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride, const int32_t *seqs,
                               const int32_t *in_pos, const sjd_rope *rope, const int32_t *axis_pos, void *q_out, int64_t q_out_stride,
                               void *cuda_stream) {
  const int rc = check_pool(pool, false);
  if (rc != SJD_OK) return rc;
  if (dtype != SJD_F32 && dtype != SJD_BF16) return SJD_ERR_UNSUPPORTED;
  if (layer < 0 || layer >= pool->n_layers || batch < 1 || window < 1 || !k || !v || !in_pos || (q && (n_heads < 1 || !q_out)))
    return SJD_ERR_BAD_ARG;
  if ((int64_t)batch * window > 0x7FFFFFFF) return SJD_ERR_CAPACITY;
  const int hd = pool->head_dim;
  const int64_t kv_row = (int64_t)pool->n_kv_heads * hd, q_row = q ? (int64_t)n_heads * hd : 0;
  if (k_stride < kv_row || v_stride < kv_row || (q && (q_stride < q_row || q_out_stride < q_row))) return SJD_ERR_BAD_ARG;
  if (((k_stride | v_stride) & 1) || (q && ((q_stride | q_out_stride) & 1))) return SJD_ERR_BAD_ARG;
  const uintptr_t align = dtype == SJD_F32 ? 7 : 3;
  if ((((uintptr_t)k | (uintptr_t)v | (q ? (uintptr_t)q | (uintptr_t)q_out : 0)) & align) != 0) return SJD_ERR_BAD_ARG;
  AppendParams p;
  memset(&p, 0, sizeof(p));
  p.pool = *pool;
  p.layer = layer;
  p.batch = batch;
  p.window = window;
  p.n_heads = q ? n_heads : 0;
  p.q = q;
  p.k = k;
  p.v = v;
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.out_stride = q_out_stride;
  p.seqs = seqs;
  p.in_pos = in_pos;
  p.axis_pos = axis_pos;
  p.q_out = q_out;
  if (rope) {
    if (rope->n_axes < 1 || rope->n_axes > 3 || !(rope->theta > 0.0) || rope->theta > 1e300) return SJD_ERR_BAD_ARG;
    int left[3] = {0, 0, 0}, sum = 0;
    for (int a = 0; a < rope->n_axes; ++a) {
      if (rope->pairs[a] < 0 || rope->pairs[a] > hd / 2) return SJD_ERR_BAD_ARG;
      sum += left[a] = rope->pairs[a];
    }
    if (sum != hd / 2) return SJD_ERR_BAD_ARG;
    p.rotate = 1;
    p.n_axes = rope->n_axes;
    for (int i = 0, a = 0; i < hd / 2; ++i) {
      while (left[a] == 0) a = (a + 1) % rope->n_axes;   // (some axis has pairs left: they add up to hd / 2)
      p.axis[i] = (uint8_t)a;
      const int own = rope->pairs[a] - left[a]--;
      const double f = rope->per_axis ? (double)own / rope->pairs[a] : 2.0 * i / hd;
      p.turns[i] = pow(rope->theta, -f) / 3.14159265358979323846;
      if (rope->interleaved) a = (a + 1) % rope->n_axes;
    }
  }
  int dev = 0, sms = 0;
  SJD_CUDA(cudaGetDevice(&dev));
  SJD_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  p.blocks_per_seq = (window + kPoolBlock - 2) / kPoolBlock + 1;
  const int heads = p.n_heads + 2 * pool->n_kv_heads;
  const long blocks = (long)batch * p.blocks_per_seq;
  if (blocks > 0x7FFFFFFF) return SJD_ERR_CAPACITY;
  // a warp takes one head as long as that does not fill the device a few times over: the angles are computed once for a block's heads
  int turns = 1;
  while (turns < 8 && turns * kAppendWarps < heads && blocks * ((heads + turns * kAppendWarps - 1) / (turns * kAppendWarps)) > 8L * sms) ++turns;
  p.heads_per_block = turns * kAppendWarps;
  const dim3 grid((unsigned)blocks, (unsigned)((heads + p.heads_per_block - 1) / p.heads_per_block));
  if (grid.y > 65535) return SJD_ERR_CAPACITY;
  auto launch = [&](auto kernel) -> int {
    SJD_CUDA(launch_kernel(kernel, grid, dim3(kAppendThreads), 0, (cudaStream_t)cuda_stream, p));
    SJD_CHECK_LAUNCH();
    return SJD_OK;
  };
  if (dtype == SJD_F32) return hd == 128 ? launch(pool_append_kernel<float, 128>) : launch(pool_append_kernel<float, 64>);
  return hd == 128 ? launch(pool_append_kernel<__nv_bfloat16, 128>) : launch(pool_append_kernel<__nv_bfloat16, 64>);
}
