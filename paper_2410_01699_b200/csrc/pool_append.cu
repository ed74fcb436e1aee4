// Rotary step with several axes and append to the 8-bit paged cache.
//
// A block of threads owns a block of 16 positions of a sequence and some heads, a warp one head (of the queries, keys or values) at a time:
// it loads the head's rows, rotates them, reduces the largest entry, and stores 16 x head_dim bytes under one power-of-two scale.  Rows that
// were in the block before are read, scaled to what they stand for, and take part; nothing outside the block's rows up to the last
// new one is touched, so no two warps meet.  A lane holds four pairs (i, i + head_dim / 2) of half of the rows (64: a quarter), so that
// the rotation needs no exchange.
//   (a, b) -> (a c - b s, b c + a s), angle = position * theta^(-2 f / rot)
// Angles are products in 64 bits (a position of 10^6 times a frequency in 32 bits is off by 0.06), their cosine and sine are rounded to
// 32 bits once and shared by the heads of a block of threads through shared memory.  Products and sums are single 32-bit operations
// (no fused multiply-add), so that an entry next to a rounding border falls on the side that the formula says.
// Rounding: q to its own type, k and v to e4m3 (half a step is 2^-4 of an entry) under a scale that lets the largest entry reach
// 224 to 448; the scale itself is exact.
// Bound: bytes, one pass over q, k, v: 4224 rows of 32 + 2 x 8 heads, bf16, 95 MB, 23.1 us, 4.1 TB/s (the loads of a warp's next head
// wait for the stores of the one before; issued earlier they cost registers that spill: 22.9, and fp32, which spills 204 bytes with heads of
// 128 as it is, 45.7 -> 45.9); 8 windows of
// 32 rows of 32 + 2 x 32 heads, fp32, three axes, 18.9 MB, 9.4 us.  Two blocks a SM: one, which no register limit binds, takes 37.5 and 11.2.
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

// four neighbouring entries as floats
template <typename T> struct Four;
template <> struct Four<float> {
  typedef float4 raw;
  static __device__ __forceinline__ float4 get(raw r) { return r; }
  static __device__ __forceinline__ raw put(float4 v) { return v; }
};
template <> struct Four<__nv_bfloat16> {
  typedef uint2 raw;
  static __device__ __forceinline__ float4 get(raw r) {
    return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xFFFF0000u), __uint_as_float(r.y << 16), __uint_as_float(r.y & 0xFFFF0000u));
  }
  static __device__ __forceinline__ raw put(float4 v) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    return make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
  }
};

// four e4m3 numbers of a word, the first in the low byte; NaN stays NaN, the rest saturates
__device__ __forceinline__ uint32_t to_e4m3(float4 v) {
  uint32_t r;
  asm("{\n\t.reg .b16 a, b;\n\tcvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\tmov.b32 %0, {a, b};\n\t}"
      : "=r"(r)
      : "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w));
  return r;
}
__device__ __forceinline__ float4 from_e4m3(uint32_t v) {
  float4 f;
  asm("{\n\t.reg .b16 a, b, c, d;\n\t.reg .b32 x, y;\n\tmov.b32 {a, b}, %4;\n\tcvt.rn.f16x2.e4m3x2 x, a;\n\tcvt.rn.f16x2.e4m3x2 y, b;\n\t"
      "mov.b32 {a, b}, x;\n\tmov.b32 {c, d}, y;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\tcvt.f32.f16 %2, c;\n\tcvt.f32.f16 %3, d;\n\t}"
      : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w)
      : "r"(v));
  return f;
}
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.0f;   // (NaN too)
}
__device__ __forceinline__ float scaled(float x, float s) { return fabsf(x) < INFINITY ? x * s : __int_as_float(0x7FFFFFFF); }

__device__ __forceinline__ float4 scaled(float4 v, float s) { return make_float4(scaled(v.x, s), scaled(v.y, s), scaled(v.z, s), scaled(v.w, s)); }
__device__ __forceinline__ float finite_abs(float4 v) { return fmaxf(fmaxf(finite_abs(v.x), finite_abs(v.y)), fmaxf(finite_abs(v.z), finite_abs(v.w))); }

template <typename T, int HD>
__global__ void __launch_bounds__(kAppendThreads, 2) pool_append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int HALF = HD / 2;
  constexpr int LANES = HD / 8;              // lanes of a row: four pairs each
  constexpr int STEP = 32 / LANES;           // rows a warp works on at once
  constexpr int N = kPoolBlock / STEP;       // rows of a lane
  __shared__ alignas(16) float cosine[kPoolBlock][HALF], sine[kPoolBlock][HALF];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b = blockIdx.x / p.blocks_per_seq, j = blockIdx.x - b * p.blocks_per_seq;
  const int32_t *pos = p.in_pos + (long)b * p.window;
  const int seq = p.seqs ? p.seqs[b] : b;
  const int start = pos[0];
  if (start >= p.pool.pages_per_seq * KV_PAGE) {   // (at most 2^26: the sums below stay in 32 bits)
    if (tid == 0) pool_fault(p.pool.status, SJD_ERR_BAD_ARG);
    return;
  }
  const int base = (start < 0 ? 0 : start / kPoolBlock * kPoolBlock) + j * kPoolBlock;
  // rows of the window in this block: k0 .. k1 - 1, of which the first n_new are active
  const int k0 = start < 0 ? j * kPoolBlock : max(0, base - start), k1 = min(p.window, start < 0 ? k0 + kPoolBlock : base + kPoolBlock - start);
  if (k0 >= k1) return;
  bool bad = seq < 0 || seq >= p.pool.n_seqs;
  int page = -1;
  if (!bad && start >= 0 && base < p.pool.pages_per_seq * KV_PAGE) page = p.pool.table[(long)seq * p.pool.pages_per_seq + base / KV_PAGE];
  int active = 0;
  if (tid < k1 - k0) {
    const int at = pos[k0 + tid];
    active = at >= 0;
    bad |= at < -1 || (active && (start < 0 || at != start + k0 + tid));
    if (active && k0 + tid > 0 && pos[k0 + tid - 1] < 0) bad = true;   // a hole before an active row
  }
  for (int i = tid; p.seqs && i < p.batch; i += kAppendThreads) bad |= i != b && p.seqs[i] == seq;
  const int n_new = __syncthreads_count(active);
  bad |= n_new > 0 && (page < 0 || page >= p.pool.n_pages);
  if (__syncthreads_or(bad)) {
    if (tid == 0) pool_fault(p.pool.status, SJD_ERR_BAD_ARG);
    return;
  }
  if (n_new == 0) return;
  const long m0 = (long)b * p.window + k0;      // first new row
  const int row0 = start + k0 - base;           // its place in the block; rows before it are kept

  typedef typename Four<T>::raw raw;
  const int sub = lane / LANES, d = (lane % LANES) * 4;   // lane's row of a step, its first pair
  const int h_begin = blockIdx.y * p.heads_per_block, h_all = p.n_heads + 2 * p.pool.n_kv_heads;
  const int h_end = min(h_all, h_begin + p.heads_per_block);
  raw ra[N], rb[N];   // new rows as they are loaded
  auto load = [&](int h) {
    const bool is_q = h < p.n_heads, is_k = !is_q && h < p.n_heads + p.pool.n_kv_heads;
    const int kh = is_q ? h : is_k ? h - p.n_heads : h - p.n_heads - p.pool.n_kv_heads;
    const long stride = is_q ? p.q_stride : is_k ? p.k_stride : p.v_stride;
    const T *src = (const T *)(is_q ? p.q : is_k ? p.k : p.v) + (m0 - row0) * stride + (long)kh * HD + d;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = i * STEP + sub;
      if (r >= row0 && r < row0 + n_new) {
        ra[i] = *reinterpret_cast<const raw *>(src + r * stride);
        rb[i] = *reinterpret_cast<const raw *>(src + r * stride + HALF);
      }
    }
  };
  int h = h_begin + warp;
  if (h < h_end) load(h);   // (under way while the angles are computed)
  if (p.rotate && h_begin < p.n_heads + p.pool.n_kv_heads) {
    for (int i = tid; i < n_new * HALF; i += kAppendThreads) {
      const int r = i / HALF, f = i % HALF;
      const int at = p.axis_pos ? p.axis_pos[(m0 + r) * p.n_axes + p.axis[f]] : start + k0 + r;
      double s, c;
      sincospi((double)at * p.turns[f], &s, &c);
      cosine[row0 + r][f] = (float)c;
      sine[row0 + r][f] = (float)s;
    }
    __syncthreads();
  }

  for (; h < h_end; h += kAppendWarps) {
    const bool is_q = h < p.n_heads, is_k = !is_q && h < p.n_heads + p.pool.n_kv_heads;
    const int kh = is_q ? h : is_k ? h - p.n_heads : h - p.n_heads - p.pool.n_kv_heads;
    float4 a[N], c[N];   // rows of the block: new ones, and with keys and values those that stay
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = i * STEP + sub;
      a[i] = c[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (r < row0 || r >= row0 + n_new) continue;
      const float4 x = Four<T>::get(ra[i]), y = Four<T>::get(rb[i]);
      a[i] = x;
      c[i] = y;
      if (p.rotate && (is_q || is_k)) {
        const float4 cs = *reinterpret_cast<const float4 *>(&cosine[r][d]), sn = *reinterpret_cast<const float4 *>(&sine[r][d]);
        a[i].x = __fsub_rn(__fmul_rn(x.x, cs.x), __fmul_rn(y.x, sn.x));
        a[i].y = __fsub_rn(__fmul_rn(x.y, cs.y), __fmul_rn(y.y, sn.y));
        a[i].z = __fsub_rn(__fmul_rn(x.z, cs.z), __fmul_rn(y.z, sn.z));
        a[i].w = __fsub_rn(__fmul_rn(x.w, cs.w), __fmul_rn(y.w, sn.w));
        c[i].x = __fadd_rn(__fmul_rn(y.x, cs.x), __fmul_rn(x.x, sn.x));
        c[i].y = __fadd_rn(__fmul_rn(y.y, cs.y), __fmul_rn(x.y, sn.y));
        c[i].z = __fadd_rn(__fmul_rn(y.z, cs.z), __fmul_rn(x.z, sn.z));
        c[i].w = __fadd_rn(__fmul_rn(y.w, cs.w), __fmul_rn(x.w, sn.w));
      }
    }
    if (is_q) {
      T *dst = (T *)p.q_out + (m0 - row0) * p.out_stride + (long)kh * HD + d;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = i * STEP + sub;
        if (r < row0 || r >= row0 + n_new) continue;
        *reinterpret_cast<raw *>(dst + r * p.out_stride) = Four<T>::put(a[i]);
        *reinterpret_cast<raw *>(dst + r * p.out_stride + HALF) = Four<T>::put(c[i]);
      }
    } else {
      const long plane = (((long)page * p.pool.n_layers + p.layer) * 2 + (is_k ? 0 : 1)) * p.pool.n_kv_heads + kh;
      uint8_t *bytes = (uint8_t *)p.pool.pages + (plane * KV_PAGE + base % KV_PAGE) * HD + d;
      int8_t *exp_at = p.pool.exps + plane * kPoolBlocks + base % KV_PAGE / kPoolBlock;
      if (row0 > 0) {   // rows that stay: at most 15, only in the window's first block
        const float s = two_to(pool_exp(*exp_at));
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int r = i * STEP + sub;
          if (r >= row0) continue;
          a[i] = from_e4m3(*reinterpret_cast<const uint32_t *>(bytes + r * HD));
          c[i] = from_e4m3(*reinterpret_cast<const uint32_t *>(bytes + r * HD + HALF));
          a[i].x *= s, a[i].y *= s, a[i].z *= s, a[i].w *= s;
          c[i].x *= s, c[i].y *= s, c[i].z *= s, c[i].w *= s;
        }
        __syncwarp();   // (every lane has read the exponent)
      }
      float top = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) top = fmaxf(top, fmaxf(finite_abs(a[i]), finite_abs(c[i])));
      top = warp_max(top);
      // top = f 2^e, 1/2 <= f < 1: the smallest power of two that brings it to 448 = 7/8 2^9 at most
      int e = 0;
      if (top > 0.0f) {
        const float f = frexpf(top, &e);
        e = pool_exp(e - 9 + (f > 0.875f));
      }
      const float inv = two_to(-e);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = i * STEP + sub;
        if (r >= row0 + n_new) continue;
        *reinterpret_cast<uint32_t *>(bytes + r * HD) = to_e4m3(scaled(a[i], inv));
        *reinterpret_cast<uint32_t *>(bytes + r * HD + HALF) = to_e4m3(scaled(c[i], inv));
      }
      if (lane == 0) *exp_at = (int8_t)e;
    }
    if (h + kAppendWarps < h_end) load(h + kAppendWarps);
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
  if (((k_stride | v_stride) & 3) || (q && ((q_stride | q_out_stride) & 3))) return SJD_ERR_BAD_ARG;
  const uintptr_t align = dtype == SJD_F32 ? 15 : 7;
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
  // A warp takes one head while all blocks then find room at once (two on a SM), and more where they do not: the angles are computed once for a
  // block's heads, and no block waits for another.  4224 rows of 48 heads, bf16: 23.1 us (six heads a warp); with room for
  // four rounds of blocks, two heads a warp, 26.9; with eight rounds, one head, 29.0.
  int turns = 1;
  while (turns < 8 && turns * kAppendWarps < heads && blocks * ((heads + turns * kAppendWarps - 1) / (turns * kAppendWarps)) > 2L * sms) ++turns;
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
