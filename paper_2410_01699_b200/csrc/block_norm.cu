// The norm after a block, its gate, the residual and the norm before the next block, in one pass over the rows:
//   t = N(y) g1 + b1    h' = h + scale * gate * t    z = N(h') g2 + b2        N(x) = x / sqrt(mean(x^2) + eps), or of x - mean(x)
//
// A row is a block's (a warp's, up to 1024 entries): its entries stay in registers between the sums, which are in 32 bits; the mean goes
// off before the squares are summed (squares of the entries less the mean's square would lose what a large mean leaves of them).  z is
// taken of h' before that is rounded to its type.  A thread has N vectors of VEC entries, T threads apart.  A row's
// entries are read by the thread that writes them, before it does: that is why outputs may lie where inputs do.
//
// Few rows are bound by the launch and two or four round trips (256 rows of 4096, gate and residual: 10.6 us).  Many are bound by the bytes, and where
// a block has one row at a time, by what it waits for between fetching a row and writing it: those of block_norm_rows_kernel keep the
// next rows coming (16892 rows of 4096, layer norms, gate, bf16: 235 us with a row a block, 140 with two vectors a thread, 113 now,
// 86 are the bytes; RMS 100; residual stream in fp32, whose rows are fetched by halves of sectors, 185 to 195, RMS 169, and 129 by the bytes).
#include <algorithm>

#include "common.cuh"

namespace sjd {
namespace {

constexpr int kMaxD = 32768;
constexpr int kWarpRows = 4;   // rows of a block whose warps have one each

struct NormParams {
  const void *h, *y, *post_gain, *post_bias, *gate, *pre_gain, *pre_bias;
  void *h_out, *z;
  long h_stride, y_stride, h_out_stride, z_stride;
  int rows, d, layer, gate_rows, gate_tanh;
  int wide_h, wide_z;   // rows of h_out, of z start on 32 bytes (with vectors)
  float eps, scale, inv_d;
};

template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T *p, float *v) {
  if constexpr (VEC == 1) {
    v[0] = (float)*p;
  } else if constexpr (sizeof(T) == 4) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
// wide: p is a multiple of 32 bytes (two stores of half a sector each take 228 us instead of 195 where h is fp32)
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T *p, const float *v, bool wide) {
  if constexpr (VEC == 1) {
    *p = (T)v[0];   // (to the nearest)
  } else if constexpr (sizeof(T) == 4) {
    if (wide) {
      asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                   ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                   : "memory");
    } else {
      reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// Y: type of y, gains, biases, gate and z; H: of h and h_out.  ROW: threads of a row are the block (else a warp).
template <typename Y, typename H, int VEC, int N, bool ROW>
__global__ void __launch_bounds__(ROW ? 1024 : 32 * kWarpRows) block_norm_kernel(const __grid_constant__ NormParams p) {
  __shared__ float red[2][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int T = ROW ? blockDim.x : 32, t = ROW ? threadIdx.x : lane;
  const long row = ROW ? blockIdx.x : (long)blockIdx.x * kWarpRows + warp;
  pdl_wait();
  pdl_trigger();
  if (!ROW && row >= p.rows) return;
  int sums = 0;
  auto sum_of_row = [&](float v) {
    v = warp_sum(v);
    if constexpr (ROW) {
      float *r = red[sums++ & 1];   // (the one before may still be read)
      if (lane == 0) r[warp] = v;
      __syncthreads();
      v = warp_sum(lane < T >> 5 ? r[lane] : 0.0f);
    }
    return v;
  };
  auto at = [&](int i) { return (i * T + t) * VEC; };
  auto each = [&](auto f) {   // vectors that there are (d is a multiple of VEC)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (at(i) < p.d) f(i, at(i));
  };
  // x = N(x) gain + bias
  auto normalise = [&](float (&x)[N][VEC], const Y *gain, const Y *bias) {
    float mean = 0.0f;
    if (p.layer) {
      float s = 0.0f;
      each([&](int i, int) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) s += x[i][e];
      });
      mean = sum_of_row(s) * p.inv_d;
    }
    float s = 0.0f;
    each([&](int i, int) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        x[i][e] -= mean;
        s = fmaf(x[i][e], x[i][e], s);
      }
    });
    const float f = rsqrtf(fmaf(sum_of_row(s), p.inv_d, p.eps));
    each([&](int i, int k) {
      float g[VEC], b[VEC];
      load_vec<Y, VEC>(gain + k, g);
#pragma unroll
      for (int e = 0; e < VEC; ++e) b[e] = 0.0f;
      if (bias) load_vec<Y, VEC>(bias + k, b);
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[i][e] = fmaf(x[i][e] * f, g[e], b[e]);
    });
  };

  // With up to 16 entries a thread both loads are under way at once; with 32, h comes when it is needed (64 registers of 1024 threads).
  constexpr bool EARLY = N * VEC <= 16;
  float x[N][VEC], h[EARLY ? N : 1][VEC];
  const H *hp = (const H *)p.h + row * p.h_stride;
  if (p.y) {
    const Y *y = (const Y *)p.y + row * p.y_stride;
    each([&](int i, int k) { load_vec<Y, VEC>(y + k, x[i]); });
    if constexpr (EARLY) each([&](int i, int k) { load_vec<H, VEC>(hp + k, h[i]); });
    if (p.post_gain) normalise(x, (const Y *)p.post_gain, (const Y *)p.post_bias);
    const Y *gate = (const Y *)p.gate + (p.gate ? row / p.gate_rows * p.d : 0);
    each([&](int i, int k) {
      if (p.gate) {
        float g[VEC];
        load_vec<Y, VEC>(gate + k, g);
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[i][e] *= p.gate_tanh ? tanhf(g[e]) : g[e];
      }
      if constexpr (!EARLY) load_vec<H, VEC>(hp + k, h[0]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[i][e] = fmaf(p.scale, x[i][e], h[EARLY ? i : 0][e]);
      store_vec<H, VEC>((H *)p.h_out + row * p.h_out_stride + k, x[i], p.wide_h);
    });
  } else {
    each([&](int i, int k) { load_vec<H, VEC>(hp + k, x[i]); });
  }
  if (p.z) {
    normalise(x, (const Y *)p.pre_gain, (const Y *)p.pre_bias);
    each([&](int i, int k) { store_vec<Y, VEC>((Y *)p.z + row * p.z_stride + k, x[i], p.wide_z); });
  }
}

// ---- many rows: persistent blocks, the next row's entries on their way to shared memory
// A group of T threads has a row, four vectors of eight entries each thread (fewer entries, and what a warp does once a row, the sums
// and the root, is most of its instructions: 512 threads a row of 4096 took 235 us for what a block of 128 threads for each row did in 140).  Gains and biases
// stay in shared memory, the same for all groups of a block; a slot of a group is filled with the next row as soon as its thread has read it.
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
// Threads of a block: with 1024 (64 registers, 40 to 70 bytes laid aside) the case above takes 120 us, with 640 118, with 512 119.  With these nothing is laid aside where h is
// bf16, and 8 to 24 bytes where it is fp32.
constexpr int kN = 4, kMaxGroups = 32, kMaxWarps = 8, kRowsThreads = 768;

// 16 bytes to shared memory, and the groups of such copies of this thread
__device__ __forceinline__ void copy_async(void *dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// eight entries, as pairs, from the units of a vector `step` units apart
template <typename T>
__device__ __forceinline__ void load_pairs(const uint4 *from, int step, float2 *v) {
  if constexpr (sizeof(T) == 4) {
    const float4 a = *reinterpret_cast<const float4 *>(from), b = *reinterpret_cast<const float4 *>(from + step);
    v[0] = make_float2(a.x, a.y), v[1] = make_float2(a.z, a.w), v[2] = make_float2(b.x, b.y), v[3] = make_float2(b.z, b.w);
  } else {
    const uint4 a = *from;
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
  }
}

// FULL: a row has an entry for every thread's every vector
template <typename Y, typename H, bool FULL>
__global__ void __launch_bounds__(kRowsThreads, 1) block_norm_rows_kernel(const __grid_constant__ NormParams p, int T) {
  constexpr int YU = sizeof(Y) / 2, HU = sizeof(H) / 2;   // 16-byte units of a vector
  __shared__ alignas(16) float red[kMaxGroups][2][kMaxWarps];
  extern __shared__ __align__(16) uint4 shared[];   // gains [4][kN YU][T], slots [group][kN (YU + HU)][T]
  const int g = threadIdx.x / T, t = threadIdx.x - g * T, lane = threadIdx.x & 31, groups = blockDim.x / T, warps = T >> 5;
  uint4 *kept = shared + t, *slot = shared + (4 * kN * YU + g * kN * (YU + HU)) * T + t;
  pdl_wait();
  pdl_trigger();
  auto each = [&](auto f) {
#pragma unroll
    for (int i = 0; i < kN; ++i)
      if (FULL || (i * T + t) * 8 < p.d) f(i, (i * T + t) * 8);
  };
  auto fetch = [&](const void *base, auto type, long stride, long row, uint4 *to) {   // a row's vectors to the slot
    constexpr int U = sizeof(type) / 2;
    const uint4 *from = (const uint4 *)((const decltype(type) *)base + row * stride);
    if (row < p.rows)
      each([&](int i, int k) {
#pragma unroll
        for (int u = 0; u < U; ++u) copy_async(to + (i * U + u) * T, from + k / 8 * U + u);
      });
    copies_commit();
  };
  const long first = (long)blockIdx.x * groups + g, step = (long)gridDim.x * groups;
  uint4 *y_slot = slot, *h_slot = slot + kN * YU * T;
  if (p.y) fetch(p.y, Y(), p.y_stride, first, y_slot);
  fetch(p.h, H(), p.h_stride, first, h_slot);
  if (g == 0) {
    const void *from[4] = {p.post_gain, p.post_bias, p.pre_gain, p.pre_bias};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (from[j])
        each([&](int i, int k) {
#pragma unroll
          for (int u = 0; u < YU; ++u) kept[(j * kN * YU + i * YU + u) * T] = ((const uint4 *)from[j])[k / 8 * YU + u];
        });
  }
  __syncthreads();
  int sums = 0;
  auto sum_of_row = [&](float v) {
    v = warp_sum(v);
    if (warps > 1) {
      float *r = red[g][sums++ & 1];   // (the one before may still be read)
      if (lane == 0) r[t >> 5] = v;
      asm volatile("bar.sync %0, %1;" ::"r"(g), "r"(T) : "memory");
      v = r[0];
      for (int w = 1; w < warps; ++w) v += r[w];
    }
    return v;
  };
  auto normalise = [&](float2 (&x)[kN][4], int j, bool bias) {   // x = N(x) gain j + bias j + 1
    if (p.layer) {
      float2 s = make_float2(0.0f, 0.0f);
      each([&](int i, int) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s = add2(s, x[i][e]);
      });
      const float mean = sum_of_row(s.x + s.y) * p.inv_d;
      each([&](int i, int) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i][e] = add2(x[i][e], make_float2(-mean, -mean));
      });
    }
    float2 s = make_float2(0.0f, 0.0f);
    each([&](int i, int) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s = fma2(x[i][e], x[i][e], s);
    });
    const float f = rsqrtf(fmaf(sum_of_row(s.x + s.y), p.inv_d, p.eps));
    each([&](int i, int) {
      float2 w[4];
      load_pairs<Y>(kept + (j * kN * YU + i * YU) * T, T, w);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][e] = mul2(x[i][e], make_float2(f, f));
      if (bias) {
        float2 b[4];
        load_pairs<Y>(kept + ((j + 1) * kN * YU + i * YU) * T, T, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i][e] = fma2(x[i][e], w[e], b[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i][e] = mul2(x[i][e], w[e]);
      }
    });
  };
  for (long row = first; row < p.rows; row += step) {
    float2 x[kN][4];
    if (p.y) {
      copies_wait<1>();   // (h may be under way)
      each([&](int i, int) { load_pairs<Y>(y_slot + i * YU * T, T, x[i]); });
      fetch(p.y, Y(), p.y_stride, row + step, y_slot);
      if (p.post_gain) normalise(x, 0, p.post_bias);
      if (p.gate) {
        const Y *gate = (const Y *)p.gate + row / p.gate_rows * p.d;
        each([&](int i, int k) {
          float2 w[4];
          load_pairs<Y>((const uint4 *)(gate + k), 1, w);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[i][e] = mul2(x[i][e], p.gate_tanh ? make_float2(tanhf(w[e].x), tanhf(w[e].y)) : w[e]);
        });
      }
      copies_wait<1>();   // (y of the next row may be)
      each([&](int i, int k) {
        float2 h[4];
        load_pairs<H>(h_slot + i * HU * T, T, h);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i][e] = fma2(x[i][e], make_float2(p.scale, p.scale), h[e]);
        store_vec<H, 8>((H *)p.h_out + row * p.h_out_stride + k, &x[i][0].x, p.wide_h);
      });
    } else {
      copies_wait<0>();
      each([&](int i, int) { load_pairs<H>(h_slot + i * HU * T, T, x[i]); });
    }
    fetch(p.h, H(), p.h_stride, row + step, h_slot);
    if (p.z) {
      normalise(x, 2, p.pre_bias);
      each([&](int i, int k) { store_vec<Y, 8>((Y *)p.z + row * p.z_stride + k, &x[i][0].x, p.wide_z); });
    }
  }
  copies_wait<0>();
}

template <typename Y, typename H>
int launch_rows(const NormParams &p, int sms, cudaStream_t stream) {
  const int T = (p.d + kN * 256 - 1) / (kN * 256) * 32;
  const size_t kept = 4ull * kN * sizeof(Y) / 2 * 16 * T, slot = (size_t)kN * (sizeof(Y) + sizeof(H)) / 2 * 16 * T, most = 224 * 1024;   // (of 227 KB; the rest is static)
  const int groups = std::min(std::min(kRowsThreads / T, kMaxGroups), (int)((most - kept) / slot));
  auto launch = [&](auto kernel) -> int {
    const int rc = allow_smem(kernel, most);
    if (rc != SJD_OK) return rc;
    g_pdl = true;   // (waits for the launch before it itself)
    const cudaError_t e = launch_kernel(kernel, dim3((unsigned)std::min<long>(sms, (p.rows + groups - 1) / groups)), dim3(groups * T), kept + groups * slot, stream, p, T);
    g_pdl = false;
    SJD_CUDA(e);
    SJD_CHECK_LAUNCH();
    return SJD_OK;
  };
  return p.d == T * 8 * kN ? launch(block_norm_rows_kernel<Y, H, true>) : launch(block_norm_rows_kernel<Y, H, false>);
}

template <typename Y, typename H>
int launch_norm(const NormParams &p, bool vec, int sms, cudaStream_t stream) {
  auto launch = [&](auto kernel, int rows_of_block, int threads) -> int {
    g_pdl = true;   // (waits for the launch before it itself)
    const cudaError_t e = launch_kernel(kernel, dim3((unsigned)((p.rows + (long)rows_of_block - 1) / rows_of_block)), dim3(threads), 0, stream, p);
    g_pdl = false;
    SJD_CUDA(e);
    SJD_CHECK_LAUNCH();
    return SJD_OK;
  };
  auto threads = [&](int per_thread) { return (p.d + 32 * per_thread - 1) / (32 * per_thread) * 32; };
  if (vec && p.d <= kMaxWarps * 32 * 8 * kN && (long)p.rows * p.d > 4l * sms * 4096) return launch_rows<Y, H>(p, sms, stream);
  if (vec) {
    if (p.d <= 256) return launch(block_norm_kernel<Y, H, 8, 1, false>, kWarpRows, 32 * kWarpRows);
    if (p.d <= 512) return launch(block_norm_kernel<Y, H, 8, 2, false>, kWarpRows, 32 * kWarpRows);
    if (p.d <= 1024) return launch(block_norm_kernel<Y, H, 8, 4, false>, kWarpRows, 32 * kWarpRows);
    if (p.d <= 8192 && p.rows <= 512) return launch(block_norm_kernel<Y, H, 8, 1, true>, 1, threads(8));
    if (p.d <= 16384) return launch(block_norm_kernel<Y, H, 8, 2, true>, 1, threads(16));
    return launch(block_norm_kernel<Y, H, 8, 4, true>, 1, threads(32));
  }
  if (p.d <= 256) return launch(block_norm_kernel<Y, H, 1, 8, false>, kWarpRows, 32 * kWarpRows);
  if (p.d <= 8192) return launch(block_norm_kernel<Y, H, 1, 8, true>, 1, threads(8));
  return launch(block_norm_kernel<Y, H, 1, 32, true>, 1, threads(32));
}

}  // namespace
}  // namespace sjd

using namespace sjd;

extern "C" int sjd_block_norm(int rows, int d, int kind, float eps, int dtype, int h_dtype, const void *h, int64_t h_stride, const void *y,
                              int64_t y_stride, const void *post_gain, const void *post_bias, const void *gate, int gate_rows,
                              int gate_tanh, float scale, void *h_out, int64_t h_out_stride, const void *pre_gain, const void *pre_bias,
                              void *z, int64_t z_stride, void *cuda_stream) {
  if ((dtype != SJD_F32 && dtype != SJD_BF16) || (h_dtype != SJD_F32 && h_dtype != SJD_BF16)) return SJD_ERR_UNSUPPORTED;
  if (kind != SJD_NORM_RMS && kind != SJD_NORM_LAYER) return SJD_ERR_UNSUPPORTED;
  if (rows < 0 || d < 1 || !(eps >= 0.0f) || eps > 1e30f) return SJD_ERR_BAD_ARG;
  if (rows == 0 && d <= kMaxD) return SJD_OK;
  if (!h) return SJD_ERR_BAD_ARG;
  if (!y != !h_out || !pre_gain != !z || (!y && !z)) return SJD_ERR_BAD_ARG;
  if ((!y && (post_gain || gate)) || (post_bias && !post_gain) || (pre_bias && !pre_gain) || (gate && gate_rows < 1)) return SJD_ERR_BAD_ARG;
  if (h_stride < d || (y && (y_stride < d || h_out_stride < d)) || (z && z_stride < d)) return SJD_ERR_BAD_ARG;
  const int size = dtype == SJD_F32 ? 4 : 2, h_size = h_dtype == SJD_F32 ? 4 : 2;
  const uintptr_t of_y = (uintptr_t)y | (uintptr_t)post_gain | (uintptr_t)post_bias | (uintptr_t)gate | (uintptr_t)pre_gain | (uintptr_t)pre_bias | (uintptr_t)z;
  const uintptr_t of_h = (uintptr_t)h | (uintptr_t)h_out;
  if ((of_y & (size - 1)) != 0 || (of_h & (h_size - 1)) != 0) return SJD_ERR_BAD_ARG;
  if (d > kMaxD) return SJD_ERR_UNSUPPORTED;
  NormParams p;
  memset(&p, 0, sizeof(p));
  p.h = h, p.y = y, p.post_gain = post_gain, p.post_bias = post_bias, p.gate = gate, p.pre_gain = pre_gain, p.pre_bias = pre_bias;
  p.h_out = h_out, p.z = z;
  p.h_stride = h_stride, p.y_stride = y_stride, p.h_out_stride = h_out_stride, p.z_stride = z_stride;
  p.rows = rows, p.d = d, p.layer = kind == SJD_NORM_LAYER, p.gate_rows = gate_rows, p.gate_tanh = gate_tanh != 0;
  p.eps = eps, p.scale = scale, p.inv_d = 1.0f / (float)d;
  // vectors of eight entries where all rows start on 16 bytes
  const int64_t strides = (y ? y_stride | h_out_stride : 0) | (z ? z_stride : 0) | h_stride;
  const bool vec = d % 8 == 0 && (strides & 7) == 0 && ((of_y | of_h) & 15) == 0;
  p.wide_h = ((uintptr_t)h_out & 31) == 0, p.wide_z = ((uintptr_t)z & 31) == 0;
  int dev = 0, sms = 0;
  SJD_CUDA(cudaGetDevice(&dev));
  SJD_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (dtype == SJD_F32)
    return h_dtype == SJD_F32 ? launch_norm<float, float>(p, vec, sms, stream) : launch_norm<float, __nv_bfloat16>(p, vec, sms, stream);
  return h_dtype == SJD_F32 ? launch_norm<__nv_bfloat16, float>(p, vec, sms, stream) : launch_norm<__nv_bfloat16, __nv_bfloat16>(p, vec, sms, stream);
}
