// Residual sum and RMS norms between two blocks: y = x + scale * gate * post(h), z = norm(y) * w_pre, in one pass.
//
// A workgroup holds a row in registers, eight elements a vector and up to four vectors a thread, so that every element is read once and
// written once; memory bounds it from a few hundred rows on, the two reductions (one behind the other where there are both norms) and the launch below.
// Measured: 2048 rows of 8192, stream in 32 bits, both norms and a gate, 201 MB in 38.8 us, 5.2 TB/s (a large copy reaches 4.9); one row of 4096 2.5 us in a
// graph, of which an empty launch is 2, and 3.9 from the host, 5.2 where it allocates both results.
#include "vq_kv.hpp"

namespace vq {

namespace {

struct NormParams {
  const __half *h, *w_post, *gate, *w_pre;
  const void *x;
  void *y;
  __half *z;
  long long ldh, ldx, ldgate, ldy, ldz;
  float scale, eps;
  int width;
};

struct Eight {
  float e[8];
};

typedef float float4b __attribute__((ext_vector_type(4), aligned(4)));

// Elements [i, i + 8) of a row, zeros past its end.  ONCE: read past the caches, where what is read once would push out what the call writes
// for the next one (2048 x 8192, both norms, stream in 32 bits: 51.6 us with ordinary loads, 39.2 so).
template <bool ONCE>
__device__ __forceinline__ Eight load8(const __half *row, int i, int width) {
  Eight r;
  if (i + 8 <= width) {
    const uint4b *at = reinterpret_cast<const uint4b *>(row + i);
    const uint4v u = ONCE ? __builtin_nontemporal_load(at) : *at;
    const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const half2v v = half2_of(w[j]);
      r.e[2 * j] = (float)v.x;
      r.e[2 * j + 1] = (float)v.y;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) r.e[j] = i + j < width ? __half2float(row[i + j]) : 0.f;
  }
  return r;
}
template <bool ONCE>
__device__ __forceinline__ Eight load8(const float *row, int i, int width) {
  Eight r;
  if (i + 8 <= width) {
    const float4b *at = reinterpret_cast<const float4b *>(row + i);
    const float4v a = ONCE ? __builtin_nontemporal_load(at) : *at, b = ONCE ? __builtin_nontemporal_load(at + 1) : at[1];
    r.e[0] = a.x; r.e[1] = a.y; r.e[2] = a.z; r.e[3] = a.w;
    r.e[4] = b.x; r.e[5] = b.y; r.e[6] = b.z; r.e[7] = b.w;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) r.e[j] = i + j < width ? row[i + j] : 0.f;
  }
  return r;
}
__device__ __forceinline__ void store8(__half *row, int i, int width, const Eight &r) {
  if (i + 8 <= width) {
    unsigned w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = (unsigned)__half_as_ushort(__float2half_rn(r.e[2 * j])) | ((unsigned)__half_as_ushort(__float2half_rn(r.e[2 * j + 1])) << 16);
    *reinterpret_cast<uint4b *>(row + i) = uint4v{w[0], w[1], w[2], w[3]};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i + j < width) row[i + j] = __float2half_rn(r.e[j]);
  }
}
__device__ __forceinline__ void store8(float *row, int i, int width, const Eight &r) {
  if (i + 8 <= width) {
    *reinterpret_cast<float4b *>(row + i) = float4v{r.e[0], r.e[1], r.e[2], r.e[3]};
    *reinterpret_cast<float4b *>(row + i + 4) = float4v{r.e[4], r.e[5], r.e[6], r.e[7]};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i + j < width) row[i + j] = r.e[j];
  }
}

// Sum over the workgroup, in every thread; the order does not depend on anything but the workgroup's size.
__device__ __forceinline__ float block_sum(float x, float *waves) {
  x = wave_sum(x);
  if (blockDim.x == 64) return x;
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
  __syncthreads();
  const int n = (int)(blockDim.x >> 6);
  float s = 0.f;
  for (int w = 0; w < n; ++w) s += waves[w];
  return s;
}

template <typename Stream, int NV>
__global__ __launch_bounds__(1024) void residual_norm_kernel(const NormParams p) {
  __shared__ float sums[2][16];
  const long long row = blockIdx.x;
  const int stride = (int)blockDim.x * 8, i0 = (int)threadIdx.x * 8, width = p.width;
  const Stream *x = static_cast<const Stream *>(p.x) + row * p.ldx;
  // Rows of one vector a thread are few: what the reductions wait for counts, and the weights are asked for in front of them.
  constexpr bool EARLY = NV == 1;
  Eight w_pre{}, w_post{};
  if (EARLY && p.z) w_pre = load8<false>(p.w_pre, i0, width);
  if (EARLY && p.w_post) w_post = load8<false>(p.w_post, i0, width);
  Eight y[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) y[v] = load8<true>(x, i0 + v * stride, width);
  if (p.h) {
    const __half *h = p.h + row * p.ldh;
    Eight f[NV];
    float ss = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      f[v] = load8<true>(h, i0 + v * stride, width);
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = __fmaf_rn(f[v].e[j], f[v].e[j], ss);
    }
    float r = p.scale;
    if (p.w_post) {
      r = 1.f / __fsqrt_rn(block_sum(ss, sums[0]) / (float)width + p.eps);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const Eight w = EARLY ? w_post : load8<false>(p.w_post, i0 + v * stride, width);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[v].e[j] *= w.e[j];
      }
      r *= p.scale;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (p.gate) {
        const Eight g = load8<false>(p.gate + row * p.ldgate, i0 + v * stride, width);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[v].e[j] *= g.e[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) y[v].e[j] = __fmaf_rn(f[v].e[j], r, y[v].e[j]);
    }
  }
  if (p.y) {
    Stream *to = static_cast<Stream *>(p.y) + row * p.ldy;
#pragma unroll
    for (int v = 0; v < NV; ++v) store8(to, i0 + v * stride, width, y[v]);
  }
  if (!p.z) return;
  float ss = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) ss = __fmaf_rn(y[v].e[j], y[v].e[j], ss);
  const float r = 1.f / __fsqrt_rn(block_sum(ss, sums[1]) / (float)width + p.eps);
  __half *to = p.z + row * p.ldz;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Eight w = EARLY ? w_pre : load8<false>(p.w_pre, i0 + v * stride, width);
#pragma unroll
    for (int j = 0; j < 8; ++j) y[v].e[j] = y[v].e[j] * r * w.e[j];
    store8(to, i0 + v * stride, width, y[v]);
  }
}

template <typename Stream>
int launch(const NormParams &p, int rows, hipStream_t s) {
  // Where there are two workgroups for a compute unit or less, as many threads as a row has vectors; more rows have vectors enough on their way, and fewer waves
  // to wait for one another.  (us in a graph, by up to 256 threads and up to 1024: 1 row of 4096 3.0 and 2.5, of 8192 with both norms 5.2 and 3.6; 512 rows 13.9 and
  // 11.8; 1024 20.0 and 22.3; 2048 39.9 and 42.5, of 4096 12.5 and 14.2.)
  const int vectors = (p.width + 7) / 8, most = rows <= 2 * cu_count() ? 1024 : 256;
  int nv = 1;
  while (nv < 4 && (vectors + nv - 1) / nv > most) nv *= 2;
  const int threads = ((vectors + nv - 1) / nv + 63) / 64 * 64;
  auto kernel = nv == 1 ? residual_norm_kernel<Stream, 1> : nv == 2 ? residual_norm_kernel<Stream, 2> : residual_norm_kernel<Stream, 4>;
  constexpr int MOST = 1 << 21;                                     // rows of a launch (a grid has fewer than 2^32 threads)
  for (int row0 = 0; row0 < rows; row0 += MOST) {
    NormParams q = p;
    q.x = static_cast<const Stream *>(p.x) + row0 * p.ldx;
    if (p.h) q.h = p.h + row0 * p.ldh;
    if (p.gate) q.gate = p.gate + row0 * p.ldgate;
    if (p.y) q.y = static_cast<Stream *>(p.y) + row0 * p.ldy;
    if (p.z) q.z = p.z + row0 * p.ldz;
    hipLaunchKernelGGL(kernel, dim3(rows - row0 < MOST ? rows - row0 : MOST), dim3(threads), 0, s, q);
    if (rows - row0 <= MOST) break;
  }
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace

int launch_residual_norm(const __half *h, long long ldh, const void *x, long long ldx, const __half *w_post, const __half *gate, long long ldgate,
                         float scale, const __half *w_pre, float eps, bool stream32, int rows, int width, void *y, long long ldy, __half *z,
                         long long ldz, hipStream_t s) {
  const NormParams p{h, w_post, gate, w_pre, x, y, z, ldh, ldx, ldgate, ldy, ldz, scale, eps, width};
  return stream32 ? launch<float>(p, rows, s) : launch<__half>(p, rows, s);
}

}  // namespace vq
