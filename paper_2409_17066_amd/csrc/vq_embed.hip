// Rows of an embedding table, scaled, into the residual stream: y[r] = scale * table[ids[r]].
//
// Memory bounds it: a row's elements are read and written once, sixteen bytes a thread, and all of a thread's vectors of a row are asked for before the first is written.
#include "vq_kv.hpp"

namespace vq {

namespace {

typedef float float4b __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ void store8(float *to, const float (&e)[8]) {
  reinterpret_cast<float4b *>(to)[0] = float4v{e[0], e[1], e[2], e[3]};
  reinterpret_cast<float4b *>(to)[1] = float4v{e[4], e[5], e[6], e[7]};
}
__device__ __forceinline__ void store8(__half *to, const float (&e)[8]) {
  const half8v h = {(_Float16)e[0], (_Float16)e[1], (_Float16)e[2], (_Float16)e[3], (_Float16)e[4], (_Float16)e[5], (_Float16)e[6], (_Float16)e[7]};
  *reinterpret_cast<uint4b *>(to) = __builtin_bit_cast(uint4v, h);
}
__device__ __forceinline__ void store1(float *to, float e) { *to = e; }
__device__ __forceinline__ void store1(__half *to, float e) { *to = __float2half_rn(e); }

constexpr int THREADS = 256;

// 2^shift threads to a row, the workgroup's rows next to each other.
template <typename Stream>
__global__ __launch_bounds__(THREADS) void embed_kernel(const int *ids, int rows, const __half *table, long long ld, int vocabulary, int width, float scale, Stream *y,
                                                        long long ldy, int shift) {
  const long long row = (long long)blockIdx.x * (THREADS >> shift) + (threadIdx.x >> shift);
  if (row >= rows) return;
  const int id = ids[row], step = 8 << shift;
  const bool there = (unsigned)id < (unsigned)vocabulary;
  const __half *from = table + (there ? id : 0) * ld;
  Stream *to = y + row * ldy;
  for (int i = (int)(threadIdx.x & ((1 << shift) - 1)) * 8; i < width; i += step) {
    if (i + 8 <= width) {
      const half8v h = __builtin_bit_cast(half8v, (uint4v)*reinterpret_cast<const uint4b *>(from + i));
      float e[8] = {(float)h[0], (float)h[1], (float)h[2], (float)h[3], (float)h[4], (float)h[5], (float)h[6], (float)h[7]};
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = there ? e[j] * scale : 0.f;
      store8(to + i, e);
    } else {
      for (int j = i; j < width; ++j) store1(to + j, there ? __half2float(from[j]) * scale : 0.f);
    }
  }
}

template <typename Stream>
int launch(const int *ids, int rows, const __half *table, long long ld, int vocabulary, int width, float scale, Stream *y, long long ldy, hipStream_t s) {
  int shift = 0;
  while (shift < 8 && (8 << shift) < width) ++shift;
  const int each = THREADS >> shift;
  constexpr int MOST = 1 << 21;                                     // workgroups of a launch
  for (long long row0 = 0; row0 < rows; row0 += (long long)MOST * each) {
    const long long left = rows - row0, blocks = (left + each - 1) / each;
    hipLaunchKernelGGL(embed_kernel<Stream>, dim3((unsigned)(blocks < MOST ? blocks : MOST)), dim3(THREADS), 0, s, ids + row0, (int)left, table, ld, vocabulary, width, scale,
                       y + row0 * ldy, ldy, shift);
  }
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace

int launch_embed(const int *ids, int rows, const __half *table, long long ld, int vocabulary, int width, float scale, bool stream32, void *y, long long ldy, hipStream_t s) {
  return stream32 ? launch(ids, rows, table, ld, vocabulary, width, scale, static_cast<float *>(y), ldy, s)
                  : launch(ids, rows, table, ld, vocabulary, width, scale, static_cast<__half *>(y), ldy, s);
}

}  // namespace vq
