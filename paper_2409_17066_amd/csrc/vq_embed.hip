// Rows of an embedding table, scaled, into the residual stream: y[r] = scale * table[ids[r]].
//
// Memory bounds it: a row's elements are read and written once.  A lane takes what makes sixteen bytes of the result, next to those of the lanes beside it, and asks for four of its
// pieces of a row before it writes the first.
// Measured: 8192 rows of 8192 (5700 different ones) from a table of 32000 into 32 bits 70 us, 5.7 TB/s of rows read and written; 58 where the same rows are read again, which the caches hold then; whether
// the result is a new tensor makes no difference.  Stores of 32 bytes a lane, piece after piece, took 92 (the same rows again).  16 rows of 4096 2.6 us in a graph, of which an empty launch is 2.
#include "vq_kv.hpp"

namespace vq {

namespace {

constexpr int THREADS = 256, AHEAD = 4;

// What a lane takes of a row.
template <typename Stream>
struct Piece;
template <>
struct Piece<float> {
  static constexpr int ELEMENTS = 4;
  typedef unsigned Words __attribute__((ext_vector_type(2), aligned(2)));
  typedef float Out __attribute__((ext_vector_type(4), aligned(4)));
  static __device__ __forceinline__ Out scaled(Words w, float scale) {
    const half2v a = half2_of(w.x), b = half2_of(w.y);
    return Out{(float)a.x * scale, (float)a.y * scale, (float)b.x * scale, (float)b.y * scale};
  }
};
template <>
struct Piece<__half> {
  static constexpr int ELEMENTS = 8;
  typedef uint4b Words;
  typedef uint4b Out;
  static __device__ __forceinline__ unsigned two(unsigned w, float scale) {
    const half2v a = half2_of(w);
    return __builtin_bit_cast(unsigned, half2v{(_Float16)((float)a.x * scale), (_Float16)((float)a.y * scale)});
  }
  static __device__ __forceinline__ Out scaled(Words w, float scale) { return Out{two(w.x, scale), two(w.y, scale), two(w.z, scale), two(w.w, scale)}; }
};
__device__ __forceinline__ void store1(float *to, float e) { *to = e; }
__device__ __forceinline__ void store1(__half *to, float e) { *to = __float2half_rn(e); }

// 2^shift threads to a row, the workgroup's rows next to each other.  ONCE: written past the caches.
template <typename Stream, bool ONCE>
__global__ __launch_bounds__(THREADS) void embed_kernel(const int *ids, int rows, const __half *table, long long ld, int vocabulary, int width, float scale, Stream *y,
                                                        long long ldy, int shift) {
  typedef Piece<Stream> P;
  constexpr int N = P::ELEMENTS;
  const long long row = (long long)blockIdx.x * (THREADS >> shift) + (threadIdx.x >> shift);
  if (row >= rows) return;
  const int id = ids[row], step = N << shift;
  const bool there = (unsigned)id < (unsigned)vocabulary;
  const __half *from = table + (there ? id : 0) * ld;
  Stream *to = y + row * ldy;
  auto read = [&](int i) { return *reinterpret_cast<const typename P::Words *>(from + i); };
  auto write = [&](int i, typename P::Words w) {
    // (stored here, where the type says how little its address may be aligned: a template's argument would be the type without)
    typename P::Out *at = reinterpret_cast<typename P::Out *>(to + i), x = there ? P::scaled(w, scale) : typename P::Out{0, 0, 0, 0};
    if (ONCE) __builtin_nontemporal_store(x, at);
    else *at = x;
  };
  int i = (int)(threadIdx.x & ((1 << shift) - 1)) * N;
  for (; i + (AHEAD - 1) * step + N <= width; i += AHEAD * step) {
    const typename P::Words a = read(i), b = read(i + step), c = read(i + 2 * step), d = read(i + 3 * step);
    write(i, a);
    write(i + step, b);
    write(i + 2 * step, c);
    write(i + 3 * step, d);
  }
  for (; i + N <= width; i += step) write(i, read(i));
  for (int j = i; j < width && j < i + N; ++j) store1(to + j, there ? __half2float(from[j]) * scale : 0.f);
}

// Results of so many bytes are written past the caches: what reads them next finds nothing of them there in either case.  (us alone and with the residual norm behind it, rows of 8192 in 32
// bits, through the caches and past them: 8192 rows, 268 MB, 73 and 203, 59 and 202; 4096 rows 39 and 91, 29 and 100; 1024 rows 9.1 and 24.7, 8.5 and 26.6.)
constexpr long long ONCE_FROM = 192ll << 20;

template <typename Stream>
int launch(const int *ids, int rows, const __half *table, long long ld, int vocabulary, int width, float scale, Stream *y, long long ldy, hipStream_t s) {
  int shift = 0;
  while (shift < 8 && (Piece<Stream>::ELEMENTS << shift) < width) ++shift;
  const int each = THREADS >> shift;
  constexpr int MOST = 1 << 21;                                     // workgroups of a launch
  auto kernel = (long long)rows * width * (long long)sizeof(Stream) >= ONCE_FROM ? embed_kernel<Stream, true> : embed_kernel<Stream, false>;
  for (long long row0 = 0; row0 < rows; row0 += (long long)MOST * each) {
    const long long left = rows - row0, blocks = (left + each - 1) / each;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(blocks < MOST ? blocks : MOST)), dim3(THREADS), 0, s, ids + row0, (int)left, table, ld, vocabulary, width, scale, y + row0 * ldy, ldy, shift);
  }
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace

int launch_embed(const int *ids, int rows, const __half *table, long long ld, int vocabulary, int width, float scale, bool stream32, void *y, long long ldy, hipStream_t s) {
  return stream32 ? launch(ids, rows, table, ld, vocabulary, width, scale, static_cast<float *>(y), ldy, s)
                  : launch(ids, rows, table, ld, vocabulary, width, scale, static_cast<__half *>(y), ldy, s);
}

}  // namespace vq
