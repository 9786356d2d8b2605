// New keys and values into a paged cache, and the rotation of queries and keys by their positions on the way.
//
// One launch.  A workgroup takes one page, head and matrix (keys or values) that a sequence's new tokens reach; others take queries, 256 threads
// of eight elements each.  Memory bounds it: every element is read once, rotated in binary32 and written once.  In 8 bits the page's scale has to be known
// before the first code is, so a workgroup holds its elements in registers between the two (small pages) or reads them again (from L1 or L2).
#include "vq_kv.hpp"

namespace vq {

namespace {

constexpr int THREADS = 256;

struct AppendParams {
  KvParams c;
  const __half *k, *v, *q;
  long long ldk, ldv, ldq, ldq_out;
  __half *q_out;
  int q_heads, slots, kv_blocks, q_tiles;     // pages a sequence can reach; workgroups for keys and values; for a sequence's queries
  Rotary r;
};

typedef float float8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float8 widened(uint4v u) {
  float8 x;
  half2v a = half2_of(u.x), b = half2_of(u.y), c = half2_of(u.z), d = half2_of(u.w);
  x.s0 = (float)a.x; x.s1 = (float)a.y; x.s2 = (float)b.x; x.s3 = (float)b.y;
  x.s4 = (float)c.x; x.s5 = (float)c.y; x.s6 = (float)d.x; x.s7 = (float)d.y;
  return x;
}

// Elements [d, d + 8) of one head of one token, rotated.  d is a multiple of 8, rotary.dim is even.
__device__ __forceinline__ float8 rotated(const __half *x, int d, const Rotary &r, int at, float8 own) {
  if (d >= r.dim) return own;
  const long long row = (long long)at * r.ld;
  float e[8] = {own.s0, own.s1, own.s2, own.s3, own.s4, own.s5, own.s6, own.s7};
  if (r.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (d + 2 * i >= r.dim) break;
      const float c = r.cos[row + d / 2 + i], s = r.sin[row + d / 2 + i], a = e[2 * i], b = e[2 * i + 1];
      e[2 * i] = a * c - b * s;
      e[2 * i + 1] = b * c + a * s;
    }
  } else {
    const int half = r.dim / 2;
    if ((half & 7) == 0) {                       // the eight elements have their partners in eight others
      const bool second = d >= half;
      const int j = second ? d - half : d;
      const float8 o = widened(*reinterpret_cast<const uint4b *>(x + (second ? j : d + half)));
      const float p[8] = {o.s0, o.s1, o.s2, o.s3, o.s4, o.s5, o.s6, o.s7};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float c = r.cos[row + j + i], s = r.sin[row + j + i], far = p[i] * s;
        e[i] = second ? e[i] * c + far : e[i] * c - far;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (d + i >= r.dim) break;
        const bool second = d + i >= half;
        const int j = second ? d + i - half : d + i;
        const float c = r.cos[row + j], s = r.sin[row + j], far = __half2float(x[second ? j : j + half]) * s;
        e[i] = second ? e[i] * c + far : e[i] * c - far;
      }
    }
  }
  return float8{e[0], e[1], e[2], e[3], e[4], e[5], e[6], e[7]};
}

__device__ __forceinline__ int rotary_row(const Rotary &r, int row, int place) {
  return min(max(r.position ? r.position[row] : place, 0), r.positions - 1);
}

__device__ __forceinline__ float largest(float8 x, float so_far) {
  const float e[8] = {x.s0, x.s1, x.s2, x.s3, x.s4, x.s5, x.s6, x.s7};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = __builtin_fabsf(e[i]);
    so_far = a <= 3.402823466e38f ? fmaxf(so_far, a) : so_far;       // (what is not finite does not take part)
  }
  return so_far;
}

// The smallest power of two S >= 2^-64 with amax <= 448 S: 448 is 1.75 * 2^8.
__device__ __forceinline__ float scale_for(float amax) {
  const unsigned u = __builtin_bit_cast(unsigned, amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __builtin_bit_cast(float, (unsigned)(max(e, -64) + 127) << 23);
}

__device__ __forceinline__ float encodable(float x) { return __builtin_fabsf(x) <= 448.f ? x : __builtin_nanf(""); }

__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(encodable(a), encodable(b), 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(encodable(c), encodable(d), w, true);
}

// Four codes times the power of two `ratio` (at most 1), as codes again.
__device__ __forceinline__ unsigned recoded(unsigned w, float ratio) {
  const float2v lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return codes4(lo.x * ratio, lo.y * ratio, hi.x * ratio, hi.y * ratio);
}

__device__ __forceinline__ unsigned packed(float a, float b) {
  return (unsigned)__half_as_ushort(__float2half_rn(a)) | ((unsigned)__half_as_ushort(__float2half_rn(b)) << 16);
}
__device__ __forceinline__ uint4v halves8(float8 x) { return uint4v{packed(x.s0, x.s1), packed(x.s2, x.s3), packed(x.s4, x.s5), packed(x.s6, x.s7)}; }

__device__ void append_queries(const AppendParams &p, int block) {
  const int b = block / p.q_tiles, tile = block - b * p.q_tiles;
  const Sequence s = sequence(p.c, b);
  const int per_head = p.c.head_dim / 8, per_row = per_head * p.q_heads;
  const int units = THREADS / per_head * per_head;                  // whole heads
  const int unit = tile * units + (int)threadIdx.x, t = unit / per_row;
  if ((int)threadIdx.x >= units || t >= s.rows) return;
  const int in_row = unit - t * per_row, head = in_row / per_head, d = (in_row - head * per_head) * 8;
  const int row = s.row0 + t;
  const __half *x = p.q + row * p.ldq + (long long)head * p.c.head_dim;
  const uint4v raw = *reinterpret_cast<const uint4b *>(x + d);
  const float8 y = rotated(x, d, p.r, rotary_row(p.r, row, s.first + t), widened(raw));
  __syncthreads();                                                  // in place: the elements' partners, of the same head, have been read
  *reinterpret_cast<uint4b *>(p.q_out + row * p.ldq_out + (long long)head * p.c.head_dim + d) = halves8(y);
}

__global__ __launch_bounds__(THREADS) void kv_append_kernel(const AppendParams p) {
  __shared__ float wave_max[THREADS / 64];
  extern __shared__ __attribute__((aligned(16))) unsigned char tile[];
  const KvParams &c = p.c;
  if ((int)blockIdx.x >= p.kv_blocks) return append_queries(p, (int)blockIdx.x - p.kv_blocks);
  int at = (int)blockIdx.x;
  const bool values = at & 1;
  at >>= 1;
  const int head = at % c.kv_heads, slot = at / c.kv_heads % p.slots, b = at / c.kv_heads / p.slots;
  const Sequence s = sequence(c, b);
  const int size = 1 << c.page_shift, d_all = c.head_dim;
  const int first = max(s.first, 0), last = min(s.first + s.rows, s.end);       // places [first, last) are written
  const int block = (first >> c.page_shift) + slot;
  if (first >= last || block > (last - 1) >> c.page_shift) return;
  const int page = page_of(c, b, block);
  if (page < 0) return;
  const int begin = max(first - (block << c.page_shift), 0), end = min(last - (block << c.page_shift), size);   // tokens of the page
  const int row0 = s.row0 + (block << c.page_shift) - s.first;                  // row of the page's token 0
  const int per_token = d_all / 8, units = (end - begin) * per_token;
  const __half *x = (values ? p.v : p.k) + (long long)head * d_all;
  const long long ld = values ? p.ldv : p.ldk;
  const bool turn = !values && p.r.cos;
  auto element = [&](int unit, int &t, int &d) {
    t = begin + unit / per_token;
    d = (unit % per_token) * 8;
    const int row = row0 + t;
    const __half *from = x + row * ld;
    const float8 own = widened(*reinterpret_cast<const uint4b *>(from + d));
    return turn ? rotated(from, d, p.r, rotary_row(p.r, row, (block << c.page_shift) + t), own) : own;
  };
  unsigned char *to = values ? c.v_pages + page * c.v_page_bytes : c.k_pages + page * c.k_page_bytes;
  const int bytes = c.e4m3 ? 1 : 2;
  to += (long long)head * size * d_all * bytes;
  float inverse = 1.f;
  if (c.e4m3) {
    float amax = 0.f;
    for (int u = threadIdx.x; u < units; u += THREADS) {
      int t, d;
      amax = largest(element(u, t, d), amax);
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) amax = fmaxf(amax, __shfl_xor(amax, m));
    if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = amax;
    float *slot_of_scale = (values ? c.v_scales : c.k_scales) + (long long)page * c.kv_heads + head;
    const float before = begin > 0 ? *slot_of_scale : 0.f;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) amax = fmaxf(amax, wave_max[w]);
    const float needed = scale_for(amax), scale = fmaxf(needed, before);
    inverse = 1.f / scale;
    if (begin > 0 && scale > before) {                                  // what the page holds already, in the new scale
      const float ratio = before * inverse;
      if (values) {
        for (int u = threadIdx.x; u < d_all * begin; u += THREADS) {
          unsigned char *code = to + (u / begin) * size + u % begin;
          *code = (unsigned char)recoded(*code, ratio);
        }
      } else {
        for (int u = threadIdx.x; u < begin * (d_all / 16); u += THREADS) {
          uint4v *code = reinterpret_cast<uint4v *>(to) + u;
          const uint4v w = *code;
          *code = uint4v{recoded(w.x, ratio), recoded(w.y, ratio), recoded(w.z, ratio), recoded(w.w, ratio)};
        }
      }
    }
    if (threadIdx.x == 0 && !(begin > 0 && scale == before)) *slot_of_scale = scale;
  }
  if (!values) {
    for (int u = threadIdx.x; u < units; u += THREADS) {
      int t, d;
      const float8 y = element(u, t, d);
      if (c.e4m3) {
        const uint2v w = {codes4(y.s0 * inverse, y.s1 * inverse, y.s2 * inverse, y.s3 * inverse), codes4(y.s4 * inverse, y.s5 * inverse, y.s6 * inverse, y.s7 * inverse)};
        *reinterpret_cast<uint2v *>(to + t * d_all + d) = w;
      } else {
        *reinterpret_cast<uint4v *>(to + (t * d_all + d) * 2) = halves8(y);
      }
    }
    return;
  }
  // Values, whose tokens lie next to each other: through LDS, 64 tokens at a time.
  const int step = min(size, 64);
  for (int t0 = begin & ~(step - 1); t0 < end; t0 += step) {
    const int from = max(begin, t0), till = min(end, t0 + step), here = (till - from) * per_token;
    __syncthreads();
    for (int u = threadIdx.x; u < here; u += THREADS) {
      int t, d;
      const float8 y = element(u + (from - begin) * per_token, t, d);
      const float e[8] = {y.s0, y.s1, y.s2, y.s3, y.s4, y.s5, y.s6, y.s7};
      if (c.e4m3) {
        const unsigned lo = codes4(e[0] * inverse, e[1] * inverse, e[2] * inverse, e[3] * inverse), hi = codes4(e[4] * inverse, e[5] * inverse, e[6] * inverse, e[7] * inverse);
#pragma unroll
        for (int i = 0; i < 8; ++i) tile[(d + i) * step + t - t0] = (unsigned char)((i < 4 ? lo : hi) >> (8 * (i & 3)));
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) reinterpret_cast<__half *>(tile)[(d + i) * step + t - t0] = __float2half_rn(e[i]);
      }
    }
    __syncthreads();
    if (till - from == step) {
      const int pieces = step * bytes / 16;                             // 16-byte pieces of a row of the tile
      for (int u = threadIdx.x; u < d_all * pieces; u += THREADS) {
        const int d = u / pieces, i = u - d * pieces;
        *reinterpret_cast<uint4v *>(to + (d * size + t0) * bytes + i * 16) = *reinterpret_cast<const uint4v *>(tile + d * step * bytes + i * 16);
      }
    } else {
      const int n = till - from;
      for (int u = threadIdx.x; u < d_all * n; u += THREADS) {
        const int d = u / n, t = from + u - d * n;
        if (c.e4m3) to[d * size + t] = tile[d * step + t - t0];
        else reinterpret_cast<__half *>(to)[d * size + t] = reinterpret_cast<const __half *>(tile)[d * step + t - t0];
      }
    }
  }
}

}  // namespace

int launch_kv_append(const KvParams &c, const __half *k, long long ldk, const __half *v, long long ldv, const __half *q, long long ldq, int q_heads,
                     __half *q_out, long long ldq_out, const Rotary &r, hipStream_t s) {
  AppendParams p{c, k, v, q, ldk, ldv, ldq, ldq_out, q_out, q_heads, 0, 0, 0, r};
  const int size = 1 << c.page_shift;
  p.slots = (c.max_new + size - 2) / size + 1;
  const long long kv_blocks = 2LL * c.n_seqs * p.slots * c.kv_heads;
  const int heads_at_once = THREADS / (c.head_dim / 8);
  p.q_tiles = q ? (int)(((long long)c.max_new * q_heads + heads_at_once - 1) / heads_at_once) : 0;
  const long long blocks = kv_blocks + (long long)c.n_seqs * p.q_tiles;
  if (blocks > 0x7fffffff) return VQ_ERR_SHAPE;
  p.kv_blocks = (int)kv_blocks;
  const int lds = c.head_dim * (size < 64 ? size : 64) * (c.e4m3 ? 1 : 2);
  hipLaunchKernelGGL(kv_append_kernel, dim3((unsigned)blocks), dim3(THREADS), lds, s, p);
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace vq
