// New keys and values into a paged cache, and the rotation of queries and keys by their positions on the way.
//
// One launch.  A team of one, two or four waves takes one page, head and matrix (keys or values) that a sequence's new tokens reach, other waves take a head
// of some queries.  A lane takes eight elements of four tokens at a time: memory bounds it, and with fewer bytes on their way in each wave the chain from lengths to
// page table to elements to scale does.  Every element is read once, rotated in binary32 and written once; in 8 bits the page's scale has to be known
// before the first code is, so a lane keeps its first four tokens in registers between the two, and reads what large pages hold beyond that again (from L2).
#include "vq_kv.hpp"

namespace vq {

namespace {

constexpr int WAVES = 4, WAVE_LDS = 4096;

struct AppendParams {
  KvParams c;
  const __half *k, *v, *q;
  long long ldk, ldv, ldq, ldq_out;
  __half *q_out;
  int q_heads, slots, team;                   // pages a sequence can reach; waves of a team
  int kv_blocks, q_tiles;                     // workgroups for keys and values; waves for one head of a sequence's queries
  int columns, groups, tokens;                // lanes of a token, groups of four tokens of a wave, tokens of a wave at a time
  Rotary r;
};

struct Eight {
  float e[8];
};
typedef float float4b __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ Eight widened(uint4v u) {
  const half2v a = half2_of(u.x), b = half2_of(u.y), c = half2_of(u.z), d = half2_of(u.w);
  return Eight{{(float)a.x, (float)a.y, (float)b.x, (float)b.y, (float)c.x, (float)c.y, (float)d.x, (float)d.y}};
}

// Elements [d, d + 8) of one head of one token, rotated.  d is a multiple of 8, rotary.dim is even.  EIGHTS: pairs lie half of rotary.dim apart, and
// eight elements have their partners in eight others.
template <bool EIGHTS>
__device__ __forceinline__ Eight rotated(const __half *x, int d, const Rotary &r, int at, Eight y) {
  if (d >= r.dim) return y;
  const long long row = (long long)at * r.ld;
  float (&e)[8] = y.e;
  const int half = r.dim / 2;
  if constexpr (EIGHTS) {
    const bool second = d >= half;
    const int j = second ? d - half : d;
    const Eight p = widened(*reinterpret_cast<const uint4b *>(x + (second ? j : d + half)));
    const float4v c0 = *reinterpret_cast<const float4b *>(r.cos + row + j), c1 = *reinterpret_cast<const float4b *>(r.cos + row + j + 4);
    const float4v s0 = *reinterpret_cast<const float4b *>(r.sin + row + j), s1 = *reinterpret_cast<const float4b *>(r.sin + row + j + 4);
    const float c[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w}, s[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float far = p.e[i] * s[i];
      e[i] = second ? e[i] * c[i] + far : e[i] * c[i] - far;
    }
  } else if (r.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (d + 2 * i >= r.dim) break;
      const float c = r.cos[row + d / 2 + i], s = r.sin[row + d / 2 + i], a = e[2 * i], b = e[2 * i + 1];
      e[2 * i] = a * c - b * s;
      e[2 * i + 1] = b * c + a * s;
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
  return y;
}

__device__ __forceinline__ float largest(const Eight &x, float so_far) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = __builtin_fabsf(x.e[i]);
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
__device__ __forceinline__ uint4v halves8(const Eight &x) {
  return uint4v{packed(x.e[0], x.e[1]), packed(x.e[2], x.e[3]), packed(x.e[4], x.e[5]), packed(x.e[6], x.e[7])};
}

// What the lanes of a wave take: column `d` of tokens 4 group ... 4 group + 3 of every `tokens` tokens (lanes left over: none).
struct Place {
  int d, group;
  bool lane;
};
__device__ __forceinline__ Place place_of(const AppendParams &p) {
  const int lane = (int)threadIdx.x & 63, group = lane / p.columns;
  return Place{(lane - group * p.columns) * 8, group, group < p.groups};
}

// Four tokens' elements: rows row0 + t ... of x, where t < end (and t >= begin), rotated if `turn`.
template <bool EIGHTS>
__device__ __forceinline__ void take(const Rotary &r, const __half *x, long long ld, int row0, int place0, int d, int t, int begin, int end, bool turn,
                                     Eight (&y)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (EIGHTS && k == 2) __builtin_amdgcn_sched_barrier(0);          // (two tokens' operands at a time: registers)
    y[k] = Eight{};
    if (t + k < begin || t + k >= end) continue;
    const __half *from = x + (row0 + t + k) * ld;
    y[k] = widened(*reinterpret_cast<const uint4b *>(from + d));
    if (turn) y[k] = rotated<EIGHTS>(from, d, r, min(max(r.position ? r.position[row0 + t + k] : place0 + t + k, 0), r.positions - 1), y[k]);
  }
}

template <bool EIGHTS>
__device__ __forceinline__ void append_queries(const AppendParams &p, int wave) {
  const int head = wave % p.q_heads, tile = wave / p.q_heads % p.q_tiles, b = wave / p.q_heads / p.q_tiles;
  if (b >= p.c.n_seqs) return;
  const Sequence s = sequence(p.c, b);
  const Place at = place_of(p);
  const int t = tile * p.tokens + at.group * 4;
  if (!at.lane || t >= s.rows) return;
  Eight y[4];
  const long long from = (long long)head * p.c.head_dim;
  take<EIGHTS>(p.r, p.q + from, p.ldq, s.row0, s.first, at.d, t, 0, s.rows, p.r.cos != nullptr, y);
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (t + k < s.rows) *reinterpret_cast<uint4b *>(p.q_out + (s.row0 + t + k) * p.ldq_out + from + at.d) = halves8(y[k]);
}

template <bool E4M3, bool EIGHTS>
__global__ __launch_bounds__(64 * WAVES, EIGHTS ? 4 : 2) void kv_append_kernel(const AppendParams p) {
  __shared__ float wave_max[WAVES];
  __shared__ __attribute__((aligned(16))) unsigned char tiles[WAVES][WAVE_LDS];
  const KvParams &c = p.c;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  if ((int)blockIdx.x >= p.kv_blocks) return append_queries<EIGHTS>(p, ((int)blockIdx.x - p.kv_blocks) * WAVES + wave);
  const int in_team = wave & (p.team - 1);
  int unit = ((int)blockIdx.x * WAVES + wave) / p.team;
  const bool values = unit & 1;
  unit >>= 1;
  const int head = unit % c.kv_heads, slot = unit / c.kv_heads % p.slots, b = unit / c.kv_heads / p.slots;
  if (b >= c.n_seqs) return;
  const Sequence s = sequence(c, b);
  const int size = 1 << c.page_shift, d_all = c.head_dim;
  const int first = max(s.first, 0), last = min(s.first + s.rows, s.end);       // places [first, last) are written
  const int block = (first >> c.page_shift) + slot;
  if (first >= last || block > (last - 1) >> c.page_shift) return;
  const int page = page_of(c, b, block);
  const int place0 = block << c.page_shift;
  const int begin = max(first - place0, 0), end = min(last - place0, size);     // tokens of the page
  const int row0 = s.row0 + place0 - s.first;                                   // row of the page's token 0
  const __half *x = (values ? p.v : p.k) + (long long)head * d_all;
  const long long ld = values ? p.ldv : p.ldk;
  const bool turn = !values && p.r.cos;
  constexpr int bytes = E4M3 ? 1 : 2;
  const Place at = place_of(p);
  // this wave's tokens: [t, t + 4) of the lane, every p.tokens * p.team
  const int stride = p.tokens * p.team, start = (begin & -stride) + in_team * p.tokens;
  const int lane_end = at.lane ? end : 0;
  Eight held[4];
  take<EIGHTS>(p.r, x, ld, row0, place0, at.d, start + at.group * 4, begin, lane_end, turn, held);
  if (page < 0) return;                                                          // (the elements are on their way beside the page's number)
  unsigned char *to = (values ? c.v_pages + page * c.v_page_bytes : c.k_pages + page * c.k_page_bytes) + (long long)head * size * d_all * bytes;
  float *scale_at = (values ? c.v_scales : c.k_scales) + (E4M3 ? (long long)page * c.kv_heads + head : 0);
  const float before = E4M3 && begin > 0 ? *scale_at : 0.f;
  float inverse = 1.f;
  if (E4M3) {
    float amax = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) amax = largest(held[k], amax);
    for (int t0 = start + stride; t0 < end; t0 += stride) {
      Eight y[4];
      take<EIGHTS>(p.r, x, ld, row0, place0, at.d, t0 + at.group * 4, begin, lane_end, turn, y);
#pragma unroll
      for (int k = 0; k < 4; ++k) amax = largest(y[k], amax);
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) amax = fmaxf(amax, __shfl_xor(amax, m));
    if (p.team > 1) {
      if (lane == 0) wave_max[wave] = amax;
      __syncthreads();
      for (int w = 0; w < p.team; ++w) amax = fmaxf(amax, wave_max[wave - in_team + w]);
    }
    const float scale = fmaxf(scale_for(amax), before);
    inverse = 1.f / scale;
    if (begin > 0 && scale > before) {                                  // what the page holds already, in the new scale
      const float ratio = before * inverse;
      const int me = in_team * 64 + lane, all = p.team * 64;
      if (values) {
        for (int u = me; u < d_all * begin; u += all) {
          unsigned char *code = to + (u / begin) * size + u % begin;
          *code = (unsigned char)recoded(*code, ratio);
        }
      } else {
        for (int u = me; u < begin * (d_all / 16); u += all) {
          uint4v *code = reinterpret_cast<uint4v *>(to) + u;
          const uint4v w = *code;
          *code = uint4v{recoded(w.x, ratio), recoded(w.y, ratio), recoded(w.z, ratio), recoded(w.w, ratio)};
        }
      }
    }
    if (in_team == 0 && lane == 0 && !(begin > 0 && scale == before)) *scale_at = scale;
  }
  for (int t0 = start; t0 < end; t0 += stride) {
    const int t = t0 + at.group * 4;
    if (t0 != start) take<EIGHTS>(p.r, x, ld, row0, place0, at.d, t, begin, lane_end, turn, held);
    unsigned code[4][2];                                                // a token's eight codes
    uint4v half[4];                                                     // or its halfs
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const Eight &y = held[k];
      if (E4M3) {
        code[k][0] = codes4(y.e[0] * inverse, y.e[1] * inverse, y.e[2] * inverse, y.e[3] * inverse);
        code[k][1] = codes4(y.e[4] * inverse, y.e[5] * inverse, y.e[6] * inverse, y.e[7] * inverse);
      } else {
        half[k] = halves8(y);
      }
    }
    if (!values) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (t + k < begin || t + k >= lane_end) continue;
        if (E4M3) *reinterpret_cast<uint2v *>(to + (t + k) * d_all + at.d) = uint2v{code[k][0], code[k][1]};
        else *reinterpret_cast<uint4v *>(to + ((t + k) * d_all + at.d) * 2) = half[k];
      }
      continue;
    }
    // Values, whose tokens lie next to each other in the cache.
    if (t0 < begin || t0 + p.tokens > end) {                            // some tokens of these: one by one
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (t + k < begin || t + k >= lane_end) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (E4M3) {
            to[(at.d + i) * size + t + k] = (unsigned char)(code[k][i >> 2] >> (8 * (i & 3)));
          } else {
            const unsigned w = i < 2 ? half[k].x : i < 4 ? half[k].y : i < 6 ? half[k].z : half[k].w;
            reinterpret_cast<unsigned short *>(to)[(at.d + i) * size + t + k] = (unsigned short)(w >> (16 * (i & 1)));
          }
        }
      }
      continue;
    }
    // All of them: through LDS, where element 8 column + i is row i * columns + column of `tokens` tokens (adjacent lanes write adjacent rows).
    unsigned char *tile = tiles[wave];
    const int row_bytes = p.tokens * bytes;
    if (at.lane) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        unsigned char *w = tile + (i * p.columns + (at.d >> 3)) * row_bytes + at.group * 4 * bytes;
        if (E4M3) {
          const int sh = 8 * (i & 3);
          *reinterpret_cast<unsigned *>(w) = (code[0][i >> 2] >> sh & 255) | (code[1][i >> 2] >> sh & 255) << 8 | (code[2][i >> 2] >> sh & 255) << 16 | (code[3][i >> 2] >> sh & 255) << 24;
        } else {
          unsigned h[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) h[k] = (i < 2 ? half[k].x : i < 4 ? half[k].y : i < 6 ? half[k].z : half[k].w) >> (16 * (i & 1)) & 0xffffu;
          *reinterpret_cast<uint2v *>(w) = uint2v{h[0] | h[1] << 16, h[2] | h[3] << 16};
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int pieces = row_bytes >= 16 ? row_bytes / 16 : 1, wide = row_bytes / pieces;      // of a row: 16 bytes, or the eight that it has
    for (int u = lane; u < d_all * pieces; u += 64) {
      const int d = u / pieces, i = u - d * pieces;
      const unsigned char *from = tile + ((d & 7) * p.columns + (d >> 3)) * row_bytes + i * wide;
      unsigned char *w = to + ((long long)d * size + t0) * bytes + i * wide;
      if (wide == 16) *reinterpret_cast<uint4v *>(w) = *reinterpret_cast<const uint4v *>(from);
      else *reinterpret_cast<uint2v *>(w) = *reinterpret_cast<const uint2v *>(from);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace

int launch_kv_append(const KvParams &c, const __half *k, long long ldk, const __half *v, long long ldv, const __half *q, long long ldq, int q_heads,
                     __half *q_out, long long ldq_out, const Rotary &r, hipStream_t s) {
  AppendParams p{c, k, v, q, ldk, ldv, ldq, ldq_out, q_out, q_heads, 0, 1, 0, 1, 0, 1, 0, r};
  const int size = 1 << c.page_shift;
  p.columns = c.head_dim / 8;
  while (p.groups * 2 * p.columns <= 64 && p.groups * 8 <= size) p.groups *= 2;
  p.tokens = 4 * p.groups;
  p.slots = (c.max_new + size - 2) / size + 1;
  // a wave to the tokens that it holds at a time, of those that a sequence can bring to a page
  const int most = c.max_new < size ? c.max_new : size;
  while (p.team < WAVES && p.team * p.tokens < most) p.team *= 2;
  const long long kv_blocks = (2LL * c.n_seqs * p.slots * c.kv_heads * p.team + WAVES - 1) / WAVES;
  p.q_tiles = (c.max_new + p.tokens - 1) / p.tokens;
  const long long q_waves = q ? (long long)c.n_seqs * p.q_tiles * q_heads : 0, blocks = kv_blocks + (q_waves + WAVES - 1) / WAVES;
  if (blocks > 0x7fffffff / WAVES) return VQ_ERR_SHAPE;
  p.kv_blocks = (int)kv_blocks;
  const bool eights = !r.cos || (!r.interleaved && r.dim % 16 == 0);
  auto kernel = c.e4m3 ? (eights ? kv_append_kernel<true, true> : kv_append_kernel<true, false>) : (eights ? kv_append_kernel<false, true> : kv_append_kernel<false, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * WAVES), 0, s, p);
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace vq
