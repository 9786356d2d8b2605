// New keys and values into a paged cache, and the rotation of queries and keys by their positions on the way.
//
// One launch.  A team of one, two or four waves takes one page, head and matrix (keys or values) that a sequence's new tokens reach, other waves take a head
// of some queries.  Memory bounds long prompts (four users' of 2624 tokens of 32 + 32 + 32 heads of 128 elements, 8 bits: 115 MB in 25.4 us, 4.5 TB/s, where a
// large copy reaches 4.9), below that the chain from lengths to page table to elements to scale (one token: 4.2 us, of which an empty launch is half).  Every
// element is read once, rotated in binary32 and written once; in 8 bits the page's scale has to be known
// before the first code is, so a lane keeps its tokens in registers between the two; of pages that hold more than a team's lanes it reads them again (from L2).
// A lane takes 32 elements at a time: of two tokens eight elements and the eight half a head further on, so that what it rotates are pairs and a token's
// cosines and sines are read once for both (half the loads through L1 of one half each: those prompts 40 -> 31 us), or, where the rotation pairs
// other elements, eight elements of four tokens.  Conversions that scale, and maxima of three at a time: 31 -> 29; 66 registers, and so seven
// waves a SIMD, by not keeping addresses from round to round: 29 -> 25.
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
  int columns, by_columns, groups, tokens;    // lanes of a token (and 2^16 over them, rounded up), groups of tokens of a wave, tokens of a wave at a time
  Rotary r;
};

struct Eight {
  float e[8];
};
typedef short short2v __attribute__((ext_vector_type(2)));
typedef float float4b __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ Eight widened(uint4v u) {
  const half2v a = half2_of(u.x), b = half2_of(u.y), c = half2_of(u.z), d = half2_of(u.w);
  return Eight{{(float)a.x, (float)a.y, (float)b.x, (float)b.y, (float)c.x, (float)c.y, (float)d.x, (float)d.y}};
}

__device__ __forceinline__ Eight eight_of(const float *from) {
  const float4v a = *reinterpret_cast<const float4b *>(from), b = *reinterpret_cast<const float4b *>(from + 4);
  return Eight{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}

// Pairs (a[i], b[i]) of elements j + i and dim / 2 + j + i, rotated.
__device__ __forceinline__ void rotate_pairs(const Rotary &r, int at, int j, Eight &a, Eight &b) {
  const unsigned long long row = (unsigned long long)(unsigned)at * (unsigned long long)r.ld + j;
  const Eight c = eight_of(r.cos + row), s = eight_of(r.sin + row);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = a.e[i], y = b.e[i];
    a.e[i] = x * c.e[i] - y * s.e[i];
    b.e[i] = y * c.e[i] + x * s.e[i];
  }
}

// Elements [d, d + 8) of one head of one token, rotated, whatever the pairs are.  d is a multiple of 8, rotary.dim is even.
__device__ __forceinline__ void rotate_eight(const Rotary &r, int at, const __half *x, int d, Eight &y) {
  if (d >= r.dim) return;
  const long long row = (long long)at * r.ld;
  float (&e)[8] = y.e;
  const int half = r.dim / 2;
  if (r.interleaved) {
    float c[4], s[4];
    if (d + 8 <= r.dim) {
      const float4v cv = *reinterpret_cast<const float4b *>(r.cos + row + d / 2), sv = *reinterpret_cast<const float4b *>(r.sin + row + d / 2);
      c[0] = cv.x; c[1] = cv.y; c[2] = cv.z; c[3] = cv.w;
      s[0] = sv.x; s[1] = sv.y; s[2] = sv.z; s[3] = sv.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool turns = d + 2 * i < r.dim;
        c[i] = turns ? r.cos[row + d / 2 + i] : 1.f;
        s[i] = turns ? r.sin[row + d / 2 + i] : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (d + 2 * i >= r.dim) break;
      const float a = e[2 * i], b = e[2 * i + 1];
      e[2 * i] = a * c[i] - b * s[i];
      e[2 * i + 1] = b * c[i] + a * s[i];
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

// Codes of the numbers over a power of two that makes them at most 448 in size; NaN stays NaN.
__device__ __forceinline__ unsigned scaled_codes4(float a, float b, float c, float d, float scale) {
  short2v w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(short2v{0, 0}, a, b, scale, false);
  return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true));
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

// What a lane takes of every `tokens` tokens: TOKENS of them from TOKENS * group on, PARTS times eight elements (lanes left over: none).
template <bool PAIRED>
struct Share {
  static constexpr int TOKENS = PAIRED ? 2 : 4, PARTS = PAIRED ? 2 : 1;
  Eight y[TOKENS][PARTS];
};
// Largest size of the finite elements, `so_far` among them; odd: whether there are others.  (Three operations of the vector ALU for four elements but where
// there are others.)
__device__ __forceinline__ float max3_of_sizes(float so_far, float a, float b) {
  float m;
  asm("v_max3_f32 %0, %1, |%2|, |%3|" : "=v"(m) : "v"(so_far), "v"(a), "v"(b));
  return m;
}
template <bool PAIRED>
__device__ __forceinline__ float largest(const Share<PAIRED> &x, float so_far, bool &odd) {
  float m = so_far;
  bool nan = false;
#pragma unroll
  for (int k = 0; k < Share<PAIRED>::TOKENS; ++k)
#pragma unroll
    for (int i = 0; i < Share<PAIRED>::PARTS; ++i)
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const float a = x.y[k][i].e[j], b = x.y[k][i].e[j + 1];
        nan |= __builtin_isunordered(a, b);
        m = max3_of_sizes(m, a, b);
      }
  if (__builtin_expect(!__any(nan || m > 3.402823466e38f), 1)) return m;
  odd = true;
  m = so_far;
#pragma unroll
  for (int k = 0; k < Share<PAIRED>::TOKENS; ++k)
#pragma unroll
    for (int i = 0; i < Share<PAIRED>::PARTS; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = __builtin_fabsf(x.y[k][i].e[j]);
        m = a <= 3.402823466e38f ? fmaxf(m, a) : m;
      }
  return m;
}

struct Place {
  int d0, half, group;                                              // elements of the parts: d0 and half a head further
  bool lane;
  __device__ __forceinline__ int d(int part) const { return d0 + part * half; }
};
template <bool PAIRED>
__device__ __forceinline__ Place place_of(const AppendParams &p) {
  const int lane = (int)threadIdx.x & 63, group = lane * p.by_columns >> 16, d = (lane - group * p.columns) * 8;
  return Place{d, p.c.head_dim / 2, group, group < p.groups};
}

// A lane's tokens: rows row0 + t ... of x, rotated if `turn`; the nearest of [begin, end) in place of others, so that nothing branches.
template <bool PAIRED>
__device__ __forceinline__ void take(const Rotary &r, const __half *x, long long ld, int row0, int place0, const Place &at, int t, int begin, int end, bool turn,
                                     Share<PAIRED> &s) {
#pragma unroll
  for (int k = 0; k < Share<PAIRED>::TOKENS; ++k) {
    const int token = min(max(t + k, begin), end - 1);
    const __half *from = x + (unsigned long long)(unsigned)(row0 + token) * (unsigned long long)ld;
#pragma unroll
    for (int i = 0; i < Share<PAIRED>::PARTS; ++i) s.y[k][i] = widened(*reinterpret_cast<const uint4b *>(from + at.d(i)));
    if (!turn) continue;
    const int row = min(max(r.position ? r.position[row0 + token] : place0 + token, 0), r.positions - 1);
    if constexpr (PAIRED) rotate_pairs(r, row, at.d0, s.y[k][0], s.y[k][1]);
    else rotate_eight(r, row, from, at.d0, s.y[k][0]);
  }
}

template <bool PAIRED>
__device__ __forceinline__ void append_queries(const AppendParams &p, int wave) {
  const int head = wave % p.q_heads, tile = wave / p.q_heads % p.q_tiles, b = wave / p.q_heads / p.q_tiles;
  if (b >= p.c.n_seqs) return;
  const Sequence s = sequence(p.c, b);
  const Place at = place_of<PAIRED>(p);
  Share<PAIRED> q;
  const int t = tile * p.tokens + at.group * q.TOKENS;
  if (!at.lane || t >= s.rows) return;
  const long long from = (long long)head * p.c.head_dim;
  take<PAIRED>(p.r, p.q + from, p.ldq, s.row0, s.first, at, t, 0, s.rows, p.r.cos != nullptr, q);
#pragma unroll
  for (int k = 0; k < q.TOKENS; ++k)
#pragma unroll
    for (int i = 0; i < q.PARTS; ++i)
      if (t + k < s.rows) *reinterpret_cast<uint4b *>(p.q_out + (s.row0 + t + k) * p.ldq_out + from + at.d(i)) = halves8(q.y[k][i]);
}

template <bool E4M3, bool PAIRED>
__global__ __launch_bounds__(64 * WAVES, PAIRED && E4M3 ? 5 : 2) void kv_append_kernel(const AppendParams p) {
  __shared__ float wave_max[WAVES];
  __shared__ __attribute__((aligned(16))) unsigned char tiles[WAVES][WAVE_LDS];
  const KvParams &c = p.c;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  if ((int)blockIdx.x >= p.kv_blocks) return append_queries<PAIRED>(p, ((int)blockIdx.x - p.kv_blocks) * WAVES + wave);
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
  const Place at = place_of<PAIRED>(p);
  constexpr int TOKENS = Share<PAIRED>::TOKENS, PARTS = Share<PAIRED>::PARTS;
  // this wave's tokens: [t, t + TOKENS) of the lane, every p.tokens * p.team
  const int stride = p.tokens * p.team, start = (begin & -stride) + in_team * p.tokens;
  const int lane_end = at.lane ? end : 0;
  Share<PAIRED> held;
  take<PAIRED>(p.r, x, ld, row0, place0, at, start + at.group * TOKENS, begin, end, turn, held);
  if (page < 0) return;                                                          // (the elements are on their way beside the page's number)
  unsigned char *to = (values ? c.v_pages + page * c.v_page_bytes : c.k_pages + page * c.k_page_bytes) + (long long)head * size * d_all * bytes;
  float *scale_at = (values ? c.v_scales : c.k_scales) + (E4M3 ? (long long)page * c.kv_heads + head : 0);
  const float before = E4M3 && begin > 0 ? *scale_at : 0.f;
  float scale = 1.f;
  bool odd = false;                                                              // some element is not finite
  if (E4M3) {
    float amax = 0.f;
    amax = largest<PAIRED>(held, amax, odd);
    for (int t0 = start + stride; t0 < end; t0 += stride) {
      take<PAIRED>(p.r, x, ld, row0, place0, at, t0 + at.group * TOKENS, begin, end, turn, held);
      amax = largest<PAIRED>(held, amax, odd);
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) amax = fmaxf(amax, __shfl_xor(amax, m));
    if (p.team > 1) {
      if (lane == 0) wave_max[wave] = amax;
      __syncthreads();
      for (int w = 0; w < p.team; ++w) amax = fmaxf(amax, wave_max[wave - in_team + w]);
    }
    scale = fmaxf(scale_for(amax), before);
    if (begin > 0 && scale > before) {                                  // what the page holds already, in the new scale
      const float ratio = before / scale;
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
  const Place mine = at;
  for (int t0 = start; t0 < end; t0 += stride) {
    Place at = mine;
    asm volatile("" : "+v"(at.d0), "+v"(at.group));                     // (what follows from them is not kept from round to round: registers)
    const int t = t0 + at.group * TOKENS;
    if (E4M3 ? start + stride < end : t0 != start) take<PAIRED>(p.r, x, ld, row0, place0, at, t, begin, end, turn, held);
    uint4v word[TOKENS][PARTS];                                         // eight halfs, or in x and y eight codes
#pragma unroll
    for (int k = 0; k < TOKENS; ++k)
#pragma unroll
      for (int i = 0; i < PARTS; ++i) {
        Eight &y = held.y[k][i];
        if (E4M3) {
          if (__builtin_expect(odd, 0))
#pragma unroll
            for (int j = 0; j < 8; ++j) y.e[j] = __builtin_fabsf(y.e[j]) <= 3.402823466e38f ? y.e[j] : __builtin_nanf("");
          word[k][i] = uint4v{scaled_codes4(y.e[0], y.e[1], y.e[2], y.e[3], scale), scaled_codes4(y.e[4], y.e[5], y.e[6], y.e[7], scale), 0, 0};
        }
        else word[k][i] = halves8(y);
      }
    // element j of them
    auto element = [&](int k, int i, int j) {
      const uint4v w = word[k][i];
      if (E4M3) return (j < 4 ? w.x : w.y) >> (8 * (j & 3)) & 0xffu;
      return (j < 2 ? w.x : j < 4 ? w.y : j < 6 ? w.z : w.w) >> (16 * (j & 1)) & 0xffffu;
    };
    if (!values) {
#pragma unroll
      for (int k = 0; k < TOKENS; ++k) {
        if (t + k < begin || t + k >= lane_end) continue;
#pragma unroll
        for (int i = 0; i < PARTS; ++i) {
          if (E4M3) *reinterpret_cast<uint2v *>(to + (t + k) * d_all + at.d(i)) = uint2v{word[k][i].x, word[k][i].y};
          else *reinterpret_cast<uint4v *>(to + ((t + k) * d_all + at.d(i)) * 2) = word[k][i];
        }
      }
      continue;
    }
    // Values, whose tokens lie next to each other in the cache.
    if (t0 < begin || t0 + p.tokens > end) {                            // some tokens of these: one by one
#pragma unroll
      for (int k = 0; k < TOKENS; ++k) {
        if (t + k < begin || t + k >= lane_end) continue;
#pragma unroll
        for (int i = 0; i < PARTS; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int at_element = (at.d(i) + j) * size + t + k;
            if (E4M3) to[at_element] = (unsigned char)element(k, i, j);
            else reinterpret_cast<unsigned short *>(to)[at_element] = (unsigned short)element(k, i, j);
          }
      }
      continue;
    }
    // All of them: through LDS, where element 8 e + j is row j * (head_dim / 8) + e of `tokens` tokens (adjacent lanes write adjacent rows).
    unsigned char *tile = tiles[wave];
    const int row_bytes = p.tokens * bytes, eighths = d_all / 8;
    if (at.lane) {
#pragma unroll
      for (int i = 0; i < PARTS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          unsigned char *w = tile + (j * eighths + (at.d(i) >> 3)) * row_bytes + at.group * TOKENS * bytes;
          if constexpr (PAIRED) {
            const unsigned both = element(0, i, j) | element(1, i, j) << (8 * bytes);
            if (E4M3) *reinterpret_cast<unsigned short *>(w) = (unsigned short)both;
            else *reinterpret_cast<unsigned *>(w) = both;
          } else {
            const unsigned low = element(0, i, j) | element(1, i, j) << (8 * bytes), high = element(2, i, j) | element(TOKENS - 1, i, j) << (8 * bytes);
            if (E4M3) *reinterpret_cast<unsigned *>(w) = low | high << 16;
            else *reinterpret_cast<uint2v *>(w) = uint2v{low, high};
          }
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int pieces = row_bytes >= 16 ? row_bytes / 16 : 1, wide = row_bytes / pieces;      // of a row: 16 bytes, or the eight that it has
    for (int u = lane; u < d_all * pieces; u += 64) {
      const int d = u / pieces, i = u - d * pieces;
      const unsigned char *from = tile + ((d & 7) * eighths + (d >> 3)) * row_bytes + i * wide;
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
  AppendParams p{c, k, v, q, ldk, ldv, ldq, ldq_out, q_out, q_heads, 0, 1, 0, 1, 0, 0, 1, 0, r};
  const int size = 1 << c.page_shift;
  const bool paired = !r.cos || (!r.interleaved && r.dim == c.head_dim);
  const int each = paired ? 2 : 4;
  p.columns = c.head_dim / (paired ? 16 : 8);
  p.by_columns = 65535 / p.columns + 1;
  while (p.groups * 2 * p.columns <= 64 && p.groups * 2 * each <= size) p.groups *= 2;
  p.tokens = each * p.groups;
  p.slots = (c.max_new + size - 2) / size + 1;
  // a wave to the tokens that it holds at a time, of those that a sequence can bring to a page
  const int most = c.max_new < size ? c.max_new : size;
  while (p.team < WAVES && p.team * p.tokens < most) p.team *= 2;
  const long long kv_blocks = (2LL * c.n_seqs * p.slots * c.kv_heads * p.team + WAVES - 1) / WAVES;
  p.q_tiles = (c.max_new + p.tokens - 1) / p.tokens;
  const long long q_waves = q ? (long long)c.n_seqs * p.q_tiles * q_heads : 0, blocks = kv_blocks + (q_waves + WAVES - 1) / WAVES;
  if (blocks > 0xffffffffll / (64 * WAVES)) return VQ_ERR_SHAPE;     // (threads of a grid)
  p.kv_blocks = (int)kv_blocks;
  auto kernel = c.e4m3 ? (paired ? kv_append_kernel<true, true> : kv_append_kernel<true, false>) : (paired ? kv_append_kernel<false, true> : kv_append_kernel<false, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * WAVES), 0, s, p);
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace vq
