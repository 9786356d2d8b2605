// What the attention kernels share: which keys a tile of rows looks at, and how partial results are passed on (internal).
#pragma once
#include "vq_kv.hpp"

namespace vq {

// How a sequence's keys are cut into parts: part p takes every `parts`-th run of `run` chunks of 64 keys (a power of two) from run p on, so that what a workgroup
// looks at first does not depend on the sequence's length.
struct Split {
  int parts, run;
  float *o, *ml;               // partial outputs [seq][kv head][part][row][head_dim], maxima and sums [seq][kv head][part][row][2]
};

// Chunks of a run, one for each wave of the decode kernel.
constexpr int DECODE_RUN = 8, PROMPT_RUN = 4;
int attention_decode_run(const KvParams &c);                       // DECODE_RUN, or half of it
int attention_decode_waves(const KvParams &c, int parts);          // waves of a workgroup of the decode kernel
// The decode kernel, which takes every head: rows of a key head to a workgroup.
int attention_decode_rows(const KvParams &c, const AttentionParams &a);
int launch_attention_decode(const KvParams &c, const AttentionParams &a, const Split &s, hipStream_t stream);
// The prompt kernel: rows of a key head to a workgroup, and whether it takes heads of this size.
int attention_prompt_rows();
bool attention_prompt_takes(const KvParams &c);
int launch_attention_prompt(const KvParams &c, const AttentionParams &a, const Split &s, hipStream_t stream);
// The launch that joins parts: whether a grid can have so many rows and sequences.
bool attention_join_takes(const KvParams &c, const AttentionParams &a);
int launch_attention_join(const KvParams &c, const AttentionParams &a, const Split &s, int tile_rows, hipStream_t stream);

// Bytes from a page's start to word w (of the keys, sixteen bytes each, four lane groups apart) that lane n + 16 g of the decode kernel loads of a key in tile t of a chunk whose sixteen
// keys begin at `place`; in place of words past the key's end its first one, which is not used: behind a pool's last key there is nothing.
constexpr long long key_word_at(int kv_head, int page_shift, int place, int t, int w, int n, int g, int row_bytes) {
  return (((long long)kv_head << page_shift) + (place & ((1 << page_shift) - 1)) + (n & 3)) * row_bytes + t * 4 * row_bytes +
         (w * 64 + g * 16 < row_bytes ? w * 64 + g * 16 : 0);
}

#ifdef __HIPCC__
// The rows of a key head are (new token t, query head of its group), t * group + g.  A tile of them sees keys [low, end) and [0, sinks), of
// which some rows may see fewer; they are looked at in chunks of 64 keys: `sink_chunks` from 0 on, the others from `first` on.
struct Span {
  int place_min, place_max, low, end, first, sink_chunks, chunks;
  __device__ __forceinline__ int chunk(int i) const { return i < sink_chunks ? i : first + i - sink_chunks; }
};
// The new token of a row of a key head.
__device__ __forceinline__ int token_of(const AttentionParams &a, int row) { return a.group > 1 ? (int)__umulhi((unsigned)row, a.by_group) : row; }
__device__ __forceinline__ Span span_of(const AttentionParams &a, const Sequence &s, int row0, int rows) {
  Span v;
  v.place_min = s.first + token_of(a, row0);
  v.place_max = s.first + token_of(a, min(row0 + rows, s.rows * a.group) - 1);
  v.end = max(min(v.place_max + 1, s.end), 0);
  v.low = a.window > 0 ? max(v.place_min - a.window + 1, 0) : 0;
  v.first = v.low >> 6;
  v.sink_chunks = min((min(a.sinks, v.low) + 63) >> 6, v.first);
  v.chunks = v.end > 0 ? v.sink_chunks + max(((v.end + 63) >> 6) - v.first, 0) : 0;
  return v;
}
// Parts that have chunks, one at least.
__device__ __forceinline__ int parts_of(const Split &s, int chunks) { return max(min(s.parts, (chunks + s.run - 1) / s.run), 1); }

// Maximum and sum over the four rows of sixteen lanes, in every lane.  (The exchanged words are named before they are reinterpreted: a bit cast of
// a vector's element was compiled as that of its first.)
__device__ __forceinline__ void across_halves(float x, float &low, float &high) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const unsigned a = r[0], b = r[1];
  low = __uint_as_float(a);
  high = __uint_as_float(b);
}
__device__ __forceinline__ void across_rows(float x, float &even, float &odd) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const unsigned a = r[0], b = r[1];
  even = __uint_as_float(a);
  odd = __uint_as_float(b);
}
__device__ __forceinline__ float rows_max(float x) {
  float a, b;
  across_halves(x, a, b);
  across_rows(fmaxf(a, b), a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float rows_sum(float x) {
  float a, b;
  across_halves(x, a, b);
  across_rows(a + b, a, b);
  return a + b;
}

// Scales past 2^7, with which a code may stand for more than binary16 holds (448 times 2^7 is 57344; 65504 is stored as the code of 256 times 2^8).  Keys are widened with
// 2^7 and what is left of the scale multiplies their scores.  Values beyond the largest number count as that, as an infinity would be not a number in the sums of rows that do
// not see it: of the widened ones (finite_of), or where those are not together in registers of the codes, at 2^16, of which the probability takes a factor of two.
constexpr float WIDEST = 128.f;
__device__ __forceinline__ bool is_wide(float scale) { return !(scale <= WIDEST); }
__device__ __forceinline__ float rest_of(float scale) { return is_wide(scale) ? scale * (1.f / WIDEST) : 1.f; }
__device__ __forceinline__ unsigned finite_of(unsigned halves) {
  return halves - ((halves & 0x7fffu) == 0x7c00u ? 1u : 0u) - ((halves & 0x7fff0000u) == 0x7c000000u ? 0x10000u : 0u);
}
// Codes of values past 2^16 as those of 2^16; NaN stays.
__device__ __forceinline__ unsigned limited(unsigned codes, float scale) {
  const int k = 16 - ((int)(__float_as_uint(scale) >> 23 & 0xff) - 127);       // code 8 (k + 7) is 2^k, down to 2^-6, below that 2^(k + 9)
  const unsigned most = (k >= -6 ? 8 * (k + 7) : 1u << max(k + 9, 0)) * 0x01010101u, size = codes & 0x7f7f7f7fu;
  const unsigned more = (size + (0x7f7f7f7fu - most)) & ~(size + 0x01010101u) & 0x80808080u, all = more | (more - (more >> 7));
  return (codes & ~(all & 0x7f7f7f7fu)) | (most & all);
}
__device__ __forceinline__ half8v finite_of(half8v x) {
  const uint4v u = __builtin_bit_cast(uint4v, x);
  return __builtin_bit_cast(half8v, uint4v{finite_of(u.x), finite_of(u.y), finite_of(u.z), finite_of(u.w)});
}

__device__ __forceinline__ half8v halves_of_e4m3(unsigned a, unsigned b, float scale) {
  const half2v w = halves_of_e4m3<false>(a, scale), x = halves_of_e4m3<true>(a, scale), y = halves_of_e4m3<false>(b, scale), z = halves_of_e4m3<true>(b, scale);
  return half8v{w.x, w.y, x.x, x.y, y.x, y.y, z.x, z.y};
}

// Which of the places [base, base + 16) a token at `place` sees, as bits.
__device__ __forceinline__ unsigned seen_of(const AttentionParams &a, const Sequence &s, int place, int base) {
  auto below = [&](int limit) { return (1u << min(max(limit - base, 0), 16)) - 1u; };
  const unsigned most = below(min(place + 1, s.end));
  return a.window > 0 ? most & (~below(place - a.window + 1) | below(a.sinks)) : most;
}
// x where bit r of `seen` is set, else minus infinity.
__device__ __forceinline__ float where_seen(unsigned seen, int r, float x) {
  const unsigned all = (unsigned)((int)(seen << (31 - r)) >> 31);
  return __uint_as_float((__float_as_uint(x) & all) | (0xff800000u & ~all));
}

// Values that are not finite, of keys that some rows of a tile see and others do not: zero times them would reach the rows that do not.  They are taken
// out of the operands (Odd::clean) and come back as a sum that is not finite for the rows that see them: bits of 64 keys for each element and kind.
template <bool E4M3>
struct Odd {
  static constexpr int KINDS = E4M3 ? 1 : 3, KEYS = E4M3 ? 16 : 8;           // NaN, and in 16 bits both infinities; keys of a 16-byte word
  static __device__ __forceinline__ bool any(uint4v w) {
    const unsigned exponent = E4M3 ? 0x7f7f7f7fu : 0x7c007c00u, one = E4M3 ? 0x01010101u : 0x04000400u, carry = E4M3 ? 0x80808080u : 0x80008000u;
    return ((((w.x & exponent) + one) | ((w.y & exponent) + one) | ((w.z & exponent) + one) | ((w.w & exponent) + one)) & carry) != 0;
  }
  // Bits of the word's keys by kind; the word without them.
  static __device__ __forceinline__ uint4v clean(uint4v w, unsigned (&bits)[KINDS]) {
    unsigned x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int k = 0; k < KINDS; ++k) bits[k] = 0;
#pragma unroll
    for (int i = 0; i < KEYS; ++i) {
      const int per = KEYS / 4, shift = i % per * (32 / per);
      const unsigned v = x[i / per] >> shift & (E4M3 ? 0xffu : 0xffffu);
      const bool odd = E4M3 ? (v & 0x7f) == 0x7f : (v & 0x7c00) == 0x7c00;
      const int kind = E4M3 || (v & 0x3ff) ? 0 : v & 0x8000 ? 2 : 1;
#pragma unroll
      for (int k = 0; k < KINDS; ++k) bits[k] |= odd && kind == k ? 1u << i : 0u;
      if (odd) x[i / per] &= ~((E4M3 ? 0xffu : 0xffffu) << shift);
    }
    return uint4v{x[0], x[1], x[2], x[3]};
  }
  // The bits lie in LDS from address `bits` on, [KINDS][elements], eight bytes each.  (Addresses of LDS as numbers, made opaque where they are used: the compiler
  // would keep each in a register through the loops around, for what hardly ever happens.)
  static __device__ __forceinline__ void put(unsigned at, int kind, int elements, unsigned of) {
    typedef __attribute__((address_space(3))) unsigned short *Shorts;
    typedef __attribute__((address_space(3))) unsigned char *Bytes;
    if (E4M3) *(Shorts)(size_t)(at + kind * elements * 8) = (unsigned short)of;
    else *(Bytes)(size_t)(at + kind * elements * 8) = (unsigned char)of;
  }
  // What they add to an element, whose bits of the first kind are at `at`, of a row that sees the keys of `seen`.
  static __device__ __forceinline__ float sum(unsigned at, int elements, unsigned long long seen) {
    typedef const __attribute__((address_space(3))) unsigned long long *Longs;
    const float inf = __builtin_inff();
    float x = *(Longs)(size_t)at & seen ? __builtin_nanf("") : 0.f;
    if constexpr (!E4M3) {
      if (*(Longs)(size_t)(at + elements * 8) & seen) x += inf;
      if (*(Longs)(size_t)(at + 2 * elements * 8) & seen) x -= inf;
    }
    return x;
  }
};
// Which of 64 places from `base` on a token sees.
__device__ __forceinline__ unsigned long long seen64_of(const AttentionParams &a, const Sequence &s, int place, int base) {
  return (unsigned long long)(seen_of(a, s, place, base) | seen_of(a, s, place, base + 16) << 16) |
         (unsigned long long)(seen_of(a, s, place, base + 32) | seen_of(a, s, place, base + 48) << 16) << 32;
}

// A finite stand-in for the base of a row that has seen nothing yet.
__device__ __forceinline__ float base_of(float m) { return m == -__builtin_inff() ? 0.f : m; }
// The base of a row's exponents lies 2^7 below its maximum and follows it when that has grown by 2^7 more: probabilities of up to 2^14 in binary16, which rounds to zero below
// 2^-25, at least 2^-32 of the largest.  With the base at the maximum a long tail behind a key that outweighs it (a first token, say) is lost from 17 below on, where
// it may be all that comes out.  (The difference is exact; m + 14 is not.)  Every row's by its own scores
// alone, so that no result depends on what rows a tile puts side by side.
constexpr float BELOW = 7.f;
__device__ __forceinline__ bool outgrown(float now, float m) { return now - m > 2.f * BELOW; }
// Exponents are score * scale - base in one rounding and the base is a rounded product: past 2^22 they would be off by more than they may grow, and from 2^28 on
// probabilities infinite.  There the products are rounded as the base is.
__device__ __forceinline__ bool is_large(float base) { return __builtin_fabsf(base) > 4194304.f; }
// One over a softmax's sum; zero for a row that sees nothing; what is not a number stays none.
__device__ __forceinline__ float inverse_of(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -__builtin_inff() : (m + __log2f(l)) * 0.6931471805599453f; }
#endif

}  // namespace vq
