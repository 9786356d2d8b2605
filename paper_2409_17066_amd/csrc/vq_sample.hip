// The next token of each row of logits: by temperature, the top_k largest, the smallest set that holds top_p of what they weigh, what weighs at least min_p of the largest, and a
// given random number.
//
// Logits are binary16, of which there are 31744 finite sizes and two signs: a row's counts by value say all but which of equal tokens is meant.  So nothing is sorted and no
// token's weight is computed: a workgroup counts its row in LDS by value, sums counts and weights over the values in binary64, the largest first, finds the borders and the
// value that the random number falls on by these sums, and then that value's n-th occurrence in the row.
//
// 32 neighbouring values of a sign (a run) lie a constant distance apart, so that their weights are w q^i, one exponential and a polynomial in q with the counts as coefficients.
// Sums are of 64 bits, in an order that depends on nothing: which token a number falls on is decided by sums over the vocabulary, whose rounding in 32 bits (2^-24 times a sum's
// terms) is as large as a rare token's share.
//
// Latency bounds it: few rows, each the work of one compute unit, in phases behind one another (clocks of a row of 32000: counts 9400, sums of the runs 6500, over the runs 2000, borders and the number's
// place 3000 to 6400, its occurrence 3000); of many long rows the counts, 12 to 19 clocks for 64 additions to LDS.  Measured: one row of 32000 with all settings 14 us, 20 rows of 50261
// with 40 % masked 18, 64 rows of 128000 with top_p 24, 256 of 131072 30 (2.2 TB/s), which keep a row in registers; 256 of 151936, read twice, 39, of 256000 54.  Rows on odd addresses are read from
// the first multiple of sixteen bytes on: 20 rows of 50261 16 us, of which such reads without took 21.
// That is with masks of minus infinity, which are counted aside.  A mask of a finite number (-65504, say) is counted like others, 64 lanes in turn at the same word, and beyond 65535 of them the row is
// counted again in 32 bits: 64 rows of 128000 60 us with 40 % masked so, 233 with 70 %, in place of 26.
#include "vq_kv.hpp"

namespace vq {

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;
// Words of LDS by size (the number without its sign): occurrences of the positive number in the lower half, of the negative one in the upper.  Sizes from INF on are not finite.
constexpr int INF = 0x7C00, WORDS = 0x8000, RUN = 32, RUNS = INF / RUN;
// Runs in the order of their values: those of positive numbers, from the largest on, then those of negative ones.  Zero, of either sign, is the last value of the former.
constexpr int ENTRIES = 2 * RUNS, PADDED = 2 * THREADS;
constexpr int OCTAVES = INF / 1024;
static_assert(ENTRIES <= PADDED && INF % RUN == 0 && 1024 % RUN == 0, "runs lie within a power of two");

typedef __attribute__((address_space(3))) unsigned *Lds;
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));

// A value's place in the order of all: the i-th of run `entry`.
struct Place {
  int entry, i;
};
// Where a sum reaches a border: what stands in front of `at` and `n` of that value's tokens are in front of it, and weigh `mass`.
struct Border {
  Place at;
  int n;
  double mass;
};
__device__ __forceinline__ int order_of(Place p) { return p.entry * RUN + p.i; }
__device__ __forceinline__ bool in_front(Border a, Border b) { return order_of(a.at) < order_of(b.at) || (order_of(a.at) == order_of(b.at) && a.n < b.n); }
__device__ __forceinline__ int size_of(Place p) { return p.entry < RUNS ? (RUNS - 1 - p.entry) * RUN + RUN - 1 - p.i : (p.entry - RUNS) * RUN + p.i; }
__device__ __forceinline__ unsigned bits_of(Place p) { return (unsigned)size_of(p) | (p.entry < RUNS ? 0u : 0x8000u); }
__device__ __forceinline__ Place place_of(unsigned bits) {
  const int size = (int)(bits & 0x7FFFu), run = size / RUN;
  return bits & 0x8000u && size ? Place{RUNS + run, size % RUN} : Place{RUNS - 1 - run, RUN - 1 - size % RUN};
}
__device__ __forceinline__ float number_of(unsigned bits) { return __half2float(__ushort_as_half((unsigned short)bits)); }

// exp(y), y <= 0: 2^n times the series of exp on half a factor of two on either side of one, whose 14th term is below 2^-57.
__device__ __forceinline__ double exp_of(double y) {
  y = fmax(y, -1000.0);
  const double n = __builtin_rint(y * 1.4426950408889634074), r = __fma_rn(n, -0x1.abc9e3b39803fp-56, __fma_rn(n, -0x1.62e42fefa39efp-1, y));
  double p = 1.0 / 6227020800.0;
#define VQ_TERM(FACTORIAL) p = __fma_rn(p, r, 1.0 / FACTORIAL)
  VQ_TERM(479001600.0); VQ_TERM(39916800.0); VQ_TERM(3628800.0); VQ_TERM(362880.0); VQ_TERM(40320.0); VQ_TERM(5040.0); VQ_TERM(720.0); VQ_TERM(120.0);
  VQ_TERM(24.0); VQ_TERM(6.0); VQ_TERM(2.0); VQ_TERM(1.0); VQ_TERM(1.0);
#undef VQ_TERM
  return ldexp(p, (int)n);
}

// Vectors of eight numbers are read from addresses of sixteen bytes: `head` numbers stand in front of a row's first one, and fewer than eight behind its last.
struct Row {
  const __half *logits;          // the first vector
  int vocabulary, head, vectors;
  float temperature, top_p, min_p, uniform;
  int top_k;
};

// What the workgroup shares beside the counts: the sums up to each run's end, and what its waves tell each other.
struct Scratch {
  double mass[PADDED];
  unsigned count[PADDED];
  double wave_mass[WAVES], mass_up_to[WAVES];
  double powers[OCTAVES][RUN / 4], factors[OCTAVES];      // by the power of two of a run's sizes: the factor from a number's weight to the next one's, and its (4 i)-th power
  double below_mass;
  int below_entry, below_i;
  unsigned wave_count[WAVES], count_up_to[WAVES], wave_valid[WAVES], wave_top[WAVES], wave_size[WAVES], counts[RUN];
  int found[WAVES], at_front, behind_all, bits, nth;
  float probability;
};

// A wave's part of a range of vectors of eight numbers.
struct Walk {
  int begin, end;
};
__device__ __forceinline__ Walk walk_of(int first, int vectors, int wave) {
  const int each = (vectors + WAVES * 64 - 1) / (WAVES * 64) * 64;
  return Walk{first + min(wave * each, vectors), first + min((wave + 1) * each, vectors)};
}
constexpr unsigned NONE = 0xFC00FC00u;                              // two minus infinities
__device__ __forceinline__ uint4v load8(const Row &r, int vector) { return *reinterpret_cast<const uint4b *>(r.logits + (long long)vector * 8); }
// What stands in front of the vectors, in the workgroup's first thread, and what stands behind them, in its last: the row's first and last eight numbers, of which the others, and those of other
// threads, are minus infinities.
__device__ __forceinline__ uint4v ends_read(const Row &r, int tid) {
  const __half *row = r.logits - r.head;
  if (r.vocabulary >= 8) return *reinterpret_cast<const uint4b *>(tid ? row + r.vocabulary - 8 : row);
  unsigned h[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) h[j] = j >= 8 - r.vocabulary ? __half_as_ushort(row[r.vocabulary - 8 + j]) : 0xFC00u;
  return uint4v{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
}
__device__ __forceinline__ int behind(const Row &r) { return r.vocabulary - r.head - r.vectors * 8; }
__device__ __forceinline__ uint4v ends_of(const Row &r, uint4v read, int tid) {
  const int from = tid == THREADS - 1 ? 8 - behind(r) : tid ? 8 : 0, to = tid ? 8 : r.head;
  auto two = [&](unsigned w, int j) { return (j >= from && j < to ? w & 0xffff : 0xFC00u) | (j + 1 >= from && j + 1 < to ? w & 0xffff0000u : 0xFC000000u); };
  return uint4v{two(read.x, 0), two(read.y, 2), two(read.z, 4), two(read.w, 6)};
}
__device__ __forceinline__ bool has_end(const Row &r, int tid) { return (tid == 0 && r.head) || (tid == THREADS - 1 && behind(r)); }
// The first HELD of a lane's vectors stay in registers.
template <int HELD>
struct Held {
  uint4v x[HELD];
};
// f(a vector's four words) for this wave's vectors, AHEAD of which are on their way at once.
template <int AHEAD, typename F>
__device__ __forceinline__ void walk(const Row &r, Walk w, int lane, F f) {
  for (int v0 = w.begin; v0 < w.end; v0 += 64 * AHEAD) {
    uint4v x[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) x[u] = load8(r, min(v0 + u * 64 + lane, w.end - 1));
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (v0 + u * 64 + lane < w.end) f(x[u]);
  }
}
__device__ __forceinline__ unsigned half_at(uint4v x, int j) {
  const unsigned w = j < 2 ? x.x : j < 4 ? x.y : j < 6 ? x.z : x.w;
  return j & 1 ? w >> 16 : w & 0xffff;
}

__device__ __forceinline__ void add(unsigned address, unsigned n) {
  __hip_atomic_fetch_add((Lds)(size_t)address, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
// factor * the lower or upper half of a word + more
template <bool UPPER>
__device__ __forceinline__ unsigned of_half(unsigned word, unsigned factor, unsigned more) {
  unsigned r;
  if (UPPER) asm("v_mad_u32_u16 %0, %1, %2, %3 op_sel:[1,0,0,0]" : "=v"(r) : "v"(word), "v"(factor), "v"(more));
  else asm("v_mad_u32_u16 %0, %1, %2, %3" : "=v"(r) : "v"(word), "v"(factor), "v"(more));
  return r;
}

// Inclusive sums over the wave's lanes, by DPP: within rows of sixteen lanes, then the rows.
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double x) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, x);
  const unsigned low = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)u, CTRL, ROWS, 0xF, false), high = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), CTRL, ROWS, 0xF, false);
  return __builtin_bit_cast(double, (unsigned long long)low | (unsigned long long)high << 32);
}
__device__ __forceinline__ double sums_of(double x) {
  x += moved<0x111, 0xF>(x);
  x += moved<0x112, 0xF>(x);
  x += moved<0x114, 0xF>(x);
  x += moved<0x118, 0xF>(x);
  x += moved<0x142, 0xA>(x);
  x += moved<0x143, 0xC>(x);
  return x;
}
__device__ __forceinline__ unsigned sums_of(unsigned x) {
#define VQ_MOVED(CTRL, ROWS) x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false)
  VQ_MOVED(0x111, 0xF); VQ_MOVED(0x112, 0xF); VQ_MOVED(0x114, 0xF); VQ_MOVED(0x118, 0xF); VQ_MOVED(0x142, 0xA); VQ_MOVED(0x143, 0xC);
#undef VQ_MOVED
  return x;
}
__device__ __forceinline__ double of_lane(double x, int lane) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, x);
  const unsigned low = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)u, lane), high = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(u >> 32), lane);
  return __builtin_bit_cast(double, (unsigned long long)low | (unsigned long long)high << 32);
}
__device__ __forceinline__ unsigned of_lane(unsigned x, int lane) { return (unsigned)__builtin_amdgcn_readlane((int)x, lane); }

// WIDE: counts of 32 bits, of one sign after the other, for rows in which a number occurs more than 65535 times.
template <bool WIDE>
struct Drawer {
  const Row &r;
  unsigned *words;
  Scratch &s;
  int tid, lane, wave;
  double top, per;                 // the largest logit; one over the temperature
  unsigned largest_size;           // of the finite logits

  // (1 for numbers above the largest, of which there are none)
  __device__ __forceinline__ double weight(unsigned bits) const { return exp_of(fmin(((double)number_of(bits) - top) * per, 0.0)); }

  // Counts the row (WIDE: its numbers of one sign; zeros are positive); -> of this thread's numbers, those that are finite (WIDE: or infinite and positive), and the largest ones of either half.
  template <int HELD>
  __device__ __forceinline__ unsigned count(bool negative, half2v &largest, Held<HELD> &held) {
    const Walk of_wave = walk_of(0, r.vectors, wave);
    const uint4v ends = ends_read(r, tid);
    if constexpr (HELD > 0) {
      // (all of them, the last one in place of those behind it: of conditional loads the compiler would wait for all in front of the first use)
      if (r.vectors > 0) {
#pragma unroll
        for (int u = 0; u < HELD; ++u) held.x[u] = load8(r, min(of_wave.begin + u * 64 + lane, r.vectors - 1));
      }
    }
    uint4v *all = reinterpret_cast<uint4v *>(words);
    for (int i = tid; i < WORDS / 4; i += THREADS) all[i] = uint4v{0, 0, 0, 0};
    __syncthreads();
    const unsigned base = (unsigned)(size_t)(Lds)words;
    unsigned valid = 0;
    ushort2v largest_sizes = {0, 0}, infinities = {0, 0};
    largest = half2v{(_Float16)-__builtin_inff(), (_Float16)-__builtin_inff()};
    // Infinities (a grammar's mask, mostly) go to a word behind the sizes that no other lane of the wave adds to: 64 lanes that add to the same one take 64 turns.
    const unsigned aside = (1 + (unsigned)tid % 1023) * 4;
    auto one = [&](uint4v x) {
      const uint4v size = x & 0x7FFF7FFFu;
      auto larger = [](unsigned a, unsigned b) { return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(ushort2v, a), __builtin_bit_cast(ushort2v, b))); };
      const unsigned sizes = larger(larger(size.x, size.y), larger(size.z, size.w));
      const bool odd = ((sizes + 0x04000400u) & 0x80008000u) != 0, nan = ((sizes + 0x03FF03FFu) & 0x80008000u) != 0, alike = x.x == x.y && x.x == x.z && x.x == x.w;
      largest = __builtin_elementwise_max(largest, __builtin_elementwise_max(__builtin_elementwise_max(half2_of(x.x), half2_of(x.y)), __builtin_elementwise_max(half2_of(x.z), half2_of(x.w))));
      if (WIDE || nan || alike) {
        // NaN, which is not counted, and eight times the same, as masks of a number leave it: one addition
        if (!WIDE && alike && x.x == NONE) return;
        const bool same = alike && (x.x & 0xffff) == x.x >> 16;
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {
          const unsigned bits = half_at(x, j), m = bits & 0x7FFF, n = same ? 8 : 1;
          const bool minus = bits >= 0x8000u && m;
          if (m > INF || (m == INF && (!WIDE || minus)) || (same && j)) continue;
          valid += n;
          if (m < INF) largest_sizes = __builtin_elementwise_max(largest_sizes, (ushort2v){(unsigned short)m, 0});
          if (!WIDE) add(base + m * 4, bits & 0x8000u ? n << 16 : n);
          else if (minus == negative) add(base + m * 4, n);
        }
        return;
      }
      valid += 8;
      const uint4v sign = (x >> 15) & 0x00010001u;
      if (!__ballot(odd)) {
        largest_sizes = __builtin_elementwise_max(largest_sizes, __builtin_bit_cast(ushort2v, sizes));
        auto two = [&](unsigned m, unsigned minus) {
          add(of_half<false>(m, 4, base), of_half<false>(minus, 0xFFFF, 1));
          add(of_half<true>(m, 4, base), of_half<true>(minus, 0xFFFF, 1));
        };
        two(size.x, sign.x); two(size.y, sign.y); two(size.z, sign.z); two(size.w, sign.w);
        return;
      }
      auto two = [&](unsigned m, unsigned minus) {
        const ushort2v of = __builtin_bit_cast(ushort2v, m), most = {INF - 1, INF - 1}, all = {INF, INF}, infinite = __builtin_elementwise_sub_sat(of, most);     // (one or zero)
        infinities += infinite;
        largest_sizes = __builtin_elementwise_max(largest_sizes, of - infinite * all);
        const unsigned which = __builtin_bit_cast(unsigned, infinite);
        add(of_half<false>(which, aside, of_half<false>(m, 4, base)), of_half<false>(minus, 0xFFFF, 1));
        add(of_half<true>(which, aside, of_half<true>(m, 4, base)), of_half<true>(minus, 0xFFFF, 1));
      };
      two(size.x, sign.x); two(size.y, sign.y); two(size.z, sign.z); two(size.w, sign.w);
    };
    if constexpr (HELD > 0) {
#pragma unroll
      for (int u = 0; u < HELD; ++u)
        if (of_wave.begin + u * 64 + lane < of_wave.end) one(held.x[u]);
    } else {
      walk<WIDE ? 2 : 8>(r, of_wave, lane, one);
    }
    if (has_end(r, tid)) one(ends_of(r, ends, tid));
    largest_size = max(largest_sizes.x, largest_sizes.y);
    return valid - infinities.x - infinities.y;
  }
  // The sum of all threads' `valid` and the largest number, for all of them.
  __device__ __forceinline__ void tell(unsigned valid, half2v largest, unsigned &valid_of_all, float &top_of_all) {
    float x = fmaxf((float)largest.x, (float)largest.y);
    valid = sums_of(valid);
    unsigned size = largest_size;
#define VQ_LARGER(CTRL, ROWS) size = max(size, (unsigned)__builtin_amdgcn_update_dpp((int)size, (int)size, CTRL, ROWS, 0xF, false))
    VQ_LARGER(0x111, 0xF); VQ_LARGER(0x112, 0xF); VQ_LARGER(0x114, 0xF); VQ_LARGER(0x118, 0xF); VQ_LARGER(0x142, 0xA); VQ_LARGER(0x143, 0xC);
#undef VQ_LARGER
#define VQ_LARGER(CTRL, ROWS) x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), CTRL, ROWS, 0xF, false)))
    VQ_LARGER(0x111, 0xF); VQ_LARGER(0x112, 0xF); VQ_LARGER(0x114, 0xF); VQ_LARGER(0x118, 0xF); VQ_LARGER(0x142, 0xA); VQ_LARGER(0x143, 0xC);
#undef VQ_LARGER
    if (lane == 63) {
      s.wave_valid[wave] = valid;
      s.wave_top[wave] = __float_as_uint(x);
      s.wave_size[wave] = size;
    }
    __syncthreads();
    valid_of_all = largest_size = 0;
    top_of_all = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      valid_of_all += s.wave_valid[w];
      top_of_all = fmaxf(top_of_all, __uint_as_float(s.wave_top[w]));
      largest_size = max(largest_size, s.wave_size[w]);
    }
  }

  // How far numbers of a power of two are apart.
  __device__ __forceinline__ static double distance(int octave) { return (double)number_of((unsigned)octave * 1024 + 1) - (double)number_of((unsigned)octave * 1024); }
  __device__ __forceinline__ void make_powers() {
    constexpr int EACH = RUN / 4 + 1;
    if (tid >= OCTAVES * EACH) return;
    const int octave = tid / EACH, i = tid % EACH;
    const double f = exp_of(-distance(octave) * per * (double)(i < EACH - 1 ? 4 * i : 1));
    if (i < EACH - 1) s.powers[octave][i] = f;
    else s.factors[octave] = f;
  }
  // Counts and weights of the runs of both signs (WIDE: of one), of a thread's 32 sizes, to the scratch.  That of the row's largest number is summed value by value by the last wave, half of which has
  // no other: weights relative to its neighbours could be too large for a number there, and of equal logits the sums are whole numbers so, whose weight is one without a rounding.
  __device__ __forceinline__ void sum_runs(bool negative) {
    const unsigned of_top = __half_as_ushort(__float2half_rn((float)top)), top_size = of_top & 0x7FFFu;
    const bool top_minus = of_top >= 0x8000u && top_size;
    if (wave == WAVES - 1) {
      s.mass[ENTRIES + lane] = 0.0;                                 // (entries behind the last run)
      s.count[ENTRIES + lane] = 0;
      if (!WIDE || negative == top_minus) {
        const int entry = place_of(of_top).entry;
        const unsigned bits = bits_of(Place{entry, lane & (RUN - 1)}), w = words[bits & 0x7FFFu];
        unsigned n = WIDE ? w : bits & 0x8000u ? w >> 16 : bits ? w & 0xffff : (w & 0xffff) + (w >> 16);
        if (lane >= RUN || bits == 0x8000u) n = 0;                  // (minus zero is counted as zero)
        const double m = sums_of((double)n * weight(bits));
        n = sums_of(n);
        if (lane == 63) {
          s.mass[entry] = m;
          s.count[entry] = n;
        }
      }
    }
    if (tid >= RUNS) return;
    const unsigned least = (unsigned)tid * RUN;
    const bool has_top = top_size / RUN == (unsigned)tid, plus_too = (!WIDE || !negative) && !(has_top && !top_minus), minus_too = (!WIDE || negative) && !(has_top && top_minus);
    double plus = 0.0, minus = 0.0;
    unsigned n_plus = 0, n_minus = 0;
    if (least <= largest_size) {
      // A run's powers of q begin at its largest number, that of largest size of the positive and of smallest size of the negative ones.  Lanes begin in different quarters of their runs,
      // whose first words lie in the same bank of LDS for every second lane.
      const uint4v *from = reinterpret_cast<const uint4v *>(words) + tid * (RUN / 4);
      const double *powers = s.powers[tid / (1024 / RUN)];
      const double q = s.factors[tid / (1024 / RUN)];
      int c = (lane >> 1) & 7;
      uint4v w = from[c];
      // (one after the other: there are few registers beside those of a row that is kept)
#pragma unroll 1
      for (int j = 0; j < RUN / 4; ++j) {
        const int next = (c + 1) & 7;
        const uint4v ahead = from[next];
        const double p_plus = powers[7 - c], p_minus = powers[c];
        unsigned a0 = WIDE ? w.x : w.x & 0xffff, b0 = WIDE ? w.x : w.x >> 16;
        const unsigned a1 = WIDE ? w.y : w.y & 0xffff, a2 = WIDE ? w.z : w.z & 0xffff, a3 = WIDE ? w.w : w.w & 0xffff;
        const unsigned b1 = WIDE ? w.y : w.y >> 16, b2 = WIDE ? w.z : w.z >> 16, b3 = WIDE ? w.w : w.w >> 16;
        if (!WIDE && (tid | c) == 0) {                              // zeros
          a0 += b0;
          b0 = 0;
        }
        n_plus += (a0 + a1) + (a2 + a3);
        n_minus += (b0 + b1) + (b2 + b3);
        plus = __fma_rn(__fma_rn(__fma_rn(__fma_rn((double)a0, q, (double)a1), q, (double)a2), q, (double)a3), p_plus, plus);
        minus = __fma_rn(__fma_rn(__fma_rn(__fma_rn((double)b3, q, (double)b2), q, (double)b1), q, (double)b0), p_minus, minus);
        c = next;
        w = ahead;
      }
      if (n_plus) plus *= weight(least + RUN - 1);
      if (n_minus) minus *= weight(least | 0x8000u);
    }
    if (plus_too) {
      s.mass[RUNS - 1 - tid] = plus;
      s.count[RUNS - 1 - tid] = n_plus;
    }
    if (minus_too) {
      s.mass[RUNS + tid] = minus;
      s.count[RUNS + tid] = n_minus;
    }
  }

  // Sums up to each run's end in place of its own.
  __device__ __forceinline__ void scan() {
    __syncthreads();
    const double m0 = s.mass[2 * tid], m1 = s.mass[2 * tid + 1];
    const unsigned c0 = s.count[2 * tid], c1 = s.count[2 * tid + 1];
    const double m = sums_of(m0 + m1);
    const unsigned c = sums_of(c0 + c1);
    if (lane == 63) {
      s.wave_mass[wave] = m;
      s.wave_count[wave] = c;
    }
    __syncthreads();
    // lane w: the sums up to wave w's end
    const double up_to = sums_of(lane < WAVES ? s.wave_mass[lane] : 0.0);
    const unsigned count_up_to = sums_of(lane < WAVES ? s.wave_count[lane] : 0u);
    const double before = wave ? of_lane(up_to, wave - 1) : 0.0;
    const unsigned count_before = wave ? of_lane(count_up_to, wave - 1) : 0;
    if (wave == 0 && lane < WAVES) {
      s.mass_up_to[lane] = up_to;
      s.count_up_to[lane] = count_up_to;
    }
    s.mass[2 * tid + 1] = before + m;
    s.count[2 * tid + 1] = count_before + c;
    s.mass[2 * tid] = before + m - m1;
    s.count[2 * tid] = count_before + c - c1;
    __syncthreads();
  }

  // One run: lane i of the wave has its i-th value (lanes from RUN on: none): its bits, how often it occurs, its weight, and the sums up to it.
  struct Value {
    unsigned bits, n, count;
    double weight, mass, before;   // before: in front of the run
  };
  __device__ __forceinline__ Value values_of(int entry) {
    Value v;
    const Place p{entry, lane & (RUN - 1)};
    v.bits = bits_of(p);
    if (WIDE) {
      // the row once more, equal ones in succession added together
      __syncthreads();
      if (tid < RUN) s.counts[tid] = 0;
      __syncthreads();
      unsigned n = 0;
      int of = 0;
      auto flush = [&] {
        if (n) atomicAdd(&s.counts[of], n);
      };
      auto one = [&](uint4v x) {
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {
          const unsigned bits = half_at(x, j);
          if ((bits & 0x7FFFu) >= INF) continue;
          const Place here = place_of(bits);
          if (here.entry != entry) continue;
          if (here.i != of) {
            flush();
            n = 0;
            of = here.i;
          }
          ++n;
        }
      };
      walk<1>(r, walk_of(0, r.vectors, wave), lane, one);
      if (has_end(r, tid)) one(ends_of(r, ends_read(r, tid), tid));
      flush();
      __syncthreads();
      v.n = s.counts[p.i];
    } else {
      const unsigned w = words[size_of(p)];
      v.n = v.bits & 0x8000u ? w >> 16 : v.bits ? w & 0xffff : (w & 0xffff) + (w >> 16);
      if (v.bits == 0x8000u) v.n = 0;                               // (counted as zero)
    }
    if (lane >= RUN) v.n = 0;
    v.weight = weight(v.bits);
    v.before = entry ? s.mass[entry - 1] : 0.0;
    v.mass = v.before + sums_of((double)v.n * v.weight);
    v.count = (entry ? s.count[entry - 1] : 0) + sums_of(v.n);
    return v;
  }

  // The first run whose sums `is` says yes to; -1: none.
  template <typename Is>
  __device__ __forceinline__ int entry_where(Is is) const {
    // (of the sixteen stretches that the waves have added up, then two runs a lane; where rounding leaves the sums in no order, the stretch's last one)
    constexpr int EACH = PADDED / WAVES;
    static_assert(EACH == 128, "two runs a lane");
    const unsigned long long stretch = __ballot(lane < WAVES && is(s.count_up_to[lane & (WAVES - 1)], s.mass_up_to[lane & (WAVES - 1)]));
    if (!stretch) return -1;
    const int from = __builtin_ctzll(stretch) * EACH, at = from + 2 * lane;
    const bool first = is(s.count[at], s.mass[at]), second = is(s.count[at + 1], s.mass[at + 1]);
    const unsigned long long both = __ballot(first || second);
    if (!both) return from + EACH - 1;
    const int l = __builtin_ctzll(both);
    return from + 2 * l + (__ballot(first) >> l & 1 ? 0 : 1);
  }

  __device__ __forceinline__ Border end() const { return Border{{PADDED, 0}, 0, s.mass[PADDED - 1]}; }
  // A border in front of the n-th token of value i.
  __device__ __forceinline__ Border border_at(int entry, const Value &v, int i, int n) const {
    return Border{{entry, i}, n, (i ? of_lane(v.mass, i - 1) : v.before) + (double)n * of_lane(v.weight, i)};
  }
  // Behind the k-th token (of more).
  __device__ __forceinline__ Border kth(unsigned k) {
    const int entry = entry_where([&](unsigned c, double) { return c >= k; });
    const Value v = values_of(entry);
    const int i = __builtin_ctzll(__ballot(v.n && v.count >= k) | 1ull << 63) & (RUN - 1);
    return border_at(entry, v, i, (int)(k - (of_lane(v.count, i) - of_lane(v.n, i))));
  }
  // In front of the token whose weight takes the sum past `target`; BEHIND: behind the one that takes it there.
  template <bool BEHIND>
  __device__ __forceinline__ Border token_at(double target) {
    auto reaches = [&](double m) { return BEHIND ? m >= target : m > target; };
    // (where rounding lets a run without tokens reach it: the next one; where it keeps all sums below: the last token)
    int entry = entry_where([&](unsigned c, double m) { return c > 0 && reaches(m); });
    const unsigned all = s.count[PADDED - 1];
    if (entry >= 0) {
      const unsigned up_to = s.count[entry];
      if (up_to == (entry ? s.count[entry - 1] : 0)) entry = entry_where([&](unsigned c, double) { return c > up_to; });
    }
    if (entry < 0) entry = entry_where([&](unsigned c, double) { return c == all; });
    const Value v = values_of(entry);
    const unsigned long long some = __ballot(v.n != 0), here = __ballot(v.n != 0 && reaches(v.mass));
    const int i = here ? __builtin_ctzll(here) : some ? 63 - __builtin_clzll(some) : 0;
    const double before = i ? of_lane(v.mass, i - 1) : v.before, ahead = (target - before) / of_lane(v.weight, i);
    // tokens of this value in front: as many as whole weights fit; behind: one that ends at the target is enough
    const double n = fmin(fmax(BEHIND ? ceil(ahead) - 1.0 : floor(ahead), 0.0), (double)of_lane(v.n, i) - 1.0);
    return border_at(entry, v, i, (int)n + BEHIND);
  }
  // In front of the first value that weighs less than min_p: among every 1024th one, every sixteenth of those in front of that, each of those in front of that.  By the weights themselves: around
  // max + T log(min_p) it is not to be looked for, as at high temperatures any number of weights round to the same (all of them to 1, which min_p = 1 keeps).
  __device__ __forceinline__ Border below_min_p() {
    constexpr int VALUES = ENTRIES * RUN, FAR = 1024, NEAR = 16;
    static_assert(VALUES <= 63 * FAR && FAR == 64 * NEAR, "three steps of 64 lanes");
    auto below = [&](int order) { return order >= VALUES || weight(bits_of(Place{order / RUN, order % RUN})) < (double)r.min_p; };
    // (the largest number is never below, as no weight is more than 1 and min_p at most that; behind the values everything is)
    const int far_end = (int)__builtin_ctzll(__ballot(lane > 0 && below(lane * FAR))) * FAR;
    const int near_end = far_end - FAR + ((int)__builtin_ctzll(__ballot(lane == 63 || below(far_end - FAR + (lane + 1) * NEAR))) + 1) * NEAR;
    const int first = near_end - NEAR + (int)__builtin_ctzll(__ballot(lane >= NEAR - 1 || below(near_end - NEAR + lane + 1))) + 1;
    if (first >= VALUES) return end();
    return border_at(first / RUN, values_of(first / RUN), first % RUN, 0);
  }

  // What top_k and top_p keep.
  __device__ __forceinline__ Border kept() {
    Border e = end();
    if (r.top_k > 0 && (unsigned)r.top_k < s.count[PADDED - 1]) e = kth((unsigned)r.top_k);
    if (r.top_p < 1.f) {
      const Border p = token_at<true>((double)fmaxf(r.top_p, 0.f) * e.mass);
      if (in_front(p, e)) e = p;
    }
    return e;
  }
  // The token among the row's in front of a border, by the value's order and how many equal ones stand in front of it, and its probability.
  __device__ __forceinline__ Border drawn(Border e, float &probability) {
    const Border t = token_at<false>((double)r.uniform * e.mass);
    probability = (float)(weight(bits_of(t.at)) / e.mass);
    return t;
  }
};

// Infinite logits, n of them: of equal weight, and nothing else has any.
__device__ __forceinline__ Border infinite_of(const Row &r, unsigned n, float &probability) {
  if (r.top_k > 0) n = min(n, (unsigned)r.top_k);
  if (r.top_p < 1.f) n = max((unsigned)ceil((double)fmaxf(r.top_p, 0.f) * (double)n), 1u);
  probability = (float)(1.0 / (double)n);
  return Border{{0, 0}, (int)((double)r.uniform * (double)n), 0.0};
}

// HELD: vectors of eight numbers that a lane keeps (all of its row's), or 0: the row is read again at the end.
template <int HELD>
__global__ __launch_bounds__(THREADS) void sample_kernel(const SampleParams p) {
  extern __shared__ __attribute__((aligned(16))) unsigned words[];
  Scratch &s = *reinterpret_cast<Scratch *>(words + WORDS);
  const int row = (int)blockIdx.x, tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Row r;
  r.logits = p.logits + row * p.ld;
  r.vocabulary = p.vocabulary;
  r.head = p.vocabulary < 16 ? 0 : (int)(-((unsigned)(size_t)r.logits >> 1) & 7);
  r.logits += r.head;
  r.vectors = (r.vocabulary - r.head) / 8;
  r.temperature = p.temperatures ? p.temperatures[row] : p.temperature;
  r.top_k = p.top_ks ? p.top_ks[row] : p.top_k;
  r.top_p = p.top_ps ? p.top_ps[row] : p.top_p;
  r.min_p = p.min_ps ? p.min_ps[row] : p.min_p;
  r.uniform = fminf(fmaxf(p.uniform[row], 0.f), 0x1.fffffep-1f);
  if (!(r.top_p < 1.f)) r.top_p = 1.f;                              // (NaN too)
  r.min_p = r.min_p > 0.f ? fminf(r.min_p, 1.f) : 0.f;
  Drawer<false> d{r, words, s, tid, lane, wave};
  half2v largest;
  Held<HELD> held;
  unsigned valid = d.count(false, largest, held);
  float top;
  const bool hot = r.temperature > 0.f;
  d.per = 1.0 / (double)r.temperature;
  if (hot) d.make_powers();
  d.tell(valid, largest, valid, top);
  if (valid == 0 && !(top > 0.f)) {                                  // (infinite logits are not counted, but there)
    if (tid == 0) {
      p.tokens[row] = -1;
      if (p.probabilities) p.probabilities[row] = 0.f;
    }
    return;
  }
  unsigned bits = __half_as_ushort(__float2half_rn(top));
  int nth = 0;
  float probability = 1.f;
  if (hot) {
    d.top = (double)top;
    const bool infinite = bits == INF;
    bool overflown = infinite;                                      // (infinite ones: by wide counts)
    if (!infinite) {
      d.sum_runs(false);
      d.scan();
      overflown = s.count[PADDED - 1] != valid;
    }
    if (overflown) {
      Drawer<true> e{r, words, s, tid, lane, wave, d.top, d.per, INF};
      half2v unused;
      Held<0> none;
      __syncthreads();
      e.count(false, unused, none);
      __syncthreads();
      if (infinite) {
        nth = infinite_of(r, words[INF], probability).n;
      } else {
        e.largest_size = d.largest_size;                            // (of all of the row)
        e.sum_runs(false);
        __syncthreads();
        e.count(true, unused, none);
        __syncthreads();
        e.largest_size = d.largest_size;
        e.sum_runs(true);
        e.scan();
        Border kept = e.kept();
        if (r.min_p > 0.f) {
          const Border m = e.below_min_p();
          if (in_front(m, kept)) kept = m;
        }
        const Border t = e.drawn(kept, probability);
        bits = bits_of(t.at);
        nth = t.n;
      }
    } else {
      // (one wave: it needs nothing of the others, which would be in its way, but for the border of min_p, which depends on none of its own)
      Border e;
      if (wave == 1 && r.min_p > 0.f) {
        const Border m = d.below_min_p();
        if (lane == 0) {
          s.below_entry = m.at.entry;
          s.below_i = m.at.i;
          s.below_mass = m.mass;
        }
      }
      if (wave == 0) e = d.kept();
      if (r.min_p > 0.f) __syncthreads();
      if (wave == 0) {
        if (r.min_p > 0.f) {
          const Border m{{s.below_entry, s.below_i}, 0, s.below_mass};
          if (in_front(m, e)) e = m;
        }
        const Border t = d.drawn(e, probability);
        if (lane == 0) {
          s.bits = (int)bits_of(t.at);
          s.nth = t.n;
          s.probability = probability;
        }
      }
      __syncthreads();
      bits = (unsigned)s.bits;
      nth = s.nth;
      probability = s.probability;
    }
  }

  // Where the number's nth occurrence (from zero) is.  A half of zero bits in what `differs` leaves is the number.
  const unsigned zeros = (bits & 0x7FFFu) == 0 ? 0x7FFF7FFFu : 0xFFFFFFFFu, both = (bits | bits << 16) & zeros;
  auto differs = [&](uint4v x) { return (x & zeros) ^ both; };
  auto matches = [&](uint4v x) {
    const uint4v d = differs(x);
    auto smaller = [](unsigned a, unsigned b) {
      return __builtin_bit_cast(unsigned, __builtin_elementwise_min(__builtin_bit_cast(ushort2v, a), __builtin_bit_cast(ushort2v, b)));
    };
    const unsigned least = smaller(smaller(d.x, d.y), smaller(d.z, d.w));
    unsigned n = 0;
    if (!(least & 0xffff) || !(least >> 16)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) n += half_at(d, j) == 0;
    }
    return n;
  };
  auto write = [&](uint4v x, int skip, int from) {                // the lane whose vector it is
    const uint4v d = differs(x);
    int token = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (half_at(d, j) == 0 && skip-- == 0) token = from + j;
    p.tokens[row] = token;
    if (p.probabilities) p.probabilities[row] = probability;
  };
  // Numbers of matches of the waves, of which the one with the nth is found; nth: what is left of it there.
  auto wave_with_nth = [&](unsigned n_of_wave) {
    __syncthreads();
    if (lane == 0) s.found[wave] = (int)n_of_wave;
    __syncthreads();
    int of = 0;
    while (of < WAVES - 1 && s.found[of] <= nth) nth -= s.found[of++];
    return of;
  };
  const uint4v ends = ends_of(r, ends_read(r, tid), tid);                     // (again: they would take four registers all the way)
  const unsigned at_end = matches(ends);
  const int at_front = (int)of_lane(at_end, 0), behind_all = (int)of_lane(at_end, 63);      // (of the first wave and of the last)
  int first = 0, vectors = r.vectors;
  if constexpr (HELD > 0) {
    const Walk w = walk_of(first, vectors, wave);
    unsigned n = 0;
#pragma unroll
    for (int u = 0; u < HELD; ++u)
      if (w.begin + u * 64 + lane < w.end) n += matches(held.x[u]);
    n += at_end;
    if (wave != wave_with_nth(of_lane(sums_of(n), 63))) return;
    if (wave == 0) {
      if (nth < at_front) {
        if (tid == 0) write(ends, nth, 0);
        return;
      }
      nth -= at_front;
    }
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
      if (w.begin + u * 64 >= w.end) break;
      const unsigned here = w.begin + u * 64 + lane < w.end ? matches(held.x[u]) : 0;
      if (!__ballot(here != 0)) continue;
      const unsigned up_to = sums_of(here);
      if ((int)up_to > nth && (int)(up_to - here) <= nth) write(held.x[u], nth - (int)(up_to - here), r.head + (w.begin + u * 64 + lane) * 8);
      nth -= (int)of_lane(up_to, 63);
      if (nth < 0) return;
    }
    if (tid == THREADS - 1) write(ends, nth, p.vocabulary - 8);
  } else {
    // the wave in whose part of the row it is, the part of that, the lane
    for (bool whole = true;; whole = false) {
      const Walk w = walk_of(first, vectors, wave);
      unsigned n = 0;
      uint4v mine{};
      walk<8>(r, w, lane, [&](uint4v x) {
        mine = x;
        n += matches(x);
      });
      const unsigned up_to = sums_of(n);
      if (whole && tid == 0) s.at_front = at_front;
      if (whole && tid == THREADS - 1) s.behind_all = behind_all;
      const int of = wave_with_nth(of_lane(up_to, 63) + (whole ? at_front + behind_all : 0));
      if (whole && of == 0) {
        if (nth < s.at_front) {
          if (tid == 0) write(ends, nth, 0);
          return;
        }
        nth -= s.at_front;
      }
      if (whole && of == WAVES - 1 && nth >= s.found[of] - s.behind_all) {
        if (tid == THREADS - 1) write(ends, nth - (s.found[of] - s.behind_all), p.vocabulary - 8);
        return;
      }
      if (vectors <= WAVES * 64) {                                  // one vector to a lane
        if (wave == of && (int)up_to > nth && (int)(up_to - n) <= nth) write(mine, nth - (int)(up_to - n), r.head + (w.begin + lane) * 8);
        return;
      }
      const Walk there = walk_of(first, vectors, of);
      first = there.begin;
      vectors = there.end - there.begin;
    }
  }
}

}  // namespace

int launch_sample(const SampleParams &p, int rows, hipStream_t s) {
  // As many registers as the row needs, for rows that fit them: 20 rows of 32000 logits 12.7 us with 4 vectors a lane; of 32776 13.7 with 8 and 15.3 with 16; of 65536 15.9 and 17.3; of
  // 131072 22.4 with 16, of 131080, read twice, 25.1.
  VQ_ALLOW_FULL_LDS(sample_kernel<4>);
  VQ_ALLOW_FULL_LDS(sample_kernel<8>);
  VQ_ALLOW_FULL_LDS(sample_kernel<16>);
  VQ_ALLOW_FULL_LDS(sample_kernel<0>);
  constexpr int EACH = 8 * THREADS;
  auto kernel = p.vocabulary <= 4 * EACH ? sample_kernel<4> : p.vocabulary <= 8 * EACH ? sample_kernel<8> : p.vocabulary <= 16 * EACH ? sample_kernel<16> : sample_kernel<0>;
  constexpr int MOST = 1 << 21;                                     // rows of a launch (a grid has fewer than 2^32 threads)
  for (int row0 = 0; row0 < rows; row0 += MOST) {
    SampleParams q = p;
    q.logits += row0 * p.ld;
    q.uniform += row0;
    if (q.temperatures) q.temperatures += row0;
    if (q.top_ks) q.top_ks += row0;
    if (q.top_ps) q.top_ps += row0;
    if (q.min_ps) q.min_ps += row0;
    q.tokens += row0;
    if (q.probabilities) q.probabilities += row0;
    hipLaunchKernelGGL(kernel, dim3(rows - row0 < MOST ? rows - row0 : MOST), dim3(THREADS), WORDS * 4 + sizeof(Scratch), s, q);
    if (rows - row0 <= MOST) break;
  }
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace vq
