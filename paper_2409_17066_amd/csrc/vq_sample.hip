// The next token of each row of logits: by temperature, the top_k largest, the smallest set that holds top_p of what they weigh, what weighs at least min_p of the largest, and a
// given random number.
//
// Logits are binary16, of which there are 63489 values above minus infinity: a row's counts by value say all but which of equal tokens is meant.  So nothing is sorted and no token's
// weight is computed: a workgroup counts its row in LDS (one bin for each value, the largest first), sums counts and weights over the bins in binary64, finds the borders
// and the value that the random number falls on by these sums, and then that value's n-th occurrence in the row.
//
// Sums are of 64 bits, in an order that depends on nothing: which token a number falls on is decided by sums over the vocabulary, whose rounding in 32 bits (2^-24 times a sum's
// terms) is as large as a rare token's share.
#include "vq_kv.hpp"

namespace vq {

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;
// Bins in descending order of the values they stand for: infinity is bin 0, -65504 is bin LAST; what is left (minus infinity, NaN) has larger numbers.  A thread's sums are of slices of sixteen bins,
// slice r * THREADS + thread for r < ROUNDS.
constexpr int TOP_KEY = 0xFC00, LAST = TOP_KEY - 0x400, SLICE = 16, ROUNDS = 4, BINS = ROUNDS * THREADS * SLICE;
static_assert(BINS > LAST && BINS == 65536, "a bin for every value");

typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
typedef short short2v __attribute__((ext_vector_type(2)));

// Bins of the two numbers of a word; -0 counts as +0.
__device__ __forceinline__ unsigned bins_of(unsigned word) {
  const half2v zero = {(_Float16)0.f, (_Float16)0.f};
  const short2v x = __builtin_bit_cast(short2v, half2_of(word) + zero);
  const short2v sign = x >> 15;
  const ushort2v key = __builtin_bit_cast(ushort2v, x ^ (sign | (short2v){(short)0x8000, (short)0x8000}));
  return __builtin_bit_cast(unsigned, (ushort2v){(unsigned short)TOP_KEY, (unsigned short)TOP_KEY} - key);
}
__device__ __forceinline__ float value_of(int bin) {
  const unsigned key = (unsigned)(TOP_KEY - bin);
  return __half2float(__ushort_as_half((unsigned short)(key & 0x8000u ? key ^ 0x8000u : key ^ 0xFFFFu)));
}

// Where a sum reaches a border: bins below `bin` and `n` of that bin's tokens are in front of it.
struct Border {
  int bin, n;
};
__device__ __forceinline__ Border nearer(Border a, Border b) { return a.bin < b.bin || (a.bin == b.bin && a.n < b.n) ? a : b; }

struct Row {
  const __half *logits;
  int vocabulary;
  float temperature, top_p, min_p, uniform;
  int top_k;
};

// What the workgroup shares beside the bins.
struct Scratch {
  double mass[64], before_mass;
  unsigned count[64], before_count, counts[SLICE];
  int top, slice, below, valid, found[WAVES];
};

// A workgroup's walk over a row: eight numbers a lane, each wave a range of its own.
struct Walk {
  int begin, end;                   // vectors of eight, of this wave
};
__device__ __forceinline__ Walk walk_of(int first, int vectors, int wave) {
  const int each = (vectors + WAVES * 64 - 1) / (WAVES * 64) * 64;
  Walk w;
  w.begin = first + min(wave * each, vectors);
  w.end = first + min((wave + 1) * each, vectors);
  return w;
}
__device__ __forceinline__ uint4v load8(const Row &r, int vector) {
  const int i = vector * 8;
  if (i + 8 <= r.vocabulary) return *reinterpret_cast<const uint4b *>(r.logits + i);
  unsigned w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int at = i + 2 * j;
    const unsigned low = at < r.vocabulary ? __half_as_ushort(r.logits[at]) : 0xFC00u, high = at + 1 < r.vocabulary ? __half_as_ushort(r.logits[at + 1]) : 0xFC00u;
    w[j] = low | high << 16;
  }
  return uint4v{w[0], w[1], w[2], w[3]};
}
// f(bins of a vector's four words, vector) for this wave's vectors; those past the end are of minus infinities.
template <int AHEAD, typename F>
__device__ __forceinline__ void walk(const Row &r, Walk w, int lane, F f) {
  for (int v0 = w.begin; v0 < w.end; v0 += 64 * AHEAD) {
    uint4v x[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int v = v0 + u * 64 + lane;
      x[u] = v < w.end ? load8(r, v) : uint4v{0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u};
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (v0 + u * 64 < w.end) f(uint4v{bins_of(x[u].x), bins_of(x[u].y), bins_of(x[u].z), bins_of(x[u].w)}, v0 + u * 64 + lane);
  }
}

// WIDE: counts of 32 bits, half of the bins at a time, for a row in which a value occurs more than 65535 times; otherwise two bins to a word.
template <bool WIDE>
struct Drawer {
  const Row &r;
  unsigned *bins;
  Scratch &s;
  int tid, lane, wave;
  // sums up to the end of this thread's slices, and in front of them
  unsigned count[ROUNDS], count_before[ROUNDS];
  double mass[ROUNDS], mass_before[ROUNDS], per;          // per: one over the temperature
  unsigned total_count;
  double total_mass;
  float top;

  __device__ __forceinline__ double weight(int bin) const { return s.top == 0 ? (bin == 0 ? 1.0 : 0.0) : exp(((double)value_of(bin) - (double)top) * per); }

  // Counts the row's numbers with bins from `low` on; -> numbers of this thread that have a bin.
  __device__ __forceinline__ unsigned count_bins(int low) {
    uint4v *words = reinterpret_cast<uint4v *>(bins);
    for (int i = tid; i < BINS / 8; i += THREADS) words[i] = uint4v{0, 0, 0, 0};
    __syncthreads();
    unsigned valid = 0;
    auto add = [&](unsigned bin, unsigned n) {
      if (WIDE ? bin - low < BINS / 2 && bin <= LAST : bin <= LAST) {
        valid += n;
        if (WIDE) atomicAdd(bins + (bin - low), n);
        else atomicAdd(bins + (bin >> 1), bin & 1 ? n << 16 : n);
      }
    };
    walk<WIDE ? 4 : 8>(r, walk_of(0, (r.vocabulary + 7) / 8, wave), lane, [&](uint4v b, int) {
      // (eight times the same, as masks leave it: one addition)
      if (b.x == b.y && b.z == b.w && b.x == b.z && (b.x & 0xffff) == b.x >> 16) {
        add(b.x & 0xffff, 8);
        return;
      }
      add(b.x & 0xffff, 1); add(b.x >> 16, 1); add(b.y & 0xffff, 1); add(b.y >> 16, 1);
      add(b.z & 0xffff, 1); add(b.z >> 16, 1); add(b.w & 0xffff, 1); add(b.w >> 16, 1);
    });
    __syncthreads();
    return valid;
  }

  // The words of a slice, and which of its bins are not empty.
  struct Words {
    uint4v a, b, c, d;
  };
  __device__ __forceinline__ Words words_of(int slice) const {
    const uint4v *w = reinterpret_cast<const uint4v *>(bins) + slice * (WIDE ? 4 : 2);
    Words x{w[0], w[1], uint4v{0, 0, 0, 0}, uint4v{0, 0, 0, 0}};
    if (WIDE) {
      x.c = w[2];
      x.d = w[3];
    }
    return x;
  }
  __device__ __forceinline__ static unsigned some(const Words &x) {
    const unsigned w[16] = {x.a.x, x.a.y, x.a.z, x.a.w, x.b.x, x.b.y, x.b.z, x.b.w, x.c.x, x.c.y, x.c.z, x.c.w, x.d.x, x.d.y, x.d.z, x.d.w};
    unsigned mask = 0;
#pragma unroll
    for (int i = 0; i < SLICE; ++i) mask |= (WIDE ? w[i] : i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffff) != 0 ? 1u << i : 0u;
    return mask;
  }
  __device__ __forceinline__ unsigned count_at(int slice, int i) const {      // (slice: among those that are counted)
    return WIDE ? bins[slice * SLICE + i] : reinterpret_cast<const unsigned short *>(bins)[slice * SLICE + i];
  }

  // Counts and weights of this thread's slices of the bins that are counted; the first of all bins that is not empty is the row's maximum.
  template <int FROM, int TO>
  __device__ __forceinline__ void sum_slices() {
    unsigned mask[TO - FROM];
    int first = BINS;
#pragma unroll
    for (int q = FROM; q < TO; ++q) {
      mask[q - FROM] = some(words_of((q - FROM) * THREADS + tid));
      if (mask[q - FROM] && first == BINS) first = (q * THREADS + tid) * SLICE + __builtin_ctz(mask[q - FROM]);
    }
    first = (int)wave_min_u32((unsigned)first);
    if (lane == 0 && first < BINS) atomicMin(&s.top, first);
    __syncthreads();
    top = value_of(min(s.top, LAST));
    int below = BINS;
#pragma unroll
    for (int q = FROM; q < TO; ++q) {
      unsigned c = 0, left = mask[q - FROM];
      double m = 0.0;
      while (left) {
        const int i = __builtin_ctz(left), bin = (q * THREADS + tid) * SLICE + i;
        left &= left - 1;
        const unsigned n = count_at((q - FROM) * THREADS + tid, i);
        const double w = weight(bin);
        c += n;
        m += (double)n * w;
        if (w < (double)r.min_p && bin < below) below = bin;
      }
      count[q] = c;
      mass[q] = m;
    }
    if (below < BINS) atomicMin(&s.below, below);
  }

  // The slices' sums, from the first on.
  __device__ __forceinline__ void scan() {
#pragma unroll
    for (int q = 0; q < ROUNDS; ++q) {
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const unsigned c = __shfl_up(count[q], d);
        const double m = __shfl_up(mass[q], d);
        if (lane >= d) {
          count[q] += c;
          mass[q] += m;
        }
      }
      if (lane == 63) {
        s.count[q * WAVES + wave] = count[q];
        s.mass[q * WAVES + wave] = mass[q];
      }
      count_before[q] = __shfl_up(count[q], 1);
      mass_before[q] = __shfl_up(mass[q], 1);
      if (lane == 0) {
        count_before[q] = 0;
        mass_before[q] = 0.0;
      }
    }
    __syncthreads();
    unsigned c = s.count[lane];
    double m = s.mass[lane];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const unsigned pc = __shfl_up(c, d);
      const double pm = __shfl_up(m, d);
      if (lane >= d) {
        c += pc;
        m += pm;
      }
    }
    total_count = __shfl(c, 63);
    total_mass = __shfl(m, 63);
#pragma unroll
    for (int q = 0; q < ROUNDS; ++q) {
      const int at = q * WAVES + wave;
      const unsigned pc = __shfl(c, (at - 1) & 63);
      const double pm = __shfl(m, (at - 1) & 63);
      if (at > 0) {
        count[q] += pc;
        count_before[q] += pc;
        mass[q] += pm;
        mass_before[q] += pm;
      }
    }
  }

  // One slice: lane i of every wave has bin i (lanes 0 .. 15, others an empty one): its count and weight, and the sums up to the bin's end.
  struct Bin {
    int bin;
    unsigned n, count;
    double weight, mass;
  };
  __device__ __forceinline__ Bin bin_of(int slice) {
    Bin b;
    b.bin = slice * SLICE + lane;
    if (WIDE) {
      if (tid < SLICE) s.counts[tid] = 0;
      __syncthreads();
      unsigned n = 0, of = 0;                                     // (equal ones in a row are added together)
      auto flush = [&] {
        if (n) atomicAdd(&s.counts[of], n);
      };
      walk<1>(r, walk_of(0, (r.vocabulary + 7) / 8, wave), lane, [&](uint4v x, int) {
        const unsigned w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const unsigned bin = j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xffff;
          if ((int)(bin / SLICE) != slice) continue;
          if (bin % SLICE != of) {
            flush();
            n = 0;
            of = bin % SLICE;
          }
          ++n;
        }
      });
      flush();
      __syncthreads();
      b.n = lane < SLICE ? s.counts[lane] : 0;
    } else {
      b.n = lane < SLICE ? count_at(slice, lane) : 0;
    }
    b.weight = b.n ? weight(b.bin) : 0.0;
    b.count = b.n;
    b.mass = (double)b.n * b.weight;
#pragma unroll
    for (int d = 1; d < SLICE; d <<= 1) {
      const unsigned c = __shfl_up(b.count, d);
      const double m = __shfl_up(b.mass, d);
      if (lane >= d) {
        b.count += c;
        b.mass += m;
      }
    }
    b.count += s.before_count;
    b.mass += s.before_mass;
    return b;
  }

  // The first slice with tokens that `is` says yes to, by the sums up to its end; -1: none.  Leaves the sums in front of it in the scratch.
  template <typename Is>
  __device__ __forceinline__ int slice_where(Is is) {
    int first = BINS;
#pragma unroll
    for (int q = 0; q < ROUNDS; ++q)
      if (first == BINS && count[q] != count_before[q] && is(q)) first = q * THREADS + tid;
    __syncthreads();                                              // (what is there has been read)
    if (tid == 0) s.slice = BINS;
    __syncthreads();
    const int of_wave = (int)wave_min_u32((unsigned)first);
    if (lane == 0 && of_wave < BINS) atomicMin(&s.slice, of_wave);
    __syncthreads();
    const int slice = s.slice;
    if (slice == BINS) return -1;
#pragma unroll
    for (int q = 0; q < ROUNDS; ++q)
      if (q * THREADS + tid == slice) {
        s.before_count = count_before[q];
        s.before_mass = mass_before[q];
      }
    __syncthreads();
    return slice;
  }

  // What the tokens in front of a border weigh.
  __device__ __forceinline__ double mass_until(Border e) {
    if (e.bin > LAST) return total_mass;
    const int slice = e.bin / SLICE;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < ROUNDS; ++q)
      if (q * THREADS + tid == slice) {
        s.before_count = count_before[q];
        s.before_mass = mass_before[q];
      }
    __syncthreads();
    const Bin b = bin_of(slice);
    const int at = e.bin % SLICE;
    return in_front(b, at) + (double)e.n * __shfl(b.weight, at);
  }
  __device__ __forceinline__ double in_front(const Bin &b, int at) const { return at ? __shfl(b.mass, at - 1) : s.before_mass; }

  // Behind the k-th token.
  __device__ __forceinline__ Border kth(unsigned k) {
    const int slice = slice_where([&](int q) { return count[q] >= k; });
    if (slice < 0) return Border{BINS, 0};
    const Bin b = bin_of(slice);
    const int at = __builtin_ctzll(__ballot(lane < SLICE && b.n && b.count >= k) | 1ull << 63) & (SLICE - 1);
    return Border{slice * SLICE + at, (int)(k - (__shfl(b.count, at) - __shfl(b.n, at)))};
  }
  // The token whose weight takes the sum to `target` (BEYOND: past it): the tokens in front of it.  The last one where rounding keeps all sums below.
  template <bool BEYOND>
  __device__ __forceinline__ Border token_at(double target) {
    auto reaches = [&](double m) { return BEYOND ? m > target : m >= target; };
    int slice = slice_where([&](int q) { return reaches(mass[q]); });
    if (slice < 0) slice = slice_where([&](int q) { return count[q] == total_count; });
    const Bin b = bin_of(slice);
    const unsigned long long some = __ballot(lane < SLICE && b.n), here = __ballot(lane < SLICE && b.n && reaches(b.mass));
    const int at = here ? __builtin_ctzll(here) : 63 - __builtin_clzll(some);
    const double w = __shfl(b.weight, at), ahead = (target - in_front(b, at)) / w;
    // tokens of the bin whose sums stay in front: as many as whole weights fit, but for one that ends at the target where that is enough
    double n = BEYOND ? floor(ahead) : ceil(ahead) - 1.0;
    n = fmin(fmax(n, 0.0), (double)__shfl(b.n, at) - 1.0);
    return Border{slice * SLICE + at, (int)n};
  }

  // The token among the row's (bin, how many equal ones stand in front of it) that is drawn, and its probability.
  __device__ __forceinline__ Border drawn(float &probability) {
    Border end{BINS, 0};
    if (r.top_k > 0 && (unsigned)r.top_k < total_count) end = kth((unsigned)r.top_k);
    if (r.top_p < 1.f) {
      Border p = token_at<false>((double)fmaxf(r.top_p, 0.f) * mass_until(end));
      ++p.n;
      end = nearer(end, p);
    }
    if (s.below < BINS) end = nearer(end, Border{s.below, 0});
    const double all = mass_until(end);
    Border t = token_at<true>((double)r.uniform * all);
    if (!(t.bin < end.bin || (t.bin == end.bin && t.n < end.n))) {
      // (rounding: the last one in front of the border)
      t = end.n > 0 ? Border{end.bin, end.n - 1} : t;
    }
    probability = (float)(weight(t.bin) / all);
    return t;
  }
};

__global__ __launch_bounds__(THREADS) void sample_kernel(const SampleParams p) {
  extern __shared__ __attribute__((aligned(16))) unsigned bins[];
  Scratch &s = *reinterpret_cast<Scratch *>(bins + BINS / 2);
  const int row = (int)blockIdx.x, tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  Row r;
  r.logits = p.logits + row * p.ld;
  r.vocabulary = p.vocabulary;
  r.temperature = p.temperatures ? p.temperatures[row] : p.temperature;
  r.top_k = p.top_ks ? p.top_ks[row] : p.top_k;
  r.top_p = p.top_ps ? p.top_ps[row] : p.top_p;
  r.min_p = p.min_ps ? p.min_ps[row] : p.min_p;
  r.uniform = fminf(fmaxf(p.uniform[row], 0.f), 0x1.fffffep-1f);
  if (!(r.top_p < 1.f)) r.top_p = 1.f;                              // (NaN too)
  r.min_p = r.min_p > 0.f ? fminf(r.min_p, 1.f) : 0.f;
  if (tid == 0) {
    s.top = BINS;
    s.below = BINS;
    s.valid = 0;
  }
  Border at{BINS, 0};
  float probability = 0.f;
  const bool hot = r.temperature > 0.f;
  Drawer<false> d{r, bins, s, tid, lane, wave};
  d.per = hot ? 1.0 / (double)r.temperature : 0.0;
  const unsigned valid = d.count_bins(0);
  if (p.vocabulary > 65535) {
    unsigned all = valid;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) all += __shfl_xor(all, x);
    if (lane == 0) atomicAdd(&s.valid, (int)all);
  }
  d.sum_slices<0, ROUNDS>();
  d.scan();
  if (p.vocabulary > 65535 && d.total_count != (unsigned)s.valid) {
    // a bin has overflowed: once more, half of the bins after the other
    __syncthreads();
    if (tid == 0) {
      s.top = BINS;
      s.below = BINS;
    }
    Drawer<true> e{r, bins, s, tid, lane, wave};
    e.per = d.per;
    e.count_bins(0);
    e.sum_slices<0, ROUNDS / 2>();
    __syncthreads();
    e.count_bins(BINS / 2);
    e.sum_slices<ROUNDS / 2, ROUNDS>();
    e.scan();
    if (e.total_count) {
      at = Border{s.top, 0};
      probability = 1.f;
      if (hot) at = e.drawn(probability);
    }
  } else if (d.total_count) {
    at = Border{s.top, 0};
    probability = 1.f;
    if (hot) at = d.drawn(probability);
  }

  // where the value's at.n-th occurrence (from zero) is: the wave in whose range it is, the step of that range, the token
  int token = -1;
  if (at.bin < BINS) {
    int first = 0, vectors = (p.vocabulary + 7) / 8, left = at.n;
    for (;;) {
      const Walk w = walk_of(first, vectors, wave);
      unsigned n = 0;
      walk<8>(r, w, lane, [&](uint4v b, int) {
        const unsigned x[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) n += ((x[j] & 0xffff) == (unsigned)at.bin) + ((x[j] >> 16) == (unsigned)at.bin);
      });
      unsigned up_to = n;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const unsigned x = __shfl_up(up_to, d);
        if (lane >= d) up_to += x;
      }
      __syncthreads();
      if (lane == 63) s.found[wave] = (int)up_to;
      __syncthreads();
      int of = 0, before = 0;
      while (of < WAVES - 1 && before + s.found[of] <= left) before += s.found[of++];
      left -= before;
      if (vectors <= WAVES * 64) {                                  // one vector to a lane: wave `of`'s lane with the token knows it
        if (wave == of && (int)up_to > left && (int)(up_to - n) <= left) {
          int skip = left - (int)(up_to - n);
          const uint4v x = load8(r, w.begin + lane);
          const unsigned b[4] = {bins_of(x.x), bins_of(x.y), bins_of(x.z), bins_of(x.w)};
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if ((j & 1 ? b[j / 2] >> 16 : b[j / 2] & 0xffff) == (unsigned)at.bin && skip-- == 0) token = (w.begin + lane) * 8 + j;
        }
        break;
      }
      const Walk there = walk_of(first, vectors, of);
      first = there.begin;
      vectors = there.end - there.begin;
    }
    if (token >= 0) {
      p.tokens[row] = token;
      if (p.probabilities) p.probabilities[row] = probability;
    }
  } else if (tid == 0) {
    p.tokens[row] = -1;
    if (p.probabilities) p.probabilities[row] = 0.f;
  }
}

}  // namespace

int launch_sample(const SampleParams &p, int rows, hipStream_t s) {
  VQ_ALLOW_FULL_LDS(sample_kernel);
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
    hipLaunchKernelGGL(sample_kernel, dim3(rows - row0 < MOST ? rows - row0 : MOST), dim3(THREADS), BINS * 2 + sizeof(Scratch), s, q);
    if (rows - row0 <= MOST) break;
  }
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace vq
