// Attention of many rows a key head (a prompt, or a chunk of one) over a paged cache: the prompt path.
//
// The matrix cores bound it, and the vector ALUs' softmax beside them.  Four waves of a workgroup take 32 rows each, two workgroups share a compute
// unit.  Chunks of 64 keys pass through LDS as binary16 numbers, in two buffers: the next chunk's words are loaded before a chunk is computed and are converted and
// stored behind it.  Scores come transposed, S^T = K Q^T (v_mfma_f32_32x32x16_f16): a lane holds sixteen keys a tile of one row, so that a row's maximum is
// one exchange between two lanes, and the running maximum scales registers of the same lane.  Rows of a key tile are stored in an order that makes a lane's scores those of
// sixteen consecutive keys, eight of which are what the lane has to give as operand B of O^T = V^T P^T: the probabilities never leave their registers.
//
// Measured, 8 bits, heads of 128 elements: chunks of 1024 tokens behind up to 15360, 64 query and 8 key heads, 1.12 to 1.16 ms, 900 to 935 TFLOP/s, where a large product of
// matrices reaches 1100; a prompt of 2048 tokens, 32 heads, 57 us (604 TFLOP/s: one round of workgroups, whose last chunks run alone), of 64 elements 42.  Matrix cores, vector ALUs and
// LDS are each busy 40 % of the clocks of long contexts; fewer vector operations (scale in a vector register, four maxima side by side) and two chains of
// products in place of one changed nothing: what is left is LDS (without its traffic 36 % less) and the power limit.
#include "vq_attention.hpp"
#include <type_traits>

namespace vq {

namespace {

constexpr int WAVES = 4, THREADS = 64 * WAVES, ROWS = 32 * WAVES;
typedef float float16v __attribute__((ext_vector_type(16)));
struct Sixteen {
  float f[16];
};

// Row of LDS for key (of 64): within 32 keys, key 16 h + 4 a + i is row 8 a + 4 h + i.
__device__ __forceinline__ int row_of_key(int key) { return (key & 32) | ((key & 12) << 1) | ((key & 16) >> 2) | (key & 3); }

// The sequence that has `n` longer ones (of equal ones the first comes first; as they are numbered, where there are more than a wave has lanes).
__device__ __forceinline__ int nth_longest(const KvParams &c, int n, int lane) {
  if (c.n_seqs == 1 || c.n_seqs > 64) return n;
  const int mine = lane < c.n_seqs ? max(c.lengths[lane], 0) : -1;
  int before = 0;
  for (int j = 0; j < c.n_seqs; ++j) {
    const int other = __builtin_amdgcn_readlane(mine, j);
    before += other > mine || (other == mine && j < lane);
  }
  return (int)__builtin_ctzll(__ballot(lane < c.n_seqs && before == n));
}

// D: elements of a head, or (not EXACT) more, zeros behind the head's own.
template <bool E4M3, int D, bool EXACT>
__global__ __launch_bounds__(THREADS, 2) void attention_prompt_kernel(const KvParams c, const AttentionParams a, const Split split, int tiles, int zigzag) {
  const int dim = EXACT ? D : c.head_dim;
  constexpr int BYTES = E4M3 ? 1 : 2;
  constexpr int KU = D * BYTES / 16, VU = 64 * BYTES / 16;        // 16-byte words of a key, and of an element's 64 keys
  constexpr int REPS = 64 * KU / THREADS, SLOTS = D / 8;          // words a thread brings; 16-byte slots of a key in LDS
  constexpr int K_BYTES = 64 * D * 2, BUFFER = 2 * K_BYTES;
  constexpr int STEPS = D / 16, DT = D / 32, AHEAD = 6;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  unsigned char *there = lds + 2 * BUFFER;                         // [2][4]: bit 0, whether each sixteen keys of a buffer have a page; 1: values to be put back; 2: rests of keys' scales
  auto bits_of = [](int buffer) { return 2 * BUFFER + 16 + buffer * (Odd<E4M3>::KINDS * D * 8); };
  auto rests_of = [=](int buffer) { return bits_of(2) + buffer * (REPS * WAVES * 4); };      // [word][wave]
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;

  // Long sequences first and of each the rows that see most, so that short work fills the end; where all workgroups are resident at once, so that
  // the two of a compute unit have equal work together.  Those of a key head go to one XCD where the heads are a multiple of eight.
  const int kv_head = (int)(blockIdx.x % c.kv_heads), rest = (int)(blockIdx.x / c.kv_heads);
  int b, part, rank;
  if (zigzag) {
    b = rest % c.n_seqs;
    part = rest / c.n_seqs % split.parts;
    rank = rest / c.n_seqs / split.parts;
  } else {
    part = rest % split.parts;
    rank = rest / split.parts % tiles;
    b = nth_longest(c, rest / split.parts / tiles, lane);
  }
  const int longer = (tiles + 1) / 2, tile = !zigzag || rank < longer ? tiles - 1 - rank : rank - longer;
  const Sequence s = sequence(c, b);
  const int rows = s.rows * a.group, row0 = tile * ROWS;
  if (row0 >= rows) return;
  const Span span = span_of(a, s, row0, ROWS);
  // chunks of this part: runs, every split.parts-th
  if (part > 0 && part * split.run >= span.chunks) return;
  const int jump = (split.parts - 1) * split.run, run_mask = split.run - 1;
  auto following = [&](int chunk) { return chunk + 1 + (((chunk + 1) & run_mask) == 0 ? jump : 0); };
  auto first_of = [&](int chunk) { return (chunk < span.sink_chunks ? chunk : chunk + span.first - span.sink_chunks) * 64; };

  // this wave's rows
  const int wave_row = row0 + wave * 32;
  const bool has_rows = wave_row < rows;
  const int row = min(wave_row + n, rows - 1), token = token_of(a, row), place = s.first + token;
  const int place_min = s.first + token_of(a, min(wave_row, rows - 1)), place_max = s.first + token_of(a, min(wave_row + 31, rows - 1));
  half8v q[STEPS];
  {
    const __half *x = a.q + (s.row0 + token) * a.ldq + ((long long)kv_head * a.group + row - token * a.group) * dim + h * 8;
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
      q[i] = __builtin_bit_cast(half8v, EXACT || i * 16 < dim ? (uint4v)*reinterpret_cast<const uint4b *>(x + i * 16) : uint4v{0, 0, 0, 0});
  }
  float m = -__builtin_inff(), l = 0.f;
  float16v o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = float16v{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

  // What a thread brings of a chunk: REPS words of keys and of values.  All lanes of a wave bring words of one page, so that its number, address and scale
  // are scalars: of the keys eight tokens (four, sixteen) of a wave are adjacent, of the values a wave takes sixteen tokens, or, where a page
  // holds a whole chunk, the workgroup all of them, so that adjacent lanes read adjacent words.
  const int shift = c.page_shift;
  const bool wide = shift >= 6;
  constexpr int K_STEP = THREADS / KU, V_STEP = THREADS / VU;       // keys and elements from one word of a thread to its next
  const int k_key = tid / KU, k_piece = tid % KU, wave_key = wave * (64 / KU);
  const int v_piece = wide ? tid % VU : wave * BYTES + lane % BYTES, v_d = wide ? tid / VU : lane / BYTES, v_key = v_piece * (16 / BYTES);
  const bool k_has = EXACT || k_piece * 16 < dim * BYTES;
  const unsigned k_offset = (unsigned)((k_key - wave_key) * (dim * BYTES) + (k_has ? k_piece * 16 : 0));
  const unsigned v_offset = (unsigned)((v_d << shift) * BYTES + (wide ? v_piece * 16 : lane % BYTES * 16)), v_step = (unsigned)(V_STEP * BYTES) << shift;
  // (elements behind the head's: its last one again, for outputs that nobody stores)
  auto v_of = [&](int r) { return EXACT ? v_offset : v_offset - ((unsigned)(max(v_d + r * V_STEP - (dim - 1), 0) * BYTES) << shift); };
  uint4v kw[REPS], vw[REPS];
  float ks[REPS], vs = 1.f;
  int k_entry[REPS], v_entry = -1;
  bool v_there = false;
  // (Numbers and scales come by vector loads of one address: scalar loads would share a counter with the reads of LDS and come in any order, so that
  // every wait for LDS behind them would wait for them as well.)
  auto buffer = [](const void *at) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(at), 0, 0xffffffffu, 0x00020000); };
  auto word_at = [](__amdgpu_buffer_rsrc_t from, unsigned lane_offset, unsigned offset) {
    return __builtin_bit_cast(uint4v, __builtin_amdgcn_raw_buffer_load_b128(from, lane_offset, offset, 0));
  };
  auto number_at = [](__amdgpu_buffer_rsrc_t from, unsigned offset) { return __builtin_amdgcn_raw_buffer_load_b32(from, 0, offset, 0); };
  const __amdgpu_buffer_rsrc_t table = buffer(c.page_table + b * c.table_stride), k_scales = buffer(c.k_scales + kv_head), v_scales = buffer(c.v_scales + kv_head);
  const int last_entry = c.table_pages - 1, mask = (1 << shift) - 1;
  int k_place[REPS];                                                // of this wave's keys in a chunk
  unsigned k_in_page[REPS];
#pragma unroll
  for (int r = 0; r < REPS; ++r) {
    k_place[r] = wave_key + r * K_STEP;
    k_in_page[r] = (unsigned)(k_place[r] & mask) * (dim * BYTES);
  }
  const int v_place = wide ? 0 : wave * 16;
  const unsigned v_in_page = (unsigned)(v_place & mask) * BYTES;
  const unsigned char *k_head = c.k_pages + ((long long)kv_head << shift) * (dim * BYTES), *v_head = c.v_pages + (((long long)kv_head * dim) << shift) * BYTES;
  // Entries of the page table; past its end, where no key is, the last one's.
  auto entries = [&](int j0) {
#pragma unroll
    for (int r = 0; r < REPS; ++r) k_entry[r] = (int)number_at(table, (unsigned)min((j0 + k_place[r]) >> shift, last_entry) * 4u);
    v_entry = (int)number_at(table, (unsigned)min((j0 + v_place) >> shift, last_entry) * 4u);
  };
  // (instead of a page that is not there page 0 is read, and what comes of it is not used)
  auto load = [&](int j0) {
    const unsigned in_page = (unsigned)(j0 & mask);
#pragma unroll
    for (int r = 0; r < REPS; ++r) {
      const unsigned entry = (unsigned)__builtin_amdgcn_readfirstlane(k_entry[r]), page = entry < (unsigned)c.n_pages ? entry : 0u;
      kw[r] = word_at(buffer(k_head + (unsigned long long)page * (unsigned)c.k_page_bytes), k_offset, in_page * (dim * BYTES) + k_in_page[r]);
      if (E4M3) ks[r] = __uint_as_float(number_at(k_scales, page * (unsigned)c.kv_heads * 4u));
    }
    const unsigned entry = (unsigned)__builtin_amdgcn_readfirstlane(v_entry);
    v_there = entry < (unsigned)c.n_pages;
    const unsigned page = v_there ? entry : 0u;
    const __amdgpu_buffer_rsrc_t from = buffer(v_head + (unsigned long long)page * (unsigned)c.v_page_bytes);
#pragma unroll
    for (int r = 0; r < REPS; ++r) vw[r] = word_at(from, v_of(r) + (EXACT ? 0u : r * v_step), in_page * BYTES + v_in_page + (EXACT ? r * v_step : 0u));
    if (E4M3) vs = __uint_as_float(number_at(v_scales, page * (unsigned)c.kv_heads * 4u));
  };
  using Zero = std::integral_constant<int, 0>;
  using One = std::integral_constant<int, 1>;
  // Where this thread's words go: slots of sixteen bytes whose number is mixed with the row's, for reads without conflicts.  Its other words lie constant
  // distances further on, and the second half of one that is converted is the neighbour.
  const unsigned lds_at = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)lds;
  const int k_row = row_of_key(k_key);
  unsigned k_to = lds_at + (k_row * SLOTS + ((E4M3 ? 2 * k_piece : k_piece) ^ (SLOTS == 16 ? k_row & 15 : (k_row >> 1) & 7))) * 16;
  unsigned v_to = lds_at + K_BYTES + (v_d * 8 + ((E4M3 ? 2 * v_piece : v_piece) ^ ((v_d >> 1) & 7))) * 16;
  auto put = [](unsigned at, uint4v x) { *(__attribute__((address_space(3))) uint4v *)(size_t)at = x; };
  auto store = [&](int j0, auto into) {
    constexpr int INTO = decltype(into)::value;
    if (!EXACT)
#pragma unroll
      for (int r = 0; r < REPS; ++r) kw[r] = k_has ? kw[r] : uint4v{0, 0, 0, 0};
    if (j0 + 64 > span.end || j0 < span.low || !v_there) {          // values that no row looks at may be anything: cleared
      unsigned keep[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        keep[w] = 0;
#pragma unroll
        for (int r = 0; r < 4 / BYTES; ++r) {
          const int j = j0 + v_key + w * (4 / BYTES) + r;
          if (v_there && j < span.end && (j >= span.low || j < a.sinks)) keep[w] |= (E4M3 ? 0xffu : 0xffffu) << (8 * BYTES * r);
        }
      }
#pragma unroll
      for (int r = 0; r < REPS; ++r) vw[r] &= uint4v{keep[0], keep[1], keep[2], keep[3]};
      if (!(keep[0] | keep[1] | keep[2] | keep[3])) vs = 1.f;         // (the scale may be anything too)
    }
    bool odd = false;
    if (span.place_min != span.place_max && (j0 + 63 > span.place_min || (a.window > 0 && j0 <= span.place_max - a.window))) {
      unsigned bits = lds_at + bits_of(INTO) + v_d * 8 + v_piece * (Odd<E4M3>::KEYS / 8);
      asm volatile("" : "+v"(bits));
#pragma unroll
      for (int r = 0; r < REPS; ++r) {
        odd |= Odd<E4M3>::any(vw[r]);
        unsigned of[Odd<E4M3>::KINDS];
        vw[r] = Odd<E4M3>::clean(vw[r], of);
#pragma unroll
        for (int kind = 0; kind < Odd<E4M3>::KINDS; ++kind) Odd<E4M3>::put(bits + r * V_STEP * 8, kind, D, of[kind]);
        __builtin_amdgcn_sched_barrier(0);                            // (one after the other: registers)
      }
      odd = __ballot(odd) != 0;
    }
    auto words = [&](auto any_wide) {
      constexpr bool WIDE = decltype(any_wide)::value;
#pragma unroll
      for (int r = 0; r < REPS; ++r) {
        const int row = row_of_key(r * K_STEP);                     // how far key k_key + r * K_STEP is from k_key: row 4 has its slots mixed otherwise
        const unsigned mixed = (SLOTS == 16 ? row & 15 : 0) * 16u, k_further = INTO * BUFFER + row * SLOTS * 16, v_further = INTO * BUFFER + r * V_STEP * 8 * 16;
        if constexpr (E4M3) {
          const float by = WIDE ? fminf(ks[r], WIDEST) : ks[r];
          auto value = [&](unsigned a, unsigned b) {
            const half8v x = halves_of_e4m3(a, b, vs);
            return __builtin_bit_cast(uint4v, WIDE ? finite_of(x) : x);
          };
          put((k_to ^ mixed) + k_further, __builtin_bit_cast(uint4v, halves_of_e4m3(kw[r].x, kw[r].y, by)));
          put((k_to ^ mixed ^ 16u) + k_further, __builtin_bit_cast(uint4v, halves_of_e4m3(kw[r].z, kw[r].w, by)));
          put(v_to + v_further, value(vw[r].x, vw[r].y));
          put((v_to ^ 16u) + v_further, value(vw[r].z, vw[r].w));
        } else {
          put((k_to ^ mixed) + k_further, kw[r]);
          put(v_to + v_further, vw[r]);
        }
      }
    };
    float widest = vs;
    if (E4M3)
#pragma unroll
      for (int r = 0; r < REPS; ++r) widest = fmaxf(widest, ks[r]);
    const bool any_wide = E4M3 && __ballot(is_wide(widest)) != 0;
    if (E4M3 && __builtin_expect(any_wide, 0)) {
      words(std::true_type{});
      // What is left of the scales of keys, of which a wave brings sixteen or, of heads of more than 64 elements, eight of every 32.
      if (lane == 0)
#pragma unroll
        for (int r = 0; r < REPS; ++r)
          *(__attribute__((address_space(3))) float *)(size_t)(lds_at + rests_of(INTO) + (r * WAVES + wave) * 4) = rest_of(ks[r]);
    } else {
      words(std::false_type{});
    }
    if (lane == 0) there[INTO * 4 + wave] = (unsigned char)(v_there | odd << 1 | any_wide << 2);
  };

  // first places of the chunks that are computed, stored to LDS and looked up in the page table next
  int chunk = part * split.run, j_now = first_of(chunk), j_next = 0, j_after = 0;
  const bool any = chunk < span.chunks;
  if (any) {
    entries(j_now);
    load(j_now);
    chunk = following(chunk);
    j_next = first_of(chunk);
    entries(j_next);
    store(j_now, Zero{});
  }
  // (the queries have arrived here: a wait for them inside the loop would wait for the next chunk's loads too)
#pragma unroll
  for (int i = 0; i < STEPS; ++i) asm volatile("" : "+v"(q[i]));
  // Where this lane's operands lie in the first buffer; what else an address consists of is a constant.
  auto lds_halves = [](unsigned at) { return *(const __attribute__((address_space(3))) half8v *)(size_t)at; };
  unsigned k_from[STEPS], v_from[4];
#pragma unroll
  for (int st = 0; st < STEPS; ++st) {
    k_from[st] = lds_at + (n * SLOTS + ((2 * st + h) ^ (SLOTS == 16 ? n & 15 : (n >> 1) & 7))) * 16;
    asm volatile("" : "+v"(k_from[st]));
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    v_from[u] = lds_at + K_BYTES + (n * 8 + ((4 * (u >> 1) + 2 * h + (u & 1)) ^ ((n >> 1) & 7))) * 16;
    asm volatile("" : "+v"(v_from[u]));
  }
  __syncthreads();
  // One chunk; whether there is another.  (The buffers take turns; a constant one makes their addresses immediates.)
  auto step = [&](auto of) {
    constexpr int OF = decltype(of)::value;
    const bool more = chunk < span.chunks;
    if (more) {
      load(j_next);
      chunk = following(chunk);
      j_after = first_of(chunk);
      entries(j_after);
    }
    const int j0 = j_now;
    const bool looks = has_rows && j0 <= place_max && (a.window <= 0 || j0 + 63 > place_min - a.window || j0 < a.sinks);
    if (looks) {
      Sixteen sc[2];
      const int pages = *(const __attribute__((address_space(3))) int *)(size_t)(lds_at + 2 * BUFFER + OF * 4);
      __builtin_amdgcn_sched_barrier(0);                           // (in front of the operands: it is waited for alone)
      // operands are read from LDS several products ahead
      half8v f[2 * STEPS];
#pragma unroll
      for (int u = 0; u < 2 * STEPS; ++u) f[u] = lds_halves(k_from[u % STEPS] + OF * BUFFER + u / STEPS * 32 * SLOTS * 16);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float16v x = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < STEPS; ++st) x = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[t * STEPS + st], q[st], x, 0, 0, 0);
        sc[t] = __builtin_bit_cast(Sixteen, x);
      }
      half8v vf[4 * DT];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) vf[dt] = lds_halves(v_from[0] + OF * BUFFER + dt * 32 * 8 * 16);
      __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
      for (int u = 0; u < 2 * STEPS + DT - AHEAD; ++u) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x8, AHEAD - DT, 0);
      const unsigned is = (unsigned)__builtin_amdgcn_readfirstlane(pages);
      if (is != 0x01010101u || j0 + 63 > place_min || j0 + 64 > s.end || (a.window > 0 && j0 <= place_max - a.window)) {
        if (E4M3 && (is & 0x04040404u)) {
          // (what the wave that brought this lane's keys of a tile has left of their scale)
          auto rest_at = [&](int r, int by) {
            return is >> (8 * by) & 4 ? *(const __attribute__((address_space(3))) float *)(size_t)(lds_at + rests_of(OF) + (r * WAVES + by) * 4) : 1.f;
          };
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const float rest = REPS == 1 ? rest_at(0, 2 * t + h) : rest_at(t, 2 * h);
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[t].f[r] *= rest;
          }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const unsigned seen = is >> (16 * t + 8 * h) & 1 ? seen_of(a, s, place, j0 + 32 * t + 16 * h) : 0;
#pragma unroll
          for (int r = 0; r < 16; ++r) sc[t].f[r] = where_seen(seen, r, sc[t].f[r]);
        }
      }
      float top = fmaxf(sc[0].f[0], sc[1].f[0]);
#pragma unroll
      for (int r = 1; r < 16; ++r) top = fmaxf(fmaxf(top, sc[0].f[r]), sc[1].f[r]);
      float low, high;
      across_halves(top, low, high);
      const float now = fmaxf(low, high) * a.scale;
      float base = base_of(m);
      if (__ballot(outgrown(now, m) || is_large(base))) {
        const float next = outgrown(now, m) ? now - BELOW : m, again = __builtin_amdgcn_exp2f(m - base_of(next));
        l *= again;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] *= again;
        m = next;
        base = base_of(next);
        if (is_large(base)) {                                        // (the differences in place of the scores: one more value in the loop costs scalar spills)
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[t].f[r] = (sc[t].f[r] * a.scale - base) * (1.f / a.scale);
          base = 0.f;
        }
      }
      half8v p[2][2];
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float e[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) e[r] = __builtin_amdgcn_exp2f(__fmaf_rn(sc[t].f[8 * u + r], a.scale, -base));
          sum += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
          p[t][u] = half8v{(_Float16)e[0], (_Float16)e[1], (_Float16)e[2], (_Float16)e[3], (_Float16)e[4], (_Float16)e[5], (_Float16)e[6], (_Float16)e[7]};
        }
      l += sum;
#pragma unroll
      for (int u = DT; u < 4 * DT; ++u) vf[u] = lds_halves(v_from[u / DT] + OF * BUFFER + u % DT * 32 * 8 * 16);
#pragma unroll
      for (int u = 0; u < 4 * DT; ++u) o[u % DT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[u], p[u / DT / 2][u / DT % 2], o[u % DT], 0, 0, 0);
#pragma unroll
      for (int u = 0; u < 3 * DT; ++u) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x8, DT, 0);
      if (is & 0x02020202u) {
        const unsigned long long seen = seen64_of(a, s, place, j0);
        unsigned bits = lds_at + bits_of(OF) + h * 4 * 8;
        asm volatile("" : "+v"(bits));
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          Sixteen x = __builtin_bit_cast(Sixteen, o[dt]);
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            x.f[r] += Odd<E4M3>::sum(bits + (32 * dt + 8 * (r >> 2) + (r & 3)) * 8, D, seen);
            if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);
          }
          o[dt] = __builtin_bit_cast(float16v, x);
        }
      }
    }
    if (more) store(j_next, std::integral_constant<int, 1 - OF>{});
    j_now = j_next;
    j_next = j_after;
    __syncthreads();
    return more;
  };
  if (any)
    while (step(Zero{}) && step(One{})) {}

  float low, high;
  across_halves(l, low, high);
  const float total = low + high;
  if (wave_row + n >= rows) return;
  const bool whole = parts_of(split, span.chunks) == 1;
  const float inverse = inverse_of(total);
  const int head = kv_head * a.group + row - token * a.group;
  const long long to = (((long long)b * c.kv_heads + kv_head) * split.parts + part) * ((long long)c.max_new * a.group) + row;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    const Sixteen x = __builtin_bit_cast(Sixteen, o[dt]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int d = 32 * dt + 8 * w + 4 * h;
      if (!EXACT && d >= dim) continue;
      const float y0 = x.f[4 * w], y1 = x.f[4 * w + 1], y2 = x.f[4 * w + 2], y3 = x.f[4 * w + 3];
      if (whole) {
        typedef _Float16 half4b __attribute__((ext_vector_type(4), aligned(2)));
        *reinterpret_cast<half4b *>(a.out + (s.row0 + token) * a.ldo + (long long)head * dim + d) =
            half4b{(_Float16)(y0 * inverse), (_Float16)(y1 * inverse), (_Float16)(y2 * inverse), (_Float16)(y3 * inverse)};
      } else {
        *reinterpret_cast<float4v *>(split.o + to * dim + d) = float4v{y0, y1, y2, y3};
      }
    }
  }
  if (h == 0) {
    if (!whole) *reinterpret_cast<float2v *>(split.ml + to * 2) = float2v{m, total};
    else if (a.lse) a.lse[(long long)(s.row0 + token) * a.q_heads + head] = lse_of(m, total);
  }
}

template <bool E4M3, int D, bool EXACT = true>
int launch(const KvParams &c, const AttentionParams &a, const Split &s, hipStream_t stream) {
  const int tiles = (c.max_new * a.group + ROWS - 1) / ROWS;
  const long long blocks = (long long)c.n_seqs * c.kv_heads * tiles * s.parts;
  if (blocks > 0xffffffffll / THREADS) return VQ_ERR_SHAPE;        // (threads of a grid)
  VQ_ALLOW_FULL_LDS((attention_prompt_kernel<E4M3, D, EXACT>));
  hipLaunchKernelGGL((attention_prompt_kernel<E4M3, D, EXACT>), dim3((unsigned)blocks), dim3(THREADS), 2 * 2 * 64 * D * 2 + 16 + 2 * Odd<E4M3>::KINDS * D * 8 + (E4M3 ? 2 * (D / 64) * WAVES * 4 : 0), stream, c, a, s, tiles,
                     blocks <= 2 * cu_count());
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace

int attention_prompt_rows() { return ROWS; }
bool attention_prompt_takes(const KvParams &c) { return c.head_dim <= 128; }

int launch_attention_prompt(const KvParams &c, const AttentionParams &a, const Split &s, hipStream_t stream) {
  if (c.head_dim < 64) return c.e4m3 ? launch<true, 64, false>(c, a, s, stream) : launch<false, 64, false>(c, a, s, stream);
  if (c.head_dim > 64 && c.head_dim < 128) return c.e4m3 ? launch<true, 128, false>(c, a, s, stream) : launch<false, 128, false>(c, a, s, stream);
  if (c.head_dim == 64) return c.e4m3 ? launch<true, 64>(c, a, s, stream) : launch<false, 64>(c, a, s, stream);
  return c.e4m3 ? launch<true, 128>(c, a, s, stream) : launch<false, 128>(c, a, s, stream);
}

}  // namespace vq
