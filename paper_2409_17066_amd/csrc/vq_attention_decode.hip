// Attention of few rows a key head (one token or a few drafted ones, times the query heads that share it) over a paged cache: the decode path.
//
// Bytes of keys and values bound it, so nothing is staged: eight waves of a workgroup take chunks of 64 keys in turn, each lane loading sixteen bytes
// that are already what it feeds to the matrix cores, and the next chunk's keys and values are on their way while this one's are used.  With
// v_mfma_f32_16x16x32_f16 the scores come transposed, S^T = K Q^T: a lane (row n of sixteen, lane group g of four) gets four keys of
// each of the chunk's four tiles.  Which key is which row of a tile is free: key 16 g + 4 tile + r makes a lane's sixteen scores those of keys 16 g ..
// 16 g + 15, and the same lane group then holds exactly these keys of the values, whose tokens lie next to each other in the cache, as
// operand A of O^T = V^T P^T.  Likewise the elements of a head are dealt to the lanes sixteen bytes at a time, in the queries as in the keys.  So there
// are no shuffles but for the maximum over four lane groups, and the running maximum of a row scales registers of the same lane.
//
// Measured, 64 query and 8 key heads of 128 elements, 8 bits: one sequence of 131071 tokens 49 us, 5.5 TB/s (a large copy reaches 4.9 of reads and writes), and 4.6 for the second
// launch that joins its 32 parts; sixteen sequences of up to 4096 21.6 and 3.9, 4.2 TB/s: start-up and the last chunks of the longest.  32
// heads, one sequence of 509 tokens: 7.2, launch and the chain from page table to keys to the join of the waves.  Heads of other sizes (16 sequences of
// 4096 tokens): 80 elements 22, 256 63, whose keys and values are not in registers together.
#include "vq_attention.hpp"

namespace vq {

namespace {

// Waves of a workgroup, at most: as many as have room in LDS for what they join.
constexpr int waves_of(bool e4m3, int dim) { return !e4m3 && dim > 192 ? DECODE_RUN / 2 : DECODE_RUN; }

// RT: tiles of sixteen rows; D: elements of a head, or (not EXACT) the next multiple of 64, zeros behind the head's own; MANY: rows may be of several new
// tokens, which see different keys.
template <bool E4M3, int D, int RT, bool MANY, bool EXACT>
__global__ __launch_bounds__(64 * waves_of(E4M3, D)) void attention_decode_kernel(const KvParams c, const AttentionParams a, const Split split, int tiles, int tile0, int waves) {
  const int dim = EXACT ? D : c.head_dim;
  constexpr int BYTES = E4M3 ? 1 : 2, KL = D * BYTES / 64, VL = BYTES, DT = D / 16, STEPS = D / 32, PITCH = D + 4;
  // The next chunk is loaded ahead where there are registers for it beside those of the rows' differences, and its values where the keys leave them room.
  constexpr bool AHEAD = !MANY || D == 64 || (E4M3 && D <= 128), V_AHEAD = D == 64 || (D == 128 && (EXACT || E4M3));
  static_assert(!AHEAD || V_AHEAD, "the next keys are loaded by page numbers that are asked for in front of them only where the values are");
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  // (tiles of the same keys a multiple of all key heads apart: on the same XCD where those are a multiple of eight)
  const int b = (int)blockIdx.x, kv_head = (int)blockIdx.y, part = tiles > 1 ? (int)blockIdx.z / tiles : (int)blockIdx.z, tile = tile0 + (tiles > 1 ? (int)blockIdx.z % tiles : 0);
  const int shift = c.page_shift, mask = (1 << shift) - 1;
  // Entries of the page table for places [of, of + 16).  Without a window the first ones do not depend on the sequence's length, and are asked for beside it.
  auto entry = [&](int of) { return of >> shift < c.table_pages ? c.page_table[b * c.table_stride + (of >> shift)] : -1; };
  int i = part * waves + wave, k_entry = 0, v_entry = 0;
  float *ml = lds, *out = lds + 2 * 16 * waves, *put_back = out;      // (a wave's first part of put_back is read before its results take the place)
  bool any_odd = false;
  if (a.window == 0) {
    k_entry = entry(i * 64 + 16 * (n >> 2));
    v_entry = entry(i * 64 + 16 * g);
  }
  const Sequence s = sequence(c, b);
  const int rows = s.rows * a.group, row0 = tile * 16 * RT, here = min(rows - row0, 16 * RT);
  if (here <= 0) return;
  const Span span = span_of(a, s, row0, 16 * RT);
  const int begin = part * waves, end = span.chunks, stride = split.parts * waves;
  if (part > 0 && begin >= end) return;
  const int active = min(max(end - begin, 0), waves);            // waves that have a chunk
  if (a.window != 0 && i < end) {
    k_entry = entry(span.chunk(i) * 64 + 16 * (n >> 2));
    v_entry = entry(span.chunk(i) * 64 + 16 * g);
  }

  // the rows of this lane: new token, query head, place
  half8v q[RT][STEPS];
  int place[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = min(row0 + rt * 16 + n, rows - 1), t = token_of(a, r);
    place[rt] = s.first + t;
    const __half *x = a.q + (s.row0 + t) * a.ldq + ((long long)kv_head * a.group + r - t * a.group) * dim;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int at = E4M3 ? (i >> 1) * 64 + g * 16 + (i & 1) * 8 : i * 32 + g * 8;
      const uint4v w = *reinterpret_cast<const uint4b *>(x + (EXACT || at < dim ? at : 0));
      q[rt][i] = __builtin_bit_cast(half8v, EXACT || at < dim ? w : uint4v{0, 0, 0, 0});
    }
  }

  float m[RT], l[RT];
  float4v o[RT][DT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = -__builtin_inff();
    l[rt] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[rt][dt] = float4v{0.f, 0.f, 0.f, 0.f};
  }

  // page of sixteen places where a row looks at some of them, else page 0, whose contents are not used (nor its scale: it may be anything)
  auto page_at = [&](int of, int entry, bool &there) {
    there = (unsigned)entry < (unsigned)c.n_pages && of < span.end && (of + 15 >= span.low || of < a.sinks);
    return there ? entry : 0;
  };
  uint4v k[4][KL], v[DT][VL];
  auto has = [&](int dt) {                                         // whether the head has elements 16 dt ... 16 dt + 15
    int of = dim;
    if (!EXACT) asm volatile("" : "+s"(of));                       // (compared where it is asked: kept from round to round it would be two scalar registers for each)
    return EXACT || dt * 16 < of;
  };
  float k_scale = 1.f, v_scale = 1.f;
  bool v_there = false;
  auto entries_of = [&](int i) {
    k_entry = entry(span.chunk(i) * 64 + 16 * (n >> 2));
    v_entry = entry(span.chunk(i) * 64 + 16 * g);
  };
  auto load_k = [&](int i) {
    const int j = span.chunk(i) * 64 + 16 * (n >> 2);
    bool there;
    const int page = page_at(j, k_entry, there);
    const unsigned char *from = c.k_pages + page * c.k_page_bytes;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int w = 0; w < KL; ++w) {
        const uint4v x = *reinterpret_cast<const uint4v *>(from + key_word_at(kv_head, shift, j, t, w, n, g, dim * BYTES));
        k[t][w] = EXACT || w * 64 + g * 16 < dim * BYTES ? x : uint4v{0, 0, 0, 0};
      }
    if (E4M3) k_scale = c.k_scales[(long long)page * c.kv_heads + kv_head];
  };
  auto load_v = [&](int i) {
    const int j = span.chunk(i) * 64 + 16 * g;
    const int page = page_at(j, v_entry, v_there);
    const unsigned char *from = c.v_pages + page * c.v_page_bytes + (((((long long)kv_head * dim + n) << shift) + (j & mask)) * BYTES);
    const int step = 16 * BYTES << shift;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int w = 0; w < VL; ++w) v[dt][w] = has(dt) ? *reinterpret_cast<const uint4v *>(from + dt * step + w * 16) : uint4v{0, 0, 0, 0};
    if (E4M3) v_scale = v_there ? c.v_scales[(long long)page * c.kv_heads + kv_head] : 1.f;
  };

  if (V_AHEAD && i < end) {
    load_k(i);
    load_v(i);
  }
  for (; i < end; i += stride) {
    const int j0 = span.chunk(i) * 64, next = i + stride;
    if (V_AHEAD && next < end) entries_of(next);
    if (!V_AHEAD) load_k(i);
    float4v sc[RT][4];
    bool odd = false;
    const float k_by = E4M3 ? fminf(k_scale, WIDEST) : 1.f;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      half8v f[STEPS];
#pragma unroll
      for (int w = 0; w < KL; ++w) {
        if constexpr (E4M3) {
          f[2 * w] = halves_of_e4m3(k[t][w].x, k[t][w].y, k_by);
          f[2 * w + 1] = halves_of_e4m3(k[t][w].z, k[t][w].w, k_by);
        } else {
          f[w] = __builtin_bit_cast(half8v, k[t][w]);
        }
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float4v x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < STEPS; ++w) x = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[w], q[rt][w], x, 0, 0, 0);
        sc[rt][t] = x;
      }
    }
    if (E4M3 && __builtin_expect(__ballot(is_wide(k_scale)) != 0, 0)) {
      const float rest = rest_of(__shfl(k_scale, 4 * g));           // (that lane has loaded keys of this one's sixteen)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int t = 0; t < 4; ++t) sc[rt][t] *= rest;
    }
    if (AHEAD && next < end) load_k(next);
    if (!V_AHEAD) {
      __builtin_amdgcn_sched_barrier(0);                           // (not beside the keys: registers)
      load_v(i);
      if (next < end) entries_of(next);
    }
    // keys that some row does not see: hidden from it; those that no row sees may hold anything, so their values are cleared
    const bool all_there = __ballot(!v_there) == 0;
    if (!all_there || j0 + 63 > span.place_min || j0 + 64 > s.end || (a.window > 0 && j0 <= span.place_max - a.window)) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const unsigned seen = v_there ? seen_of(a, s, place[rt], j0 + 16 * g) : 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float4v x = sc[rt][t];
          sc[rt][t] = float4v{where_seen(seen, 4 * t, x.x), where_seen(seen, 4 * t + 1, x.y), where_seen(seen, 4 * t + 2, x.z), where_seen(seen, 4 * t + 3, x.w)};
        }
      }
      unsigned keep[4 * VL];
#pragma unroll
      for (int w = 0; w < 4 * VL; ++w) {
        keep[w] = 0;
#pragma unroll
        for (int r = 0; r < 4 / BYTES; ++r) {
          const int j = j0 + 16 * g + w * (4 / BYTES) + r;
          if (v_there && j < span.end && (j >= span.low || j < a.sinks)) keep[w] |= (E4M3 ? 0xffu : 0xffffu) << (8 * BYTES * r);
        }
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int w = 0; w < VL; ++w) v[dt][w] &= uint4v{keep[4 * w], keep[4 * w + 1], keep[4 * w + 2], keep[4 * w + 3]};
      if (MANY && span.place_min != span.place_max) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int w = 0; w < VL; ++w) odd |= Odd<E4M3>::any(v[dt][w]);
        odd = __ballot(odd) != 0;
        if (odd) {
          unsigned bits = (unsigned)(size_t)(__attribute__((address_space(3))) float *)(put_back + RT * waves * 16 * PITCH) + wave * (Odd<E4M3>::KINDS * D * 8) + n * 8 + g * 2;
          asm volatile("" : "+v"(bits));
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int w = 0; w < VL; ++w) {
              unsigned of[Odd<E4M3>::KINDS];
              v[dt][w] = Odd<E4M3>::clean(v[dt][w], of);
#pragma unroll
              for (int kind = 0; kind < Odd<E4M3>::KINDS; ++kind) Odd<E4M3>::put(bits + dt * 16 * 8 + w, kind, D, of[kind]);
              __builtin_amdgcn_sched_barrier(0);                    // (one after the other: registers)
            }
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          __builtin_amdgcn_wave_barrier();
        }
      }
    }
    half8v p[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float top = fmaxf(fmaxf(fmaxf(sc[rt][0].x, sc[rt][0].y), fmaxf(sc[rt][0].z, sc[rt][0].w)), fmaxf(fmaxf(sc[rt][1].x, sc[rt][1].y), fmaxf(sc[rt][1].z, sc[rt][1].w)));
      top = fmaxf(top, fmaxf(fmaxf(fmaxf(sc[rt][2].x, sc[rt][2].y), fmaxf(sc[rt][2].z, sc[rt][2].w)), fmaxf(fmaxf(sc[rt][3].x, sc[rt][3].y), fmaxf(sc[rt][3].z, sc[rt][3].w))));
      const float now = rows_max(top) * a.scale;
      if (__ballot(outgrown(now, m[rt]))) {
        const float next = outgrown(now, m[rt]) ? now - BELOW : m[rt], again = __builtin_amdgcn_exp2f(m[rt] - base_of(next));
        l[rt] *= again;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[rt][dt] *= again;
        m[rt] = next;
      }
      const float base = base_of(m[rt]);
      float scale = a.scale;
      if (__builtin_expect(is_large(base), 0)) {
#pragma unroll
        for (int t = 0; t < 4; ++t) sc[rt][t] *= a.scale;
        scale = 1.f;
      }
      float sum = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float e[8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float4v x = sc[rt][2 * h + u];
          e[4 * u] = __builtin_amdgcn_exp2f(__fmaf_rn(x.x, scale, -base));
          e[4 * u + 1] = __builtin_amdgcn_exp2f(__fmaf_rn(x.y, scale, -base));
          e[4 * u + 2] = __builtin_amdgcn_exp2f(__fmaf_rn(x.z, scale, -base));
          e[4 * u + 3] = __builtin_amdgcn_exp2f(__fmaf_rn(x.w, scale, -base));
        }
        sum += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
        // (rounded to nearest: what the matrix cores take; the sum is that of the unrounded ones)
        p[rt][h] = half8v{(_Float16)e[0], (_Float16)e[1], (_Float16)e[2], (_Float16)e[3], (_Float16)e[4], (_Float16)e[5], (_Float16)e[6], (_Float16)e[7]};
      }
      l[rt] += sum;
    }
    if (E4M3 && __builtin_expect(__ballot(is_wide(v_scale)) != 0, 0)) {
      const _Float16 two = is_wide(v_scale) ? (_Float16)2.f : (_Float16)1.f;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int h = 0; h < 2; ++h) p[rt][h] *= half8v{two, two, two, two, two, two, two, two};
      if (is_wide(v_scale)) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int w = 0; w < VL; ++w) v[dt][w] = uint4v{limited(v[dt][w].x, v_scale), limited(v[dt][w].y, v_scale), limited(v[dt][w].z, v_scale), limited(v[dt][w].w, v_scale)};
        v_scale *= 0.5f;
      }
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      half8v f[2];
      if (!has(dt)) continue;
      if constexpr (E4M3) {
        f[0] = halves_of_e4m3(v[dt][0].x, v[dt][0].y, v_scale);
        f[1] = halves_of_e4m3(v[dt][0].z, v[dt][0].w, v_scale);
      } else {
        f[0] = __builtin_bit_cast(half8v, v[dt][0]);
        f[1] = __builtin_bit_cast(half8v, v[dt][VL - 1]);
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        o[rt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[0], p[rt][0], o[rt][dt], 0, 0, 0);
        o[rt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[1], p[rt][1], o[rt][dt], 0, 0, 0);
      }
    }
    if (MANY && odd) {                                             // (to LDS, and from there to the outputs behind the loop: beside what is loaded there are no registers)
      const unsigned bits = (unsigned)(size_t)(__attribute__((address_space(3))) float *)(put_back + RT * waves * 16 * PITCH) + wave * (Odd<E4M3>::KINDS * D * 8) + g * 4 * 8;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const unsigned long long seen = seen64_of(a, s, place[rt], j0);
        for (int dt = 0; dt < DT && has(dt); ++dt) {
          const unsigned at = bits + dt * 16 * 8;
          float4v *to = reinterpret_cast<float4v *>(put_back + ((rt * waves + wave) * 16 + n) * PITCH + dt * 16 + g * 4);
          const float4v x = {Odd<E4M3>::sum(at, D, seen), Odd<E4M3>::sum(at + 8, D, seen), Odd<E4M3>::sum(at + 16, D, seen), Odd<E4M3>::sum(at + 24, D, seen)};
          *to = any_odd ? *to + x : x;
        }
      }
      any_odd = true;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    if (next < end) {
      if (V_AHEAD && !AHEAD) load_k(next);
      if (V_AHEAD) load_v(next);
    }
  }

  // the waves' results, joined through LDS, sixteen rows at a time
  const bool whole = parts_of(split, span.chunks) == 1;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int left = here - rt * 16;
    if (left <= 0) break;
    __syncthreads();
    if (MANY && any_odd) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[rt][dt] += *reinterpret_cast<const float4v *>(put_back + ((rt * waves + wave) * 16 + n) * PITCH + dt * 16 + g * 4);
    }
    const float sum = rows_sum(l[rt]);
    if (wave < active && lane < 16) {
      ml[2 * (wave * 16 + n)] = m[rt];
      ml[2 * (wave * 16 + n) + 1] = sum;
    }
    if (wave < active && n < left) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<float4v *>(out + (wave * 16 + n) * PITCH + dt * 16 + g * 4) = o[rt][dt];
    }
    __syncthreads();
    for (int u = (int)threadIdx.x; u < min(left, 16) * (D / 4); u += 64 * waves) {
      const int r = u / (D / 4), d = (u - r * (D / 4)) * 4;
      if (!EXACT && d >= dim) continue;
      float top = -__builtin_inff();
      for (int w = 0; w < active; ++w) top = fmaxf(top, ml[2 * (w * 16 + r)]);
      const float base = base_of(top);
      float total = 0.f;
      float4v x = {0.f, 0.f, 0.f, 0.f};
      for (int w = 0; w < active; ++w) {
        const float f = __builtin_amdgcn_exp2f(ml[2 * (w * 16 + r)] - base);
        total = __fmaf_rn(ml[2 * (w * 16 + r) + 1], f, total);
        const float4v y = *reinterpret_cast<const float4v *>(out + (w * 16 + r) * PITCH + d);
        x.x = __fmaf_rn(y.x, f, x.x); x.y = __fmaf_rn(y.y, f, x.y); x.z = __fmaf_rn(y.z, f, x.z); x.w = __fmaf_rn(y.w, f, x.w);
      }
      const int row = row0 + rt * 16 + r;
      if (whole) {
        const int t = token_of(a, row), head = kv_head * a.group + row - t * a.group;
        x *= inverse_of(total);
        typedef _Float16 half4b __attribute__((ext_vector_type(4), aligned(2)));
        *reinterpret_cast<half4b *>(a.out + (s.row0 + t) * a.ldo + (long long)head * dim + d) = half4b{(_Float16)x.x, (_Float16)x.y, (_Float16)x.z, (_Float16)x.w};
        if (a.lse && d == 0) a.lse[(long long)(s.row0 + t) * a.q_heads + head] = lse_of(top, total);
      } else {
        const long long to = (((long long)b * c.kv_heads + kv_head) * split.parts + part) * ((long long)c.max_new * a.group) + row;
        *reinterpret_cast<float4v *>(split.o + to * dim + d) = x;
        if (d == 0) *reinterpret_cast<float2v *>(split.ml + to * 2) = float2v{top, total};
      }
    }
  }
}

// Joins the parts of a sequence's keys: a workgroup to a row, whose threads take four elements of a share of the parts each.  D: elements of a head, or more.
constexpr int JOIN_THREADS = 256;

template <int D>
__global__ __launch_bounds__(JOIN_THREADS) void attention_join_kernel(const KvParams c, const AttentionParams a, const Split split, int tile_rows) {
  constexpr int LANES = D / 4, SHARES = JOIN_THREADS / LANES;
  __shared__ __attribute__((aligned(16))) float shares[SHARES][D];
  __shared__ float factors[64];
  const int rows_most = c.max_new * a.group, dim = c.head_dim, lane = (int)threadIdx.x & 63;
  const int row = (int)blockIdx.x, kv_head = (int)blockIdx.y, b = (int)blockIdx.z;
  const long long from = ((long long)b * c.kv_heads + kv_head) * split.parts * rows_most + row;
  // lane w < parts of every wave takes part w's maximum and sum (64 parts at most); loaded, as the outputs are, before it is known how many there are
  const float2v mine = lane < split.parts ? *reinterpret_cast<const float2v *>(split.ml + (from + (long long)lane * rows_most) * 2) : float2v{0.f, 0.f};
  const int share = (int)threadIdx.x / LANES, d = (int)(threadIdx.x % LANES) * 4;
  float4v y[4];
  auto load = [&](int w0) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int w = w0 + u * SHARES;
      y[u] = w < split.parts && d < dim ? *reinterpret_cast<const float4v *>(split.o + (from + (long long)w * rows_most) * dim + d) : float4v{0.f, 0.f, 0.f, 0.f};
    }
  };
  load(share);
  const Sequence s = sequence(c, b);
  if (row >= s.rows * a.group) return;
  const int parts = parts_of(split, span_of(a, s, row & -tile_rows, tile_rows).chunks);
  if (parts == 1) return;                                        // written already
  const float m = lane < parts ? mine.x : -__builtin_inff();
  float top = m;
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
  const float f = __builtin_amdgcn_exp2f(m - base_of(top)), total = wave_sum(lane < parts ? mine.y * f : 0.f);
  if (threadIdx.x < 64) factors[lane] = f;
  __syncthreads();
  float4v x = {0.f, 0.f, 0.f, 0.f};
  for (int w0 = share; w0 < parts; w0 += 4 * SHARES) {
    if (w0 != share) load(w0);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int w = w0 + u * SHARES;
      if (w >= parts) break;                                     // (what is there was not written by this call)
      const float fw = factors[w];
      x.x = __fmaf_rn(y[u].x, fw, x.x); x.y = __fmaf_rn(y[u].y, fw, x.y); x.z = __fmaf_rn(y[u].z, fw, x.z); x.w = __fmaf_rn(y[u].w, fw, x.w);
    }
  }
  *reinterpret_cast<float4v *>(&shares[share][d]) = x;
  __syncthreads();
  const int t = token_of(a, row), head = kv_head * a.group + row - t * a.group;
  if ((int)threadIdx.x < dim) {
    float y = 0.f;
#pragma unroll
    for (int w = 0; w < SHARES; ++w) y += shares[w][threadIdx.x];
    a.out[(s.row0 + t) * a.ldo + (long long)head * dim + threadIdx.x] = __float2half_rn(y * inverse_of(total));
  }
  if (a.lse && threadIdx.x == 0) a.lse[(long long)(s.row0 + t) * a.q_heads + head] = lse_of(top, total);
}

template <bool E4M3, int D, int RT, bool MANY, bool EXACT = true>
int launch(const KvParams &c, const AttentionParams &a, const Split &s, hipStream_t stream) {
  const int waves = attention_decode_waves(c, s.parts);
  const int tiles = (c.max_new * a.group + 16 * RT - 1) / (16 * RT), most = 65535 / s.parts;     // (more tiles than a grid has layers: several launches)
  if (c.n_seqs > 0x7fffffff / 512) return VQ_ERR_SHAPE;
  const int lds = (2 * 16 + 16 * (D + 4) * (MANY ? RT : 1)) * waves * 4 + (MANY ? waves * Odd<E4M3>::KINDS * D * 8 : 0);
  VQ_ALLOW_FULL_LDS((attention_decode_kernel<E4M3, D, RT, MANY, EXACT>));
  for (int tile0 = 0; tile0 < tiles; tile0 += most) {
    const int now = tiles - tile0 < most ? tiles - tile0 : most;
    hipLaunchKernelGGL((attention_decode_kernel<E4M3, D, RT, MANY, EXACT>), dim3(c.n_seqs, c.kv_heads, now * s.parts), dim3(64 * waves), lds, stream, c, a, s, now, tile0, waves);
  }
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace

// Two tiles share the conversions and loads of a chunk, where the registers are there: not beside 64 of a 16-bit chunk's keys and as many of its values, nor
// (heads of 128 elements) beside what rows of several tokens need.
int attention_decode_rows(const KvParams &c, const AttentionParams &a) {
  return (long long)c.max_new * a.group > 16 && (c.head_dim == 64 || (c.head_dim == 128 && c.e4m3 && c.max_new == 1)) ? 32 : 16;
}
// Where no sequence has a chunk for every wave, no more waves than chunks: more workgroups share a compute unit (8 bits: 36 sequences of up to 13
// tokens, 32 heads of 64 elements, 10.9 us by eight waves and 7.0 by one; 64 of 250 tokens, 8 key heads of 128, 12.7 by eight and 9.4 by four).
int attention_decode_waves(const KvParams &c, int parts) {
  int waves = waves_of(c.e4m3, c.head_dim);
  while (parts == 1 && waves > 1 && c.max_length <= 32 * waves) waves /= 2;
  return waves;
}
int attention_decode_run(const KvParams &c) { return waves_of(c.e4m3, c.head_dim); }

template <bool MANY>
static int launch_decode(const KvParams &c, const AttentionParams &a, const Split &s, hipStream_t stream) {
  const bool two = attention_decode_rows(c, a) == 32;
  if (c.head_dim == 64) return c.e4m3 ? (two ? launch<true, 64, 2, MANY>(c, a, s, stream) : launch<true, 64, 1, MANY>(c, a, s, stream))
                                      : (two ? launch<false, 64, 2, MANY>(c, a, s, stream) : launch<false, 64, 1, MANY>(c, a, s, stream));
  if constexpr (!MANY)
    if (two) return launch<true, 128, 2, MANY>(c, a, s, stream);
  return c.e4m3 ? launch<true, 128, 1, MANY>(c, a, s, stream) : launch<false, 128, 1, MANY>(c, a, s, stream);
}

// Heads of other sizes: rows of one token as well by what takes several.
template <int D>
static int launch_padded(const KvParams &c, const AttentionParams &a, const Split &s, hipStream_t stream) {
  return c.e4m3 ? launch<true, D, 1, true, false>(c, a, s, stream) : launch<false, D, 1, true, false>(c, a, s, stream);
}

int launch_attention_decode(const KvParams &c, const AttentionParams &a, const Split &s, hipStream_t stream) {
  if (c.head_dim != 64 && c.head_dim != 128)
    return c.head_dim < 64 ? launch_padded<64>(c, a, s, stream) : c.head_dim < 128 ? launch_padded<128>(c, a, s, stream) :
           c.head_dim <= 192 ? launch_padded<192>(c, a, s, stream) : launch_padded<256>(c, a, s, stream);
  return c.max_new > 1 ? launch_decode<true>(c, a, s, stream) : launch_decode<false>(c, a, s, stream);
}

bool attention_join_takes(const KvParams &c, const AttentionParams &a) {
  return c.n_seqs <= 65535 && (long long)c.max_new * a.group <= 0xffffffffll / JOIN_THREADS;
}
int launch_attention_join(const KvParams &c, const AttentionParams &a, const Split &s, int tile_rows, hipStream_t stream) {
  const dim3 blocks(c.max_new * a.group, c.kv_heads, c.n_seqs);
  auto kernel = c.head_dim <= 64 ? attention_join_kernel<64> : c.head_dim <= 128 ? attention_join_kernel<128> : attention_join_kernel<256>;
  hipLaunchKernelGGL(kernel, blocks, dim3(JOIN_THREADS), 0, stream, c, a, s, tile_rows);
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace vq
