// Attention of new tokens over a paged cache: dispatch, and the kernel that takes every layout.
#include "vq_attention.hpp"
#include <algorithm>

namespace vq {

namespace {

// One wave to a new token and query head, 64 keys at a time: a lane computes one key's score, the wave the running maximum and sum, and then
// each lane up to four elements of the output.
constexpr int MOST_DIM = 256;

template <bool E4M3>
__global__ __launch_bounds__(64) void attention_wave_kernel(const KvParams c, const AttentionParams a) {
  __shared__ __attribute__((aligned(16))) float q[MOST_DIM];
  __shared__ __attribute__((aligned(16))) float p[64];
  const int lane = (int)threadIdx.x, d_all = c.head_dim, head = (int)blockIdx.x % a.q_heads, t = (int)blockIdx.x / a.q_heads % c.max_new,
            b = (int)(blockIdx.x / a.q_heads / c.max_new);
  const Sequence s = sequence(c, b);
  if (t >= s.rows) return;
  const long long row = s.row0 + t;
  const int place = s.first + t, keys = min(place + 1, s.end), low = a.window > 0 ? max(place - a.window + 1, 0) : 0;
  const int kv_head = head / a.group, size = 1 << c.page_shift;
  for (int d = lane; d < d_all; d += 64) q[d] = __half2float(a.q[row * a.ldq + (long long)head * d_all + d]);
  float m = -__builtin_inff(), l = 0.f, o[MOST_DIM / 64] = {};
  const int sink_chunks = (min(a.sinks, low) + 63) / 64;
  for (int j0 = sink_chunks ? 0 : low & ~63; j0 < keys; j0 = j0 + 64 < sink_chunks * 64 ? j0 + 64 : max(j0 + 64, low & ~63)) {
    const int j = j0 + lane;
    bool sees = j < keys && (j >= low || j < a.sinks);
    const int page = sees ? page_of(c, b, j >> c.page_shift) : -1;
    sees = page >= 0;
    float score = -__builtin_inff();
    __syncthreads();
    if (sees) {
      float dot = 0.f;
      const unsigned char *k = c.k_pages + page * c.k_page_bytes + ((long long)(kv_head << c.page_shift) + (j & (size - 1))) * d_all * (E4M3 ? 1 : 2);
      const float scale = E4M3 ? c.k_scales[(long long)page * c.kv_heads + kv_head] : 1.f;
      for (int d = 0; d < d_all; d += E4M3 ? 16 : 8) {
        const uint4v u = *reinterpret_cast<const uint4v *>(k + d * (E4M3 ? 1 : 2));
        const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (E4M3) {
            const half2v lo = halves_of_e4m3<false>(w[i], scale), hi = halves_of_e4m3<true>(w[i], scale);
            dot = __fmaf_rn((float)lo.x, q[d + 4 * i], dot);
            dot = __fmaf_rn((float)lo.y, q[d + 4 * i + 1], dot);
            dot = __fmaf_rn((float)hi.x, q[d + 4 * i + 2], dot);
            dot = __fmaf_rn((float)hi.y, q[d + 4 * i + 3], dot);
          } else {
            const half2v x = half2_of(w[i]);
            dot = __fmaf_rn((float)x.x, q[d + 2 * i], dot);
            dot = __fmaf_rn((float)x.y, q[d + 2 * i + 1], dot);
          }
        }
      }
      score = dot * a.scale;
    }
    float top = score;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
    const float now = fmaxf(m, top), base = now == -__builtin_inff() ? 0.f : now;
    const float again = exp2f(m - base), mine = exp2f(score - base);
    p[lane] = mine;
    l = l * again + wave_sum(mine);
    m = now;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MOST_DIM / 64; ++i) o[i] *= again;
    const unsigned long long seen = __ballot(sees);
    for (int k = 0; k < 64; ++k) {
      if (!(seen >> k & 1)) continue;                       // (what nobody sees may hold anything)
      const int at = j0 + k, of = __builtin_amdgcn_readlane(page, k);
      const float scale = E4M3 ? c.v_scales[(long long)of * c.kv_heads + kv_head] : 1.f;
      const unsigned char *v = c.v_pages + of * c.v_page_bytes + (long long)(kv_head << c.page_shift) * d_all * (E4M3 ? 1 : 2);
#pragma unroll
      for (int i = 0; i < MOST_DIM / 64; ++i) {
        const int d = lane + 64 * i;
        if (d >= d_all) break;
        const int element = (d << c.page_shift) + (at & (size - 1));
        const float x = E4M3 ? (float)halves_of_e4m3<false>(v[element], scale).x : __half2float(reinterpret_cast<const __half *>(v)[element]);
        o[i] = __fmaf_rn(p[k], x, o[i]);
      }
    }
  }
  const float inverse = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;      // (a sum that is not a number stays one)
#pragma unroll
  for (int i = 0; i < MOST_DIM / 64; ++i) {
    const int d = lane + 64 * i;
    if (d < d_all) a.out[row * a.ldo + (long long)head * d_all + d] = __float2half_rn(o[i] * inverse);
  }
  if (a.lse && lane == 0) a.lse[row * a.q_heads + head] = l == 0.f ? -__builtin_inff() : (m + __log2f(l)) * 0.6931471805599453f;
}

}  // namespace

namespace {

// How a call is taken: `tile_rows` rows of a key head to a workgroup (0: the wave kernel), by the prompt or the decode kernel, the keys in up to `parts` parts.
struct Plan {
  int tile_rows, parts;
  bool prompt;
  size_t o_bytes, ml_bytes;
};

// The kernel and number of parts whose time is estimated the least, in us, from measurements on heads of 64 and 128 elements, 8 and 16 bits, 8 and 32 key heads,
// 1 to 16 sequences of 1024 to 32768 tokens with 16 to 256 rows a key head:
//   decode: a workgroup to a compute unit, rounds of 3.2 us for eight chunks of 16 KB (more bytes take longer, and more rows more workgroups) behind 9 us;
//   prompt: two to a compute unit, 1.3 us a chunk of both for up to 32 rows and 0.6 more for each further 32 of 128, behind 12 us, and where there is one
//   alone 1.3 and 0.1 (half of that for 64 elements);
// and for parts the second launch that joins them, 5 us and what it moves.  Measured (64 query and 8 key heads of 128 elements, 8 bits, us by the decode and by
// the prompt kernel): 16 sequences of 4096 tokens 32 and 38 for 32 rows a key head, 59 and 49 for 64, 218 and 99 for 256; one of 1024 tokens 13 and 16 for 32
// rows, 13 and 19 for 256.  Parts (16 rows): 4 sequences of 2048 tokens 17 in one and 14 in four, one of 1024 13 in one and 14 in two.
Plan plan_of(const KvParams &c, const AttentionParams &a, bool parts_allowed) {
  Plan best{0, 1, false, 0, 0};
  if (c.head_dim != 64 && c.head_dim != 128) return best;
  const long long rows = (long long)c.max_new * a.group, slots = cu_count();
  float least = 0.f;
  for (const bool prompt : {false, true}) {
    if (!prompt && rows > 512) continue;
    const int tile = prompt ? attention_prompt_rows() : attention_decode_rows(c, a), run = prompt ? PROMPT_RUN : DECODE_RUN;
    // tokens that a tile's rows look at: a window's and the first ones, or on the average all before half of the new ones
    const long long all = c.max_length - (rows > tile ? c.max_new / 2 : 0), reach = a.window > 0 ? (long long)a.window + a.sinks + tile / a.group + 64 : all;
    const long long chunks = (std::max(std::min(all, reach), 1LL) + 63) / 64, groups = (long long)c.n_seqs * c.kv_heads * ((rows + tile - 1) / tile);
    const float quarters = (float)std::min((rows + 31) / 32, 4LL), size = (float)c.head_dim / 128.f;
    const long long most = parts_allowed ? std::min((chunks + run - 1) / run, 64LL) : 1;
    for (long long parts = 1;; parts *= 2) {
      parts = std::min(parts, most);
      const float rounds = std::max((float)(groups * parts) / (float)((prompt ? 2 : 1) * slots), 1.f), runs = (float)(((chunks + run - 1) / run + parts - 1) / parts);
      const float step = !prompt ? 3.2f * size * (c.e4m3 ? 1.f : 2.f) : run * size * (groups * parts > slots ? 0.7f + 0.6f * quarters : 1.2f + 0.1f * quarters);
      const float join = parts > 1 ? 5.f + (float)(c.n_seqs * parts * c.kv_heads * rows) * size * 1024.f / 4.5e6f : 0.f;
      const float time = (prompt ? 12.f : 9.f) + join + rounds * runs * step;
      if (least == 0.f || time < least) {
        least = time;
        best.tile_rows = tile;
        best.parts = (int)parts;
        best.prompt = prompt;
      }
      if (parts == most) break;
    }
  }
  if (best.parts > 1) {
    best.o_bytes = (size_t)c.n_seqs * c.kv_heads * best.parts * rows * c.head_dim * 4;
    best.ml_bytes = (size_t)c.n_seqs * c.kv_heads * best.parts * rows * 8;
  }
  return best;
}

}  // namespace

size_t attention_workspace_bytes(const KvParams &c, const AttentionParams &a) {
  const Plan p = plan_of(c, a, true);
  return (p.o_bytes + p.ml_bytes + 255) / 256 * 256;
}

int launch_attention(const KvParams &c, const AttentionParams &a, void *workspace, size_t workspace_bytes, hipStream_t s) {
  Plan p = plan_of(c, a, true);
  if (p.parts > 1 && workspace_bytes < p.o_bytes + p.ml_bytes) p = plan_of(c, a, false);
  if (p.tile_rows) {
    float *o = static_cast<float *>(workspace);
    const Split split{p.parts, p.prompt ? PROMPT_RUN : DECODE_RUN, o, p.parts > 1 ? o + p.o_bytes / 4 : nullptr};
    const int rc = p.prompt ? launch_attention_prompt(c, a, split, s) : launch_attention_decode(c, a, split, s);
    return rc != VQ_OK || p.parts == 1 ? rc : launch_attention_join(c, a, split, p.tile_rows, s);
  }
  const long long blocks = (long long)c.n_seqs * c.max_new * a.q_heads;
  if (blocks > 0xffffffffll / 64) return VQ_ERR_SHAPE;
  if (c.e4m3) hipLaunchKernelGGL((attention_wave_kernel<true>), dim3((unsigned)blocks), dim3(64), 0, s, c, a);
  else hipLaunchKernelGGL((attention_wave_kernel<false>), dim3((unsigned)blocks), dim3(64), 0, s, c, a);
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace vq
