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

Plan plan_of(const KvParams &c, const AttentionParams &a) {
  Plan p{0, 1, false, 0, 0};
  if (c.head_dim != 64 && c.head_dim != 128) return p;
  const long long rows = (long long)c.max_new * a.group;
  p.prompt = rows > 64;
  p.tile_rows = p.prompt ? attention_prompt_rows() : attention_decode_rows(c, a);
  const long long seen = a.window > 0 ? std::min<long long>(c.max_length, (long long)a.window + a.sinks + p.tile_rows / a.group + 64) : c.max_length;
  const long long chunks = (seen + 63) / 64, groups = (long long)c.n_seqs * c.kv_heads * ((rows + p.tile_rows - 1) / p.tile_rows);
  // Parts until there is a workgroup to a compute unit (of the prompt kernel two), of two runs at least: a second launch costs about 4 us.
  const long long wanted = std::min((p.prompt ? 2LL : 1LL) * cu_count() / groups, chunks / (2 * RUN));
  p.parts = (int)std::max(1LL, std::min(wanted, 64LL));
  if (p.parts > 1) {
    p.o_bytes = (size_t)c.n_seqs * c.kv_heads * p.parts * rows * c.head_dim * 4;
    p.ml_bytes = (size_t)c.n_seqs * c.kv_heads * p.parts * rows * 8;
  }
  return p;
}

}  // namespace

size_t attention_workspace_bytes(const KvParams &c, const AttentionParams &a) {
  const Plan p = plan_of(c, a);
  return (p.o_bytes + p.ml_bytes + 255) / 256 * 256;
}

int launch_attention(const KvParams &c, const AttentionParams &a, void *workspace, size_t workspace_bytes, hipStream_t s) {
  const Plan p = plan_of(c, a);
  if (p.tile_rows) {
    const bool room = p.parts > 1 && workspace_bytes >= p.o_bytes + p.ml_bytes;
    float *o = static_cast<float *>(workspace);
    const Split split{room ? p.parts : 1, o, room ? o + p.o_bytes / 4 : nullptr};
    const int rc = p.prompt ? launch_attention_prompt(c, a, split, s) : launch_attention_decode(c, a, split, s);
    return rc != VQ_OK || !room ? rc : launch_attention_join(c, a, split, p.tile_rows, s);
  }
  const long long blocks = (long long)c.n_seqs * c.max_new * a.q_heads;
  if (blocks > 0x7fffffff) return VQ_ERR_SHAPE;
  if (c.e4m3) hipLaunchKernelGGL((attention_wave_kernel<true>), dim3((unsigned)blocks), dim3(64), 0, s, c, a);
  else hipLaunchKernelGGL((attention_wave_kernel<false>), dim3((unsigned)blocks), dim3(64), 0, s, c, a);
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace vq
