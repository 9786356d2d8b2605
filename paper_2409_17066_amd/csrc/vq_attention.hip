// Attention of new tokens over a paged cache: dispatch, and the kernel that takes every layout.
#include "vq_kv.hpp"

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

size_t attention_workspace_bytes(const KvParams &, const AttentionParams &) { return 0; }

int launch_attention(const KvParams &c, const AttentionParams &a, void *, size_t, hipStream_t s) {
  const long long blocks = (long long)c.n_seqs * c.max_new * a.q_heads;
  if (blocks > 0x7fffffff) return VQ_ERR_SHAPE;
  if (c.e4m3) hipLaunchKernelGGL((attention_wave_kernel<true>), dim3((unsigned)blocks), dim3(64), 0, s, c, a);
  else hipLaunchKernelGGL((attention_wave_kernel<false>), dim3((unsigned)blocks), dim3(64), 0, s, c, a);
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace vq
