// Attention behind shared prefixes, the launch behind its halves: partial results of a prefix and of a sequence's own keys become outputs.
//
// Latency bounds it: a launch, what a sequence has, the parts' maxima, the parts.  Measured: 4 us for 1024 rows of 128 elements, 6.2 for 4096 with ten parts each (20 MB), 8.6 for 8192; by a workgroup for each
// row, which looked everything up anew, 11 to 20.  A workgroup takes as many rows (of a token's heads) as it has lanes for at four elements each; what it has to know of its sequence it looks up once for all of them.  A lane takes a part's
// maximum and sum as well, and passes its factor on.
#include "vq_attention.hpp"

namespace vq {

namespace {

constexpr int JOIN_THREADS = 256;

template <int D>
__global__ __launch_bounds__(JOIN_THREADS) void attention_join_halves_kernel(const KvParams c, const AttentionParams a, const Split own, int own_tile_rows, const Split prefix, const Prefixes x) {
  constexpr int LANES = D / 4, ROWS_HERE = JOIN_THREADS / LANES, EACH = 2 * HALF_PARTS / LANES;     // (parts that a lane looks after)
  static_assert(EACH * LANES == 2 * HALF_PARTS, "");
  const int b = (int)blockIdx.y, dim = c.head_dim, lane = (int)threadIdx.x % LANES, d = lane * 4;
  const Sequence s = sequence(c, b);
  const Behind h = behind(c, x, s, b);
  const int row = (int)blockIdx.x * ROWS_HERE + (int)threadIdx.x / LANES;
  const bool there = row < s.rows * a.q_heads;
  if (!__ballot(there)) return;
  const int t = there ? row / a.q_heads : 0, head = there ? row - t * a.q_heads : 0, kv_head = token_of(a, head), of_head = t * a.group + head - kv_head * a.group;
  Sequence behind_prefix = s;
  behind_prefix.begin = h.length;
  const int before = h.prefix < 0 ? 0 : parts_of(prefix, (h.length + 63) >> 6);
  const int parts = there ? before + parts_of(own, span_of<OWN>(a, behind_prefix, of_head / own_tile_rows * own_tile_rows, own_tile_rows).chunks) : 0;
  const long long own_most = (long long)c.max_new * a.group, own_from = ((long long)b * c.kv_heads + kv_head) * own.parts * own_most + of_head;
  const long long prefix_most = x.partial_tokens * a.group, prefix_from = (long long)kv_head * prefix.parts * prefix_most + (prefix_partials(x, max(h.prefix, 0), s.row0 - h.row) + h.row) * a.group + of_head;
  auto from = [&](int w) { return w < before ? prefix_from + w * prefix_most : own_from + (long long)(w - before) * own_most; };
  float2v ml[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int w = i * LANES + lane;
    ml[i] = w < parts ? *reinterpret_cast<const float2v *>((w < before ? prefix.ml : own.ml) + from(w) * 2) : float2v{-__builtin_inff(), 0.f};
  }
  constexpr int AHEAD = 4;
  float4v y[AHEAD];
  auto load = [&](int w0) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      y[u] = w0 + u < parts && d < dim ? *reinterpret_cast<const float4v *>((w0 + u < before ? prefix.o : own.o) + from(w0 + u) * dim + d) : float4v{0.f, 0.f, 0.f, 0.f};
  };
  load(0);
  float top = ml[0].x;
#pragma unroll
  for (int i = 1; i < EACH; ++i) top = fmaxf(top, ml[i].x);
#pragma unroll
  for (int i = 1; i < LANES; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
  float f[EACH], total = 0.f;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    f[i] = __builtin_amdgcn_exp2f(ml[i].x - base_of(top));
    total = __fmaf_rn(ml[i].y, f[i], total);
  }
#pragma unroll
  for (int i = 1; i < LANES; i <<= 1) total += __shfl_xor(total, i);
  float4v o = {0.f, 0.f, 0.f, 0.f};
  for (int w0 = 0; __ballot(w0 < parts); w0 += AHEAD) {
    if (w0) load(w0);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int w = w0 + u;
      float fw = 0.f;
#pragma unroll
      for (int i = 0; i < EACH; ++i)
        if (w / LANES == i) fw = __shfl(f[i], w % LANES, LANES);
      // (nothing of parts that there are not: zero times zero)
      o.x = __fmaf_rn(y[u].x, fw, o.x); o.y = __fmaf_rn(y[u].y, fw, o.y); o.z = __fmaf_rn(y[u].z, fw, o.z); o.w = __fmaf_rn(y[u].w, fw, o.w);
    }
  }
  if (!there) return;
  if (d < dim) {
    o *= inverse_of(total);
    typedef _Float16 half4b __attribute__((ext_vector_type(4), aligned(2)));
    *reinterpret_cast<half4b *>(a.out + (s.row0 + t) * a.ldo + (long long)head * dim + d) = half4b{(_Float16)o.x, (_Float16)o.y, (_Float16)o.z, (_Float16)o.w};
  }
  if (a.lse && lane == 0) a.lse[(long long)(s.row0 + t) * a.q_heads + head] = lse_of(top, total);
}

template <int D>
int launch(const KvParams &c, const AttentionParams &a, const Split &own, int own_tile_rows, const Split &prefix, const Prefixes &x, hipStream_t stream) {
  const long long rows = (long long)c.max_new * a.q_heads;
  constexpr int HERE = JOIN_THREADS / (D / 4);
  hipLaunchKernelGGL(attention_join_halves_kernel<D>, dim3((unsigned)((rows + HERE - 1) / HERE), c.n_seqs), dim3(JOIN_THREADS), 0, stream, c, a, own, own_tile_rows, prefix, x);
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace

int launch_attention_join_halves(const KvParams &c, const AttentionParams &a, const Split &own, int own_tile_rows, const Split &prefix, const Prefixes &x, hipStream_t stream) {
  return c.head_dim <= 64 ? launch<64>(c, a, own, own_tile_rows, prefix, x, stream) : c.head_dim <= 128 ? launch<128>(c, a, own, own_tile_rows, prefix, x, stream)
                                                                                                        : launch<256>(c, a, own, own_tile_rows, prefix, x, stream);
}

}  // namespace vq
