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

// RT: tiles of sixteen rows; D: elements of a head, or (not EXACT) the next multiple of 64, zeros behind the head's own; MANY: rows may be of several new
// tokens, which see different keys.
template <bool E4M3, int D, int RT, bool MANY, bool EXACT, Half HALF>
__global__ __launch_bounds__(64 * waves_of(E4M3, D)) void attention_decode_kernel(const KvParams c, const AttentionParams a, const Split split, int tiles, int tile0, int waves, const PrefixesOf<HALF> x) {
  const int block_seq = (int)blockIdx.x, block_head = (int)blockIdx.y, block_rest = (int)blockIdx.z;
#include "vq_attention_decode.inc"
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

template <bool E4M3, int D, int RT, bool MANY, bool EXACT, Half HALF>
int launch(const KvParams &c, const AttentionParams &a, const Split &s, const Prefixes &x, hipStream_t stream) {
  const int waves = attention_decode_waves(c, s.parts, HALF == OWN ? x.max_own : c.max_length);
  const int tiles = (c.max_new * a.group + 16 * RT - 1) / (16 * RT), most = 65535 / s.parts;     // (more tiles than a grid has layers: several launches)
  if (c.n_seqs > 0x7fffffff / 512) return VQ_ERR_SHAPE;
  const int lds = decode_lds_bytes(E4M3, D, RT, MANY, waves);
  VQ_ALLOW_FULL_LDS((attention_decode_kernel<E4M3, D, RT, MANY, EXACT, HALF>));
  for (int tile0 = 0; tile0 < tiles; tile0 += most) {
    const int now = tiles - tile0 < most ? tiles - tile0 : most;
    hipLaunchKernelGGL((attention_decode_kernel<E4M3, D, RT, MANY, EXACT, HALF>), dim3(c.n_seqs, c.kv_heads, now * s.parts), dim3(64 * waves), lds, stream, c, a, s, now, tile0, waves,
                       prefixes_of<HALF>(x));
  }
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // namespace

// Two tiles share the conversions and loads of a chunk, where the registers are there: not beside 64 of a 16-bit chunk's keys and as many of its values, nor
// (heads of 128 elements) beside what rows of several tokens need.
int attention_decode_rows(const KvParams &c, const AttentionParams &a, bool alike) {
  return (long long)c.max_new * a.group > 16 && (c.head_dim == 64 || (c.head_dim == 128 && c.e4m3 && alike)) ? 32 : 16;
}
// Where no sequence has a chunk for every wave, no more waves than chunks: more workgroups share a compute unit (8 bits: 36 sequences of up to 13
// tokens, 32 heads of 64 elements, 10.9 us by eight waves and 7.0 by one; 64 of 250 tokens, 8 key heads of 128, 12.7 by eight and 9.4 by four).
int attention_decode_waves(const KvParams &c, int parts, int length) {
  int waves = waves_of(c.e4m3, c.head_dim);
  while (parts == 1 && waves > 1 && length <= 32 * waves) waves /= 2;
  return waves;
}
int attention_decode_run(const KvParams &c) { return waves_of(c.e4m3, c.head_dim); }

template <bool MANY, Half HALF>
static int launch_decode(const KvParams &c, const AttentionParams &a, const Split &s, const Prefixes &x, hipStream_t stream) {
  const bool two = attention_decode_rows(c, a, !MANY) == 32;
  if (c.head_dim == 64) return c.e4m3 ? (two ? launch<true, 64, 2, MANY, true, HALF>(c, a, s, x, stream) : launch<true, 64, 1, MANY, true, HALF>(c, a, s, x, stream))
                                      : (two ? launch<false, 64, 2, MANY, true, HALF>(c, a, s, x, stream) : launch<false, 64, 1, MANY, true, HALF>(c, a, s, x, stream));
  if constexpr (!MANY)
    if (two) return launch<true, 128, 2, MANY, true, HALF>(c, a, s, x, stream);
  return c.e4m3 ? launch<true, 128, 1, MANY, true, HALF>(c, a, s, x, stream) : launch<false, 128, 1, MANY, true, HALF>(c, a, s, x, stream);
}

// Heads of other sizes: rows of one token as well by what takes several.
template <int D, Half HALF>
static int launch_padded(const KvParams &c, const AttentionParams &a, const Split &s, const Prefixes &x, hipStream_t stream) {
  return c.e4m3 ? launch<true, D, 1, true, false, HALF>(c, a, s, x, stream) : launch<false, D, 1, true, false, HALF>(c, a, s, x, stream);
}

template <Half HALF>
static int launch_half(const KvParams &c, const AttentionParams &a, const Split &s, const Prefixes &x, hipStream_t stream) {
  if (c.head_dim != 64 && c.head_dim != 128)
    return c.head_dim < 64 ? launch_padded<64, HALF>(c, a, s, x, stream) : c.head_dim < 128 ? launch_padded<128, HALF>(c, a, s, x, stream) :
           c.head_dim <= 192 ? launch_padded<192, HALF>(c, a, s, x, stream) : launch_padded<256, HALF>(c, a, s, x, stream);
  if constexpr (HALF != PREFIX)
    if (c.max_new > 1) return launch_decode<true, HALF>(c, a, s, x, stream);
  return launch_decode<false, HALF>(c, a, s, x, stream);
}
int launch_attention_decode(const KvParams &c, const AttentionParams &a, const Split &s, hipStream_t stream) { return launch_half<WHOLE>(c, a, s, Prefixes{}, stream); }
int launch_attention_decode(const KvParams &c, const AttentionParams &a, const Split &s, const Prefixes &x, Half half, hipStream_t stream) {
  return half == PREFIX ? launch_half<PREFIX>(c, a, s, x, stream) : launch_half<OWN>(c, a, s, x, stream);
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
