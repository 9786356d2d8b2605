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

namespace vq {

namespace {

// D: elements of a head, or (not EXACT) more, zeros behind the head's own.
template <bool E4M3, int D, bool EXACT, Half HALF>
__global__ __launch_bounds__(THREADS, 2) void attention_prompt_kernel(const KvParams c, const AttentionParams a, const Split split, int tiles, int zigzag, const PrefixesOf<HALF> x) {
  const unsigned block = blockIdx.x;
#include "vq_attention_prompt.inc"
}

template <bool E4M3, int D, bool EXACT, Half HALF>
int launch(const KvParams &c, const AttentionParams &a, const Split &s, const Prefixes &x, hipStream_t stream) {
  const int tiles = (c.max_new * a.group + ROWS - 1) / ROWS;
  const long long blocks = (long long)c.n_seqs * c.kv_heads * tiles * s.parts;
  if (blocks > 0xffffffffll / THREADS) return VQ_ERR_SHAPE;        // (threads of a grid)
  const int lds = prompt_lds_bytes(E4M3, D), zigzag = blocks <= 2 * cu_count() || (HALF == PREFIX && x.by_token);
  VQ_ALLOW_FULL_LDS((attention_prompt_kernel<E4M3, D, EXACT, HALF>));
  hipLaunchKernelGGL((attention_prompt_kernel<E4M3, D, EXACT, HALF>), dim3((unsigned)blocks), dim3(THREADS), lds, stream, c, a, s, tiles, zigzag, prefixes_of<HALF>(x));
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

template <Half HALF>
int launch_half(const KvParams &c, const AttentionParams &a, const Split &s, const Prefixes &x, hipStream_t stream) {
  if (c.head_dim < 64) return c.e4m3 ? launch<true, 64, false, HALF>(c, a, s, x, stream) : launch<false, 64, false, HALF>(c, a, s, x, stream);
  if (c.head_dim > 64 && c.head_dim < 128) return c.e4m3 ? launch<true, 128, false, HALF>(c, a, s, x, stream) : launch<false, 128, false, HALF>(c, a, s, x, stream);
  if (c.head_dim == 64) return c.e4m3 ? launch<true, 64, true, HALF>(c, a, s, x, stream) : launch<false, 64, true, HALF>(c, a, s, x, stream);
  return c.e4m3 ? launch<true, 128, true, HALF>(c, a, s, x, stream) : launch<false, 128, true, HALF>(c, a, s, x, stream);
}

}  // namespace

int attention_prompt_rows() { return ROWS; }
bool attention_prompt_takes(const KvParams &c) { return c.head_dim <= 128; }

int launch_attention_prompt(const KvParams &c, const AttentionParams &a, const Split &s, hipStream_t stream) { return launch_half<WHOLE>(c, a, s, Prefixes{}, stream); }
int launch_attention_prompt(const KvParams &c, const AttentionParams &a, const Split &s, const Prefixes &x, Half half, hipStream_t stream) {
  return half == PREFIX ? launch_half<PREFIX>(c, a, s, x, stream) : launch_half<OWN>(c, a, s, x, stream);
}

}  // namespace vq
