// Both halves of attention behind shared prefixes in one launch: what the matrix cores bound (many rows over a prefix) and what memory bounds (few rows over each sequence's own keys) share
// the compute units.  Workgroups of four waves, two to a compute unit, as the prompt kernel's are.
// Measured (64 query and 8 key heads of 128 elements, 8 bits): 16 sequences behind 2048 tokens 10.6 us (with a launch for each half 18), 64 behind 8192 41.5 (56): one workgroup of the prefix on each
// compute unit, 16 chunks of 64 keys one behind the other at about 1.8 us by itself and 2.5 beside a workgroup of the own keys, so that a chunk's latency bounds it (matrix cores busy 17 % of the
// clocks); 128 behind 32768 168 (209): two workgroups of the prefix on each, a chunk of both in 2.5 us, as in long prompts.  (Internal; instantiated for each type of cache by a file of its own.)
#pragma once
#include "vq_attention.hpp"

namespace vq {

namespace {

// PRT: 0: the prefix by the prompt kernel, else by the decode kernel in tiles of 16 PRT rows.  Workgroups that begin together take different halves: `first` of the
// prefix's, which are the longer ones, then the sequences' own, then the rest.  Those of a key head go to one XCD where the heads are a multiple of eight.
// (The bodies find what they expect under its name: those of the prefix in scopes of their own.)
template <bool E4M3, int D, int PRT, int ORT, bool OWN_MANY>
__global__ __launch_bounds__(THREADS, 2) void attention_halves_kernel(const KvParams c, const AttentionParams a, const Split split, const Split prefix, const Prefixes x, const HalvesGrid g) {
  constexpr bool EXACT = true;
  constexpr int waves = HALVES_WAVES, tile0 = 0;
  const int own_block = (int)blockIdx.x - g.first;
  if (own_block >= 0 && own_block < g.own_blocks) {
    constexpr int RT = ORT;
    constexpr bool MANY = OWN_MANY;
    constexpr Half HALF = OWN;
    const int tiles = g.own_tiles, rest = own_block / c.kv_heads, block_seq = rest % c.n_seqs, block_head = own_block % c.kv_heads, block_rest = rest / c.n_seqs;
#include "vq_attention_decode.inc"
  } else {
    const KvParams of_prefix = as_sequences(c, x);
    const Split &of_prefix_split = prefix;
    const unsigned block = own_block < 0 ? blockIdx.x : blockIdx.x - (unsigned)g.own_blocks;
    const KvParams &c = of_prefix;
    const Split &split = of_prefix_split;
    constexpr Half HALF = PREFIX;
    const int tiles = g.prefix_tiles;
    if constexpr (PRT == 0) {
      const int zigzag = g.zigzag;
#include "vq_attention_prompt.inc"
    } else {
      constexpr int RT = PRT;
      constexpr bool MANY = false;
      const int rest = (int)block / c.kv_heads, block_seq = rest % c.n_seqs, block_head = (int)block % c.kv_heads, block_rest = rest / c.n_seqs;
#include "vq_attention_decode.inc"
    }
  }
}

template <bool E4M3, int D, int PRT, int RT, bool MANY>
int launch(const KvParams &c, const AttentionParams &a, const Split &own, const Split &prefix, const Prefixes &x, const HalvesGrid &g, hipStream_t stream) {
  const int by_own = decode_lds_bytes(E4M3, D, RT, MANY, HALVES_WAVES), by_prefix = PRT == 0 ? prompt_lds_bytes(E4M3, D) : decode_lds_bytes(E4M3, D, PRT, false, HALVES_WAVES);
  VQ_ALLOW_FULL_LDS((attention_halves_kernel<E4M3, D, PRT, RT, MANY>));
  hipLaunchKernelGGL((attention_halves_kernel<E4M3, D, PRT, RT, MANY>), dim3((unsigned)(g.prefix_blocks + g.own_blocks)), dim3(THREADS), by_own > by_prefix ? by_own : by_prefix, stream, c, a, own,
                     prefix, x, g);
  return hipGetLastError() == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}
template <bool E4M3, int D, int PRT>
int launch_own(const KvParams &c, const AttentionParams &a, const Split &own, const Split &prefix, const Prefixes &x, const HalvesGrid &g, hipStream_t stream) {
  const bool many = c.max_new > 1, two = attention_decode_rows(c, a, !many) == 32;
  if constexpr (D == 64) {
    if (many) return two ? launch<E4M3, D, PRT, 2, true>(c, a, own, prefix, x, g, stream) : launch<E4M3, D, PRT, 1, true>(c, a, own, prefix, x, g, stream);
  } else if (many) {
    return launch<E4M3, D, PRT, 1, true>(c, a, own, prefix, x, g, stream);
  }
  if constexpr (D == 64 || E4M3)
    if (two) return launch<E4M3, D, PRT, 2, false>(c, a, own, prefix, x, g, stream);
  return launch<E4M3, D, PRT, 1, false>(c, a, own, prefix, x, g, stream);
}
template <bool E4M3, int D>
int launch_prefix(const KvParams &c, const AttentionParams &a, const Split &own, const Split &prefix, const Prefixes &x, const HalvesGrid &g, bool prompt, hipStream_t stream) {
  if (prompt) return launch_own<E4M3, D, 0>(c, a, own, prefix, x, g, stream);
  if constexpr (D == 64 || E4M3)
    if (attention_decode_rows(as_sequences(c, x), a, true) == 32) return launch_own<E4M3, D, 2>(c, a, own, prefix, x, g, stream);
  return launch_own<E4M3, D, 1>(c, a, own, prefix, x, g, stream);
}

}  // namespace

template <bool E4M3>
int launch_attention_halves(const KvParams &c, const AttentionParams &a, const Split &own, const Split &prefix, const Prefixes &x, const HalvesGrid &g, bool prompt, hipStream_t stream) {
  return c.head_dim == 64 ? launch_prefix<E4M3, 64>(c, a, own, prefix, x, g, prompt, stream) : launch_prefix<E4M3, 128>(c, a, own, prefix, x, g, prompt, stream);
}

}  // namespace vq
