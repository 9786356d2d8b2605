// The paged cache of keys and values as kernels take it (internal; include/vq.h describes the layout).
#pragma once
#include "vq_common.hpp"

namespace vq {

struct KvParams {
  int e4m3, kv_heads, head_dim, page_shift, n_pages, n_seqs, n_tokens, max_new, max_length, table_pages;
  int each;                      // new tokens of every sequence where `starts` is not given
  unsigned char *k_pages, *v_pages;
  long long k_page_bytes, v_page_bytes, table_stride;
  float *k_scales, *v_scales;
  const int *page_table, *lengths, *starts;
};

struct Rotary {
  const float *cos, *sin;
  long long ld;
  int positions, dim, interleaved;
  const int *position;
};

// Host-side validation shared by the entry points; fills `p` on success.
int make_kv_params(const vq_kv_desc *d, KvParams *p);

int launch_kv_append(const KvParams &c, const __half *k, long long ldk, const __half *v, long long ldv, const __half *q, long long ldq, int q_heads,
                     __half *q_out, long long ldq_out, const Rotary &r, hipStream_t s);

struct AttentionParams {
  const __half *q;
  long long ldq;
  __half *out;
  long long ldo;
  float *lse;
  float scale;                   // of the scores, times log2(e)
  int q_heads, group, window, sinks;
  unsigned by_group;             // 2^32 / group, rounded up: r / group is the upper half of r * by_group for all rows r (group > 1)
};
size_t attention_workspace_bytes(const KvParams &c, const AttentionParams &a);
int launch_attention(const KvParams &c, const AttentionParams &a, void *workspace, size_t workspace_bytes, hipStream_t s);

// Prefixes that sequences have in common.
struct Prefixes {
  int n, most, max_length, max_own;  // prefixes; sequences of one, tokens of one and of what a sequence holds behind its own, at most
  int n_seqs, table_pages;           // sequences of the call; entries of a row of page_table
  int rows_most;                     // new tokens of one prefix's sequences, at most
  int by_token;                      // partial results lie where the call's new tokens do, or each prefix's behind the other's: what needs less
  long long partial_tokens;          // new tokens that these have room for, n_tokens or n * rows_most
  const int *page_table, *lengths, *members;
  long long table_stride;
};
size_t attention_shared_workspace_bytes(const KvParams &c, const Prefixes &x, const AttentionParams &a);
int launch_attention_shared(const KvParams &c, const Prefixes &x, const AttentionParams &a, void *workspace, size_t workspace_bytes, hipStream_t s);

int launch_residual_norm(const __half *h, long long ldh, const void *x, long long ldx, const __half *w_post, const __half *gate, long long ldgate,
                         float scale, const __half *w_pre, float eps, bool stream32, int rows, int width, void *y, long long ldy, __half *z,
                         long long ldz, hipStream_t s);

int launch_embed(const int *ids, int rows, const __half *table, long long ld, int vocabulary, int width, float scale, bool stream32, void *y, long long ldy, hipStream_t s);

// Settings of a row: an array's entry, or the number where there is none.
struct SampleParams {
  const __half *logits;
  long long ld;
  int vocabulary, top_k;
  float temperature, top_p, min_p;
  const float *uniform, *temperatures, *top_ps, *min_ps;
  const int *top_ks;
  int *tokens;
  float *probabilities;
};
int launch_sample(const SampleParams &p, int rows, hipStream_t s);

#ifdef __HIPCC__
typedef unsigned uint4v __attribute__((ext_vector_type(4)));
typedef unsigned uint2v __attribute__((ext_vector_type(2)));
typedef unsigned uint4b __attribute__((ext_vector_type(4), aligned(2)));      // 16 bytes that begin at any half
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));

// A sequence of the call: its new tokens are rows row0 ... row0 + rows - 1, token t stands at place first + t, and places
// below `end` exist, of which those from `begin` on are looked at.
struct Sequence {
  int row0, rows, first, end, begin;
};
__device__ __forceinline__ Sequence sequence(const KvParams &c, int b) {
  Sequence s;
  int brings;
  if (c.starts) {
    s.row0 = min(max(c.starts[b], 0), c.n_tokens);
    brings = min(max(c.starts[b + 1], s.row0), c.n_tokens) - s.row0;
  } else {
    brings = c.each;
    s.row0 = b * brings;
  }
  const int length = max(c.lengths[b], 0);
  s.rows = min(brings, c.max_new);
  s.first = length - brings;
  s.end = min(length, c.max_length);
  s.begin = 0;
  return s;
}

// First row of sequence i's new tokens (i may be n_seqs: the row behind the last).
__device__ __forceinline__ int row_of(const KvParams &c, int i) { return c.starts ? min(max(c.starts[i], 0), c.n_tokens) : i * c.each; }

// The rows of a prefix: new tokens of its sequences, [row0, row0 + rows); what stands behind rows_most is left out.
struct PrefixRows {
  int first, last, row0, rows;       // sequences [first, last)
};
__device__ __forceinline__ PrefixRows prefix_rows(const KvParams &c, const Prefixes &x, int g) {
  PrefixRows r;
  r.first = x.members ? min(max(x.members[g], 0), x.n_seqs) : 0;
  r.last = min(x.members ? min(max(x.members[g + 1], r.first), x.n_seqs) : x.n_seqs, r.first + x.most);
  r.row0 = row_of(c, r.first);
  r.rows = min(max(row_of(c, r.last) - r.row0, 0), x.rows_most);
  return r;
}

// Page of block `block` (< table_pages) of sequence b, -1 where there is none.
__device__ __forceinline__ int page_of(const KvParams &c, int b, int block) {
  const int page = c.page_table[b * c.table_stride + block];
  return (unsigned)page < (unsigned)c.n_pages ? page : -1;
}

__device__ __forceinline__ half2v half2_of(unsigned u) { return __builtin_bit_cast(half2v, u); }

// Two e4m3 codes of a word (its lower or upper half) as binary16 numbers, times the power of two `scale`.
template <bool UPPER>
__device__ __forceinline__ half2v halves_of_e4m3(unsigned word, float scale) {
  return __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, scale, UPPER));
}
#endif

}  // namespace vq
