// The choice of kernels of vq_attention_shared for a call of the largest sizes that its arguments allow, with what it launches in place of the kernels: prints which were launched.  Built with
// checks of signed arithmetic, which end the program.
#include <cstdio>
#include <cstdlib>

#include "vq_attention.hip"

namespace vq {
const char *launched = "nothing";
int cu_count() { return 256; }
const Switches &switches() {
  static Switches sw;
  sw.shared = '1';
  return sw;
}
int attention_decode_run(const KvParams &) { return DECODE_RUN; }
int attention_decode_waves(const KvParams &, int, int) { return DECODE_RUN; }
int attention_decode_rows(const KvParams &, const AttentionParams &, bool) { return 16; }
int attention_prompt_rows() { return ROWS; }
bool attention_prompt_takes(const KvParams &) { return true; }
bool attention_join_takes(const KvParams &, const AttentionParams &) { return true; }
int note(const char *what) {
  launched = what;
  return VQ_OK;
}
int launch_attention_decode(const KvParams &, const AttentionParams &, const Split &, hipStream_t) { return note("whole"); }
int launch_attention_prompt(const KvParams &, const AttentionParams &, const Split &, hipStream_t) { return note("whole"); }
int launch_attention_decode(const KvParams &, const AttentionParams &, const Split &, const Prefixes &, Half, hipStream_t) { return note("half"); }
int launch_attention_prompt(const KvParams &, const AttentionParams &, const Split &, const Prefixes &, Half, hipStream_t) { return note("half"); }
int launch_attention_join(const KvParams &, const AttentionParams &, const Split &, int, hipStream_t) { return VQ_OK; }
int launch_attention_join_halves(const KvParams &, const AttentionParams &, const Split &, int, const Split &, const Prefixes &, hipStream_t) { return VQ_OK; }
template <bool E4M3>
int launch_attention_halves(const KvParams &, const AttentionParams &, const Split &, const Split &, const Prefixes &, const HalvesGrid &g, bool, hipStream_t) {
  if (g.prefix_blocks < 1 || g.own_blocks < 1 || g.first < 1 || g.first > g.prefix_blocks) abort();
  return note("halves");
}
template int launch_attention_halves<true>(const KvParams &, const AttentionParams &, const Split &, const Split &, const Prefixes &, const HalvesGrid &, bool, hipStream_t);
template int launch_attention_halves<false>(const KvParams &, const AttentionParams &, const Split &, const Split &, const Prefixes &, const HalvesGrid &, bool, hipStream_t);
}  // namespace vq

// sequences, prefixes, key heads, new tokens of a sequence, tokens of a prefix and behind it
int main(int, char **argv) {
  vq::KvParams c{};
  c.e4m3 = 1;
  c.head_dim = 64;
  c.page_shift = 4;
  c.n_pages = 1;
  c.n_seqs = atoi(argv[1]);
  c.kv_heads = atoi(argv[3]);
  c.max_new = atoi(argv[4]);
  const long long tokens = (long long)c.n_seqs * c.max_new;
  c.n_tokens = (int)(tokens < 1 << 30 ? tokens : 1 << 30);
  c.max_length = 1 << 30;
  vq::Prefixes x{};
  x.n = atoi(argv[2]);
  x.most = x.n_seqs = c.n_seqs;
  x.max_length = atoi(argv[5]);
  x.max_own = atoi(argv[6]);
  x.rows_most = c.n_tokens;
  x.by_token = x.n > 1;
  x.partial_tokens = c.n_tokens;
  vq::AttentionParams a{};
  a.group = 1;
  a.q_heads = c.kv_heads;
  const size_t bytes = vq::attention_shared_workspace_bytes(c, x, a);
  const int rc = vq::launch_attention_shared(c, x, a, bytes ? malloc(256) : nullptr, bytes, nullptr);
  printf("%d %s\n", rc, vq::launched);
  return 0;
}
