// Attention of new tokens over a paged cache: which kernel takes a call, and in how many parts.
#include "vq_attention.hpp"
#include <algorithm>
#include <cmath>

namespace vq {

namespace {

// How a call is taken: `tile_rows` rows of a key head to a workgroup, by the prompt or the decode kernel, the keys in up to `parts` parts of runs of `run` chunks.
struct Plan {
  int tile_rows, parts, run;
  bool prompt;
  size_t o_bytes, ml_bytes;
};

// The kernel and number of parts whose time is estimated the least, in us, from measurements on heads of 64 and 128 elements, 8 and 16 bits, 8 and 32 key heads,
// 1 to 200 sequences of 15 to 32768 tokens with 1 to 4144 rows a key head (heads of other sizes count as the next multiple of 64, as the kernels take them; every sequence as the longest):
//   decode: a workgroup of eight waves to a compute unit (more of smaller ones), rounds of 3.2 us for eight chunks of 16 KB behind 9 us;
//   prompt: one workgroup to a compute unit takes 1.3 us a chunk for up to 32 rows and 0.1 more for each further 32 of 128, two 1.3 and 0.6, behind 12 us and 5
//   for every further round of workgroups;
// and for parts the second launch that joins them, 5 us, 0.3 ns a row and what it moves.  Measured (64 query and 8 key heads of 128 elements, 8 bits, us by the
// decode and by the prompt kernel): 16 sequences of 4096 tokens 32 and 39 for 32 rows a key head, 59 and 50 for 64, 217 and 102 for 256; one of 1024 tokens 11 and
// 13 for 32 rows, 12 and 19 for 256; 64 of 100 tokens, 32 key heads, one row 15 and 39.  Parts (16 rows): 4 sequences of 2048 tokens 18 in one and 12 in four, one of 1024 11
// in one and in two; heads of 64 elements, 518 tokens behind 1909 (prompt kernel) 58 in one and 95 in two.  Of 115 layouts by both kernels in 1 to 32 parts (profiles/attention_plan.txt) what is
// chosen takes up to 10 % longer than the least in 100, and up to 29 % in the others.
Plan plan_of(const KvParams &c, const AttentionParams &a, bool parts_allowed) {
  Plan best{};
  const long long rows = (long long)c.max_new * a.group, slots = cu_count();
  float least = 0.f;
  parts_allowed = parts_allowed && attention_join_takes(c, a);
  for (const bool prompt : {false, true}) {
    const char forced = attention_prompt_takes(c) ? switches().attention : 'd';
    if (forced == 'd' || forced == 'p' ? prompt != (forced == 'p') : !prompt && rows > 512) continue;
    const int tile = prompt ? attention_prompt_rows() : attention_decode_rows(c, a), run = prompt ? PROMPT_RUN : attention_decode_run(c);
    // tokens that a tile's rows look at: a window's and the first ones, or on the average all before half of the new ones
    const long long all = c.max_length - (rows > tile ? c.max_new / 2 : 0), reach = a.window > 0 ? (long long)a.window + a.sinks + tile / a.group + 64 : all;
    const long long chunks = (std::max(std::min(all, reach), 1LL) + 63) / 64, groups = (long long)c.n_seqs * c.kv_heads * ((rows + tile - 1) / tile);
    const float quarters = (float)std::min((rows + 31) / 32, 4LL), size = (float)((c.head_dim + 63) / 64) / 2.f;
    const long long most = parts_allowed ? std::min((chunks + run - 1) / run, 64LL) : 1;
    for (long long parts = 1;; parts *= 2) {
      if (switches().parts >= 0) parts = 1LL << switches().parts;
      parts = std::min(parts, most);
      const float alone = (float)slots * (prompt ? 1.f : (float)run / (float)std::min(attention_decode_waves(c, (int)parts), run));   // workgroups side by side
      const float most_at_once = prompt ? 2.f * alone : alone, work = (float)(groups * parts), rounds = prompt ? std::max(work / most_at_once, 1.f) : std::ceil(work / most_at_once);
      const float turns = parts > 1 ? (float)(((chunks + run - 1) / run + parts - 1) / parts) : prompt ? (float)chunks / (float)run : (float)((chunks + run - 1) / run);
      const float one = 1.2f + 0.1f * quarters, two = 0.7f + 0.6f * quarters, shared = std::min(std::max(work / alone - 1.f, 0.f), 1.f);
      const float step = !prompt ? 3.2f * size * (c.e4m3 ? 1.f : 2.f) : run * size * (one + (two - one) * shared);
      const float join = parts > 1 ? 5.f + (float)((long long)c.n_seqs * c.kv_heads * rows) * (0.3e-3f + (float)parts * size * 1024.f / 4.5e6f) : 0.f;
      const float time = (prompt ? 12.f + 5.f * size * (rounds - 1.f) : 9.f) + join + rounds * turns * step;
      if (least == 0.f || time < least) {
        least = time;
        best.tile_rows = tile;
        best.parts = (int)parts;
        best.run = run;
        best.prompt = prompt;
      }
      if (parts == most || switches().parts >= 0) break;
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
  float *o = static_cast<float *>(workspace);
  const Split split{p.parts, p.run, o, p.parts > 1 ? o + p.o_bytes / 4 : nullptr};
  const int rc = p.prompt ? launch_attention_prompt(c, a, split, s) : launch_attention_decode(c, a, split, s);
  return rc != VQ_OK || p.parts == 1 ? rc : launch_attention_join(c, a, split, p.tile_rows, s);
}

}  // namespace vq
