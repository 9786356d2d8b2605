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
  float time, beside;            // estimated, us; the same to be held against attention behind shared prefixes
};

// Rows that a prefix is taken to have, of up to `rows`: an even share of the call's.  Where max_members bounds little (by default each prefix may have all of the call's sequences) most
// workgroups find no rows and end at once, of which a compute unit takes one in EMPTY us.  (Counted as work, ten prefixes of twelve sequences each without that bound were not computed once at all.
// Measured, 4096 tokens each, 64 query and 8 key heads of 128 elements, 8 bits: 46.6 us with the bound, 47.0 without, 93 by themselves.)
constexpr float EMPTY = 0.2f;
long long even_rows(const KvParams &c, const AttentionParams &a, long long prefixes, long long rows) {
  return std::min(rows, ((long long)c.n_tokens * a.group + prefixes - 1) / prefixes);
}

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
// A prefix is a sequence all of whose rows see all of it; of what lies behind there are `length` keys at most.  Both always leave parts for another launch, which is not counted here.
Plan plan_of(const KvParams &c, const AttentionParams &a, bool parts_allowed, Half half, long long length) {
  Plan best{};
  const long long rows = (long long)c.max_new * a.group, slots = cu_count(), even = half == PREFIX ? even_rows(c, a, c.n_seqs, rows) : rows;
  const long long all_rows = half == PREFIX ? std::min(c.n_seqs * rows, (long long)c.n_tokens * a.group) : c.n_seqs * rows;
  float least = 0.f;
  parts_allowed = parts_allowed && attention_join_takes(c, a);
  const int forced_parts = half == PREFIX && switches().prefix_parts >= 0 ? switches().prefix_parts : switches().parts;
  const char forced_kernel = half == PREFIX && switches().prefix ? switches().prefix : switches().attention;
  for (const bool prompt : {false, true}) {
    const char forced = attention_prompt_takes(c) ? forced_kernel : 'd';
    if (forced == 'd' || forced == 'p' ? prompt != (forced == 'p') : !prompt && rows > 512) continue;
    const int tile = prompt ? attention_prompt_rows() : attention_decode_rows(c, a, half == PREFIX || c.max_new == 1), run = prompt ? PROMPT_RUN : attention_decode_run(c);
    // tokens that a tile's rows look at: a window's and the first ones, or on the average all before half of the new ones
    const long long all = length - (rows > tile && half != PREFIX ? c.max_new / 2 : 0), reach = a.window > 0 ? (long long)a.window + a.sinks + tile / a.group + 64 : all;
    const long long chunks = (std::max(std::min(all, reach), 1LL) + 63) / 64;
    const long long heads = (long long)c.n_seqs * c.kv_heads, all_groups = heads * ((rows + tile - 1) / tile), groups = heads * ((even + tile - 1) / tile);
    const float quarters = (float)std::min((even + 31) / 32, 4LL), size = (float)((c.head_dim + 63) / 64) / 2.f;
    const long long most = parts_allowed ? std::min((chunks + run - 1) / run, half == WHOLE ? 64LL : (long long)HALF_PARTS) : 1;
    for (long long parts = 1;; parts *= 2) {
      if (forced_parts >= 0) parts = 1LL << forced_parts;
      parts = std::min(parts, most);
      const float alone = (float)slots * (prompt ? 1.f : (float)run / (float)std::min(attention_decode_waves(c, (int)parts, (int)length), run));   // workgroups side by side
      const float most_at_once = prompt ? 2.f * alone : alone, work = (float)(groups * parts), rounds = prompt ? std::max(work / most_at_once, 1.f) : std::ceil(work / most_at_once);
      const float turns = parts > 1 ? (float)(((chunks + run - 1) / run + parts - 1) / parts) : prompt ? (float)chunks / (float)run : (float)((chunks + run - 1) / run);
      const float one = 1.2f + 0.1f * quarters, two = 0.7f + 0.6f * quarters, shared = std::min(std::max(work / alone - 1.f, 0.f), 1.f);
      const float step = !prompt ? 3.2f * size * (c.e4m3 ? 1.f : 2.f) : run * size * (one + (two - one) * shared);
      const float join = parts > 1 ? (half == WHOLE ? 5.f : 0.f) + (float)(c.kv_heads * all_rows) * (0.3e-3f + (float)parts * size * 1024.f / 4.5e6f) : 0.f;
      const float empty = (float)((all_groups - groups) * parts) / (float)slots * EMPTY;
      const float time = (prompt ? 12.f + 5.f * size * (rounds - 1.f) : 9.f) + join + rounds * turns * step + empty;
      if (least == 0.f || time < least) {
        least = time;
        best.tile_rows = tile;
        best.parts = (int)parts;
        best.run = run;
        best.prompt = prompt;
        best.time = time;
        best.beside = prompt ? (half == WHOLE ? time : time - 5.f) : 1.2f + empty + join + rounds * (2.f + 3.1f * (float)std::max(c.head_dim, 64) / 128.f * (c.e4m3 ? 1.f : 2.f) * turns);
      }
      if (parts == most || forced_parts >= 0) break;
    }
  }
  if (best.parts > 1 || half != WHOLE) {
    best.o_bytes = (size_t)c.kv_heads * best.parts * all_rows * c.head_dim * 4;
    best.ml_bytes = (size_t)c.kv_heads * best.parts * all_rows * 8;
  }
  return best;
}

Plan plan_of(const KvParams &c, const AttentionParams &a, bool parts_allowed) { return plan_of(c, a, parts_allowed, WHOLE, c.max_length); }

// Attention behind shared prefixes: the prefixes and what lies behind, in one launch or one each, and one that joins them.
struct SharedPlan {
  KvParams prefixes;             // as sequences
  Plan prefix, own;
  bool shares, together;         // or every sequence by itself, where that is estimated to be faster; both halves in one launch
  HalvesGrid grid;
  static size_t bytes(const Plan &half) { return (half.o_bytes + half.ml_bytes + 255) / 256 * 256; }
  size_t bytes() const { return bytes(prefix) + bytes(own); }
};
// What a half moves to the launch that joins them.
void size_partials(Plan &half, int kv_heads, long long rows, int head_dim) {
  half.o_bytes = (size_t)kv_heads * half.parts * rows * head_dim * 4;
  half.ml_bytes = (size_t)kv_heads * half.parts * rows * 8;
}

// Both halves in one launch: the kernel of the prefixes and the parts of either half whose time is estimated the least, in us.  A workgroup of 256 threads takes runs of four chunks of 64 keys; two
// share a compute unit.  With `size` for the elements of a head (1: 128) and `element` for the bytes of one, and q for quarters of a prompt workgroup's 128 rows that are there:
//   a workgroup by itself      prefix, prompt kernel 1.75 + 4 size (1.19 + 0.16 q) a run     prefix, decode kernel 2 + 2.25 size element     own keys 3.2 + 0.73 size element
//   of a full compute unit     1.7 + 4 size (0.57 + 0.157 q)                                 0.8 + 2 size element                             0.73 of 1.3 + 2.7 size element
// (sequences are shorter than the longest), a prefix's once more on all compute units where some have one more; the halves overlap, but for 0.32 of the smaller one, behind 4 us; the launch that
// joins them takes 3.8 us and 0.34 for each MB of partial results.
// Fitted to 44 layouts by both kernels in 1 to 32 parts of the prefix and 1 to 4 of the rest.  Of the 60 in the first table of profiles/shared_plan.txt, these among them, what is chosen takes up to 5 % longer
// than the least in 49, up to 10 % in 55, up to 19 % in the others.
// Measured (64 query and 8 key heads of 128 elements, 8 bits): 64 sequences behind 8192 tokens with up to 1021 of their own 45 us by the prompt kernel in 8 parts, 51 by the decode kernel in 2,
// 119 by themselves; 16 behind 8192 with 300 26 (prompt, 32), 21.5 (decode, 8) and 38; 4 behind 4096 with 100 16, 15 and 13.
void plan_together(const KvParams &c, const Prefixes &x, const AttentionParams &a, SharedPlan &p) {
  const float size = (float)((c.head_dim + 63) / 64) / 2.f, moved = size * (c.e4m3 ? 1.f : 2.f), cus = (float)cu_count();
  const long long rows = (long long)x.rows_most * a.group, own_rows = (long long)c.max_new * a.group;
  const long long runs = std::max<long long>((x.max_length + 255) / 256, 1), own_runs = std::max<long long>((x.max_own + 255) / 256, 1);
  const long long even = even_rows(c, a, x.n, rows);
  const float quarters = (float)std::min((even + 31) / 32, 4LL);
  const int own_tile = attention_decode_rows(c, a, c.max_new == 1);
  const long long own_tiles = (own_rows + own_tile - 1) / own_tile;
  const char kernel = switches().prefix ? switches().prefix : switches().attention;
  const int prefix_parts = switches().prefix_parts >= 0 ? switches().prefix_parts : switches().parts;
  constexpr long long most = 0x7fffffff / THREADS;               // workgroups of a launch
  p.prefix.time = 0.f;
  for (const bool prompt : {false, true}) {
    if ((kernel == 'd' || kernel == 'p') && prompt != (kernel == 'p')) continue;
    const int tile = prompt ? attention_prompt_rows() : attention_decode_rows(p.prefixes, a, true);
    const long long tiles = (rows + tile - 1) / tile;
    for (int i = prefix_parts >= 0 ? prefix_parts : 0; i <= (prefix_parts >= 0 ? prefix_parts : 5); ++i) {
      const long long parts = std::min(std::min(1LL << i, runs), (long long)HALF_PARTS), blocks = (long long)x.n * c.kv_heads * tiles * parts;
      const long long with_rows = (long long)x.n * c.kv_heads * ((even + tile - 1) / tile) * parts;
      const float turns = (float)((runs + parts - 1) / parts);
      const float one = prompt ? 1.75f + turns * 4.f * size * (1.19f + 0.16f * quarters) : 2.f + turns * 2.25f * moved;
      const float each = (float)with_rows / cus, rounds = each > 1.f ? 0.93f * std::ceil(each) + 0.07f * each : each;
      const float all = rounds * (prompt ? 1.7f + turns * 4.f * size * (0.57f + 0.157f * quarters) : 0.8f + turns * 2.f * moved) + (float)(blocks - with_rows) / cus * EMPTY;
      for (int k = switches().parts >= 0 ? switches().parts : 0; k <= (switches().parts >= 0 ? switches().parts : 2); ++k) {
        const long long own_parts = std::min(std::min(1LL << k, own_runs), (long long)HALF_PARTS), own_blocks = (long long)c.n_seqs * c.kv_heads * own_tiles * own_parts;
        const float own_turns = (float)((own_runs + own_parts - 1) / own_parts), own_one = 3.2f + own_turns * 0.73f * moved, own_all = (float)own_blocks / cus * 0.73f * (1.3f + own_turns * 2.7f * moved);
        const float join = 3.8f + (float)((long long)c.n_seqs * own_rows * c.kv_heads) * (float)(parts + own_parts) * (float)c.head_dim * 4e-6f * 0.34f;
        const float time = 4.f + std::max(std::max(one, own_one), std::max(all, own_all) + 0.32f * std::min(all, own_all)) + join;
        if (blocks > most || own_blocks > most - blocks || (p.prefix.time != 0.f && time >= p.prefix.time)) continue;
        p.prefix.time = time;
        p.prefix.prompt = prompt;
        p.prefix.tile_rows = tile;
        p.prefix.parts = (int)parts;
        p.own.parts = (int)own_parts;
        p.grid = HalvesGrid{(int)blocks, (int)own_blocks, (int)std::min(blocks, (long long)cu_count()), (int)tiles, (int)own_tiles, blocks <= 2 * cu_count() || x.by_token};
      }
    }
  }
  p.together = p.prefix.time != 0.f;
  p.prefix.run = p.own.run = HALVES_WAVES;
  p.own.tile_rows = own_tile;
  size_partials(p.prefix, c.kv_heads, x.partial_tokens * a.group, c.head_dim);
  size_partials(p.own, c.kv_heads, c.n_seqs * own_rows, c.head_dim);
}

// (a call is launched whole or refused: a launch that a grid has no room for, and partial results whose bytes 64 bits do not count, are found before the first launch)
bool half_fits(const KvParams &c, const AttentionParams &a, const Plan &half) {
  const long long rows = (long long)c.max_new * a.group;
  return (!half.prompt || (long long)c.n_seqs * c.kv_heads * ((rows + half.tile_rows - 1) / half.tile_rows) * half.parts <= 0xffffffffll / THREADS) &&
         (double)c.n_seqs * c.kv_heads * half.parts * (double)rows * (c.head_dim * 4 + 8) < 4e18;
}

SharedPlan shared_plan_of(const KvParams &c, const Prefixes &x, const AttentionParams &a) {
  SharedPlan p{};
  p.prefixes = as_sequences(c, x);
  // (rows of a prefix: token_of()'s division and a grid's layers; rows of a sequence: threads of the launch that joins, up to 64 a row)
  if (!attention_join_takes(c, a) || x.max_length == 0 || (long long)x.rows_most * a.group * a.group >= 1ll << 30 || (long long)c.max_new * a.q_heads >= 1ll << 25) return p;
  const char forced = switches().shared;
  const Plan whole = plan_of(c, a, true);
  // A launch for each half, by either kernel.
  p.prefix = plan_of(p.prefixes, a, true, PREFIX, x.max_length);
  p.own = plan_of(c, a, true, OWN, std::min(x.max_own, c.max_length));
  const float apart = p.prefix.time + p.own.time + 5.f;
  // (what plan_of estimates is good for the choice among its own: held against others it is 6 us too much for one short round of the decode kernel, a quarter too little for many, and 5 us too much
  // for a half by the prompt kernel.  Of 44 layouts the slower one is chosen here in five, by 1 to 17 %.  Of 200 others of heads of 32 to 256 elements, drawn at random, which profiles/shared_plan.txt
  // lists, what is chosen takes up to 5 % longer than the least of all ways in 158, up to 20 % in 185, and up to 56 % in the others, of which ten are calls of 9 to 17 us.)
  const bool fit = half_fits(p.prefixes, a, p.prefix) && half_fits(c, a, p.own);
  p.shares = fit && (forced ? forced != '0' : p.prefix.beside + p.own.beside + 5.f < whole.beside);
  if ((c.head_dim == 64 || c.head_dim == 128) && forced != '2') {
    SharedPlan both = p;
    plan_together(c, x, a, both);
    if (both.together && both.prefix.time < apart) {
      p = both;
      p.shares = forced ? forced != '0' : p.prefix.time < whole.beside + 1.f;
    }
  }
  return p;
}

}  // namespace

size_t attention_shared_workspace_bytes(const KvParams &c, const Prefixes &x, const AttentionParams &a) {
  const SharedPlan p = shared_plan_of(c, x, a);
  return p.shares ? p.bytes() : attention_workspace_bytes(c, a);
}

int launch_attention_shared(const KvParams &c, const Prefixes &x, const AttentionParams &a, void *workspace, size_t workspace_bytes, hipStream_t s) {
  const SharedPlan p = shared_plan_of(c, x, a);
  if (!p.shares || workspace_bytes < p.bytes()) return launch_attention(c, a, workspace, workspace_bytes, s);
  float *at = static_cast<float *>(workspace);
  auto split_of = [&](const Plan &half) {
    const Split split{half.parts, half.run, at, at + half.o_bytes / 4};
    at += SharedPlan::bytes(half) / 4;
    return split;
  };
  const Split prefix = split_of(p.prefix), own = split_of(p.own);
  if (p.together) {
    const int rc = c.e4m3 ? launch_attention_halves<true>(c, a, own, prefix, x, p.grid, p.prefix.prompt, s) : launch_attention_halves<false>(c, a, own, prefix, x, p.grid, p.prefix.prompt, s);
    return rc != VQ_OK ? rc : launch_attention_join_halves(c, a, own, p.own.tile_rows, prefix, x, s);
  }
  int rc = p.prefix.prompt ? launch_attention_prompt(p.prefixes, a, prefix, x, PREFIX, s) : launch_attention_decode(p.prefixes, a, prefix, x, PREFIX, s);
  if (rc == VQ_OK) rc = p.own.prompt ? launch_attention_prompt(c, a, own, x, OWN, s) : launch_attention_decode(c, a, own, x, OWN, s);
  return rc != VQ_OK ? rc : launch_attention_join_halves(c, a, own, p.own.tile_rows, prefix, x, s);
}

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
