#!/usr/bin/env python3
"""A stack of decoder layers over a paged cache: prompts of several sequences at once, then their next tokens one by one from a captured graph.

One layer is eight calls on one stream (prompts of more than sixteen tokens take a call for each product):

    x += h; z = norm(x)             residual_norm      (h: what the layer before left)
    q, k, v = products of z         gemv_multi / gemm
    rotate q and k, store k and v   kv_append
    a = attention(q, cache)         attention          (attention_shared where the sequences begin with the same tokens)
    h = product of a                gemv / gemm
    x += h; z = norm(x)             residual_norm
    g, u = products of z            gemv_multi / gemm
    h = product of silu(g) * u      gemv / gemm        (silu by torch)

    python examples/decoder_layer.py [--layers 2] [--seqs 16] [--prompt 512] [--steps 64] [--bits 8]

runs layers of the sizes 4096 / 11008 with 32 heads of 128 elements (seeded synthetic weights of 12-bit indices with residuals) and prints the times of
the prompts and of a step.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2409_17066_amd as vq  # noqa: E402
import vq_synth  # noqa: E402


class PagedCache:
    """Pages of one layer's keys and values (bits: 16, or 8 for e4m3 codes with a scale for every page and head)."""

    def __init__(self, pages, kv_heads, page_tokens, head_dim, bits):
        kind = torch.float8_e4m3fn if bits == 8 else torch.float16
        self.k = torch.empty((pages, kv_heads, page_tokens, head_dim), dtype=kind, device="cuda")
        self.v = torch.empty((pages, kv_heads, head_dim, page_tokens), dtype=kind, device="cuda")
        self.k_scales, self.v_scales = (torch.ones((pages, kv_heads), device="cuda") if bits == 8 else None for _ in "kv")


class Sequences:
    """Which pages each sequence has, how long it is, and which rows are its new tokens; shared by all layers.  shared: so many tokens, whole pages of them, that all sequences
    begin with, in pages that they have in common; first() is the sequence of these alone, whose tokens come first."""

    def __init__(self, n_seqs, page_tokens, longest, shared=0):
        assert shared % page_tokens == 0
        common, each = shared // page_tokens, -(-(longest - shared) // page_tokens)
        self.page_tokens, self.n_seqs, self.longest = page_tokens, n_seqs, longest
        # (a server hands pages out as sequences grow; here each gets its own beforehand, interleaved as they would come to lie)
        own = common + torch.arange(n_seqs * each, dtype=torch.int32, device="cuda").reshape(each, n_seqs).t()
        prefix = torch.arange(common, dtype=torch.int32, device="cuda").expand(n_seqs, -1)
        self.table = torch.cat((prefix, own), 1).contiguous()
        self.pages = common + n_seqs * each
        self.lengths = torch.full((n_seqs,), shared, dtype=torch.int32, device="cuda")
        self.starts, self.max_new, self.max_length = None, 1, longest
        self.prefix = None
        if shared:
            self.prefix = dict(prefix_table=prefix[:1].contiguous(), prefix_lengths=self.lengths[:1].clone(), max_prefix=shared, max_own=longest - shared)

    def first(self):
        """The tokens that all sequences begin with as a sequence of its own, without a length so far."""
        alone = Sequences(1, self.page_tokens, self.prefix["max_prefix"])
        alone.table = self.prefix["prefix_table"]
        return alone

    def begin(self, news):
        """news: how many new tokens each sequence brings."""
        self.starts = torch.cumsum(torch.tensor([0] + list(news)), 0).to(dtype=torch.int32, device="cuda")
        self.lengths += torch.tensor(list(news), dtype=torch.int32, device="cuda")
        self.max_new = max(news)

    def one_each(self):
        self.starts, self.max_new = None, 1

    def where(self, cache):
        return dict(k_pages=cache.k, v_pages=cache.v, k_scales=cache.k_scales, v_scales=cache.v_scales, page_table=self.table, lengths=self.lengths,
                    starts=self.starts, max_new=self.max_new, max_length=self.max_length)


def products(layers, z):
    """Each of the layers times z's rows."""
    return vq.gemv_multi(layers, z) if z.shape[0] <= 16 else [vq.gemm(layer, z) for layer in layers]


class DecoderLayer:
    def __init__(self, weights, norm1, norm2, heads, kv_heads, head_dim):
        """weights: the seven products by name, DeviceLayer each; norm1, norm2: fp16 weights of the norms before attention and before the rest."""
        self.w, self.norm1, self.norm2, self.heads, self.kv_heads, self.head_dim = weights, norm1, norm2, heads, kv_heads, head_dim

    def __call__(self, h, x, seqs, cache, cos, sin):
        """h: what the layer before leaves to be added (None: nothing), x: the residual stream, fp32 [tokens][width], updated in place -> h."""
        w, where = self.w, seqs.where(cache)
        _, z = vq.residual_norm(h, x, pre=self.norm1, y=x)
        q, k, v = products([w["q"], w["k"], w["v"]], z)
        q, k, v = (t.unflatten(1, (-1, self.head_dim)) for t in (q, k, v))
        vq.kv_append(k, v, q=q, q_out=q, cos=cos, sin=sin, **where)
        a = vq.attention(q, **where) if seqs.prefix is None else vq.attention_shared(q, **seqs.prefix, **where)
        h, = products([w["o"]], a.flatten(1))
        _, z = vq.residual_norm(h, x, pre=self.norm2, y=x)
        gate, up = products([w["gate"], w["up"]], z)
        h, = products([w["down"]], torch.nn.functional.silu(gate) * up)
        return h


class Decoder:
    """Layers, their caches and the last norm: new tokens' rows in, normalised rows out."""

    def __init__(self, layers, last_norm, cos, sin, seqs, bits):
        pages = seqs.pages
        self.layers, self.last_norm, self.cos, self.sin, self.seqs = layers, last_norm, cos, sin, seqs
        self.caches = [PagedCache(pages, l.kv_heads, seqs.page_tokens, l.head_dim, bits) for l in layers]

    def __call__(self, x, seqs=None):
        """seqs: the sequences that x's rows are of (None: the decoder's)."""
        x, h = x.float(), None
        for layer, cache in zip(self.layers, self.caches):
            h = layer(h, x, seqs or self.seqs, cache, self.cos, self.sin)
        return vq.residual_norm(h, x, pre=self.last_norm, y=x)[1]

    def capture(self, x):
        """A graph of one step of a token a sequence on x: [sequences][width], and its result; every replay first makes each sequence a token longer."""
        self.seqs.one_each()
        kept = self.seqs.lengths.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):                   # (a first run outside of the graph, with idle slots: they store nothing)
            self.seqs.lengths.zero_()
            self(x)
            self.seqs.lengths.copy_(kept)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.seqs.lengths += 1
            out = self(x)
        return graph, out


def rotations(positions, head_dim, base=10000.0):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, head_dim, 2, dtype=torch.float64) / head_dim)
    return angle.cos().float().cuda(), angle.sin().float().cuda()


def random_layers(n, width, inner, heads, kv_heads, head_dim, v=6, k=4096, k_res=4096, seed=2):
    """(synthetic layers by name, norm weights) of n decoder layers, on the host."""
    shapes = dict(q=(heads * head_dim, width), k=(kv_heads * head_dim, width), v=(kv_heads * head_dim, width), o=(width, heads * head_dim), gate=(inner, width),
                  up=(inner, width), down=(width, inner))
    made = []
    for i in range(n):
        weights = {name: vq_synth.make_layer(seed, name, *shape, v, k, k_res, layer_ordinal=7 * i + j) for j, (name, shape) in enumerate(shapes.items())}
        norms = [vq_synth.to_fp16(0.5 + vq_synth.uniform01(1000 * seed + 2 * i + j, width)) for j in range(2)]
        made.append((weights, norms))
    return made


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--seqs", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=512)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 16))
    a = ap.parse_args()
    width, inner, heads, head_dim = 4096, 11008, 32, 128
    made = random_layers(a.layers, width, inner, heads, heads, head_dim)
    layers = [DecoderLayer({name: vq.DeviceLayer(w) for name, w in weights.items()}, *(torch.from_numpy(n).cuda() for n in norms), heads, heads, head_dim)
              for weights, norms in made]
    seqs = Sequences(a.seqs, 16, a.prompt + a.steps + 1)
    decoder = Decoder(layers, torch.ones(width, dtype=torch.float16, device="cuda"), *rotations(seqs.longest, head_dim), seqs, a.bits)
    generator = torch.Generator(device="cuda").manual_seed(0)
    rows = torch.randn((a.seqs * a.prompt, width), device="cuda", generator=generator).half()

    def timed(work):
        before, after = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        before.record()
        work()
        after.record()
        torch.cuda.synchronize()
        return before.elapsed_time(after)
    seqs.begin([a.prompt] * a.seqs)
    decoder(rows)                                       # (first run: code objects and memory)
    prompt = timed(lambda: decoder(rows))               # the same tokens again, which changes nothing
    x = rows[: a.seqs].clone()
    graph, out = decoder.capture(x)
    graph.replay()
    step = timed(lambda: [graph.replay() for _ in range(a.steps - 1)]) / max(a.steps - 1, 1)
    assert torch.isfinite(out).all() and seqs.lengths.tolist() == [a.prompt + a.steps] * a.seqs
    print("%d layers, %d sequences, %d bits: prompts of %d tokens %.2f ms (%.0f tokens/s), step at %d tokens %.3f ms (%.0f tokens/s)"
          % (a.layers, a.seqs, a.bits, a.prompt, prompt, 1e3 * a.seqs * a.prompt / prompt, a.prompt + a.steps, step, 1e3 * a.seqs / step))


if __name__ == "__main__":
    main()
