#!/usr/bin/env python3
"""From token numbers to token numbers: a decoder (decoder_layer.py) with an embedding table in front and a vector-quantized head behind, for sequences that begin with the same tokens.

The tokens that all sequences begin with pass through the decoder once; each sequence's own prompt follows behind them, and then its next tokens, one by one, from a captured graph whose
every replay is a whole step:

    x = scale * table[tokens]       embed
    z = decoder(x)                  decoder_layer.py: kv_append, attention_shared, residual_norm and the products
    logits = head * z               gemv
    tokens = draw(logits)           sample            (random numbers are written into `uniform` between the replays)

    python examples/generate.py [--layers 2] [--seqs 16] [--shared 2048] [--prompt 64] [--steps 64] [--bits 8] [--vocabulary 32000]

runs layers of the sizes 4096 / 11008 with 32 heads of 128 elements (seeded synthetic weights of 12-bit indices with residuals) and prints the times of the prompts and of a step.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import decoder_layer as dl  # noqa: E402
import paper_2409_17066_amd as vq  # noqa: E402
import vq_synth  # noqa: E402


class Generator:
    def __init__(self, decoder, table, head, scale=1.0, **how):
        """table: fp16 [vocabulary][width], head: DeviceLayer [vocabulary][width], how: sample()'s settings."""
        n = decoder.seqs.n_seqs
        self.decoder, self.table, self.head, self.scale, self.how = decoder, table, head, scale, how
        self.tokens = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.uniform = torch.zeros(n, device="cuda")
        self.logits = None

    def rows(self, tokens, seqs=None):
        """The decoder's last rows for new tokens (int32 [tokens])."""
        return self.decoder(vq.embed(tokens, self.table, scale=self.scale, dtype=torch.float32), seqs)

    def draw(self, z):
        """The next token of each row into self.tokens."""
        self.logits, = dl.products([self.head], z)
        return vq.sample(self.logits, self.uniform, out=self.tokens, **self.how)

    def prefix(self, tokens):
        """What all sequences begin with."""
        first = self.decoder.seqs.first()
        first.begin([len(tokens)])
        self.rows(tokens, first)

    def prompts(self, tokens, news):
        """Each sequence's own prompt, news[i] tokens of it -> the first tokens behind them."""
        self.decoder.seqs.begin(news)
        z = self.rows(tokens)
        last = torch.cumsum(torch.tensor(news), 0).cuda() - 1
        return self.draw(z[last])

    def capture(self):
        """A graph of one step: self.tokens, drawn before, join their sequences, and the next ones take their place."""
        seqs = self.decoder.seqs
        seqs.one_each()
        kept, tokens = seqs.lengths.clone(), self.tokens.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):                   # (a first run outside of the graph, with idle slots: they store nothing)
            seqs.lengths.zero_()
            self.draw(self.rows(self.tokens))
            seqs.lengths.copy_(kept)
            self.tokens.copy_(tokens)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            seqs.lengths += 1
            self.draw(self.rows(self.tokens))
        return graph


def random_head(vocabulary, width, v=6, k=4096, k_res=4096, seed=2):
    return vq_synth.make_layer(seed, "head", vocabulary, width, v, k, k_res, layer_ordinal=10 ** 4)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--seqs", type=int, default=16)
    ap.add_argument("--shared", type=int, default=2048)
    ap.add_argument("--prompt", type=int, default=64)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 16))
    ap.add_argument("--vocabulary", type=int, default=32000)
    a = ap.parse_args()
    width, inner, heads, head_dim = 4096, 11008, 32, 128
    made = dl.random_layers(a.layers, width, inner, heads, heads, head_dim)
    layers = [dl.DecoderLayer({name: vq.DeviceLayer(w) for name, w in weights.items()}, *(torch.from_numpy(n).cuda() for n in norms), heads, heads, head_dim)
              for weights, norms in made]
    seqs = dl.Sequences(a.seqs, 16, a.shared + a.prompt + a.steps + 1, a.shared)
    decoder = dl.Decoder(layers, torch.ones(width, dtype=torch.float16, device="cuda"), *dl.rotations(seqs.longest, head_dim), seqs, a.bits)
    g = torch.Generator(device="cuda").manual_seed(0)
    table = torch.randn((a.vocabulary, width), device="cuda", generator=g).half()
    model = Generator(decoder, table, vq.DeviceLayer(random_head(a.vocabulary, width)), temperature=0.8, top_k=50, top_p=0.9)

    def drawn(n):
        return torch.randint(a.vocabulary, (n,), device="cuda", generator=g, dtype=torch.int32)

    def timed(work):
        before, after = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        before.record()
        work()
        after.record()
        torch.cuda.synchronize()
        return before.elapsed_time(after)
    if a.shared:
        model.prefix(drawn(a.shared))
    tokens = drawn(a.seqs * a.prompt)
    model.prompts(tokens, [a.prompt] * a.seqs)          # (first run: code objects and memory)
    seqs.lengths -= a.prompt
    prompt = timed(lambda: model.prompts(tokens, [a.prompt] * a.seqs))
    graph = model.capture()
    numbers = torch.rand((a.steps, a.seqs), device="cuda", generator=g)

    def step(i):
        model.uniform.copy_(numbers[i])
        graph.replay()
    step(0)
    each = timed(lambda: [step(i) for i in range(1, a.steps)]) / max(a.steps - 1, 1)
    assert ((model.tokens >= 0) & (model.tokens < a.vocabulary)).all() and seqs.lengths.tolist() == [a.shared + a.prompt + a.steps] * a.seqs
    print("%d layers, %d sequences behind %d tokens, %d bits: prompts of %d tokens %.2f ms, step %.3f ms (%.0f tokens/s)"
          % (a.layers, a.seqs, a.shared, a.bits, a.prompt, prompt, each, 1e3 * a.seqs / each))


if __name__ == "__main__":
    main()
