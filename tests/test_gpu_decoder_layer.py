"""examples/decoder_layer.py, the products and the operators between them as one program, against 64 bits.

The reference rounds where the program does (norms' results, products, rotated queries, attention, gate and up to binary16, the cache's codes), so that
the two differ where a rounding falls on the other side: each of the eleven roundings of a layer moves its value by up to 2^-10 (one unit) in relative terms, two
layers' and the last one's add up in the norm's result to at most 23 * 2^-10 of its rows' largest elements if every one were off in the same direction; a code of the cache
that falls on the other side moves one element of one token by 2^-3.  Weights that vq_gemm rounds to binary16 are 2^-11 off each, in sums of hundreds."""
import os
import sys

import numpy as np
import pytest

import kv_reference as ref

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu

WIDTH, INNER, HEADS, KV_HEADS, DIM = 256, 384, 4, 2, 64


def _half(x):
    return np.asarray(x, np.float64).astype(np.float16)


def _norm(x, w):
    return _half(x / np.sqrt((x ** 2).mean(1, keepdims=True) + 1e-5) * w.astype(np.float64))


class Reference:
    def __init__(self, made, cos, sin, table, bits):
        rng = np.random.default_rng(31)
        self.made, self.cos, self.sin, self.table = made, cos, sin, table
        self.caches = [ref.Cache(rng, table.size, KV_HEADS, 16, DIM, bits) for _ in made]

    def __call__(self, x, lengths, news):
        import oracle
        x, h = x.astype(np.float64), None
        for (w, (n1, n2)), cache in zip(self.made, self.caches):
            x = x if h is None else x + h.astype(np.float64)
            z = _norm(x, n1)
            q, k, v = (_half(oracle.matmul(w[n], z)).reshape(len(z), -1, DIM) for n in "qkv")
            cache.append(k, v, self.table, lengths, news, self.cos, self.sin)
            row = 0
            for length, new in zip(lengths, news):
                for t in range(new):
                    q[row] = ref.rotate(q[row], self.cos[length - new + t], self.sin[length - new + t], False).astype(np.float16)
                    row += 1
            a = _half(ref.attention(q, cache, self.table, lengths, news, DIM ** -0.5)[0])
            x = x + _half(oracle.matmul(w["o"], a.reshape(len(z), -1))).astype(np.float64)
            z = _norm(x, n2)
            gate, up = (_half(oracle.matmul(w[n], z)).astype(np.float64) for n in ("gate", "up"))
            h = _half(oracle.matmul(w["down"], _half(_half(gate / (1 + np.exp(-gate))).astype(np.float64) * up)))
        return _norm(x + h.astype(np.float64), np.ones(WIDTH))


@pytest.mark.parametrize("bits", [16, 8])
def test_prompts_and_steps_of_a_graph(gpu_lib, bits):
    import torch
    import decoder_layer as example
    made = example.random_layers(2, WIDTH, INNER, HEADS, KV_HEADS, DIM, k=256, k_res=256, seed=30)
    up = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    layers = [example.DecoderLayer({n: gpu_lib.DeviceLayer(w) for n, w in weights.items()}, *map(up, norms), HEADS, KV_HEADS, DIM) for weights, norms in made]
    seqs = example.Sequences(3, 16, 64)
    cos, sin = example.rotations(64, DIM)
    decoder = example.Decoder(layers, torch.ones(WIDTH, dtype=torch.float16, device="cuda"), cos, sin, seqs, bits)
    reference = Reference(made, cos.cpu().numpy(), sin.cpu().numpy(), seqs.table.cpu().numpy(), bits)
    rng = np.random.default_rng(32)
    bound = 23 * 2.0 ** -10

    def check(got, want):
        got, want = got.float().cpu().numpy(), want.astype(np.float64)
        most = np.abs(want).max(1, keepdims=True)
        assert (np.abs(got - want) <= bound * most).all(), (np.abs(got - want) / most).max()
    lengths = [0, 0, 0]
    for news in ([21, 1, 16], [4, 4, 4], [0, 17, 3]):
        lengths = [n + m for n, m in zip(lengths, news)]
        seqs.begin(news)
        x = rng.standard_normal((sum(news), WIDTH)).astype(np.float16)
        check(decoder(up(x)), reference(x, lengths, news))
    x = torch.zeros((3, WIDTH), dtype=torch.float16, device="cuda")
    graph, out = decoder.capture(x)
    for _ in range(4):
        lengths = [n + 1 for n in lengths]
        rows = rng.standard_normal((3, WIDTH)).astype(np.float16)
        x.copy_(up(rows))
        graph.replay()
        torch.cuda.synchronize()
        check(out, reference(rows, lengths, [1, 1, 1]))
    assert seqs.lengths.tolist() == lengths
