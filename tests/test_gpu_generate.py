"""examples/generate.py: embedding, decoder behind a shared prefix, head and drawing as one program of captured steps, against 64 bits.

Decoder rows are held to test_gpu_decoder_layer.py's bound, from the program's own tokens on.  Logits are sums of a row's elements times the head's weights (restored exactly, rounded
once to binary16): a row that is off by up to `bound` of its largest element moves a logit by up to that times the sum of its weights' sizes.  Which token is drawn is
decided by the logits of the program exactly."""
import os
import sys

import numpy as np
import pytest

from test_gpu_decoder_layer import DIM, HEADS, INNER, KV_HEADS, WIDTH, Reference
from test_gpu_sample import _one

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu

VOCABULARY, SHARED = 1003, 48


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("switches", ["", "shared=1"])
def test_a_shared_prefix_prompts_and_steps_of_a_graph(gpu_lib, monkeypatch, bits, switches):
    import oracle
    import torch
    import decoder_layer as dl
    import generate
    monkeypatch.setenv("VQ_SWITCHES", switches)
    made = dl.random_layers(2, WIDTH, INNER, HEADS, KV_HEADS, DIM, k=256, k_res=256, seed=40)
    up = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    layers = [dl.DecoderLayer({n: gpu_lib.DeviceLayer(w) for n, w in weights.items()}, *map(up, norms), HEADS, KV_HEADS, DIM) for weights, norms in made]
    seqs = dl.Sequences(3, 16, 128, SHARED)
    cos, sin = dl.rotations(128, DIM)
    decoder = dl.Decoder(layers, torch.ones(WIDTH, dtype=torch.float16, device="cuda"), cos, sin, seqs, bits)
    rng = np.random.default_rng(41)
    table = rng.standard_normal((VOCABULARY, WIDTH)).astype(np.float16)
    head = generate.random_head(VOCABULARY, WIDTH, k=256, k_res=0, seed=42)
    sizes = np.abs(oracle.dequant(head).astype(np.float64)).sum(1)
    how = dict(temperature=0.7, top_k=200, top_p=0.9, min_p=0.001)
    model = generate.Generator(decoder, up(table), gpu_lib.DeviceLayer(head), scale=2.0, **how)
    whole = seqs.table.cpu().numpy()
    reference = Reference(made, cos.cpu().numpy(), sin.cpu().numpy(), whole, bits)
    bound = 23 * 2.0 ** -10

    def embedded(tokens):
        return (table[tokens].astype(np.float64) * 2.0).astype(np.float32)

    def check(z, uniform):
        """The logits against the reference's rows, the tokens against the logits."""
        want, logits = oracle.matmul(head, z), model.logits.cpu().numpy()
        off = bound * np.abs(z.astype(np.float64)).max(1, keepdims=True) * sizes + 2.0 ** -10 * np.abs(want) + 2.0 ** -24
        assert (np.abs(logits.astype(np.float64) - want) <= off).all()
        drawn = [_one(x, u, np.float32(how["temperature"]), how["top_k"], np.float32(how["top_p"]), np.float32(how["min_p"]))[0] for x, u in zip(logits, uniform)]
        assert model.tokens.tolist() == drawn
    tokens = rng.integers(0, VOCABULARY, SHARED).astype(np.int32)
    model.prefix(up(tokens))
    reference.table = whole[:1, : SHARED // 16]
    reference(embedded(tokens), [SHARED], [SHARED])
    reference.table = whole
    news, lengths = [5, 20, 1], [SHARED + 5, SHARED + 20, SHARED + 1]
    tokens, uniform = rng.integers(0, VOCABULARY, sum(news)).astype(np.int32), rng.random(3, dtype=np.float32)
    model.uniform.copy_(up(uniform))
    model.prompts(up(tokens), news)
    torch.cuda.synchronize()
    check(reference(embedded(tokens), lengths, news)[np.cumsum(news) - 1], uniform)
    before = model.tokens.tolist()
    graph = model.capture()
    assert model.tokens.tolist() == before and seqs.lengths.tolist() == lengths
    for _ in range(5):
        tokens, uniform = np.array(model.tokens.tolist()), rng.random(3, dtype=np.float32)
        model.uniform.copy_(up(uniform))
        graph.replay()
        torch.cuda.synchronize()
        lengths = [n + 1 for n in lengths]
        check(reference(embedded(tokens), lengths, [1, 1, 1]), uniform)
    assert seqs.lengths.tolist() == lengths
