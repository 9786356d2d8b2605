"""vq_kv_append and vq_attention over layouts drawn at random: the cache bit for bit, attention within the bound of tests/test_gpu_attention_long.py."""
import numpy as np
import pytest

import kv_reference as ref
from test_gpu_attention import Device, _problem, _tables
from test_gpu_attention_long import _attention, _check

pytestmark = pytest.mark.gpu


def _layout(seed):
    rng = np.random.default_rng(1000 + seed)
    pick = lambda *a: a[rng.integers(len(a))]  # noqa: E731
    dim, bits, size = int(pick(64, 128, 128, 16 * int(rng.integers(1, 17)))), int(pick(8, 8, 16)), int(pick(16, 16, 32, 64, 128, 256))
    heads, group, seqs = int(rng.integers(1, 4)), int(pick(1, 1, 2, 3, 4, 7, 8, 16)), int(pick(1, 2, 3, 9))
    longest = int(pick(1, 17, 100, 700, 2200))
    most = int(pick(1, 1, 4, 30, 150))
    lengths = [int(n) for n in rng.integers(0, longest + 1, seqs)]
    lengths[int(rng.integers(seqs))] = longest
    uniform = rng.random() < 0.5
    news = [most] * seqs if uniform else [int(n) for n in rng.integers(0, most + 1, seqs)]
    if sum(news) == 0:
        news[0] = 1
    window, sinks = (0, 0) if rng.random() < 0.6 else (int(pick(1, 5, 64, 300, 2000)), int(pick(0, 1, 4, 70)))
    return dim, bits, size, heads, group, lengths, news, window, sinks


@pytest.mark.parametrize("switches", ["", "attention=d", "attention=p", "attention=d,parts=2", "attention=p,parts=3", "attention=d,parts=6"])
@pytest.mark.parametrize("seed", range(60))
def test_layouts_drawn_at_random(gpu_lib, monkeypatch, seed, switches):
    """The kernels that are chosen, and each of the two in one part and in several."""
    import torch
    monkeypatch.setenv("VQ_SWITCHES", switches)
    dim, bits, size, heads, group, lengths, news, window, sinks = _layout(seed)
    if max(lengths) * heads * dim * (1 + group * max(news)) > 3e8:
        news = [min(n, 8) for n in news]
    lost = [(b, i) for b, (n, m) in enumerate(zip(lengths, news)) for i in range(-(-n // size))
            if window and (i + 1) * size <= n - m - window + 1 and i * size >= sinks]
    rng, cache, table, k, v, q = _problem(2000 + seed, lengths, news, heads * group, heads, dim, size, bits, fill="nan" if seed % 3 else "stale", spare=seed % 2, lost=lost)
    pairs, interleaved = (int(rng.integers(1, dim // 2 + 1)), bool(seed & 1)) if seed % 4 else (dim // 2, False)
    cos, sin = _tables(rng, max(max(lengths), 1), pairs)
    dev = Device(cache, table, lengths, news, uniform=len(set(news)) == 1, pitch=16 * (seed % 3))
    up = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    # rows of q, k and v in one matrix, as a joint product leaves them
    wide = torch.cat([up(a).flatten(1) for a in (q, k, v)], 1)
    qd, kd, vd = (t.unflatten(1, (-1, dim)) for t in wide.split([q[0].size, k[0].size, v[0].size], 1))
    args = dict(starts=dev.starts, max_new=max(news), max_length=max(lengths))
    rotated = gpu_lib.kv_append(kd, vd, *dev.cache, q=qd, cos=up(cos), sin=up(sin), interleaved=interleaved, **args)
    out, lse = gpu_lib.attention(rotated, *dev.cache, window=window, sinks=sinks, return_lse=True, **args)
    torch.cuda.synchronize()
    cache.append(k, v, table, lengths, news, cos, sin, None, interleaved)
    dev.equals(cache)
    row = 0
    for length, new in zip(lengths, news):
        for t in range(new):
            at = min(max(length - new + t, 0), len(cos) - 1)
            q[row] = ref.rotate(q[row], cos[at], sin[at], interleaved).astype(np.float16)
            row += 1
    assert np.array_equal(rotated.cpu().numpy().view(np.uint16), q.view(np.uint16))
    _check(out.cpu().numpy(), lse.cpu().numpy(), *_attention(q, cache, table, lengths, news, dim ** -0.5, window, sinks), dim, max(lengths))
