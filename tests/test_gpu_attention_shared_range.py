"""vq_attention_shared at the ends of its numbers' ranges, with what is not finite, in pools past 32 bits and in graphs that share a workspace: against 64 bits or against vq_attention's
own results."""
import numpy as np
import pytest

from test_gpu_attention import Device
from test_gpu_attention_long import _attention
from test_gpu_attention_range import _margin
from test_gpu_attention_shared import Problem

pytestmark = pytest.mark.gpu

ROUTES = ["shared=1,prefix=d,attention=d", "shared=1,prefix=p,attention=d", "shared=2,prefix=d,attention=d", "shared=2,prefix=p,attention=p"]
LAYOUTS = [
    # prefixes, alone, q heads, heads, dim, page, bits
    ([(256, 256, [(70, 1), (9, 1), (1, 1)]), (128, 120, [(40, 1), (200, 1)])], [(90, 1)], 8, 2, 128, 16, 8),
    ([(512, 490, [(70, 5), (9, 5), (100, 9)])], [], 4, 2, 64, 32, 16),
    ([(192, 192, [(70, 7), (33, 2)])], [(20, 3)], 2, 1, 80, 16, 8),
    ([(256, 256, [(150, 140), (90, 33)])], [], 4, 2, 128, 64, 16),
]


def _call(gpu_lib, p, q, cache=None, **kw):
    import torch
    dev, prefix = p.up()
    if cache is not None:
        dev = Device(cache, p.table, p.lengths, p.news)
    return gpu_lib.attention_shared(torch.from_numpy(q).cuda(), dev.k, dev.v, dev.table, dev.lengths, k_scales=dev.k_scales, v_scales=dev.v_scales,
                                    starts=torch.tensor(np.concatenate([[0], np.cumsum(p.news)]), dtype=torch.int32, device="cuda"), return_lse=True, max_new=max(p.news), **prefix, **kw)


def _plain(gpu_lib, p, q, cache):
    import torch
    dev = Device(cache, p.table, p.lengths, p.news)
    return gpu_lib.attention(torch.from_numpy(q).cuda(), *dev.cache, starts=dev.starts, max_new=max(p.news), return_lse=True)


@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda c: "%d of %d bits" % c[-3::2])
@pytest.mark.parametrize("switches", ROUTES)
@pytest.mark.parametrize("size", [2.0 ** 5, 2.0 ** 8, 2.0 ** 14])
def test_scores_of_every_size(gpu_lib, monkeypatch, layout, switches, size):
    """As the test of this name for vq_attention, with queries and keys of up to 50000: scores of up to 10^10 in either half; rows of one key get that key's value."""
    import torch
    monkeypatch.setenv("VQ_SWITCHES", switches)
    p = Problem(41, *layout, spread=size)
    rng = np.random.default_rng(42)
    q = (rng.standard_normal(p.q.shape) * size).clip(-50000, 50000).astype(np.float16)
    out, lse = _call(gpu_lib, p, q)
    torch.cuda.synchronize()
    out, lse = out.cpu().numpy(), lse.cpu().numpy()
    want, want_lse, _, _, terms = _attention(q, p.cache, p.table, p.lengths, p.news, p.dim ** -0.5, 0, 0)
    error = (p.dim + 2) * 2.0 ** -24 * terms
    assert np.isfinite(out).all() and np.isfinite(lse).all()
    assert (np.abs(lse - want_lse) <= error[..., 0] + 2.0 ** -10 + 2.0 ** -22 * np.abs(want_lse)).all()
    alone = _margin(q, p.cache, p.table, p.lengths, p.news, p.dim ** -0.5, 0, 0) > 4 * error[..., 0] + 40
    assert size < 2.0 ** 8 or alone.mean() > 0.9
    off = np.abs(out[alone].astype(np.float64) - want[alone]) - ((2.0 ** -10 + 2.0 ** -18) * np.abs(want[alone]) + 2.0 ** -24)
    assert off.max(initial=0) <= 0, off.max()


@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda c: "%d of %d bits" % c[-3::2])
@pytest.mark.parametrize("switches", ROUTES)
def test_rows_do_not_depend_on_one_another(gpu_lib, monkeypatch, layout, switches):
    """Every second query of another size: the others get the same bits, though their tiles' maxima grow at other keys."""
    import torch
    monkeypatch.setenv("VQ_SWITCHES", switches)
    p = Problem(43, *layout)
    results = []
    for gain in (1, 12):
        q = p.q.copy()
        q[:, ::2] *= np.float16(gain)
        results.append(_call(gpu_lib, p, q))
    torch.cuda.synchronize()
    assert torch.equal(results[0][0][:, 1::2], results[1][0][:, 1::2]) and torch.equal(results[0][1][:, 1::2], results[1][1][:, 1::2])
    assert not torch.equal(results[0][0], results[1][0])


@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda c: "%d of %d bits" % c[-3::2])
@pytest.mark.parametrize("switches", ROUTES)
def test_values_that_are_not_finite_reach_those_who_see_them_alone(gpu_lib, monkeypatch, layout, switches):
    """One value of a prefix and one of the middle of a sequence's new tokens: the others' results stay, bit for bit, and who sees one gets what vq_attention gives."""
    p = Problem(44, *layout)
    monkeypatch.setenv("VQ_SWITCHES", switches)
    clean = _call(gpu_lib, p, p.q)
    for kind in ["nan"] if p.cache.bits == 8 else ["nan", "inf", "-inf"]:
        _one_value(gpu_lib, monkeypatch, p, clean, switches, kind)


def _one_value(gpu_lib, monkeypatch, p, clean, switches, kind):
    import copy
    import torch
    monkeypatch.setenv("VQ_SWITCHES", switches)
    cache, size = copy.deepcopy(p.cache), p.cache.size
    bad = 0x7F if p.cache.bits == 8 else np.float16(kind)
    cache.v[p.prefix_table[0, 40 // size], 0, 3, 40 % size] = bad
    first = int(p.members[1]) - 1                                   # the first prefix's last sequence
    place = p.lengths[first] - 1 - p.news[first] // 2
    cache.v[p.table[first, place // size], 0, 5, place % size] = bad
    out, lse = _call(gpu_lib, p, p.q, cache)
    monkeypatch.setenv("VQ_SWITCHES", "")
    want, want_lse = _plain(gpu_lib, p, p.q, cache)
    torch.cuda.synchronize()
    assert torch.equal(lse, clean[1])
    for same in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(same(out), same(want))
    fine = torch.isfinite(out)
    assert torch.equal(out[fine], clean[0][fine])
    group, rows = p.q.shape[1] // p.cache.heads, np.concatenate([[0], np.cumsum(p.news)])
    hit = np.zeros(out.shape, bool)
    hit[: rows[p.members[1]], :group, 3] = True
    hit[rows[first] + p.news[first] - 1 - p.news[first] // 2: rows[first + 1], :group, 5] = True
    assert np.array_equal(~fine.cpu().numpy(), hit)


@pytest.mark.parametrize("switches", ROUTES)
@pytest.mark.parametrize("bits", [8, 16])
def test_pages_past_32_bits(gpu_lib, monkeypatch, switches, bits):
    """The same tokens in the first pages of a small pool and in the last ones of a pool of more than 2^32 bytes (a short cut of views of it)."""
    import torch
    monkeypatch.setenv("VQ_SWITCHES", switches)
    p = Problem(45, [(256, 250, [(70, 2), (9, 2)])], [], 4, 2, 128, 64, bits)
    dev, prefix = p.up()
    kind, raw, element = (torch.float8_e4m3fn, torch.uint8, 1) if bits == 8 else (torch.float16, torch.float16, 2)
    pitch, pages = 48 * 2 ** 20 // element, 100                     # pages 48 MiB apart: the hundredth lies behind 4.5 GiB
    first = pages - len(p.cache.k)
    room = torch.empty(2 * pages * pitch, dtype=raw, device="cuda").view(kind)
    views, scales = [], [None, None]
    for i, (theirs, scale) in enumerate(((dev.k, dev.k_scales), (dev.v, dev.v_scales))):
        view = room.as_strided((pages,) + tuple(theirs.shape[1:]), (pitch,) + theirs.stride()[1:], i * pages * pitch)
        view[first:].view(raw).copy_(theirs.view(raw))
        views.append(view)
        if bits == 8:
            scales[i] = torch.ones((pages, 2), device="cuda")
            scales[i][first:] = scale
    q = torch.from_numpy(p.q).cuda()
    small = gpu_lib.attention_shared(q, dev.k, dev.v, dev.table, dev.lengths, k_scales=dev.k_scales, v_scales=dev.v_scales, max_new=2, **prefix)
    moved = lambda t: torch.where(t >= 0, t + first, t)  # noqa: E731
    prefix["prefix_table"] = moved(prefix["prefix_table"])
    large = gpu_lib.attention_shared(q, *views, moved(dev.table), dev.lengths, k_scales=scales[0], v_scales=scales[1], max_new=2, **prefix)
    torch.cuda.synchronize()
    assert torch.equal(small, large)


def test_graphs_that_share_a_workspace(gpu_lib, monkeypatch):
    """Two calls of different layouts captured with the same workspace, replayed in turn with eager calls between."""
    import torch
    monkeypatch.setenv("VQ_SWITCHES", "shared=1")
    workspace, graphs = torch.empty(64 << 20, dtype=torch.uint8, device="cuda"), []
    for seed, layout in ((46, LAYOUTS[0]), (47, LAYOUTS[1])):
        p = Problem(seed, *layout)
        dev, prefix = p.up()
        args = (torch.from_numpy(p.q).cuda(), dev.k, dev.v, dev.table, dev.lengths)
        kw = dict(k_scales=dev.k_scales, v_scales=dev.v_scales, starts=dev.starts, max_new=max(p.news), workspace=workspace, **prefix)

        def call(args=args, kw=kw):
            return gpu_lib.attention_shared(*args, **kw)
        want = call().clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        graphs.append((graph, out, want, call))
    for i in range(6):
        graph, out, want, call = graphs[i % 2]
        out.zero_()
        graph.replay()
        assert torch.equal(graphs[1 - i % 2][3](), graphs[1 - i % 2][2])
        torch.cuda.synchronize()
        assert torch.equal(out, want)
