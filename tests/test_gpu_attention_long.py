"""vq_attention where sequences are cut into parts and where offsets pass 32 bits, and what the tensor entry points refuse.

Bound of the error: that of short sequences (probabilities rounded to binary16: relative 2^-11, absolute 2^-25 below; scores of binary32 sums,
relative (head_dim + 2) 2^-24 of the sizes of their terms, once in the probability and once in the sum; exp2, divisions and the join of parts within 2^-18; the result rounded to
binary16: 2^-11), and for n keys the binary32 sums of up to n terms, added at least sixteen at a time: n / 16 + 64 roundings of 2^-24 of the terms' sizes."""
import numpy as np
import pytest

import kv_reference as ref
from test_gpu_attention import Device, _problem

pytestmark = pytest.mark.gpu


def _whole(cache, pages, length, h):
    """Keys and values [length][head_dim] of a sequence in 64 bits, and which of its places have a page."""
    blocks = -(-length // cache.size)
    there = np.array([0 <= p < len(cache.k) for p in pages[:blocks]], bool)
    use = np.where(there, pages[:blocks], 0)
    k, v = cache.k[use, h], np.swapaxes(cache.v[use, h], 1, 2)
    if cache.bits == 8:
        k, v = ref.values(k) * cache.k_scales[use, h][:, None, None], ref.values(v) * cache.v_scales[use, h][:, None, None]
    flat = [a.astype(np.float64).reshape(-1, cache.dim)[:length] for a in (k, v)]
    return (*flat, np.repeat(there, cache.size)[:length])


def _attention(q, cache, table, lengths, news, scale, window, sinks):
    """As kv_reference.attention, a sequence's head at a time."""
    tokens, q_heads, dim = q.shape
    group = q_heads // cache.heads
    out, weight, floor = (np.zeros((tokens, q_heads, dim)) for _ in range(3))
    lse, terms = np.full((tokens, q_heads), -np.inf), np.zeros((tokens, q_heads, 1))
    row = 0
    for pages, length, new in zip(table, lengths, news):
        rows, places = np.arange(row, row + new), np.arange(length)
        at = length - new + np.arange(new)
        row += new
        if not length or not new:
            continue
        for h in range(cache.heads):
            K, V, there = _whole(cache, pages, length, h)
            sees = there & (places <= at[:, None])
            if window:
                sees &= (places > at[:, None] - window) | (places < sinks)
            anyone = sees.any(0)
            K, V, sees = K[anyone], V[anyone], sees[:, anyone]
            some = sees.any(1)
            if not some.any():
                continue
            for g in range(h * group, (h + 1) * group):
                x = q[rows[some], g].astype(np.float64)
                s = np.where(sees[some], x @ K.T * scale, -np.inf)
                most = s.max(1, keepdims=True)
                p = np.exp(s - most)
                total = p.sum(1, keepdims=True)
                out[rows[some], g] = p @ V / total
                weight[rows[some], g] = p @ np.abs(V) / total
                floor[rows[some], g] = sees[some].astype(float) @ np.abs(V) / total
                lse[rows[some], g] = (most + np.log(total))[:, 0]
                terms[rows[some], g, 0] = np.where(sees[some], np.abs(x) @ np.abs(K).T, 0).max(1) * scale
    return out, lse, weight, floor, terms


def _check(got, lse, want, want_lse, weight, floor, terms, dim, keys):
    sums = (keys / 16 + 64) * 2.0 ** -24
    scores = 2 * (dim + 2) * 2.0 ** -24 * terms
    bound = (2.0 ** -10 + 2.0 ** -18 + 2 * sums + scores) * weight + 2.0 ** -25 * floor + 2.0 ** -24
    off = np.abs(got.astype(np.float64) - want) - bound
    assert np.isfinite(got).all() and off.max() <= 0, (np.unravel_index(off.argmax(), off.shape), off.max())
    empty = ~np.isfinite(want_lse)
    assert np.array_equal(empty, lse == -np.inf)
    near = np.abs(lse[~empty] - want_lse[~empty])
    assert (near <= scores[..., 0][~empty] + 2.0 ** -18 + sums + 2.0 ** -22 * np.abs(want_lse[~empty])).all(), near.max()


LONG = [
    # lengths, news, q heads, heads, dim, page, bits, window, sinks
    ([5000, 3, 0], [1, 1, 1], 8, 2, 128, 16, 8, 0, 0),              # beside sequences that have one part or none
    ([4097, 4096], [1, 1], 4, 1, 64, 64, 16, 0, 0),
    ([9001], [1], 32, 1, 128, 128, 8, 0, 0),                        # more queries a key than sixteen
    ([3000, 700], [8, 5], 8, 2, 128, 16, 16, 0, 0),                 # drafted tokens, ragged
    ([2800, 1000], [9, 9], 8, 2, 64, 32, 8, 0, 0),
    ([6000, 2500], [1, 1], 8, 2, 128, 16, 8, 3001, 7),              # a window of parts
    ([6000, 2500], [3, 2], 4, 2, 64, 16, 16, 2050, 130),
    ([2600, 2050], [70, 64], 4, 2, 128, 16, 8, 0, 0),               # short chunks behind long contexts
    ([2600, 2050, 30], [257, 64, 30], 4, 2, 128, 64, 16, 0, 0),
    ([3100], [200], 2, 1, 64, 256, 8, 0, 0),
    ([5000], [150], 4, 1, 128, 32, 8, 2200, 100),
    ([200, 2600], [300, 300], 2, 1, 64, 16, 16, 1500, 40),          # rows that see nothing beside ones of parts
]


@pytest.mark.parametrize("case", LONG, ids=str)
def test_sequences_in_parts(gpu_lib, case):
    import torch
    lengths, news, q_heads, heads, dim, size, bits, window, sinks = case
    lost = [(b, i) for b, (n, m) in enumerate(zip(lengths, news)) for i in range(-(-n // size))
            if window and (i + 1) * size <= n - m - window + 1 and i * size >= sinks]
    rng, cache, table, k, v, q = _problem(21, lengths, news, q_heads, heads, dim, size, bits, fill="nan", lost=lost)
    cache.append(k, v, table, lengths, news)
    scale = 1.1 / np.sqrt(dim)
    dev = Device(cache, table, lengths, news, uniform=len(set(news)) == 1)
    qd = torch.from_numpy(q).cuda()
    args = dict(starts=dev.starts, scale=scale, window=window, sinks=sinks, max_new=max(news), max_length=max(lengths), return_lse=True)
    want = _attention(q, cache, table, lengths, news, scale, window, sinks)
    # its own parts, one part, and whatever fits the bounds that are known when nobody says more (the table's)
    for more in (dict(), dict(workspace=torch.empty(0, dtype=torch.uint8, device="cuda")), dict(max_length=None)):
        out, lse = gpu_lib.attention(qd, *dev.cache, **dict(args, **more))
        again, lse2 = gpu_lib.attention(qd, *dev.cache, **dict(args, **more))
        torch.cuda.synchronize()
        assert torch.equal(out, again) and torch.equal(lse, lse2)
        _check(out.cpu().numpy(), lse.cpu().numpy(), *want, dim, max(lengths))


def test_long_cases_are_cut(gpu_lib):
    """Most of the cases above are taken in parts: their workspace is not empty."""
    import ctypes
    cut = 0
    for lengths, news, q_heads, heads, dim, size, bits, window, sinks in LONG:
        d = gpu_lib.vq_kv_desc(struct_size=ctypes.sizeof(gpu_lib.vq_kv_desc), type=gpu_lib.VQ_KV_E4M3 if bits == 8 else gpu_lib.VQ_KV_FP16, kv_heads=heads,
                               head_dim=dim, page_tokens=size, n_pages=1, n_seqs=len(news), n_tokens=sum(news), max_new=max(news), max_length=max(lengths),
                               table_pages=1000, k_pages=16, v_pages=16, k_page_stride=heads * dim * size, v_page_stride=heads * dim * size, k_scales=16,
                               v_scales=16, page_table=16, table_stride=1000, lengths=16, starts=16)
        cut += gpu_lib.vq_attention_workspace_bytes(d, q_heads, window, sinks) > 0
    assert cut >= 9


@pytest.mark.parametrize("dim", [16, 32, 48, 80, 96, 112, 144, 192, 208, 256])
@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("lengths,news,q_heads,heads,window,sinks", [
    ([1900, 3, 64], [1, 1, 1], 8, 2, 0, 0),
    ([1400, 90], [5, 3], 4, 2, 500, 5),
    ([700, 40], [300, 40], 2, 1, 0, 0),
    ([1700], [140], 2, 2, 0, 0),
], ids=str)
def test_heads_of_other_sizes(gpu_lib, dim, bits, lengths, news, q_heads, heads, window, sinks):
    """Between heads stand NaN (unseen places of the pages) and other heads; the last page of the pool is in use."""
    import torch
    size = 16 if dim < 100 else 64
    rng, cache, table, k, v, q = _problem(25, lengths, news, q_heads, heads, dim, size, bits, fill="nan", spare=0)
    cache.append(k, v, table, lengths, news)
    dev = Device(cache, table, lengths, news)
    qd = torch.from_numpy(q).cuda()
    args = dict(starts=dev.starts, window=window, sinks=sinks, max_new=max(news), max_length=max(lengths), return_lse=True)
    out, lse = gpu_lib.attention(qd, *dev.cache, **args)
    again, lse2 = gpu_lib.attention(qd, *dev.cache, **args)
    torch.cuda.synchronize()
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    _check(out.cpu().numpy(), lse.cpu().numpy(), *_attention(q, cache, table, lengths, news, dim ** -0.5, window, sinks), dim, max(lengths))


@pytest.mark.parametrize("dim,bits", [(80, 8), (80, 16), (48, 16), (192, 8), (192, 16), (256, 8), (256, 16)])
@pytest.mark.parametrize("news", [[7, 1], [150, 60]], ids=str)
def test_values_that_are_not_finite_in_heads_of_other_sizes(gpu_lib, dim, bits, news):
    """In the last element of the first head, and the first of the second: rows that see them get what the sums give, others what they get without."""
    import torch
    lengths, heads, size = [300, 190], 2, 16
    rng, cache, table, k, v, q = _problem(26, lengths, news, 2, heads, dim, size, bits)
    cache.append(k, v, table, lengths, news)
    args = dict(max_new=max(news), max_length=max(lengths))

    def run():
        dev = Device(cache, table, lengths, news)
        return gpu_lib.attention(torch.from_numpy(q).cuda(), *dev.cache, starts=dev.starts, **args)
    want = run()
    place = lengths[0] - 3                              # seen by the last three of the first sequence's tokens
    for head, element, value in ((0, dim - 1, np.nan if bits == 8 else -np.inf), (1, 0, np.nan)):
        cache.v[table[0, place // size], head, element, place % size] = 0x7f if bits == 8 else value
    got = run()
    torch.cuda.synchronize()
    hit = torch.zeros(got.shape, dtype=torch.bool, device="cuda")
    rows = slice(max(news[0] - 3, 0), news[0])
    hit[rows, 0, dim - 1] = hit[rows, 1, 0] = True
    assert torch.equal(got[~hit], want[~hit])
    assert torch.isnan(got[rows, 1, 0]).all() and (torch.isnan(got[rows, 0, dim - 1]) if bits == 8 else got[rows, 0, dim - 1] == -np.inf).all()


@pytest.mark.parametrize("dim", [64, 80, 128])
def test_windows_and_first_tokens_longer_than_any_sequence(gpu_lib, dim):
    """The largest numbers see what no window sees, also beside tokens that see nothing (more new tokens than the sequence holds)."""
    import torch
    for lengths, news in (([3, 700], [8, 8]), ([5, 500], [90, 90])):
        rng, cache, table, k, v, q = _problem(27, lengths, news, 4, 2, dim, 16, 8)
        cache.append(k, v, table, lengths, news)
        dev, qd = Device(cache, table, lengths, news, uniform=True), torch.from_numpy(q).cuda()
        args = dict(max_new=news[0], max_length=max(lengths), return_lse=True)
        want = gpu_lib.attention(qd, *dev.cache, **args)
        for window, sinks in ((2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (max(lengths), 0), (1, 2 ** 31 - 1), (40, max(lengths))):
            got = gpu_lib.attention(qd, *dev.cache, window=window, sinks=sinks, **args)
            torch.cuda.synchronize()
            _check(got[0].cpu().numpy(), got[1].cpu().numpy(), *_attention(q, cache, table, lengths, news, dim ** -0.5, 0, 0), dim, max(lengths))
            assert torch.equal(got[1] == -float("inf"), want[1] == -float("inf"))


def test_many_sequences(gpu_lib):
    import torch
    rng = np.random.default_rng(22)
    lengths, heads, dim, size = list(rng.integers(0, 90, 150)), 2, 64, 16
    for bits in (8, 16):
        _, cache, table, k, v, q = _problem(22, lengths, [1] * 150, 4, heads, dim, size, bits, fill="nan")
        cache.append(k, v, table, lengths, [1] * 150)
        dev = Device(cache, table, lengths, [1] * 150, uniform=True)
        out, lse = gpu_lib.attention(torch.from_numpy(q).cuda(), *dev.cache, return_lse=True)
        torch.cuda.synchronize()
        _check(out.cpu().numpy(), lse.cpu().numpy(), *_attention(q, cache, table, lengths, [1] * 150, dim ** -0.5, 0, 0), dim, 90)


@pytest.mark.parametrize("news,dim,bits", [([1], 128, 8), ([1], 64, 16), ([90], 128, 8), ([40], 64, 16)])
def test_an_infinity_in_a_later_part(gpu_lib, news, dim, bits):
    """A value's infinity (in 8 bits NaN) far behind the first part reaches its element of every row that sees it, and no other."""
    import torch
    lengths, heads, size = [4500], 1, 16
    rng, cache, table, k, v, q = _problem(23, lengths, news, 4, heads, dim, size, bits)
    cache.append(k, v, table, lengths, news)
    args = dict(max_new=news[0], max_length=lengths[0])
    want = gpu_lib.attention(torch.from_numpy(q).cuda(), *Device(cache, table, lengths, news, uniform=True).cache, **args)
    place = 3900
    cache.v[table[0, place // size], 0, 5, place % size] = 0x7f if bits == 8 else -np.inf
    got = gpu_lib.attention(torch.from_numpy(q).cuda(), *Device(cache, table, lengths, news, uniform=True).cache, **args)
    torch.cuda.synchronize()
    hit = torch.zeros(dim, dtype=torch.bool, device="cuda")
    hit[5] = True
    assert torch.equal(got[..., ~hit], want[..., ~hit])
    assert (torch.isnan(got[..., 5]) if bits == 8 else got[..., 5] == -np.inf).all()


@pytest.mark.parametrize("dim,bits", [(128, 8), (64, 16), (80, 8)])
@pytest.mark.parametrize("news", [[1, 1], [60, 33]], ids=str)
def test_pages_past_32_bits(gpu_lib, dim, bits, news):
    """The same tokens in the first pages of a small pool and in the last ones of a pool of more than 2^32 bytes (a short cut of views of it)."""
    import torch
    lengths, heads, size = [700, 90], 2, 64
    rng, cache, table, k, v, q = _problem(24, lengths, news, 4, heads, dim, size, bits)
    small = Device(cache, table, lengths, news)
    up = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    kind, element = (torch.float8_e4m3fn, 1) if bits == 8 else (torch.float16, 2)
    pitch = 48 * 2 ** 20 // element                     # pages 48 MiB apart: the hundredth lies behind 4.5 GiB
    pages = 100
    first = pages - len(cache.k)
    table2 = np.where(table >= 0, table + first, -1).astype(np.int32)
    big = Device(cache, table2, lengths, news)
    room = torch.empty(2 * pages * pitch, dtype=torch.uint8 if bits == 8 else kind, device="cuda").view(kind)
    assert (pages - 1) * pitch * element > 2 ** 32
    views = []
    for i, theirs in enumerate((small.k, small.v)):
        view = room.as_strided((pages,) + tuple(theirs.shape[1:]), (pitch,) + theirs.stride()[1:], i * pages * pitch)
        view[first:].view(torch.uint8 if bits == 8 else kind).copy_(theirs.view(torch.uint8 if bits == 8 else kind))
        views.append(view)
    scales = [None, None]
    if bits == 8:
        for i, theirs in enumerate((small.k_scales, small.v_scales)):
            scales[i] = torch.ones((pages, heads), device="cuda")
            scales[i][first:] = theirs
    results = []
    for k_pages, v_pages, t, k_scales, v_scales in ((small.k, small.v, small.table, small.k_scales, small.v_scales), (*views, big.table, *scales)):
        place = (k_pages, v_pages, t, small.lengths, k_scales, v_scales)
        gpu_lib.kv_append(up(k), up(v), *place, starts=small.starts, max_new=max(news))
        results.append(gpu_lib.attention(up(q), *place, starts=small.starts, max_new=max(news), max_length=max(lengths)))
    torch.cuda.synchronize()
    assert torch.equal(*results)
    raw = torch.uint8 if bits == 8 else torch.float16
    for view, theirs in zip(views, (small.k, small.v)):
        assert torch.equal(view[first:].contiguous().view(raw), theirs.contiguous().view(raw))


def _small(torch, bits=8):
    kind = torch.float8_e4m3fn if bits == 8 else torch.float16
    pages = [torch.zeros(s, dtype=torch.float16, device="cuda").to(kind) for s in ((6, 2, 16, 64), (6, 2, 64, 16))]
    table, lengths = torch.arange(6, dtype=torch.int32, device="cuda").reshape(2, 3), torch.tensor([20, 40], dtype=torch.int32, device="cuda")
    scales = [torch.ones((6, 2), device="cuda") if bits == 8 else None for _ in range(2)]
    new = lambda heads: torch.zeros((4, heads, 64), dtype=torch.float16, device="cuda")  # noqa: E731
    return pages + [table, lengths] + scales, new


def test_tensors_that_are_refused(gpu_lib):
    import torch
    cache, new = _small(torch)
    bad_caches = {
        0: [cache[0].float(), cache[0][0], cache[0].transpose(2, 3), cache[0][:, :1], cache[0].cpu(), None, 7],
        1: [cache[1].transpose(2, 3), cache[1][:5], cache[1].view(torch.uint8), cache[0]],
        2: [cache[2].long(), cache[2][:1], cache[2][0], cache[2].t().contiguous().t(), cache[2].cpu()],
        3: [cache[3].long(), cache[3][:1], cache[3].float(), cache[3].reshape(2, 1), torch.zeros(4, dtype=torch.int32, device="cuda")[::2]],
        4: [None, cache[4].half(), cache[4][:5], cache[4].t().contiguous().t(), cache[4][:, :1]],
        5: [None, cache[5].double(), cache[5].reshape(-1)],
    }
    for i, bads in bad_caches.items():
        for bad in bads:
            place = list(cache)
            place[i] = bad
            with pytest.raises(ValueError):
                gpu_lib.kv_append(new(2), new(2), *place)
            with pytest.raises(ValueError):
                gpu_lib.attention(new(4), *place)
    sixteen, _ = _small(torch, 16)
    with pytest.raises(ValueError):
        gpu_lib.attention(new(4), *sixteen[:4], k_scales=cache[4], v_scales=cache[5])           # 16-bit pages have no scales
    table = torch.zeros((48, 32), device="cuda")
    for kw in (dict(k=new(3)), dict(k=new(2)[:3]), dict(v=new(2).float()), dict(k=new(2).transpose(0, 1)), dict(k=torch.zeros((4, 2, 80), dtype=torch.float16, device="cuda")),
               dict(q=new(4)[:2]), dict(q=new(4)[..., :32]), dict(q=new(4), q_out=new(2)), dict(q_out=new(4)), dict(cos=table), dict(sin=table),
               dict(cos=table, sin=table.half()), dict(cos=table, sin=table[:, :16]), dict(cos=table.t(), sin=table.t()), dict(cos=table, sin=table, position=cache[3]),
               dict(starts=cache[3]), dict(max_new="2"), dict(max_length=2 ** 40)):
        with pytest.raises(ValueError):
            gpu_lib.kv_append(**dict(dict(zip(("k", "v", "k_pages", "v_pages", "page_table", "lengths", "k_scales", "v_scales"), [new(2), new(2)] + cache)), **kw))
    for kw in (dict(q=new(4).float()), dict(q=new(4)[0]), dict(q=new(4)[..., ::2]), dict(out=new(2)), dict(out=new(4).cpu()), dict(scale="x"), dict(window=1.5),
               dict(workspace=torch.zeros(4, device="cuda")), dict(starts=cache[3]), dict(sinks=2 ** 33)):
        with pytest.raises(ValueError):
            gpu_lib.attention(**dict(dict(zip(("q", "k_pages", "v_pages", "page_table", "lengths", "k_scales", "v_scales"), [new(4)] + cache)), **kw))
    # what the library itself refuses
    for call in (lambda: gpu_lib.attention(new(3), *cache), lambda: gpu_lib.attention(new(4)[:3], *cache), lambda: gpu_lib.attention(new(4), *cache, max_new=1),
                 lambda: gpu_lib.attention(new(4), *cache, max_length=49), lambda: gpu_lib.attention(new(4), *cache, scale=0.0),
                 lambda: gpu_lib.attention(new(4)[:0], *cache), lambda: gpu_lib.kv_append(new(2)[:0], new(2)[:0], *cache),
                 lambda: gpu_lib.kv_append(new(2)[:1].expand(4, 2, 64), new(2), *cache)):
        with pytest.raises(gpu_lib.VQError):
            call()
    torch.cuda.synchronize()
    assert not cache[0].view(torch.uint8).any() and not cache[1].view(torch.uint8).any()


def test_rows_and_weights_that_are_refused(gpu_lib):
    import torch
    x = torch.zeros((3, 64), dtype=torch.float16, device="cuda")
    w = torch.ones(64, dtype=torch.float16, device="cuda")
    for kw in (dict(h=x[:2]), dict(h=x[:, :32]), dict(h=x.float()), dict(x=x.double()), dict(x=x.cpu()), dict(x=x[0]), dict(pre=w[:32]), dict(pre=w.float()),
               dict(post=w[None]), dict(gate=x[:2]), dict(gate=w[:3]), dict(y=x.float()), dict(y=x[:2]), dict(z=x.t()), dict(z=x, pre=None), dict(eps="x"), dict(scale=None),
               dict(h=torch.zeros((64, 3), dtype=torch.float16, device="cuda").t()), dict(h=None, x=None)):
        with pytest.raises(ValueError):
            gpu_lib.residual_norm(**dict(dict(h=x, x=x, pre=w), **kw))
    for kw in (dict(h=None, gate=w), dict(h=None, post=w), dict(eps=-1.0), dict(x=x[:0], h=x[:0]), dict(x=x[:1].expand(3, 64))):
        with pytest.raises(gpu_lib.VQError):
            gpu_lib.residual_norm(**dict(dict(h=x, x=x, pre=w), **kw))
