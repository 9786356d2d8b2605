"""vq_kv_append and vq_attention on the GPU: the cache bit for bit, attention against 64 bits.

Bound of attention's error, element by element, from its arithmetic: the probabilities are rounded to binary16 (relative 2^-11, absolute
2^-25 where they are subnormal), scores are binary32 sums of exact products (head_dim terms, then the scale: relative (head_dim + 2) 2^-24 of the sum of
the terms' sizes; an error e of a score is one of e of its probability, and once more in the sum), exp2, the running sums over up to n
keys and the division are within 2^-18, and the result is rounded to binary16 (2^-11, subnormal 2^-25)."""
import numpy as np
import pytest

import kv_reference as ref

pytestmark = pytest.mark.gpu


def _problem(seed, lengths, news, q_heads, heads, dim, size, bits, fill="stale", spare=2, lost=()):
    """A cache whose sequences hold their tokens but for the new ones, those, and the queries.  lost: (sequence, block) entries of the
    table that are -1."""
    rng = np.random.default_rng(seed)
    blocks = [-(-n // size) for n in lengths]
    pool = sum(blocks) + spare
    pages = rng.permutation(pool)
    table = np.full((len(lengths), max(blocks + [1]) + 1), -1, np.int32)
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = pages[at: at + n]
        at += n
    for b, block in lost:
        table[b, block] = -1
    cache = ref.Cache(rng, pool, heads, size, dim, bits, fill)
    gain = np.exp(rng.standard_normal((heads, dim)) * 0.5)

    def rows(n):
        return ((rng.standard_normal((n, heads, dim)) * gain).astype(np.float16), rng.standard_normal((n, heads, dim)).astype(np.float16))
    before = [max(0, n - m) for n, m in zip(lengths, news)]
    cache.append(*rows(sum(before)), table, before, before)
    k, v = rows(sum(news))
    q = rng.standard_normal((sum(news), q_heads, dim)).astype(np.float16)
    return rng, cache, table, k, v, q


class Device:
    def __init__(self, cache, table, lengths, news, uniform=False, pitch=0):
        import torch
        def up(a):
            return None if a is None else torch.from_numpy(a).cuda()
        kind = torch.float8_e4m3fn if cache.bits == 8 else torch.float16

        def pages(a):
            """With a pitch, pages lie further apart than their size."""
            t = up(a)
            t = t.view(kind) if cache.bits == 8 else t
            if not pitch:
                return t
            room = torch.zeros((t.shape[0], t[0].numel() + pitch), dtype=torch.uint8 if cache.bits == 8 else torch.float16, device="cuda")
            room = room.view(kind)
            view = room[:, : t[0].numel()].view(t.shape) if t.shape[0] == 1 else room.as_strided(t.shape, (room.shape[1],) + t.stride()[1:])
            view.copy_(t)
            return view
        self.k, self.v, self.k_scales, self.v_scales = pages(cache.k), pages(cache.v), up(cache.k_scales), up(cache.v_scales)
        self.table, self.lengths = up(table), torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.starts = None if uniform else torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32, device="cuda")
        self.cache = (self.k, self.v, self.table, self.lengths, self.k_scales, self.v_scales)

    def equals(self, cache):
        import torch
        for mine, theirs in ((self.k, cache.k), (self.v, cache.v)):
            mine = mine.contiguous().view(torch.uint8).cpu().numpy() if cache.bits == 8 else mine.cpu().numpy().view(np.uint16)
            theirs = theirs if cache.bits == 8 else theirs.view(np.uint16)
            if cache.bits == 8:                          # NaN is NaN, of either sign
                same = (mine == theirs) | ((mine & 0x7f == 0x7f) & (theirs & 0x7f == 0x7f))
            else:
                nan = lambda x: (x & 0x7fff) > 0x7c00  # noqa: E731
                same = (mine == theirs) | (nan(mine) & nan(theirs))
            assert same.all(), np.argwhere(~same)[:4]
        for mine, theirs in ((self.k_scales, cache.k_scales), (self.v_scales, cache.v_scales)):
            assert theirs is None or np.array_equal(mine.cpu().numpy(), theirs)


def _tables(rng, positions, pairs):
    angle = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(pairs) / pairs)
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


APPENDS = [
    # lengths, news, q heads, heads, dim, page, bits, pairs, interleaved
    ([1], [1], 4, 4, 128, 16, 8, 64, False),                        # the very first token
    ([9], [1], 4, 4, 128, 16, 8, 64, False),                        # behind eight others in a page
    ([17], [1], 2, 2, 64, 16, 8, 32, True),                         # the first of a page
    ([16, 33, 5], [16, 33, 5], 4, 2, 64, 16, 8, 32, False),         # prompts
    ([40, 21, 130], [5, 5, 5], 8, 2, 128, 32, 8, 64, False),        # drafted tokens across pages
    ([50, 0, 7], [3, 0, 7], 3, 1, 96, 16, 16, 48, False),           # a sequence without any, 16 bits
    ([300, 129], [260, 129], 2, 2, 64, 128, 8, 32, True),           # more than one tile of a page
    ([300, 257], [299, 1], 2, 1, 32, 256, 16, 16, False),
    ([70, 70], [70, 3], 5, 5, 80, 64, 8, 10, False),                # partial rotation, pairs that are no multiple of eight
    ([70, 70], [70, 3], 5, 5, 80, 64, 8, 10, True),
    ([70, 4], [37, 4], 2, 2, 16, 16, 8, 0, False),                  # no rotation, the smallest head
    ([20, 3], [20, 3], 2, 1, 256, 16, 8, 128, False),
]


@pytest.mark.parametrize("case", APPENDS, ids=str)
@pytest.mark.parametrize("in_place", [False, True])
def test_append_bit_for_bit(gpu_lib, case, in_place):
    import torch
    lengths, news, q_heads, heads, dim, size, bits, pairs, interleaved = case
    rng, cache, table, k, v, q = _problem(7, lengths, news, q_heads, heads, dim, size, bits)
    k *= np.float16(4)                                              # scales grow, and what is there is encoded again
    cos, sin = _tables(rng, max(lengths) - 2 if max(lengths) > 4 else max(lengths), pairs) if pairs else (None, None)      # (places past the table take its last row)
    dev = Device(cache, table, lengths, news)
    up = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    # rows further apart than their heads, and not on 16 bytes
    wide = torch.zeros((len(q), 2 * heads * dim + q_heads * dim + 1), dtype=torch.float16, device="cuda")
    at = 0
    views = []
    for a in (k, v, q):
        n = a.shape[1] * dim
        views.append(wide[:, at: at + n].unflatten(1, (a.shape[1], dim)))
        views[-1].copy_(up(a))
        at += n
    args = dict(q=views[2], cos=up(cos), sin=up(sin), interleaved=interleaved, starts=dev.starts, max_new=max(news), q_out=views[2] if in_place else None)
    got = gpu_lib.kv_append(views[0], views[1], *dev.cache, **args)
    torch.cuda.synchronize()
    cache.append(k, v, table, lengths, news, cos, sin, None, interleaved)
    dev.equals(cache)
    row = 0
    for length, new in zip(lengths, news):
        for t in range(new):
            at = min(length - new + t, len(cos) - 1) if pairs else 0
            want = ref.rotate(q[row], cos[at], sin[at], interleaved).astype(np.float16) if pairs else q[row]
            assert np.array_equal(got[row].cpu().numpy().view(np.uint16), want.view(np.uint16)), (row, t)
            row += 1
    if not in_place:                                                # the same call again changes nothing
        again = gpu_lib.kv_append(views[0], views[1], *dev.cache, **args)
        torch.cuda.synchronize()
        dev.equals(cache)
        assert torch.equal(again, got)


def test_append_of_what_is_not_finite_and_of_positions_of_its_own(gpu_lib):
    import torch
    lengths, news, heads, dim, size = [30, 12], [13, 12], 2, 64, 16
    for bits in (8, 16):
        rng, cache, table, k, v, q = _problem(8, lengths, news, 2, heads, dim, size, bits)
        k[3, 0, 5], k[4, 1, 60], v[2, 0, 1], v[7, 1, 9] = np.inf, np.nan, -np.inf, np.nan
        k[13:16] = 0                                                # a page's head of zeros but for later tokens
        v[13:25, 1] = 0                                             # of zeros alone
        v[20, 0, 3] = 65504
        k[20] = np.float16(2.0 ** -24)
        position = rng.integers(-3, 50, sum(news)).astype(np.int32)
        cos, sin = _tables(rng, 40, 32)
        dev = Device(cache, table, lengths, news)
        up = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
        gpu_lib.kv_append(up(k), up(v), *dev.cache, cos=up(cos), sin=up(sin), position=up(position), starts=dev.starts)
        torch.cuda.synchronize()
        cache.append(k, v, table, lengths, news, cos, sin, position)
        dev.equals(cache)


def test_append_leaves_out_what_the_arrays_name_outside_of_the_buffers(gpu_lib):
    """Entries of the table that name no page, lengths shorter than the new tokens and beyond the longest, more new tokens than max_new."""
    import torch
    heads, dim, size = 2, 64, 16
    lengths, news = [40, 5, 20], [30, 5, 20]
    rng, cache, table, k, v, q = _problem(9, lengths, news, 2, heads, dim, size, 8, lost=((0, 1),))
    table[2, 1] = 10 ** 6
    dev = Device(cache, table, lengths, news)
    up = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    gpu_lib.kv_append(up(k), up(v), *dev.cache, starts=dev.starts)
    torch.cuda.synchronize()
    cache.append(k, v, table, lengths, news)
    dev.equals(cache)
    # sequence 0 is two tokens long and brings thirty, 1 has none, 2 is longer than max_length, and rows end early
    dev.lengths.copy_(torch.tensor([2, 0, 1000], dtype=torch.int32))
    dev.starts.copy_(torch.tensor([0, 30, 35, 4000], dtype=torch.int32))
    gpu_lib.kv_append(up(k), up(v), *dev.cache, starts=dev.starts, max_new=30, max_length=40)
    torch.cuda.synchronize()
    cache.append(k[28:30], v[28:30], table[:1], [2], [2])
    dev.equals(cache)


def _check(got, lse, want, want_lse, weight, floor, terms, dim):
    scores = 2 * (dim + 2) * 2.0 ** -24 * terms
    bound = (2.0 ** -10 + 2.0 ** -18 + scores) * weight + 2.0 ** -25 * floor + 2.0 ** -24
    off = np.abs(got.astype(np.float64) - want) - bound
    assert np.isfinite(got).all() and off.max() <= 0, (np.unravel_index(off.argmax(), off.shape), off.max())
    if lse is not None:
        empty = ~np.isfinite(want_lse)
        assert np.array_equal(empty, lse == -np.inf)
        near = np.abs(lse[~empty] - want_lse[~empty])
        assert (near <= scores[..., 0][~empty] + 2.0 ** -18 + 2.0 ** -22 * np.abs(want_lse[~empty])).all(), near.max()


ATTENDS = [
    # lengths, news, q heads, heads, dim, page, bits, window, sinks
    ([1], [1], 1, 1, 128, 16, 8, 0, 0),                             # a token that sees itself alone
    ([1], [1], 4, 4, 64, 16, 16, 0, 0),
    ([63], [1], 8, 8, 128, 16, 8, 0, 0),
    ([64, 65, 130], [1, 1, 1], 8, 1, 128, 16, 8, 0, 0),
    ([509, 31], [1, 1], 28, 4, 128, 32, 8, 0, 0),                   # seven queries a key
    ([1023, 2, 700], [1, 1, 1], 8, 2, 64, 64, 16, 0, 0),
    ([1500], [1], 64, 1, 128, 128, 8, 0, 0),                        # more queries a key than a tile has rows
    ([700, 300], [4, 4], 8, 8, 128, 16, 16, 0, 0),                  # drafted tokens
    ([200, 90, 77], [5, 1, 3], 16, 2, 128, 16, 8, 0, 0),            # ragged ones
    ([333, 70], [16, 16], 8, 2, 64, 256, 8, 0, 0),
    ([900, 400, 30], [1, 1, 1], 8, 2, 128, 16, 8, 100, 4),          # window and first tokens
    ([900, 400, 30], [1, 1, 1], 8, 2, 64, 16, 16, 64, 0),
    ([900, 130], [9, 9], 4, 2, 128, 32, 8, 1, 70),                  # a window of the token itself
    ([300], [300], 2, 2, 128, 16, 8, 0, 0),                         # a prompt
    ([257, 100, 1], [257, 40, 1], 4, 1, 64, 16, 16, 0, 0),
    ([520, 300], [129, 300], 4, 2, 128, 64, 8, 90, 5),              # chunks with a window
    ([450], [200], 6, 2, 64, 128, 8, 33, 130),
    ([200], [100], 4, 1, 80, 16, 8, 0, 0),                          # heads of other sizes
    ([200, 50], [1, 1], 6, 3, 256, 16, 8, 60, 2),
    ([77], [30], 2, 1, 16, 32, 16, 0, 0),
    ([3, 150], [8, 8], 4, 2, 128, 16, 8, 0, 0),                     # more new tokens than the sequence holds: rows that see nothing
    ([0, 90], [1, 1], 8, 2, 128, 16, 8, 0, 0),                      # an empty slot
    ([2, 150], [90, 90], 4, 2, 64, 16, 16, 20, 1),
]


@pytest.mark.parametrize("case", ATTENDS, ids=str)
@pytest.mark.parametrize("with_workspace", [True, False])
def test_attention(gpu_lib, case, with_workspace):
    import torch
    lengths, news, q_heads, heads, dim, size, bits, window, sinks = case
    # what nobody sees is NaN; with a window, its pages are given back
    lost = [(b, i) for b, (n, m) in enumerate(zip(lengths, news)) for i in range(-(-n // size))
            if window and (i + 1) * size <= n - m - window + 1 and i * size >= sinks]
    rng, cache, table, k, v, q = _problem(11, lengths, news, q_heads, heads, dim, size, bits, fill="nan", lost=lost)
    cache.append(k, v, table, lengths, news)
    scale = 1.3 / np.sqrt(dim)
    dev = Device(cache, table, lengths, news, uniform=len(set(news)) == 1, pitch=0 if with_workspace else 32)
    qd = torch.zeros((len(q), q_heads * dim + 3), dtype=torch.float16, device="cuda")[:, 1: 1 + q_heads * dim].unflatten(1, (q_heads, dim))
    qd.copy_(torch.from_numpy(q))
    args = dict(starts=dev.starts, scale=scale, window=window, sinks=sinks, max_new=max(news), return_lse=True,
                workspace=None if with_workspace else torch.empty(0, dtype=torch.uint8, device="cuda"))
    out, lse = gpu_lib.attention(qd, *dev.cache, **args)
    again, lse2 = gpu_lib.attention(qd, *dev.cache, **args)
    torch.cuda.synchronize()
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    want = ref.attention(q, cache, table, lengths, news, scale, window, sinks)
    _check(out.cpu().numpy(), lse.cpu().numpy(), *want, dim)


def test_attention_bounds_that_are_larger_than_needed_and_a_given_output(gpu_lib):
    """max_new and max_length left to their defaults (all tokens, the whole table), an output of a pitch of its own, no rows beyond the
    sequences' written."""
    import torch
    lengths, news, q_heads, heads, dim, size = [100, 20], [3, 2], 8, 2, 128, 16
    rng, cache, table, k, v, q = _problem(12, lengths, news, q_heads, heads, dim, size, 8, fill="nan")
    cache.append(k, v, table, lengths, news)
    dev = Device(cache, table, lengths, news)
    qd = torch.from_numpy(np.concatenate([q, q[:2]])).cuda()
    out = torch.full((7, q_heads * dim + 8), 7.0, dtype=torch.float16, device="cuda")
    got = gpu_lib.attention(qd, *dev.cache, starts=dev.starts, out=out[:, : q_heads * dim].unflatten(1, (q_heads, dim)))
    torch.cuda.synchronize()
    want = ref.attention(q, cache, table, lengths, news, dim ** -0.5)
    _check(got[:5].cpu().numpy(), None, *want, dim)
    assert (out[5:] == 7).all() and (out[:, q_heads * dim:] == 7).all()


def test_attention_of_large_scores_and_of_keys_whose_scales_differ(gpu_lib):
    """Scores of some hundreds (a softmax of one key), falling and rising along the sequence, and pages whose scales are far apart."""
    import torch
    for lengths, news in (([600], [1]), ([300], [120])):
        heads, dim, size = 2, 128, 16
        rng, cache, table, k, v, q = _problem(13, lengths, news, 4, heads, dim, size, 8)
        for n, slope in ((0, 60.0), (1, -60.0)):
            place = np.arange(lengths[0])
            x = rng.standard_normal((lengths[0], heads, dim)) * np.exp(slope * (place / lengths[0] - (1 if slope > 0 else 0)) / 6)[:, None, None]
            y = rng.standard_normal(x.shape) * np.exp2(rng.integers(-12, 12, (lengths[0] + size - 1) // size)).repeat(size)[: lengths[0], None, None]
            cache.append((x * 8).astype(np.float16), y.astype(np.float16), table, lengths, lengths)
            dev = Device(cache, table, lengths, news)
            out, lse = gpu_lib.attention(torch.from_numpy(q).cuda(), *dev.cache, starts=dev.starts, max_new=news[0], return_lse=True)
            torch.cuda.synchronize()
            want = ref.attention(q, cache, table, lengths, news, dim ** -0.5)
            _check(out.cpu().numpy(), lse.cpu().numpy(), *want, dim)


def test_step_in_a_graph(gpu_lib):
    """Appending and attending captured once and replayed as the sequences grow; every replay against the eager calls."""
    import torch
    lengths, news, q_heads, heads, dim, size = [61, 14, 200], [1, 1, 1], 8, 2, 128, 16
    rng, cache, table, k, v, q = _problem(14, [n + 8 for n in lengths], news, q_heads, heads, dim, size, 8)
    cos, sin = (torch.from_numpy(a).cuda() for a in _tables(rng, 256, 64))
    both = [Device(cache, table, lengths, news, uniform=True) for _ in range(2)]
    x = [torch.from_numpy(a).cuda() for a in (k, v, q)]

    def step(dev):
        rotated = gpu_lib.kv_append(x[0], x[1], *dev.cache, q=x[2], cos=cos, sin=sin, max_new=1)
        return rotated, gpu_lib.attention(rotated, *dev.cache, max_new=1)
    for dev in both:
        step(dev)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(both[0])
    for i in range(5):
        for dev in both:
            dev.lengths.add_(1)
        for a in x:
            a.copy_(torch.from_numpy(rng.standard_normal(tuple(a.shape)).astype(np.float16)))
        graph.replay()
        eager = step(both[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, eager)), i
        assert torch.equal(both[0].k.view(torch.uint8), both[1].k.view(torch.uint8))


def test_attention_on_a_stream_of_its_own(gpu_lib):
    import torch
    lengths, news = [900, 250], [1, 1]
    rng, cache, table, k, v, q = _problem(15, lengths, news, 8, 2, 128, 16, 8)
    dev, qd = Device(cache, table, lengths, news, uniform=True), torch.from_numpy(q).cuda()
    want = gpu_lib.attention(qd, *dev.cache)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = gpu_lib.attention(qd, *dev.cache)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("lengths,news,q_heads,heads,dim,size,bits,window,sinks", [
    ([200, 70], [4, 4], 8, 2, 128, 16, 8, 0, 0),
    ([200, 70], [4, 4], 8, 2, 128, 16, 16, 0, 0),
    ([150, 90], [7, 16], 2, 1, 64, 32, 16, 40, 3),
    ([150, 90], [7, 16], 8, 2, 64, 64, 8, 40, 3),
    ([300, 130], [130, 129], 4, 2, 128, 16, 8, 0, 0),
    ([300, 130], [130, 129], 2, 2, 128, 64, 16, 70, 2),
    ([300, 130], [130, 129], 2, 2, 64, 16, 16, 0, 0),
    ([300], [300], 2, 1, 64, 128, 8, 90, 1),
    ([90], [40], 2, 1, 80, 16, 16, 33, 2),
])
def test_keys_and_values_that_are_not_finite_reach_the_tokens_that_see_them_alone(gpu_lib, lengths, news, q_heads, heads, dim, size, bits, window, sinks):
    """One token in the middle of the new ones of each sequence has a value that is NaN (in 16 bits also infinities, of one sign and of both), another a key:
    tokens that do not see them get what they get without, bit for bit, the others what the sums give."""
    import torch
    rng, cache, table, k, v, q = _problem(16, lengths, news, q_heads, heads, dim, size, bits)
    args = dict(max_new=max(news), window=window, sinks=sinks)

    def run(k, v):
        import copy
        mine = copy.deepcopy(cache)
        with np.errstate(invalid="ignore", over="ignore"):
            mine.append(k, v, table, lengths, news)
        dev = Device(mine, table, lengths, news)
        out, lse = gpu_lib.attention(torch.from_numpy(q).cuda(), *dev.cache, starts=dev.starts, return_lse=True, **args)
        torch.cuda.synchronize()
        return out.cpu().numpy(), lse.cpu().numpy()
    want, want_lse = run(k, v)
    rows = [0] + list(np.cumsum(news))
    for what, kinds in (("value", [np.nan] if bits == 8 else [np.nan, np.inf, -np.inf, None]), ("key", [np.nan])):
        for kind in kinds:
            k2, v2, hit = k.copy(), v.copy(), np.zeros((len(q), dim), bool)
            for b, (length, new) in enumerate(zip(lengths, news)):
                t = new // 2
                places = (t, t + 1) if kind is None else (t,)
                for place in places:
                    if place >= new:
                        continue
                    sign = kind if kind is not None else (np.inf if place == t else -np.inf)
                    (v2 if what == "value" else k2)[rows[b] + place, 0, dim // 2 + 1] = sign
                    for u in range(new):
                        at, j = length - new + u, length - new + place
                        if j <= at and (not window or j > at - window or j < sinks):
                            hit[rows[b] + u, dim // 2 + 1 if what == "value" else slice(None)] = True
            got, lse = run(k2, v2)
            group = q_heads // heads
            hit = np.repeat(hit[:, None, :], q_heads, 1)
            hit[:, group:] = False                                  # other key heads are not touched
            # (in 8 bits a page's scale is that of its finite elements, of which one is gone: the others' codes may differ where it was the largest)
            same = got.view(np.uint16)[~hit] == want.view(np.uint16)[~hit]
            assert same.all(), (what, kind, (~same).sum())
            assert not np.isfinite(got[hit]).any(), (what, kind)
            if kind is not None and np.isinf(kind):
                assert (got[hit] == kind).all()
