"""vq_attention at the ends of its numbers' ranges, against 64 bits.

Bound of the error behind a long tail: that of tests/test_gpu_attention_long.py but for the probabilities' absolute error.  They are binary16 numbers relative to a
base at least 2^7 below the largest so far, so that the absolute error 2^-25 of the small ones is 2^-32 of the largest."""
import numpy as np
import pytest

from test_gpu_attention import Device, _problem
from test_gpu_attention_long import _attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths,news,q_heads,heads,dim,bits,window,sinks", [
    ([700, 33, 1], [1, 1, 1], 4, 2, 128, 8, 0, 0),
    ([9000], [1], 2, 1, 64, 16, 0, 0),                               # in parts
    ([700, 90], [4, 4], 4, 2, 128, 16, 0, 0),
    ([700, 90], [9, 5], 8, 2, 64, 8, 100, 3),
    ([300, 40], [7, 1], 2, 1, 80, 8, 0, 0),
    ([300, 40], [7, 40], 2, 1, 256, 16, 0, 0),
    ([700, 200], [300, 200], 2, 1, 128, 8, 0, 0),                    # prompts
    ([700, 200], [300, 200], 2, 2, 64, 16, 90, 1),
    ([200], [200], 1, 1, 112, 16, 0, 0),
])
@pytest.mark.parametrize("size", [2.0, 2.0 ** 5, 2.0 ** 8, 2.0 ** 14])
def test_scores_of_every_size(gpu_lib, lengths, news, q_heads, heads, dim, bits, window, sinks, size):
    """Queries and keys of up to 50000: scores of up to 10^10, whose rounding steps are larger than what a softmax tells apart.  The largest score of a token is far
    above its next in all but a few rows (left out): what comes out is that key's value."""
    import torch
    rng, cache, table, k, v, q = _problem(33, lengths, news, q_heads, heads, dim, 16, bits, fill="nan")
    keys, values = ((rng.standard_normal((sum(lengths), heads, dim)) * gain).clip(-50000, 50000).astype(np.float16) for gain in (size, 1))
    q = (rng.standard_normal(q.shape) * size).clip(-50000, 50000).astype(np.float16)
    cache.append(keys, values, table, lengths, lengths)
    dev = Device(cache, table, lengths, news)
    out, lse = gpu_lib.attention(torch.from_numpy(q).cuda(), *dev.cache, starts=dev.starts, window=window, sinks=sinks, max_new=max(news), max_length=max(lengths),
                                 return_lse=True)
    torch.cuda.synchronize()
    out, lse = out.cpu().numpy(), lse.cpu().numpy()
    want, want_lse, _, _, terms = _attention(q, cache, table, lengths, news, dim ** -0.5, window, sinks)
    error = (dim + 2) * 2.0 ** -24 * terms                           # of a score
    assert np.isfinite(out).all() and np.isfinite(lse).all()
    assert (np.abs(lse - want_lse) <= error[..., 0] + 2.0 ** -10 + 2.0 ** -22 * np.abs(want_lse)).all()
    # rows of one key: whose largest score is above all others by more than the errors of both and what a softmax tells apart.  The probability and the result are
    # rounded to binary16, and what else there is lies within 2^-18
    alone = _margin(q, cache, table, lengths, news, dim ** -0.5, window, sinks) > 4 * error[..., 0] + 40
    assert size < 2.0 ** 8 or alone.mean() > 0.9
    off = np.abs(out[alone].astype(np.float64) - want[alone]) - ((2.0 ** -10 + 2.0 ** -18) * np.abs(want[alone]) + 2.0 ** -24)
    assert off.max(initial=0) <= 0, off.max()


def _margin(q, cache, table, lengths, news, scale, window, sinks):
    """How far the largest score of every row lies above its next (infinitely where it is the only one)."""
    from test_gpu_attention_long import _whole
    margin = np.zeros(q.shape[:2])
    group, row = q.shape[1] // cache.heads, 0
    for pages, length, new in zip(table, lengths, news):
        at, places = length - new + np.arange(new)[:, None], np.arange(length)
        sees = places <= at
        if window:
            sees &= (places > at - window) | (places < sinks)
        for g in range(q.shape[1]):
            K, _, there = _whole(cache, pages, length, g // group)
            s = np.where(sees & there, q[row: row + new, g].astype(np.float64) @ np.where(there[:, None], K, 0).T * scale, -np.inf)
            top = np.sort(np.concatenate([np.full((new, 1), -np.inf), s], 1), 1)[:, -2:]
            margin[row: row + new, g] = top[:, 1] - top[:, 0]
        row += new
    return margin


@pytest.mark.parametrize("lengths,news,q_heads,heads,dim,bits", [
    ([300, 90], [1, 1], 16, 1, 128, 8), ([300, 90], [5, 9], 4, 2, 64, 16), ([300, 90], [5, 9], 4, 2, 80, 8), ([300, 200], [130, 200], 2, 1, 128, 16), ([300, 200], [130, 200], 2, 2, 64, 8),
])
def test_a_query_of_large_scores_beside_others(gpu_lib, lengths, news, q_heads, heads, dim, bits):
    """The other rows get what they get without it, bit for bit."""
    import torch
    rng, cache, table, k, v, q = _problem(34, lengths, news, q_heads, heads, dim, 16, bits)
    cache.append(k, v, table, lengths, news)
    dev = Device(cache, table, lengths, news)
    results = []
    for gain in (1, 10000):
        q2 = q.copy()
        q2[::7, 0] *= np.float16(gain)
        results.append(gpu_lib.attention(torch.from_numpy(q2).cuda(), *dev.cache, starts=dev.starts, max_new=max(news), max_length=max(lengths), return_lse=True, scale=500.0))
    torch.cuda.synchronize()
    others = torch.ones(q.shape[:2], dtype=torch.bool, device="cuda")
    others[::7, 0] = False
    assert (results[1][1][::7, 0].abs() > 4194304).any() and all(torch.isfinite(x).all() for x in results[1])
    assert torch.equal(results[0][0][others], results[1][0][others]) and torch.equal(results[0][1][others], results[1][1][others])


@pytest.mark.parametrize("lengths,news,q_heads,heads,dim,bits", [
    ([700, 90], [1, 1], 16, 1, 128, 8), ([700, 90], [1, 1], 8, 1, 64, 16), ([700, 90], [5, 9], 4, 2, 64, 16), ([700, 90], [5, 9], 4, 2, 80, 8),
    ([700, 200], [130, 200], 2, 1, 128, 16), ([700, 200], [130, 200], 2, 2, 64, 8),
])
def test_rows_do_not_depend_on_one_another(gpu_lib, lengths, news, q_heads, heads, dim, bits):
    """Every second query of another size: the others get the same bits, though their tiles' maxima grow at other keys."""
    import torch
    rng, cache, table, k, v, q = _problem(35, lengths, news, q_heads, heads, dim, 16, bits)
    cache.append(k, v, table, lengths, news)
    dev = Device(cache, table, lengths, news)
    results = []
    for gain in (1, 12):
        q2 = q.copy()
        q2[:, ::2] *= np.float16(gain)
        results.append(gpu_lib.attention(torch.from_numpy(q2).cuda(), *dev.cache, starts=dev.starts, max_new=max(news), max_length=max(lengths), return_lse=True))
    torch.cuda.synchronize()
    assert torch.equal(results[0][0][:, 1::2], results[1][0][:, 1::2]) and torch.equal(results[0][1][:, 1::2], results[1][1][:, 1::2])


def _check(got, lse, want, want_lse, weight, floor, terms, dim, keys, values=0.0):
    sums = (keys / 16 + 64) * 2.0 ** -24
    scores = 2 * (dim + 2) * 2.0 ** -24 * terms
    bound = (2.0 ** -10 + 2.0 ** -18 + values + 2 * sums + scores) * weight + 2.0 ** -32 * floor + 2.0 ** -24
    off = np.abs(got.astype(np.float64) - want) - bound
    assert np.isfinite(got).all() and off.max() <= 0, (np.unravel_index(off.argmax(), off.shape), off.max())
    near = np.abs(lse - want_lse)
    assert (near <= scores[..., 0] + 2.0 ** -18 + sums + 2.0 ** -22 * np.abs(want_lse)).all(), near.max()


TAILS = [
    # lengths, news, q heads, heads, dim, bits, window, sinks
    ([3000, 70], [1, 1], 2, 2, 128, 8, 0, 0),
    ([3000, 70], [1, 1], 2, 2, 64, 16, 0, 0),
    ([9000], [1], 1, 1, 128, 8, 0, 0),                               # in parts
    ([5000, 900], [4, 4], 4, 2, 128, 16, 0, 0),                      # drafted tokens
    ([2000], [9], 4, 2, 64, 8, 0, 0),
    ([2500, 600], [1, 3], 2, 1, 80, 8, 0, 0),                        # padded heads
    ([2500], [1], 2, 1, 256, 16, 0, 0),
    ([3000], [140], 1, 1, 128, 8, 0, 0),                             # chunks of prompts
    ([2600, 700], [90, 33], 4, 2, 64, 16, 0, 0),
    ([1500], [70], 1, 1, 96, 16, 0, 0),
    ([4000, 500], [1, 1], 4, 2, 128, 8, 1500, 1),                    # the dominant key is a first token that stays
    ([4000], [70], 2, 2, 128, 16, 1500, 4),
]


@pytest.mark.parametrize("case", TAILS, ids=str)
@pytest.mark.parametrize("gap", [14.0, 17.0, 19.0])
def test_the_tail_behind_a_key_of_no_value(gpu_lib, case, gap):
    """Each sequence's first key has a score `gap` above all others and a value of zeros: what comes out is the tail alone."""
    import torch
    lengths, news, q_heads, heads, dim, bits, window, sinks = case
    rng, cache, table, k, v, q = _problem(31, lengths, news, q_heads, heads, dim, 16, bits, fill="nan")
    along = rng.standard_normal((heads, dim))
    along /= np.linalg.norm(along, axis=1, keepdims=True)
    tokens = sum(lengths)
    keys = (0.3 * rng.standard_normal((tokens, heads, dim))).astype(np.float16)
    values = (1 + 0.25 * rng.standard_normal((tokens, heads, dim))).astype(np.float16)
    first = np.concatenate([[0], np.cumsum(lengths)])[:-1]
    keys[first] = along * gap * np.sqrt(dim) / 8
    values[first] = 0
    q = (8 * np.repeat(along, q_heads // heads, 0) + 0.01 * rng.standard_normal(q.shape)).astype(np.float16)
    cache.append(keys, values, table, lengths, lengths)
    dev = Device(cache, table, lengths, news)
    out, lse = gpu_lib.attention(torch.from_numpy(q).cuda(), *dev.cache, starts=dev.starts, window=window, sinks=sinks, max_new=max(news), max_length=max(lengths),
                                 return_lse=True)
    torch.cuda.synchronize()
    _check(out.cpu().numpy(), lse.cpu().numpy(), *_attention(q, cache, table, lengths, news, dim ** -0.5, window, sinks), dim, max(lengths))


LARGE = [
    # lengths, news, q heads, heads, dim, page, window, sinks
    ([200, 70], [4, 4], 8, 2, 128, 16, 0, 0),
    ([150, 90], [7, 16], 8, 2, 64, 64, 40, 3),
    ([150, 90], [20, 16], 2, 1, 64, 16, 0, 0),
    ([300, 130], [130, 129], 4, 2, 128, 16, 0, 0),
    ([300, 130], [130, 129], 2, 2, 64, 128, 70, 2),
    ([300], [300], 2, 2, 128, 64, 0, 0),
    ([90, 170], [40, 3], 2, 1, 80, 16, 33, 2),
    ([90], [90], 2, 2, 48, 32, 0, 0),
    ([200, 90], [9, 5], 2, 2, 192, 16, 0, 0),
    ([200, 90], [9, 5], 2, 2, 256, 32, 50, 1),
    ([3000, 500], [4, 4], 2, 2, 128, 16, 0, 0),                      # in parts
    ([400, 33], [1, 1], 4, 2, 128, 16, 0, 0),                        # single tokens
    ([400, 33], [1, 1], 4, 2, 112, 16, 0, 0),
]


@pytest.mark.parametrize("case", LARGE, ids=str)
@pytest.mark.parametrize("switches", ["", "attention=d", "attention=p"])
@pytest.mark.parametrize("top", [2.0 ** 8, 2.0 ** 12])
def test_codes_that_stand_for_more_than_binary16_holds(gpu_lib, monkeypatch, case, switches, top):
    """65504 and -65504 appended in 8 bits are the codes of 256 times 2^8.  In the pages of a token in the middle of the new ones of each sequence scales are that, or larger
    yet: tokens that do not see it get, bit for bit, what they get where it stands for half of that, the others what the sums in 64 bits are.  Values beyond count as
    65536 or as the largest number of binary16, 2^-11 less."""
    import torch
    monkeypatch.setenv("VQ_SWITCHES", switches)
    lengths, news, q_heads, heads, dim, size, window, sinks = case
    rng, cache, table, k, v, q = _problem(32, lengths, news, q_heads, heads, dim, size, 8)
    cache.append(k, v, table, lengths, news)
    q = (q * np.float16(2.0 ** -6)).astype(np.float16)              # (scores of keys that large stay small)
    hit = np.zeros(len(q), bool)
    at = []
    row = 0
    for b, (length, new) in enumerate(zip(lengths, news)):
        place = length - new + new // 2
        page = table[b, place // size]
        cache.k_scales[page] = cache.v_scales[page] = top
        cache.k[page], cache.v[page] = cache.k[page] & 0x9f, cache.v[page] & 0x9f          # (the page's other tokens: below 2^-3, times that)
        at.append((page, place % size))
        for u in range(new):
            here = length - new + u
            hit[row + u] = place <= here and (not window or place > here - window or place < sinks)
        row += new

    def run(code, key):
        for page, offset in at:
            cache.v[page, :, ::2, offset], cache.v[page, :, 1::2, offset] = code, code | 0x80
            cache.k[page, :, offset, 1] = key
        dev = Device(cache, table, lengths, news)
        out, lse = gpu_lib.attention(torch.from_numpy(q).cuda(), *dev.cache, starts=dev.starts, window=window, sinks=sinks, max_new=max(news), max_length=max(lengths),
                                     return_lse=True)
        torch.cuda.synchronize()
        return out.cpu().numpy(), lse.cpu().numpy()
    half, half_lse = run(0x70, 0x70)
    for code, key in ((0x78, 0x70), (0x70, 0x7b), (0x78, 0xfb)):     # 256; 352, which a rotated key reaches, and -352
        got, lse = run(code, key)
        assert np.array_equal(got[~hit].view(np.uint16), half[~hit].view(np.uint16)) and np.array_equal(lse[~hit], half_lse[~hit])
        if top > 256:
            for page, offset in at:
                cache.v[page, :, ::2, offset], cache.v[page, :, 1::2, offset] = 0x58, 0xd8          # 16 times 2^12
        want = _attention(q, cache, table, lengths, news, dim ** -0.5, window, sinks)
        fits = np.abs(want[0]) < 65000                               # (a token that sees little else: more than the result's type holds)
        assert np.array_equal(np.sign(got[~fits]), np.sign(want[0][~fits]))
        _check(np.where(fits, got, 0), lse, np.where(fits, want[0], 0), *want[1:], dim, max(lengths), values=2.0 ** -11)
