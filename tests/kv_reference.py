"""Rotation, paged cache and attention written out in numpy, token by token (test infrastructure)."""
import numpy as np
import torch

E4M3_MAX = 448.0


def e4m3(x):
    """Values of binary32 numbers rounded to e4m3 (ties to even), as codes; what is not finite becomes NaN."""
    x = np.where(np.abs(x) <= E4M3_MAX, x, np.nan).astype(np.float32)
    return torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def values(codes):
    return torch.from_numpy(np.ascontiguousarray(codes)).view(torch.float8_e4m3fn).float().numpy()


def power_for(x):
    """The smallest power of two S, 2^-64 at least, with |x| <= 448 S for the finite x."""
    x = np.abs(x[np.isfinite(x)])
    amax = np.float64(x.max()) if x.size else 0.0
    s = 2.0 ** -64
    while s * E4M3_MAX < amax:
        s *= 2.0
    return np.float32(s)


def rotate(x, cos, sin, interleaved):
    """x: [heads][dim] fp16 of one token, cos, sin: one row; every operation rounded to binary32."""
    x, half = x.astype(np.float32), cos.shape[0]
    y = x.copy()
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    with np.errstate(all="ignore"):
        y[:, a] = x[:, a] * cos - x[:, b] * sin
        y[:, b] = x[:, b] * cos + x[:, a] * sin
    return y


class Cache:
    """Pages in host memory, as the descriptor lays them out."""

    def __init__(self, rng, pages, heads, size, dim, bits, fill="stale"):
        self.size, self.bits, self.heads, self.dim = size, bits, heads, dim
        shape_k, shape_v = (pages, heads, size, dim), (pages, heads, dim, size)
        if bits == 8:
            make = {"stale": lambda s: rng.integers(0, 0x7f, s, dtype=np.uint8), "nan": lambda s: np.full(s, 0x7f, np.uint8)}[fill]
            self.k_scales, self.v_scales = (np.exp2(rng.integers(-9, -3, (pages, heads))).astype(np.float32) for _ in "kv")
        else:
            make = {"stale": lambda s: rng.standard_normal(s).astype(np.float16), "nan": lambda s: np.full(s, np.nan, np.float16)}[fill]
            self.k_scales = self.v_scales = None
        self.k, self.v = make(shape_k), make(shape_v)

    def append(self, k, v, table, lengths, news, cos=None, sin=None, position=None, interleaved=False):
        row = 0
        for pages, length, new in zip(table, lengths, news):
            turned = []
            for t in range(new):
                place = length - new + t
                at = place if position is None else position[row + t]
                at = 0 if cos is None else min(max(at, 0), len(cos) - 1)
                turned.append(k[row + t].astype(np.float32) if cos is None else rotate(k[row + t], cos[at], sin[at], interleaved))
            places = [length - new + t for t in range(new)]
            for block in sorted({p // self.size for p in places if p >= 0}):
                page = pages[block]
                if not 0 <= page < len(self.k):
                    continue
                here = [(t, p % self.size) for t, p in enumerate(places) if p >= 0 and p // self.size == block]
                begin = here[0][1]
                for h in range(self.heads):
                    for matrix, scales, rows in ((self.k[page, h], self.k_scales, turned), (self.v[page, h].T, self.v_scales, None)):
                        fresh = np.stack([rows[t][h] if rows is not None else v[row + t, h].astype(np.float32) for t, _ in here])
                        if self.bits == 16:
                            with np.errstate(over="ignore"):
                                matrix[begin: begin + len(here)] = fresh.astype(np.float16)
                            continue
                        s = power_for(fresh)
                        if begin:
                            s = max(s, scales[page, h])
                            matrix[:begin] = e4m3(values(matrix[:begin]) * (scales[page, h] / s))
                        scales[page, h] = s
                        with np.errstate(invalid="ignore"):
                            matrix[begin: begin + len(here)] = e4m3(fresh / s)
            row += new

    def read(self, page, offset, h):
        if self.bits == 16:
            return self.k[page, h, offset].astype(np.float64), self.v[page, h, :, offset].astype(np.float64)
        return values(self.k[page, h, offset]).astype(np.float64) * self.k_scales[page, h], values(self.v[page, h, :, offset]).astype(np.float64) * self.v_scales[page, h]


def attention(q, cache, table, lengths, news, scale, window=0, sinks=0):
    """(out, lse, weight of the largest error): out[t][h] in 64 bits; for every element sum_j p_j |V_j| and sum_j |V_j| / sum exp(score - largest),
    which a bound of the rounding errors of p is made of; and the largest of sum |q_i K_i|, of the scores'."""
    tokens, q_heads, dim = q.shape
    group = q_heads // cache.heads
    out, weight, floor = (np.zeros((tokens, q_heads, dim)) for _ in range(3))
    lse = np.full((tokens, q_heads), -np.inf)
    terms = np.zeros((tokens, q_heads, 1))
    row = 0
    for pages, length, new in zip(table, lengths, news):
        low = max(0, length - new - window + 1) if window else 0
        places = [j for j in range(length) if (j >= low or j < sinks) and 0 <= pages[j // cache.size] < len(cache.k)]
        for h in range(cache.heads):
            if places:
                K, V = (np.stack(m) for m in zip(*[cache.read(pages[j // cache.size], j % cache.size, h) for j in places]))
            for t in range(new):
                at = length - new + t
                sees = [i for i, j in enumerate(places) if j <= at and (not window or j > at - window or j < sinks)]
                if not sees:
                    continue
                for g in range(h * group, (h + 1) * group):
                    x = q[row + t, g].astype(np.float64)
                    s = K[sees] @ x * scale
                    p = np.exp(s - s.max())
                    out[row + t, g] = p @ V[sees] / p.sum()
                    weight[row + t, g] = p @ np.abs(V[sees]) / p.sum()
                    floor[row + t, g] = np.abs(V[sees]).sum(0) / p.sum()
                    lse[row + t, g] = s.max() + np.log(p.sum())
                    terms[row + t, g] = (np.abs(K[sees]) @ np.abs(x)).max() * scale
        row += new
    return out, lse, weight, floor, terms
