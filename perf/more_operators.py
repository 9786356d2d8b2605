"""From token numbers to token numbers: what a serving step does around its decoder layers, as cases whose time can be measured.

A step of a model that is served from a paged cache
  * looks its tokens up in the embedding table (embed),
  * lets the new tokens of many sequences attend to a cache whose sequences begin with the same tokens, a system prompt or a document
    that many questions are asked about: its pages are in all of their tables, and its keys and values are read once for all of
    them (attention_shared),
  * draws the next token of each sequence from its logits (sample): by temperature, the top_k largest, the smallest set that holds
    top_p of what is left, what has at least min_p of the largest one's probability, and a given random number.
The cache is held as the package's kv_append leaves it: 8 bits (e4m3) with one power-of-two scale for each page and head, keys and
values apart, or 16 bits; keys [page][head][token][element], values [page][head][element][token].

run() computes these in plain torch operations (own = False), or calls the package (own = True).
"""
import math

import numpy as np
import torch

own = False

E4M3_MAX = 448.0


# ---- cases ------------------------------------------------------------------------------------------------------------
def _attend(prefixes, members, own_length, new, q_heads, kv_heads, head_dim, page, bits, alone=0, ragged=False):
    """prefixes: how many; the first is `prefix` tokens long, each further one shorter; members: sequences of each; alone: sequences
    without a prefix; own_length: tokens of the longest sequence behind its prefix, the new ones included."""
    count, prefix = prefixes
    return dict(op="attention", count=count, prefix=prefix, members=members, alone=alone, own=own_length, new=new, q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, page=page, bits=bits, ragged=ragged)


def _sample(rows, vocabulary, filters, temperature, masked=0.0, idle=0):
    """filters: "none", "k", "p", "min", "all", or "mixed" (each row its own, some without randomness); masked: share of the logits
    that a grammar has set to -inf; idle: rows whose logits all are."""
    return dict(op="sample", rows=rows, vocabulary=vocabulary, filters=filters, temperature=temperature, masked=masked, idle=idle)


def _embed(rows, width, vocabulary, stream, scale=1.0):
    return dict(op="embed", rows=rows, width=width, vocabulary=vocabulary, stream=stream, scale=scale)


def listed():
    """7B-shaped layers have 32 heads of 128 elements for queries and for keys, 70B-shaped ones 64 and 8."""
    return [
        # Four users of a 7B-shaped layer behind a short system prompt, a decoding step: launches are most of it.
        dict(name="four behind 512", **_attend((1, 512), 4, 61, 1, 32, 32, 128, 16, 8)),
        # Sixteen users of a 70B-shaped layer behind a system prompt, one token each.
        dict(name="sixteen behind 2048", **_attend((1, 2048), 16, 509, 1, 64, 8, 128, 16, 8)),
        # 64 users of a 70B-shaped layer behind a long system prompt with examples.
        dict(name="64 behind 8192", **_attend((1, 8192), 64, 1021, 1, 64, 8, 128, 32, 8)),
        # Eight answers to one long document, drawn side by side, on a 70B-shaped layer.
        dict(name="eight behind 131072", **_attend((1, 131072), 8, 201, 1, 64, 8, 128, 64, 8)),
        # Three applications with a prompt each, 24 users and two others without, whose drafted tokens are checked; smaller heads, 16 bits.
        dict(name="drafts behind three", **_attend((3, 4096), 8, 333, 4, 32, 8, 64, 16, 16, alone=2, ragged=True)),
        # 128 users of a 70B-shaped layer behind a book: the largest call.
        dict(name="128 behind 32768", **_attend((1, 32768), 128, 257, 1, 64, 8, 128, 64, 8)),
        # One user's next token: the smallest call.
        dict(name="sample one", **_sample(1, 32000, "all", 0.7)),
        # Four users' drafted tokens, an odd vocabulary of which a grammar allows a part, each row with its own settings, one slot idle.
        dict(name="sample 20 mixed", **_sample(20, 50261, "mixed", 1.0, masked=0.4, idle=1)),
        # 64 users, the smallest set that holds nine tenths.
        dict(name="sample 64 top-p", **_sample(64, 128000, "p", 0.8)),
        # 256 users at a high temperature, nothing left out.
        dict(name="sample 256 whole", **_sample(256, 131072, "none", 1.3)),
        # A decoding step of 16 users.
        dict(name="embed 16", **_embed(16, 4096, 32000, 16)),
        # The prompts of several users at once, into a residual stream of 32 bits, scaled by the root of the width.
        dict(name="embed 8192", **_embed(8192, 8192, 32000, 32, math.sqrt(8192.0))),
    ]


def _size(rng, low, high):
    """A size between low and high, even over its logarithm."""
    return low if high <= low else min(high, max(low, int(math.exp(rng.uniform(math.log(low), math.log(high))) + 0.5)))


HEADS = ((32, 32), (64, 8), (64, 8), (32, 8), (40, 40), (28, 4), (8, 1), (16, 2))
#: What the largest listed cases cost: a drawn one stays below.
MOST_BYTES, MOST_PAIRS, MOST_LOGITS, MOST_ELEMENTS = 300e6, 128 * 64 * 32768, 256 * 131072, 8192 * 8192


def draw(rng):
    op = rng.choice(("attention", "attention", "attention", "sample", "sample", "embed"))
    if op == "embed":
        width = rng.choice((64, 512, 1024, 2048, 4096, 5120, 8192, rng.randrange(65, 4096)))
        return _embed(_size(rng, 1, MOST_ELEMENTS // max(width, 4096)), width, _size(rng, 500, 64000), rng.choice((16, 32)), rng.choice((1.0, 0.25, math.sqrt(width))))
    if op == "sample":
        vocabulary = rng.choice((32000, 128000, 131072, _size(rng, 2, 32000), _size(rng, 1000, 262144), _size(rng, 1000, 262144)))
        rows = _size(rng, 1, min(512, MOST_LOGITS // vocabulary))
        return _sample(rows, vocabulary, rng.choice(("none", "k", "p", "min", "all", "mixed", "mixed")), rng.choice((0.3, 0.7, 1.0, 1.5)),
                       rng.choice((0.0, 0.0, 0.4, 0.98)), rng.choice((0, 0, 1)) if rows > 1 else 0)
    q_heads, kv_heads = rng.choice(HEADS)
    head_dim, page, bits = rng.choice((64, 128, 128, 128, 80)), rng.choice((16, 16, 32, 64, 128)), rng.choice((8, 8, 16))
    token = 2 * kv_heads * head_dim * bits // 8
    count = rng.choice((1, 1, 1, 2, 3, 5))
    members = _size(rng, 2, 128 // count)
    new = rng.choice((1, 1, 1, rng.randrange(2, 9)))
    alone = rng.choice((0, 0, rng.randrange(1, 5)))
    most = min(65536, int(0.7 * MOST_BYTES / (count * token)), MOST_PAIRS // (count * members * q_heads * new))
    prefix = max(page, _size(rng, 64, max(64, most)) // page * page)
    own_length = max(new, _size(rng, max(new, 16), max(new, min(2048, int(0.3 * MOST_BYTES / ((count * members + alone) * token))))))
    return _attend((count, prefix), members, own_length, new, q_heads, kv_heads, head_dim, page, bits, alone, ragged=rng.random() < 0.5)


def _lengths(case):
    """Length of each prefix; for each sequence the number of its prefix (-1: none), what it holds behind it, and how many of that are
    new: the first has the case's numbers, the others spread from a quarter of them up, the new ones where the case is ragged."""
    count, page = case["count"], case["page"]
    prefixes = [max(1, int(case["prefix"] * (1.0 - 0.6 * i / count)) // page) * page for i in range(count)]
    of = [i for i in range(count) for _ in range(case["members"])] + [-1] * case["alone"]
    part = [(i * 0.6180339887) % 1.0 for i in range(len(of))]
    news = [case["new"] if not case["ragged"] or i == 0 else max(1, int(case["new"] * (1.0 - 0.75 * part[i]))) for i in range(len(of))]
    held = [case["own"] if i == 0 else max(news[i], int(case["own"] * (1.0 - 0.75 * part[i]))) for i in range(len(of))]
    return prefixes, of, held, news


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _power(amax):
    """The smallest power of two times 448 that is no smaller (32 bits; 2^-64 at least)."""
    mantissa, exponent = torch.frexp(amax / E4M3_MAX)
    power = exponent - (mantissa == 0.5).int()
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), power.clamp(min=-64)), torch.full_like(amax, 2.0 ** -64))


def _cache(pool, heads, rows, columns, bits, gain, generator):
    """Pages of normal values whose channels are of different sizes, as keys' are, and their scales."""
    x = torch.randn((pool, heads, rows, columns), device="cuda", generator=generator)
    x *= gain
    if bits == 16:
        return x.half(), None
    scale = _power(x.abs().amax((2, 3)))
    return (x / scale[:, :, None, None]).to(torch.float8_e4m3fn), scale


def _prepare_attention(case, seed, g):
    prefixes, of, held, news = _lengths(case)
    page, heads, d = case["page"], case["kv_heads"], case["head_dim"]
    # pages scattered over the pool, as they come and go in a server; a prefix's are in the tables of all of its sequences
    shared, mine = [n // page for n in prefixes], [-(-n // page) for n in held]
    pool = sum(shared) + sum(mine) + 3
    free = iter(np.random.default_rng(seed).permutation(pool).tolist())
    of_prefix = [[next(free) for _ in range(n)] for n in shared]
    rows = [(of_prefix[p] if p >= 0 else []) + [next(free) for _ in range(n)] for p, n in zip(of, mine)]

    def table(lists):
        t = np.full((len(lists), max(len(x) for x in lists)), -1, np.int32)
        for i, x in enumerate(lists):
            t[i, : len(x)] = x
        return torch.from_numpy(t).cuda()
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    lengths = [n + (prefixes[p] if p >= 0 else 0) for p, n in zip(of, held)]
    members = [i * case["members"] for i in range(case["count"] + 1)]
    state = {"op": "attention", "page_table": table(rows), "lengths": ints(lengths), "prefix_table": table(of_prefix), "prefix_lengths": ints(prefixes),
             "members": None if members == [0, len(of)] else ints(members), "starts": ints([0] + list(np.cumsum(news))) if case["ragged"] else None,
             # what a server knows without asking the GPU
             "known": {"lengths": lengths, "prefixes": prefixes, "members": members, "starts": [0] + np.cumsum(news).tolist()},
             "max_new": max(news), "max_length": max(lengths), "max_prefix": max(prefixes), "max_members": case["members"], "max_own": max(held)}
    k_gain = torch.exp(0.5 * torch.randn((1, heads, 1, d), device="cuda", generator=g))
    state["k_pages"], state["k_scales"] = _cache(pool, heads, page, d, case["bits"], k_gain, g)
    state["v_pages"], state["v_scales"] = _cache(pool, heads, d, page, case["bits"], 1.0, g)
    state["q"] = torch.randn((sum(news), case["q_heads"], d), device="cuda", generator=g).half()
    return state


def _prepare_sample(case, g):
    rows, n = case["rows"], case["vocabulary"]
    rand = lambda *s: torch.rand(s, device="cuda", generator=g)  # noqa: E731
    # most of a vocabulary far below a few dozen candidates, whose lead falls off as their rank grows
    logits = 2.2 * torch.randn((rows, n), device="cuda", generator=g) - 2.0
    few = min(n, 60)
    at = torch.randint(n, (rows, few), device="cuda", generator=g)
    lead = 14.0 - 1.9 * torch.log1p(torch.arange(few, device="cuda", dtype=torch.float32)) + rand(rows, few)
    logits.scatter_reduce_(1, at, lead, "amax")                           # (the same token twice: the larger one)
    if case["masked"]:
        logits.masked_fill_(rand(rows, n) < case["masked"], -math.inf)
    if case["idle"]:
        logits[rows // 2: rows // 2 + case["idle"]] = -math.inf
    state = {"op": "sample", "logits": logits.half(), "uniform": rand(rows)}
    filters, per_row = case["filters"], torch.arange(rows, device="cuda")
    full = lambda x: torch.full((rows,), x, device="cuda")  # noqa: E731
    state["temperature"], state["top_k"], state["top_p"], state["min_p"] = full(case["temperature"]), None, None, None
    if filters in ("k", "all"):
        state["top_k"] = torch.full((rows,), 50, dtype=torch.int32, device="cuda")
    if filters in ("p", "all"):
        state["top_p"] = full(0.9)
    if filters in ("min", "all"):
        state["min_p"] = full(0.02)
    if filters == "mixed":
        state["temperature"] = torch.where(per_row % 5 == 2, 0.0, case["temperature"] * (0.5 + rand(rows)))
        state["top_k"] = torch.where(per_row % 3 == 0, 0, torch.randint(1, 2000, (rows,), device="cuda", generator=g)).int()
        state["top_p"] = torch.where(per_row % 4 == 1, torch.ones((), device="cuda"), 0.3 + 0.69 * rand(rows))
        state["min_p"] = torch.where(per_row % 2 == 0, torch.zeros((), device="cuda"), 0.1 * rand(rows))
    return state


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "attention":
        return _prepare_attention(case, seed, g)
    if case["op"] == "sample":
        return _prepare_sample(case, g)
    table = torch.randn((case["vocabulary"], case["width"]), device="cuda", generator=g, dtype=torch.float16)
    # some tokens are far more frequent than others
    ids = (case["vocabulary"] * torch.rand(case["rows"], device="cuda", generator=g) ** 3).int().clamp(max=case["vocabulary"] - 1)
    return {"op": "embed", "table": table, "ids": ids, "scale": case["scale"], "dtype": torch.float16 if case["stream"] == 16 else torch.float32}


# ---- one pass ---------------------------------------------------------------------------------------------------------
def _held(s, pages):
    """Keys and values of a list of pages as [heads][tokens][element], 32 bits."""
    def of(pool, scales):
        if scales is None:
            return pool[pages].float()
        return pool.view(torch.uint8)[pages].view(torch.float8_e4m3fn).float() * scales[pages][..., None, None]
    k, v = of(s["k_pages"], s["k_scales"]), of(s["v_pages"], s["v_scales"])
    return k.transpose(0, 1).flatten(1, 2), v.permute(1, 0, 3, 2).flatten(1, 2)


def _plain_attention(s):
    """The rows of all of a prefix's sequences against its keys in one product for each head, then each sequence's own ones."""
    q = s["q"].float()
    heads, size, d = s["k_pages"].shape[1:]
    group, table = q.shape[1] // heads, s["page_table"].long()
    lengths, prefixes, members, starts = (s["known"][name] for name in ("lengths", "prefixes", "members", "starts"))
    n = len(lengths)
    out = torch.empty_like(q)

    def rows_of(a, b):
        return q[a:b].reshape(b - a, heads, group, d).transpose(0, 1).reshape(heads, (b - a) * group, d)

    def one(b, first, before, values):
        """Sequence b, whose keys from place `first` on are its own; before: scores against those in front of them."""
        new, length = starts[b + 1] - starts[b], lengths[b]
        K, V = _held(s, table[b, first // size: -(-length // size)])
        place = (length - new + torch.arange(new, device="cuda")).repeat_interleave(group)
        score = rows_of(starts[b], starts[b + 1]) @ K.transpose(1, 2) * d ** -0.5
        score = score.masked_fill(first + torch.arange(K.shape[1], device="cuda") > place[:, None], -math.inf)
        if before is not None:
            score = torch.cat((before, score), 2)
        p = (score - score.amax(2, keepdim=True)).exp()
        total = p.sum(2, keepdim=True)
        o = p[:, :, first:] @ V
        if before is not None:
            o = o + p[:, :, :first] @ values
        out[starts[b]: starts[b + 1]] = (o / total).view(heads, new, group, d).transpose(0, 1).reshape(new, heads * group, d)
    for i, prefix in enumerate(prefixes):
        a, b = members[i], members[i + 1]
        K, V = _held(s, s["prefix_table"][i, : -(-prefix // size)].long())
        K, V = K[:, :prefix], V[:, :prefix]
        score = rows_of(starts[a], starts[b]) @ K.transpose(1, 2) * d ** -0.5
        for m in range(a, b):
            at = (starts[m] - starts[a]) * group, (starts[m + 1] - starts[a]) * group
            one(m, prefix, score[:, at[0]: at[1]], V)
    for b in range(members[-1], n):
        one(b, 0, None, None)
    return out.half()


def _plain_sample(s):
    """In 64 bits: which token a random number falls on is decided by sums over a whole vocabulary."""
    x = s["logits"].double()
    rows, n = x.shape
    order = x.sort(dim=1, descending=True, stable=True)                     # (stable: of equal ones the lowest token first)
    top = order.values[:, :1]
    hot = s["temperature"] > 0
    temperature = torch.where(hot, s["temperature"], torch.ones((), device="cuda")).double()[:, None]
    w = torch.where(order.values > -math.inf, ((order.values - top) / temperature).exp(), torch.zeros((), device="cuda", dtype=torch.float64))
    rank = torch.arange(n, device="cuda")
    k = s["top_k"] if s["top_k"] is not None else torch.zeros(rows, dtype=torch.int32, device="cuda")
    k = torch.where(hot, torch.where(k > 0, k, n), 1)[:, None]
    w = torch.where(rank < k, w, torch.zeros((), device="cuda", dtype=torch.float64))
    if s["top_p"] is not None:
        sums = w.cumsum(1)
        p = s["top_p"].double()[:, None]
        keep = (sums - w < p * sums[:, -1:]) | (p >= 1)
        keep[:, 0] = True
        w = w * keep
    if s["min_p"] is not None:
        w = w * (w >= s["min_p"].double()[:, None])
    sums = w.cumsum(1)
    total = sums[:, -1:]
    at = (sums <= s["uniform"].double()[:, None] * total).sum(1, keepdim=True).clamp(max=n - 1)
    some = total[:, 0] > 0
    token = torch.where(some, order.indices.gather(1, at)[:, 0], -1).int()
    return token, torch.where(some, (w.gather(1, at) / total)[:, 0], torch.zeros((), device="cuda", dtype=torch.float64)).float()


def run(state):
    s = state
    if own:
        import paper_2409_17066_amd as vq
    if s["op"] == "attention":
        if own:
            return vq.attention_shared(s["q"], s["k_pages"], s["v_pages"], s["page_table"], s["lengths"], s["prefix_table"], s["prefix_lengths"],
                                       s["k_scales"], s["v_scales"], members=s["members"], starts=s["starts"], max_new=s["max_new"],
                                       max_length=s["max_length"], max_prefix=s["max_prefix"], max_members=s["max_members"], max_own=s["max_own"])
        return _plain_attention(s)
    if s["op"] == "sample":
        if own:
            given = {name: s[name] for name in ("top_k", "top_p", "min_p") if s[name] is not None}
            return vq.sample(s["logits"], s["uniform"], temperature=s["temperature"], return_prob=True, **given)
        return _plain_sample(s)
    if own:
        return vq.embed(s["ids"], s["table"], scale=s["scale"], dtype=s["dtype"])
    return (s["table"][s["ids"].long()].float() * s["scale"]).to(s["dtype"])


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------
def _exact_attention(case, s):
    """Sequence by sequence over its own table, nothing shared."""
    prefixes, of, held, news = _lengths(case)
    size, heads, d, group = case["page"], case["kv_heads"], case["head_dim"], case["q_heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for b, (p, own_length, new) in enumerate(zip(of, held, news)):
        length = own_length + (prefixes[p] if p >= 0 else 0)
        at = torch.arange(length, device="cuda")
        pages = s["page_table"][b].long()[at // size]
        for h in range(heads):
            if case["bits"] == 8:
                k = s["k_pages"][:, h].view(torch.uint8)[pages, at % size].view(torch.float8_e4m3fn).double() * s["k_scales"][pages, h].double()[:, None]
                v = s["v_pages"][:, h].view(torch.uint8)[pages, :, at % size].view(torch.float8_e4m3fn).double() * s["v_scales"][pages, h].double()[:, None]
            else:
                k, v = s["k_pages"][:, h][pages, at % size].double(), s["v_pages"][:, h][pages, :, at % size].double()
            q = s["q"][row: row + new, h * group:(h + 1) * group].double().reshape(-1, d)
            here = torch.arange(length - new, length, device="cuda").repeat_interleave(group)[:, None]
            w = torch.softmax(torch.where(at <= here, q @ k.T.contiguous() / math.sqrt(d), -math.inf), -1)
            out[row: row + new, h * group:(h + 1) * group] = (w @ v).view(new, group, d)
        row += new
    return out


def _exact_sample(s):
    host = {name: None if s[name] is None else s[name].cpu().numpy() for name in ("logits", "uniform", "temperature", "top_k", "top_p", "min_p")}
    tokens, probabilities = [], []
    for r, x in enumerate(host["logits"].astype(np.float64)):
        places = np.argsort(-x, kind="stable")[: int(np.isfinite(x).sum())]
        if not len(places):
            tokens.append(-1)
            probabilities.append(0.0)
            continue
        if host["temperature"][r] <= 0:
            tokens.append(int(places[0]))
            probabilities.append(1.0)
            continue
        if host["top_k"] is not None and host["top_k"][r] > 0:
            places = places[: host["top_k"][r]]
        w = np.exp((x[places] - x[places[0]]) / np.float64(host["temperature"][r]))
        if host["top_p"] is not None and host["top_p"][r] < 1:
            sums = np.cumsum(w.astype(np.longdouble))
            w = w[: 1 + np.searchsorted(sums, np.longdouble(host["top_p"][r]) * sums[-1], side="left")]
        if host["min_p"] is not None:
            w = w[w >= np.float64(host["min_p"][r])]
        sums = np.cumsum(w.astype(np.longdouble))
        at = int(np.searchsorted(sums, np.longdouble(host["uniform"][r]) * sums[-1], side="right"))
        tokens.append(int(places[at]))
        probabilities.append(float(w[at] / sums[-1]))
    return torch.tensor(tokens, dtype=torch.int32, device="cuda"), torch.tensor(probabilities, dtype=torch.float64, device="cuda")


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attention":
        return _exact_attention(case, s)
    if case["op"] == "sample":
        return _exact_sample(s)
    out = torch.empty((case["rows"], case["width"]), dtype=torch.float64, device="cuda")
    for r in range(0, case["rows"], 512):
        out[r: r + 512] = torch.index_select(s["table"], 0, s["ids"][r: r + 512]).double().mul(s["scale"])
    return out


# ---- what a pass cannot do without -------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "embed":
        n, distinct = case["rows"] * case["width"], min(case["rows"], case["vocabulary"]) * case["width"]
        return {"bytes": 2 * distinct + n * case["stream"] // 8 + 4 * case["rows"], "flops": n}
    if case["op"] == "sample":
        given = {"none": 1, "k": 2, "p": 2, "min": 2, "all": 4, "mixed": 4}[case["filters"]]
        return {"bytes": 2 * case["rows"] * case["vocabulary"] + 4 * case["rows"] * (3 + given), "flops": 4 * case["rows"] * case["vocabulary"]}
    prefixes, of, held, news = _lengths(case)
    heads, q_heads, d, page = case["kv_heads"], case["q_heads"], case["head_dim"], case["page"]
    seen = sum(prefixes) + sum(held)
    pages = sum(n // page for n in prefixes) + sum(-(-n // page) for n in held)
    pairs = sum(m * (n + (prefixes[p] if p >= 0 else 0)) - m * (m - 1) // 2 for p, n, m in zip(of, held, news))
    return {"bytes": 2 * seen * heads * d * case["bits"] // 8 + 4 * sum(news) * q_heads * d + pages * (4 + (8 * heads if case["bits"] == 8 else 0)),
            "flops": 4 * d * q_heads * pairs}
