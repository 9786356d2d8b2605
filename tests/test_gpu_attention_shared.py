"""vq_attention_shared on the GPU: attention behind shared prefixes against 64 bits over every sequence by itself, to the bound of vq_attention's error (test_gpu_attention.py): joining
partial sums adds a rounding of 2^-24 for each of up to 64 parts, which its allowance of 2^-18 holds."""
import numpy as np
import pytest

import kv_reference as ref
from test_gpu_attention import Device, _check

pytestmark = pytest.mark.gpu


class Problem:
    """prefixes: (tokens in whole pages, tokens that the call names as the prefix, [(own, new), ...]) each; alone: [(own, new), ...].  An `own` that is a text is the
    whole length of a sequence that ends inside of the prefix's pages or is empty."""

    def __init__(self, seed, prefixes, alone, q_heads, heads, dim, size, bits, spread=1.0):
        rng = np.random.default_rng(seed)
        flat = [(g, own, new) for g, (_, _, seqs) in enumerate(prefixes) for own, new in seqs] + [(-1, own, new) for own, new in alone]
        commons = [common for common, _, _ in prefixes]
        assert all(n % size == 0 for n in commons)
        self.lengths = [int(own) if isinstance(own, str) else own + (commons[g] if g >= 0 else 0) for g, own, _ in flat]
        self.news = [new for _, _, new in flat]
        most = max(-(-n // size) for n in self.lengths + [1])
        pool = sum(n // size for n in commons) + sum(-(-own // size) for _, own, _ in flat if not isinstance(own, str)) + 2
        free = iter(rng.permutation(pool))
        self.prefix_table = np.full((max(len(prefixes), 1), max([n // size for n in commons] + [1]) + 1), -1, np.int32)
        self.table = np.full((len(flat), most + 1), -1, np.int32)
        for g, n in enumerate(commons):
            self.prefix_table[g, : n // size] = [next(free) for _ in range(n // size)]
        cache = ref.Cache(rng, pool, heads, size, dim, bits, "nan")
        gain = np.exp(rng.standard_normal((heads, dim)) * 0.5) * spread

        def rows(n):
            return (rng.standard_normal((n, heads, dim)) * gain).clip(-50000, 50000).astype(np.float16), rng.standard_normal((n, heads, dim)).astype(np.float16)
        for g, n in enumerate(commons):
            cache.append(*rows(n), self.prefix_table[g: g + 1], [n], [n])
        for b, (g, own, _) in enumerate(flat):
            shared = commons[g] // size if g >= 0 else 0
            if isinstance(own, str):
                self.table[b, : -(-int(own) // size)] = self.prefix_table[g, : -(-int(own) // size)]
                continue
            self.table[b, :shared] = self.prefix_table[g, :shared]
            self.table[b, shared: shared + -(-own // size)] = [next(free) for _ in range(-(-own // size))]
            cache.append(*rows(own), self.table[b: b + 1], [self.lengths[b]], [own])
        self.cache, self.dim, self.prefix_lengths = cache, dim, [named for _, named, _ in prefixes]
        self.members = np.concatenate([[0], np.cumsum([len(seqs) for _, _, seqs in prefixes])]).astype(np.int32)
        self.most = max(len(seqs) for _, _, seqs in prefixes)
        self.q = rng.standard_normal((sum(self.news), q_heads, dim)).astype(np.float16)
        self.one = len(prefixes) == 1 and not alone

    def up(self):
        import torch
        dev = Device(self.cache, self.table, self.lengths, self.news, uniform=len(set(self.news)) == 1)
        prefix = dict(prefix_table=torch.from_numpy(self.prefix_table).cuda(), prefix_lengths=torch.tensor(self.prefix_lengths, dtype=torch.int32, device="cuda"),
                      members=None if self.one else torch.from_numpy(self.members).cuda())
        return dev, prefix

    def want(self, scale):
        return ref.attention(self.q, self.cache, self.table, self.lengths, self.news, scale)


CASES = [
    # prefixes, alone, q heads, heads, dim, page, bits
    ([(16, 16, [(1, 1), (1, 1)])], [], 1, 1, 128, 16, 8),                                        # the smallest
    ([(64, 64, [(5, 1), (33, 1), (64, 1)])], [], 8, 2, 128, 16, 8),
    ([(512, 512, [(61, 1), (20, 1), (5, 1), (64, 1)])], [], 4, 4, 128, 16, 8),
    ([(320, 317, [(40, 3), (7, 3), (90, 3)])], [], 8, 1, 128, 32, 8),                            # a prefix that ends inside of a page
    ([(128, 65, [(1, 1), (200, 1)])], [], 4, 2, 64, 64, 16),                                     # ... and one key behind a chunk
    ([(256, 256, [(30, 2), (64, 5), (11, 1)]), (96, 90, [(9, 4), (70, 4)])], [(150, 3), (3, 3)], 8, 2, 64, 32, 16),
    ([(256, 256, [(30, 1)] * 20)], [], 28, 4, 128, 128, 8),                                      # seven queries a key, more rows than a tile
    ([(1024, 1024, [(100, 4)] * 10), (64, 64, []), (512, 500, [(50, 2)] * 3)], [], 8, 1, 128, 16, 8),      # a prefix nobody has
    ([(400, 400, [(80, 1), (17, 1)])], [(33, 1)], 4, 1, 80, 16, 8),                              # heads of other sizes
    ([(160, 160, [(20, 2), (40, 2)])], [], 6, 3, 256, 16, 8),
    ([(96, 96, [(20, 1), (40, 1)])], [], 2, 1, 16, 32, 16),
    ([(160, 150, [(20, 2), (40, 2)])], [], 4, 2, 192, 16, 16),
    ([(96, 0, [(20, 1), (40, 1)])], [(5, 1)], 4, 2, 128, 16, 8),                                 # a prefix of no tokens
    ([(192, 192, [(200, 200), (90, 70)])], [], 4, 2, 128, 64, 8),                                # prompts behind it
    ([(192, 192, [(30, 1), ("0", 1), (5, 1)])], [("0", 1)], 8, 2, 128, 16, 8),                   # idle slots
    ([(192, 192, [(30, 4), ("100", 4), ("194", 4), ("2", 4), ("192", 4)])], [], 8, 2, 64, 16, 8),       # sequences whose new tokens are (partly) the prefix's own
    ([(192, 180, [(3, 15), (12, 15)])], [], 4, 2, 128, 16, 16),                                  # new tokens that begin exactly at its end and in front of it
    ([(64, 64, [(2, 1)] * 90)], [(70, 1)] * 3, 2, 2, 64, 16, 8),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c)[:100])
@pytest.mark.parametrize("switches", ["", "shared=1", "shared=1,attention=d,parts=0", "shared=1,attention=d,parts=2", "shared=1,attention=p,parts=0", "shared=1,attention=p,parts=3", "shared=0", "shared=2", "shared=2,attention=d,parts=2", "shared=2,attention=p,parts=1"])
def test_against_every_sequence_by_itself(gpu_lib, monkeypatch, case, switches):
    import torch
    monkeypatch.setenv("VQ_SWITCHES", switches)
    p = Problem(21, *case)
    dev, prefix = p.up()
    scale = 1.3 / np.sqrt(p.dim)
    q = torch.zeros((len(p.q), p.q.shape[1] * p.dim + 3), dtype=torch.float16, device="cuda")[:, 1: 1 + p.q.shape[1] * p.dim].unflatten(1, (p.q.shape[1], p.dim))
    q.copy_(torch.from_numpy(p.q))
    tight = dict(max_new=max(p.news), max_length=max(p.lengths), max_prefix=max(p.prefix_lengths), max_members=p.most, max_own=100)
    for bounds in (tight, dict(max_new=max(p.news))):
        args = dict(k_scales=dev.k_scales, v_scales=dev.v_scales, starts=dev.starts, scale=scale, return_lse=True, **prefix, **bounds)
        out, lse = gpu_lib.attention_shared(q, dev.k, dev.v, dev.table, dev.lengths, **args)
        again, lse2 = gpu_lib.attention_shared(q, dev.k, dev.v, dev.table, dev.lengths, **args)
        torch.cuda.synchronize()
        assert torch.equal(out, again) and torch.equal(lse, lse2)
        _check(out.cpu().numpy(), lse.cpu().numpy(), *p.want(scale), p.dim)


def test_bounds_that_leave_members_and_tokens_out(gpu_lib, monkeypatch):
    """Sequences beyond max_members, prefixes longer than max_prefix, members in no order and out of range: every sequence is still looked at as a whole."""
    import torch
    monkeypatch.setenv("VQ_SWITCHES", "shared=1")
    p = Problem(22, [(256, 256, [(30, 2)] * 5), (128, 128, [(9, 2)] * 3)], [(40, 2)], 8, 2, 128, 16, 8)
    dev, prefix = p.up()
    want = p.want(p.dim ** -0.5)

    def check(**kw):
        out, lse = gpu_lib.attention_shared(torch.from_numpy(p.q).cuda(), dev.k, dev.v, dev.table, dev.lengths, k_scales=dev.k_scales, v_scales=dev.v_scales,
                                            return_lse=True, **dict(prefix, max_new=2, **kw))
        torch.cuda.synchronize()
        _check(out.cpu().numpy(), lse.cpu().numpy(), *want, p.dim)
    check(max_members=1)
    check(max_members=4)
    check(max_prefix=100)
    check(max_prefix=0)
    check(max_own=0)
    prefix["prefix_lengths"] = torch.tensor([256, -7], dtype=torch.int32, device="cuda")
    check()
    prefix["prefix_lengths"] = torch.tensor([10 ** 9, 128], dtype=torch.int32, device="cuda")
    check(max_prefix=256)
    for members in ([0, 0, 0], [2, 4, 4], [0, 5, 5], [-9, 5, 100], [0, 5, 8]):
        prefix["prefix_lengths"] = torch.tensor([256, 128], dtype=torch.int32, device="cuda")
        prefix["members"] = torch.tensor(members, dtype=torch.int32, device="cuda")
        if members[2] == 100:                                      # (the ninth sequence is none of the second prefix's: a prefix that says so would be wrong)
            prefix["prefix_lengths"][1] = 0
        check()


def test_without_room_it_is_attention(gpu_lib, monkeypatch):
    import torch
    monkeypatch.setenv("VQ_SWITCHES", "shared=1")
    p = Problem(23, [(256, 256, [(30, 1)] * 5)], [], 8, 2, 128, 16, 8)
    dev, prefix = p.up()
    q = torch.from_numpy(p.q).cuda()
    cache = (dev.k, dev.v, dev.table, dev.lengths)
    scales = dict(k_scales=dev.k_scales, v_scales=dev.v_scales)
    for room in (0, 256):
        ws = torch.empty(room, dtype=torch.uint8, device="cuda")
        got = gpu_lib.attention_shared(q, *cache, **scales, **prefix, workspace=ws)
        want = gpu_lib.attention(q, *cache, **scales, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_nothing_is_read_where_the_prefixs_table_names_no_page(gpu_lib, monkeypatch):
    """Entries of -1 and beyond the pool are seen by nobody, in the prefix as in a sequence."""
    import torch
    monkeypatch.setenv("VQ_SWITCHES", "shared=1")
    p = Problem(24, [(256, 256, [(30, 1)] * 5)], [], 8, 2, 128, 16, 8)
    p.prefix_table[0, 3], p.prefix_table[0, 15] = -1, 10 ** 6
    p.table[:, 3], p.table[:, 15] = -1, -1
    dev, prefix = p.up()
    out, lse = gpu_lib.attention_shared(torch.from_numpy(p.q).cuda(), dev.k, dev.v, dev.table, dev.lengths, k_scales=dev.k_scales, v_scales=dev.v_scales, return_lse=True, **prefix)
    torch.cuda.synchronize()
    _check(out.cpu().numpy(), lse.cpu().numpy(), *p.want(p.dim ** -0.5), p.dim)


def test_scores_far_apart_in_the_two_halves(gpu_lib, monkeypatch):
    """Keys that outweigh the other half altogether, either way, and scores of some hundreds."""
    import torch
    monkeypatch.setenv("VQ_SWITCHES", "shared=1")
    for spread in (8.0, 40.0):
        p = Problem(25, [(256, 256, [(30, 1), (100, 1), (2, 1)])], [], 8, 2, 128, 16, 16, spread=spread)
        p.cache.k[p.prefix_table[0, :16]] *= np.float16(0.05)
        dev, prefix = p.up()
        out, lse = gpu_lib.attention_shared(torch.from_numpy(p.q).cuda(), dev.k, dev.v, dev.table, dev.lengths, return_lse=True, **prefix)
        torch.cuda.synchronize()
        _check(out.cpu().numpy(), lse.cpu().numpy(), *p.want(p.dim ** -0.5), p.dim)


def test_in_a_graph_as_sequences_and_prefixes_change(gpu_lib, monkeypatch):
    """Captured once; sequences grow, become idle and the prefix gets shorter between replays."""
    import torch
    monkeypatch.setenv("VQ_SWITCHES", "shared=1")
    p = Problem(26, [(256, 256, [(50, 1)] * 6), (64, 64, [(50, 1)] * 2)], [(60, 1)], 8, 2, 128, 16, 8)
    dev, prefix = p.up()
    q = torch.from_numpy(p.q).cuda()
    bounds = dict(max_new=1, max_length=320, max_prefix=256, max_members=6, max_own=64)

    def call():
        return gpu_lib.attention_shared(q, dev.k, dev.v, dev.table, dev.lengths, k_scales=dev.k_scales, v_scales=dev.v_scales, return_lse=True, **prefix, **bounds)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = call()
    for i in range(5):
        dev.lengths.copy_(torch.tensor([max(0, n - 7 * i) if b != i else 0 for b, n in enumerate(p.lengths)], dtype=torch.int32))
        prefix["prefix_lengths"].copy_(torch.tensor([256 - 19 * i, 64 - 16 * i], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        eager = call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])
        want = ref.attention(p.q, p.cache, p.table, dev.lengths.tolist(), p.news, p.dim ** -0.5)
        _check(got[0].cpu().numpy(), got[1].cpu().numpy(), *want, p.dim)


def test_two_streams_at_once(gpu_lib, monkeypatch):
    import torch
    monkeypatch.setenv("VQ_SWITCHES", "shared=1")
    p = Problem(27, [(512, 512, [(50, 2)] * 6)], [], 8, 2, 128, 16, 8)
    dev, prefix = p.up()
    q = torch.from_numpy(p.q).cuda()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []

    def call(x):
        return gpu_lib.attention_shared(x, dev.k, dev.v, dev.table, dev.lengths, k_scales=dev.k_scales, v_scales=dev.v_scales, max_new=2, **prefix)
    other = q.flip(0)
    want = call(q), call(other)
    torch.cuda.synchronize()
    for _ in range(4):
        for s, x in zip(streams, (q, other)):
            with torch.cuda.stream(s):
                got.append((s is streams[0], call(x)))
    torch.cuda.synchronize()
    for first, out in got:
        assert torch.equal(out, want[0] if first else want[1])


def test_what_the_package_refuses(gpu_lib):
    import torch
    p = Problem(28, [(64, 64, [(5, 1)] * 3)], [], 4, 2, 64, 16, 16)
    dev, prefix = p.up()
    q = torch.from_numpy(p.q).cuda()
    good = dict(q=q, k_pages=dev.k, v_pages=dev.v, page_table=dev.table, lengths=dev.lengths, **prefix)
    gpu_lib.attention_shared(**good)
    for bad in (dict(prefix_table=prefix["prefix_table"].long()), dict(prefix_table=prefix["prefix_table"][0]), dict(prefix_table=prefix["prefix_table"].repeat(2, 1)),
                dict(prefix_lengths=prefix["prefix_lengths"].float()), dict(prefix_lengths=None), dict(members=torch.zeros(3, dtype=torch.int32, device="cuda")),
                dict(prefix_lengths=prefix["prefix_lengths"].repeat(2), prefix_table=prefix["prefix_table"].repeat(2, 1)), dict(max_prefix=0.5), dict(max_members="x"),
                dict(prefix_table=torch.zeros((1, 8), dtype=torch.int32, device="cuda")[:, ::2]), dict(k_scales=torch.ones(1, device="cuda")), dict(q=q[..., :32])):
        with pytest.raises(ValueError):
            gpu_lib.attention_shared(**dict(good, **bad))
    for bad in (dict(max_prefix=10 ** 6), dict(max_members=0), dict(max_own=-1), dict(max_prefix=-1), dict(scale=-1.0)):
        with pytest.raises(gpu_lib.VQError):
            gpu_lib.attention_shared(**dict(good, **bad))


@pytest.mark.parametrize("switches", ["shared=0", "shared=1", "shared=1,prefix=p", "shared=2"])
def test_tokens_beyond_max_length_are_left_out(gpu_lib, monkeypatch, switches):
    """A bound of the sequences' lengths inside of the prefix: what the prefix has behind it is seen by no token, as in vq_attention."""
    import torch
    monkeypatch.setenv("VQ_SWITCHES", switches)
    p = Problem(29, [(256, 256, [(30, 1), (100, 1), (2, 1)])], [(150, 1)], 8, 2, 128, 16, 8)
    dev, prefix = p.up()
    table = p.table.copy()
    table[:, 192 // 16:] = -1
    want = ref.attention(p.q, p.cache, table, p.lengths, p.news, p.dim ** -0.5)
    out, lse = gpu_lib.attention_shared(torch.from_numpy(p.q).cuda(), dev.k, dev.v, dev.table, dev.lengths, k_scales=dev.k_scales, v_scales=dev.v_scales, return_lse=True, max_length=192,
                                        max_prefix=256, **prefix)
    torch.cuda.synchronize()
    _check(out.cpu().numpy(), lse.cpu().numpy(), *want, p.dim)


@pytest.mark.parametrize("prefixes,members,common,own", [(1, 16, 2048, 60), (3, 12, 2048, 50), (10, 6, 1024, 20)])
def test_prefixes_are_computed_once_without_bounds(gpu_lib, monkeypatch, prefixes, members, common, own):
    """Without max_own, max_members and max_prefix, which only the tables' sizes bound then, the results are those of the shared halves, bit for bit, and not vq_attention's."""
    import torch
    monkeypatch.setenv("VQ_SWITCHES", "")
    p = Problem(30, [(common, common, [(own, 1)] * members)] * prefixes, [], 64, 8, 128, 16, 8)
    dev, prefix = p.up()
    q, cache, scales = torch.from_numpy(p.q).cuda(), (dev.k, dev.v, dev.table, dev.lengths), dict(k_scales=dev.k_scales, v_scales=dev.v_scales)
    got, plain = gpu_lib.attention_shared(q, *cache, **scales, **prefix), gpu_lib.attention(q, *cache, **scales)
    monkeypatch.setenv("VQ_SWITCHES", "shared=1")
    length, of_prefix = (16 * t.shape[1] for t in (p.table, p.prefix_table))
    shared = gpu_lib.attention_shared(q, *cache, **scales, **prefix, max_length=length, max_prefix=of_prefix, max_members=prefixes * members, max_own=length - of_prefix)
    torch.cuda.synchronize()
    assert torch.equal(got, shared) and not torch.equal(got, plain)


@pytest.mark.parametrize("q_heads,heads,dim,bits", [(4, 2, 16, 16), (6, 2, 80, 8), (8, 2, 64, 16), (14, 2, 128, 8), (4, 2, 192, 8), (2, 1, 256, 16)])
@pytest.mark.parametrize("switches", ["shared=1", "shared=2", "shared=1,prefix=p,prefix_parts=1", "shared=2,attention=d,parts=2", "shared=2,attention=p,parts=1"])
def test_several_prefixes_without_bounds(gpu_lib, monkeypatch, q_heads, heads, dim, bits, switches):
    """Prefixes of which each may have all of the sequences, whose partial results lie by the call's new tokens: of one sequence, of none, of most, with sequences in front of, between and behind them."""
    import torch
    monkeypatch.setenv("VQ_SWITCHES", switches)
    p = Problem(31, [(128, 128, [(9, 2)]), (64, 64, []), (320, 317, [(20, 3)] * 11 + [("330", 1), ("0", 2)]), (96, 96, [(70, 5), (4, 4)])], [(33, 2), (1, 1)], q_heads, heads, dim, 16, bits)
    dev, prefix = p.up()
    args = dict(k_scales=dev.k_scales, v_scales=dev.v_scales, starts=dev.starts, max_new=max(p.news), return_lse=True)
    want = p.want(dim ** -0.5)

    def check(**kw):
        out, lse = gpu_lib.attention_shared(torch.from_numpy(p.q).cuda(), dev.k, dev.v, dev.table, dev.lengths, **args, **prefix, **kw)
        torch.cuda.synchronize()
        _check(out.cpu().numpy(), lse.cpu().numpy(), *want, dim)
    check()
    check(max_members=12)
    # the first sequence as one without a prefix, the third prefix's last ones too
    prefix["members"] = torch.tensor([1, 1, 1, 9, 14], dtype=torch.int32, device="cuda")
    prefix["prefix_lengths"] = torch.tensor([128, 64, 317, 0], dtype=torch.int32, device="cuda")
    check()
