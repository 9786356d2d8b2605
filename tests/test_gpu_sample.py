"""vq_sample on the GPU against the definition in 64 bits: the token exactly, its probability to a rounding."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _one(x, u, temperature, top_k, top_p, min_p):
    """(token, probability) of a row of logits, written out."""
    x = x.astype(np.float64)
    u = min(max(float(u), 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    order = np.argsort(np.where(np.isnan(x), np.inf, -x), kind="stable")
    order = order[: int((x > -np.inf).sum())]
    if not len(order):
        return -1, 0.0
    if not temperature > 0:
        return int(order[0]), 1.0
    largest = x[order[0]]
    with np.errstate(invalid="ignore", over="ignore"):
        w = (x[order] == np.inf).astype(np.float64) if largest == np.inf else np.exp((x[order] - largest) / np.float64(temperature))
    keep = len(order) if top_k <= 0 else min(int(top_k), len(order))
    w = w[:keep]
    if top_p < 1:
        sums = np.concatenate([[0.0], np.cumsum(w)])
        w = w[: max(1, int((sums[:-1] < np.float64(max(top_p, np.float32(0))) * sums[-1]).sum()))]
    if min_p > 0:
        w = w[w >= min(np.float64(min_p), 1.0)]
    sums = np.cumsum(w)
    at = min(int((sums <= u * sums[-1]).sum()), len(w) - 1)
    return int(order[at]), float(w[at] / sums[-1])


def _check(gpu_lib, logits, uniform, out=None, **how):
    """logits: fp16 device tensor [rows][vocabulary] of any pitch; settings: numbers or numpy arrays."""
    import torch
    given = {k: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for k, v in how.items()}
    rows = logits.shape[0]
    token, p = gpu_lib.sample(logits, torch.from_numpy(uniform).cuda(), return_prob=True, out=out, **given)
    again = gpu_lib.sample(logits, torch.from_numpy(uniform).cuda(), **given)
    torch.cuda.synchronize()
    assert torch.equal(token, again)
    token, p, x = token.cpu().numpy(), p.cpu().numpy(), logits.cpu().numpy()
    default = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    for r in range(rows):
        mine = {k: (how[k][r] if isinstance(how[k], np.ndarray) else np.float32(how[k])) if k in how else default[k] for k in default}
        want, probability = _one(x[r], uniform[r], **mine)
        assert token[r] == want, (r, mine, uniform[r], int(token[r]), want)
        # (binary64 throughout, rounded once to binary32; subnormal numbers to 2^-150)
        assert abs(p[r] - probability) <= 2.0 ** -23 * probability + 2.0 ** -149, (r, p[r], probability)


def _logits(rng, rows, n):
    x = 2.2 * rng.standard_normal((rows, n)) - 2.0
    for r in range(rows):
        few = rng.integers(0, n, min(n, 40))
        x[r, few] = 14.0 - 1.9 * np.log1p(np.arange(len(few)))
    return x.astype(np.float16)


SETTINGS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=50, temperature=1.5), dict(top_p=0.9), dict(top_p=0.3, temperature=2.5), dict(min_p=0.05),
            dict(top_k=40, top_p=0.95, min_p=0.02, temperature=0.8), dict(temperature=0.0), dict(top_k=10 ** 9), dict(temperature=100.0), dict(temperature=1e-3), dict(temperature=float("inf"), top_p=0.5)]


@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 63, 511, 513, 1000, 8191, 8192, 8193, 32000, 65536, 100003, 131079, 300001])
def test_vocabularies(gpu_lib, n):
    import torch
    rng = np.random.default_rng(n)
    rows = 3
    wide = torch.zeros((rows, n + 3), dtype=torch.float16, device="cuda")
    for how in SETTINGS:
        # rows of an odd pitch, of which none is on 16 bytes
        view = wide[:, 1: n + 1]
        view.copy_(torch.from_numpy(_logits(rng, rows, n)))
        _check(gpu_lib, view, rng.random(rows, dtype=np.float32), **how)


def test_each_row_its_own_settings(gpu_lib):
    import torch
    rng = np.random.default_rng(3)
    rows, n = 300, 5003
    how = dict(temperature=rng.choice(np.float32([0, -1, np.nan, 0.3, 1, 1.7, np.inf, 1e-30]), rows), top_k=rng.choice(np.int32([-5, 0, 1, 2, 17, 400, 5003, 2 ** 31 - 1]), rows),
               top_p=rng.choice(np.float32([-1, 0, 1e-6, 0.1, 0.5, 0.97, 1 - 2.0 ** -24, 1, 7, np.nan]), rows),
               min_p=rng.choice(np.float32([-1, 0, 1e-30, 0.01, 0.4, 1, 3, np.nan]), rows))
    uniform = rng.choice(np.float32([0, -0.5, 1e-30, 0.25, 0.5, 0.75, 1 - 2.0 ** -24, 1, 5, np.nan]), rows)
    uniform[::2] = rng.random(rows, dtype=np.float32)[::2]
    _check(gpu_lib, torch.from_numpy(_logits(rng, rows, n)).cuda(), uniform, **how)


def test_equal_logits_are_told_apart_by_their_tokens(gpu_lib):
    """Few different values, so that borders lie among equal ones, whose sums are whole numbers: what is on a border counts."""
    import torch
    rng = np.random.default_rng(4)
    for n, values in ((1000, [2.0]), (1024, [0.0, -0.0]), (4000, [1.5, 1.5, -1e4]), (777, [0.0, -np.inf])):
        x = rng.choice(np.float16(values), (40, n))
        uniform = (np.arange(40) / 40).astype(np.float32)
        for how in (dict(), dict(top_p=0.5), dict(top_k=100), dict(top_p=0.25, top_k=200), dict(min_p=1.0), dict(temperature=0.0)):
            _check(gpu_lib, torch.from_numpy(x).cuda(), uniform, **how)


def test_values_that_occur_more_than_65535_times(gpu_lib):
    """Counts beyond 16 bits: all alike (a warm-up on zeros), masks of the type's lowest value with and without a temperature at which they weigh something, and one
    more or less than a count holds, of even and of odd bins."""
    import torch
    rng = np.random.default_rng(5)
    n = 140001
    rows = []
    rows.append(np.zeros(n, np.float16))
    x = _logits(rng, 1, n)[0]
    x[rng.random(n) < 0.9] = -65504
    rows.append(x)
    for value in (np.float16(1.0), np.nextafter(np.float16(1.0), np.float16(2.0))):
        for count in (65535, 65536, 131072):
            x = (np.float16(-3.0) * np.ones(n)).astype(np.float16) if count == 131072 else (rng.standard_normal(n) * 0.01 - 3).astype(np.float16)
            x[rng.permutation(n)[:count]] = value
            rows.append(x)
    x = np.full(n, -np.inf, np.float16)
    x[rng.permutation(n)[:65536]] = 65504
    rows.append(x)
    x = rows[0].copy()
    x[::2] = -0.0
    rows.append(x)
    logits = torch.from_numpy(np.stack(rows)).cuda()
    for how in (dict(), dict(temperature=1e6), dict(top_k=70000, top_p=0.6), dict(top_p=0.3, temperature=50.0), dict(temperature=0.0), dict(min_p=0.5)):
        _check(gpu_lib, logits, rng.random(len(rows), dtype=np.float32), **how)


@pytest.mark.parametrize("n", [15, 16, 17, 70003, 140008, 140015])
def test_first_and_last_of_equal_logits(gpu_lib, n):
    """Each of the first and last tokens of a row of equal logits, at each distance from sixteen bytes."""
    import torch
    asked = np.array(sorted({i % n for i in range(-17, 17)}))
    uniform = ((asked + 0.5) / n).astype(np.float32)
    wide = torch.full((len(asked), n + 16), 3.0, dtype=torch.float16, device="cuda")
    for first in range(8):
        for how in (dict(), dict(temperature=0.25, top_p=1.0 - 2.0 ** -24)):
            token, p = gpu_lib.sample(wide[:, first: first + n], torch.from_numpy(uniform).cuda(), return_prob=True, **how)
            assert token.tolist() == asked.tolist(), (first, how)
            assert np.abs(p.cpu().numpy() * n - 1).max() <= 2.0 ** -22        # (binary32, rounded once, and this product)


@pytest.mark.parametrize("n", [129, 4000, 40005, 131100])
def test_where_vectors_begin(gpu_lib, n):
    """Rows at each distance from sixteen bytes, with what lies around them larger than anything in them."""
    import torch
    rng = np.random.default_rng(n)
    wide = torch.full((4, n + 17), 60000.0, dtype=torch.float16, device="cuda")
    for first in range(9):
        wide.fill_(60000.0)
        view = wide[:, first: first + n]
        x = _logits(rng, 4, n)
        x[1, 0] = x[2, -1] = 20.0
        x[3, 1:9] = x[3, -9:-1] = 17.0
        view.copy_(torch.from_numpy(x))
        for how in (dict(temperature=0.8), dict(top_k=12, top_p=0.97, min_p=0.001)):
            _check(gpu_lib, view, rng.random(4, dtype=np.float32), **how)


def test_logits_that_are_not_finite(gpu_lib):
    import torch
    rng = np.random.default_rng(6)
    x = _logits(rng, 12, 900)
    x[0] = -np.inf                                                  # an idle slot
    x[1] = np.nan
    x[2, ::3], x[2, 1::3] = np.nan, -np.nan
    x[3, 5], x[3, 700] = np.inf, np.inf
    x[4] = np.inf
    x[5, 1:] = -np.inf
    x[6] = -65504
    x[7, :] = np.float16(2.0 ** -24)                                # subnormal ones
    x[7, ::2] = -np.float16(2.0 ** -24)
    x[8] = np.where(np.arange(900) % 2, np.inf, np.nan)
    x[9, 10:] = -65504
    x[10] = 65504
    for how in (dict(), dict(top_k=3), dict(top_p=0.5, temperature=3.0), dict(min_p=0.1), dict(temperature=0.0), dict(temperature=1e30), dict(top_k=1, temperature=1e-30)):
        _check(gpu_lib, torch.from_numpy(x).cuda(), rng.random(12, dtype=np.float32), **how)


def test_given_output_and_nothing_else_written(gpu_lib):
    import torch
    rng = np.random.default_rng(7)
    room = torch.full((9,), 77, dtype=torch.int32, device="cuda")
    logits = torch.from_numpy(_logits(rng, 5, 333)).cuda()
    got = gpu_lib.sample(logits, torch.full((5,), 0.3, device="cuda"), out=room[2:7])
    torch.cuda.synchronize()
    assert got.data_ptr() == room[2:].data_ptr() and (room[:2] == 77).all() and (room[7:] == 77).all()
    _check(gpu_lib, logits, np.full(5, 0.3, np.float32), out=room[2:7])


def test_in_a_graph_and_on_two_streams(gpu_lib):
    import torch
    rng = np.random.default_rng(8)
    logits, uniform = torch.from_numpy(_logits(rng, 6, 20001)).cuda(), torch.rand(6, device="cuda")
    how = dict(top_k=torch.full((6,), 300, dtype=torch.int32, device="cuda"), top_p=0.9)
    gpu_lib.sample(logits, uniform, **how)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = gpu_lib.sample(logits, uniform, return_prob=True, **how)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(4):
        logits.copy_(torch.from_numpy(_logits(rng, 6, 20001)))
        uniform.uniform_()
        how["top_k"].fill_(2 + 100 * i)
        graph.replay()
        want = gpu_lib.sample(logits, uniform, return_prob=True, **how)
        torch.cuda.synchronize()
        side = []
        for s in streams:
            with torch.cuda.stream(s):
                side.append(gpu_lib.sample(logits, uniform, return_prob=True, **how))
        torch.cuda.synchronize()
        for got in [captured] + side:
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_rows_whose_offsets_pass_32_bits(gpu_lib):
    import torch
    rows, n = 5, 1000
    room = torch.empty((rows - 1) * ((1 << 30) - 7) + n, dtype=torch.float16, device="cuda")
    logits = room.as_strided((rows, n), ((1 << 30) - 7, 1))
    rng = np.random.default_rng(9)
    logits.copy_(torch.from_numpy(_logits(rng, rows, n)))
    _check(gpu_lib, logits, rng.random(rows, dtype=np.float32), top_p=0.9)


def test_what_the_package_refuses(gpu_lib):
    import torch
    x, u = torch.zeros((4, 50), dtype=torch.float16, device="cuda"), torch.zeros(4, device="cuda")
    for bad in (dict(logits=x.float()), dict(logits=x.t()), dict(logits=x[0]), dict(logits=x.cpu()), dict(uniform=u.double()), dict(uniform=u[:3]), dict(uniform=None),
                dict(temperature=u.half()), dict(temperature="x"), dict(top_k=u), dict(top_k=2.5), dict(top_p=torch.zeros(5, device="cuda")), dict(min_p=torch.zeros((4, 1), device="cuda")),
                dict(out=torch.zeros(4, dtype=torch.int64, device="cuda")), dict(out=torch.zeros(8, dtype=torch.int32, device="cuda")[::2]), dict(top_k=2 ** 40)):
        with pytest.raises(ValueError):
            gpu_lib.sample(**dict(dict(logits=x, uniform=u), **bad))
    with pytest.raises(gpu_lib.VQError):
        gpu_lib.sample(x[:0], u[:0])


def test_min_p_where_many_weights_are_alike(gpu_lib):
    """Temperatures at which weights far apart in the order of the values are still within min_p of one another: up to all of them, where every weight rounds to 1 in binary64."""
    import torch
    rng = np.random.default_rng(10)
    n = 3001
    x = np.concatenate([_logits(rng, 2, n), rng.uniform(-30000, 30000, (2, n)).astype(np.float16), (rng.standard_normal((2, n)) * 1e-4).astype(np.float16)])
    long = np.concatenate([np.full((6, 70000), -65504, np.float16), x], 1)         # (counted in 32 bits)
    for logits in (torch.from_numpy(x).cuda(), torch.from_numpy(long).cuda()):
        for how in (dict(temperature=1e30, min_p=1.0), dict(temperature=3e38, min_p=7.0), dict(temperature=1e25, min_p=1 - 2.0 ** -24), dict(temperature=1e30, min_p=1.0, top_k=2000),
                    dict(temperature=1e30, min_p=1.0, top_p=0.7), dict(temperature=1e10, min_p=1 - 2.0 ** -24), dict(temperature=1e6, min_p=0.997), dict(temperature=1e-30, min_p=1e-38)):
            _check(gpu_lib, logits, rng.random(6, dtype=np.float32), **how)
