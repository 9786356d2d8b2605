"""vq_residual_norm on the GPU against 64 bits.

Bounds from its arithmetic: y is x plus a product of up to five binary32 factors (eight roundings with the norm's root and division, and the
norm's sum over up to 128 partial sums in each of its levels: 2^-18 of the product covers them), rounded once more to its type; z is y before
that rounding times a factor of the same kind, rounded to binary16."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _reference(h, x, pre, post, gate, scale, eps):
    norm = lambda a, w: a / np.sqrt((a ** 2).mean(1, keepdims=True) + eps) * w  # noqa: E731
    f = np.zeros_like(x) if h is None else h
    if post is not None:
        f = norm(f, post)
    if gate is not None:
        f = f * gate
    y = x + scale * f
    return y, np.abs(x) + np.abs(scale * f), None if pre is None else norm(y, pre)


@pytest.mark.parametrize("rows,width", [(1, 4096), (3, 1), (2, 7), (5, 64), (7, 65), (2, 513), (33, 1000), (1, 8192), (3, 2049), (2, 11008), (2, 16384), (1, 32768), (300, 512)])
@pytest.mark.parametrize("stream", [16, 32])
@pytest.mark.parametrize("post,gate,scale", [(False, None, 1.0), (True, None, 0.5), (False, "channel", 0.125), (True, "token", -1.0)])
@pytest.mark.parametrize("pitch", [0, 3])
def test_residual_norm(gpu_lib, rows, width, stream, post, gate, scale, pitch):
    import torch
    rng = np.random.default_rng(rows * 100003 + width)
    kind, eps = (np.float16 if stream == 16 else np.float32), 1e-5
    make = lambda shape, s=1.0, k=np.float16: (rng.standard_normal(shape) * s).astype(k)  # noqa: E731
    h, x = make((rows, width)), make((rows, width), 4.0, kind)
    pre, post = make(width), make(width) if post else None
    gate = {None: None, "channel": make(width), "token": make((rows, width))}[gate]

    def up(a):
        if a is None:
            return None
        t = torch.from_numpy(a).cuda()
        if not pitch or a.ndim == 1:
            return t
        room = torch.zeros((rows, width + pitch), dtype=t.dtype, device="cuda")
        room[:, 1: 1 + width] = t
        return room[:, 1: 1 + width]
    y, z = gpu_lib.residual_norm(up(h), up(x), pre=up(pre), post=up(post), gate=up(gate), scale=scale, eps=eps)
    torch.cuda.synchronize()
    wide = lambda a: None if a is None else a.astype(np.float64)  # noqa: E731
    want_y, size, want_z = _reference(wide(h), wide(x), wide(pre), wide(post), wide(gate), scale, eps)
    ulp = 2.0 ** -11 if stream == 16 else 2.0 ** -24
    off = np.abs(y.cpu().numpy().astype(np.float64) - want_y)
    assert (off <= ulp * np.abs(want_y) + 2.0 ** -18 * size + 2.0 ** -25).all(), off.max()
    # the errors of y and of its norm: y's own, relative to the row's size where y is a difference
    factor = np.abs(wide(pre)) / np.sqrt((want_y ** 2).mean(1, keepdims=True) + eps)
    off = np.abs(z.cpu().numpy().astype(np.float64) - want_z)
    root = np.sqrt((size ** 2).mean(1, keepdims=True)) / np.sqrt((want_y ** 2).mean(1, keepdims=True) + eps)
    assert (off <= 2.0 ** -11 * np.abs(want_z) + 2.0 ** -18 * (size * factor + np.abs(want_z) * (1 + root)) + 2.0 ** -25).all(), off.max()


@pytest.mark.parametrize("rows,width", [(600, 1000), (700, 2049), (600, 4100), (530, 8192), (520, 12000)])
@pytest.mark.parametrize("stream", [16, 32])
def test_residual_norm_of_many_rows(gpu_lib, rows, width, stream):
    test_residual_norm(gpu_lib, rows, width, stream, True, "channel", 0.5, 0)
    test_residual_norm(gpu_lib, rows, width, stream, False, "token", 1.0, 5)


def test_more_rows_than_one_launch_takes(gpu_lib):
    """Every row of a matrix of 2^21 + 2^20 + 5 rows gets what it gets by itself."""
    import torch
    rows, width = 2 ** 21 + 2 ** 20 + 5, 16
    g = torch.Generator(device="cuda").manual_seed(5)
    h, x, w = (torch.randn(s, device="cuda", generator=g).half() for s in ((rows, width), (rows, width), (width,)))
    gate = torch.randn((rows, width), device="cuda", generator=g).half()
    y, z = gpu_lib.residual_norm(h, x, pre=w, post=w, gate=gate)
    for at in (slice(0, 300), slice(2 ** 21 - 100, 2 ** 21 + 100), slice(rows - 200, rows)):
        want = gpu_lib.residual_norm(h[at], x[at], pre=w, post=w, gate=gate[at])
        assert torch.equal(y[at], want[0]) and torch.equal(z[at], want[1])


def test_norm_alone_sum_alone_and_in_place(gpu_lib):
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    h, x, w = (torch.randn(s, device="cuda", generator=g).half() for s in ((17, 1280), (17, 1280), (1280,)))
    y, z = gpu_lib.residual_norm(h, x, pre=w)
    alone, none = gpu_lib.residual_norm(h, x)
    assert none is None and torch.equal(alone, y)
    same, first = gpu_lib.residual_norm(None, x, pre=w)                # a model's first norm
    assert torch.equal(same, x) and torch.equal(first, gpu_lib.residual_norm(torch.zeros_like(h), x, pre=w)[1])
    a, b = x.clone(), h.clone()
    got = gpu_lib.residual_norm(b, a, pre=w, y=a, z=b)
    assert got[0] is a and got[1] is b and torch.equal(a, y) and torch.equal(b, z)


def test_what_is_not_finite_stays_in_its_row(gpu_lib):
    import torch
    x = torch.ones((4, 300), dtype=torch.float16, device="cuda")
    h, w = torch.ones_like(x), torch.ones(300, dtype=torch.float16, device="cuda")
    want = gpu_lib.residual_norm(h, x, pre=w, post=w)
    h[1, 7], x[2, 299] = float("inf"), float("nan")
    y, z = gpu_lib.residual_norm(h, x, pre=w, post=w)
    torch.cuda.synchronize()
    for r in (0, 3):
        assert torch.equal(y[r], want[0][r]) and torch.equal(z[r], want[1][r])
    assert z[1].isnan().any() and z[2].isnan().all()
    zero = torch.zeros((1, 300), dtype=torch.float16, device="cuda")
    assert (gpu_lib.residual_norm(zero, zero, pre=w, post=w)[1] == 0).all()      # no division by nothing
