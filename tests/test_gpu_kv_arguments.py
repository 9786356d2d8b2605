"""Arguments of kv_append() and attention() that say the same thing in different ways, or nothing."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _place(torch):
    pages = [torch.zeros(s, dtype=torch.float16, device="cuda") for s in ((6, 2, 16, 64), (6, 2, 64, 16))]
    table, lengths = torch.arange(6, dtype=torch.int32, device="cuda").reshape(2, 3), torch.tensor([20, 40], dtype=torch.int32, device="cuda")
    return pages + [table, lengths], lambda heads: torch.ones((4, heads, 64), dtype=torch.float16, device="cuda")


@pytest.mark.parametrize("truth", [True, 1, np.True_, "yes", False, 0, np.False_, None])
def test_any_truth_value_asks_for_the_sums(gpu_lib, truth):
    import torch
    place, new = _place(torch)
    got = gpu_lib.attention(new(4), *place, return_lse=truth)
    if truth:
        out, lse = got
        assert out.shape == (4, 4, 64) and lse.shape == (4, 4)
    else:
        assert got.shape == (4, 4, 64)
    with pytest.raises(ValueError):
        gpu_lib.attention(new(4), *place, return_lse=torch.zeros(2, device="cuda"))


def test_positions_without_tables_are_refused(gpu_lib):
    """A caller who gives positions expects a rotation."""
    import torch
    place, new = _place(torch)
    position = torch.zeros(4, dtype=torch.int32, device="cuda")
    table = torch.ones((48, 32), device="cuda")
    for bad in (position, position.long(), 3):
        with pytest.raises(ValueError):
            gpu_lib.kv_append(new(2), new(2), *place, position=bad)
    gpu_lib.kv_append(new(2), new(2), *place, cos=table, sin=table, position=position)
    torch.cuda.synchronize()
    assert place[0].any()


def test_a_call_that_is_repeated_with_queries_in_place(gpu_lib):
    """The cache stays as it is; queries are rotated by every call, so that a repeated one needs them as they were."""
    import torch
    place, _ = _place(torch)
    rng = torch.Generator(device="cuda").manual_seed(3)
    k, v, q = (torch.randn((4, n, 64), generator=rng, device="cuda").half() for n in (2, 2, 4))
    angle = torch.arange(48, device="cuda")[:, None] * 0.1 * torch.ones(32, device="cuda")
    tables = dict(cos=angle.cos(), sin=angle.sin())
    want = gpu_lib.kv_append(k, v, *place, q=q, **tables)
    pages = [p.clone() for p in place[:2]]
    mine = q.clone()
    assert gpu_lib.kv_append(k, v, *place, q=mine, q_out=mine, **tables) is mine
    assert torch.equal(mine, want) and all(torch.equal(a, b) for a, b in zip(pages, place))
    gpu_lib.kv_append(k, v, *place, q=mine, q_out=mine, **tables)
    assert not torch.equal(mine, want) and all(torch.equal(a, b) for a, b in zip(pages, place))
    mine.copy_(q)
    gpu_lib.kv_append(k, v, *place, q=mine, q_out=mine, **tables)
    assert torch.equal(mine, want) and all(torch.equal(a, b) for a, b in zip(pages, place))
