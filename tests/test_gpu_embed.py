"""vq_embed on the GPU: scale * table[ids], the product in binary32 and rounded once, bit for bit."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _bits(x):
    x = x.contiguous().cpu().numpy()
    return x.view(np.uint16 if x.dtype == np.float16 else np.uint32)


@pytest.mark.parametrize("rows,width,vocabulary", [(1, 1, 1), (1, 4096, 100), (3, 7, 5), (40, 8, 9), (17, 9, 1000), (5, 2049, 33), (300, 64, 50), (2, 20000, 3), (70, 100, 64), (33, 24, 7)])
@pytest.mark.parametrize("stream", ["fp16", "fp32"])
def test_rows(gpu_lib, rows, width, vocabulary, stream):
    import torch
    kind = torch.float16 if stream == "fp16" else torch.float32
    g = torch.Generator().manual_seed(rows * width)
    for pitch in (0, 3):
        room = torch.randn((vocabulary, width + pitch), generator=g).half().cuda()
        table = room[:, : width]
        ids = torch.randint(-2, vocabulary + 2, (rows,), generator=g, dtype=torch.int32)      # some name no row
        ids[0] = 2 ** 31 - 1 if rows > 1 else 0
        there = ((ids >= 0) & (ids < vocabulary)).cuda()
        for scale in (1.0, 0.3, -width ** 0.5):
            want = torch.where(there[:, None], table[ids.clamp(0, vocabulary - 1).long().cuda()].float() * torch.tensor(scale, dtype=torch.float32, device="cuda"), torch.zeros((), device="cuda")).to(kind)
            got = gpu_lib.embed(ids.cuda(), table, scale=scale, dtype=kind)
            out = torch.full((rows, width + 2 * pitch), 7.0, dtype=kind, device="cuda")
            given = gpu_lib.embed(ids.cuda(), table, scale=scale, out=out[:, pitch: pitch + width])
            torch.cuda.synchronize()
            assert np.array_equal(_bits(got), _bits(want)) and np.array_equal(_bits(given), _bits(want))
            assert (out[:, :pitch] == 7).all() and (out[:, pitch + width:] == 7).all()


def test_what_is_not_finite_and_what_is_too_large(gpu_lib):
    import torch
    table = torch.tensor([[float("nan"), float("inf"), -float("inf"), 65504.0, 2.0 ** -24, -0.0, 1.0, -1.0, 3.0]], dtype=torch.float16, device="cuda")
    ids = torch.zeros(2, dtype=torch.int32, device="cuda")
    got = gpu_lib.embed(ids, table, scale=4.0)
    torch.cuda.synchronize()
    want = (table.float() * 4).half().expand(2, -1)
    assert torch.equal(got.nan_to_num(9, 8, 7), want.nan_to_num(9, 8, 7)) and got[0, 0].isnan() and got[0, 3] == float("inf")


def test_tables_beyond_32_bits(gpu_lib):
    import torch
    width, vocabulary = 4096, (1 << 32) // 4096 + 40
    table = torch.empty((vocabulary, width), dtype=torch.float16, device="cuda")
    ids = torch.tensor([0, vocabulary - 1, vocabulary // 2 + 3, vocabulary], dtype=torch.int32, device="cuda")
    for i in ids[:3].tolist():
        table[i] = torch.arange(width, device="cuda") % 97 + i % 31
    got = gpu_lib.embed(ids, table, dtype=torch.float32)
    torch.cuda.synchronize()
    assert torch.equal(got[:3], table[ids[:3].long()].float()) and (got[3] == 0).all()


def test_in_a_graph(gpu_lib):
    import torch
    table, ids = torch.randn((50, 300), device="cuda").half(), torch.zeros(6, dtype=torch.int32, device="cuda")
    gpu_lib.embed(ids, table)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = gpu_lib.embed(ids, table, scale=0.5, dtype=torch.float32)
    for i in range(3):
        ids.copy_(torch.arange(6) * 7 + i)
        graph.replay()
        want = gpu_lib.embed(ids, table, scale=0.5, dtype=torch.float32)
        torch.cuda.synchronize()
        assert torch.equal(captured, want)


def test_what_the_package_refuses(gpu_lib):
    import torch
    ids, table = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros((5, 8), dtype=torch.float16, device="cuda")
    for bad in (dict(ids=ids.long()), dict(ids=ids[None]), dict(ids=torch.zeros(6, dtype=torch.int32, device="cuda")[::2]), dict(table=table.float()), dict(table=table.t()),
                dict(ids=ids.cpu()), dict(dtype=torch.bfloat16), dict(dtype="fp16"), dict(scale="x"), dict(out=torch.zeros((3, 7), dtype=torch.float16, device="cuda")),
                dict(out=torch.zeros((3, 8), device="cuda"), dtype=torch.float16), dict(out=torch.zeros((8, 3), dtype=torch.float16, device="cuda").t())):
        with pytest.raises(ValueError):
            gpu_lib.embed(**dict(dict(ids=ids, table=table), **bad))
    for bad in (dict(ids=ids[:0]), dict(scale=float("nan")), dict(scale=float("inf"))):
        with pytest.raises(gpu_lib.VQError):
            gpu_lib.embed(**dict(dict(ids=ids, table=table), **bad))


@pytest.mark.parametrize("stream", ["fp16", "fp32"])
@pytest.mark.parametrize("width", [4099, 4096])
def test_results_of_more_than_the_caches_hold(gpu_lib, stream, width):
    """Results of 192 MB and more are written past the caches: from addresses of no more than an element's alignment on, of odd widths too, with ids that name no row."""
    import torch
    kind, element = (torch.float16, 2) if stream == "fp16" else (torch.float32, 4)
    rows, vocabulary = (192 << 20) // (width * element) + 5, 70
    g = torch.Generator(device="cuda").manual_seed(width)
    table = torch.randn((vocabulary, width + 1), device="cuda", generator=g).half()[:, 1:]
    ids = torch.randint(-2, vocabulary + 2, (rows,), device="cuda", generator=g, dtype=torch.int32)
    there = (ids >= 0) & (ids < vocabulary)
    want = torch.where(there[:, None], table[ids.clamp(0, vocabulary - 1).long()].float() * torch.tensor(0.3, dtype=torch.float32, device="cuda"), torch.zeros((), device="cuda")).to(kind)
    out = torch.full((rows, width + 3), 7.0, dtype=kind, device="cuda")
    got, given = gpu_lib.embed(ids, table, scale=0.3, dtype=kind), gpu_lib.embed(ids, table, scale=0.3, out=out[:, 1: 1 + width])
    torch.cuda.synchronize()
    bits = torch.int16 if stream == "fp16" else torch.int32
    assert torch.equal(got.view(bits), want.view(bits)) and torch.equal(given.contiguous().view(bits), want.view(bits))
    assert (out[:, 0] == 7).all() and (out[:, 1 + width:] == 7).all()


@pytest.mark.parametrize("stream", ["fp16", "fp32"])
def test_rows_of_the_result_past_32_bits(gpu_lib, stream):
    import torch
    kind = torch.float16 if stream == "fp16" else torch.float32
    rows, width, pitch = 4, 100, (1 << 30) + 3
    out = torch.empty((rows - 1) * pitch + width, dtype=kind, device="cuda").as_strided((rows, width), (pitch, 1))
    table, ids = torch.randn((9, width), device="cuda").half(), torch.tensor([3, 8, 9, 1], dtype=torch.int32, device="cuda")
    gpu_lib.embed(ids, table, out=out)
    torch.cuda.synchronize()
    want = table[ids.clamp(max=8).long()].to(kind)
    want[2] = 0
    assert torch.equal(out, want)
