"""vq_kv_append, vq_attention and vq_residual_norm at the C-ABI boundary on the host: what they refuse (no GPU work is enqueued)."""
import ctypes

import pytest

import paper_2409_17066_amd as vq

HEADS, DIM, PAGE = 2, 64, 16


def _cache(**kw):
    """A cache of 8-bit pages for three sequences of up to 64 tokens that bring two new ones each."""
    d = vq.vq_kv_desc(struct_size=ctypes.sizeof(vq.vq_kv_desc), type=vq.VQ_KV_E4M3, kv_heads=HEADS, head_dim=DIM, page_tokens=PAGE, n_pages=12, n_seqs=3,
                      n_tokens=6, max_new=2, max_length=64, table_pages=4, reserved=0, k_pages=0x10000, v_pages=0x20000,
                      k_page_stride=HEADS * DIM * PAGE, v_page_stride=HEADS * DIM * PAGE, k_scales=0x30000, v_scales=0x31000, page_table=0x40000,
                      table_stride=4, lengths=0x41000, starts=0x42000)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _append(cache=None, **kw):
    a = dict(k_ptr=0x1000, ldk=HEADS * DIM, v_ptr=0x2000, ldv=HEADS * DIM, q_ptr=0x3000, ldq=4 * DIM, q_heads=4, q_out_ptr=0x4000, ldq_out=4 * DIM)
    a.update(kw)
    return vq.vq_kv_append(cache if cache is not None else _cache(), **a)


def _attend(cache=None, **kw):
    a = dict(q_ptr=0x3000, ldq=4 * DIM, q_heads=4, softmax_scale=0.125, window=0, sinks=0, out_ptr=0x4000, ldo=4 * DIM)
    a.update(kw)
    return vq.vq_attention(cache if cache is not None else _cache(), **a)


BAD_CACHES = [
    (dict(struct_size=8), vq.VQ_ERR_SHAPE), (dict(reserved=1), vq.VQ_ERR_SHAPE),
    (dict(type=2), vq.VQ_ERR_SHAPE), (dict(type=-1), vq.VQ_ERR_SHAPE),
    (dict(kv_heads=0), vq.VQ_ERR_SHAPE), (dict(kv_heads=-2), vq.VQ_ERR_SHAPE), (dict(kv_heads=65536), vq.VQ_ERR_SHAPE),
    (dict(head_dim=0), vq.VQ_ERR_SHAPE), (dict(head_dim=72), vq.VQ_ERR_SHAPE), (dict(head_dim=272), vq.VQ_ERR_SHAPE),
    (dict(page_tokens=8), vq.VQ_ERR_SHAPE), (dict(page_tokens=48), vq.VQ_ERR_SHAPE), (dict(page_tokens=512), vq.VQ_ERR_SHAPE),
    (dict(n_pages=0), vq.VQ_ERR_SHAPE), (dict(n_seqs=0), vq.VQ_ERR_SHAPE), (dict(n_tokens=0), vq.VQ_ERR_SHAPE),
    (dict(max_new=0), vq.VQ_ERR_SHAPE), (dict(max_new=7), vq.VQ_ERR_SHAPE),
    (dict(max_length=-1), vq.VQ_ERR_SHAPE), (dict(max_length=65), vq.VQ_ERR_SHAPE),
    (dict(max_length=2 ** 30 + 1, table_pages=2 ** 27, table_stride=2 ** 27), vq.VQ_ERR_SHAPE),
    (dict(table_pages=-1), vq.VQ_ERR_SHAPE), (dict(table_stride=3), vq.VQ_ERR_SHAPE),
    (dict(starts=None, n_tokens=7), vq.VQ_ERR_SHAPE),                       # not as many for each
    (dict(starts=None, max_new=1), vq.VQ_ERR_SHAPE),                        # two each
    (dict(k_pages=None), vq.VQ_ERR_NULL), (dict(v_pages=None), vq.VQ_ERR_NULL), (dict(lengths=None), vq.VQ_ERR_NULL),
    (dict(page_table=None), vq.VQ_ERR_NULL), (dict(k_scales=None), vq.VQ_ERR_NULL), (dict(v_scales=None), vq.VQ_ERR_NULL),
    (dict(k_page_stride=HEADS * DIM * PAGE - 16), vq.VQ_ERR_SHAPE), (dict(v_page_stride=0), vq.VQ_ERR_SHAPE),
    (dict(k_page_stride=1 << 32), vq.VQ_ERR_SHAPE), (dict(type=vq.VQ_KV_FP16, v_page_stride=1 << 31), vq.VQ_ERR_SHAPE),
    (dict(k_page_stride=HEADS * DIM * PAGE + 8), vq.VQ_ERR_ALIGNMENT), (dict(type=vq.VQ_KV_FP16, v_page_stride=HEADS * DIM * PAGE + 4), vq.VQ_ERR_ALIGNMENT),
    (dict(k_pages=0x10008), vq.VQ_ERR_ALIGNMENT), (dict(v_pages=0x20001), vq.VQ_ERR_ALIGNMENT),
    (dict(lengths=0x41002), vq.VQ_ERR_ALIGNMENT), (dict(page_table=0x40001), vq.VQ_ERR_ALIGNMENT), (dict(starts=0x42002), vq.VQ_ERR_ALIGNMENT),
    (dict(k_scales=0x30002), vq.VQ_ERR_ALIGNMENT), (dict(v_scales=0x31001), vq.VQ_ERR_ALIGNMENT),
]


@pytest.mark.parametrize("kw,status", BAD_CACHES, ids=str)
def test_caches_that_are_refused(kw, status):
    assert _append(_cache(**kw)) == status
    assert _attend(_cache(**kw)) == status
    assert vq.vq_attention_workspace_bytes(_cache(**kw), 4) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(k_ptr=None), vq.VQ_ERR_NULL), (dict(v_ptr=None), vq.VQ_ERR_NULL), (dict(q_out_ptr=None), vq.VQ_ERR_NULL),
    (dict(ldk=HEADS * DIM - 1), vq.VQ_ERR_SHAPE), (dict(ldv=0), vq.VQ_ERR_SHAPE), (dict(ldq=4 * DIM - 1), vq.VQ_ERR_SHAPE),
    (dict(ldq_out=-4 * DIM), vq.VQ_ERR_SHAPE), (dict(q_heads=0), vq.VQ_ERR_SHAPE), (dict(q_heads=65536, ldq=1 << 30, ldq_out=1 << 30), vq.VQ_ERR_SHAPE),
    (dict(k_ptr=0x1001), vq.VQ_ERR_ALIGNMENT), (dict(v_ptr=0x2001), vq.VQ_ERR_ALIGNMENT), (dict(q_ptr=0x3001), vq.VQ_ERR_ALIGNMENT),
    (dict(q_out_ptr=0x4001), vq.VQ_ERR_ALIGNMENT),
], ids=str)
def test_appends_that_are_refused(kw, status):
    assert _append(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(cos=None), vq.VQ_ERR_NULL), (dict(sin=None), vq.VQ_ERR_NULL), (dict(positions=0), vq.VQ_ERR_SHAPE),
    (dict(rotary_dim=0), vq.VQ_ERR_SHAPE), (dict(rotary_dim=33), vq.VQ_ERR_SHAPE), (dict(rotary_dim=DIM + 2), vq.VQ_ERR_SHAPE),
    (dict(ld=31), vq.VQ_ERR_SHAPE), (dict(cos=0x50002), vq.VQ_ERR_ALIGNMENT), (dict(sin=0x51001), vq.VQ_ERR_ALIGNMENT),
    (dict(position=0x52002), vq.VQ_ERR_ALIGNMENT),
], ids=str)
def test_rotations_that_are_refused(kw, status):
    r = vq.vq_rotary(cos=0x50000, sin=0x51000, ld=32, positions=64, rotary_dim=64, interleaved=0, position=None)
    for k, v in kw.items():
        setattr(r, k, v)
    assert _append(rotary=r) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q_ptr=None), vq.VQ_ERR_NULL), (dict(out_ptr=None), vq.VQ_ERR_NULL),
    (dict(q_heads=0), vq.VQ_ERR_SHAPE), (dict(q_heads=3, ldq=1024, ldo=1024), vq.VQ_ERR_SHAPE),          # no multiple of the key heads
    (dict(q_heads=65536, ldq=1 << 30, ldo=1 << 30), vq.VQ_ERR_SHAPE), (dict(window=-1), vq.VQ_ERR_SHAPE), (dict(sinks=-1, window=4), vq.VQ_ERR_SHAPE),
    (dict(ldq=4 * DIM - 1), vq.VQ_ERR_SHAPE), (dict(ldo=0), vq.VQ_ERR_SHAPE),
    (dict(softmax_scale=0.0), vq.VQ_ERR_SHAPE), (dict(softmax_scale=-1.0), vq.VQ_ERR_SHAPE), (dict(softmax_scale=float("nan")), vq.VQ_ERR_SHAPE),
    (dict(softmax_scale=float("inf")), vq.VQ_ERR_SHAPE),
    (dict(q_ptr=0x3001), vq.VQ_ERR_ALIGNMENT), (dict(out_ptr=0x4001), vq.VQ_ERR_ALIGNMENT), (dict(lse_ptr=0x5002), vq.VQ_ERR_ALIGNMENT),
    (dict(workspace_ptr=0x6010, workspace_bytes=4096), vq.VQ_ERR_ALIGNMENT),
], ids=str)
def test_attentions_that_are_refused(kw, status):
    assert _attend(**kw) == status


def test_rows_beyond_what_the_kernels_count():
    """2^15 tokens of 2^8 queries a key head."""
    many = _cache(kv_heads=1, n_tokens=1 << 15, max_new=1 << 15, k_page_stride=DIM * PAGE, v_page_stride=DIM * PAGE)
    assert _attend(many, q_heads=256, ldq=256 * DIM, ldo=256 * DIM) == vq.VQ_ERR_SHAPE
    assert vq.vq_attention_workspace_bytes(many, 256) == 0


def test_no_cache():
    assert vq.vq_kv_append(None, 0x1000, 128, 0x2000, 128) == vq.VQ_ERR_NULL
    assert vq.vq_attention(None, 0x3000, 256, 4, 0.125, 0, 0, 0x4000, 256) == vq.VQ_ERR_NULL


@pytest.mark.parametrize("kw,status", [
    (dict(x_ptr=None), vq.VQ_ERR_NULL), (dict(y_ptr=None, z_ptr=None), vq.VQ_ERR_NULL), (dict(w_pre_ptr=None), vq.VQ_ERR_NULL),
    (dict(h_ptr=None), vq.VQ_ERR_NULL), (dict(h_ptr=None, w_post_ptr=None), vq.VQ_ERR_NULL), (dict(h_ptr=None, gate_ptr=None), vq.VQ_ERR_NULL),
    (dict(rows=0), vq.VQ_ERR_SHAPE), (dict(width=0), vq.VQ_ERR_SHAPE),
    (dict(width=32769, ldh=1 << 16, ldx=1 << 16, ldy=1 << 16, ldz=1 << 16), vq.VQ_ERR_SHAPE),
    (dict(ldh=99), vq.VQ_ERR_SHAPE), (dict(ldx=0), vq.VQ_ERR_SHAPE), (dict(ldy=99), vq.VQ_ERR_SHAPE), (dict(ldz=-100), vq.VQ_ERR_SHAPE),
    (dict(ldgate=50), vq.VQ_ERR_SHAPE), (dict(eps=-1e-6), vq.VQ_ERR_SHAPE), (dict(eps=float("nan")), vq.VQ_ERR_SHAPE),
    (dict(x_ptr=0x1002, stream32=1), vq.VQ_ERR_ALIGNMENT), (dict(y_ptr=0x3002, stream32=1), vq.VQ_ERR_ALIGNMENT), (dict(x_ptr=0x1001), vq.VQ_ERR_ALIGNMENT),
    (dict(h_ptr=0x2001), vq.VQ_ERR_ALIGNMENT), (dict(z_ptr=0x4001), vq.VQ_ERR_ALIGNMENT), (dict(w_post_ptr=0x5001), vq.VQ_ERR_ALIGNMENT),
    (dict(gate_ptr=0x6001), vq.VQ_ERR_ALIGNMENT), (dict(w_pre_ptr=0x7001), vq.VQ_ERR_ALIGNMENT),
], ids=str)
def test_norms_that_are_refused(kw, status):
    a = dict(h_ptr=0x2000, ldh=100, x_ptr=0x1000, ldx=100, w_post_ptr=0x5000, gate_ptr=0x6000, ldgate=0, scale=1.0, w_pre_ptr=0x7000, eps=1e-5, stream32=0,
             rows=3, width=100, y_ptr=0x3000, ldy=100, z_ptr=0x4000, ldz=100)
    a.update(kw)
    assert vq.vq_residual_norm(**a) == status


def test_the_workspace_follows_from_the_sizes_alone():
    """Sequences too short to be cut need none, and neither do windows."""
    long = dict(n_seqs=1, n_tokens=1, max_new=1, starts=None, table_pages=4096, table_stride=4096, max_length=65536)
    sizes = vq.vq_attention_workspace_bytes(_cache(**long), 4)
    parts = sizes // (4 * (DIM * 4 + 8))
    assert parts > 1 and sizes % 256 == 0 and sizes >= parts * 4 * (DIM * 4 + 8)
    assert vq.vq_attention_workspace_bytes(_cache(**dict(long, max_length=64)), 4) == 0
    assert vq.vq_attention_workspace_bytes(_cache(**long), 4, window=64, sinks=4) == 0
    assert vq.vq_attention_workspace_bytes(_cache(**long), 3) == 0 == vq.vq_attention_workspace_bytes(_cache(**long), 4, window=-1)
