"""vq_attention_shared, vq_embed and vq_sample at the C-ABI boundary on the host: what they refuse (no GPU work is enqueued)."""
import ctypes

import pytest

import paper_2409_17066_amd as vq
from test_kv_boundary import BAD_CACHES, DIM, _cache


def _prefix(**kw):
    d = vq.vq_prefix_desc(struct_size=ctypes.sizeof(vq.vq_prefix_desc), n_prefixes=2, max_members=2, max_length=32, max_own=32, table_pages=2, page_table=0x50000,
                          table_stride=2, lengths=0x51000, members=0x52000)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _attend(cache=None, prefix=None, **kw):
    a = dict(q_ptr=0x3000, ldq=4 * DIM, q_heads=4, softmax_scale=0.125, out_ptr=0x4000, ldo=4 * DIM)
    a.update(kw)
    return vq.vq_attention_shared(cache if cache is not None else _cache(), prefix if prefix is not None else _prefix(), **a)


@pytest.mark.parametrize("kw,status", BAD_CACHES, ids=str)
def test_caches_that_are_refused(kw, status):
    assert _attend(_cache(**kw)) == status
    assert vq.vq_attention_shared_workspace_bytes(_cache(**kw), _prefix(), 4) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), vq.VQ_ERR_SHAPE), (dict(n_prefixes=0), vq.VQ_ERR_SHAPE), (dict(n_prefixes=65536), vq.VQ_ERR_SHAPE), (dict(max_members=0), vq.VQ_ERR_SHAPE),
    (dict(max_length=-1), vq.VQ_ERR_SHAPE), (dict(max_length=33), vq.VQ_ERR_SHAPE), (dict(max_length=2 ** 30 + 1, table_pages=2 ** 27, table_stride=2 ** 27), vq.VQ_ERR_SHAPE),
    (dict(max_own=-1), vq.VQ_ERR_SHAPE), (dict(table_pages=-1), vq.VQ_ERR_SHAPE), (dict(table_stride=1), vq.VQ_ERR_SHAPE), (dict(members=None), vq.VQ_ERR_SHAPE),
    (dict(lengths=None), vq.VQ_ERR_NULL), (dict(page_table=None), vq.VQ_ERR_NULL),
    (dict(page_table=0x50002), vq.VQ_ERR_ALIGNMENT), (dict(lengths=0x51001), vq.VQ_ERR_ALIGNMENT), (dict(members=0x52002), vq.VQ_ERR_ALIGNMENT),
], ids=str)
def test_prefixes_that_are_refused(kw, status):
    assert _attend(prefix=_prefix(**kw)) == status
    assert vq.vq_attention_shared_workspace_bytes(_cache(), _prefix(**kw), 4) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(q_ptr=None), vq.VQ_ERR_NULL), (dict(out_ptr=None), vq.VQ_ERR_NULL), (dict(q_heads=3), vq.VQ_ERR_SHAPE), (dict(q_heads=0), vq.VQ_ERR_SHAPE),
    (dict(ldq=4 * DIM - 1), vq.VQ_ERR_SHAPE), (dict(ldo=0), vq.VQ_ERR_SHAPE), (dict(softmax_scale=0.0), vq.VQ_ERR_SHAPE), (dict(softmax_scale=float("nan")), vq.VQ_ERR_SHAPE),
    (dict(q_ptr=0x3001), vq.VQ_ERR_ALIGNMENT), (dict(out_ptr=0x4001), vq.VQ_ERR_ALIGNMENT), (dict(lse_ptr=0x6002), vq.VQ_ERR_ALIGNMENT),
    (dict(workspace_ptr=0x6080, workspace_bytes=256), vq.VQ_ERR_ALIGNMENT),
], ids=str)
def test_calls_that_are_refused(kw, status):
    assert _attend(**kw) == status


def test_missing_descriptors():
    assert vq.vq_attention_shared(None, _prefix(), 0x3000, 4 * DIM, 4, 0.1, 0x4000, 4 * DIM) == vq.VQ_ERR_NULL
    assert vq.vq_attention_shared(_cache(), None, 0x3000, 4 * DIM, 4, 0.1, 0x4000, 4 * DIM) == vq.VQ_ERR_NULL
    assert vq.load().vq_attention_shared_workspace_bytes(None, None, 4) == 0
    assert vq.vq_sample(0x1000, 8, 1, 8, 0x2000, None, 0x3000) == vq.VQ_ERR_NULL


@pytest.mark.parametrize("kw,status", [
    (dict(ids_ptr=None), vq.VQ_ERR_NULL), (dict(table_ptr=None), vq.VQ_ERR_NULL), (dict(y_ptr=None), vq.VQ_ERR_NULL), (dict(rows=0), vq.VQ_ERR_SHAPE), (dict(rows=-3), vq.VQ_ERR_SHAPE),
    (dict(vocabulary=0), vq.VQ_ERR_SHAPE), (dict(vocabulary=2 ** 24 + 1), vq.VQ_ERR_SHAPE), (dict(width=0), vq.VQ_ERR_SHAPE),
    (dict(width=2 ** 24 + 1, ld=2 ** 25, ldy=2 ** 25), vq.VQ_ERR_SHAPE), (dict(ld=63), vq.VQ_ERR_SHAPE), (dict(ldy=-64), vq.VQ_ERR_SHAPE),
    (dict(scale=float("inf")), vq.VQ_ERR_SHAPE), (dict(scale=float("nan")), vq.VQ_ERR_SHAPE),
    (dict(ids_ptr=0x1002), vq.VQ_ERR_ALIGNMENT), (dict(table_ptr=0x2001), vq.VQ_ERR_ALIGNMENT), (dict(y_ptr=0x3001), vq.VQ_ERR_ALIGNMENT),
    (dict(y_ptr=0x3002, stream32=1), vq.VQ_ERR_ALIGNMENT),
], ids=str)
def test_lookups_that_are_refused(kw, status):
    a = dict(ids_ptr=0x1000, rows=3, table_ptr=0x2000, ld=64, vocabulary=100, width=64, scale=1.0, stream32=0, y_ptr=0x3000, ldy=64)
    a.update(kw)
    assert vq.vq_embed(**a) == status


@pytest.mark.parametrize("kw,status", [
    (dict(logits_ptr=None), vq.VQ_ERR_NULL), (dict(uniform_ptr=None), vq.VQ_ERR_NULL), (dict(tokens_ptr=None), vq.VQ_ERR_NULL), (dict(rows=0), vq.VQ_ERR_SHAPE),
    (dict(vocabulary=0), vq.VQ_ERR_SHAPE), (dict(vocabulary=2 ** 24 + 1, ld=2 ** 25), vq.VQ_ERR_SHAPE), (dict(ld=99), vq.VQ_ERR_SHAPE), (dict(how=dict(struct_size=4)), vq.VQ_ERR_SHAPE),
    (dict(logits_ptr=0x1001), vq.VQ_ERR_ALIGNMENT), (dict(uniform_ptr=0x2002), vq.VQ_ERR_ALIGNMENT), (dict(tokens_ptr=0x3002), vq.VQ_ERR_ALIGNMENT),
    (dict(probabilities_ptr=0x4001), vq.VQ_ERR_ALIGNMENT), (dict(how=dict(temperatures=0x5002)), vq.VQ_ERR_ALIGNMENT), (dict(how=dict(top_ks=0x5001)), vq.VQ_ERR_ALIGNMENT),
    (dict(how=dict(top_ps=0x5002)), vq.VQ_ERR_ALIGNMENT), (dict(how=dict(min_ps=0x5003)), vq.VQ_ERR_ALIGNMENT),
], ids=str)
def test_samples_that_are_refused(kw, status):
    how = vq.vq_sampling(**dict(dict(struct_size=ctypes.sizeof(vq.vq_sampling), top_k=0, temperature=1.0, top_p=1.0, min_p=0.0), **kw.pop("how", {})))
    a = dict(logits_ptr=0x1000, ld=100, rows=2, vocabulary=100, uniform_ptr=0x2000, how=how, tokens_ptr=0x3000)
    a.update(kw)
    assert vq.vq_sample(**a) == status
