"""Refusals of the paged-cache operators (no GPU): the binding's checks before a
pointer is taken, and the C ABI's own before any launch."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

import paper_2406_13868_amd as sdq  # noqa: E402
from paper_2406_13868_amd import _lib  # noqa: E402

P = 1 << 20  # stands for a device pointer in calls that are refused before it is used


def _cache(**kw):
    f = dict(k=P, v=P, k_scale=None, v_scale=None, position=None, weight=None, pages=10, page_stride=8 * 16 * 64, head_stride=16 * 64,
             slot_stride=64, dtype=_lib.DTYPE_BF16, heads=8, page_size=16, dim=64)
    return _lib.sdq_kv_cache(**(f | kw))


def _append(t=None, qkv=P, x=0, M=1, ld=24 * 64, pos=P, slot=P, out=P, qd=0, **kw):
    f = dict(qkv=qkv, pos=pos, slot=slot, q_out=out, q_weight=None, k_weight=None, cos_sin=P, M=M, row_stride=ld, positions=10, x_dtype=x,
             q_dtype=qd, heads_q=8, rot_dim=64, interleaved=0, eps=1e-6)
    return _lib.lib().sdq_qkv_append(C.byref(_cache(**kw)), C.byref(_lib.sdq_append_args(**(f | (t or {})))), None)


def _attend(q=P, qt=0, B=2, hq=8, qs=8 * 64, table=P, ts=4, mp=4, lens=P, max_len=64, scale=1.0, out=P, lse=None, w=None, ws=P,
            nbytes=1 << 40, **kw):
    t = _lib.sdq_attn_args(q=q, page_table=table, seq_lens=lens, out=out, lse=lse, weight_out=w, workspace=ws, ws_bytes=nbytes, B=B,
                           q_stride=qs, table_stride=ts, max_pages=mp, max_len=max_len, dtype=qt, heads_q=hq, scale=scale)
    return _lib.lib().sdq_attn_decode(C.byref(_cache(**kw)), C.byref(t), None)


def _evict(B=2, table=P, ts=4, mp=4, lens=P, max_len=64, budget=8, recent=2, lo=P, po=P, wo=P, ws=P, nbytes=1 << 40, **kw):
    t = _lib.sdq_evict_args(page_table=table, seq_lens=lens, lens_out=lo, position_out=po, weight_out=wo, workspace=ws, ws_bytes=nbytes,
                            B=B, table_stride=ts, max_pages=mp, max_len=max_len, budget=budget, recent=recent)
    return _lib.lib().sdq_cache_evict(C.byref(_cache(**(dict(position=P, weight=P) | kw))), C.byref(t), None)


def test_null_arguments():
    L, c = _lib.lib(), C.byref(_cache(position=P, weight=P))
    for f in (L.sdq_qkv_append, L.sdq_attn_decode, L.sdq_cache_evict):
        assert f(c, None, None) == NULL and f(None, None, None) == NULL


NULL, SHAPE, CONFIG, SMALL, VALUE = -1, -2, -3, -4, -7


@pytest.mark.parametrize("kw, status", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(dtype=0), CONFIG), (dict(dtype=2), NULL), (dict(dtype=2, k_scale=P), NULL),
    (dict(heads=0), SHAPE), (dict(heads=1025), SHAPE), (dict(dim=8), SHAPE), (dict(dim=72), SHAPE), (dict(dim=272), SHAPE),
    (dict(page_size=0), SHAPE), (dict(page_size=1 << 21), SHAPE), (dict(pages=0), SHAPE), (dict(pages=1 << 28), SHAPE),
    (dict(k=P + 8), SHAPE), (dict(slot_stride=68), SHAPE), (dict(head_stride=-64), SHAPE), (dict(page_stride=1 << 41), SHAPE),
])
def test_caches(kw, status):
    assert _append(**kw) == status and _attend(**kw) == status and _evict(**kw) == status
    n = C.c_size_t()
    assert _lib.lib().sdq_attn_decode_workspace_size(C.byref(_cache(**kw)), 1, 8, 64, 0, C.byref(n)) == status
    assert _lib.lib().sdq_cache_evict_workspace_size(C.byref(_cache(**kw)), 1, 64, 8, C.byref(n)) == status


@pytest.mark.parametrize("kw, status", [
    (dict(x=2), CONFIG), (dict(qd=2), CONFIG), (dict(t=dict(rot_dim=63)), CONFIG), (dict(t=dict(rot_dim=66)), CONFIG),
    (dict(t=dict(rot_dim=-2)), CONFIG), (dict(t=dict(interleaved=2)), CONFIG), (dict(t=dict(q_weight=P)), CONFIG),
    (dict(t=dict(q_weight=P, k_weight=P, eps=-1.0)), CONFIG), (dict(t=dict(q_weight=P, k_weight=P, eps=float("nan"))), CONFIG),
    (dict(t=dict(heads_q=0)), SHAPE), (dict(t=dict(heads_q=12)), SHAPE), (dict(t=dict(positions=-1)), SHAPE), (dict(M=-1), SHAPE),
    (dict(M=1 << 26), SHAPE), (dict(ld=24 * 64 - 16), SHAPE), (dict(ld=24 * 64 + 2), SHAPE), (dict(qkv=None), NULL), (dict(slot=None), NULL),
    (dict(out=None), NULL), (dict(pos=None), NULL), (dict(t=dict(cos_sin=None)), NULL), (dict(t=dict(rot_dim=0), position=P, pos=None), NULL),
    (dict(qkv=P + 4), SHAPE), (dict(out=P + 4), SHAPE), (dict(t=dict(cos_sin=P + 4)), SHAPE), (dict(t=dict(q_weight=P + 4, k_weight=P)), SHAPE),
    (dict(M=0, qkv=None, slot=None, out=None), 0),
])
def test_append(kw, status):
    assert _append(**kw) == status


@pytest.mark.parametrize("kw, status", [
    (dict(qt=2), CONFIG), (dict(B=-1), SHAPE), (dict(B=(1 << 20) + 1), SHAPE), (dict(max_len=-1), SHAPE), (dict(mp=-1), SHAPE),
    (dict(ts=-1), SHAPE), (dict(hq=0), SHAPE), (dict(hq=12), SHAPE), (dict(hq=1032), SHAPE), (dict(qs=8 * 64 - 16), SHAPE),
    (dict(qs=8 * 64 + 2), SHAPE), (dict(lens=None), NULL), (dict(table=None), NULL), (dict(q=None), NULL), (dict(out=None), NULL),
    (dict(ws=None), NULL), (dict(w=P), NULL), (dict(scale=float("inf")), VALUE), (dict(q=P + 4), SHAPE), (dict(out=P + 4), SHAPE),
    (dict(ws=P + 4), SHAPE), (dict(nbytes=100), SMALL), (dict(B=1 << 20, mp=1 << 20, max_len=1 << 24), SHAPE),
    (dict(B=0, q=None, table=None, lens=None), 0),
])
def test_attend(kw, status):
    assert _attend(**kw) == status


@pytest.mark.parametrize("kw, status", [
    (dict(position=None), NULL), (dict(weight=None), NULL), (dict(B=-1), SHAPE), (dict(budget=0), SHAPE), (dict(recent=-1), SHAPE),
    (dict(recent=9), SHAPE), (dict(lo=None), NULL), (dict(po=None), NULL), (dict(wo=None), NULL), (dict(ws=None), NULL),
    (dict(lens=None), NULL), (dict(table=None), NULL), (dict(wo=2 * P), CONFIG), (dict(po=2 * P), CONFIG), (dict(ws=P + 4), SHAPE),
    (dict(nbytes=64), SMALL), (dict(B=0, table=None, lens=None, lo=None), 0),
])
def test_evict(kw, status):
    assert _evict(**kw) == status


def test_workspace_sizes():
    c, n = _cache(), C.c_size_t()
    L = _lib.lib()
    assert L.sdq_attn_decode_workspace_size(C.byref(c), 2, 8, 64, 0, C.byref(n)) == 0 and n.value > 0
    plain = n.value
    assert L.sdq_attn_decode_workspace_size(C.byref(c), 2, 8, 64, 1, C.byref(n)) == 0 and n.value >= plain + 2 * 8 * 64 * 4
    assert L.sdq_attn_decode_workspace_size(C.byref(c), 2, 8, 64, 0, None) == NULL
    assert L.sdq_attn_decode_workspace_size(C.byref(c), 2, 12, 64, 0, C.byref(n)) == SHAPE
    assert L.sdq_cache_evict_workspace_size(C.byref(c), 2, 64, 0, C.byref(n)) == SHAPE
    assert L.sdq_cache_evict_workspace_size(C.byref(c), 2, 64, 8, None) == NULL


def _raises(fn, match):
    with pytest.raises(ValueError, match=match):
        fn()


def test_the_binding_checks_the_cache():
    k = torch.zeros((4, 2, 8, 32), dtype=torch.bfloat16)
    f8 = torch.zeros((4, 2, 8, 32), dtype=torch.float8_e4m3fn)
    s = torch.zeros((4, 2, 8))
    _raises(lambda: sdq.KVCache(k[0], k[0]), "k must be a")
    _raises(lambda: sdq.KVCache(k.float(), k.float()), "bfloat16 or float8")
    _raises(lambda: sdq.KVCache(k, f8), "v must be")
    _raises(lambda: sdq.KVCache(k, k[:3]), "v must be")
    _raises(lambda: sdq.KVCache(k, torch.zeros((4, 8, 2, 32), dtype=torch.bfloat16).transpose(1, 2)), "same strides")
    t = torch.zeros((4, 2, 32, 8), dtype=torch.bfloat16).transpose(2, 3)
    _raises(lambda: sdq.KVCache(t, t), "contiguous")
    e = torch.zeros((1, 2, 8, 32), dtype=torch.bfloat16).expand(4, 2, 8, 32)
    _raises(lambda: sdq.KVCache(e, e), "overlap")
    _raises(lambda: sdq.KVCache(k[:0], k[:0]), "at least one")
    _raises(lambda: sdq.KVCache(k, k, s, s), "belong to an e4m3")
    _raises(lambda: sdq.KVCache(f8, f8), "belong to an e4m3")
    _raises(lambda: sdq.KVCache(f8, f8, s[:3], s), "k_scale must be")
    _raises(lambda: sdq.KVCache(k, k, position=s), "position must be")
    _raises(lambda: sdq.KVCache(k, k, weight=s.double()), "weight must be")
    _raises(lambda: sdq.KVCache(k, k), "CUDA")
    _raises(lambda: sdq.KVCache.empty(1, 1, 1, 16, "f16"), "dtype must be")


class _Stub:
    """A cache as the calls see it, without a GPU."""
    pages, heads, page_size, dim, device = 4, 2, 8, 32, torch.device("cpu")
    k = v = torch.zeros((4, 2, 8, 32), dtype=torch.bfloat16)
    k_scale = v_scale = position = weight = None
    _index = -1


def test_the_binding_checks_the_calls():
    c = _Stub()
    qkv, slot = torch.zeros((3, 8 * 32)), torch.zeros(3, dtype=torch.int64)
    _raises(lambda: sdq.qkv_append(qkv[:, :-1], None, slot, c, 4), "qkv must be")
    _raises(lambda: sdq.qkv_append(qkv, None, slot, c, 5), "qkv must be")
    _raises(lambda: sdq.qkv_append(qkv, None, slot, c, 4), "CUDA")
    table, lens = torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    q = torch.zeros((3, 4, 32))
    _raises(lambda: sdq.attn_decode(q, c, table.long(), lens), "page_table must be")
    _raises(lambda: sdq.attn_decode(q, c, table[0], lens), "page_table must be")
    _raises(lambda: sdq.attn_decode(q, c, table, lens[:2]), "seq_lens must be")
    _raises(lambda: sdq.attn_decode(q, c, table, lens), "CUDA")
    _raises(lambda: sdq.cache_evict(c, table, lens.long(), 4), "seq_lens must be")


OK = 0


@pytest.mark.parametrize("B,heads,heads_q,max_len,track,status", [
    (1 << 20, 8, 8, 64, 0, OK), (1 << 20, 16, 16, 64, 0, SHAPE), ((1 << 20) + 1, 1, 1, 64, 0, SHAPE),
    (4096, 32, 32, 100000, 0, OK), (4096, 32, 32, 100000, 1, OK), (4096, 32, 32, 131072, 1, SHAPE),
    (1 << 14, 32, 32, 1 << 20, 0, SHAPE),
])
def test_attention_counts_that_no_launch_holds_are_refused(B, heads, heads_q, max_len, track, status):
    n = C.c_size_t()
    c = _cache(heads=heads)
    assert _lib.lib().sdq_attn_decode_workspace_size(C.byref(c), B, heads_q, max_len, track, C.byref(n)) == status


@pytest.mark.parametrize("B,heads,status", [(1 << 20, 3, OK), (1 << 20, 4, SHAPE), (4096, 1023, OK), (4096, 1024, SHAPE)])
def test_eviction_counts_that_no_launch_holds_are_refused(B, heads, status):
    n = C.c_size_t()
    c = _cache(heads=heads)
    assert _lib.lib().sdq_cache_evict_workspace_size(C.byref(c), B, 64, 8, C.byref(n)) == status
