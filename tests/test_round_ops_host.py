"""What the entry points around a speculation round refuse on the host, before anything is launched (no GPU needed: the
pointers are never followed)."""
import ctypes

import pytest

from paper_2607_27735_b200 import binding

P = 1 << 20  # an aligned address that nothing reads
INVALID, SHAPE, SMALL = -1, -2, -3


def _kv(**kw):
    d = dict(k=P, v=P, layer_stride=1 << 20, page_stride=4096, head_stride=2048, slot_stride=128, n_layers=1, page_size=16, page_table=None,
             max_pages=4, batch=1, n_q_heads=8, n_kv_heads=2, head_dim=128, n_pages=4, sm_scale=0.0, kv_dtype=0, k_scale=None, v_scale=None)
    d.update(kw)
    return ctypes.byref(binding._KV(*(d[n] for n, _ in binding._KV._fields_)))


def _pages(**kw):
    d = dict(first=P, new=P, batch=2, ps=16, table=P, max_pages=4, held=P, pool=P, n_pages=8, n_free=P, max_rows=4, cu=P, pos=P, slots=P,
             ws=P, bytes=4096)
    d.update(kw)
    return binding.load().spec_assign_pages(*d.values(), None)


@pytest.mark.parametrize("change,code", [
    (dict(batch=-1), INVALID), (dict(ps=0), INVALID), (dict(max_pages=0), INVALID), (dict(n_pages=0), INVALID), (dict(max_rows=-1), INVALID),
    (dict(first=None), INVALID), (dict(new=None), INVALID), (dict(table=None), INVALID), (dict(held=None), INVALID),
    (dict(pool=None), INVALID), (dict(n_free=None), INVALID), (dict(cu=None), INVALID), (dict(pos=None), INVALID),
    (dict(slots=None), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 16), INVALID), (dict(bytes=511), SMALL),
    (dict(n_pages=1 << 27), SHAPE), (dict(batch=2048, max_pages=1 << 20), SHAPE), (dict(batch=2049), SHAPE),
])
def test_assign_pages_refuses(change, code):
    assert _pages(**change) == code


def _append(kv=None, **kw):
    d = dict(q=P, ql=0, qr=1024, k=P, kl=0, kr=256, v=P, vl=0, vr=256, n=3, pos=P, slots=P, qw=None, kw=None, eps=1e-6, cs=P, max_pos=9,
             rot=128, out=P, ws=P, bytes=256, flags=0)
    d.update(kw)
    return binding.load().spec_qkv_append(kv or _kv(), *d.values(), None)


@pytest.mark.parametrize("change,code", [
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(slots=None), INVALID),
    (dict(pos=None), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 128), INVALID), (dict(bytes=255), SMALL), (dict(n=-1), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(q=P + 8), INVALID), (dict(kw=P + 2), INVALID), (dict(out=P + 4), INVALID),
    (dict(cs=P + 4), INVALID), (dict(qr=1025), INVALID), (dict(vr=-256), INVALID), (dict(rot=8), INVALID), (dict(rot=136), INVALID),
    (dict(rot=40), INVALID), (dict(max_pos=0), INVALID), (dict(flags=2), INVALID),
])
def test_qkv_append_refuses(change, code):
    assert _append(**change) == code


@pytest.mark.parametrize("change,code", [
    (dict(head_dim=96), SHAPE), (dict(kv_dtype=3), INVALID), (dict(kv_dtype=2), INVALID), (dict(kv_dtype=2, k_scale=P), INVALID),
    (dict(head_stride=0), INVALID), (dict(page_stride=0), INVALID), (dict(n_layers=2, layer_stride=0), INVALID),
    (dict(n_pages=1 << 28), SHAPE), (dict(slot_stride=64), INVALID), (dict(kv_dtype=1, head_stride=2056), INVALID),
])
def test_qkv_append_refuses_the_cache(change, code):
    assert _append(_kv(**change)) == code


def test_page_scales_need_room_for_the_rows():
    assert _append(_kv(kv_dtype=2, k_scale=P, v_scale=P), bytes=256 + 47) == SMALL


def test_no_rows_is_nothing_to_do():
    assert _append(n=0) == 0


@pytest.mark.parametrize("change,code", [
    (dict(logits=None), INVALID), (dict(out=None), INVALID), (dict(dtype=2), INVALID), (dict(rows=-1), INVALID), (dict(vocab=0), INVALID),
    (dict(stride=99), INVALID), (dict(out_stride=99), INVALID), (dict(rows=65536), SHAPE), (dict(rows=0), 0),
    (dict(vocab=(1 << 30) + 1, stride=1 << 31, out_stride=1 << 31), SHAPE),
])
def test_token_probs_refuses(change, code):
    d = dict(logits=P, dtype=1, rows=2, vocab=100, stride=100, temp=None, out=P, out_stride=100)
    d.update(change)
    assert binding.load().spec_token_probs(*d.values(), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(p=None), INVALID), (dict(u=None), INVALID), (dict(n=None), INVALID), (dict(token=None), INVALID), (dict(draft=None), INVALID),
    (dict(batch=-1), INVALID), (dict(k1=0), INVALID), (dict(vocab=0), INVALID), (dict(pr=-1), INVALID), (dict(qb=-1), INVALID),
    (dict(batch=65536), SHAPE), (dict(batch=0), 0), (dict(vocab=(1 << 30) + 1), SHAPE),
])
def test_accept_sample_refuses(change, code):
    d = dict(p=P, pb=300, pr=100, q=P, qb=200, qr=100, draft=P, nd=None, u=P, batch=2, k1=3, vocab=100, n=P, token=P)
    d.update(change)
    assert binding.load().spec_accept_sample(*d.values(), None) == code


def test_workspaces_and_the_new_code():
    assert binding.pages_workspace_bytes() == 512 and binding.append_workspace_bytes() == 256 + (1 << 20)
    size = binding.load().spec_workspace_bytes
    assert size(binding.WS_APPEND, _kv(), 1000, 0, 0) == 256
    assert size(binding.WS_APPEND, _kv(kv_dtype=2, k_scale=P, v_scale=P, n_layers=3), 1000, 0, 0) == 256 + 2 * 3 * 1000 * 8
    assert size(binding.WS_APPEND, _kv(), -1, 0, 0) == 0
    assert binding.strerror(-7) == "too few free pages"
