"""Refusals of the operators between the linear layers: every one is decided on the host, before anything is
launched, so made-up aligned addresses will do."""
import ctypes as C

import pytest

from paper_2509_22951_b200 import binding as tq

A = 1 << 20  # an aligned address that is never followed
lib = tq._lib


def _ws_bytes():
    n = C.c_uint64()
    assert lib.tq_attn_workspace_size(C.byref(n)) == tq.TQ_OK
    return n.value


NORM = dict(h=A, ht=0, hs=64, d=A, dt=1, ds=64, w=A, eps=1e-5, rows=4, cols=64, ho=A, out=A)


@pytest.mark.parametrize("change,status", [
    (dict(h=None), -1), (dict(w=None), -1), (dict(out=None), -1), (dict(ht=2), -1), (dict(dt=7), -1), (dict(cols=0), -1),
    (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(h=A + 1), -1), (dict(w=A + 2), -1), (dict(d=A + 2), -1), (dict(ho=A + 1), -1),
    (dict(out=A + 1), -1), (dict(hs=63), -1), (dict(ds=63), -1), (dict(cols=tq.TQ_NORM_MAX_COLS + 1, hs=1 << 20, ds=1 << 20), -4),
    (dict(rows=0), 0), (dict(rows=0, h=None, w=None, out=None), 0),
])
def test_rmsnorm(change, status):
    a = dict(NORM, **change)
    head = (a["h"], a["ht"], a["hs"], a["d"], a["dt"], a["ds"], a["w"], a["eps"], a["rows"], a["cols"], a["ho"])
    assert lib.tq_rmsnorm(*head, a["out"], None) == status
    if "out" not in change or a["out"] is None:  # 8-bit levels have no alignment
        assert lib.tq_rmsnorm_q8(*head, a["out"], a["out"], None) == status


def test_rmsnorm_q8_wants_its_scales():
    a = NORM
    head = (a["h"], a["ht"], a["hs"], None, 0, 0, a["w"], a["eps"], a["rows"], a["cols"], None)
    assert lib.tq_rmsnorm_q8(*head, A, None, None) == -1
    assert lib.tq_rmsnorm_q8(*head, None, A, None) == -1
    assert lib.tq_rmsnorm_q8(*head, A, A + 2, None) == -1


CACHE = dict(d_k=A, d_v=A, n_pages=4, page_size=16, n_kv_heads=2, head_dim=64, page_stride=2048, head_stride=1024, slot_stride=64, d_status=None)
BAD_CACHES = [
    (dict(d_k=None), -1), (dict(d_v=A + 8), -1), (dict(n_pages=0), -1), (dict(page_size=0), -1), (dict(n_kv_heads=0), -1),
    (dict(page_stride=2047), -1), (dict(head_stride=1), -1), (dict(slot_stride=-64), -1), (dict(d_status=A + 1), -1),
    (dict(head_dim=96), -4), (dict(head_dim=256), -4), (dict(n_pages=1 << 31), -4),
]


def _cache(**change):
    return tq._KvCache(**dict(CACHE, **change))


ROPE = dict(q=A, k=A, v=A, xt=1, qs=256, ks=128, vs=128, T=3, H=4, table=A, n_pos=10, rot=64, pos=A, sec=(32,), inter=0, slots=A, out=A)


def _rope(cache, **change):
    a = dict(ROPE, **change)
    sec = None if a["sec"] is None else (C.c_uint32 * max(1, len(a["sec"])))(*a["sec"])
    n = a.get("axes", 0 if a["sec"] is None else len(a["sec"]))
    return lib.tq_rope_append(a["q"], a["k"], a["v"], a["xt"], a["qs"], a["ks"], a["vs"], a["T"], a["H"], a["table"], a["n_pos"], a["rot"], a["pos"],
                              sec, n, a["inter"], a["slots"], None if cache is None else C.byref(cache), a["out"], None)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), -1), (dict(k=A + 8), -1), (dict(v=None), -1), (dict(table=None), -1), (dict(pos=None), -1), (dict(slots=A + 2), -1),
    (dict(out=None), -1), (dict(xt=3), -1), (dict(qs=252), -1), (dict(ks=4), -1), (dict(vs=1), -1), (dict(H=0), -1), (dict(n_pos=0), -1),
    (dict(rot=0, sec=(0,)), -1), (dict(rot=60, sec=(30,)), -1), (dict(rot=72, sec=(36,)), -1), (dict(sec=(31,)), -1), (dict(sec=(16, 17)), -1),
    (dict(sec=()), -1), (dict(sec=None), -1), (dict(sec=(8, 8, 8, 8)), -1), (dict(T=0), 0),
])
def test_rope_append(change, status):
    assert _rope(_cache(), **change) == status


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_caches(change, status):
    c = _cache(**change)
    assert _rope(c) == status
    assert lib.tq_paged_attention(C.byref(c), A, 256, 2, 4, A, 8, A, 1.0, A, None, A, _ws_bytes(), None) == status


def test_no_cache():
    assert _rope(None) == -1
    assert lib.tq_paged_attention(None, A, 256, 2, 4, A, 8, A, 1.0, A, None, A, _ws_bytes(), None) == -1


PAGED = dict(scale=0.125, q=A, qs=256, B=2, H=4, table=A, max_pages=8, lens=A, out=A, lse=None, ws=A, short=0)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), -1), (dict(q=A + 8), -1), (dict(qs=4), -1), (dict(H=0), -1), (dict(H=5), -1), (dict(table=None), -1), (dict(max_pages=0), -1),
    (dict(lens=None), -1), (dict(out=A + 2), -1), (dict(lse=A + 1), -1), (dict(ws=None), -1), (dict(ws=A + 16), -1), (dict(short=1), -3), (dict(B=0), 0),
    (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1),
])
def test_paged_attention(change, status):
    a, c = dict(PAGED, **change), _cache()
    assert lib.tq_paged_attention(C.byref(c), a["q"], a["qs"], a["B"], a["H"], a["table"], a["max_pages"], a["lens"], a["scale"], a["out"], a["lse"], a["ws"],
                                  _ws_bytes() - a["short"], None) == status


KV = dict(d_k=A, d_v=A, n_seqs=2, n_states=100, n_kv_heads=2, head_dim=64, batch_stride=12800, state_stride=128, head_stride=64)
CROSS = dict(scale=0.125, q=A, qb=1024, qt=256, T=4, H=4, kv_len=None, mask=None, block=0, out=A, lse=None, ws=A, short=0)


@pytest.mark.parametrize("kv,change,status", [
    (dict(d_k=None), {}, -1), (dict(d_v=A + 8), {}, -1), (dict(n_kv_heads=0), {}, -1), (dict(batch_stride=4), {}, -1), (dict(state_stride=-128), {}, -1),
    (dict(head_stride=1), {}, -1), (dict(head_dim=80), {}, -4), (dict(n_states=1 << 31), {}, -4), (dict(n_seqs=0), {}, 0),
    ({}, dict(q=None), -1), ({}, dict(q=A + 8), -1), ({}, dict(qb=4), -1), ({}, dict(qt=4), -1), ({}, dict(H=3), -1), ({}, dict(H=0), -1),
    ({}, dict(kv_len=A + 1), -1), ({}, dict(mask=A), -1), ({}, dict(out=None), -1), ({}, dict(lse=A + 2), -1), ({}, dict(ws=None), -1),
    ({}, dict(short=1), -3), ({}, dict(T=0), 0), ({}, dict(T=1 << 30, H=4), -4),
    ({}, dict(scale=0.0), -1), ({}, dict(scale=float("nan")), -1),
])
def test_cross_attention(kv, change, status):
    a, e = dict(CROSS, **change), tq._EncoderKv(**dict(KV, **kv))
    assert lib.tq_cross_attention(C.byref(e), a["q"], a["qb"], a["qt"], a["T"], a["H"], a["kv_len"], a["mask"], a["block"], a["scale"], a["out"], a["lse"],
                                  a["ws"], _ws_bytes() - a["short"], None) == status


def test_workspace_arguments():
    assert lib.tq_attn_workspace_size(None) == -1
    assert lib.tq_attn_workspace_init(None, _ws_bytes(), None) == -1
    assert lib.tq_attn_workspace_init(A + 16, _ws_bytes(), None) == -1
    assert lib.tq_attn_workspace_init(A, _ws_bytes() - 1, None) == -3
    st = C.c_uint32()
    assert lib.tq_attn_status(None, None, C.byref(st)) == -1 and lib.tq_attn_status(A, None, None) == -1
