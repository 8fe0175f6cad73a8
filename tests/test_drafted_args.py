"""Refusals of the operators of a decode step with drafted tokens: every one is decided on the host, before anything is launched, so
made-up aligned addresses will do."""
import ctypes as C

import pytest

from paper_2509_22951_b200 import binding as tq

A = 1 << 20  # an aligned address that is never followed
lib = tq._lib
CACHE = dict(d_k=A, d_v=A, n_pages=4, page_size=16, n_kv_heads=2, head_dim=64, page_stride=2048, head_stride=1024, slot_stride=64, d_status=None)
BAD_CACHES = [(dict(d_k=None), -1), (dict(d_v=A + 8), -1), (dict(n_pages=0), -1), (dict(page_size=0), -1), (dict(slot_stride=-64), -1),
              (dict(d_status=A + 1), -1), (dict(head_dim=96), -4), (dict(n_pages=1 << 31), -4)]


def _cache(**change):
    return tq._KvCache(**dict(CACHE, **change))


def _ws_bytes():
    n = C.c_uint64()
    assert lib.tq_attn_workspace_size(C.byref(n)) == tq.TQ_OK
    return n.value


HEADS = dict(q=A, k=A, v=A, xt=1, qs=256, ks=128, vs=128, T=3, H=4, qw=A, kw=A, eps=1e-5, table=A, n_pos=10, rot=64, pos=A, sec=(32,), inter=0, slots=A, out=A)


def _heads(cache, **change):
    a = dict(HEADS, **change)
    sec = None if a["sec"] is None else (C.c_uint32 * max(1, len(a["sec"])))(*a["sec"])
    return lib.tq_qk_norm_rope_append(a["q"], a["k"], a["v"], a["xt"], a["qs"], a["ks"], a["vs"], a["T"], a["H"], a["qw"], a["kw"], a["eps"], a["table"],
                                      a["n_pos"], a["rot"], a["pos"], sec, 0 if a["sec"] is None else len(a["sec"]), a["inter"], a["slots"],
                                      None if cache is None else C.byref(cache), a["out"], None)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), -1), (dict(k=A + 8), -1), (dict(v=None), -1), (dict(qw=None), -1), (dict(kw=A + 2), -1), (dict(eps=-1e-5), -1),
    (dict(eps=float("nan")), -1), (dict(table=None), -1), (dict(pos=None), -1), (dict(slots=A + 2), -1), (dict(out=None), -1), (dict(xt=3), -1),
    (dict(qs=252), -1), (dict(H=0), -1), (dict(n_pos=0), -1), (dict(rot=72, sec=(36,)), -1), (dict(sec=(31,)), -1), (dict(sec=None), -1),
    (dict(T=0), 0), (dict(T=0, qw=None, kw=None), 0),
])
def test_qk_norm_rope_append(change, status):
    assert _heads(_cache(), **change) == status


TREE = dict(q=A, qs=256, T=9, B=2, H=4, first=A, table=A, max_pages=8, lens=A, mask=None, words=0, scale=0.125, out=A, lse=None, ws=A, short=0)


def _tree(cache, **change):
    a = dict(TREE, **change)
    return lib.tq_tree_attention(None if cache is None else C.byref(cache), a["q"], a["qs"], a["T"], a["B"], a["H"], a["first"], a["table"], a["max_pages"],
                                 a["lens"], a["mask"], a["words"], a["scale"], a["out"], a["lse"], a["ws"], _ws_bytes() - a["short"], None)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), -1), (dict(q=A + 8), -1), (dict(qs=4), -1), (dict(H=0), -1), (dict(H=5), -1), (dict(first=None), -1), (dict(first=A + 2), -1),
    (dict(table=None), -1), (dict(max_pages=0), -1), (dict(lens=None), -1), (dict(mask=A), -1), (dict(mask=A + 1, words=1), -1), (dict(out=A + 2), -1),
    (dict(lse=A + 1), -1), (dict(ws=None), -1), (dict(ws=A + 16), -1), (dict(short=1), -3), (dict(scale=0.0), -1), (dict(scale=float("nan")), -1),
    (dict(scale=float("inf")), -1), (dict(T=1 << 30), -4), (dict(T=1 << 24, max_pages=1 << 27), -4), (dict(B=0), 0), (dict(T=0), 0),
])
def test_tree_attention(change, status):
    assert _tree(_cache(), **change) == status


SAMPLE = dict(x=A, xt=1, stride=100, rows=3, vocab=100, u=A, t=None, k=None, p=None, m=None, out=A, lp=None)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), -1), (dict(x=A + 2), -1), (dict(x=A + 1, xt=0), -1), (dict(xt=2), -1), (dict(vocab=0), -1), (dict(vocab=tq.TQ_SAMPLE_MAX_VOCAB + 1), -4),
    (dict(u=None), -1), (dict(u=A + 1), -1), (dict(t=A + 2), -1), (dict(k=A + 1), -1), (dict(p=A + 2), -1), (dict(m=A + 3), -1), (dict(out=None), -1),
    (dict(out=A + 2), -1), (dict(lp=A + 1), -1), (dict(rows=0), 0), (dict(rows=0, x=None, u=None, out=None), 0), (dict(rows=1 << 31, vocab=1 << 15), -4),
])
def test_sample(change, status):
    a = dict(SAMPLE, **change)
    assert lib.tq_sample(a["x"], a["xt"], a["stride"], a["rows"], a["vocab"], a["u"], a["t"], a["k"], a["p"], a["m"], a["out"], a["lp"], None) == status


ACCEPT = dict(n=None, table=A, max_pages=8, B=2, T=9, first=A, lens=A + 64, tokens=A, parents=A, sampled=A, max_path=4, out=A, path=A, count=A, lens_out=A)


def _accept(caches, **change):
    a = dict(ACCEPT, **change)
    n = len(caches) if a["n"] is None else a["n"]
    return lib.tq_tree_accept((tq._KvCache * len(caches))(*caches) if caches else None, n, a["table"], a["max_pages"], a["B"], a["T"], a["first"], a["lens"],
                              a["tokens"], a["parents"], a["sampled"], a["max_path"], a["out"], a["path"], a["count"], a["lens_out"], None)


@pytest.mark.parametrize("change,status", [
    (dict(table=None), -1), (dict(max_pages=0), -1), (dict(first=None), -1), (dict(lens=A + 1), -1), (dict(tokens=None), -1), (dict(parents=None), -1),
    (dict(sampled=A + 2), -1), (dict(max_path=0), -1), (dict(max_path=tq.TQ_TREE_MAX_PATH + 1), -4), (dict(out=None), -1), (dict(path=None), -1),
    (dict(count=A + 1), -1), (dict(lens_out=None), -1), (dict(lens_out=A + 64), -1), (dict(T=1 << 31), -4), (dict(B=0), 0),
])
def test_tree_accept(change, status):
    assert _accept([_cache(), _cache(d_k=A + 32)], **change) == status


def test_tree_accept_wants_caches_that_are_alike():
    for change in (dict(n_pages=5), dict(page_size=8), dict(n_kv_heads=1), dict(head_dim=128), dict(page_stride=4096), dict(head_stride=2048), dict(slot_stride=128)):
        assert _accept([_cache(), _cache(**change)]) == -1
    assert _accept([_cache()] * (tq.TQ_MAX_CACHES + 1)) == -4
    assert _accept([], n=1) == -1


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_caches(change, status):
    c = _cache(**change)
    assert _heads(c) == status and _tree(c) == status and _accept([c]) == status


def test_no_cache():
    assert _heads(None) == -1 and _tree(None) == -1
