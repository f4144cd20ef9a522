"""What the calls that share a paged cache and keep it within bounds refuse, on the host (no GPU needed: nothing is launched)."""
import ctypes

import pytest
import torch

from tests.test_paged_refusals import INVALID, L, ODD, OK, P, SHAPES, UNSUPPORTED, WORKSPACE, pages  # noqa: F401

MISALIGNED4, P2 = ctypes.c_void_p(4096 + 4), ctypes.c_void_p(8192)


def ref(s):
    return ctypes.byref(s) if s is not None else None


def append_at(L, s, **kw):
    a = dict(q=P, qs=8 * 128, k=P, ks=2 * 128, v=P, vs=2 * 128, n=2, off=P, len=P, table=P, rope=P, position=P, n_axes=3, axis=P, q_out=P,
             kp=P, vp=P, k_scale=None, v_scale=None)
    a.update(kw)
    return L.binding._lib.kv_page_append_at(ref(s), a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["n"], a["off"], a["len"], a["table"],
                                            a["rope"], a["position"], a["n_axes"], a["axis"], a["q_out"], a["kp"], a["vp"], a["k_scale"],
                                            a["v_scale"], None, None, None, None, None)


def shared(L, s, **kw):
    a = dict(q=P, kp=P, vp=P, ks=None, vs=None, table=P, len=P, n=1, off=P, pages=P, out=P, lse=None, ws=P, nbytes=1 << 40)
    a.update(kw)
    return L.binding._lib.page_attention_decode_shared(ref(s), a["q"], a["kp"], a["vp"], a["ks"], a["vs"], a["table"], a["len"], a["n"], a["off"],
                                                       a["pages"], 1.0, a["out"], a["lse"], a["ws"], a["nbytes"], None)


def weigh(L, s, **kw):
    a = dict(q=P, n=2, off=P, kp=P, ks=None, table=P, len=P, lse=P, before=None, weight=P, seen=P, ids=P)
    a.update(kw)
    return L.binding._lib.page_weight_add(ref(s), a["q"], a["n"], a["off"], a["kp"], a["ks"], a["table"], a["len"], 1.0, a["lse"], 1.0,
                                          a["before"], a["weight"], a["seen"], a["ids"], None)


def select(L, s, **kw):
    a = dict(weight=P, ids=P, seen=P, len=P, keep=P, first=None, recent=0, moves=P, m_max=4, count=P, new=P2, status=None, ws=P, nbytes=1 << 40)
    a.update(kw)
    return L.binding._lib.page_evict_select(ref(s), a["weight"], a["ids"], a["seen"], a["len"], a["keep"], a["first"], a["recent"], a["moves"],
                                            a["m_max"], a["count"], a["new"], a["status"], a["ws"], a["nbytes"], None)


def move(L, s, **kw):
    a = dict(moves=P, m_max=4, count=P, old=P, new=P, table=P, kp=P, vp=P, ks=None, vs=None, weight=None, ids=None, abstract=None)
    a.update(kw)
    return L.binding._lib.kv_page_move(ref(s), a["moves"], a["m_max"], a["count"], a["old"], a["new"], a["table"], a["kp"], a["vp"], a["ks"],
                                       a["vs"], a["weight"], a["ids"], a["abstract"], None, None, None)


CALLS = [append_at, shared, weigh, select, move]


@pytest.mark.parametrize("fields,status", SHAPES, ids=[str(f) for f, _ in SHAPES])
def test_shapes(L, fields, status):
    s = pages(L, **fields)
    assert [call(L, s) for call in CALLS] == [status] * len(CALLS)
    assert [call(L, None) for call in CALLS] == [INVALID] * len(CALLS)
    assert L.leoam_page_shared_workspace_bytes(s, 1) == 0 and L.leoam_page_shared_workspace_min(s) == 0
    assert L.leoam_page_evict_workspace_bytes(s) == 0


def test_append_at(L):
    s = pages(L, rot=64, rope=10)
    for n_axes, status in ((0, INVALID), (-1, INVALID), (9, UNSUPPORTED)):
        assert append_at(L, s, n_axes=n_axes) == status
    for name in ("position", "axis", "rope", "len", "table", "kp", "vp", "q", "q_out", "k", "v"):
        assert append_at(L, s, **{name: None}) == INVALID, name
    for name in ("rope", "kp", "vp", "q", "q_out", "k", "v"):
        assert append_at(L, s, **{name: ODD}) == INVALID, name
    assert append_at(L, s, n=-1) == INVALID and append_at(L, s, n=3, off=None) == INVALID
    assert append_at(L, s, qs=4) == INVALID and append_at(L, pages(L, kv=4, rot=64, rope=10)) == INVALID
    assert append_at(L, s, n=0) == OK and append_at(L, s, n=0, position=None, axis=None) == OK


def test_shared(L):
    s = pages(L)
    for name in ("q", "kp", "vp", "table", "len", "off", "pages", "out"):
        assert shared(L, s, **{name: None}) == INVALID, name
    for name in ("q", "kp", "vp", "out"):
        assert shared(L, s, **{name: ODD}) == INVALID, name
    assert shared(L, s, n=0) == INVALID and shared(L, s, n=3) == INVALID and shared(L, pages(L, kv=4)) == INVALID
    least = L.leoam_page_shared_workspace_min(s)
    assert 0 < least <= L.leoam_page_shared_workspace_bytes(s, 2) <= 70 << 20
    assert shared(L, s, ws=None) == WORKSPACE and shared(L, s, ws=ODD) == WORKSPACE and shared(L, s, nbytes=least - 1) == WORKSPACE
    assert L.leoam_page_shared_workspace_bytes(s, 0) == 0 and L.leoam_page_shared_workspace_bytes(s, 3) == 0


def test_weigh(L):
    s = pages(L)
    for name in ("q", "kp", "table", "len", "lse", "weight", "seen", "ids"):      # numbers: both or neither
        assert weigh(L, s, **{name: None}) == INVALID, name
    for name in ("q", "kp"):
        assert weigh(L, s, **{name: ODD}) == INVALID, name
    assert weigh(L, s, n=-1) == INVALID and weigh(L, s, n=3, off=None) == INVALID and weigh(L, pages(L, kv=4)) == INVALID
    assert weigh(L, s, n=0) == OK


def test_select(L):
    s = pages(L)
    for name in ("weight", "len", "keep", "moves", "count", "new", "ids", "seen"):
        assert select(L, s, **{name: None}) == INVALID, name
    assert select(L, s, recent=-1) == INVALID and select(L, s, m_max=0) == INVALID and select(L, s, moves=MISALIGNED4) == INVALID
    assert select(L, s, new=P) == INVALID and select(L, s, new=P, keep=P2) == INVALID and select(L, s, new=P, len=P2) == INVALID
    assert select(L, s, ws=None) == WORKSPACE and select(L, s, ws=ODD) == WORKSPACE
    assert select(L, s, nbytes=L.leoam_page_evict_workspace_bytes(s) - 1) == WORKSPACE


def test_move(L):
    s = pages(L)
    for name in ("moves", "count", "old", "new", "table", "kp", "vp"):
        assert move(L, s, **{name: None}) == INVALID, name
    for name in ("kp", "vp", "abstract"):
        assert move(L, s, **{name: ODD}) == INVALID, name
    assert move(L, s, m_max=0) == INVALID and move(L, s, moves=MISALIGNED4) == INVALID
    assert move(L, pages(L, kv=4)) == INVALID and move(L, pages(L, kv=4), ks=P) == INVALID


def test_binding_looks_at_its_tensors(L):
    s, t = pages(L), torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        L.kv_page_append_at(s, t, t, t, None, t, t, None, None, None, t, t, t)
    with pytest.raises(ValueError):
        L.page_attention_decode_shared(s, t, t, t, None, None, t, t, t, t, 1.0, t, None, t)
    with pytest.raises(ValueError):
        L.page_weight_add(s, t, None, t, None, t, t, 1.0, t, 1.0, None, t)
    with pytest.raises(ValueError):
        L.page_evict_select(s, t, None, None, t, t, None, 0, t, t, t, None, t)
    with pytest.raises(ValueError):
        L.kv_page_move(s, t, t, t, t, t, t, t)
    with pytest.raises(TypeError):
        L.binding._bind.kv_page_move(s, t)
