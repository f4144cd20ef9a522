"""What the paged cache's entry points refuse, on the host (no GPU needed: nothing is launched)."""
import ctypes

import pytest
import torch

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -3, -4
P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4096 + 8)


@pytest.fixture(scope="module")
def L():
    import paper_2506_20187_amd as lib
    return lib


def pages(L, batch=2, hq=8, hkv=2, d=128, n_pages=10, page=64, max_pages=5, dtype=2, kv=2, rot=0, inter=0, rope=0):
    return L.Pages(batch, hq, hkv, d, n_pages, page, max_pages, dtype, kv, rot, inter, rope)


def append(L, s, **kw):
    a = dict(q=P, qs=8 * 128, k=P, ks=2 * 128, v=P, vs=2 * 128, n=0, off=P, len=P, table=P, rope=None, q_out=P, kp=P, vp=P, k_scale=None,
             v_scale=None, abstract=None, chunk_off=None, n_chunks=None, status=None)
    a.update(kw)
    return L.binding._lib.kv_page_append(ctypes.byref(s) if s is not None else None, a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["n"],
                                         a["off"], a["len"], a["table"], a["rope"], a["q_out"], a["kp"], a["vp"], a["k_scale"],
                                         a["v_scale"], a["abstract"], a["chunk_off"], a["n_chunks"], a["status"], None)


def decode(L, s, **kw):
    a = dict(q=P, kp=P, vp=P, ks=None, vs=None, table=P, len=P, idx=None, count=None, k_max=0, out=P, lse=None, ws=None, nbytes=0)
    a.update(kw)
    return L.binding._lib.page_attention_decode(ctypes.byref(s) if s is not None else None, a["q"], a["kp"], a["vp"], a["ks"], a["vs"],
                                                a["table"], a["len"], a["idx"], a["count"], a["k_max"], 1.0, a["out"], a["lse"], a["ws"],
                                                a["nbytes"], None)


def prefill(L, s, **kw):
    a = dict(q=P, n=5, off=P, kp=P, vp=P, ks=None, vs=None, table=P, len=P, out=P, lse=None, ws=None, nbytes=0)
    a.update(kw)
    return L.binding._lib.page_attention_prefill(ctypes.byref(s) if s is not None else None, a["q"], a["n"], a["off"], a["kp"], a["vp"],
                                                 a["ks"], a["vs"], a["table"], a["len"], 1.0, a["out"], a["lse"], a["ws"], a["nbytes"], None)


SHAPES = [(dict(batch=0), INVALID), (dict(hq=7), INVALID), (dict(hkv=0), INVALID), (dict(n_pages=0), INVALID), (dict(page=0), INVALID),
          (dict(max_pages=0), INVALID), (dict(rot=8), INVALID), (dict(rot=144, rope=10), INVALID), (dict(rot=64), INVALID),
          (dict(rot=-16), INVALID), (dict(inter=2), INVALID), (dict(d=64), UNSUPPORTED), (dict(hq=6), UNSUPPORTED),
          (dict(hq=32), UNSUPPORTED), (dict(page=8), UNSUPPORTED), (dict(page=48), UNSUPPORTED), (dict(page=512), UNSUPPORTED),
          (dict(max_pages=1 << 24), UNSUPPORTED), (dict(dtype=3, kv=3), UNSUPPORTED), (dict(dtype=4, kv=4), UNSUPPORTED),
          (dict(dtype=0, kv=4), UNSUPPORTED), (dict(dtype=1, kv=2), UNSUPPORTED), (dict(kv=3), UNSUPPORTED),
          (dict(batch=70000), UNSUPPORTED), (dict(hkv=5000, hq=5000), UNSUPPORTED)]


@pytest.mark.parametrize("fields,status", SHAPES, ids=[str(f) for f, _ in SHAPES])
def test_shapes(L, fields, status):
    s = pages(L, **fields)
    assert append(L, s) == status and decode(L, s) == status and prefill(L, s) == status
    assert L.leoam_page_workspace_bytes(s, 10) == 0 and L.leoam_page_workspace_min(s) == 0


def test_append(L):
    # (two rows: a call that is refused launches nothing; no rows: a call that is not has nothing to do)
    s, rot, e4 = pages(L), pages(L, rot=64, rope=10), pages(L, kv=4)
    assert append(L, None) == INVALID
    assert append(L, s, n=0) == OK and append(L, s, n=0, q=None, k=None, v=None) == OK
    for name in ("len", "table", "kp", "vp", "q", "q_out", "k", "v"):           # q and q_out only together
        assert append(L, s, n=2, **{name: None}) == INVALID, name
    for name in ("q", "k", "v", "q_out", "kp", "vp", "abstract"):
        assert append(L, s, n=2, **{name: ODD}) == INVALID, name
    assert append(L, s, n=-1) == INVALID and append(L, s, n=3, off=None) == INVALID and append(L, s, n=0, off=None) == INVALID
    assert append(L, rot, n=2) == INVALID and append(L, rot, n=2, rope=ODD) == INVALID
    assert append(L, e4, n=2) == INVALID and append(L, e4, n=2, k_scale=P) == INVALID
    for name, heads in (("qs", 8), ("ks", 2), ("vs", 2)):
        for stride in (0, -128, heads * 128 - 8, heads * 128 + 4, 1 << 40):
            assert append(L, s, n=3, **{name: stride}) == INVALID, (name, stride)
    assert append(L, s, n=3, q_out=P, q=P, qs=12 * 128) == INVALID    # in place needs contiguous rows


def test_attention(L):
    s, e4 = pages(L), pages(L, kv=4)
    assert decode(L, None) == INVALID and prefill(L, None) == INVALID
    for name in ("q", "kp", "vp", "table", "len", "out"):
        assert decode(L, s, **{name: None}) == INVALID and prefill(L, s, **{name: None}) == INVALID, name
    for name in ("q", "kp", "vp", "out"):
        assert decode(L, s, **{name: ODD}) == INVALID and prefill(L, s, **{name: ODD}) == INVALID, name
    assert decode(L, e4) == INVALID and prefill(L, e4) == INVALID
    assert decode(L, s) == WORKSPACE and prefill(L, s) == WORKSPACE   # none given
    assert decode(L, s, ws=ODD, nbytes=1 << 30) == WORKSPACE
    least = L.leoam_page_workspace_min(s)
    if least > 0:
        assert decode(L, s, ws=P, nbytes=least - 1) == WORKSPACE
    big = dict(ws=P, nbytes=1 << 30)
    assert decode(L, s, idx=P, **big) == INVALID and decode(L, s, count=P, **big) == INVALID
    assert decode(L, s, idx=P, count=P, k_max=0, **big) == INVALID
    assert decode(L, s, idx=P, count=P, k_max=1 << 24, **big) == UNSUPPORTED
    assert prefill(L, s, n=-1, **big) == INVALID and prefill(L, s, n=3, off=None, **big) == INVALID
    assert prefill(L, s, n=0) == OK


def test_workspace_sizes(L):
    for s in (pages(L), pages(L, kv=4), pages(L, dtype=0, kv=0), pages(L, hq=64, hkv=8, batch=300)):
        assert 0 <= L.leoam_page_workspace_min(s) <= L.leoam_page_workspace_bytes(s) <= 64 << 20
        for n in (1, 100, 1 << 20):
            assert L.leoam_page_workspace_min(s) <= L.leoam_page_workspace_bytes(s, n) <= 72 << 20


def test_binding_looks_at_its_tensors(L):
    s = pages(L)
    t = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        L.page_attention_decode(s, t, t, t, None, None, t, t, None, None, 1.0, t, None, t)
    with pytest.raises(TypeError):
        L.page_attention_decode(L.make_shape(1, 8, 2, 128, 64, 4, 4, torch.bfloat16), t, t, t, None, None, t, t, None, None, 1.0, t, None, t)
    with pytest.raises(ValueError):
        L.kv_page_append(s, t, t, t, None, t, t, None, t, t, t)
    with pytest.raises(ValueError):
        L.page_attention_prefill(s, None, None, t, t, None, None, t, t, 1.0, t, None, t)


def test_rope_table(L):
    table = L.rope_table(7, 16, 100.0).double()
    for p in range(7):
        for i in range(8):
            angle = p * 100.0 ** (-i / 8)
            assert abs(float(table[p, i]) - float(torch.tensor(angle, dtype=torch.float64).cos())) <= 2.0 ** -24
            assert abs(float(table[p, 8 + i]) - float(torch.tensor(angle, dtype=torch.float64).sin())) <= 2.0 ** -24
