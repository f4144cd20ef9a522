"""kv_page_append where sequences do not simply grow: infinities beside zeros, steps back, batch rows that change hands, pages of
other sequences, lists that descend.  What is expected is read from the definition in include/leoam.h."""
import math

import pytest
import torch

from tests.test_gpu_paged import BF16, F16, F32, KIND_IDS, KINDS, L, scratch, spread  # noqa: F401

pytestmark = pytest.mark.gpu
i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731


class Pool:
    """An empty cache (NaN wherever no token is) with the buffers of a selection."""

    def __init__(self, L, dtype, q8, batch, hkv, page, max_pages, n_pages, hq=None):
        self.L, self.dtype, self.q8, self.hkv, self.page = L, dtype, q8, hkv, page
        store = torch.float8_e4m3fn if q8 else dtype
        self.hq = hq or hkv
        self.pages = L.make_pages(batch, self.hq, hkv, 128, n_pages, page, max_pages, dtype, L.E4M3 if q8 else None)
        self.k = torch.full((n_pages, hkv, page, 128), math.nan).to(store).cuda()
        self.v = self.k.clone()
        self.ks, self.vs = (torch.full((n_pages, hkv), math.nan).cuda() for _ in "kv") if q8 else (None, None)
        self.abstract = torch.full((batch, hkv, max_pages, 2, 128), 77.0, dtype=dtype).cuda()
        self.off = torch.full((batch, max_pages + 1), -7, dtype=torch.int32).cuda()
        self.n_chunks = torch.zeros(batch, dtype=torch.int32).cuda()
        self.status = torch.full((batch,), -7, dtype=torch.int32).cuda()

    def append(self, k, v, new_off, seq_len, table, abstract=True, n_chunks=True):
        self.L.kv_page_append(self.pages, None, k, v, new_off, i32(seq_len), table.cuda(), None, None, self.k, self.v, self.ks, self.vs,
                              self.abstract if abstract else None, self.off if abstract else None,
                              self.n_chunks if abstract and n_chunks else None, self.status)
        torch.cuda.synchronize()

    def values(self, which, ids, n):
        """[Hkv, n, 128] float64: the first n tokens of the pages `ids`."""
        pool, scale = (self.k, self.ks) if which == 0 else (self.v, self.vs)
        x = pool.float().double()[ids]
        if self.q8:
            x = x * scale.double()[ids][..., None, None]
        return x.transpose(0, 1).reshape(self.hkv, -1, 128)[:, :n]

    def check_rows(self, b, table, n):
        """Row b's abstract and boundaries are those of its n stored tokens."""
        ids = table[b, : -(-n // self.page)].long().cuda()
        K = self.values(0, ids, n)
        assert torch.isfinite(K).all()
        for p in range(len(ids)):
            kept = K[:, p * self.page: (p + 1) * self.page]
            assert torch.equal(self.abstract[b, :, p, 0].double(), kept.amax(1)), f"maximum, sequence {b}, page {p}"
            assert torch.equal(self.abstract[b, :, p, 1].double(), kept.amin(1)), f"minimum, sequence {b}, page {p}"
        assert int(self.n_chunks[b]) == len(ids)
        assert self.off[b, : len(ids) + 1].tolist() == [min(p * self.page, n) for p in range(len(ids) + 1)]


# ---- 8 bits: a page of zeros and infinities -------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("single", [True, False], ids=["tokens", "prompt"])
def test_infinities_beside_zeros_are_zero(L, dtype, single):
    # scale 0, so +-448 scale is 0; NaN stays NaN; and nothing changes when the scale grows
    c = Pool(L, dtype, True, 1, 2, 16, 2, 3)
    table = torch.tensor([[2, 0]], dtype=torch.int32)
    k = torch.zeros(3, 2, 128)
    v = torch.zeros(3, 2, 128)
    k[0, 0, 5], k[1, 0, 6], k[2, 1, 100] = math.inf, -math.inf, math.nan
    v[0, 1, 0], v[2, 0, 127] = -math.inf, math.nan
    k, v = k.to(dtype).cuda(), v.to(dtype).cuda()
    if single:
        for i in range(3):
            c.append(k[i: i + 1], v[i: i + 1], None, [i + 1], table)
    else:
        c.append(k, v, i32([0, 3]), [3], table)
    for grown in (False, True):
        if grown:
            one = torch.ones(1, 2, 128, dtype=dtype, device="cuda")
            c.append(one, one, None, [4], table)
        for which, x in ((0, k), (1, v)):
            got, gone = c.values(which, [2], 3).transpose(0, 1), torch.isnan(x)
            assert torch.equal(torch.isnan(got), gone)
            assert (got[~gone] == 0).all()
        assert (c.ks[2] == (2.0 ** -8 if grown else 0)).all() and (c.vs[2] == (2.0 ** -8 if grown else 0)).all()


# ---- the abstract is that of the stored keys ------------------------------------------------------------------

@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("single", [True, False], ids=["tokens", "prompt"])
def test_rejected_tokens_leave_the_abstract(L, dtype, q8, page, single):
    # some tokens are taken back and others stored in their places
    g = torch.Generator().manual_seed(page)
    c = Pool(L, dtype, q8, 2, 3, page, 4, 9)
    table = torch.tensor([[5, 2, 7, 1], [0, 8, 3, 4]], dtype=torch.int32)
    make = lambda n, gain: (torch.randn(n, 3, 128, generator=g) * gain).to(dtype).cuda()  # noqa: E731
    first = [page + 11, 9]
    off = [0, first[0], sum(first)]
    c.append(make(off[2], 1.0), make(off[2], 1.0), i32(off), first, table)
    rejected = [n + 4 for n in first]
    c.append(make(8, 30.0), make(8, 1.0), i32([0, 4, 8]), rejected, table)      # far beyond the others
    for b in (0, 1):
        c.check_rows(b, table, rejected[b])
    now = [rejected[0] - 3, rejected[1] - 4]      # one of them stays, or none
    for _ in range(2):
        if single:
            now = [n + 1 for n in now]
            c.append(make(2, 0.5), make(2, 1.0), None, now, table)
        else:
            now = [now[0] + 2, now[1] + 1]
            c.append(make(3, 0.5), make(3, 1.0), i32([0, 2, 3]), now, table)
        for b in (0, 1):
            c.check_rows(b, table, now[b])


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("single", [True, False], ids=["tokens", "prompt"])
def test_abstract_of_a_page_begun_without_one(L, dtype, q8, single):
    # (the rows held something else: of whoever had this place in the batch before)
    g = torch.Generator().manual_seed(3)
    c = Pool(L, dtype, q8, 1, 2, 32, 2, 3)
    table = torch.tensor([[1, 2]], dtype=torch.int32)
    make = lambda n: torch.randn(n, 2, 128, generator=g).to(dtype).cuda()  # noqa: E731
    c.append(make(13), make(13), i32([0, 13]), [13], table, abstract=False)
    n = 14 if single else 17
    c.append(make(n - 13), make(n - 13), None if single else i32([0, n - 13]), [n], table)
    c.check_rows(0, table, n)


def test_an_idle_sequence_has_no_chunks(L):
    c = Pool(L, BF16, False, 3, 2, 16, 3, 8)
    table = torch.tensor([[0, 1, 2], [3, 4, 5], [6, 7, -1]], dtype=torch.int32)
    x = torch.randn(60, 2, 128, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    c.append(x, x, i32([0, 20, 40, 60]), [20, 20, 20], table)
    assert c.n_chunks.tolist() == [2, 2, 2]
    c.append(x[:3], x[:3], None, [21, 0, 21], table)
    assert c.n_chunks.tolist() == [2, 0, 2] and c.status.tolist() == [0, 0, 0]
    c.append(x[:1], x[:1], i32([0, 1, 1, 1]), [22, 0, 21], table)      # (the last takes in nothing and stays as it is)
    assert c.n_chunks.tolist() == [2, 0, 2]
    c.append(x[:1], x[:1], i32([0, 1, 1, 1]), [23, 0, 0], table)
    assert c.n_chunks.tolist() == [2, 0, 0]


# ---- pages that others filled ---------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("single", [True, False], ids=["tokens", "prompt"])
def test_rows_of_shared_pages(L, dtype, q8, single):
    # a sequence that begins behind the pages of another: n_chunks says how many of its rows are there already
    g = torch.Generator().manual_seed(5)
    page, hkv = 16, 3
    c = Pool(L, dtype, q8, 3, hkv, page, 8, 24)
    table = torch.randperm(24, generator=g).to(torch.int32).reshape(3, 8)
    make = lambda n: torch.randn(n, hkv, 128, generator=g).to(dtype).cuda()  # noqa: E731
    c.append(make(100 + 30), make(130), i32([0, 100, 100, 130]), [100, 0, 30], table)
    table[1, :5], table[2, :6] = table[0, :5], table[0, :6]
    c.n_chunks[2] = 0      # (it had a sequence of its own before)
    lens = [101, 81, 97] if single else [100, 85, 120]
    c.append(make(3) if single else make(29), make(3) if single else make(29), None if single else i32([0, 0, 5, 29]), lens, table)
    assert c.status.tolist() == [0, 0, 0]
    for b in range(3):
        c.check_rows(b, table, lens[b])
    # rows that are there are not looked at; pages outside the pool are passed over
    c.abstract[1, :, :2] = 55.0
    c.abstract[1, :, 3] = 66.0
    c.n_chunks[1] = 2
    table[1, 3] = -1
    lens[1] += 1
    c.append(make(1), make(1), i32([0, 0, 1, 1]), lens, table)
    assert (c.abstract[1, :, :2] == 55).all() and (c.abstract[1, :, 3] == 66).all()
    K = c.values(0, table[1, 2:3].long().cuda(), page)
    assert torch.equal(c.abstract[1, :, 2, 0].double(), K.amax(1)) and torch.equal(c.abstract[1, :, 2, 1].double(), K.amin(1))
    assert c.off[1, :7].tolist() == [0, 16, 32, 48, 64, 80, lens[1]]


@pytest.mark.parametrize("dtype,q8", [(BF16, False), (F16, True), (F32, False)], ids=["bf16", "f16-e4m3", "f32"])
@pytest.mark.parametrize("reused", [False, True], ids=["fresh", "reused"])
def test_layer_selects_among_shared_pages(L, dtype, q8, reused):
    """A sequence behind another's pages, under a budget, against the same tokens in pages of its own."""
    g = torch.Generator().manual_seed(6)
    hq, hkv, page, head = 8, 2, 16, 96      # six pages in common
    n = [150, 130]
    x = torch.randn(n[0], hq + 2 * hkv, 128, generator=g)
    y = torch.randn(n[1] - head, hq + 2 * hkv, 128, generator=g)
    tail = torch.cat([x[:head], y]).to(dtype).cuda()      # the second sequence, whole
    x, y = x.to(dtype).cuda(), y.to(dtype).cuda()
    steps = [torch.randn(2, hq + 2 * hkv, 128, generator=g).to(dtype).cuda() for _ in range(3)]
    parts = lambda t: (t[:, :hq], t[:, hq: hq + hkv], t[:, hq + hkv:])  # noqa: E731
    table, n_pages = spread([160, 160], page, g)
    got = []
    for shared in (False, True):
        t = table.clone()
        seq_len = i32([0, 0])
        if shared:
            t[1, : head // page] = t[0, : head // page]
        layer = L.PagedLayer(t.cuda(), seq_len, hq, hkv, n_pages, page, dtype, L.E4M3 if q8 else None, token_budget=64)
        if reused:      # somebody was there before, behind pages of his own, and left
            mine = layer.page_table.clone()
            layer.page_table.copy_(table)
            seq_len.copy_(i32([1, 140]))
            layer.prompt(*parts(torch.cat([x, x])[:141]), i32([0, 1, 141]))
            seq_len.zero_()
            layer.step(*parts(x[:2]))
            layer.page_table.copy_(mine)
        else:
            layer.abstract.fill_(9.0)
        seq_len.copy_(i32([n[0], 0]))
        layer.prompt(*parts(x), i32([0, n[0], n[0]]))
        seq_len.copy_(i32(n))
        new = parts(y) if shared else parts(tail)
        out = layer.prompt(*new, i32([0, 0, new[0].shape[0]]))[-y.shape[0]:]
        kept = [out]
        for s in steps:
            seq_len.add_(1)
            layer.step(*parts(s))
            kept += [layer.out.clone(), layer.lse.clone(), layer.sel_count.clone(), layer.sel_idx.clone()]
        torch.cuda.synchronize()
        got.append(kept)
    for i, (a, b) in enumerate(zip(*got)):
        if i and i % 4 == 0:      # (entries past the count may be anything)
            listed = torch.arange(a.shape[2], device="cuda") < got[0][i - 1][..., None]
            a, b = a[listed], b[listed]
        if i == 0:
            assert torch.isfinite(a).all() and float((a.double() - b.double()).abs().max()) < 0.1      # (rows in other tiles)
        else:
            assert torch.equal(a, b), i


# ---- lists that descend ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,q8", [(BF16, False), (F16, True)], ids=["bf16", "f16-e4m3"])
@pytest.mark.parametrize("off", [[0, 100, 5, 12], [0, 10, 5, 12], [0, 12, -4, 12], [0, 5, 200, 12], [3, 1, 90, 100], [0, 40, 20, 60, 30, 100],
                                 [0, 100] + [0] * 70 + [100], [0] * 70 + [90, 80, 100]],
                         ids=lambda o: "-".join(map(str, o)) if len(o) < 9 else f"{len(o) - 1}-sequences" + str(o[-2]))
def test_tokens_of_a_descending_list_are_reported(L, dtype, q8, off):
    """Status 0 says that all of a sequence's tokens are stored and its queries are written."""
    batch, page, hkv, hq = len(off) - 1, 16, 1, 2
    new = [max(0, off[b + 1] - off[b]) for b in range(batch)]
    per = 14
    table = torch.arange(batch * per, dtype=torch.int32).reshape(batch, per)
    x = torch.randn(100, hq + 2 * hkv, 128, generator=torch.Generator().manual_seed(7)).to(dtype).cuda()
    c = Pool(L, dtype, q8, batch, hkv, page, per, batch * per, hq=hq)
    q_out = torch.full((100, hq, 128), 7.0, dtype=dtype, device="cuda")
    L.kv_page_append(c.pages, x[:, :hq], x[:, hq: hq + 1], x[:, hq + 1:], i32(off), i32([min(n, per * page) for n in new]), table.cuda(), None, q_out,
                     c.k, c.v, c.ks, c.vs, c.abstract, c.off, c.n_chunks, c.status)
    torch.cuda.synchronize()
    status = c.status.tolist()
    for b in range(batch):
        assert status[b] in (0, 1)
        if off[b] > off[b + 1] or off[b] < 0 or off[b + 1] > 100:
            assert status[b] == 1, b
        elif status[b] == 0 and new[b]:
            K = c.values(0, table[b].long().cuda(), new[b])
            assert torch.isfinite(K).all(), f"sequence {b} is said to be stored"
            assert torch.equal(q_out[off[b]: off[b + 1]], x[off[b]: off[b + 1], :hq]), f"queries of sequence {b}"
    if off == [0, 100, 5, 12]:
        assert status[1] == 1 and 1 in (status[0], status[2])


# ---- layers that share workspaces -------------------------------------------------------------------------------

def test_layers_share_workspaces(L):
    g = torch.Generator().manual_seed(8)
    hq, hkv, page, n = 8, 2, 32, [700, 40]
    table, n_pages = spread([n[0] + 4, n[1] + 4], page, g)
    x = [torch.randn(sum(n), hq + 2 * hkv, 128, generator=g).to(BF16).cuda() for _ in range(3)]
    s = [torch.randn(2, hq + 2 * hkv, 128, generator=g).to(BF16).cuda() for _ in range(3)]
    parts = lambda t: (t[:, :hq], t[:, hq: hq + hkv], t[:, hq + hkv:])  # noqa: E731
    got = []
    for together in (False, True):
        seq_len = i32(n)
        layers = []
        for i in range(3):
            layers.append(L.PagedLayer(table.cuda(), seq_len, hq, hkv, n_pages, page, BF16, L.E4M3 if i == 1 else None, token_budget=96 * (i == 2),
                                       workspaces_of=layers[0] if together and i else None))
        out = [layer.prompt(*parts(a), i32([0, n[0], sum(n)])) for layer, a in zip(layers, x)]
        seq_len.add_(1)
        out += [layer.step(*parts(a)) for layer, a in zip(layers, s)]
        torch.cuda.synchronize()
        got.append(out)
        held = {w.data_ptr(): w.numel() for layer in layers for w in [layer.workspace] + layer.prompt_workspaces}
        assert len(held) == (2 if together else 6)
    for a, b in zip(*got):
        assert torch.equal(a, b)
