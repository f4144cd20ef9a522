"""Attention over pages where rows and units are cut into pieces, with operands whose results are known to the last bit or nearly.

Every query of `Marked` is a unit vector and a key's channel is 0 or -40, so a token's weight is 1 or e^-40 (1/2 of the tokens each, other
ones for every head); a value row is a unit vector by the token's place.  Weights, their sum and the products with the values are whole
numbers: an output is a count by a count.  A token that is lost, seen twice, or weighed as its neighbour moves some channel by 1 in about
n / 256, far beyond the rounding.  Tolerances: where a row sees tokens of weight e^-40 only, the reference is the rounded product
-40 log2(e), the weights are its rounding error away from 1, 58 * 2^-24 < 2^-18; a division, and the output's rounding."""
import math

import pytest
import torch

from tests.test_gpu_paged import BF16, F16, F32, HALF, KIND_IDS, KINDS, L, scratch, spread  # noqa: F401

pytestmark = pytest.mark.gpu
NONE = -40.0


class Marked:
    def __init__(self, dtype, q8, lengths, hkv, group, page, seed, columns=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.q8, self.lengths, self.hkv, self.group, self.page = dtype, q8, lengths, hkv, group, page
        self.table, self.n_pages = spread(lengths, page, g)
        if columns > self.table.shape[1]:
            wide = torch.full((len(lengths), columns), -1, dtype=torch.int32)
            wide[:, : self.table.shape[1]] = self.table
            self.table = wide
        store = torch.float8_e4m3fn if q8 else dtype
        self.marks, pools = [], []
        k = torch.full((self.n_pages, hkv, page, 128), math.nan)
        v = k.clone()
        for b, n in enumerate(lengths):
            marks = torch.rand(hkv, group, n, generator=g) < 0.5
            marks[..., :1] = True
            self.marks.append(marks)
            kb = torch.randint(-3, 4, (n, hkv, 128), generator=g).float()
            vb = torch.zeros(n, hkv, 128)
            t = torch.arange(n)
            for h in range(hkv):
                for j in range(group):
                    kb[:, h, self.channel(h, j)] = torch.where(marks[h, j], 0.0, NONE)
                vb[t, h, (t + 37 * h) % 128] = 1.0
            at = self.table[b, t // page].long()
            k[at, :, t % page], v[at, :, t % page] = kb, vb
        # (8 bits: codes of 2^1 and 2^-1)
        self.k, self.v = (k / (2.0 if q8 else 1.0)).to(store).cuda(), (v / (0.5 if q8 else 1.0)).to(store).cuda()
        self.ks = torch.full((self.n_pages, hkv), 2.0, device="cuda") if q8 else None
        self.vs = torch.full((self.n_pages, hkv), 0.5, device="cuda") if q8 else None
        self.seq_len = torch.tensor(lengths, dtype=torch.int32).cuda()

    @staticmethod
    def channel(h, j):
        return (17 * j + 5 * h + 3) % 128

    def queries(self, n):
        q = torch.zeros(n, self.hkv, self.group, 128)
        for h in range(self.hkv):
            for j in range(self.group):
                q[:, h, j, self.channel(h, j)] = 1.0
        return q.reshape(n, -1, 128).to(self.dtype).cuda()

    def pages(self, L):
        return L.make_pages(len(self.lengths), self.hkv * self.group, self.hkv, 128, self.n_pages, self.page, self.table.shape[1], self.dtype,
                            L.E4M3 if self.q8 else None)

    def expected(self, b, n):
        """[Hq, 128], [Hq] float64: what attends to the first n tokens of sequence b."""
        out = torch.zeros(self.hkv, self.group, 128, dtype=torch.float64)
        t = torch.arange(n)
        t = t[(self.table[b, t // self.page] >= 0) & (self.table[b, t // self.page] < self.n_pages)]
        if len(t) == 0:
            return out.reshape(-1, 128), torch.full((self.hkv * self.group,), -math.inf, dtype=torch.float64)
        z = torch.where(self.marks[b][..., t], 0.0, NONE).double()
        lse = torch.logsumexp(z, -1)
        p = torch.exp(z - lse[..., None])
        for h in range(self.hkv):
            out[h].index_add_(1, (t + 37 * h) % 128, p[h])
        return out.reshape(-1, 128), lse.reshape(-1)


def same(what, got, want, rel, small):
    got = got.double().cpu()
    if torch.isinf(want).any():
        assert torch.equal(got, want), what
        return
    off = (got - want).abs() - rel * want.abs()
    assert (off <= small).all(), f"{what}: off by {float(off.max()):.3g}"


def prefill(L, m, off, n, rows, kernels_of=None):
    """off: None or the list; rows: [(row, sequence, tokens it sees)]; the others stay as they were."""
    q, pages = m.queries(n), m.pages(L)
    out = torch.full(q.shape, 7.0, dtype=m.dtype, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    ws = scratch(L.leoam_page_workspace_bytes(pages, n))
    table, new_off = m.table.cuda(), None if off is None else torch.tensor(off, dtype=torch.int32).cuda()

    def call():
        L.page_attention_prefill(pages, q, new_off, m.k, m.v, m.ks, m.vs, table, m.seq_len, 1.0, out, lse, ws)
    if kernels_of:
        names = [name for name, _ in kernels_of(call)]
        assert len(names) == 2 and "page_prefill_merge_kernel" in names[1], names      # (work may be cut, pieces are merged)
    call()
    torch.cuda.synchronize()
    for row, b, seen in rows:
        want, want_lse = m.expected(b, seen)
        same(f"row {row}", out[row], want, HALF[m.dtype] + 2.0 ** -17, 2.0 ** -40)
        same(f"lse of row {row}", lse[row], want_lse, 2.0 ** -21, 2.0 ** -18)
    touched = {r for r, _, _ in rows}
    return out, lse, touched


def rows_of(m, off, some=None):
    return [(r, b, m.lengths[b] - off[b + 1] + r + 1) for b in range(len(off) - 1) for r in range(off[b], off[b + 1]) if some is None or r in some]


def offsets(new):
    return [sum(new[:b]) for b in range(len(new) + 1)]


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("new", [[5, 1, 7], [150, 20, 33]], ids=["few", "many"])
def test_prefill_pieces(L, kernels_of, dtype, q8, group, new):
    m = Marked(dtype, q8, [3000, 20, 2501], 2, group, 32, seed=group)
    off = offsets(new)
    prefill(L, m, off, off[-1], rows_of(m, off), kernels_of)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("group,new", [(1, [60, 4]), (4, [3, 16]), (8, [8, 2]), (8, [100, 20])])
def test_prefill_pieces_with_missing_pages(L, kernels_of, dtype, q8, group, new):
    # pages of 16: whole 16-key groups of a tile are missing, in either half of it
    m = Marked(dtype, q8, [2300, 1900], 2, group, 16, seed=20 + group)
    gone = torch.randperm(110, generator=torch.Generator().manual_seed(1))[:40] + 1
    m.table[0, gone] = torch.where(gone % 2 == 0, 10 ** 6, -1).to(torch.int32)
    m.table[1, 30:60] = -7      # several tiles one after the other
    m.table[1, 118] = m.n_pages      # the last page
    off = offsets(new)
    prefill(L, m, off, off[-1], rows_of(m, off), kernels_of)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("group", [1, 8])
def test_prefill_pieces_rows_of_nobody_and_negative_positions(L, kernels_of, dtype, q8, group):
    # the first sequence claims 8 new tokens and holds 3; rows 20 .. 29 belong to nobody
    m = Marked(dtype, q8, [3, 4001], 2, group, 32, seed=30)
    rows = [(i, 0, max(0, i - 4)) for i in range(8)] + [(8 + i, 1, 4001 - 11 + i) for i in range(12)]
    out, lse, _ = prefill(L, m, [0, 8, 20], 30, rows, kernels_of)
    assert (out[20:] == 7).all() and (lse[20:] == 7).all()


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_prefill_pieces_one_row_each(L, kernels_of, dtype, q8, group):
    m = Marked(dtype, q8, [3000, 0, 17, 1, 2050], 2, group, 64, seed=40)
    prefill(L, m, None, 5, [(b, b, n) for b, n in enumerate(m.lengths)], kernels_of)


@pytest.mark.parametrize("dtype,q8", [(F32, False), (BF16, False), (F16, True)], ids=["f32", "bf16", "f16-e4m3"])
@pytest.mark.parametrize("batch", [31, 32])
def test_prefill_as_many_units_as_are_cut(L, kernels_of, dtype, q8, batch):
    # 32 heads of 32 row tiles are 1024 units, the most that are shared out; one more sequence and each has a workgroup
    lengths = [5000, 40] + [3 + b for b in range(batch - 2)]
    m = Marked(dtype, q8, lengths, 32, 2, 16, seed=50)
    new = [2] * batch
    off = offsets(new)
    if batch == 31:
        new[0], off = 4, offsets([4] + new[1:])      # 64 rows of two heads
        assert off[-1] * 2 // 128 + batch == 31 + (off[-1] >= 64)
    prefill(L, m, off, off[-1], rows_of(m, off, set(range(0, 12)) | {off[-1] - 1}), kernels_of if off[-1] * 2 // 128 + batch <= 32 else None)


# ---- decode ----------------------------------------------------------------------------------------------------

def decode(L, m, kernels_of=None, keep=None):
    B = len(m.lengths)
    q, pages = m.queries(B), m.pages(L)
    out, lse = torch.full(q.shape, math.nan, device="cuda"), torch.full(q.shape[:2], math.nan, device="cuda")
    ws, table = scratch(L.leoam_page_workspace_bytes(pages)), m.table.cuda()

    def call():
        L.page_attention_decode(pages, q, m.k, m.v, m.ks, m.vs, table, m.seq_len, None, None, 1.0, out, lse, ws)
    if kernels_of:
        names = [name for name, _ in kernels_of(call)]
        assert len(names) == 2 and "page_decode_merge_kernel" in names[1], names
    call()
    torch.cuda.synchronize()
    for b, n in enumerate(m.lengths):
        want, want_lse = m.expected(b, n)
        same(f"sequence {b}", out[b], want, 2.0 ** -21, 2.0 ** -40)
        same(f"lse of sequence {b}", lse[b], want_lse, 2.0 ** -21, 2.0 ** -18)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("lengths,hkv,page", [([6001, 70, 0, 3500], 2, 16), ([2100] * 3 + [5, 900] * 4 + [7777], 8, 64)], ids=["few", "more"])
def test_decode_pieces(L, kernels_of, dtype, q8, group, lengths, hkv, page):
    decode(L, Marked(dtype, q8, lengths, hkv, group, page, seed=60 + group), kernels_of)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("group", [1, 8])
def test_decode_pieces_with_missing_pages(L, kernels_of, dtype, q8, group):
    m = Marked(dtype, q8, [6001, 4000, 300], 2, group, 16, seed=70)
    gone = torch.randperm(370, generator=torch.Generator().manual_seed(2))[:150] + 1
    m.table[0, gone] = torch.where(gone % 2 == 0, 10 ** 6, -1).to(torch.int32)
    m.table[1, 40:200] = -7      # more than a wave's part of a stretch
    m.table[2, 1:19] = m.n_pages
    decode(L, m, kernels_of)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
def test_decode_weights_to_the_last_part(L, dtype, q8):
    """Equal weights that 16 (bf16) or 11 (fp16) bits do not hold: what a lost part of them is worth would add up.

    Of 32 tokens one has logit 0 and value 0, the others logit -x and value 1: out = 31 w / (1 + 31 w), w = e^-x.  The exponent
    -x log2(e), below 4, is off by 2^-25 of itself and the rounding of its product, 2^-23, and the exponential by 2^-23: 2^-21.5 of w, of
    which a third reaches out.  The matrix cores add up 32 products and the waves four sums, 36 * 2^-24; a lane 8 weights, lanes
    and waves two and four sums, 14 * 2^-24; the division: 51.  In all below 54 * 2^-24 of out; a lost part of x as chosen is worth
    twice that."""
    def lost(x):      # relative to the weight
        w = rest = torch.exp(-x.double()).float() * (2.0 ** 15 if dtype == F16 else 1.0)
        for _ in range(1 if dtype == F16 else 2):
            rest = rest - rest.to(dtype).float()
        return (rest / w).abs()
    xs = torch.arange(64, 500) / 128.0                      # (7 + 2 bits: numbers of bf16 from 2 on and some below)
    xs = xs[xs.to(BF16).float() == xs]
    x = xs[lost(xs).argmax()] if dtype != F32 else xs[77]
    n, hq, hkv, page = 128, 8, 1, 16
    z = torch.zeros(n, hkv, 128)
    z[:, 0, 3] = -1.0
    z[::32, 0, 3] = 0.0
    v = torch.ones(n, hkv, 128)
    v[::32] = 0.0
    store = torch.float8_e4m3fn if q8 else dtype
    fill = lambda t: t.reshape(n // page, page, hkv, 128).transpose(1, 2).contiguous().to(store).cuda()  # noqa: E731
    one = torch.ones(n // page, hkv, device="cuda") if q8 else None
    q = torch.zeros(1, hq, 128)
    q[..., 3] = x
    pages = L.make_pages(1, hq, hkv, 128, n // page, page, n // page, dtype, L.E4M3 if q8 else None)
    out, lse = torch.empty(1, hq, 128, device="cuda"), torch.empty(1, hq, device="cuda")
    L.page_attention_decode(pages, q.to(dtype).cuda(), fill(z), fill(v), one, one, torch.arange(n // page, dtype=torch.int32).reshape(1, -1).cuda(),
                            torch.tensor([n], dtype=torch.int32).cuda(), None, None, 1.0, out, lse, scratch(L.leoam_page_workspace_bytes(pages)))
    w = math.exp(-float(x))
    want = 31 * w / (1 + 31 * w)
    tol = 54 * 2.0 ** -24
    assert dtype == F32 or float(lost(x[None])[0]) > 2 * tol
    assert float((out.double() / want - 1).abs().max()) <= tol
