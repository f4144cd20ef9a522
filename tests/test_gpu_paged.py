"""The paged cache: kv_page_append, page_attention_decode, page_attention_prefill against tests/paged_reference.py.

Pages that are not listed, and the places of a page behind the last token, hold NaN throughout: nothing of them may
reach a result.

Tolerances.  Appending is compared bit for bit (its definition is in binary32 operations).  Attention, with
A = max_t scale * sum_d |q_d K_td|:  a logit is a sum of 128 products in 32 bits and is scaled twice, each step off by at
most 2^-24 relative to the magnitudes summed, so it is within 140 * 2^-24 A < 2^-16 A =: dz (running sums in other
orders included), which moves a weight by a factor e^dz, numerator and denominator alike: 2 dz together.  Weights enter
P V in 16-bit pieces (decode, two or three: off by at most 2^-16) or one (prefill: 2^-8 for bf16, 2^-11 for fp16, 0 for fp32).
A sum of n terms in 32 bits is off by at most n 2^-24 of the magnitudes; exp2 and log2 by a few 2^-23.  The output is
within max|V| times all that; prefill rounds it once more."""
import math

import numpy as np
import pytest
import torch

from tests import paged_reference as R

pytestmark = pytest.mark.gpu
SCALE = 1.0 / math.sqrt(128)
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def L():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2506_20187_amd as lib
    return lib


def spread(lengths, page, gen, spare=3):
    """A page table over a shuffled pool: (table, number of pages)."""
    pages = [-(-n // page) for n in lengths]
    n_pages = sum(pages) + spare
    order = torch.randperm(n_pages, generator=gen).to(torch.int32)
    table = torch.full((len(lengths), max(max(pages), 1) + 1), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at: at + n]
        at += n
    return table, n_pages


class Made:
    """Filled pages (through the reference), with NaN wherever no token is."""

    def __init__(self, dtype, q8, lengths, hkv, page, seed, k_gain=1.0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.q8, self.lengths, self.hkv, self.page = dtype, q8, lengths, hkv, page
        self.table, self.n_pages = spread(lengths, page, g)
        shape = (self.n_pages, hkv, page, 128)
        store = torch.float8_e4m3fn if q8 else dtype
        nan = torch.full(shape, math.nan).to(store)
        sc = torch.full((self.n_pages, hkv), math.nan) if q8 else None
        self.cache = R.Cache(nan, nan, sc, sc, dtype)
        for b, n in enumerate(lengths):
            if n:
                k = (torch.randn(n, hkv, 128, generator=g) * k_gain).to(dtype).float()
                v = torch.randn(n, hkv, 128, generator=g).to(dtype).float()
                self.cache.append(k, v, 0, self.table[b], page)
        self.k_pages, self.v_pages = (p.to(torch.float32).to(store).cuda() for p in self.cache.pool)
        self.k_scale, self.v_scale = ((s.float().cuda() if q8 else None) for s in self.cache.scale)
        self.seq_len = torch.tensor(lengths, dtype=torch.int32).cuda()

    def pages(self, L, hq, **kw):
        return L.make_pages(len(self.lengths), hq, self.hkv, 128, self.n_pages, self.page, self.table.shape[1], self.dtype,
                            L.E4M3 if self.q8 else None, **kw)

    def tokens(self, which, b, positions):
        """[Hkv, n, 128] float64 of sequence b's tokens at `positions`."""
        v = self.cache.values(which)
        pos = torch.as_tensor(positions, dtype=torch.long)
        return v[self.table[b, pos // self.page].long(), :, pos % self.page].transpose(0, 1)


def scratch(nbytes):
    """A workspace: anything may stand in it."""
    return torch.full((max(16, nbytes),), 0xAA, dtype=torch.uint8, device="cuda")


def check(name, got, want, tol):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), f"{name}: not finite"
    off = (got - want).abs()
    assert (off <= tol).all(), f"{name}: off by {float((off - tol).max() + 0):.3g} more than allowed (largest {float(off.max()):.3g})"


def check_rows(L, made, out, lse, rows, weight_half, out_half, scale=SCALE):
    """rows: (index into out, q [Hq,128], per-head K, V lists)."""
    for i, q, K, V in rows:
        want, want_lse, reach = R.attend(q.double(), K, V, scale)
        n = K.shape[1]
        if n == 0:
            assert (out[i] == 0).all() and (lse[i] == -math.inf).all()
            continue
        dz = 2.0 ** -16 * reach
        top = float(V.abs().max())
        tol = top * (2 * dz + weight_half + n * 2.0 ** -24 + 2.0 ** -20) + out_half * want.abs()
        check("out", out[i], want, tol)
        check("lse", lse[i], want_lse, dz + (n + 8) * 2.0 ** -24 + 2.0 ** -21 * want_lse.abs() + 2.0 ** -21)


# ---- append --------------------------------------------------------------------------------------------------

def run_append(L, dtype, q8, hq, hkv, page, calls, rot=128, interleaved=False, seed=0, strided=True, poke=None, gain=None):
    """calls: per call the new tokens of every sequence; everything is compared after each of them."""
    g = torch.Generator().manual_seed(seed)
    B = len(calls[0])
    total = [sum(c[b] for c in calls) for b in range(B)]
    table, n_pages = spread(total, page, g)
    max_pages = table.shape[1]
    store = torch.float8_e4m3fn if q8 else dtype
    kp = torch.full((n_pages, hkv, page, 128), math.nan).to(store)
    sc = torch.full((n_pages, hkv), math.nan) if q8 else None
    ref = R.Cache(kp, kp, sc, sc, dtype)
    rope = L.rope_table(max_pages * page, rot, 10000.0) if rot else None
    pages = L.make_pages(B, hq, hkv, 128, n_pages, page, max_pages, dtype, L.E4M3 if q8 else None, rot_dim=rot,
                         interleaved=interleaved, rope_len=max_pages * page if rot else 0)
    k_pages, v_pages = kp.cuda(), kp.cuda()
    k_scale, v_scale = (sc.cuda(), sc.cuda()) if q8 else (None, None)
    abstract = torch.full((B, hkv, max_pages, 2, 128), math.nan).to(dtype).cuda()
    off = torch.full((B, max_pages + 1), -7, dtype=torch.int32).cuda()
    nch = torch.full((B,), -7, dtype=torch.int32).cuda()
    status = torch.full((B,), -7, dtype=torch.int32).cuda()
    held = [0] * B
    for ci, call in enumerate(calls):
        n = sum(call)
        width = hq + 2 * hkv
        x = torch.randn(n, width, 128, generator=g)
        if gain:
            x = x * gain[ci]
        if poke:
            poke(ci, x, hq, hkv)
        x = x.to(dtype)
        xg = x.cuda()
        q, k, v = xg[:, :hq], xg[:, hq: hq + hkv], xg[:, hq + hkv:]
        if not strided:
            q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        lens = [held[b] + call[b] for b in range(B)]
        one_each = all(c <= 1 for c in call) and n == B
        new_off = None if one_each else torch.tensor([0] + list(np.cumsum(call)), dtype=torch.int32).cuda()
        q_out = torch.full((n, hq, 128), math.nan).to(dtype).cuda()
        L.kv_page_append(pages, q, k, v, new_off, torch.tensor(lens, dtype=torch.int32).cuda(), table.cuda(),
                         rope.cuda() if rot else None, q_out, k_pages, v_pages, k_scale, v_scale, abstract, off, nch, status)
        torch.cuda.synchronize()
        assert (status == 0).all()
        row = 0
        for b in range(B):
            m = call[b]
            if m == 0:
                continue
            pos = torch.arange(held[b], lens[b])
            xb = x[row: row + m]
            qr = R.rotate(xb[:, :hq], rope, pos, rot, interleaved)
            assert torch.equal(q_out[row: row + m].cpu().float().nan_to_num(3e30), qr.to(dtype).float().nan_to_num(3e30)), "rotated queries"
            exact = R.rotate(xb[:, :hq], rope, pos, rot, interleaved, torch.float64)
            span = 2.0 ** -22 * xb[:, :hq].double().abs().amax(-1, keepdim=True) + HALF[dtype] * exact.abs() + 1e-7
            fine = torch.isfinite(exact)
            assert ((q_out[row: row + m].cpu().double() - exact).abs()[fine] <= span.expand_as(exact)[fine]).all()
            touched = ref.append(R.rotate(xb[:, hq: hq + hkv], rope, pos, rot, interleaved), xb[:, hq + hkv:].float(), held[b], table[b], page)
            held[b] = lens[b]
            row += m
            vals = ref.values(0)
            for p in touched:
                z = min(lens[b], (p + 1) * page) - p * page
                kept = vals[int(table[b, p]), :, :z]
                bare = torch.where(torch.isnan(kept), torch.full_like(kept, -math.inf), kept)
                assert torch.equal(abstract[b, :, p, 0].cpu().double(), bare.amax(1)), f"abstract max, page {p}"
                bare = torch.where(torch.isnan(kept), torch.full_like(kept, math.inf), kept)
                assert torch.equal(abstract[b, :, p, 1].cpu().double(), bare.amin(1)), f"abstract min, page {p}"
            P = -(-lens[b] // page)
            assert int(nch[b]) == P
            assert off[b, : P + 1].tolist() == [min(i * page, lens[b]) for i in range(P + 1)]
        for which, (pool, scale) in enumerate(((k_pages, k_scale), (v_pages, v_scale))):
            got = pool.cpu()
            got = got.to(torch.float64) if not q8 else R.E4M3_VALUES[got.view(torch.uint8).long()]
            want = ref.pool[which]
            assert torch.equal(torch.isnan(got), torch.isnan(want)), "NaN in other places"
            assert torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0)), "kv"[which] + " pages"
            if q8:
                assert torch.equal(scale.cpu().double().nan_to_num(-1.0), ref.scale[which].nan_to_num(-1.0)), "scales"


@pytest.mark.parametrize("dtype,q8", [(F32, False), (F16, False), (BF16, False), (F16, True), (BF16, True)],
                         ids=["f32", "f16", "bf16", "f16-e4m3", "bf16-e4m3"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_append_prompts_then_tokens(L, dtype, q8, page):
    calls = [[37, 0, 1, 2 * page, page + 3], [1, 1, 1, 1, 1], [1, 5, 0, page - 1, 1], [1, 1, 1, 1, 1], [0, 0, 130, 0, 0]]
    run_append(L, dtype, q8, 8, 2, page, calls, seed=page, gain=[1.0, 3.0, 1.0, 40.0, 0.1])


@pytest.mark.parametrize("rot,interleaved", [(0, False), (16, False), (64, False), (96, False), (128, True), (16, True), (112, True)])
@pytest.mark.parametrize("dtype,q8", [(F32, False), (BF16, False), (F16, True)], ids=["f32", "bf16", "f16-e4m3"])
def test_append_rotations(L, dtype, q8, rot, interleaved):
    run_append(L, dtype, q8, 12 if not q8 else 6, 3, 16, [[21, 3], [1, 1], [9, 30]], rot=rot, interleaved=interleaved, seed=rot)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (5, 5), (16, 2), (64, 8), (40, 40)])
def test_append_head_layouts(L, hq, hkv):
    run_append(L, BF16, True, hq, hkv, 32, [[40], [1], [2]], seed=hq, strided=hq != 16)
    run_append(L, F32, False, hq, hkv, 32, [[40], [1], [2]], seed=hq, strided=hq != 16)


def test_append_many_sequences(L):
    # more sequences than a wave looks up at once, some without new tokens
    rng = np.random.default_rng(5)
    first = [int(x) for x in rng.integers(0, 40, 200)]
    run_append(L, BF16, True, 4, 1, 16, [first, [int(x) for x in rng.integers(0, 3, 200)], [1] * 200], seed=9)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_append_8bit_special_values(L, dtype):
    def poke(ci, x, hq, hkv):
        k = x[:, hq: hq + hkv]
        if ci == 0:
            x.zero_()                                      # a page of zeros has scale 0 ...
        if ci == 1:
            k[0, 0, 5], k[0, 0, 6], x[0, -1, 0] = math.inf, -math.inf, math.nan
        if ci == 2:
            x.mul_(3e4 if dtype == F16 else 1e30)          # ... grows, by far ...
        if ci == 3:
            x.mul_(1e-6 if dtype == F16 else 1e-36)        # ... and does not shrink
        if ci == 4:
            x[:] = 448.0                                   # the border between two scales, and one step over it
            x[..., ::2] = 448.0 if dtype == F16 else 450.0
    run_append(L, dtype, True, 4, 2, 16, [[3], [1], [2], [1], [30], [1]], rot=0, seed=1, poke=poke)


def test_append_in_place_queries(L):
    g = torch.Generator().manual_seed(3)
    q = torch.randn(5, 8, 128, generator=g).to(BF16)
    kv = torch.randn(5, 2, 128, generator=g).to(BF16).cuda()
    table, n_pages = spread([5], 16, g)
    rope = L.rope_table(32, 128)
    pages = L.make_pages(1, 8, 2, 128, n_pages, 16, 2, BF16, rot_dim=128, rope_len=32)
    pool = torch.zeros(n_pages, 2, 16, 128, dtype=BF16, device="cuda")
    qg = q.cuda()
    L.kv_page_append(pages, qg, kv, kv, torch.tensor([0, 5], dtype=torch.int32).cuda(), torch.tensor([5], dtype=torch.int32).cuda(),
                     table.cuda(), rope.cuda(), qg, pool, pool.clone())
    assert torch.equal(qg.cpu(), R.rotate(q, rope, torch.arange(5), 128, False).to(BF16))


def test_append_leaves_refused_sequences_alone(L):
    # lengths that do not fit, pages outside the pool, positions beyond the table
    g = torch.Generator().manual_seed(4)
    hq, hkv, page = 4, 2, 16
    new = [4, 20, 3, 2, 2, 0]
    lens = [3, 24, 3, 50, 2000, 7]                         # fewer than new; fine; bad page; beyond the table; beyond capacity; none
    table = torch.tensor([[0, -1, -1, -1], [1, 2, -1, -1], [99, -1, -1, -1], [3, 4, 5, 6], [7, 8, 9, 10], [11, -1, -1, -1]], dtype=torch.int32)
    n = sum(new)
    x = torch.randn(n, hq + 2 * hkv, 128, generator=g).to(BF16).cuda()
    rope = L.rope_table(40, 128)
    pages = L.make_pages(6, hq, hkv, 128, 12, page, 4, BF16, rot_dim=128, rope_len=40)
    pool = torch.full((12, hkv, page, 128), 7.0, dtype=BF16, device="cuda")
    vpool = pool.clone()
    q_out = torch.full((n, hq, 128), 7.0, dtype=BF16, device="cuda")
    status = torch.full((6,), -7, dtype=torch.int32).cuda()
    off = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32).cuda()
    L.kv_page_append(pages, x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:], off, torch.tensor(lens, dtype=torch.int32).cuda(),
                     table.cuda(), rope.cuda(), q_out, pool, vpool, status=status)
    torch.cuda.synchronize()
    assert status.tolist() == [1, 0, 2, 3, 1, 0]
    for b, untouched in ((0, [0]), (3, [3, 4, 5, 6]), (4, [7, 8, 9, 10]), (5, [11])):
        assert (pool[untouched] == 7).all() and (vpool[untouched] == 7).all(), b
    assert (q_out[:4] == 7).all() and (q_out[27:31] == 7).all()
    assert not (q_out[4:27] == 7).all(dim=-1).any()
    assert (pool[1, :, :4] == 7).all() and not (pool[1, :, 4:] == 7).all() and (pool[2, :, 8:] == 7).all()


# ---- decode --------------------------------------------------------------------------------------------------

KINDS = [(F32, False), (F16, False), (BF16, False), (F16, True), (BF16, True)]
KIND_IDS = ["f32", "f16", "bf16", "f16-e4m3", "bf16-e4m3"]


def run_decode(L, made, hq, seed=0, keep=None, workspace_bytes=None, scale=SCALE):
    B, hkv = len(made.lengths), made.hkv
    g = torch.Generator().manual_seed(seed + 77)
    q = torch.randn(B, hq, 128, generator=g).to(made.dtype)
    pages = made.pages(L, hq)
    out = torch.full((B, hq, 128), math.nan, device="cuda")
    lse = torch.full((B, hq), math.nan, device="cuda")
    nbytes = L.leoam_page_workspace_bytes(pages) if workspace_bytes is None else workspace_bytes
    ws = scratch(nbytes)
    idx = count = None
    if keep is not None:
        idx, count = keep
    L.page_attention_decode(pages, q.cuda(), made.k_pages, made.v_pages, made.k_scale, made.v_scale, made.table.cuda(), made.seq_len,
                            idx.cuda() if keep else None, count.cuda() if keep else None, scale, out, lse, ws)
    torch.cuda.synchronize()
    G = hq // hkv
    half = 0.0 if made.dtype == F32 else 2.0 ** -16
    for b, n in enumerate(made.lengths):
        if not keep:
            rows = [(b, q[b], made.tokens(0, b, range(n)), made.tokens(1, b, range(n)))]
            check_rows(L, made, out, lse, rows, half, 2.0 ** -23, scale)
            continue
        for h in range(hkv):
            pos = []
            for j in range(min(max(int(count[b, h]), 0), idx.shape[2])):
                p = int(idx[b, h, j])
                if p >= 0:
                    pos += [t for t in range(p * made.page, (p + 1) * made.page) if t < n]
            K, V = made.tokens(0, b, pos)[h: h + 1], made.tokens(1, b, pos)[h: h + 1]
            o, l = out[b, h * G: (h + 1) * G][None], lse[b, h * G: (h + 1) * G][None]
            check_rows(L, made, o, l, [(0, q[b, h * G: (h + 1) * G], K, V)], half, 2.0 ** -23)
    return q, out, lse


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_decode_lengths(L, dtype, q8, group):
    made = Made(dtype, q8, [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 300], 2, 16, seed=group)
    run_decode(L, made, 2 * group, seed=group)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("page", [32, 64, 128, 256])
def test_decode_page_sizes(L, dtype, q8, page):
    made = Made(dtype, q8, [5 * page + 7, page, 1, 4097 if page == 64 else 700], 3, page, seed=page)
    run_decode(L, made, 12, seed=page)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("page", [16, 128])
def test_decode_kept_pages(L, dtype, q8, page):
    made = Made(dtype, q8, [10 * page + 5, 3 * page, 0, 7 * page + 1], 2, page, seed=page + 1)
    idx = torch.full((4, 2, 5), -1, dtype=torch.int32)
    count = torch.zeros(4, 2, dtype=torch.int32)
    for (b, h), pages in {(0, 0): [0, 3, 10], (0, 1): [1, 2, 4, 5, 9], (1, 0): [2], (1, 1): [], (2, 0): [0], (3, 0): [7, 0], (3, 1): [3, 50, -4, 6]}.items():
        idx[b, h, : len(pages)] = torch.tensor(pages, dtype=torch.int32)
        count[b, h] = len(pages)
    count[0, 1] = 900                                      # clamped to k_max
    run_decode(L, made, 8, keep=(idx, count))


@pytest.mark.parametrize("dtype,q8", [(F32, False), (BF16, False), (BF16, True)], ids=["f32", "bf16", "bf16-e4m3"])
def test_decode_long_and_few(L, dtype, q8):
    run_decode(L, Made(dtype, q8, [20011], 1, 64, seed=3), 4)
    run_decode(L, Made(dtype, q8, [9001, 1, 40], 2, 16, seed=4, k_gain=4.0), 2)


@pytest.mark.parametrize("dtype,q8", [(F32, False), (BF16, False), (F16, True)], ids=["f32", "bf16", "f16-e4m3"])
@pytest.mark.parametrize("hkv,lengths", [(8, [9000]), (8, [3000, 1, 0, 700]), (9, [40, 2500, 33]), (16, [64] * 5)])
def test_decode_rows_in_pieces(L, dtype, q8, hkv, lengths):
    made = Made(dtype, q8, lengths, hkv, 64, seed=hkv)
    first = run_decode(L, made, hkv * (2 if hkv == 8 else 1))
    for _ in range(3):
        again = run_decode(L, made, hkv * (2 if hkv == 8 else 1))
        assert torch.equal(first[1], again[1]) and torch.equal(first[2], again[2])


def widened(made, columns):
    """The same pages behind a table with room for more."""
    table = torch.full((made.table.shape[0], columns), -1, dtype=torch.int32)
    table[:, : made.table.shape[1]] = made.table
    made.table = table
    return made


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
def test_decode_short_rows_behind_a_wide_table(L, dtype, q8):
    # short rows are not cut; whether they are short shows only on the device
    run_decode(L, widened(Made(dtype, q8, [100, 0, 500, 128, 1, 129], 2, 16, seed=41), 700), 8)
    run_decode(L, widened(Made(dtype, q8, [2000, 33] + [100] * 6, 16, 64, seed=42), 300), 32)


@pytest.mark.parametrize("dtype,q8", [(F32, False), (BF16, False), (F16, True)], ids=["f32", "bf16", "f16-e4m3"])
@pytest.mark.parametrize("longest", [120, 6000])
def test_decode_more_rows_than_shares(L, dtype, q8, longest):
    lengths = [longest] + [0, 1, 17, 40] * 16
    run_decode(L, widened(Made(dtype, q8, lengths, 8, 16, seed=43), 400), 8)


@pytest.mark.parametrize("dtype,q8", [(F32, False), (BF16, False), (F16, True)], ids=["f32", "bf16", "f16-e4m3"])
def test_decode_short_rows_beside_long_ones(L, dtype, q8):
    made = Made(dtype, q8, [70, 3] * 7 + [5000] + [0, 3, 170, 1, 129] * 5, 4, 32, seed=66)
    most, least = L.leoam_page_workspace_bytes(made.pages(L, 8)), L.leoam_page_workspace_min(made.pages(L, 8))
    for nbytes in (most, most * 7 // 8, most // 3, least):
        run_decode(L, made, 8, workspace_bytes=max(nbytes // 16 * 16, least))


@pytest.mark.parametrize("dtype,q8", [(F32, False), (BF16, True)], ids=["f32", "bf16-e4m3"])
def test_many_sequences(L, dtype, q8):
    # more sequences than a workgroup has threads: long ones first, in the middle and last
    lengths = [4000] + [0, 1, 17, 40, 16, 130] * 50 + [3001] + [5, 33, 2] * 100 + [2500]
    made = Made(dtype, q8, lengths, 1, 16, seed=68)
    run_decode(L, made, 4)
    new = [min(n, b % 3) for b, n in enumerate(lengths)]
    run_prefill(L, made, 4, new)


@pytest.mark.parametrize("dtype,q8", [(F32, False), (F16, True), (BF16, False)], ids=["f32", "f16-e4m3", "bf16"])
def test_decode_small_workspaces(L, dtype, q8):
    made = Made(dtype, q8, [900, 0, 3, 1500], 2, 32, seed=5)
    pages = made.pages(L, 8)
    least, most = L.leoam_page_workspace_min(pages), L.leoam_page_workspace_bytes(pages)
    assert least <= most
    for nbytes in (least, 3 * least + 16, (least + most) // 32 * 16):
        run_decode(L, made, 8, workspace_bytes=max(nbytes, 16))


def test_decode_bad_page_ids_hold_no_tokens(L):
    made = Made(BF16, False, [100, 64], 1, 16, seed=6)
    made.table[0, 2], made.table[1, 0] = 10 ** 6, -5
    g = torch.Generator().manual_seed(1)
    q = torch.randn(2, 4, 128, generator=g).to(BF16)
    out, lse = torch.empty(2, 4, 128, device="cuda"), torch.empty(2, 4, device="cuda")
    pages = made.pages(L, 4)
    ws = scratch(L.leoam_page_workspace_bytes(pages))
    L.page_attention_decode(pages, q.cuda(), made.k_pages, made.v_pages, None, None, made.table.cuda(), made.seq_len, None, None,
                            SCALE, out, lse, ws)
    for b, pos in ((0, [t for t in range(100) if t // 16 != 2]), (1, list(range(16, 64)))):
        check_rows(L, made, out, lse, [(b, q[b], made.tokens(0, b, pos), made.tokens(1, b, pos))], 2.0 ** -16, 2.0 ** -23)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("scale", [-0.07, 0.0, 1.0])
def test_scales_of_any_sign(L, dtype, q8, scale):
    made = Made(dtype, q8, [70, 33], 2, 16, seed=21)
    run_decode(L, made, 4, scale=scale)
    run_prefill(L, made, 4, [20, 33], scale=scale)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
def test_one_heavy_token_among_many_light_ones(L, dtype, q8):
    # weights down to 2^-26 of the largest, thousands of them: together they count
    made = Made(dtype, q8, [6000], 1, 64, seed=22, k_gain=2.0)
    run_decode(L, made, 2, scale=0.25)
    run_prefill(L, made, 2, [3], scale=0.25)
    run_prefill(L, made, 2, [6000], scale=0.25, rows={0, 64, 3000, 5999})


@pytest.mark.parametrize("dtype,q8", [(BF16, False), (F16, True)], ids=["bf16", "f16-e4m3"])
def test_a_page_listed_twice_counts_twice(L, dtype, q8):
    made = Made(dtype, q8, [50], 1, 16, seed=23)
    idx, count = torch.tensor([[[1, 1, 3, 3]]], dtype=torch.int32), torch.tensor([[4]], dtype=torch.int32)
    run_decode(L, made, 4, keep=(idx, count))


@pytest.mark.parametrize("dtype,q8", [(F32, False), (BF16, False), (BF16, True)], ids=["f32", "bf16", "bf16-e4m3"])
def test_sequences_that_share_pages(L, dtype, q8):
    made = Made(dtype, q8, [96, 40, 96], 2, 16, seed=24)
    made.table[2, :4] = made.table[0, :4]                  # the first 64 tokens of the third are those of the first
    run_decode(L, made, 8)
    run_prefill(L, made, 8, [30, 40, 50])


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
def test_pages_behind_4_gib(L, dtype, q8):
    page, hkv = 256, 1
    size = page * hkv * 128 * (1 if q8 else 4 if dtype == F32 else 2)
    n_pages = (1 << 32) // size + 300
    store = torch.float8_e4m3fn if q8 else dtype
    g = torch.Generator().manual_seed(25)
    k_pages = torch.empty(n_pages, hkv, page, 128, dtype=store, device="cuda")
    v_pages = torch.empty_like(k_pages)
    ks = torch.zeros(n_pages, hkv, device="cuda") if q8 else None
    vs = torch.zeros(n_pages, hkv, device="cuda") if q8 else None
    n, hq = 300, 2
    table = torch.tensor([[n_pages - 1, n_pages - 7]], dtype=torch.int32)
    pages = L.make_pages(1, hq, hkv, 128, n_pages, page, 2, dtype, L.E4M3 if q8 else None)
    x = torch.randn(n, hq + 2 * hkv, 128, generator=g).to(dtype)
    xg = x.cuda()
    q, out, lse = torch.empty(n, hq, 128, dtype=dtype, device="cuda"), torch.empty(n, hq, 128, dtype=dtype, device="cuda"), torch.empty(n, hq, device="cuda")
    off, seq_len = torch.tensor([0, n], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda()
    L.kv_page_append(pages, xg[:, :hq], xg[:, hq: hq + hkv], xg[:, hq + hkv:], off, seq_len, table.cuda(), None, q, k_pages, v_pages, ks, vs)
    ws = scratch(max(L.leoam_page_workspace_bytes(pages, n), L.leoam_page_workspace_bytes(pages)))
    L.page_attention_prefill(pages, q, off, k_pages, v_pages, ks, vs, table.cuda(), seq_len, SCALE, out, lse, ws)
    dout, dlse = torch.empty(1, hq, 128, device="cuda"), torch.empty(1, hq, device="cuda")
    L.page_attention_decode(pages, q[-1:].contiguous(), k_pages, v_pages, ks, vs, table.cuda(), seq_len, None, None, SCALE, dout, dlse, ws)
    used = table[0].long()
    small = lambda t: t[used].cpu() if t is not None else None  # noqa: E731
    cache = R.Cache(small(k_pages), small(v_pages), small(ks), small(vs), dtype)
    K, V = (cache.values(w).transpose(0, 1).reshape(hkv, -1, 128)[:, :n] for w in (0, 1))
    assert torch.isfinite(K).all() and float(K.abs().max()) > 1
    weight = 0.0 if dtype == F32 else HALF[dtype]
    check_rows(L, None, out, lse, [(i, x[i, :hq], K[:, : i + 1], V[:, : i + 1]) for i in (0, 255, 256, n - 1)], weight, HALF[dtype])
    check_rows(L, None, dout, dlse, [(0, x[n - 1, :hq], K, V)], 0.0 if dtype == F32 else 2.0 ** -16, 2.0 ** -23)


# ---- prefill -------------------------------------------------------------------------------------------------

def run_prefill(L, made, hq, new, seed=0, rows=None, workspace_bytes=None, scale=SCALE):
    """new: tokens of each sequence that attend; rows: which of the call's rows are compared (None: all)."""
    g = torch.Generator().manual_seed(seed + 5)
    n = sum(new)
    q = torch.randn(n, hq, 128, generator=g).to(made.dtype)
    pages = made.pages(L, hq)
    off = [0] + [int(x) for x in np.cumsum(new)]
    out = torch.full((n, hq, 128), math.nan, dtype=made.dtype, device="cuda")
    lse = torch.full((n, hq), math.nan, device="cuda")
    nbytes = L.leoam_page_workspace_bytes(pages, n) if workspace_bytes is None else workspace_bytes
    ws = scratch(nbytes)
    L.page_attention_prefill(pages, q.cuda(), torch.tensor(off, dtype=torch.int32).cuda(), made.k_pages, made.v_pages, made.k_scale,
                             made.v_scale, made.table.cuda(), made.seq_len, scale, out, lse, ws)
    torch.cuda.synchronize()
    weight = 0.0 if made.dtype == F32 else HALF[made.dtype]
    for b, m in enumerate(new):
        length = made.lengths[b]
        K, V = made.tokens(0, b, range(length)), made.tokens(1, b, range(length))
        for i in range(m):
            if rows is not None and off[b] + i not in rows:
                continue
            t = length - m + i
            check_rows(L, made, out, lse, [(off[b] + i, q[off[b] + i], K[:, : t + 1], V[:, : t + 1])], weight, HALF[made.dtype], scale)
    return q, out, lse


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_prefill_ragged(L, dtype, q8, group):
    made = Made(dtype, q8, [1, 70, 129, 0, 33, 200], 2, 16, seed=group)
    run_prefill(L, made, 2 * group, [1, 70, 65, 0, 2, 31], seed=group)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("page", [32, 64, 128, 256])
def test_prefill_page_sizes(L, dtype, q8, page):
    made = Made(dtype, q8, [2 * page + 9, 400], 1, page, seed=page)
    run_prefill(L, made, 4, [page + 1, 150], seed=page)


@pytest.mark.parametrize("dtype,q8", [(F32, False), (BF16, False), (F16, True)], ids=["f32", "bf16", "f16-e4m3"])
def test_prefill_few_rows_behind_a_long_context(L, dtype, q8):
    made = Made(dtype, q8, [9000, 20, 6001], 1, 64, seed=7, k_gain=2.0)
    run_prefill(L, made, 4, [5, 1, 9])
    least = L.leoam_page_workspace_min(made.pages(L, 4))
    run_prefill(L, made, 4, [5, 1, 9], workspace_bytes=max(16, least))


@pytest.mark.parametrize("dtype,q8", [(F32, False), (BF16, False), (BF16, True)], ids=["f32", "bf16", "bf16-e4m3"])
def test_prefill_long_prompt(L, dtype, q8):
    made = Made(dtype, q8, [1500, 1023], 1, 128, seed=8)
    some = set(range(0, 2523, 97)) | {1499, 1500, 2522}
    run_prefill(L, made, 2, [1500, 1023], rows=some)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
def test_prefill_bad_page_ids_hold_no_tokens(L, dtype, q8):
    made = Made(dtype, q8, [150, 64], 1, 16, seed=26)
    made.table[0, 2], made.table[0, 7], made.table[1, 0] = 10 ** 6, -3, -5
    g = torch.Generator().manual_seed(6)
    q = torch.randn(70, 4, 128, generator=g).to(dtype)
    out, lse = torch.empty(70, 4, 128, dtype=dtype, device="cuda"), torch.empty(70, 4, device="cuda")
    pages = made.pages(L, 4)
    ws = scratch(L.leoam_page_workspace_bytes(pages, 70))
    L.page_attention_prefill(pages, q.cuda(), torch.tensor([0, 50, 70], dtype=torch.int32).cuda(), made.k_pages, made.v_pages, made.k_scale,
                             made.v_scale, made.table.cuda(), made.seq_len, SCALE, out, lse, ws)
    rows = []
    for b, (r0, r1, n) in enumerate(((0, 50, 150), (50, 70, 64))):
        for r in range(r0, r1):
            pos = [t for t in range(n - (r1 - r) + 1) if not (b == 0 and t // 16 in (2, 7)) and not (b == 1 and t < 16)]
            rows.append((r, q[r], made.tokens(0, b, pos), made.tokens(1, b, pos)))
    check_rows(L, made, out, lse, rows, 0.0 if dtype == F32 else HALF[dtype], HALF[dtype])


@pytest.mark.parametrize("dtype,q8", [(F32, False), (BF16, False), (F16, True)], ids=["f32", "bf16", "f16-e4m3"])
def test_prefill_rows_of_no_sequence_and_of_negative_positions(L, dtype, q8):
    made = Made(dtype, q8, [3, 40], 1, 16, seed=27)
    q = torch.randn(30, 4, 128, generator=torch.Generator().manual_seed(7)).to(dtype)
    out, lse = torch.full((30, 4, 128), 7.0, dtype=dtype, device="cuda"), torch.full((30, 4), 7.0, device="cuda")
    pages = made.pages(L, 4)
    ws = scratch(L.leoam_page_workspace_bytes(pages, 30))
    # the first sequence claims 8 new tokens and holds 3; rows 20 .. 29 belong to nobody
    L.page_attention_prefill(pages, q.cuda(), torch.tensor([0, 8, 20], dtype=torch.int32).cuda(), made.k_pages, made.v_pages, made.k_scale,
                             made.v_scale, made.table.cuda(), made.seq_len, SCALE, out, lse, ws)
    assert (out[20:] == 7).all() and (lse[20:] == 7).all()
    assert (out[:5] == 0).all() and (lse[:5] == -math.inf).all()
    rows = [(5 + i, q[5 + i], made.tokens(0, 0, range(i + 1)), made.tokens(1, 0, range(i + 1))) for i in range(3)]
    rows += [(8 + i, q[8 + i], made.tokens(0, 1, range(29 + i)), made.tokens(1, 1, range(29 + i))) for i in range(12)]
    check_rows(L, made, out, lse, rows, 0.0 if dtype == F32 else HALF[dtype], HALF[dtype])


@pytest.mark.parametrize("dtype,q8", [(F32, False), (BF16, False), (F16, True)], ids=["f32", "bf16", "f16-e4m3"])
def test_prefill_many_units(L, dtype, q8):
    # more units than are shared out, and - with one sequence less - just as many as are
    lengths = [130, 129, 128, 1, 300, 17] * 3
    for n in (18, 3):
        made = Made(dtype, q8, lengths[:n], 32, 16, seed=28)
        run_prefill(L, made, 64, lengths[:n], rows=set(range(0, sum(lengths[:n]), 61)))


@pytest.mark.parametrize("dtype,q8", [(F32, False), (BF16, False), (F16, True)], ids=["f32", "bf16", "f16-e4m3"])
def test_prefill_small_workspaces(L, dtype, q8):
    # too small to share the tiles, for about as many workgroups as there are units, for more
    some = set(range(0, 345, 23)) | {299, 300, 344}
    made = Made(dtype, q8, [900, 40, 300], 8, 32, seed=63)
    most = L.leoam_page_workspace_bytes(made.pages(L, 32), 345)
    for eighths in (1, 2, 5):
        run_prefill(L, made, 32, [300, 40, 5], rows=some, workspace_bytes=most * eighths // 8 // 16 * 16)
    # units of few tiles, more than the workgroups that a part of the workspace is enough for
    made = widened(Made(dtype, q8, [320, 200, 60], 32, 16, seed=64), 200)
    most = L.leoam_page_workspace_bytes(made.pages(L, 128), 345)
    for eighths in (5, 8):
        run_prefill(L, made, 128, [300, 40, 5], rows=some, workspace_bytes=most * eighths // 8 // 16 * 16)


@pytest.mark.parametrize("dtype,q8", [(F32, False), (BF16, False), (F16, True)], ids=["f32", "bf16", "f16-e4m3"])
def test_prefill_short_units_beside_long_ones(L, dtype, q8):
    # shares begin and end before a unit's first tile, within it, behind it
    lengths = [70, 3] * 7 + [5000] + [0, 3, 70, 1, 129] * 5
    new = [min(n, 1 + i % 4) for i, n in enumerate(lengths)]
    made = Made(dtype, q8, lengths, 8, 32, seed=65)
    most = L.leoam_page_workspace_bytes(made.pages(L, 16), sum(new))
    for eighths in (8, 7, 5):
        run_prefill(L, made, 16, new, workspace_bytes=most * eighths // 8 // 16 * 16)


def test_prefill_one_row_each(L):
    made = Made(BF16, True, [1, 300, 0, 17], 2, 16, seed=9)
    g = torch.Generator().manual_seed(2)
    q = torch.randn(4, 8, 128, generator=g).to(BF16)
    out, lse = torch.full((4, 8, 128), math.nan, dtype=BF16, device="cuda"), torch.full((4, 8), math.nan, device="cuda")
    pages = made.pages(L, 8)
    ws = scratch(L.leoam_page_workspace_bytes(pages, 4))
    L.page_attention_prefill(pages, q.cuda(), None, made.k_pages, made.v_pages, made.k_scale, made.v_scale, made.table.cuda(),
                             made.seq_len, SCALE, out, lse, ws)
    check_rows(L, made, out, lse, [(b, q[b], made.tokens(0, b, range(n)), made.tokens(1, b, range(n))) for b, n in enumerate(made.lengths)],
               2.0 ** -8, 2.0 ** -8)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_prefill_later_tokens_that_are_not_finite(L, dtype, q8, bad):
    # a token whose key or value is not finite spoils the rows from its own on, and no earlier one
    made = Made(dtype, q8, [90], 1, 32, seed=10)
    value = math.nan if q8 or bad == "nan" else math.inf
    for pool, pos in ((made.v_pages, 50), (made.k_pages, 70)):
        page = int(made.table[0, pos // 32])
        pool.view(torch.uint8 if q8 else pool.dtype)[page, 0, pos % 32, 9] = 0x7F if q8 else value
    g = torch.Generator().manual_seed(3)
    q = torch.randn(90, 4, 128, generator=g).to(dtype)
    out, lse = torch.empty(90, 4, 128, dtype=dtype, device="cuda"), torch.empty(90, 4, device="cuda")
    pages = made.pages(L, 4)
    ws = scratch(L.leoam_page_workspace_bytes(pages, 90))
    off = torch.tensor([0, 90], dtype=torch.int32).cuda()
    L.page_attention_prefill(pages, q.cuda(), off, made.k_pages, made.v_pages, made.k_scale, made.v_scale, made.table.cuda(), made.seq_len,
                             SCALE, out, lse, ws)
    K, V = made.tokens(0, 0, range(90)), made.tokens(1, 0, range(90))
    weight = 0.0 if dtype == F32 else HALF[dtype]
    check_rows(L, made, out, lse, [(i, q[i], K[:, : i + 1], V[:, : i + 1]) for i in range(50)], weight, HALF[dtype])
    assert not torch.isfinite(out[50:70, :, 9]).any()
    assert torch.isfinite(out[50:70, :, :9]).all() and torch.isfinite(out[50:70, :, 10:]).all()
    if bad == "nan":
        assert torch.isnan(out[70:]).all()


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
def test_prefill_few_rows_and_values_that_are_not_finite(L, dtype, q8):
    # the same where a few rows share a tile's keys out among the waves and their tiles among workgroups
    n, m = 2000, 12
    made = Made(dtype, q8, [n], 1, 32, seed=67)
    for pool, pos in ((made.v_pages, n - 8), (made.k_pages, n - 4)):
        page = int(made.table[0, pos // 32])
        pool.view(torch.uint8 if q8 else pool.dtype)[page, 0, pos % 32, 9] = 0x7F if q8 else math.nan
    g = torch.Generator().manual_seed(3)
    q = torch.randn(m, 4, 128, generator=g).to(dtype)
    out, lse = torch.empty(m, 4, 128, dtype=dtype, device="cuda"), torch.empty(m, 4, device="cuda")
    pages = made.pages(L, 4)
    ws = scratch(L.leoam_page_workspace_bytes(pages, m))
    off = torch.tensor([0, m], dtype=torch.int32).cuda()
    L.page_attention_prefill(pages, q.cuda(), off, made.k_pages, made.v_pages, made.k_scale, made.v_scale, made.table.cuda(), made.seq_len,
                             SCALE, out, lse, ws)
    K, V = made.tokens(0, 0, range(n)), made.tokens(1, 0, range(n))
    weight = 0.0 if dtype == F32 else HALF[dtype]
    check_rows(L, made, out, lse, [(i, q[i], K[:, : n - m + i + 1], V[:, : n - m + i + 1]) for i in range(m - 8)], weight, HALF[dtype])
    assert not torch.isfinite(out[m - 8: m - 4, :, 9]).any()
    assert torch.isfinite(out[m - 8: m - 4, :, :9]).all() and torch.isfinite(out[m - 8: m - 4, :, 10:]).all()
    assert torch.isnan(out[m - 4:]).all()


# ---- together ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,q8", [(BF16, False), (F16, True), (F32, False)], ids=["bf16", "f16-e4m3", "f32"])
@pytest.mark.parametrize("budget", [0, 100])
def test_layer_prompt_then_steps(L, dtype, q8, budget):
    """A prompt, then decode steps, as a serving program runs a layer: against the definition at every step."""
    g = torch.Generator().manual_seed(11)
    B, hq, hkv, page, steps = 3, 8, 2, 32, 4
    prompts = [150, 33, 1]
    table, n_pages = spread([p + steps for p in prompts], page, g)
    rope = L.rope_table(table.shape[1] * page, 64, 1e4)
    seq_len = torch.tensor(prompts, dtype=torch.int32).cuda()
    layer = L.PagedLayer(table.cuda(), seq_len, hq, hkv, n_pages, page, dtype, L.E4M3 if q8 else None, rope=rope.cuda(),
                         token_budget=budget)
    store = layer.k_pages.cpu()
    zero = torch.zeros(n_pages, hkv) if q8 else None
    ref = R.Cache(store, store, zero, zero, dtype)
    held = [0] * B
    for step in range(1 + steps):
        new = prompts if step == 0 else [1] * B
        n = sum(new)
        x = torch.randn(n, hq + 2 * hkv, 128, generator=g).to(dtype)
        xg = x.cuda()
        parts = xg[:, :hq], xg[:, hq: hq + hkv], xg[:, hq + hkv:]
        if step:
            seq_len.add_(1)
            out = layer.step(*parts)
        else:
            lse = torch.empty(n, hq, device="cuda")
            out = layer.prompt(*parts, torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32).cuda(), lse=lse)
        torch.cuda.synchronize()
        assert (layer.status == 0).all()
        row = 0
        for b in range(B):
            m = new[b]
            pos = torch.arange(held[b], held[b] + m)
            xb = x[row: row + m]
            q = R.rotate(xb[:, :hq], rope, pos, 64, False).to(dtype)
            ref.append(R.rotate(xb[:, hq: hq + hkv], rope, pos, 64, False), xb[:, hq + hkv:].float(), held[b], table[b], page)
            held[b] += m
            t = torch.arange(held[b])
            K, V = (ref.values(w)[table[b, t // page].long(), :, t % page].transpose(0, 1) for w in (0, 1))
            weight = 0.0 if dtype == F32 else HALF[dtype] if step == 0 else 2.0 ** -16
            for i in range(m):
                n_seen = held[b] - m + i + 1
                if step == 0 or not budget:
                    half = HALF[dtype] if step == 0 else 2.0 ** -23
                    check_rows(L, None, out, lse if step == 0 else layer.lse, [(row + i, q[i], K[:, :n_seen], V[:, :n_seen])], weight, half)
                    continue
                G = hq // hkv
                for h in range(hkv):
                    # the kept pages: by upper bound of q.k over the page, whole pages while they fit the budget
                    tokens = []
                    score = []
                    for p in range(-(-n_seen // page)):
                        kp = K[h, p * page: min(n_seen, (p + 1) * page)]
                        hi, lo = kp.amax(0), kp.amin(0)
                        qq = q[i, h * G: (h + 1) * G].double()
                        score.append(float(torch.maximum(qq * hi, qq * lo).sum(-1).max()))
                    left = budget
                    for p in sorted(range(len(score)), key=lambda p: (-score[p], p)):
                        size = min(n_seen, (p + 1) * page) - p * page
                        if size > left:
                            break
                        left -= size
                        tokens += list(range(p * page, p * page + size))
                    tokens.sort()
                    check_rows(L, None, out[row + i, h * G: (h + 1) * G][None], layer.lse[row + i, h * G: (h + 1) * G][None],
                               [(0, q[i, h * G: (h + 1) * G], K[h: h + 1, tokens], V[h: h + 1, tokens])], weight, 2.0 ** -23)
            row += m


def test_layer_step_replays_from_a_graph(L):
    """The captured step advances its own length; every replay equals the same step run eagerly."""
    g = torch.Generator().manual_seed(12)
    B, hq, hkv, page, steps = 2, 8, 2, 16, 6
    prompts = [45, 200]

    def fresh():
        gg = torch.Generator().manual_seed(13)
        table, n_pages = spread([p + steps + 2 for p in prompts], page, gg)
        seq_len = torch.tensor(prompts, dtype=torch.int32).cuda()
        layer = L.PagedLayer(table.cuda(), seq_len, hq, hkv, n_pages, page, BF16, L.E4M3, rope=L.rope_table(table.shape[1] * page, 128).cuda(),
                             token_budget=96)
        x = torch.randn(sum(prompts), hq + 2 * hkv, 128, generator=gg).to(BF16).cuda()
        layer.prompt(x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:], torch.tensor([0, 45, 245], dtype=torch.int32).cuda())
        return layer, seq_len
    xs = [torch.randn(B, hq + 2 * hkv, 128, generator=g).to(BF16).cuda() * (1 + s) for s in range(steps)]
    split = lambda x: (x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:])  # noqa: E731
    layer, seq_len = fresh()
    want = []
    for x in xs:
        seq_len.add_(1)
        layer.step(*split(x))
        torch.cuda.synchronize()
        want.append((layer.out.clone(), layer.lse.clone(), layer.k_pages.view(torch.uint8).clone(), layer.k_scale.clone(), layer.sel_idx.clone()))
    layer, seq_len = fresh()
    x = xs[0].clone()
    q_out = torch.empty(B, hq, 128, dtype=BF16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.attend(q_out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        seq_len.add_(1)
        layer.step(*split(x), q_out=q_out)
    for s in range(steps):
        x.copy_(xs[s])
        graph.replay()
        torch.cuda.synchronize()
        got = (layer.out, layer.lse, layer.k_pages.view(torch.uint8), layer.k_scale, layer.sel_idx)
        for a, b in zip(got, want[s]):
            assert torch.equal(a, b), s
        torch.randn(1000, device="cuda").sum()


def test_same_call_twice_gives_the_same_bits(L):
    made = Made(BF16, True, [3000, 17, 800], 2, 32, seed=14)
    a = run_decode(L, made, 8)
    b = run_decode(L, made, 8)
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
    a = run_prefill(L, made, 8, [40, 17, 300], rows=set())
    b = run_prefill(L, made, 8, [40, 17, 300], rows=set())
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])


def test_two_calls_at_once(L):
    """Two streams, each with a workspace of its own, against the calls one after the other."""
    made = Made(BF16, True, [5000, 900, 70], 8, 32, seed=29)
    pages = made.pages(L, 16)
    g = torch.Generator().manual_seed(8)
    q = torch.randn(3, 16, 128, generator=g).to(BF16).cuda()
    table = made.table.cuda()
    off = torch.tensor([0, 1, 2, 3], dtype=torch.int32).cuda()

    def both(streams):
        torch.cuda.synchronize()
        res = []
        for st in streams:
            out, lse, p = torch.empty(3, 16, 128, device="cuda"), torch.empty(3, 16, device="cuda"), torch.empty(3, 16, 128, dtype=BF16, device="cuda")
            res.append((out, lse, p, scratch(L.leoam_page_workspace_bytes(pages, 3))))
        torch.cuda.synchronize()
        for _ in range(5):
            for st, (out, lse, p, ws) in zip(streams, res):
                L.page_attention_decode(pages, q, made.k_pages, made.v_pages, made.k_scale, made.v_scale, table, made.seq_len, None, None, SCALE, out, lse, ws, st)
                L.page_attention_prefill(pages, q, off, made.k_pages, made.v_pages, made.k_scale, made.v_scale, table, made.seq_len, SCALE, p, None, ws, st)
        torch.cuda.synchronize()
        return res
    want = both([torch.cuda.current_stream()])[0]
    for got in both([torch.cuda.Stream(), torch.cuda.Stream()]):
        for a, b in zip(got[:3], want[:3]):
            assert torch.equal(a, b)


def test_prompt_replays_from_a_graph(L):
    made = Made(BF16, False, [700, 90], 2, 64, seed=30)
    pages = made.pages(L, 8)
    g = torch.Generator().manual_seed(9)
    new = [300, 50]
    qs = [torch.randn(350, 8, 128, generator=g).to(BF16).cuda() for _ in range(3)]
    q, out, lse = qs[0].clone(), torch.empty(350, 8, 128, dtype=BF16, device="cuda"), torch.empty(350, 8, device="cuda")
    off, table = torch.tensor([0, 300, 350], dtype=torch.int32).cuda(), made.table.cuda()
    ws = scratch(L.leoam_page_workspace_bytes(pages, sum(new)))

    def call():
        L.page_attention_prefill(pages, q, off, made.k_pages, made.v_pages, None, None, table, made.seq_len, SCALE, out, lse, ws)
    want = []
    for x in qs:
        q.copy_(x)
        call()
        torch.cuda.synchronize()
        want.append((out.clone(), lse.clone()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in (2, 0, 1, 1):
        q.copy_(qs[i])
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])


def test_refused_tensors(L):
    """What a tensor's type, size and layout must be is looked at before anything is launched."""
    made = Made(BF16, False, [50], 2, 16, seed=31)
    pages = made.pages(L, 8)
    q, out, lse = torch.zeros(1, 8, 128, dtype=BF16, device="cuda"), torch.full((1, 8, 128), 7.0, device="cuda"), torch.empty(1, 8, device="cuda")
    table, ws = made.table.cuda(), scratch(L.leoam_page_workspace_bytes(pages))
    good = [pages, q, made.k_pages, made.v_pages, None, None, table, made.seq_len, None, None, SCALE, out, lse, ws]
    bad = {1: [q.half(), q[:, :4].contiguous(), q.cpu(), None], 2: [made.k_pages[:-1], made.k_pages.transpose(2, 3), made.k_pages.half()],
           6: [table.long(), table[:, :-1].contiguous()], 7: [made.seq_len.long(), made.seq_len[:0]], 11: [out.bfloat16(), out[:, 1:]],
           12: [lse[:, 1:], lse.double()], 4: [torch.zeros(3, device="cuda", dtype=torch.int32)]}
    for i, values in bad.items():
        for v in values:
            with pytest.raises(ValueError):
                L.page_attention_decode(*good[:i], v, *good[i + 1:])
    with pytest.raises(L.LeoamError) as e:
        L.page_attention_decode(*good[:13], ws[:16])
    assert e.value.status == -4
    torch.cuda.synchronize()
    assert (out == 7).all()
    L.page_attention_decode(*good)
    kv = torch.zeros(3, 2, 128, dtype=BF16, device="cuda")
    off = torch.tensor([0, 3], dtype=torch.int32).cuda()
    call = [pages, None, kv, kv, off, made.seq_len, table, None, None, made.k_pages, made.v_pages]
    for i, values in {2: [kv[:2], kv[:, :1], kv.float(), kv[..., ::2], kv.transpose(0, 1)], 4: [off[:1], off.long()], 1: [kv]}.items():
        for v in values:
            with pytest.raises(ValueError):
                L.kv_page_append(*call[:i], v, *call[i + 1:])


def test_another_stream(L):
    made = Made(F16, False, [500, 70], 2, 64, seed=15)
    pages = made.pages(L, 4)
    q = torch.randn(2, 4, 128, generator=torch.Generator().manual_seed(1)).to(F16).cuda()
    outs = []
    for stream in (None, torch.cuda.Stream()):
        out, lse = torch.empty(2, 4, 128, device="cuda"), torch.empty(2, 4, device="cuda")
        ws = scratch(L.leoam_page_workspace_bytes(pages))
        table = made.table.cuda()
        torch.cuda.synchronize()
        L.page_attention_decode(pages, q, made.k_pages, made.v_pages, None, None, table, made.seq_len, None, None, SCALE, out, lse, ws, stream)
        torch.cuda.synchronize()
        outs.append(out)
    assert torch.equal(*outs)


@pytest.mark.parametrize("as_handle", [False, True], ids=["stream", "handle"])
def test_layer_on_another_stream_keeps_its_temporaries(L, as_handle):
    """The rotated queries of a step are freed while its kernels wait: whoever allocates next must not get them."""
    g = torch.Generator().manual_seed(61)
    B, hq, hkv, page = 4, 32, 8, 64
    table, n_pages = spread([200] * B, page, g)
    seq_len = torch.tensor([100, 7, 64, 130], dtype=torch.int32).cuda()
    off = torch.tensor([0, 100, 107, 171, 301], dtype=torch.int32).cuda()
    prompt = torch.randn(301, hq + 2 * hkv, 128, generator=g).to(BF16).cuda()
    token = torch.randn(B, hq + 2 * hkv, 128, generator=g).to(BF16).cuda()
    parts = lambda x: (x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:])
    want = got = None
    for other in (False, True):
        layer = L.PagedLayer(table.cuda(), seq_len.clone(), hq, hkv, n_pages, page, BF16)
        stream = torch.cuda.Stream() if other else None
        torch.cuda.synchronize()
        if other:
            with torch.cuda.stream(stream):
                torch.cuda._sleep(20_000_000)      # (some 10 ms)
        handle = stream.cuda_stream if other and as_handle else stream
        a = layer.prompt(*parts(prompt), off, stream=handle)
        fill = [torch.full((301, hq, 128), math.nan, dtype=BF16, device="cuda") for _ in range(4)] if other else []
        torch.cuda.synchronize()
        layer.seq_len.add_(1)
        torch.cuda.synchronize()
        if other:
            with torch.cuda.stream(stream):
                torch.cuda._sleep(20_000_000)
        b = layer.step(*parts(token), stream=handle)
        fill += [torch.full((B, hq, 128), math.nan, dtype=BF16, device="cuda") for _ in range(4)] if other else []
        torch.cuda.synchronize()
        want, got = got, (a, b.clone())
        assert all(torch.isnan(f).all() for f in fill)      # (nor may the step's kernels write to what others were given)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_layer_prompts_that_grow_share_a_workspace(L):
    g = torch.Generator().manual_seed(62)
    hq, hkv, page, lengths = 32, 8, 64, list(range(8, 2400, 230))
    table, n_pages = spread([lengths[-1]], page, g)
    seq_len = torch.zeros(1, dtype=torch.int32).cuda()
    layer = L.PagedLayer(table.cuda(), seq_len, hq, hkv, n_pages, page, BF16)
    x = torch.randn(lengths[-1], hq + 2 * hkv, 128, generator=g).to(BF16).cuda()
    parts = lambda n: (x[:n, :hq], x[:n, hq: hq + hkv], x[:n, hq + hkv:])
    for n in lengths:
        seq_len.fill_(n)
        layer.prompt(*parts(n), torch.tensor([0, n], dtype=torch.int32).cuda())
    assert sum(w.numel() for w in layer.prompt_workspaces) <= 2 * 72 << 20
