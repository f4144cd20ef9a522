"""page_weight_add, page_evict_select and kv_page_move, each against its definition in include/leoam.h written out plainly in 64 bits, and
a run of them together.

Tolerance of a weight: z = scale * q.k is within dz = 2^-16 A of its value (A as in tests/test_gpu_paged.py), the given lse is turned
to the base of 2 by a product and subtracted in one more operation, off by at most 2^-23 (|z| + |lse|) in all, exp2 by 2^-22, and the
sum of n terms by n 2^-24 of it; decay * weight_before + that is one operation.  Selections and moves are exact."""
import math

import numpy as np
import pytest
import torch

from tests import paged_reference as R
from tests.test_gpu_paged import BF16, F16, F32, KIND_IDS, KINDS, SCALE, L, Made, check, check_rows, scratch, spread  # noqa: F401

pytestmark = pytest.mark.gpu
i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731


# ---- page_weight_add -------------------------------------------------------------------------------------------

def run_weigh(L, made, hq, rows, seed=0, decay=0.75, before=True, scale=SCALE, lse_of=None, table=None, again=None, ids=True):
    """rows: new rows of each sequence (None: one each, without new_off)."""
    B, hkv, G = len(made.lengths), made.hkv, hq // made.hkv
    g = torch.Generator().manual_seed(seed + 5)
    m = [1] * B if rows is None else rows
    n = sum(m)
    table = made.table if table is None else table
    cap = table.shape[1] * made.page
    q = torch.randn(n, hq, 128, generator=g).to(made.dtype)
    starts = [sum(m[:b]) for b in range(B + 1)]
    lse = torch.rand(n, hq, generator=g) * 3 + 1.0
    if lse_of:
        lse_of(lse)
    old = torch.rand(B, hkv, cap, generator=g)
    seen = [x + 3 * b for b, x in enumerate(made.lengths)]
    weight, token_id = torch.full((B, hkv, cap), 77.0, device="cuda"), torch.full((B, hkv, cap), -7, dtype=torch.int32, device="cuda")
    pages = made.pages(L, hq)
    off = None if rows is None else i32(starts)
    call = lambda: L.page_weight_add(  # noqa: E731
        pages, qg, off, made.k_pages, made.k_scale, tg, made.seq_len, scale, lg, decay, og, weight, sg if ids else None, token_id if ids else None)
    qg, tg, lg, og, sg = q.cuda(), table.cuda(), lse.cuda(), old.cuda() if before else None, i32(seen)
    call()
    torch.cuda.synchronize()
    got, got_ids = weight.cpu().double(), token_id.cpu()
    for b, len_b in enumerate(made.lengths):
        first = len_b - m[b]
        assert (got[b, :, len_b:] == 77.0).all()
        numbers = torch.arange(cap) + seen[b] - len_b
        mine = (torch.arange(cap) < len_b) & (torch.arange(cap) >= first) & ids
        assert torch.equal(got_ids[b], torch.where(mine, numbers, -7).int().expand(hkv, cap))
        if len_b == 0:
            continue
        there = torch.tensor([0 <= int(table[b, t // made.page]) < made.n_pages for t in range(len_b)])
        K = torch.zeros(hkv, len_b, 128, dtype=torch.float64)
        K[:, there] = made.tokens(0, b, torch.nonzero(there).flatten())
        places = first + torch.arange(m[b])
        sees = (torch.arange(len_b)[None] <= places[:, None]) & there
        qb, lb = q[starts[b]: starts[b + 1]].double(), lse[starts[b]: starts[b + 1]].double()
        for h in range(hkv):
            mine_q = qb[:, h * G: (h + 1) * G]
            z = torch.einsum("rgd,td->rgt", mine_q, K[h]) * scale
            reach = float(torch.einsum("rgd,td->rgt", mine_q.abs(), K[h].abs()).max()) * abs(scale) if m[b] else 0.0
            lh = lb[:, h * G: (h + 1) * G]
            p = torch.where(sees[:, None] & (lh > -math.inf)[..., None], torch.exp(z - lh.clamp(min=-1e30)[..., None]), torch.zeros(()).double())
            add = p.sum((0, 1))
            want = add.clone()
            if before:
                want[: max(first, 0)] += decay * old[b, h, : max(first, 0)].double()
            top = float(lh[torch.isfinite(lh)].abs().max()) if torch.isfinite(lh).any() else 0.0
            tol = add * (2.0 ** -16 * reach + 2.0 ** -23 * (reach + top) * 2 + 2.0 ** -21 + m[b] * G * 2.0 ** -24) + 2.0 ** -22 * want + 1e-30
            check(f"weights of sequence {b}, head {h}", got[b, h, :len_b], want, tol)
    if again:
        again(call, weight)
    return weight, token_id


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_weigh_one_row_each(L, dtype, q8, group):
    made = Made(dtype, q8, [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 255, 257, 700], 2, 16, seed=group)
    run_weigh(L, made, 2 * group, None, seed=group)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("many", [False, True], ids=["few rows", "many rows"])
def test_weigh_ragged_rows(L, dtype, q8, group, many):
    lengths = [0, 1, 70, 64, 300, 513, 40]
    rows = [0, 1, 70, 3, 5, 200, 0] if many else [0, 1, 2, 3, 0, 5, 1]
    run_weigh(L, Made(dtype, q8, lengths, 3, 32, seed=group), 3 * group, rows, seed=group, before=group != 2)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("page", [64, 128, 256])
def test_weigh_page_sizes(L, dtype, q8, page):
    run_weigh(L, Made(dtype, q8, [5 * page + 7, page, 1, 1025], 2, page, seed=page), 8, [100, 1, 1, 40], seed=page, decay=0.0)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("rows,history", [(4, 700), (5, 700), (33, 1200), (65, 900), (65, 0), (130, 800), (150, 10)])
def test_weigh_rows_behind_a_history(L, dtype, q8, rows, history):
    run_weigh(L, Made(dtype, q8, [rows + history, rows], 2, 32, seed=rows), 8, [rows, rows], seed=rows)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("batch,rows,history", [(8, 300, 0), (20, 100, 0), (8, 70, 250), (4, 300, 20)])
def test_weigh_rows_of_many_heads(L, dtype, q8, batch, rows, history):
    """Every number of waves to a stretch of keys, and stretches of either size."""
    lengths = [rows + history - b % 3 for b in range(batch)]
    run_weigh(L, Made(dtype, q8, lengths, 8, 32, seed=rows), 32, [rows - b % 3 for b in range(batch)], seed=rows)


def test_weigh_long_prompt(L):
    run_weigh(L, Made(BF16, False, [1500], 1, 64, seed=2), 8, [1500], before=False)


@pytest.mark.parametrize("rows", [None, [1, 60, 2]])
def test_weigh_rows_that_attended_to_nothing_and_missing_pages(L, rows):
    made = Made(F16, False, [40, 90, 33], 2, 16, seed=3)
    table = made.table.clone()
    table[0, 1], table[1, 0], table[2] = -1, made.n_pages, 1 << 30

    def nothing(lse):
        lse[0, ::2] = -math.inf
        lse[-1] = -math.inf
    run_weigh(L, made, 4, rows, table=table, lse_of=nothing)


def test_weigh_scales_of_any_sign_and_without_numbers(L):
    made = Made(F32, False, [40, 90], 1, 16, seed=4)
    for scale in (-0.2, 0.0, 1.5):
        run_weigh(L, made, 2, [3, 4], scale=scale, ids=False)


def test_weigh_rows_of_negative_places_and_lists_that_descend(L):
    # more rows than tokens: those before the first token see nothing; a list that descends brings no rows
    made = Made(BF16, False, [3, 20], 1, 16, seed=5)
    q = torch.randn(8, 2, 128, generator=torch.Generator().manual_seed(5)).to(BF16).cuda()
    lse, pages = torch.zeros(8, 2).cuda(), made.pages(L, 2)
    one, two = torch.full((2, 1, 48), 7.0).cuda(), torch.full((2, 1, 48), 7.0).cuda()
    pages.max_pages = 3
    table = torch.full((2, 3), -1, dtype=torch.int32)
    table[:, : made.table.shape[1]] = made.table
    L.page_weight_add(pages, q, i32([0, 8, 8]), made.k_pages, None, table.cuda(), made.seq_len, SCALE, lse, 1.0, None, one)
    L.page_weight_add(pages, q[5:].contiguous(), i32([0, 3, 3]), made.k_pages, None, table.cuda(), made.seq_len, SCALE, lse[5:].contiguous(), 1.0,
                      None, two)
    # The two calls bring different numbers of rows, so a token's sum may be taken in another order.  It has at most six terms that are
    # not zero (three rows, two heads), all positive and the same in both calls: five additions, each off by at most 2^-24 of the sum, so
    # two orders differ by at most 10 * 2^-24 of it, below 2^-20.
    assert ((one - two).abs() <= 2.0 ** -20 * one).all() and (one[0, 0, :3] > 0).all() and (one[1, 0, :20] == 0).all()
    L.page_weight_add(pages, q, i32([5, 2, 99]), made.k_pages, None, table.cuda(), made.seq_len, SCALE, lse, 0.5, one, two)
    assert torch.equal(two[0, 0, :3], one[0, 0, :3] * 0.5) and (two[1, 0, :20] == 0).all()


def test_weigh_in_place_repeats_and_replays(L):
    made = Made(BF16, True, [300, 1000, 64], 2, 32, seed=6)

    def again(call, weight):
        first = weight.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for i in range(3):
            weight[:, :, :64] = float(i)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(weight, first)
            call()
            assert torch.equal(weight, first)
    run_weigh(L, made, 8, [20, 100, 64], again=again)
    # in place
    pages, w = made.pages(L, 8), torch.rand(3, 2, made.table.shape[1] * 32).cuda()
    q, lse, out = torch.randn(3, 8, 128).to(BF16).cuda(), torch.rand(3, 8).cuda() + 2, torch.zeros_like(w)
    args = (pages, q, None, made.k_pages, made.k_scale, made.table.cuda(), made.seq_len, SCALE, lse, 0.9)
    L.page_weight_add(*args, w, out)
    L.page_weight_add(*args, w, w)
    for b, n in enumerate(made.lengths):
        assert torch.equal(w[b, :, :n], out[b, :, :n])


def test_weigh_short_sequences_of_a_large_table(L):
    # more blocks of places than workgroups: the grid goes round
    page, max_pages, B = 256, 20000, 8
    lengths = [5, 900, 0, 70000, 257, 1, 30, 64]
    n_pages = sum(-(-n // page) for n in lengths)
    table, at = torch.full((B, max_pages), -1, dtype=torch.int32), 0
    for b, n in enumerate(lengths):
        k = -(-n // page)
        table[b, :k] = torch.arange(at, at + k)
        at += k
    K = torch.randn(n_pages, 1, page, 128).to(F16)
    pages = L.make_pages(B, 1, 1, 128, n_pages, page, max_pages, F16)
    q, lse = torch.randn(B, 1, 128).to(F16), torch.full((B, 1), 4.0)
    weight = torch.full((B, 1, max_pages * page), -1.0, device="cuda")
    L.page_weight_add(pages, q.cuda(), None, K.cuda(), None, table.cuda(), i32(lengths), SCALE, lse.cuda(), 1.0, None, weight)
    for b, n in enumerate(lengths):
        k = K[table[b, : -(-n // page)].long(), 0].reshape(-1, 128)[:n].double()
        want = torch.exp(k @ q[b, 0].double() * SCALE - 4.0)
        reach = float((k.abs() @ q[b, 0].double().abs()).max() if n else 0) * SCALE
        check(f"sequence {b}", weight[b, 0, :n], want, want * (2.0 ** -16 * reach + 2.0 ** -20))
        assert (weight[b, 0, n:] == -1.0).all()


# ---- page_evict_select ------------------------------------------------------------------------------------------

def order_of(weight, ids, n, seen, first, recent):
    t = np.arange(n)
    guarded = (t < first) | (ids[:n].astype(np.int64) >= seen - recent)
    w = weight[:n].astype(np.float64)
    w = np.where(guarded, 0.0, w)
    nan = np.isnan(w)
    return np.lexsort((t, -np.where(nan, 0.0, w), nan, ~guarded))


def run_select(L, lengths, keeps, hkv=2, page=64, first=None, recent=0, ids=True, make=None, m_max=None, seed=0):
    B = len(lengths)
    rng = np.random.default_rng(seed)
    max_pages = -(-max(lengths) // page) + 1
    cap = max_pages * page
    weight = rng.lognormal(0, 2, (B, hkv, cap)).astype(np.float32)
    token_id = np.tile(np.arange(cap, dtype=np.int32), (B, hkv, 1))
    for b in range(B):
        for h in range(hkv):
            rng.shuffle(token_id[b, h, : lengths[b]])
    if make:
        make(weight, token_id)
    most = m_max or max(1, max(min(k, n - k) for n, k in zip(lengths, keeps)))
    pages = L.make_pages(B, hkv, hkv, 128, 4, page, max_pages, BF16)
    moves = torch.full((B, hkv, most, 2), -9, dtype=torch.int32, device="cuda")
    count, new_len, status = torch.full((B, hkv), -9, dtype=torch.int32, device="cuda"), i32([-9] * B), i32([-9] * B)
    wg, ig = torch.from_numpy(weight).cuda(), torch.from_numpy(token_id).cuda() if ids else None
    ws = scratch(L.leoam_page_evict_workspace_bytes(pages))
    call = lambda: L.page_evict_select(pages, wg, ig, seen, lens, kept, firsts, recent, moves, count, new_len, status, ws)  # noqa: E731
    seen, lens, kept, firsts = i32(lengths) if ids else None, i32(lengths), i32(keeps), i32(first) if first is not None else None
    call()
    torch.cuda.synchronize()
    mv, ct = moves.cpu().numpy(), count.cpu().numpy()
    for b, (n, keep) in enumerate(zip(lengths, keeps)):
        if keep < n and min(keep, n - keep) > most:
            assert int(status[b]) == 1 and int(new_len[b]) == n and (ct[b] == 0).all() and (mv[b] == -9).all()
            continue
        assert int(status[b]) == 0 and int(new_len[b]) == min(n, keep)
        for h in range(hkv):
            if keep >= n:
                assert ct[b, h] == 0 and (mv[b, h] == -9).all()
                continue
            number = token_id[b, h] if ids else np.arange(cap)
            stay = np.sort(order_of(weight[b, h], number, n, n, first[b] if first is not None else 0, recent)[:keep])
            free, behind = np.setdiff1d(np.arange(keep), stay), stay[stay >= keep]
            assert ct[b, h] == len(free)
            assert (mv[b, h, : len(free), 0] == free).all() and (mv[b, h, : len(free), 1] == behind).all()
            assert (mv[b, h, len(free):] == -9).all()
    return call, moves, count


@pytest.mark.parametrize("ids", [True, False], ids=["numbers", "places"])
def test_select_lengths(L, ids):
    lengths = [1, 2, 63, 64, 65, 100, 1000, 1023, 1024, 1025, 5000, 64, 64, 0]
    keeps = [0, 1, 32, 63, 64, 99, 1, 1000, 512, 1024, 300, 64, 100, 5]
    run_select(L, lengths, keeps, first=[0, 1, 4, 4, 4, 4, 1, 4, 4, 4, 4, 4, 4, 4], recent=10, ids=ids)


@pytest.mark.parametrize("n", [8191, 8193, 16383, 16384, 16385, 20000, 32703, 32769, 50000, 131072])
def test_select_long_rows(L, n):
    run_select(L, [n, n - 1, n // 2], [n // 3, n - 2, n // 2 - 1], hkv=3, first=[64, 0, 1], recent=1000, seed=n)


@pytest.mark.parametrize("n", [300, 20000, 40000])
def test_select_ties_and_special_weights(L, n):
    def make(w, ids):
        w[0] = 1.0                                                      # all the same: by place
        w[1] = np.float32(0.0)
        w[1, :, ::2] = np.float32(-0.0)                                 # the same, too
        w[2, :, ::3] = np.nan
        w[3, :, ::5], w[3, :, 1::5], w[3, :, 2::7] = np.inf, -np.inf, -3.0
        w[4] = np.nan
        w[5] = np.round(w[5])
        w[6] = np.frombuffer(np.arange(w[6].size, dtype=np.uint32).tobytes(), np.float32).reshape(w[6].shape)      # subnormals
    for part in (2, 3, 10):
        run_select(L, [n] * 7, [n // part] * 7, make=make, recent=7, first=[3] * 7)
        run_select(L, [n] * 7, [n - n // part] * 7, make=make, ids=False)


@pytest.mark.parametrize("n", [40000, 65400, 70000])
def test_select_many_long_rows(L, n):
    lengths = [n, 40, n - 1, 33000] + 28 * [700]
    run_select(L, lengths, [n // 2, 39, n - 300, 1] + 28 * [5], hkv=4, first=[4] * 3 + [0] * 29, recent=100, seed=n)
    # fewer of them: by parts, long and short
    run_select(L, lengths[:20], [n // 2, 39, n - 300, 1] + 16 * [5], hkv=4, first=[4] * 3 + [0] * 17, recent=100, seed=n)


@pytest.mark.parametrize("n", [50, 700])
def test_select_many_short_rows(L, n):
    """More rows than fit the card at a time."""
    lengths = [n - b % 7 for b in range(140)]
    run_select(L, lengths, [n // 2 + b % 3 for b in range(140)], hkv=4, first=[b % 5 for b in range(140)], recent=9, seed=n)


def test_select_more_protected_than_stay(L):
    run_select(L, [500] * 4, [100] * 4, first=[100, 101, 500, 90], recent=30)
    run_select(L, [500] * 4, [100] * 4, first=[0, 99, 100, 1 << 30], recent=1 << 30, ids=False)
    run_select(L, [500] * 4, [100] * 4, first=[-5, 0, 0, 0], recent=500)


def test_select_lists_that_are_too_short_and_lengths_that_do_not_fit(L):
    run_select(L, [500, 300, 500], [450, 100, 200], m_max=50)
    pages = L.make_pages(4, 1, 1, 128, 4, 16, 4, BF16)
    w, moves, count = torch.zeros(4, 1, 64).cuda(), torch.zeros(4, 1, 8, 2, dtype=torch.int32).cuda(), i32([[9]] * 4)
    new_len, status = i32([-1] * 4), i32([-1] * 4)
    L.page_evict_select(pages, w, None, None, i32([65, -1, 64, 20]), i32([60, 0, -1, 30]), None, 0, moves, count, new_len, status,
                        scratch(L.leoam_page_evict_workspace_bytes(pages)))
    assert status.tolist() == [1, 1, 1, 0] and new_len.tolist() == [65, -1, 64, 20] and (count == 0).all()


def test_select_replays_from_a_graph(L):
    call, moves, count = run_select(L, [3000, 40000], [1000, 39000], recent=20)      # (four launches)
    want = moves.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        moves.fill_(-9)
        count.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(moves, want)
        call()
        assert torch.equal(moves, want)


# ---- kv_page_move -----------------------------------------------------------------------------------------------

class Moving:
    """A cache with its weights, numbers, abstracts and boundaries, and the same in 64 bits."""

    def __init__(self, L, dtype, q8, lengths, hkv, page, seed=0, bounds=True, gains=None):
        self.L, self.made, self.B, self.hkv, self.page = L, Made(dtype, q8, lengths, hkv, page, seed=seed), len(lengths), hkv, page
        made, g = self.made, torch.Generator().manual_seed(seed + 1)
        if q8 and gains:      # pages of other magnitudes, by their scales
            for which, s in enumerate((made.k_scale, made.v_scale)):
                f = 2.0 ** torch.randint(*gains, s.shape, generator=g).float()
                s.mul_(f.cuda())
                made.cache.scale[which].mul_(f.double())
        self.cap = made.table.shape[1] * page
        self.weight = torch.rand(self.B, hkv, self.cap, generator=g).cuda()
        self.ids = torch.randint(0, 1 << 20, (self.B, hkv, self.cap), generator=g).int().cuda()
        self.abstract = self.off = self.n_chunks = None
        if bounds:
            P = made.table.shape[1]
            self.abstract = torch.full((self.B, hkv, P, 2, 128), 55.0, dtype=dtype, device="cuda")
            self.off = torch.full((self.B, P + 1), -7, dtype=torch.int32, device="cuda")
            self.n_chunks = torch.full((self.B,), -7, dtype=torch.int32, device="cuda")

    def random_moves(self, keeps, seed=0, share=0.5):
        """Per (sequence, kv head) some of the places below the kept length and as many of those behind it."""
        rng = np.random.default_rng(seed)
        lists = {}
        for b, (n, keep) in enumerate(zip(self.made.lengths, keeps)):
            for h in range(self.hkv):
                k = 0 if keep >= n else int(rng.integers(0, int(min(keep, n - keep) * share) + 1))
                lists[b, h] = list(zip(np.sort(rng.choice(keep, k, replace=False)) if k else [], keep + np.sort(rng.choice(n - keep, k, replace=False)) if k else []))
        return lists

    def run(self, keeps, lists, extra=None, verify=True):
        made, page, hkv = self.made, self.page, self.hkv
        most = max(1, max(len(x) for x in lists.values())) + 2
        moves, count = np.full((self.B, hkv, most, 2), -9, np.int32), np.zeros((self.B, hkv), np.int32)
        for (b, h), pairs in lists.items():
            count[b, h] = len(pairs)
            for i, (to, src) in enumerate(pairs):
                moves[b, h, i] = to, src
        before_w, before_i = self.weight.cpu(), self.ids.cpu()
        pages = made.pages(self.L, self.hkv)
        args = (pages, torch.from_numpy(moves).cuda(), torch.from_numpy(count).cuda(), made.seq_len, i32(keeps), made.table.cuda(), made.k_pages,
                made.v_pages, made.k_scale, made.v_scale, self.weight, self.ids, self.abstract, self.off, self.n_chunks)
        call = lambda: self.L.kv_page_move(*args)  # noqa: E731
        call()
        torch.cuda.synchronize()
        if verify:
            self.expect(keeps, lists, before_w, before_i)
        return call

    def expect(self, keeps, lists, w, ids):
        made, page, hkv, cache = self.made, self.page, self.hkv, self.made.cache
        table = made.table
        old = [cache.values(0).clone(), cache.values(1).clone()]
        ok = lambda b, t: 0 <= int(table[b, t // page]) < made.n_pages  # noqa: E731
        abstract = None if self.abstract is None else torch.full(self.abstract.shape, 55.0, dtype=torch.float64)
        for b, (n, keep) in enumerate(zip(made.lengths, keeps)):
            for h in range(hkv):
                pairs = [(int(t), int(f)) for t, f in lists[b, h] if keep < n and 0 <= t < keep <= f < n and ok(b, t) and ok(b, f)]
                for to, src in pairs:
                    w[b, h, to], ids[b, h, to] = w[b, h, src].clone(), ids[b, h, src].clone()
                for which in (0, 1):
                    pool = cache.pool[which]
                    for p in sorted({to // page for to, _ in pairs}):
                        phys, mine = int(table[b, p]), [(t, f) for t, f in pairs if t // page == p]
                        rows = torch.stack([old[which][int(table[b, f // page]), h, f % page] for _, f in mine])
                        at = torch.tensor([t % page for t, _ in mine])
                        if not made.q8:
                            pool[phys, h, at] = rows
                            continue
                        was = float(cache.scale[which][phys, h])
                        now = max(was, R.scale_for(rows, made.dtype))
                        if now > was:
                            pool[phys, h] = R.encode(pool[phys, h] * (was / now))
                            cache.scale[which][phys, h] = now
                        pool[phys, h, at] = R.encode(rows / now if now > 0 else rows * 0.0)
                if abstract is None or keep >= n:
                    continue
                for p in sorted({to // page for to, _ in pairs} | ({(keep - 1) // page} if keep else set())):
                    if not 0 <= int(table[b, p]) < made.n_pages:
                        continue
                    kept = cache.values(0)[int(table[b, p]), h, : min(page, keep - p * page)]
                    bare = torch.where(torch.isnan(kept), torch.full_like(kept, -math.inf), kept)
                    abstract[b, h, p, 0] = bare.amax(0)
                    abstract[b, h, p, 1] = torch.where(torch.isnan(kept), torch.full_like(kept, math.inf), kept).amin(0)
            if abstract is not None:
                last = (keep - 1) // page
                changed = keep < n
                assert int(self.n_chunks[b]) == (last + 1 if changed else -7)
                want = [-7] * (made.table.shape[1] + 1)
                if changed:
                    want[last + 1] = keep
                assert self.off[b].tolist() == want
        assert torch.equal(self.weight.cpu(), w) and torch.equal(self.ids.cpu(), ids)
        for which, (pool, scale) in enumerate(((made.k_pages, made.k_scale), (made.v_pages, made.v_scale))):
            got = pool.cpu().double() if not made.q8 else R.E4M3_VALUES[pool.cpu().view(torch.uint8).long()]
            want = cache.pool[which]
            for b, keep in enumerate(keeps):      # (what stands behind the kept length may change)
                for t in range(min(keep, made.lengths[b]), made.lengths[b]):
                    if ok(b, t) and made.q8:
                        want[int(table[b, t // page]), :, t % page] = got[int(table[b, t // page]), :, t % page]
            assert torch.equal(got.nan_to_num(3e30), want.nan_to_num(3e30)), "kv"[which] + " pages"
            if made.q8:
                assert torch.equal(scale.cpu().double().nan_to_num(-1.0), cache.scale[which].nan_to_num(-1.0)), "scales"
        if abstract is not None:
            assert torch.equal(self.abstract.cpu().double(), abstract)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("bounds", [True, False], ids=["abstracts", "bare"])
def test_moves(L, dtype, q8, page, bounds):
    lengths = [5 * page + 3, 4 * page, 0, 7, 3 * page + 1, 2 * page]
    keeps = [3 * page + 2, 2 * page, 0, 7, page - 1, 2 * page - 1]      # a page that the kept length cuts, one it does not, nothing to do
    cache = Moving(L, dtype, q8, lengths, 3, page, seed=page, bounds=bounds, gains=(-3, 4))
    cache.run(keeps, cache.random_moves(keeps, seed=page, share=1.0))


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("page", [16, 256])
def test_every_row_moves_or_none_does(L, dtype, q8, page):
    lengths, keeps = [2 * page, 2 * page, 2 * page - 1, page + 5], [page, page, page - 1, 0]
    cache = Moving(L, dtype, q8, lengths, 2, page, seed=page, gains=(-3, 4))
    lists = cache.random_moves(keeps)
    for h in range(2):
        lists[0, h] = [(t, page + t) for t in range(page)]
        lists[1, h] = []
        lists[2, h] = [(t, 2 * page - 2 - t) for t in range(page - 1)]      # in another order behind, the cut page's rows among them
        lists[3, h] = []
    cache.run(keeps, lists)


def test_move_zeros_from_a_page_of_far_larger_numbers(L):
    """The quotient of the scales is beyond 32 bits, the row's codes are zero: so are they afterwards."""
    pages = L.make_pages(1, 1, 1, 128, 2, 16, 2, BF16, kv_dtype=L.E4M3)
    k, v = (torch.randint(0, 0x7e, (2, 1, 16, 128), dtype=torch.uint8, device="cuda") for _ in range(2))
    k[1, 0, 3], v[1, 0, 3] = 0, 0x80      # (-0, too)
    ks, vs = (torch.tensor([[2.0 ** -90], [2.0 ** 110]], device="cuda") for _ in range(2))
    want = [x.clone() for x in (k, v, ks, vs)]
    want[0][0, 0, 5], want[1][0, 0, 5] = 0, 0x80
    kf, vf = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
    L.kv_page_move(pages, i32([[[[5, 19]]]]), i32([[1]]), i32([32]), i32([16]), i32([[0, 1]]), kf, vf, ks, vs, None, None, None, None, None)
    for got, expected in zip((k, v, ks, vs), want):
        assert torch.equal(got, expected)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_scales_that_rise_from_zero_and_by_far(L, dtype):
    cache = Moving(L, dtype, True, [64, 64], 2, 16, seed=2)
    made = cache.made
    for which, (pool, scale) in enumerate(((made.k_pages, made.k_scale), (made.v_pages, made.v_scale))):
        for b, p, s in ((0, 0, 0.0), (0, 1, 2.0 ** -14), (0, 3, 2.0 ** 6), (1, 0, 2.0 ** -3), (1, 2, 0.0)):
            phys = int(made.table[b, p])
            scale[phys] = s
            made.cache.scale[which][phys] = s
            if s == 0.0:
                pool[phys] = 0.0
                made.cache.pool[which][phys] = 0.0
    keeps = [37, 40]
    lists = {(b, h): [(1, 40), (2, 50), (17, 63), (20, 44), (36, 62)] for b in range(2) for h in range(2)}
    lists[1, 1] = [(3, 41), (5, 47)]
    cache.run(keeps, lists)


def test_values_that_are_not_numbers_move_and_pairs_outside_are_left_out(L):
    cache = Moving(L, BF16, True, [64, 64, 64], 1, 16, seed=3)
    made = cache.made
    phys = int(made.table[0, 3])
    made.k_pages.view(torch.uint8)[phys, 0, 4, 7] = 0x7f
    made.cache.pool[0][phys, 0, 4, 7] = math.nan
    table = made.table
    table[1, 3], table[2, 0] = -1, made.n_pages
    keeps = [30, 30, 30]
    lists = {(0, 0): [(0, 52), (5, 33)], (1, 0): [(0, 33), (1, 50), (17, 40)], (2, 0): [(2, 33), (16, 34), (29, 10), (29, 64), (31, 40)]}
    cache.run(keeps, lists)


def test_lists_that_do_not_ascend_stay_within_the_buffers(L):
    cache = Moving(L, F16, False, [200], 1, 16, seed=4)
    cache.run([100], {(0, 0): [(90, 150), (3, 120), (1 << 30, 130), (-5, 140), (50, -1), (3, 190)]}, verify=False)
    cache.made.seq_len = i32([1 << 30])
    cache.run([-4], {(0, 0): [(0, 150)]}, verify=False)


@pytest.mark.parametrize("dtype,q8", [(BF16, False), (F16, True)], ids=["bf16", "f16-e4m3"])
def test_move_replays_from_a_graph(L, dtype, q8):
    # (whole pages are kept: sources keep their values, so that the call can be repeated)
    cache = Moving(L, dtype, q8, [300, 129], 2, 32, seed=5)
    call = cache.run([160, 96], cache.random_moves([160, 96], share=1.0))
    made = cache.made
    state = [t for t in (made.k_pages.view(torch.uint8), made.v_pages.view(torch.uint8), cache.weight, cache.ids, cache.abstract.view(torch.uint8))]
    want = [t.clone() for t in state]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(state, want))
        call()
        assert all(torch.equal(a, b) for a, b in zip(state, want))


# ---- all of them together, as a serving program calls them -----------------------------------------------------

@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("budget", [0, 4], ids=["all pages", "kept pages"])
def test_a_cache_that_is_kept_within_bounds(L, dtype, q8, budget):
    """Prompts, then steps with positions of their own; whenever sequences outgrow their budget they are brought down to it.  Every
    step's attention is that over the tokens that the reference holds, every weight what it adds up, every page's abstract what it holds."""
    g = torch.Generator().manual_seed(11)
    B, hq, hkv, page, max_pages, keep, recent = 3, 8, 2, 16, 9, 70, 9
    prompt, G = [100, 33, 71], 4
    n_pages = B * max_pages
    table = torch.randperm(n_pages, generator=g).int().reshape(B, max_pages).cuda()
    seq_len, n_seen = i32([0] * B), i32([0] * B)
    rope = L.rope_table(400, 128).cuda()
    layer = L.PagedLayer(table, seq_len, hq, hkv, n_pages, page, dtype, L.E4M3 if q8 else None, rope=rope, max_chunks=budget, evicts=40)
    layer.k_pages.view(torch.uint8).fill_(0x7f)
    layer.v_pages.view(torch.uint8).fill_(0x7f)
    n_first = i32([2, 0, 5])

    def held(which, b):
        n = int(seq_len[b])
        pool, scale = (layer.k_pages, layer.k_scale) if which == 0 else (layer.v_pages, layer.v_scale)
        x = pool[table[b].long()].float().double()
        if q8:
            x = x * scale[table[b].long()].double()[..., None, None]
        return x.transpose(0, 1).reshape(hkv, -1, 128)[:, :n].cpu()

    def rows(n):
        x = torch.randn(n, hq + 2 * hkv, 128, generator=g).to(dtype).cuda()
        return x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:]

    def check_bounds():
        for b in range(B):
            n, K = int(seq_len[b]), held(0, b)
            P = -(-n // page)
            assert int(layer.n_chunks[b]) == P and layer.chunk_off[b, : P + 1].tolist() == [min(page * i, n) for i in range(P + 1)]
            for p in range(P):
                kept = K[:, p * page: (p + 1) * page]
                assert torch.equal(layer.abstract[b, :, p].cpu().double(), torch.stack([kept.amax(1), kept.amin(1)], 1))

    # prompts, weighed by all of their queries
    n = sum(prompt)
    seq_len.copy_(i32(prompt))
    n_seen.copy_(i32(prompt))
    off = i32([0, 100, 133, 204])
    lse = torch.empty(n, hq, device="cuda")
    q, k, v = rows(n)
    position = torch.cat([torch.arange(m) for m in prompt]).int()[None].cuda()
    q_turned = torch.empty(n, hq, 128, dtype=dtype, device="cuda")
    layer.prompt(q, k, v, off, lse=lse, q_out=q_turned, position=position)
    layer.weigh(q_turned, n_seen, off, lse)
    torch.cuda.synchronize()
    weights = {}
    for b in range(B):
        K, row0 = held(0, b), int(off[b])
        for h in range(hkv):
            z = torch.einsum("rgd,td->rgt", q_turned[row0: row0 + prompt[b], h * G: (h + 1) * G].cpu().double(), K[h]) * SCALE
            z = z.masked_fill(torch.triu(torch.ones(prompt[b], prompt[b], dtype=torch.bool), 1)[:, None], -math.inf)
            weights[b, h] = torch.softmax(z, -1).sum((0, 1))
            # (a weight at most some percent off: dz and the lse's error, as above, are below 2^-10 here)
            assert torch.allclose(layer.weight[b, h, : prompt[b]].cpu().double(), weights[b, h], rtol=2.0 ** -10, atol=1e-12)
    assert all(torch.equal(layer.token_id[b, :, : prompt[b]].cpu(), torch.arange(prompt[b]).int().expand(hkv, -1)) for b in range(B))
    ids = {(b, h): list(range(prompt[b])) for b in range(B) for h in range(hkv)}

    for step in range(25):
        if step % 4 == 0:
            before_w, lens = layer.weight.cpu().numpy().copy(), seq_len.tolist()
            before = [(held(0, b), held(1, b)) for b in range(B)]
            seq_len.copy_(layer.evict(i32([keep] * B), n_seen, n_first, recent))
            torch.cuda.synchronize()
            assert layer.evict_status.tolist() == [0] * B and seq_len.tolist() == [min(x, keep) for x in lens]
            for b in range(B):
                now = held(0, b), held(1, b)
                for h in range(hkv):
                    have = np.array(ids[b, h])
                    stay = np.sort(order_of(before_w[b, h], have, lens[b], int(n_seen[b]), int(n_first[b]), recent)[:keep])
                    free, behind = np.setdiff1d(np.arange(min(keep, lens[b])), stay), stay[stay >= keep]
                    at = np.arange(min(keep, lens[b]))
                    at[free] = behind                              # where each token that stays came from
                    ids[b, h] = have[at].tolist()
                    weights[b, h] = weights[b, h][torch.from_numpy(at)]
                    for which in (0, 1):
                        want, got = before[b][which][h][torch.from_numpy(at)], now[which][h]
                        if q8:      # (a code's subnormal steps: half of 2^-9 of the page's new scale)
                            scale = (layer.k_scale, layer.v_scale)[which][table[b].long(), h].cpu().double().repeat_interleave(page)[: len(at)]
                            assert ((want - got).abs() <= (2.0 ** -10 * scale)[:, None]).all()
                        else:
                            assert torch.equal(want, got)
                assert [x for h in range(hkv) for x in layer.token_id[b, h, : len(ids[b, h])].tolist()] == [x for h in range(hkv) for x in ids[b, h]]
            if budget:
                check_bounds()
        q, k, v = rows(B)
        seq_len.add_(1)
        n_seen.add_(1)
        q_turned = torch.empty(B, hq, 128, dtype=dtype, device="cuda")
        out = layer.step(q, k, v, q_out=q_turned, position=(n_seen - 1)[None].contiguous())
        if not budget:      # (under a budget lse is over the kept pages: weights of the others would not be attention)
            layer.weigh(q_turned, n_seen)
        torch.cuda.synchronize()
        where = torch.tensor([int(n_seen[b]) - 1 for b in range(B)])
        assert torch.equal(q_turned.cpu(), R.rotate(q.cpu(), rope.cpu(), where, 128, False).to(dtype))
        for b in range(B):
            K, V = held(0, b), held(1, b)
            if not budget:
                check_rows(L, None, out, layer.lse, [(b, q_turned[b].cpu(), K, V)], 0.0 if dtype == F32 else 2.0 ** -16, 2.0 ** -23)
            for h in range(hkv):
                ids[b, h].append(int(n_seen[b]) - 1)
                weights[b, h] = torch.cat([weights[b, h], torch.zeros(1, dtype=torch.float64)])
                if budget:
                    layer.token_id[b, h, int(seq_len[b]) - 1] = int(n_seen[b]) - 1
                    layer.weight[b, h, int(seq_len[b]) - 1] = 0.0
                    continue
                z = q_turned[b, h * G: (h + 1) * G].cpu().double() @ K[h].T * SCALE
                weights[b, h] += torch.softmax(z, -1).sum(0)
                assert torch.allclose(layer.weight[b, h, : K.shape[1]].cpu().double(), weights[b, h], rtol=2.0 ** -10, atol=1e-12)
        if budget:
            check_bounds()


def test_a_layer_with_a_shared_prefix(L):
    """Samples of one prompt: its pages are listed by all of them; steps over the shared pages are those over each one's own list."""
    g = torch.Generator().manual_seed(12)
    B, page, prefix = 6, 16, 5
    max_pages = prefix + 3
    table = torch.full((B, max_pages), -1, dtype=torch.int32)
    table[:, :prefix] = torch.arange(prefix)
    table[:, prefix:] = torch.arange(prefix, prefix + 3 * B).reshape(B, 3)
    n_pages = prefix + 3 * B
    table, seq_len = table.cuda(), i32([prefix * page] + [0] * (B - 1))
    rope = L.rope_table(200, 128).cuda()
    layer = L.PagedLayer(table, seq_len, 8, 2, n_pages, page, BF16, rope=rope, groups=2)
    rows = lambda n: (lambda x: (x[:, :8], x[:, 8:10], x[:, 10:]))(torch.randn(n, 12, 128, generator=g).to(BF16).cuda())  # noqa: E731
    layer.prompt(*rows(prefix * page), i32([0] + [prefix * page] * B))
    off, shared = i32([0, B]), i32([prefix])
    seq_len.fill_(prefix * page)
    for _ in range(20):
        seq_len.add_(1)
        q = layer.append(*rows(B))
        plain, lse = layer.attend(q).clone(), layer.lse.clone()
        layer.out.fill_(math.nan)
        out = layer.attend_shared(q, off, shared)
        assert (out - plain).abs().max() <= 6.0 * 2 * (2 * 12 * 2.0 ** -16 + 2.0 ** -16 + 128 * 2.0 ** -24)
        assert (layer.lse - lse).abs().max() <= 2 * 12 * 2.0 ** -16
    with pytest.raises(ValueError):
        layer.attend_shared(q, i32([0, 1, 2, 3]), i32([1, 1, 1]))
    with pytest.raises(ValueError):
        layer.weigh(q, seq_len)
    with pytest.raises(ValueError):
        layer.evict(seq_len, seq_len)
