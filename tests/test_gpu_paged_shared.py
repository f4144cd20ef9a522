"""page_attention_decode_shared and kv_page_append_at against plain 64-bit forms (tests/paged_reference.py); tolerances as derived in
tests/test_gpu_paged.py: a shared prefix changes the order of the sums only, weights enter the values in two or three 16-bit
pieces, so within 2^-16, and a rotation is defined in binary32 operations, so compared bit for bit."""
import math

import pytest
import torch

from tests import paged_reference as R
from tests.test_gpu_paged import BF16, F16, F32, KIND_IDS, KINDS, SCALE, L, check_rows, scratch, spread  # noqa: F401

pytestmark = pytest.mark.gpu
i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731


class Grouped:
    """groups: (pages of the prefix, own tokens of each member; None: an idle member, a negative number: a sequence that is as much
    shorter than the prefix).  NaN wherever no token is."""

    def __init__(self, dtype, q8, hkv, page, groups, seed=0, alone_before=(), alone_after=()):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.q8, self.hkv, self.page = dtype, q8, hkv, page
        plan, self.off, self.shared = [], [], []
        for n in alone_before:
            plan.append((None, 0, n))
        for i, (pages, members) in enumerate(groups):
            self.off.append(len(plan))
            self.shared.append(pages)
            for own in members:
                whole = own is not None and own >= 0
                plan.append((i if whole else None, pages * page if whole else 0, 0 if own is None else own if whole else pages * page + own))
        self.off.append(len(plan))
        for n in alone_after:
            plan.append((None, 0, n))
        need = [-(-n // page) for _, _, n in plan]
        self.n_pages = sum(need) + sum(self.shared) + 3
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        at, prefix = 0, []
        for n in self.shared:
            prefix.append(order[at: at + n])
            at += n
        widest = max(before // page + n for (_, before, _), n in zip(plan, need)) + 1
        self.table = torch.full((len(plan), widest), -1, dtype=torch.int32)
        self.lengths = [before + n for _, before, n in plan]
        shape = (self.n_pages, hkv, page, 128)
        store = torch.float8_e4m3fn if q8 else dtype
        nan = torch.full(shape, math.nan).to(store)
        sc = torch.full((self.n_pages, hkv), math.nan) if q8 else None
        self.cache = R.Cache(nan, nan, sc, sc, dtype)
        fresh = lambda n: torch.randn(n, hkv, 128, generator=g).to(dtype).float()  # noqa: E731
        for ids in prefix:
            if len(ids):
                n = len(ids) * page
                self.cache.append(fresh(n), fresh(n), 0, ids, page)
        for b, ((i, before, n), k) in enumerate(zip(plan, need)):
            first = before // page
            if i is not None:
                self.table[b, :first] = prefix[i]
            self.table[b, first: first + k] = order[at: at + k]
            at += k
            if n:
                self.cache.append(fresh(n), fresh(n), before, self.table[b], page)
        self.k_pages, self.v_pages = (p.to(torch.float32).to(store).cuda() for p in self.cache.pool)
        self.k_scale, self.v_scale = ((s.float().cuda() if q8 else None) for s in self.cache.scale)
        self.g = g

    def tokens(self, which, b):
        pos = [t for t in range(self.lengths[b]) if 0 <= int(self.table[b, t // self.page]) < self.n_pages]
        pos = torch.tensor(pos, dtype=torch.long)
        v = self.cache.values(which)
        return v[self.table[b, pos // self.page].long(), :, pos % self.page].transpose(0, 1)


def run_shared(L, made, hq, ws=None, scale=SCALE, rows=None, verify=True, lse=True):
    B = len(made.lengths)
    q = torch.randn(B, hq, 128, generator=made.g).to(made.dtype)
    pages = L.make_pages(B, hq, made.hkv, 128, made.n_pages, made.page, made.table.shape[1], made.dtype, L.E4M3 if made.q8 else None)
    out = torch.full((B, hq, 128), math.nan, device="cuda")
    lse = torch.full((B, hq), math.nan, device="cuda")
    ws = scratch(L.leoam_page_shared_workspace_bytes(pages, len(made.shared)) if ws is None else ws(pages))
    call = lambda: L.page_attention_decode_shared(  # noqa: E731
        pages, qg, made.k_pages, made.v_pages, made.k_scale, made.v_scale, table, lens, off, shared, scale, out, lse, ws)
    qg, table, lens, off, shared = q.cuda(), made.table.cuda(), i32(made.lengths), i32(made.off), i32(made.shared)
    call()
    torch.cuda.synchronize()
    if verify:
        half = 0.0 if made.dtype == F32 else 2.0 ** -16
        check_rows(L, made, out, lse, [(b, q[b], made.tokens(0, b), made.tokens(1, b)) for b in (rows or range(B))], half, 2.0 ** -23, scale)
    return call, qg, out, lse


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_groups_of_many_kinds(L, dtype, q8, group):
    # a group of one, members without a token of their own, idle and short ones, no prefix, sequences outside
    made = Grouped(dtype, q8, 2, 16, [(3, [5]), (9, [0, 1, 16, 17, 33, None, 15, -1, -144, 200]), (0, [7, None, 0]), (2, [None, None]),
                                      (1, [31, 32])], seed=group, alone_before=(40, 0), alone_after=(0, 129))
    run_shared(L, made, 2 * group)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("members,group", [(16, 1), (17, 1), (5, 8), (9, 4), (16, 4), (17, 4), (31, 4), (32, 4), (33, 4), (67, 4), (129, 1)])
def test_columns(L, dtype, q8, members, group):
    # columns of one wave, two, four, and of several units, up to their borders
    made = Grouped(dtype, q8, 1, 32, [(9, [1 + i % 40 for i in range(members)])], seed=members)
    run_shared(L, made, group, rows=sorted({0, 1, members // 2, members - 1, min(members - 1, 31), min(members - 1, 32)}))


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("page", [16, 64, 128, 256])
def test_long_prefixes_are_cut(L, dtype, q8, page):
    made = Grouped(dtype, q8, 2, page, [(4096 // page, [3, 700, 0]), (1024 // page, [1, 5000 if page == 64 else 90])], seed=page)
    run_shared(L, made, 8)


@pytest.mark.parametrize("dtype,q8", [(BF16, False), (F16, True)], ids=["bf16", "f16-e4m3"])
def test_small_workspaces(L, dtype, q8):
    made = Grouped(dtype, q8, 2, 32, [(20, [3, 300, 0, 64]), (3, [1, 900])], seed=3)
    for extra in (0, 1, 133120, 5 * 133120 + 7):
        run_shared(L, made, 8, ws=lambda pages: L.leoam_page_shared_workspace_min(pages) + extra)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
def test_pages_that_are_missing_hold_no_tokens(L, dtype, q8):
    made = Grouped(dtype, q8, 2, 16, [(12, [3, 40, 0, 64])], seed=4)
    for b in range(4):
        made.table[b, 2], made.table[b, 7] = -1, 1 << 30
    made.table[1, 13] = made.n_pages
    run_shared(L, made, 8)
    for b in range(4):
        made.table[b, :12] = -5
    run_shared(L, made, 8)      # (of the third nothing is left)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("hkv,group", [(5, 1), (8, 2), (6, 8)])
def test_short_tails_of_many_sequences(L, dtype, q8, hkv, group):
    # four heads to a workgroup: numbers of heads that four divides and does not, tails at the border, longer and none, pages missing
    made = Grouped(dtype, q8, hkv, 16, [(2, [0, 1, 15, 16, 31, 32, 33, 64, 65, 127, 128, 129, None, -1, 200] * 2), (0, [1, 5, 130] * 5), (3, [7, 2, 90])],
                   seed=hkv, alone_after=(0, 1, 128, 129, 40))
    assert len(made.lengths) * hkv > 256
    made.table[3, 2], made.table[9, 3], made.table[26, 2:] = -1, 1 << 20, -1
    run_shared(L, made, hkv * group, rows=sorted({*range(16), 18, 25, 26, *range(29, 36), *range(len(made.lengths) - 8, len(made.lengths))}))


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1e-30, 3.0])
def test_scales_of_any_sign(L, scale):
    run_shared(L, Grouped(F16, False, 1, 16, [(5, [3, 40, 0])], seed=5), 4, scale=scale)


def test_many_groups_and_sequences(L):
    # more groups than a workgroup keeps on chip, more entries than it has threads
    groups = [(i % 4, [1 + (i * 7) % 30] * (1 + i % 2)) for i in range(600)]
    made = Grouped(BF16, False, 1, 16, groups, seed=6)
    run_shared(L, made, 2, rows=list(range(0, len(made.lengths), 13)))


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
def test_agrees_with_decoding_and_repeats_its_bits(L, dtype, q8):
    made = Grouped(dtype, q8, 4, 64, [(17, [3, 300, 0, 64, 65]), (40, [900, 1])], seed=7)
    call, q, out, lse = run_shared(L, made, 16, rows=[0, 5])
    first, first_lse = out.clone(), lse.clone()
    for _ in range(3):
        out.fill_(7.0)
        call()
        assert torch.equal(out, first) and torch.equal(lse, first_lse)
    pages = L.make_pages(7, 16, 4, 128, made.n_pages, 64, made.table.shape[1], dtype, L.E4M3 if q8 else None)
    plain, plain_lse = torch.empty_like(out), torch.empty_like(lse)
    L.page_attention_decode(pages, q, made.k_pages, made.v_pages, made.k_scale, made.v_scale, made.table.cuda(), i32(made.lengths), None,
                            None, SCALE, plain, plain_lse, scratch(L.leoam_page_workspace_bytes(pages)))
    # (both are within the tolerance of the exact value: dz = 2^-16 A, A at most 12 here, max |V| at most 6)
    tol = 6.0 * 2 * (2 * 12 * 2.0 ** -16 + 2.0 ** -16 + 4096 * 2.0 ** -24)
    assert (plain - first).abs().max() <= tol and (plain_lse - first_lse).abs().max() <= tol


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_values_that_are_not_finite_reach_those_who_attend_to_them(L, bad):
    # in one member's own pages, and in the prefix beside a member that is too short for it and so has pages of its own
    made = Grouped(F16, False, 1, 16, [(6, [20, 20, -3])], seed=8)
    own = int(made.table[0, 6])
    made.v_pages[own, 0, 3, 9] = bad
    _, _, out, _ = run_shared(L, made, 2, verify=False)
    assert not torch.isfinite(out[0, :, 9]).any() and torch.isfinite(out[1:]).all() and torch.isfinite(out[0, :, :9]).all()
    made.v_pages[own, 0, 3, 9] = 0.0
    made.v_pages[int(made.table[0, 1]), 0, 5, 77] = bad
    _, _, out, _ = run_shared(L, made, 2, verify=False)
    assert not torch.isfinite(out[:2, :, 77]).any() and torch.isfinite(out[2]).all() and torch.isfinite(out[:, :, :77]).all()


def test_lists_that_are_out_of_range_stay_within_the_buffers(L):
    made = Grouped(BF16, False, 1, 16, [(2, [5, 6]), (3, [9, 1])], seed=9)
    made.off, made.shared = [-3, 2, 99], [-1, 1 << 30]
    run_shared(L, made, 2)      # (no group has a prefix that its sequences reach: everybody by itself)
    made.off, made.shared = [3, 1, 4], [2, 2]
    run_shared(L, made, 2, verify=False)      # (descends: undefined, but within bounds)


def test_replays_from_a_graph_and_runs_on_another_stream(L):
    made = Grouped(BF16, True, 2, 32, [(20, [3, 300, 0]), (5, [64, 1])], seed=10)
    call, q, out, lse = run_shared(L, made, 8)
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        out.fill_(float(i))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out.fill_(5.0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert torch.equal(out, want)


# ---- kv_page_append_at ----------------------------------------------------------------------------------------

def turned(x, rope, position, axis, rot, interleaved, dtype=torch.float32):
    """x [n, H, 128]: pair i turned by rope[position[axis[i]]][i]; every product and sum one operation of `dtype`."""
    y = x.to(dtype).clone()
    half, i = rot // 2, torch.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    p = position.long().clamp(0, rope.shape[0] - 1)[axis.long().clamp(0, position.shape[0] - 1)].T      # [n, half]
    c, s = rope[p, i][:, None].to(dtype), rope[p, half + i][:, None].to(dtype)
    xa, xb = y[..., a].clone(), y[..., b].clone()
    y[..., a] = xa * c - xb * s
    y[..., b] = xb * c + xa * s
    return y


AXES = {"one": lambda h: torch.zeros(h), "sections": lambda h: (torch.arange(h) * 4 // h - 1).clamp(min=0), "turns": lambda h: torch.arange(h) % 3,
        "odd sections": lambda h: (torch.arange(h) >= 3).int() + (torch.arange(h) >= h - 5).int()}


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("layout", sorted(AXES))
@pytest.mark.parametrize("rot,interleaved", [(128, False), (64, True), (16, False), (96, False), (128, True)])
def test_append_at(L, dtype, q8, layout, rot, interleaved):
    g = torch.Generator().manual_seed(rot + len(layout))
    hq, hkv, page, calls = 8, 2, 32, [[37, 0, 1, 70], [1, 1, 1, 1], [2, 40, 1, 0]]
    axis = AXES[layout](rot // 2).int()
    n_axes = int(axis.max()) + 1
    table, n_pages = spread([sum(c[b] for c in calls) for b in range(4)], page, g)
    store = torch.float8_e4m3fn if q8 else dtype
    nan = torch.full((n_pages, hkv, page, 128), math.nan).to(store)
    sc = torch.full((n_pages, hkv), math.nan) if q8 else None
    ref = R.Cache(nan, nan, sc, sc, dtype)
    k_pages, v_pages = nan.cuda(), nan.cuda()
    k_scale, v_scale = (sc.cuda(), sc.cuda()) if q8 else (None, None)
    rope = L.rope_table(1000, rot, 500.0)
    pages = L.make_pages(4, hq, hkv, 128, n_pages, page, table.shape[1], dtype, L.E4M3 if q8 else None, rot_dim=rot, interleaved=interleaved,
                         rope_len=1000)
    status, held = i32([-7] * 4), [0] * 4
    abstract = torch.zeros(4, hkv, table.shape[1], 2, 128, dtype=dtype, device="cuda")
    for call in calls:
        n = sum(call)
        x = torch.randn(n, hq + 2 * hkv, 128, generator=g).to(dtype)
        position = torch.randint(0, 1000, (n_axes, n), generator=g).int()
        xg, q_out = x.cuda(), torch.full((n, hq, 128), math.nan, dtype=dtype, device="cuda")
        lens = [h + c for h, c in zip(held, call)]
        off = None if call == [1] * 4 else i32([sum(call[:b]) for b in range(5)])
        L.kv_page_append_at(pages, xg[:, :hq], xg[:, hq: hq + hkv], xg[:, hq + hkv:], off, i32(lens), table.cuda(), rope.cuda(),
                            position.cuda(), axis.cuda() if n_axes > 1 else None, q_out, k_pages, v_pages, k_scale, v_scale, abstract,
                            None, None, status)
        torch.cuda.synchronize()
        assert status.tolist() == [0] * 4
        assert torch.equal(q_out.cpu(), turned(x[:, :hq], rope, position, axis, rot, interleaved).to(dtype))
        exact = turned(x[:, :hq], rope, position, axis, rot, interleaved, torch.float64)
        half = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}[dtype]
        assert ((q_out.cpu().double() - exact).abs() <= 2.0 ** -22 * x.double().abs().amax() + half * exact.abs() + 1e-7).all()
        k, row = turned(x[:, hq: hq + hkv], rope, position, axis, rot, interleaved), 0
        for b, m in enumerate(call):
            for p in ref.append(k[row: row + m], x[row: row + m, hq + hkv:].float(), held[b], table[b], page) if m else ():
                kept = ref.values(0)[int(table[b, p]), :, : min(lens[b], (p + 1) * page) - p * page]
                assert torch.equal(abstract[b, :, p].cpu().double(), torch.stack([kept.amax(1), kept.amin(1)], 1))
            row += m
        held = lens
    for pool, want in ((k_pages, ref.pool[0]), (v_pages, ref.pool[1])):
        got = pool.cpu().double() if not q8 else R.E4M3_VALUES[pool.cpu().view(torch.uint8).long()]
        assert torch.equal(got.nan_to_num(3e30), want.nan_to_num(3e30))


def test_append_at_places_of_their_own_is_append(L):
    g = torch.Generator().manual_seed(12)
    x = torch.randn(50, 12, 128, generator=g).to(BF16).cuda()
    table, n_pages = spread([50], 16, g)
    pages = L.make_pages(1, 8, 2, 128, n_pages, 16, table.shape[1], BF16, rot_dim=128, rope_len=80)
    rope, off, lens = L.rope_table(80, 128).cuda(), i32([0, 50]), i32([50])
    got = []
    for at in (False, True):
        pools = [torch.zeros(n_pages, 2, 16, 128, dtype=BF16, device="cuda") for _ in "kv"]
        q = torch.empty(50, 8, 128, dtype=BF16, device="cuda")
        args = (x[:, :8], x[:, 8:10], x[:, 10:], off, lens, table.cuda(), rope)
        if at:
            L.kv_page_append_at(pages, *args, i32([list(range(50))]), None, q, *pools)
        else:
            L.kv_page_append(pages, *args, q, *pools)
        got.append((q, *pools))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("single", [False, True], ids=["prompt", "tokens"])
def test_append_at_positions_outside_the_table(L, single):
    # the nearest one that the table has, and status 3; a bad page comes first; places beyond the table's length are fine
    g = torch.Generator().manual_seed(13)
    new = [1, 1, 1, 1] if single else [3, 2, 4, 1]
    lens, n = [40, 60, 4, 5], sum(new)
    table, n_pages = spread(lens, 16, g)
    table[2, 0] = n_pages
    position = torch.randint(0, 20, (3, n), generator=g).int()
    starts = [sum(new[:b]) for b in range(4)]
    position[1, starts[0]], position[2, starts[2]] = -4, 20
    position[0, starts[3]] = 1 << 30
    axis = torch.arange(64).int() % 3
    axis[5], axis[60] = -2, 7      # (as the nearest axis)
    x = torch.randn(n, 12, 128, generator=g).to(F16)
    pages = L.make_pages(4, 8, 2, 128, n_pages, 16, table.shape[1], F16, rot_dim=128, rope_len=20)
    rope, status = L.rope_table(20, 128), i32([-7] * 4)
    pool, q = torch.zeros(n_pages, 2, 16, 128, dtype=F16, device="cuda"), torch.empty(n, 8, 128, dtype=F16, device="cuda")
    xg = x.cuda()
    L.kv_page_append_at(pages, xg[:, :8], xg[:, 8:10], xg[:, 10:], None if single else i32(starts + [n]), i32(lens), table.cuda(), rope.cuda(),
                        position.cuda(), axis.cuda(), q, pool, pool.clone(), status=status)
    torch.cuda.synchronize()
    assert status.tolist() == [3, 0, 2, 3]
    assert torch.equal(q.cpu(), turned(x[:, :8], rope, position, axis, 128, False).half())


def test_append_at_without_rotation_wants_no_positions(L):
    x = torch.randn(3, 4, 128).to(BF16).cuda()
    pages = L.make_pages(1, 2, 1, 128, 2, 16, 2, BF16)
    pool, v, q = torch.zeros(2, 1, 16, 128, dtype=BF16, device="cuda"), torch.zeros(2, 1, 16, 128, dtype=BF16, device="cuda"), torch.empty(3, 2, 128, dtype=BF16, device="cuda")
    L.kv_page_append_at(pages, x[:, :2], x[:, 2:3], x[:, 3:], i32([0, 3]), i32([3]), i32([[1, -1]]), None, None, None, q, pool, v)
    assert torch.equal(q, x[:, :2]) and torch.equal(pool[1, 0, :3], x[:, 2]) and torch.equal(v[1, 0, :3], x[:, 3])
