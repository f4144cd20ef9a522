"""kv_page_append_at, page_attention_decode_shared, page_weight_add, page_evict_select and kv_page_move one after the other, as a serving
program calls them: over pools beyond 32 bits, on several streams at once, captured and replayed, with batches that are idle."""
import pytest
import torch

from tests.test_gpu_paged import BF16, F16, F32, KIND_IDS, KINDS, SCALE, L, scratch  # noqa: F401

pytestmark = pytest.mark.gpu
HQ, HKV = 8, 2


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def raw(t):
    return None if t is None else t.view(torch.uint8)


class Serving:
    """Two sequences that share `shared` leading pages (written once, by the first), and a third by itself."""

    def __init__(self, L, dtype, q8, table, n_pages, page, lengths, shared, seed=3):
        self.L, self.page, self.B, self.P = L, page, len(lengths), len(table[0])
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.table, self.seq_len = dtype, i32(table), i32(lengths)
        store = torch.float8_e4m3fn if q8 else dtype
        self.k_pages = torch.empty(n_pages, HKV, page, 128, dtype=store, device="cuda")
        self.v_pages = torch.empty_like(self.k_pages)
        self.k_scale = torch.zeros(n_pages, HKV, device="cuda") if q8 else None
        self.v_scale = torch.zeros(n_pages, HKV, device="cuda") if q8 else None
        self.pages = L.make_pages(self.B, HQ, HKV, 128, n_pages, page, self.P, dtype, L.E4M3 if q8 else None, rot_dim=128, rope_len=4096)
        self.rope = L.rope_table(4096, 128).cuda()
        used = torch.unique(self.table.long().flatten())
        for t in (self.k_pages, self.v_pages):
            raw(t)[used] = 0
        n = sum(lengths)
        x = torch.randn(n, HQ + 2 * HKV, 128, generator=g).to(dtype).cuda()
        off = i32([sum(lengths[:b]) for b in range(self.B + 1)])
        where = torch.cat([torch.arange(m) for m in lengths]).int()[None].cuda() + 17
        if n:      # the second sequence's copy of the shared pages comes out the same
            if shared:
                x[lengths[0]: lengths[0] + shared * page] = x[: shared * page]
            L.kv_page_append_at(self.pages, None, x[:, HQ: HQ + HKV], x[:, HQ + HKV:], off, self.seq_len, self.table, self.rope, where, None,
                                None, self.k_pages, self.v_pages, self.k_scale, self.v_scale)
        cap = self.P * page
        self.n_seen = self.seq_len.clone()
        self.weight = torch.rand(self.B, HKV, cap, generator=g).cuda()
        self.token_id = torch.randperm(cap, generator=g).int().expand(self.B, HKV, cap).contiguous().cuda()
        self.group_off, self.group_pages = i32([0, 2]), i32([shared])
        self.keep, self.first = i32([max(1, m - 20) for m in lengths]), i32([shared * page] * 2 + [1] * (self.B - 2))
        self.q = torch.empty(self.B, HQ, 128, dtype=dtype, device="cuda")
        self.out, self.lse = torch.full((self.B, HQ, 128), 9.0, device="cuda"), torch.full((self.B, HQ), 9.0, device="cuda")
        self.moves, self.count = torch.full((self.B, HKV, 40, 2), -9, dtype=torch.int32, device="cuda"), i32([[-9] * HKV] * self.B)
        self.new_len, self.status = i32([-9] * self.B), i32([-9] * self.B)
        self.ws = scratch(L.leoam_page_shared_workspace_bytes(self.pages, 1))
        self.evict_ws = scratch(L.leoam_page_evict_workspace_bytes(self.pages))
        self.step_rows = torch.randn(self.B, HQ + 2 * HKV, 128, generator=g).to(dtype).cuda()
        self.position = (self.n_seen + 17)[None].contiguous()
        if n:
            self.seq_len += (self.seq_len > 0).int()
            self.n_seen += 1
        torch.cuda.synchronize()

    def step(self, stream=None):
        L, x = self.L, self.step_rows
        L.kv_page_append_at(self.pages, x[:, :HQ], x[:, HQ: HQ + HKV], x[:, HQ + HKV:], None, self.seq_len, self.table, self.rope, self.position,
                            None, self.q, self.k_pages, self.v_pages, self.k_scale, self.v_scale, stream=stream)
        L.page_attention_decode_shared(self.pages, self.q, self.k_pages, self.v_pages, self.k_scale, self.v_scale, self.table, self.seq_len,
                                       self.group_off, self.group_pages, SCALE, self.out, self.lse, self.ws, stream)
        L.page_weight_add(self.pages, self.q, None, self.k_pages, self.k_scale, self.table, self.seq_len, SCALE, self.lse, 0.9, self.weight,
                          self.weight, self.n_seen, self.token_id, stream)
        L.page_evict_select(self.pages, self.weight, self.token_id, self.n_seen, self.seq_len, self.keep, self.first, 5, self.moves, self.count,
                            self.new_len, self.status, self.evict_ws, stream)
        L.kv_page_move(self.pages, self.moves, self.count, self.seq_len, self.new_len, self.table, self.k_pages, self.v_pages, self.k_scale,
                       self.v_scale, self.weight, self.token_id, stream=stream)

    def state(self):
        """Everything that a step writes; of the pools what is kept."""
        got = [self.q, self.out, self.lse, self.weight, self.token_id, self.moves, self.count, self.new_len, self.status]
        for b in range(self.B):
            n = int(self.new_len[b])
            ids = self.table[b].long()
            for t in (self.k_pages, self.v_pages):
                got.append(raw(t)[ids].transpose(0, 1).flatten(1, 2)[:, :n])
            if self.k_scale is not None:
                got += [self.k_scale[ids][: -(-n // self.page)], self.v_scale[ids][: -(-n // self.page)]]
        return [t.clone() for t in got]


def same(a, b):
    assert len(a) == len(b)
    for i, (x, y) in enumerate(zip(a, b)):
        assert torch.equal(raw(x.contiguous()), raw(y.contiguous())), i


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
def test_pools_behind_4_gib(L, dtype, q8):
    """The same bits as from a pool of six pages."""
    page, lengths = 256, [300, 290, 500]
    n = (1 << 32) // (HKV * page * 128 * (1 if q8 else 4 if dtype == F32 else 2)) + 40
    far = Serving(L, dtype, q8, [[n - 1, n - 9], [n - 1, n - 30], [n - 3, n - 2]], n, page, lengths, 1)
    near = Serving(L, dtype, q8, [[5, 0], [5, 3], [1, 2]], 6, page, lengths, 1)
    for s in (far, near):
        s.step()
    torch.cuda.synchronize()
    assert near.status.tolist() == [0] * 3 and int(near.count.min()) > 0 and torch.isfinite(near.out).all()
    same(far.state(), near.state())


@pytest.mark.parametrize("dtype,q8", [(BF16, False), (F16, True), (F32, False)], ids=["bf16", "f16-e4m3", "f32"])
def test_steps_on_two_streams_at_once(L, dtype, q8):
    args = (dtype, q8, [[5, 0, 7], [5, 3, 4], [1, 2, 6]], 8, 64, [120, 130, 180], 1)
    want = []
    for seed in (3, 4):
        s = Serving(L, *args, seed=seed)
        s.step()
        torch.cuda.synchronize()
        want.append(s.state())
    both, streams = [Serving(L, *args, seed=seed) for seed in (3, 4)], [torch.cuda.Stream(), torch.cuda.Stream()]
    for stream in streams:
        stream.wait_stream(torch.cuda.current_stream())
    for s, stream in zip(both, streams):
        s.step(stream)
    torch.cuda.synchronize()
    for s, expected in zip(both, want):
        same(s.state(), expected)


@pytest.mark.parametrize("dtype,q8", [(BF16, False), (BF16, True)], ids=["bf16", "bf16-e4m3"])
def test_steps_replay_from_a_graph(L, dtype, q8):
    """Two graphs of one cache that share its workspaces, replayed in turn with eager steps; each finds the cache as it was."""
    s = Serving(L, dtype, q8, [[5, 0, 7], [5, 3, 4], [1, 2, 6]], 8, 64, [120, 130, 180], 1)
    kept = [s.k_pages, s.v_pages, s.weight, s.token_id] + ([s.k_scale, s.v_scale] if q8 else [])
    before = [raw(t).clone() for t in kept]

    def restore():
        for t, x in zip(kept, before):
            raw(t).copy_(x)
        for t in (s.out, s.lse, s.q):
            t.fill_(7.0)
        s.moves.fill_(-9)
        torch.cuda.synchronize()

    restore()
    s.step()
    torch.cuda.synchronize()
    want = s.state()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for graph in graphs:
        restore()
        with torch.cuda.graph(graph):
            s.step()
    for _ in range(3):
        for run in (graphs[0].replay, graphs[1].replay, s.step):
            restore()
            run()
            torch.cuda.synchronize()
            same(s.state(), want)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
def test_batches_that_are_idle(L, dtype, q8):
    s = Serving(L, dtype, q8, [[5, 0], [5, 3], [1, 2]], 6, 16, [0, 0, 0], 1)
    before = [raw(t).clone() for t in (s.k_pages, s.v_pages, s.weight, s.token_id)]
    s.step()
    torch.cuda.synchronize()
    assert (s.out == 0).all() and (s.lse == -float("inf")).all()
    assert (s.count == 0).all() and s.new_len.tolist() == [0] * 3 and s.status.tolist() == [0] * 3 and (s.moves == -9).all()
    for t, x in zip((s.k_pages, s.v_pages, s.weight, s.token_id), before):
        assert torch.equal(raw(t), x)


def test_one_page_listed_twice(L):
    """A table that names a page twice: its tokens count twice, and both places get the same."""
    g = torch.Generator().manual_seed(1)
    K, V = (torch.randn(3, 2, 16, 128, generator=g).to(BF16).cuda() for _ in range(2))
    q = torch.randn(2, 4, 128, generator=g).to(BF16).cuda()
    pages = L.make_pages(2, 4, 2, 128, 3, 16, 3, BF16)
    table, lens = i32([[0, 1, 0], [2, 2, 2]]), i32([48, 48])
    out, lse = torch.empty(2, 4, 128, device="cuda"), torch.empty(2, 4, device="cuda")
    L.page_attention_decode_shared(pages, q, K, V, None, None, table, lens, i32([0, 1]), i32([2]), SCALE, out, lse,
                                   scratch(L.leoam_page_shared_workspace_bytes(pages, 1)))
    weight = torch.zeros(2, 2, 48, device="cuda")
    L.page_weight_add(pages, q, None, K, None, table, lens, SCALE, lse, 1.0, None, weight)
    z = (q[0].double().reshape(2, 2, 128) @ K[[0, 1, 0]].double().transpose(0, 1).reshape(2, 48, 128).transpose(1, 2).contiguous()) * SCALE
    p = torch.softmax(z, -1)
    want = p @ V[[0, 1, 0]].double().transpose(0, 1).reshape(2, 48, 128)
    # |z| < 4 here: exponents within 2^-13, products of the weights within 2^-16 more
    assert torch.allclose(out[0].double().reshape(2, 2, 128), want, rtol=2.0 ** -12, atol=2.0 ** -12)
    assert torch.equal(weight[0, :, :16], weight[0, :, 32:]) and torch.equal(weight[1, :, :16], weight[1, :, 16:32])
    assert torch.allclose(weight[0].double(), p.sum(1), rtol=2.0 ** -12)
    assert torch.allclose(weight.sum(-1), torch.full((2, 2), 2.0, device="cuda"), rtol=2.0 ** -12)
