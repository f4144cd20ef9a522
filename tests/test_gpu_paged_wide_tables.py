"""page_weight_add and page_evict_select where the table has room for far more tokens than the sequences hold, which decides how the work is
cut up; against the definitions, with the tolerances of tests/test_gpu_paged_evict.py."""
import pytest
import torch

from tests.test_gpu_paged import BF16, F16, KIND_IDS, KINDS, L, Made  # noqa: F401
from tests.test_gpu_paged_evict import i32, run_select, run_weigh

pytestmark = pytest.mark.gpu


def widened(made, max_pages):
    made.table = torch.nn.functional.pad(made.table, (0, max_pages - made.table.shape[1]), value=-1)
    return made


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("max_pages", [64, 300, 3000])
def test_weigh_prompts(L, dtype, q8, max_pages):
    # one wave, four and eight to a stretch of keys, by what the table has; rows behind nothing and behind others
    run_weigh(L, widened(Made(dtype, q8, [700, 90, 0, 333], 2, 32, seed=max_pages), max_pages), 8, [700, 40, 0, 333], seed=max_pages)


@pytest.mark.parametrize("dtype,q8", [(BF16, False), (F16, True)], ids=["bf16", "f16-e4m3"])
@pytest.mark.parametrize("max_pages", [20, 2048])
def test_weigh_a_prompts_chunk_beside_single_tokens(L, dtype, q8, max_pages):
    # (an average of few rows: the chunk's columns go by sixteens)
    lengths = [1 + 37 * b % 300 for b in range(40)] + [450]
    run_weigh(L, widened(Made(dtype, q8, lengths, 2, 32, seed=3), max_pages), 8, [1] * 40 + [90], seed=4)


def test_select_from_a_graph(L):
    # short rows beside one that has the table's width: four launches, whose workgroups mostly have nothing to do
    lengths, keeps = [70001, 4224, 100, 0, 8193, 4096, 1, 70001], [20000, 4096, 64, 5, 8192, 4097, 0, 70000]
    call, moves, count = run_select(L, lengths, keeps, first=[4] * 8, recent=50, m_max=20001)
    want, want_count = moves.clone(), count.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        moves.fill_(-9)
        count.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(moves, want) and torch.equal(count, want_count)
        call()
        torch.cuda.synchronize()


@pytest.mark.parametrize("max_pages", [40, 1100])
def test_layers_that_share_a_workspace_evict_from_a_graph(L, max_pages):
    # as a model's layers do, one after the other; each one's moves are what they are with a workspace of its own
    g = torch.Generator().manual_seed(5)
    B, page, lengths, keep = 3, 64, [2300, 900, 2111], [2048, 1000, 1500]
    table = torch.full((B, max_pages), -1, dtype=torch.int32)
    table[:, :37] = torch.randperm(37 * B, generator=g).int().reshape(B, 37)
    table, seq_len, n_seen, keep = table.cuda(), i32(lengths), i32(lengths), i32(keep)
    make = lambda other=None: L.PagedLayer(table, seq_len, 8, 2, 37 * B, page, BF16, evicts=1000, workspaces_of=other)  # noqa: E731
    first, alone = make(), [make() for _ in range(3)]
    layers = [first, make(first), make(first)]
    assert all(x.evict_workspace is first.evict_workspace for x in layers)
    start = []
    for x, y in zip(layers, alone):
        x.weight.copy_(torch.rand(x.weight.shape, generator=g))
        x.token_id.copy_(torch.arange(max_pages * page, dtype=torch.int32).expand_as(x.token_id))
        x.k_pages.copy_(torch.randn(x.k_pages.shape, generator=g).to(BF16))
        x.v_pages.copy_(torch.randn(x.v_pages.shape, generator=g).to(BF16))
        names = ("weight", "token_id", "k_pages", "v_pages")
        for n in names:
            getattr(y, n).copy_(getattr(x, n))
        start.append([getattr(x, n).clone() for n in names])
        y.evict(keep, n_seen, n_recent=30)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x in layers:
            x.evict(keep, n_seen, n_recent=30)
    for _ in range(3):
        for x, old in zip(layers, start):
            for n, t in zip(names, old):
                getattr(x, n).copy_(t)
            x.move_count.fill_(-9)
        first.evict_workspace.fill_(0xAA)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(layers, alone):
            assert x.new_len.tolist() == [2048, 900, 1500] and x.move_count[0].min() > 0
            for n in (*names, "move_count", "new_len", "evict_status"):
                assert torch.equal(getattr(x, n), getattr(y, n)), n
