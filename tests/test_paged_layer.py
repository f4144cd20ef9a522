"""What PagedLayer refuses and which buffers its calls get (no GPU needed: the library's calls are replaced by ones that note what they were
given)."""
import pytest
import torch

import paper_2506_20187_amd as L
from paper_2506_20187_amd import paged

CALLS = ("kv_page_append", "kv_page_append_at", "chunk_score", "chunk_topk_select", "page_attention_decode", "page_attention_prefill",
         "page_attention_decode_shared", "page_weight_add", "page_evict_select", "kv_page_move")
B, HQ, HKV, PAGE, MAX_PAGES = 3, 8, 2, 16, 5


@pytest.fixture
def calls(monkeypatch):
    """[(name, arguments)] of the library's calls"""
    made = []
    for name in CALLS:
        monkeypatch.setattr(paged.B, name, lambda *a, _name=name: made.append((_name, a)))
    return made


def layer(**kw):
    table, seq_len = torch.zeros(B, MAX_PAGES, dtype=torch.int32), torch.full((B,), 20, dtype=torch.int32)
    return L.PagedLayer(table, seq_len, HQ, HKV, 9, PAGE, torch.bfloat16, **kw)


Q = torch.zeros(B, HQ, 128, dtype=torch.bfloat16)
N = torch.zeros(B, dtype=torch.int32)
GROUPS = (torch.tensor([0, B], dtype=torch.int32), torch.tensor([1], dtype=torch.int32))


def weighed_with(calls):
    name, args = calls[-1]
    assert name == "page_weight_add"
    return args[8]      # lse


@pytest.mark.parametrize("budget", [dict(max_chunks=2), dict(token_budget=20)], ids=str)
def test_weigh_refuses_the_logarithms_of_an_attention_over_kept_pages(calls, budget):
    x = layer(evicts=4, groups=1, **budget)
    with pytest.raises(ValueError, match="lse"):      # (nothing was attended to yet)
        x.weigh(Q, N)
    x.attend(Q)
    with pytest.raises(ValueError, match="lse"):
        x.weigh(Q, N)
    assert calls[-1][0] == "page_attention_decode"
    given = torch.zeros(B, HQ)
    x.weigh(Q, N, lse=given)                          # (what the caller gives is the caller's to know)
    assert weighed_with(calls) is given
    x.attend_shared(Q, *GROUPS)
    x.weigh(Q, N)
    assert weighed_with(calls) is x.lse
    x.attend(Q)
    with pytest.raises(ValueError, match="lse"):
        x.weigh(Q, N)


def test_weigh_takes_the_logarithms_of_an_attention_over_all_pages(calls):
    x = layer(evicts=4)
    with pytest.raises(ValueError, match="lse"):
        x.weigh(Q, N)
    x.attend(Q)
    x.weigh(Q, N)
    assert weighed_with(calls) is x.lse


def test_weigh_wants_the_logarithms_of_a_prompt(calls):
    # (as many rows as sequences: those that the last step left would fit, and are of other rows)
    x, lse = layer(evicts=4), torch.zeros(B, HQ)
    for off in (torch.tensor([0, 2, 2, 3], dtype=torch.int32), torch.arange(B + 1, dtype=torch.int32)):
        x.attend(Q)
        x.weigh(Q, N, off)
        assert weighed_with(calls) is x.lse
        x.prompt(Q, Q[:, :HKV], Q[:, :HKV], off, lse=lse)
        for o in (off, None):
            with pytest.raises(ValueError, match="lse"):
                x.weigh(Q, N, o)
        x.weigh(Q, N, off, lse)
        assert weighed_with(calls) is lse


def test_evict_of_a_layer_with_groups_wants_the_tokens_that_stay(calls):
    x = layer(evicts=4, groups=1)
    with pytest.raises(ValueError, match="n_first"):
        x.evict(N, N)
    assert not calls
    x.evict(N, N, N)
    assert [c[0] for c in calls] == ["page_evict_select", "kv_page_move"] and calls[0][1][6] is N
    layer(evicts=4).evict(N, N)


def test_layers_of_a_model_share_their_workspaces(calls):
    kinds = ("workspace", "shared_workspace", "evict_workspace")
    first = layer(evicts=4, groups=1)
    second = layer(evicts=4, groups=1, workspaces_of=first)
    third = layer(evicts=4, groups=1, workspaces_of=second)
    for x in (second, third):
        assert all(getattr(x, k) is getattr(first, k) for k in kinds)
        x.evict(N, N, N)
        assert calls[-2][1][-2] is first.evict_workspace
        # what a layer's calls leave for the caller is its own
        assert all(getattr(x, k) is not getattr(first, k) for k in ("new_len", "evict_status", "moves", "move_count", "weight", "token_id"))
    # of one that has none, or a smaller one: its own
    assert layer(evicts=4, workspaces_of=layer()).evict_workspace is not None
    table = torch.zeros(B, 1 << 13, dtype=torch.int32)
    long = L.PagedLayer(table, N, HQ, HKV, 9, PAGE, torch.bfloat16, evicts=4, workspaces_of=first)
    assert long.evict_workspace.numel() >= L.leoam_page_evict_workspace_bytes(long.pages) > first.evict_workspace.numel()
    assert layer(workspaces_of=first).evict_workspace is None
