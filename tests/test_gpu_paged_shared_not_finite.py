"""page_attention_decode_shared where logits are not finite: a head that attends to such a one gets NaN, as page_attention_decode has it,
whether its tokens are a shared prefix's or its own, in one piece or cut, and nobody else does.  Nothing that is compared by size
here differs from tests/test_gpu_paged_shared.py; its tolerances hold for the others."""
import math

import pytest
import torch

from tests.test_gpu_paged import BF16, F16, F32, KIND_IDS, KINDS, SCALE, L, check_rows, scratch  # noqa: F401
from tests.test_gpu_paged_shared import Grouped, i32

pytestmark = pytest.mark.gpu


def both(L, made, q):
    """(out, lse) of the shared call and of page_attention_decode"""
    B, hq = q.shape[:2]
    pages = L.make_pages(B, hq, made.hkv, 128, made.n_pages, made.page, made.table.shape[1], made.dtype, L.E4M3 if made.q8 else None)
    qg, table, lens = q.cuda(), made.table.cuda(), i32(made.lengths)
    pools = (made.k_pages, made.v_pages, made.k_scale, made.v_scale)
    got = []
    for shared in (True, False):
        out, lse = torch.full((B, hq, 128), 5.0, device="cuda"), torch.full((B, hq), 5.0, device="cuda")
        if shared:
            L.page_attention_decode_shared(pages, qg, *pools, table, lens, i32(made.off), i32(made.shared), SCALE, out, lse,
                                           scratch(L.leoam_page_shared_workspace_bytes(pages, len(made.shared))))
        else:
            L.page_attention_decode(pages, qg, *pools, table, lens, None, None, SCALE, out, lse, scratch(L.leoam_page_workspace_bytes(pages)))
        torch.cuda.synchronize()
        got += [out, lse]
    return got


def same_heads_are_nan(made, q, got, nan):
    """nan [B, Hq]: heads that have to be NaN throughout; all others are what they are without it"""
    out, lse, plain, plain_lse = (x.cpu() for x in got)
    assert torch.equal(torch.isnan(plain).all(-1), nan) and torch.equal(torch.isnan(plain_lse), nan)
    assert torch.equal(torch.isnan(out).all(-1), nan) and torch.equal(torch.isnan(out).any(-1), nan)
    assert torch.equal(torch.isnan(lse), nan)
    half = 0.0 if made.dtype == F32 else 2.0 ** -16
    for b in range(q.shape[0]):
        if nan[b].any():      # (a kv head's heads: those that are NaN are compared no further)
            continue
        check_rows(None, made, got[0], got[1], [(b, q[b], made.tokens(0, b), made.tokens(1, b))], half, 2.0 ** -23)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_queries(L, dtype, q8, bad):
    # groups with a prefix (few and many columns, with and without tokens of their own), a group without one, an idle member, a member that
    # is shorter than the prefix, sequences outside, short and cut
    made = Grouped(dtype, q8, 2, 16, [(9, [0, 5, 300, None, -3]), (4, [1 + i % 30 for i in range(20)]), (0, [7, 40])], seed=21,
                   alone_before=(40, 7), alone_after=(5000, 3))
    q = torch.randn(len(made.lengths), 8, 128, generator=made.g).to(dtype)
    nan = torch.zeros(q.shape[:2], dtype=torch.bool)
    for i, b in enumerate([0, 2, 4, 5, 6, 7, 9, 20, 26, 27, 29]):
        h = 3 * i % 8
        q[b, h, 7 * i] = bad
        nan[b, h] = made.lengths[b] > 0
    got = both(L, made, q)
    if bad == math.inf:      # (logits of one sign may come to no NaN: what page_attention_decode has is what is wanted)
        nan = torch.isnan(got[3]).cpu()
        assert nan.sum() >= 8
    same_heads_are_nan(made, q, got, nan)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
def test_all_queries_of_a_cut_prefix(L, dtype, q8):
    # a prefix in many pieces, of which no one has a number
    made = Grouped(dtype, q8, 1, 64, [(64, [3, 0, 700])], seed=22)
    q = torch.randn(3, 2, 128, generator=made.g).to(dtype)
    q[0, 1, 100] = q[2, 0, 0] = math.nan
    nan = torch.tensor([[False, True], [False, False], [True, False]])
    same_heads_are_nan(made, q, both(L, made, q), nan)


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("tokens", [1, 3])
@pytest.mark.parametrize("prefix", [23, 24, 25, 64])
def test_keys(L, dtype, q8, tokens, prefix):
    # all or some of a member's own keys, behind a prefix of some pieces (eight of 24 pages: its own one is folded apart from them), and one
    # key of another group's prefix
    made = Grouped(dtype, q8, 1, 64, [(prefix, [3, 0, 90]), (2, [5, -4])], seed=23)
    q = torch.randn(5, 4, 128, generator=made.g).to(dtype)
    places = [(int(made.table[0, prefix]), t) for t in range(tokens)] + [(int(made.table[3, 1]), 17)]
    for page, t in places:
        if q8:
            made.k_pages.view(torch.uint8)[page, 0, t, 9] = 0x7f      # NaN
        else:
            made.k_pages[page, 0, t, 9] = math.nan
    nan = torch.tensor([True, False, False, True, False])[:, None].expand(5, 4)
    same_heads_are_nan(made, q, both(L, made, q), nan)
