"""page_evict_select refuses outputs that lie over the lists which all of its workgroups read, and over one another (no GPU needed: nothing is
launched)."""
import ctypes

import pytest

from tests.test_paged_more_refusals import select
from tests.test_paged_refusals import INVALID, L, WORKSPACE, pages  # noqa: F401

BATCH, HKV = 6, 2
READ, WRITTEN = ("len", "keep", "first", "seen"), ("new", "status", "count")
WORDS = dict(len=BATCH, keep=BATCH, first=BATCH, seen=BATCH, new=BATCH, status=BATCH, count=BATCH * HKV)
PAIRS = [(w, r) for w in WRITTEN for r in READ] + [("new", "status"), ("new", "count"), ("status", "count")]


def apart():
    return {name: (i + 1) << 20 for i, name in enumerate(WORDS)}


@pytest.mark.parametrize("written,other", PAIRS, ids=["-".join(p) for p in PAIRS])
def test_select(L, written, other):
    s = pages(L, batch=BATCH, hkv=HKV)
    at = apart()
    call = lambda **kw: select(L, s, **{k: ctypes.c_void_p(v) if v else None for k, v in {**at, **kw}.items()})  # noqa: E731
    # the same place, the last word of one over the first of the other, one within the other
    for place in (at[other], at[other] + 4 * (WORDS[other] - 1), at[other] - 4 * (WORDS[written] - 1)):
        assert call(**{written: place}) == INVALID
    # (one behind the other, either way: the workspace is what is found fault with)
    for place in (at[other] + 4 * WORDS[other], at[other] - 4 * WORDS[written]):
        assert call(**{written: place}, ws=0) == WORKSPACE
    # lists that are not there lie over nothing
    assert call(first=0, status=0, ids=0, seen=0, ws=0) == WORKSPACE
