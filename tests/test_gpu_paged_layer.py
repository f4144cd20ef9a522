"""PagedLayer's calls for caches that are shared and kept within bounds, together: members of a group are evicted while the others go on
reading the pages that all of them list."""
import pytest
import torch

from tests.test_gpu_paged import BF16, F32, KIND_IDS, KINDS, L, check_rows  # noqa: F401

pytestmark = pytest.mark.gpu
i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731


@pytest.mark.parametrize("dtype,q8", KINDS, ids=KIND_IDS)
def test_members_of_a_group_are_evicted(L, dtype, q8):
    g = torch.Generator().manual_seed(31)
    B, hq, hkv, page, prefix, own, keep = 5, 8, 2, 16, 3, 4, 3 * 16 + 20
    max_pages, first = prefix + own, prefix * page
    table = torch.empty(B, max_pages, dtype=torch.int32)
    order = torch.randperm(prefix + own * B, generator=g).int()
    table[:, :prefix] = order[:prefix]
    table[:, prefix:] = order[prefix:].reshape(B, own)
    shared_pages, n_pages = order[:prefix].long().cuda(), prefix + own * B
    table, seq_len, n_seen = table.cuda(), i32([first] + [0] * (B - 1)), i32([first] * B)
    layer = L.PagedLayer(table, seq_len, hq, hkv, n_pages, page, dtype, L.E4M3 if q8 else None, rope=L.rope_table(400, 128).cuda(),
                         groups=1, evicts=32)
    # (the prefix is weighed by nobody before the steps: its numbers are its places)
    layer.token_id.copy_(torch.arange(max_pages * page, dtype=torch.int32, device="cuda").expand_as(layer.token_id))
    rows = lambda n: (lambda x: (x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:]))(  # noqa: E731
        torch.randn(n, hq + 2 * hkv, 128, generator=g).to(dtype).cuda())
    layer.prompt(*rows(first), i32([0] + [first] * B), position=torch.arange(first, dtype=torch.int32, device="cuda")[None])
    seq_len.fill_(first)

    def pools():
        return [layer.k_pages.view(torch.uint8)] + [layer.v_pages.view(torch.uint8)] + ([layer.k_scale, layer.v_scale] if q8 else [])

    def held(which, b):
        pool, scale = ((layer.k_pages, layer.k_scale), (layer.v_pages, layer.v_scale))[which]
        x = pool[table[b].long()].float().double()
        if q8:
            x = x * scale[table[b].long()].double()[..., None, None]
        return x.transpose(0, 1).reshape(hkv, -1, 128)[:, : int(seq_len[b])].cpu()

    shared, n_first, off, group_pages = [p[shared_pages].clone() for p in pools()], i32([first] * B), i32([0, B]), i32([prefix])
    evictions = 0
    for step in range(40):
        seq_len.add_(1)
        n_seen.add_(1)
        q = layer.append(*rows(B), position=(n_seen - 1)[None].contiguous())
        out = layer.attend_shared(q, off, group_pages)
        layer.weigh(q, n_seen)
        torch.cuda.synchronize()
        check_rows(L, None, out, layer.lse, [(b, q[b].cpu(), held(0, b), held(1, b)) for b in range(B)], 0.0 if dtype == F32 else 2.0 ** -16,
                   2.0 ** -23)
        if step % 7 == 6:
            # (some stay as they are)
            keeps = [keep, 1 << 20, keep + 3, keep, first]
            lens = seq_len.tolist()
            seq_len.copy_(layer.evict(i32(keeps), n_seen, n_first, 4))
            torch.cuda.synchronize()
            assert seq_len.tolist() == [min(n, k) for n, k in zip(lens, keeps)] and layer.evict_status.tolist() == [0] * B
            evictions += int(layer.move_count.sum())
            assert all(torch.equal(p[shared_pages], s) for p, s in zip(pools(), shared))
            for b in range(B):
                assert torch.equal(layer.token_id[b, :, :first].cpu(), torch.arange(first, dtype=torch.int32).expand(hkv, -1))
    assert evictions > 0
