"""The operators that keep a paged cache within bounds and share it, as cases that can be timed.

A case is a dict of plain values.  `op` names the operator:

  append  new queries, keys and values into the pages with positions of their own on one to three axes, where the place in
          the cache does not say the position: after an eviction, or for images and video
  shared  attention of one token per sequence for a batch whose groups share a prefix: its pages are read once for all
  weigh   what each cached token got of the attention of the call's queries, added to what it got before
  select  which tokens stay: the first ones, the most recent ones and those with the most weight; lists the rows that move
  move    the listed rows to the places that became free, in keys, values, weights and numbers; abstracts of those pages

`dtype` is the model's type, `store` what the pages hold: "model" or "e4m3" (8 bits with a scale for each page and kv head).
`ctx` is the longest sequence's length (with `ragged` the others are shorter; for `shared` without the prefix), `new` the
most rows of a sequence (1: one each), `groups` and `prefix` how many groups and how long the longest prefix, `keep` how many
tokens stay, `first` and `recent` how many of them whatever they weigh, `rot` the rotated channels, `pairs` which of them
rotate together, `axes` the axes of a position and `layout` which pairs belong to which ("sections" or "turns").

Pages lie scattered over the pool.  Keys and values are Gaussian with a gain of their own for each page, a few key channels
carry outliers.
"""
import math

import numpy as np
import torch

own = False

D = 128
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
ROPE_LEN = 32768
# exponents of a page's scale: scale * code stays a number of the model's type
EXPONENTS = {"f16": (-15, 7), "bf16": (-100, 118)}


def _case(op, dtype, store, batch, hq, hkv, ctx, new=1, page=64, groups=0, prefix=0, keep=0, first=0, recent=0, rot=128,
          pairs="halves", axes=1, layout="sections", ragged=True, bounds=True):
    return {"op": op, "dtype": dtype, "store": store, "batch": batch, "hq": hq, "hkv": hkv, "ctx": ctx, "new": new,
            "page": page, "groups": groups, "prefix": prefix, "keep": keep, "first": first, "recent": recent, "rot": rot,
            "pairs": pairs, "axes": axes, "layout": layout, "ragged": ragged, "bounds": bounds}


def listed():
    cases = [
        # one user's next token, after evictions: the position is not the place
        ("append 1 token bf16", _case("append", "bf16", "model", 1, 32, 8, 4095, ragged=False)),
        # prompts of text and images: time, height and width, in sections of the pairs
        ("append image prompts f16", _case("append", "f16", "model", 3, 32, 8, 5001, new=4097, axes=3)),
        # many users' next tokens into the 8-bit pages, three axes by turns
        ("append 96 tokens e4m3 3 axes", _case("append", "bf16", "e4m3", 96, 32, 8, 3000, page=32, axes=3, layout="turns")),
        # four samples of one prompt, multi-head attention in fp32
        ("shared f32 1K x4", _case("shared", "f32", "model", 4, 8, 8, 40, page=16, groups=1, prefix=1024)),
        # a system prompt and documents that everybody asks about
        ("shared bf16 32K x48", _case("shared", "bf16", "model", 48, 32, 8, 900, groups=1, prefix=32768)),
        # several prompts with some samples each, eight query heads per group, 8 bits
        ("shared e4m3 g8 9 groups x70", _case("shared", "bf16", "e4m3", 70, 64, 8, 2001, page=16, groups=9, prefix=9000)),
        # a decode step of sixteen users: every key is looked at once
        ("weigh bf16 33K x16", _case("weigh", "bf16", "model", 16, 32, 8, 33001)),
        # a prompt's tokens weighed by all of its queries
        ("weigh prompt f16 4K", _case("weigh", "f16", "model", 1, 32, 8, 4096, new=4096, ragged=False)),
        # many users that outgrew their budget by a little
        ("select 4.2K of x40", _case("select", "bf16", "model", 40, 32, 8, 4224, keep=4096, first=4, recent=512)),
        # long prompts brought down to a budget
        ("select 130K x2", _case("select", "bf16", "model", 2, 32, 8, 130001, keep=20001, first=64, recent=1001)),
        # a budget of 4096 kept up after some steps, with abstracts for the selection of pages
        ("move bf16 4.2K x40", _case("move", "bf16", "model", 40, 32, 8, 4224, keep=4095, first=4, recent=512)),
        # long prompts brought down to a budget, 8-bit pages
        ("move e4m3 60K x6", _case("move", "f16", "e4m3", 6, 32, 8, 60001, keep=16384, first=64, recent=1024)),
    ]
    return [dict(case, name=name) for name, case in cases]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["append", "shared", "shared", "weigh", "weigh", "select", "move"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    store = "model" if dtype == "f32" else rng.choice(["model", "e4m3"])
    hkv = rng.choice([1, 2, 4, 8, 8, 16, 32])
    group = min(rng.choice([1, 2, 4, 4, 8]), 64 // hkv)
    page = rng.choice([16, 32, 64, 64, 128, 256])
    c = _case(op, dtype, store, 1, hkv * group, hkv, 1, page=page, rot=rng.choice([128, 128, 64]),
              pairs=rng.choice(["halves", "neighbours"]), axes=rng.choice([1, 2, 3, 3]), layout=rng.choice(["sections", "turns"]),
              ragged=rng.random() < 0.8, bounds=rng.random() < 0.5)
    if op == "append":
        if rng.random() < 0.5:
            c["batch"], c["ctx"] = _log_uniform(rng, 1, 128), _log_uniform(rng, 64, 12000)
        else:
            c["batch"] = _log_uniform(rng, 1, 6)
            c["new"] = _log_uniform(rng, 2, 12000 // c["batch"])
            c["ctx"] = c["new"] + rng.choice([0, _log_uniform(rng, 1, 4096)])
        while c["batch"] * (c["ctx"] + page) * hkv > 1 << 21:
            c["ctx"] = c["ctx"] // 2 + 1
            c["new"] = min(c["new"], c["ctx"])
    elif op == "shared":
        most = 1 << (19 if dtype != "f32" else 16)                      # (kv head, prefix token) pairs of all groups
        c["groups"] = _log_uniform(rng, 1, 12)
        c["prefix"] = _log_uniform(rng, page, max(page, min(65536, most // (hkv * c["groups"]))))
        logits = 1 << (28 if dtype != "f32" else 24)
        c["batch"] = c["groups"] + _log_uniform(rng, 1, max(1, min(128, logits // (c["prefix"] * c["hq"]))))
        c["ctx"] = _log_uniform(rng, 1, max(1, min(4000, (1 << 20) // (c["batch"] * hkv))))
    elif op == "weigh":
        if rng.random() < 0.5:
            c["ctx"] = _log_uniform(rng, 1, 65536)
            c["batch"] = _log_uniform(rng, 1, max(1, min(64, (1 << (22 if dtype != "f32" else 19)) // (c["ctx"] * hkv))))
        else:
            logits = 1 << (29 if dtype != "f32" else 25)
            c["new"] = _log_uniform(rng, 2, 4096 if dtype != "f32" else 1024)
            c["ctx"] = c["new"] + rng.choice([0, _log_uniform(rng, 1, 32768)])
            while c["new"] * c["ctx"] * c["hq"] > logits:
                c["new"], c["ctx"] = (c["new"] // 2, c["ctx"]) if c["new"] > c["ctx"] // 2 else (c["new"], max(c["new"], c["ctx"] // 2))
            c["new"] = max(c["new"], 2)
            c["ctx"] = max(c["new"], c["ctx"])
            c["batch"] = _log_uniform(rng, 1, max(1, min(8, logits // (c["new"] * c["ctx"] * c["hq"]))))
    else:
        c["ctx"] = _log_uniform(rng, 100, 131072)
        c["batch"] = _log_uniform(rng, 1, max(1, min(64, (1 << (21 if op == "select" else 20)) // (c["ctx"] * hkv))))
        c["keep"] = min(c["ctx"] - 1, _log_uniform(rng, 64, c["ctx"])) if rng.random() < 0.5 else max(32, c["ctx"] - _log_uniform(rng, 1, 300))
        if op == "move" and store == "e4m3":
            c["keep"] = max(page, c["keep"] // page * page)            # (whole pages are kept where each has a scale)
            c["ctx"] = max(c["ctx"], c["keep"] + 1)
        c["first"] = rng.choice([0, 4, min(64, c["keep"] // 4)])
        c["recent"] = _log_uniform(rng, 1, max(1, c["keep"] // 2))
    return c


# ---- the case's lengths (of the case alone, so that work() knows them) ---------------------------------

def _lengths(case):
    """Length after the call and rows of every sequence."""
    rng = np.random.default_rng(case["ctx"] * 131 + case["batch"])
    B, ctx, new = case["batch"], case["ctx"], case["new"]
    n_new = np.full(B, new, np.int64)
    if case["ragged"] and new > 1:
        n_new[1:] = rng.integers(1, new + 1, B - 1)
    length = np.full(B, ctx, np.int64)
    if case["ragged"]:
        if case["op"] in ("select", "move") and case["keep"] > ctx // 2:      # they all outgrew their budget, but for a few
            length[1:] = rng.integers(case["keep"] - 1, ctx + 1, B - 1)
        else:
            length[1:] = n_new[1:] + (rng.random(B - 1) * (ctx - n_new[1:] + 1)).astype(np.int64)
    return length, n_new


def _groups(case):
    """group_off and the pages that each group shares."""
    rng = np.random.default_rng(case["prefix"] * 17 + case["groups"])
    n, page = case["groups"], case["page"]
    off = np.zeros(n + 1, np.int64)
    off[n] = case["batch"]
    off[1:n] = np.sort(rng.choice(np.arange(1, case["batch"]), n - 1, replace=False))
    pages = np.full(n, max(1, case["prefix"] // page), np.int64)
    pages[1:] = rng.integers(0, pages[0] + 1, n - 1)
    return off, pages


def work(case):
    length, n_new = _lengths(case)
    e = BYTES[case["dtype"]]
    es = 1 if case["store"] == "e4m3" else e
    B, hq, hkv, page = case["batch"], case["hq"], case["hkv"], case["page"]
    g = hq // hkv
    if case["op"] == "append":
        t = int(n_new.sum())
        first, last = (length - n_new) // page, (length - 1) // page
        rows = t * (2 * hq + 2 * hkv) * D * e + t * 2 * hkv * D * es + t * (case["rot"] + case["axes"]) * 4
        held = int(((length - n_new) % page).sum()) * hkv * D * es      # of pages that were begun, for their abstracts
        return {"bytes": rows + held + int((last - first + 1).sum()) * hkv * 2 * D * e, "flops": 3 * t * (hq + hkv) * case["rot"]}
    if case["op"] == "shared":
        off, pages = _groups(case)
        members = np.diff(off)
        stored = int((pages * page).sum() + length.sum()) * hkv
        seen = int((members * pages * page).sum() + length.sum()) * hq
        return {"bytes": stored * 2 * D * es + B * hq * D * (e + 4) + B * hq * 4, "flops": 4 * seen * D}
    if case["op"] == "weigh":
        tokens, rows = int(length.sum()) * hkv, int(n_new.sum())
        pairs = int((n_new * (length - n_new) + n_new * (n_new + 1) // 2).sum())
        return {"bytes": tokens * (D * es + 8) + rows * hq * (D * e + 4), "flops": 2 * hq * D * pairs}
    out = np.maximum(length - case["keep"], 0)
    if case["op"] == "select":
        return {"bytes": int(length.sum()) * hkv * 8 + int(_moved(case).sum()) * 8 + B * hkv * 4, "flops": int(length.sum()) * hkv}
    moved = _moved(case)
    moved_bytes = 2 * int(moved.sum()) * (2 * D * es + 8) + int(moved.sum()) * 8
    if not case["bounds"]:
        return {"bytes": moved_bytes, "flops": 0}
    # the pages that rows move to are read whole, for their abstracts (at most one for each row that moves)
    touched = np.minimum(moved, -(-np.minimum(length, case["keep"]) // page)[:, None])
    return {"bytes": moved_bytes + int(touched.sum()) * (page * D * es + 2 * D * e), "flops": 2 * int(touched.sum()) * page * D + int(out.sum())}


def _moved(case):
    """Rows that move, per (sequence, kv head): those that stay behind the kept length (expected: in proportion, the recent ones
    for sure)."""
    length, _ = _lengths(case)
    keep = np.minimum(case["keep"], length)
    out = length - keep
    recent = np.minimum(case["recent"], keep)
    rest = np.maximum(length - recent - case["first"], 1)
    share = np.maximum(keep - recent - case["first"], 0) / rest
    behind = np.maximum(out - recent, 0)
    moved = np.minimum(out, np.minimum(out, recent) + (behind * share).astype(np.int64))
    return np.repeat(np.minimum(moved, keep)[:, None], case["hkv"], 1)


# ---- inputs ----------------------------------------------------------------------------------------------

def _cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _pools(case, gen, n_pages, names="kv"):
    """Gaussian, each page with a gain of its own, outlier channels in the keys."""
    hkv, page, dt = case["hkv"], case["page"], DTYPES[case["dtype"]]
    got = {}
    for name in names:
        gain = 2.0 ** torch.randint(-1, 2, (n_pages, hkv, 1, 1), generator=gen, device="cuda").float()
        scale = None
        if case["store"] == "e4m3":
            pool = torch.empty(n_pages, hkv, page, D, dtype=torch.float8_e4m3fn, device="cuda")
            scale = gain.reshape(n_pages, hkv) * (2.0 ** -4 if name == "k" else 2.0 ** -6)
        else:
            pool = torch.empty(n_pages, hkv, page, D, dtype=dt, device="cuda")
        step = max(1, (1 << 26) // (hkv * page * D))
        for i in range(0, n_pages, step):
            x = torch.randn(pool[i: i + step].shape, generator=gen, device="cuda") * gain[i: i + step]
            if name == "k":
                x[..., :4] *= 4.0
            if scale is not None:
                x = (x / scale[i: i + step, :, None, None]).clamp(-448.0, 448.0)
            pool[i: i + step] = x.to(pool.dtype)
        got[name + "_pages"], got[name + "_scale"] = pool, scale
    return got


def _positions(case, rng, length, n_new):
    """Places on the axes for every new row: [axes, rows].  One axis: behind some tokens that were evicted.  More: stretches of
    text, where all axes go on together, and images, whose rows and columns count from where they begin."""
    parts = []
    for n, m in zip(length, n_new):
        if case["axes"] == 1:
            parts.append((np.arange(m) + n - m + rng.integers(0, 8000))[None])
            continue
        at, base, cols = 0, int(n - m), []
        while at < m:
            if rng.random() < 0.5:
                k = int(min(m - at, rng.integers(1, 300)))
                cols.append(np.repeat((base + np.arange(k))[None], case["axes"], 0))
                base += k
            else:
                w = int(rng.integers(4, 40))
                k = int(min(m - at, w * rng.integers(4, 40)))
                i = np.arange(k)
                cols.append(np.stack([np.full(k, base), base + i // w, base + i % w][: case["axes"]]))
                base += int(max(w, k // w + 1))
            at += k
        parts.append(np.concatenate(cols, 1))
    return np.minimum(np.concatenate(parts, 1), ROPE_LEN - 1).astype(np.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    dt, B, hq, hkv, page, op = DTYPES[case["dtype"]], case["batch"], case["hq"], case["hkv"], case["page"], case["op"]
    length, n_new = _lengths(case)
    s = {"case": case, "dtype": dt, "scale": 1.0 / math.sqrt(D)}
    if op == "select":
        return _prepare_select(s, case, gen, length)
    if op == "shared":
        off, shared = _groups(case)
        member_of = np.repeat(np.arange(case["groups"]), np.diff(off))
        before = shared[member_of]                              # pages of the prefix that each sequence lists first
        own_len = length
        length = own_len + before * page
    else:
        before = np.zeros(B, np.int64)
        own_len = length
    pages = -(-length // page)
    max_pages = int(pages.max()) + 1                            # room to grow
    n_pages = int((pages - before).sum()) + (int(shared.sum()) if op == "shared" else 0) + 3
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((B, max_pages), -1, np.int32)
    at = 0
    if op == "shared":
        for g in range(case["groups"]):
            table[off[g]: off[g + 1], : shared[g]] = order[at: at + shared[g]]
            at += shared[g]
    for b in range(B):
        table[b, before[b]: pages[b]] = order[at: at + pages[b] - before[b]]
        at += pages[b] - before[b]
    new_off = np.zeros(B + 1, np.int32)
    new_off[1:] = np.cumsum(n_new)
    s.update(_pools(case, gen, n_pages, "k" if op == "weigh" else "kv"))
    s.update(length=_cuda(length.astype(np.int32)), table=_cuda(table), n_pages=n_pages, max_pages=max_pages,
             new_off=_cuda(new_off) if case["new"] > 1 else None, widest=int(pages.max()), longest=int(length.max()))
    t = int(n_new.sum())
    if op == "append":
        return _prepare_append(s, case, gen, rng, length, n_new, new_off)
    if op == "move":
        return _prepare_move(s, case, gen, rng, length)
    s["q"] = torch.randn(t, hq, D, generator=gen, device="cuda").to(dt)
    if op == "shared":
        s.update(group_off=_cuda(off.astype(np.int32)), group_pages=_cuda(shared.astype(np.int32)),
                 groups=[(int(off[g]), int(off[g + 1]), int(shared[g])) for g in range(case["groups"])],
                 before=_cuda(before), widest_own=int((pages - before).max()),
                 out=torch.empty(B, hq, D, dtype=torch.float32, device="cuda"),
                 lse=torch.empty(B, hq, dtype=torch.float32, device="cuda"))
        return s
    # what the attention call of the same queries left: the logarithms of its sums (here: of a sample of the keys, which is
    # near enough for weights of the right size)
    cap = max_pages * page
    lse = 0.5 * float(np.log(8.0)) + torch.rand(t, hq, generator=gen, device="cuda")
    seen = torch.from_numpy(np.concatenate([np.arange(n - m + 1, n + 1) for n, m in zip(length, n_new)]).astype(np.float32)).cuda()
    s.update(lse=lse + 2.0 + seen.log()[:, None], weight_before=torch.rand(B, hkv, cap, generator=gen, device="cuda"),
             weight=torch.zeros(B, hkv, cap, device="cuda"), token_id=torch.zeros(B, hkv, cap, dtype=torch.int32, device="cuda"),
             n_seen=_cuda((length + rng.integers(0, 5000, B)).astype(np.int32)), rows=_cuda(n_new), most_new=int(n_new.max()),
             starts=_cuda(new_off[:-1].astype(np.int64)), decay=0.98)
    return s


def _prepare_append(s, case, gen, rng, length, n_new, new_off):
    dt, B, hq, hkv, page = s["dtype"], case["batch"], case["hq"], case["hkv"], case["page"]
    t, max_pages = int(n_new.sum()), s["max_pages"]
    # one projection's output: queries, keys and values of a token beside each other
    qkv = torch.randn(t, hq + 2 * hkv, D, generator=gen, device="cuda")
    qkv[:, hq: hq + hkv, :4] *= 4.0
    qkv = qkv.to(dt)
    s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq: hq + hkv], qkv[:, hq + hkv:]
    s["q_out"] = torch.empty(t, hq, D, dtype=dt, device="cuda")
    half = case["rot"] // 2
    angle = (torch.arange(ROPE_LEN, dtype=torch.float64, device="cuda")[:, None]
             * 500000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half))
    s["rope"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
    s["position"] = _cuda(_positions(case, rng, length, n_new))
    if case["layout"] == "turns":
        axis = np.arange(half) % case["axes"]
    else:                                                   # a quarter of the pairs to the first axis, the rest evenly
        first = half if case["axes"] == 1 else half // 4
        axis = np.where(np.arange(half) < first, 0, 1 + (np.arange(half) - first) * (case["axes"] - 1) // max(1, half - first))
    s["axis"] = _cuda(axis.astype(np.int32))
    s["status"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    s["chunk_off"] = (torch.arange(max_pages + 1, dtype=torch.int32, device="cuda") * page).repeat(B, 1)
    s["n_chunks"] = _cuda(((length - n_new) // page).astype(np.int32))
    # what the scheduler of a serving program knows on the host: every new token's sequence and place, and the pages that
    # the call touches
    seq = np.repeat(np.arange(B), n_new)
    pos = np.arange(t) - np.repeat(new_off[:-1], n_new) + np.repeat(length - n_new, n_new)
    first = (length - n_new) // page
    count = (length - 1) // page - first + 1
    base = np.zeros(B, np.int64)
    base[1:] = np.cumsum(count)[:-1]
    touched_seq = np.repeat(np.arange(B), count)
    touched_page = np.arange(int(count.sum())) - np.repeat(base, count) + np.repeat(first, count)
    s["seq"], s["pos"] = _cuda(seq), _cuda(pos)
    s["slot"] = _cuda(base[seq] + pos // page - first[seq])
    s["touched_seq"], s["touched_page"] = _cuda(touched_seq), _cuda(touched_page)
    s["start"] = _cuda(length - n_new)
    s["abstract"] = torch.zeros(B, hkv, max_pages, 2, D, dtype=dt, device="cuda")
    return s


def _scores(case, gen, length, cap):
    """Accumulated weights: most tokens got little, some much, a few nothing at all."""
    B, hkv = case["batch"], case["hkv"]
    w = torch.exp(2.0 * torch.randn(B, hkv, cap, generator=gen, device="cuda"))
    w[torch.rand(B, hkv, cap, generator=gen, device="cuda") < 0.05] = 0.0
    # the tokens' numbers, as earlier evictions left them: kept ones with gaps, moved ones in other ones' places
    seen = length + 5000
    ids = torch.arange(cap, device="cuda").expand(B, hkv, cap) + 5000
    swap = torch.rand(B, hkv, cap, generator=gen, device="cuda") < 0.3
    old = torch.arange(cap, device="cuda") < (_cuda(length) - case["recent"]).clamp_min(0)[:, None, None]
    ids = torch.where(swap & old, torch.randint(0, 5000, (B, hkv, cap), generator=gen, device="cuda"), ids)
    return w, ids.int(), _cuda(seen.astype(np.int32))


def _prepare_select(s, case, gen, length):
    B, hkv, page = case["batch"], case["hkv"], case["page"]
    s["max_pages"] = -(-int(length.max()) // page) + 1
    s["n_pages"] = s["max_pages"] * B
    cap = s["max_pages"] * page
    s["weight"], s["token_id"], s["n_seen"] = _scores(case, gen, length, cap)
    s["length"], s["longest"] = _cuda(length.astype(np.int32)), int(length.max())
    s["keep_len"] = torch.full((B,), case["keep"], dtype=torch.int32, device="cuda")
    s["n_first"] = torch.full((B,), case["first"], dtype=torch.int32, device="cuda")
    most = max(1, min(case["keep"], int(length.max()) - case["keep"]))
    s["moves"] = torch.full((B, hkv, most, 2), -1, dtype=torch.int32, device="cuda")
    s["move_count"] = torch.zeros(B, hkv, dtype=torch.int32, device="cuda")
    s["new_len"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    s["status"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    return s


def _prepare_move(s, case, gen, rng, length):
    """The list as a selection makes it: the i-th place that became free takes the i-th row that stays behind the kept length."""
    B, hkv, page, keep = case["batch"], case["hkv"], case["page"], case["keep"]
    cap = s["max_pages"] * page
    s["weight"], s["token_id"], _ = _scores(case, gen, length, cap)
    most = max(1, min(keep, int(length.max()) - keep))
    moves = np.full((B, hkv, most, 2), -1, np.int32)
    count = np.zeros((B, hkv), np.int32)
    for b in range(B):
        n = int(length[b])
        if n <= keep:
            continue
        for h in range(hkv):
            score = rng.random(n, dtype=np.float32)
            score[n - min(n, case["recent"]):] = 2.0
            score[: case["first"]] = 3.0
            stays = np.zeros(n, bool)
            stays[np.argpartition(-score, keep - 1)[:keep]] = True
            free, behind = np.flatnonzero(~stays[:keep]), keep + np.flatnonzero(stays[keep:])
            count[b, h] = len(free)
            moves[b, h, : len(free), 0], moves[b, h, : len(free), 1] = free, behind
    s.update(moves=_cuda(moves), move_count=_cuda(count), new_len=_cuda(np.minimum(length, keep).astype(np.int32)),
             abstract=None, chunk_off=None, n_chunks=None)
    if case["bounds"]:
        s["abstract"] = torch.zeros(B, hkv, s["max_pages"], 2, D, dtype=s["dtype"], device="cuda")
        s["chunk_off"] = (torch.arange(s["max_pages"] + 1, dtype=torch.int32, device="cuda") * page).repeat(B, 1)
        s["chunk_off"] = torch.minimum(s["chunk_off"], s["length"][:, None]).contiguous()
        s["n_chunks"] = ((s["length"] + page - 1) // page).int()
    return s


def _values(pool, scale, phys):
    """What the pages `phys` hold, in 32 bits."""
    x = pool[phys].float()
    return x if scale is None else x * scale[phys][..., None, None]


# ---- one pass ----------------------------------------------------------------------------------------------

def run(s):
    return (_OWN if own else _PLAIN)[s["case"]["op"]](s)


def _own_pages(s):
    import paper_2506_20187_amd as L
    if "pages" not in s:
        c = s["case"]
        rot = c["rot"] if c["op"] == "append" else 0
        s["pages"] = L.make_pages(c["batch"], c["hq"], c["hkv"], D, s["n_pages"], c["page"], s["max_pages"], s["dtype"],
                                  L.E4M3 if c["store"] == "e4m3" else s["dtype"], rot_dim=rot,
                                  interleaved=c["pairs"] == "neighbours", rope_len=ROPE_LEN if rot else 0)
        if c["op"] == "shared":
            s["workspace"] = torch.empty(L.leoam_page_shared_workspace_bytes(s["pages"], c["groups"]), dtype=torch.uint8, device="cuda")
        if c["op"] == "select":
            s["workspace"] = torch.empty(L.leoam_page_evict_workspace_bytes(s["pages"]), dtype=torch.uint8, device="cuda")
    return L, s["pages"]


def _own_append(s):
    L, pages = _own_pages(s)
    L.kv_page_append_at(pages, s["q"], s["k"], s["v"], s["new_off"], s["length"], s["table"], s["rope"], s["position"], s["axis"],
                        s["q_out"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["abstract"], s["chunk_off"],
                        s["n_chunks"], s["status"])
    return _appended(s)


def _own_shared(s):
    L, pages = _own_pages(s)
    L.page_attention_decode_shared(pages, s["q"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["table"], s["length"],
                                   s["group_off"], s["group_pages"], s["scale"], s["out"], s["lse"], s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_weigh(s):
    L, pages = _own_pages(s)
    L.page_weight_add(pages, s["q"], s["new_off"], s["k_pages"], s["k_scale"], s["table"], s["length"], s["scale"], s["lse"],
                      s["decay"], s["weight_before"], s["weight"], s["n_seen"], s["token_id"])
    return {"weight": s["weight"], "token_id": s["token_id"]}


def _own_select(s):
    L, pages = _own_pages(s)
    L.page_evict_select(pages, s["weight"], s["token_id"], s["n_seen"], s["length"], s["keep_len"], s["n_first"], s["case"]["recent"],
                        s["moves"], s["move_count"], s["new_len"], s["status"], s["workspace"])
    return {"moves": s["moves"], "count": s["move_count"], "new_len": s["new_len"]}


def _own_move(s):
    L, pages = _own_pages(s)
    L.kv_page_move(pages, s["moves"], s["move_count"], s["length"], s["new_len"], s["table"], s["k_pages"], s["v_pages"],
                   s["k_scale"], s["v_scale"], s["weight"], s["token_id"], s["abstract"], s["chunk_off"], s["n_chunks"])
    return _moved_to(s)


def _appended(s):
    got = {"q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"], "abstract": s["abstract"], "chunk_off": s["chunk_off"],
           "n_chunks": s["n_chunks"]}
    if s["k_scale"] is not None:
        got.update(k_scale=s["k_scale"], v_scale=s["v_scale"])
    return got


def _moved_to(s):
    got = {"k": s["k_pages"], "v": s["v_pages"], "weight": s["weight"], "token_id": s["token_id"]}
    if s["k_scale"] is not None:
        got.update(k_scale=s["k_scale"], v_scale=s["v_scale"])
    if s["abstract"] is not None:
        got.update(abstract=s["abstract"], chunk_off=s["chunk_off"], n_chunks=s["n_chunks"])
    return got


# ---- the plain forms ---------------------------------------------------------------------------------------

def _rotated(x, cos, sin, rot, pairs):
    """Rows x [T, H, D] with their first `rot` channels rotated; cos, sin [T, 1, rot / 2]."""
    if pairs == "halves":
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = x[..., 0: rot: 2], x[..., 1: rot: 2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _scale_of(amax, exponents):
    """The smallest power of two s with amax <= 448 s = 0.875 * 2^9 s, its exponent in `exponents`; 0 for 0."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(*exponents)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.zeros_like(amax))


def _codes(x, scale):
    y = torch.where(scale > 0, x / scale.clamp_min(2.0 ** -110), torch.zeros_like(x))
    return y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _append(s):
    c = s["case"]
    page, rot, half = c["page"], c["rot"], c["rot"] // 2
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    at_pair = s["position"].long()[s["axis"].long()].transpose(0, 1)          # [T, half]: a position for every pair
    pair = torch.arange(half, device="cuda")
    cos, sin = s["rope"][at_pair, pair][:, None], s["rope"][at_pair, half + pair][:, None]
    q, k = _rotated(q, cos, sin, rot, c["pairs"]), _rotated(k, cos, sin, rot, c["pairs"])
    s["q_out"].copy_(q)
    ts, tp = s["touched_seq"], s["touched_page"]
    phys = s["table"][ts, tp].long()                                       # [U]
    at = s["table"][s["seq"], s["pos"] // page].long()                     # [T] page of every new token
    slot = s["pos"] % page
    inside = tp[:, None] * page + torch.arange(page, device="cuda")        # [U, page] places
    held = inside < s["start"][ts][:, None]
    begun = held[:, 0]
    for name, x in (("k", k), ("v", v)):
        pool, scale = s[name + "_pages"], s[name + "_scale"]
        if scale is None:
            pool[at, :, slot] = x.to(pool.dtype)
            continue
        old = torch.where(begun[:, None], scale[phys], 0.0)                 # [U, Hkv]
        top = torch.zeros_like(old).scatter_reduce_(0, s["slot"][:, None].expand(-1, c["hkv"]), x.abs().amax(-1), "amax")
        now = torch.maximum(old, _scale_of(top, EXPONENTS[c["dtype"]]))
        again = _codes(pool[phys].float() * old[..., None, None], now[..., None, None])
        pool[phys] = torch.where(held[:, None, :, None], again.float(), pool[phys].float()).to(pool.dtype)
        scale[phys] = now
        pool.view(torch.uint8)[at, :, slot] = _codes(x, now[s["slot"]][..., None]).view(torch.uint8)
    stored = _values(s["k_pages"], s["k_scale"], phys)                     # [U, Hkv, page, D]
    valid = (inside < s["length"][ts][:, None])[:, None, :, None]
    s["abstract"][ts, :, tp, 0] = torch.where(valid, stored, -math.inf).amax(2).to(s["dtype"])
    s["abstract"][ts, :, tp, 1] = torch.where(valid, stored, math.inf).amin(2).to(s["dtype"])
    s["chunk_off"][ts, tp + 1] = torch.minimum((tp + 1) * page, s["length"][ts]).int()
    s["n_chunks"].copy_((s["length"] + page - 1) // page)
    return _appended(s)


def _shared(s):
    c = s["case"]
    B, hkv, g, page = c["batch"], c["hkv"], c["hq"] // c["hkv"], c["page"]
    q = s["q"].float().reshape(B, hkv, g, D)
    # each sequence's own pages
    at = s["before"][:, None] + torch.arange(s["widest_own"], device="cuda")
    phys = torch.gather(s["table"].long(), 1, at.clamp_max(s["max_pages"] - 1)).clamp_min(0)
    K, V = (_values(s[x + "_pages"], s[x + "_scale"], phys).transpose(1, 2).reshape(B, hkv, -1, D) for x in "kv")
    place = s["before"][:, None] * page + torch.arange(K.shape[2], device="cuda")
    z = torch.matmul(q, K.transpose(-1, -2)).mul_(s["scale"])
    z.masked_fill_((place >= s["length"][:, None])[:, None, None], -math.inf)
    m = z.amax(-1, keepdim=True)
    p = z.sub_(m).exp_()
    total, acc = p.sum(-1, keepdim=True), torch.matmul(p, V)
    # the prefix of each group, for all of its members at once
    for b0, b1, pages in s["groups"]:
        if pages == 0:
            continue
        ids = s["table"][b0, :pages].long()
        K, V = (_values(s[x + "_pages"], s[x + "_scale"], ids).transpose(0, 1).reshape(hkv, -1, D) for x in "kv")
        qg = q[b0:b1].transpose(0, 1).reshape(hkv, -1, D)
        z = torch.matmul(qg, K.transpose(-1, -2)).mul_(s["scale"])
        m1 = z.amax(-1, keepdim=True)
        p = z.sub_(m1).exp_()
        back = lambda x: x.reshape(hkv, b1 - b0, g, -1).transpose(0, 1)  # noqa: E731
        l1, a1, m1 = back(p.sum(-1, keepdim=True)), back(torch.matmul(p, V)), back(m1)
        m0 = m[b0:b1]
        top = torch.maximum(m0, m1)
        f0, f1 = (m0 - top).exp(), (m1 - top).exp()
        total[b0:b1] = total[b0:b1] * f0 + l1 * f1
        acc[b0:b1] = acc[b0:b1] * f0 + a1 * f1
        m[b0:b1] = top
    s["out"].copy_((acc / total).reshape(s["out"].shape))
    s["lse"].copy_((m + total.log()).reshape(s["lse"].shape))
    return {"out": s["out"], "lse": s["lse"]}


def _weigh(s):
    c = s["case"]
    B, hkv, g, page, n = c["batch"], c["hkv"], c["hq"] // c["hkv"], c["page"], s["most_new"]
    phys = s["table"][:, : s["widest"]].long().clamp_min(0)
    K = _values(s["k_pages"], s["k_scale"], phys).transpose(1, 2).reshape(B, hkv, -1, D)
    L = K.shape[2]
    i = torch.arange(n, device="cuda")
    row = s["starts"][:, None] + torch.minimum(i, s["rows"][:, None] - 1)                  # padded by the last row
    q = s["q"][row].float().reshape(B, n, hkv, g, D).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * g, D)
    z = torch.matmul(q, K.transpose(-1, -2)).mul_(s["scale"]).reshape(B, hkv, n, g, L)
    z.sub_(s["lse"][row].reshape(B, n, hkv, g).transpose(1, 2)[..., None])
    place = torch.arange(L, device="cuda")
    last = s["length"][:, None] - s["rows"][:, None] + i                                       # a row's own place
    hidden = (place > last[:, :, None]) | (i < s["rows"][:, None]).logical_not()[:, :, None]
    z.masked_fill_(hidden[:, None, :, None], -math.inf)
    add = z.exp_().sum((2, 3))                                                                 # [B, Hkv, L]
    old = (place < (s["length"] - s["rows"])[:, None])[:, None]
    inside = (place < s["length"][:, None])[:, None]
    now = add + s["decay"] * torch.where(old, s["weight_before"][..., :L], 0.0)
    s["weight"][..., :L] = torch.where(inside, now, s["weight"][..., :L])
    ids = (s["n_seen"] - s["length"])[:, None, None] + place
    s["token_id"][..., :L] = torch.where(inside & ~old, ids, s["token_id"][..., :L]).int()
    return {"weight": s["weight"], "token_id": s["token_id"]}


def _select(s):
    c = s["case"]
    L, most = s["longest"], s["moves"].shape[2]
    place = torch.arange(L, device="cuda")
    length, keep = s["length"][:, None, None], torch.minimum(s["keep_len"], s["length"])[:, None, None]
    w = s["weight"][..., :L]
    stay = (place < s["n_first"][:, None, None]) | (s["token_id"][..., :L] >= s["n_seen"][:, None, None] - c["recent"])
    w = torch.where(stay, math.inf, w)
    w = torch.where(place < length, w, -1.0)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(w, dtype=torch.bool).scatter_(2, order, place.expand_as(order) < keep)
    kept |= (length <= keep) & (place < length)
    free, behind = ~kept & (place < keep), kept & (place >= keep)
    count = free.sum(-1)
    for mask, k in ((free, 0), (behind, 1)):
        at = mask.cumsum(-1) - 1
        b, h, t = mask.nonzero(as_tuple=True)
        s["moves"][b, h, at[b, h, t], k] = t.int()
    s["move_count"].copy_(count)
    s["new_len"].copy_(keep[:, 0, 0])
    return {"moves": s["moves"], "count": s["move_count"], "new_len": s["new_len"]}


def _move(s):
    c = s["case"]
    page, hkv = c["page"], c["hkv"]
    i = torch.arange(s["moves"].shape[2], device="cuda")
    b, h, i = (i < s["move_count"][..., None]).nonzero(as_tuple=True)
    to, src = s["moves"][b, h, i, 0].long(), s["moves"][b, h, i, 1].long()
    p_to, p_src = s["table"][b, to // page].long(), s["table"][b, src // page].long()
    touched = torch.zeros(c["batch"], hkv, s["max_pages"], dtype=torch.bool, device="cuda")
    touched[b, h, to // page] = True
    tb, th, tp = touched.nonzero(as_tuple=True)
    phys = s["table"][tb, tp].long()
    for name in "kv":
        pool, scale = s[name + "_pages"], s[name + "_scale"]
        if scale is None:
            pool[p_to, h, to % page] = pool[p_src, h, src % page]
            continue
        slot = torch.zeros_like(touched, dtype=torch.long)
        slot[tb, th, tp] = torch.arange(len(tb), device="cuda")
        slot = slot[b, h, to // page]
        x = pool[p_src, h, src % page].float() * scale[p_src, h][:, None]
        old = scale[phys, th]
        top = torch.zeros_like(old).scatter_reduce_(0, slot, x.abs().amax(-1), "amax")
        now = torch.maximum(old, _scale_of(top, EXPONENTS[c["dtype"]]))
        pool[phys, th] = _codes(pool[phys, th].float() * old[:, None, None], now[:, None, None])
        scale[phys, th] = now
        pool.view(torch.uint8)[p_to, h, to % page] = _codes(x, now[slot][:, None]).view(torch.uint8)
    s["weight"][b, h, to], s["token_id"][b, h, to] = s["weight"][b, h, src], s["token_id"][b, h, src]
    if s["abstract"] is not None:
        shrunk = s["new_len"] < s["length"]
        last = (s["new_len"].long() - 1).clamp_min(0) // page
        sb = shrunk.nonzero().flatten()
        touched[sb, :, last[sb]] = True                        # (fewer tokens than it held)
        tb, th, tp = touched.nonzero(as_tuple=True)
        phys = s["table"][tb, tp].long()
        x = s["k_pages"][phys, th].float()
        if s["k_scale"] is not None:
            x = x * s["k_scale"][phys, th][:, None, None]
        valid = (tp[:, None] * page + torch.arange(page, device="cuda") < s["new_len"][tb][:, None])[..., None]
        s["abstract"][tb, th, tp, 0] = torch.where(valid, x, -math.inf).amax(1).to(s["dtype"])
        s["abstract"][tb, th, tp, 1] = torch.where(valid, x, math.inf).amin(1).to(s["dtype"])
        s["chunk_off"][sb, last[sb] + 1] = s["new_len"][sb]
        s["n_chunks"][sb] = (last[sb] + 1).int()
    return _moved_to(s)


_OWN = {"append": _own_append, "shared": _own_shared, "weigh": _own_weigh, "select": _own_select, "move": _own_move}
_PLAIN = {"append": _append, "shared": _shared, "weigh": _weigh, "select": _select, "move": _move}


# ---- the definition in 64 bits -----------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "shared": _exact_shared, "weigh": _exact_weigh, "select": _exact_select,
            "move": _exact_move}[case["op"]](case, s)


def _grid(x):
    """x to the nearest value of the 8-bit format (3 fraction bits, smallest step 2^-9, at most 448), ties to even."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 4).clamp_min(-9))
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _need(top, exponents):
    need = torch.exp2(torch.ceil(torch.log2(top / 448.0)).clamp(*exponents))
    return torch.where(top > 0, need, torch.zeros_like(need))


def _exact_append(case, s):
    length, n_new = _lengths(case)
    hkv, page, half = case["hkv"], case["page"], case["rot"] // 2
    quantised = case["store"] == "e4m3"
    first = torch.arange(half, device="cuda") * (1 if case["pairs"] == "halves" else 2)
    second = first + (half if case["pairs"] == "halves" else 1)
    rope = s["rope"].double()
    turn = torch.stack([torch.complex(rope[s["position"][int(s["axis"][i])].long(), i], rope[s["position"][int(s["axis"][i])].long(), half + i])
                        for i in range(half)], 1)                                   # [T, half]
    turned = {"v": s["v"].double()}
    for name in "qk":
        x = s[name].double().clone()
        z = torch.complex(x[..., first], x[..., second]) * turn[:, None]
        x[..., first], x[..., second] = z.real, z.imag
        turned[name] = x
    got = {"q": turned["q"], "k": s["k_pages"].double(), "v": s["v_pages"].double()}
    if quantised:
        got.update(k_scale=s["k_scale"].double(), v_scale=s["v_scale"].double())
    abstract, bounds, at = s["abstract"].double(), s["chunk_off"].clone(), 0
    table = s["table"].cpu().numpy()
    for b in range(case["batch"]):
        start, end = int(length[b] - n_new[b]), int(length[b])
        for p in range(start // page, (end - 1) // page + 1):
            phys, lo, hi = int(table[b, p]), max(start, p * page), min(end, (p + 1) * page)
            kept, i = max(0, start - p * page), at + lo - start
            for name in "kv":
                x = turned[name][i: i + hi - lo].transpose(0, 1)                    # [Hkv, new, D]
                if quantised:
                    old = got[name + "_scale"][phys] if kept else torch.zeros(hkv, dtype=torch.float64, device="cuda")
                    now = torch.maximum(old, _need(x.abs().amax((1, 2)), EXPONENTS[case["dtype"]]))
                    safe = torch.where(now > 0, now, torch.ones_like(now))[:, None, None]
                    got[name][phys, :, :kept] = _grid(got[name][phys, :, :kept] * old[:, None, None] / safe)
                    got[name + "_scale"][phys] = now
                    x = _grid(x / safe)
                got[name][phys, :, lo - p * page: hi - p * page] = x
            held = got["k"][phys, :, : hi - p * page] * (got["k_scale"][phys][:, None, None] if quantised else 1.0)
            abstract[b, :, p, 0], abstract[b, :, p, 1] = held.amax(1), held.amin(1)
            bounds[b, p + 1] = hi
        at += end - start
    got.update(abstract=abstract, chunk_off=bounds, n_chunks=torch.from_numpy((-(-length // page)).astype(np.int32)).cuda())
    return got


def _stored(s, b, h, n, name="k"):
    """The first n tokens that sequence b holds for kv head h, in 64 bits."""
    page = s["case"]["page"]
    phys = s["table"][b, : -(-n // page)].long()
    x = s[name + "_pages"][phys, h].double()
    if s[name + "_scale"] is not None:
        x = x * s[name + "_scale"][phys, h].double()[:, None, None]
    return x.flatten(0, 1)[:n]


def _exact_shared(case, s):
    """Sequence by sequence over all of its tokens, softmax shifted by its log-sum."""
    g = case["hq"] // case["hkv"]
    out, lse = torch.empty_like(s["out"], dtype=torch.float64), torch.empty_like(s["lse"], dtype=torch.float64)
    for b, n in enumerate(s["length"].tolist()):
        for h in range(case["hkv"]):
            mine = slice(h * g, (h + 1) * g)
            z = torch.matmul(s["q"][b, mine].double(), _stored(s, b, h, n).t().contiguous()) * s["scale"]
            total = torch.logsumexp(z, -1)
            out[b, mine] = torch.matmul(torch.exp(z - total[:, None]), _stored(s, b, h, n, "v"))
            lse[b, mine] = total
    return {"out": out, "lse": lse}


def _exact_weigh(case, s):
    _, n_new = _lengths(case)
    g = case["hq"] // case["hkv"]
    weight, ids, at = s["weight"].double(), s["token_id"].clone(), 0
    for b, n in enumerate(s["length"].tolist()):
        m = int(n_new[b])
        q, lse = s["q"][at: at + m].double(), s["lse"][at: at + m].double()
        at += m
        for h in range(case["hkv"]):
            K, got = _stored(s, b, h, n), torch.zeros(n, dtype=torch.float64, device="cuda")
            seen = torch.arange(n, device="cuda")[None] <= n - m + torch.arange(m, device="cuda")[:, None]
            for j in range(h * g, (h + 1) * g):
                z = torch.matmul(q[:, j], K.t().contiguous()) * s["scale"] - lse[:, j, None]
                got += torch.where(seen, torch.exp(z), 0.0).sum(0)
            got[: n - m] += s["decay"] * s["weight_before"][b, h, : n - m].double()
            weight[b, h, :n] = got
        ids[b, :, n - m: n] = int(s["n_seen"][b]) - m + torch.arange(m, device="cuda", dtype=torch.int32)
    return {"weight": weight, "token_id": ids}


def _exact_select(case, s):
    moves, count = s["moves"].cpu().numpy().copy(), s["move_count"].cpu().numpy().copy()
    weight, ids = s["weight"].cpu().numpy(), s["token_id"].cpu().numpy()
    new_len = s["new_len"].cpu().numpy().copy()
    for b, n in enumerate(s["length"].tolist()):
        keep = min(n, case["keep"])
        new_len[b] = keep
        for h in range(case["hkv"]):
            t = np.arange(n)
            stay = (t < case["first"]) | (ids[b, h, :n] >= int(s["n_seen"][b]) - case["recent"])
            order = np.lexsort((t, -weight[b, h, :n].astype(np.float64), ~stay))
            if stay.any():                                           # among those that stay anyhow the place alone counts
                k = int(stay.sum())
                order[:k] = np.sort(order[:k])
            kept = np.sort(order[:keep])
            free, behind = np.setdiff1d(t[:keep], kept), kept[kept >= keep]
            count[b, h] = len(free)
            moves[b, h, : len(free), 0], moves[b, h, : len(free), 1] = free, behind
    return {"moves": _cuda(moves), "count": _cuda(count), "new_len": _cuda(new_len)}


def _exact_move(case, s):
    hkv, page = case["hkv"], case["page"]
    quantised = case["store"] == "e4m3"
    got = {"k": s["k_pages"].double(), "v": s["v_pages"].double(), "weight": s["weight"].double(), "token_id": s["token_id"].clone()}
    if quantised:
        got.update(k_scale=s["k_scale"].double(), v_scale=s["v_scale"].double())
    table, moves, count = s["table"].cpu().numpy(), s["moves"].cpu().numpy(), s["move_count"].cpu().numpy()
    length, new_len = s["length"].tolist(), s["new_len"].tolist()
    if s["abstract"] is not None:
        abstract, bounds, chunks = s["abstract"].double(), s["chunk_off"].clone(), s["n_chunks"].clone()
    for b in range(case["batch"]):
        if new_len[b] == length[b]:
            continue
        for h in range(hkv):
            m = moves[b, h, : count[b, h]]
            to, src = _cuda(m[:, 0].astype(np.int64)), _cuda(m[:, 1].astype(np.int64))
            row = table[b]
            p_to, p_src = _cuda(row[m[:, 0] // page].astype(np.int64)), _cuda(row[m[:, 1] // page].astype(np.int64))
            pages = np.unique(m[:, 0] // page)
            phys = _cuda(row[pages].astype(np.int64))
            for name in "kv":
                pool = got[name]
                x = pool[p_src, h, src % page]
                if quantised:
                    scale = got[name + "_scale"]
                    x = x * scale[p_src, h][:, None]
                    which = _cuda(np.searchsorted(pages, m[:, 0] // page))
                    top = torch.zeros(len(pages), dtype=torch.float64, device="cuda").scatter_reduce_(0, which, x.abs().amax(-1), "amax")
                    old = scale[phys, h]
                    now = torch.maximum(old, _need(top, EXPONENTS[case["dtype"]]))
                    safe = torch.where(now > 0, now, torch.ones_like(now))
                    pool[phys, h] = _grid(pool[phys, h] * (old / safe)[:, None, None])
                    scale[phys, h] = now
                    x = _grid(x / safe[which][:, None])
                pool[p_to, h, to % page] = x
            got["weight"][b, h, to], got["token_id"][b, h, to] = got["weight"][b, h, src], got["token_id"][b, h, src]
            if s["abstract"] is None:
                continue
            pages = np.union1d(pages, [(new_len[b] - 1) // page])
            phys = _cuda(row[pages].astype(np.int64))
            x = got["k"][phys, h]
            if quantised:
                x = x * got["k_scale"][phys, h][:, None, None]
            gone = (_cuda(pages)[:, None] * page + torch.arange(page, device="cuda") >= new_len[b])[..., None]
            at = _cuda(pages.astype(np.int64))
            abstract[b, h, at, 0] = x.masked_fill(gone, -math.inf).amax(1)
            abstract[b, h, at, 1] = x.masked_fill(gone, math.inf).amin(1)
        if s["abstract"] is not None:
            bounds[b, (new_len[b] - 1) // page + 1] = new_len[b]
            chunks[b] = (new_len[b] - 1) // page + 1
    if s["abstract"] is not None:
        got.update(abstract=abstract, chunk_off=bounds, n_chunks=chunks)
    return got
