"""The operators over a paged cache, as cases that can be timed.

A case is a dict of plain values.  `op` names the operator:

  append   new queries, keys and values (slices of one projection's output): positions rotated, keys and
           values stored into the pages, the pages' abstract rows and the chunk boundaries kept up to date
  decode   attention of one token per sequence over its pages, or over the pages a selection kept
  prefill  causal attention of each sequence's new tokens over all it has cached, themselves included

`dtype` is the model's type, `store` what the pages hold: "model" or "e4m3" (8 bits with a scale for each page
and kv head).  `ctx` is the longest sequence's length after the call (with `ragged` the others are shorter),
`new` the most new tokens of a sequence (1: one each), `keep` the most pages a selection keeps (0: no selection),
`rot` the rotated channels, `pairs` which of them rotate together ("halves" or "neighbours").

Pages lie scattered over the pool.  Keys and values are Gaussian with a gain of their own for each page, a few
key channels carry outliers.
"""
import math

import numpy as np
import torch

own = False

D = 128
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
SCRATCH = 64 << 20
# exponents of a page's scale: scale * code stays a number of the model's type
EXPONENTS = {"f16": (-15, 7), "bf16": (-100, 118)}


def listed():
    def case(name, op, dtype, store, batch, hq, hkv, ctx, new=1, page=64, keep=0, rot=128, pairs="halves", ragged=True):
        return {"name": name, "op": op, "dtype": dtype, "store": store, "batch": batch, "hq": hq, "hkv": hkv, "ctx": ctx,
                "new": new, "page": page, "keep": keep, "rot": rot, "pairs": pairs, "ragged": ragged}
    return [
        # single-user decoding: one token of one layer, where only latency counts
        case("append 1 token bf16", "append", "bf16", "model", 1, 32, 8, 8191, ragged=False),
        # a decode step of many users, into the 8-bit pages
        case("append 96 tokens e4m3", "append", "bf16", "e4m3", 96, 32, 8, 5000, page=32),
        # prompts of several users, some with a history, multi-head attention in fp16
        case("append prompts f16 mha", "append", "f16", "model", 5, 32, 32, 6001, new=4001, pairs="neighbours"),
        # one long prompt into the 8-bit pages
        case("append prompt e4m3 16K", "append", "bf16", "e4m3", 1, 32, 8, 16384, new=16384, page=128),
        # the smallest decode of the benchmark's configurations: fp32, one sequence of 4096
        case("decode f32 4K", "decode", "f32", "model", 1, 8, 8, 4096, page=32, ragged=False),
        # single-user decoding at 128K, the pages that a selection kept
        case("decode bf16 128K kept pages", "decode", "bf16", "model", 1, 32, 8, 131072, keep=64, ragged=False),
        # serving many users at lengths of their own, eight query heads per group
        case("decode e4m3 g8 9K x40", "decode", "bf16", "e4m3", 40, 64, 8, 9001, page=16),
        # sixteen users of up to 128K in 8 bits, every page
        case("decode e4m3 128K x16", "decode", "f16", "e4m3", 16, 32, 8, 131072),
        # a prompt from its first token
        case("prefill bf16 8K", "prefill", "bf16", "model", 1, 32, 8, 8192, new=8192, ragged=False),
        # prompts of several users behind histories, from the 8-bit pages, odd lengths
        case("prefill e4m3 behind history x4", "prefill", "f16", "e4m3", 4, 32, 8, 6143, new=2047, page=32),
        # a few tokens checked at once behind a long context
        case("prefill bf16 9 tokens at 64K", "prefill", "bf16", "model", 2, 32, 8, 65000, new=9),
        # fp32, multi-head, short
        case("prefill f32 1K", "prefill", "f32", "model", 2, 8, 8, 1000, new=777, page=16),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "prefill", "prefill"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    store = "model" if dtype == "f32" else rng.choice(["model", "e4m3"])
    hkv = rng.choice([1, 2, 4, 8, 8, 16, 32])
    group = rng.choice([1, 2, 4, 4, 8])
    group = min(group, 64 // hkv)
    page = rng.choice([16, 32, 64, 64, 128, 256])
    new, keep = 1, 0
    if op == "append":
        if rng.random() < 0.5:
            batch, ctx = _log_uniform(rng, 1, 128), _log_uniform(rng, 64, 16384)
        else:
            batch = _log_uniform(rng, 1, 8)
            new = _log_uniform(rng, 2, 16384 // batch)
            ctx = new + rng.choice([0, _log_uniform(rng, 1, 4096)])
        while batch * (ctx + page) * hkv > 1 << 22:
            ctx = ctx // 2 + 1
            new = min(new, ctx)
    elif op == "decode":
        most = (1 << 24) if store == "e4m3" else (1 << 23) if dtype != "f32" else 1 << 21      # (kv head, token) pairs
        ctx = _log_uniform(rng, 1, 131072)
        batch = _log_uniform(rng, 1, max(1, min(128, most // (ctx * hkv))))
        if rng.random() < 0.4:
            keep = _log_uniform(rng, 1, max(2, -(-ctx // page) // 3))
    else:
        logits, cached = ((1 << 31, 1 << 23) if dtype != "f32" else (1 << 27, 1 << 20))          # at most
        new = _log_uniform(rng, 2, 8192 if dtype != "f32" else 2048)
        ctx = new + rng.choice([0, _log_uniform(rng, 1, 65536)])
        while new * ctx * hkv * group > logits or ctx * hkv > cached:
            new, ctx = (new // 2, ctx) if new > ctx // 2 else (new, max(new, ctx // 2))
        batch = _log_uniform(rng, 1, max(1, min(16, logits // (new * ctx * hkv * group), cached // (ctx * hkv))))
    return {"op": op, "dtype": dtype, "store": store, "batch": batch, "hq": hkv * group, "hkv": hkv, "ctx": ctx, "new": new,
            "page": page, "keep": keep, "rot": rng.choice([128, 128, 64, 0]), "pairs": rng.choice(["halves", "neighbours"]),
            "ragged": rng.random() < 0.8}


# ---- the case's lengths (of the case alone, so that work() knows them) ---------------------------------

def _lengths(case):
    """Length after the call and new tokens of every sequence."""
    rng = np.random.default_rng(case["ctx"] * 131 + case["batch"])
    B, ctx, new = case["batch"], case["ctx"], case["new"]
    n_new = np.full(B, new, np.int64)
    if case["ragged"] and new > 1:
        n_new[1:] = rng.integers(1, new + 1, B - 1)
    length = np.full(B, ctx, np.int64)
    if case["ragged"]:
        length[1:] = n_new[1:] + (rng.random(B - 1) * (ctx - n_new[1:] + 1)).astype(np.int64)
    return length, n_new


def _kept(case):
    """Pages that a selection keeps, per (sequence, kv head)."""
    length, _ = _lengths(case)
    pages = -(-length // case["page"])
    rng = np.random.default_rng(case["keep"])
    most = np.minimum(pages, case["keep"])[:, None]
    least = np.minimum(most, np.maximum(1, case["keep"] // 2))
    return rng.integers(least, most + 1, (case["batch"], case["hkv"]))


def work(case):
    length, n_new = _lengths(case)
    e = BYTES[case["dtype"]]
    es = 1 if case["store"] == "e4m3" else e
    hq, hkv, page = case["hq"], case["hkv"], case["page"]
    if case["op"] == "append":
        t = int(n_new.sum())
        first, last = (length - n_new) // page, (length - 1) // page
        begun = int(((length - n_new) % page > 0).sum())
        touched = int((last - first + 1).sum())
        rows = t * (2 * hq + 2 * hkv) * D * e + t * 2 * hkv * D * es + t * case["rot"] * 4
        return {"bytes": rows + (touched + begun) * hkv * 2 * D * e, "flops": 3 * t * (hq + hkv) * case["rot"]}
    if case["op"] == "decode":
        if case["keep"]:
            tokens = int(_kept(case).sum()) * page
        else:
            tokens = int(length.sum()) * hkv
        return {"bytes": tokens * 2 * D * es + case["batch"] * hq * D * (e + 4), "flops": 4 * tokens * (hq // hkv) * D}
    pairs = int((n_new * (length - n_new) + n_new * (n_new + 1) // 2).sum())
    return {"bytes": int(length.sum()) * hkv * 2 * D * es + int(n_new.sum()) * hq * D * 2 * e, "flops": 4 * hq * D * pairs}


# ---- inputs ----------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    dt, B, hq, hkv, page = DTYPES[case["dtype"]], case["batch"], case["hq"], case["hkv"], case["page"]
    length, n_new = _lengths(case)
    pages = -(-length // page)
    max_pages = int(pages.max()) + 1                      # room to grow
    n_pages = int(pages.sum()) + 3
    table = np.full((B, max_pages), -1, np.int32)
    order = rng.permutation(n_pages).astype(np.int32)
    at = 0
    for b in range(B):
        table[b, : pages[b]] = order[at: at + pages[b]]
        at += pages[b]
    new_off = np.zeros(B + 1, np.int32)
    new_off[1:] = np.cumsum(n_new)
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    s = {"case": case, "dtype": dt, "length": cuda(length.astype(np.int32)), "table": cuda(table), "n_pages": n_pages,
         "max_pages": max_pages, "new_off": cuda(new_off) if case["new"] > 1 else None, "scale": 1.0 / math.sqrt(D),
         "scratch": torch.zeros(SCRATCH, dtype=torch.uint8, device="cuda")}

    # the pool: Gaussian, each page with a gain of its own, outlier channels in the keys
    for name, outliers in (("k", True), ("v", False)):
        gain = 2.0 ** torch.randint(-1, 2, (n_pages, hkv, 1, 1), generator=gen, device="cuda").float()
        if case["store"] == "e4m3":
            pool = torch.empty(n_pages, hkv, page, D, dtype=torch.float8_e4m3fn, device="cuda")
            scale = gain.reshape(n_pages, hkv) * (2.0 ** -4 if outliers else 2.0 ** -6)
        else:
            pool = torch.empty(n_pages, hkv, page, D, dtype=dt, device="cuda")
            scale = None
        step = max(1, (1 << 26) // (hkv * page * D))
        for i in range(0, n_pages, step):
            x = torch.randn(pool[i: i + step].shape, generator=gen, device="cuda") * gain[i: i + step]
            if outliers:
                x[..., :4] *= 4.0
            if scale is not None:
                x = (x / scale[i: i + step, :, None, None]).clamp(-448.0, 448.0)
            pool[i: i + step] = x.to(pool.dtype)
        s[name + "_pages"], s[name + "_scale"] = pool, scale
    t = int(n_new.sum())
    if case["op"] == "append":
        # one projection's output: queries, keys and values of a token beside each other
        qkv = torch.randn(t, hq + 2 * hkv, D, generator=gen, device="cuda")
        qkv[:, hq: hq + hkv, :4] *= 4.0
        qkv = qkv.to(dt)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq: hq + hkv], qkv[:, hq + hkv:]
        s["q_out"] = torch.empty(t, hq, D, dtype=dt, device="cuda")
        cap = max_pages * page
        s["rope"] = None
        if case["rot"]:
            half = case["rot"] // 2
            angle = (torch.arange(cap, dtype=torch.float64, device="cuda")[:, None]
                     * 500000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half))
            s["rope"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
        s["status"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        s["chunk_off"] = (torch.arange(max_pages + 1, dtype=torch.int32, device="cuda") * page).repeat(B, 1)
        s["n_chunks"] = cuda(((length - n_new) // page).astype(np.int32))
        # what the scheduler of a serving program knows on the host: every new token's sequence and position,
        # and the pages that the call touches
        seq = np.repeat(np.arange(B), n_new)
        pos = np.arange(t) - np.repeat(new_off[:-1], n_new) + np.repeat(length - n_new, n_new)
        first = (length - n_new) // page
        count = (length - 1) // page - first + 1
        base = np.zeros(B, np.int64)
        base[1:] = np.cumsum(count)[:-1]
        touched_seq = np.repeat(np.arange(B), count)
        touched_page = np.arange(int(count.sum())) - np.repeat(base, count) + np.repeat(first, count)
        s["seq"], s["pos"] = cuda(seq), cuda(pos)
        s["slot"] = cuda(base[seq] + pos // page - first[seq])            # which touched page a token goes to
        s["touched_seq"], s["touched_page"] = cuda(touched_seq), cuda(touched_page)
        s["start"] = cuda(length - n_new)
        # abstracts of the pages as they were before the call (of a page with no token yet: anything)
        s["abstract"] = torch.zeros(B, hkv, max_pages, 2, D, dtype=dt, device="cuda")
        ts, tp = s["touched_seq"], s["touched_page"]
        phys = s["table"][ts, tp].long()
        old = _values(s["k_pages"], s["k_scale"], phys)                       # [U, Hkv, page, D]
        held = (tp[:, None] * page + torch.arange(page, device="cuda")) < s["start"][ts][:, None]
        held = held[:, None, :, None]
        s["abstract"][ts, :, tp, 0] = torch.where(held, old, -math.inf).amax(2).to(dt)
        s["abstract"][ts, :, tp, 1] = torch.where(held, old, math.inf).amin(2).to(dt)
        return s
    s["q"] = torch.randn(t, hq, D, generator=gen, device="cuda").to(dt)
    if case["op"] == "decode":
        s["out"] = torch.empty(B, hq, D, dtype=torch.float32, device="cuda")
        s["lse"] = torch.empty(B, hq, dtype=torch.float32, device="cuda")
        s["sel_idx"] = s["sel_count"] = None
        if case["keep"]:
            kept = _kept(case)
            idx = np.full((B, hkv, case["keep"]), -1, np.int32)
            for b in range(B):
                for h in range(hkv):
                    idx[b, h, : kept[b, h]] = np.sort(rng.choice(pages[b], kept[b, h], replace=False))
            s["sel_idx"], s["sel_count"] = cuda(idx), cuda(kept.astype(np.int32))
        s["widest"] = int(pages.max())
    else:
        s["out"] = torch.empty(t, hq, D, dtype=dt, device="cuda")
        s["lse"] = torch.empty(t, hq, dtype=torch.float32, device="cuda")
        s["widest"], s["most_new"] = int(pages.max()), int(n_new.max())
        s["starts"] = cuda(new_off[:-1].astype(np.int64))
        s["n_new"] = cuda(n_new)
        s["row_of"] = cuda(np.arange(t) - np.repeat(new_off[:-1], n_new) + np.repeat(np.arange(B), n_new) * int(n_new.max()))
    return s


def _values(pool, scale, phys):
    """What the pages `phys` hold, in 32 bits."""
    x = pool[phys].float()
    return x if scale is None else x * scale[phys][..., None, None]


# ---- one pass ----------------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return _own_append(s) if op == "append" else _own_decode(s) if op == "decode" else _own_prefill(s)
    return _append(s) if op == "append" else _decode(s) if op == "decode" else _prefill(s)


def _own_pages(s):
    import paper_2506_20187_amd as L
    if "pages" not in s:
        c = s["case"]
        s["pages"] = L.make_pages(c["batch"], c["hq"], c["hkv"], D, s["n_pages"], c["page"], s["max_pages"], s["dtype"],
                                  L.E4M3 if c["store"] == "e4m3" else s["dtype"], rot_dim=c["rot"] if c["op"] == "append" else 0,
                                  interleaved=c["pairs"] == "neighbours",
                                  rope_len=s["max_pages"] * c["page"] if c["op"] == "append" and c["rot"] else 0)
    return L, s["pages"]


def _own_append(s):
    L, pages = _own_pages(s)
    L.kv_page_append(pages, s["q"], s["k"], s["v"], s["new_off"], s["length"], s["table"], s["rope"], s["q_out"], s["k_pages"],
                     s["v_pages"], s["k_scale"], s["v_scale"], s["abstract"], s["chunk_off"], s["n_chunks"], s["status"])
    return _appended(s)


def _appended(s):
    got = {"q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"], "abstract": s["abstract"], "chunk_off": s["chunk_off"],
           "n_chunks": s["n_chunks"]}
    if s["k_scale"] is not None:
        got.update(k_scale=s["k_scale"], v_scale=s["v_scale"])
    return got


def _own_decode(s):
    L, pages = _own_pages(s)
    L.page_attention_decode(pages, s["q"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["table"], s["length"],
                            s["sel_idx"], s["sel_count"], s["scale"], s["out"], s["lse"], s["scratch"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_prefill(s):
    L, pages = _own_pages(s)
    L.page_attention_prefill(pages, s["q"], s["new_off"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["table"],
                             s["length"], s["scale"], s["out"], s["lse"], s["scratch"])
    return {"out": s["out"], "lse": s["lse"]}


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
    page, rot = c["page"], c["rot"]
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    if rot:
        row = s["rope"][s["pos"]]
        cos, sin = row[:, None, : rot // 2], row[:, None, rot // 2:]
        q, k = _rotated(q, cos, sin, rot, c["pairs"]), _rotated(k, cos, sin, rot, c["pairs"])
    s["q_out"].copy_(q)
    ts, tp = s["touched_seq"], s["touched_page"]
    phys = s["table"][ts, tp].long()                                       # [U]
    at = s["table"][s["seq"], s["pos"] // page].long()                     # [T] page of every new token
    slot = s["pos"] % page
    inside = tp[:, None] * page + torch.arange(page, device="cuda")        # [U, page] positions
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
    ends = torch.minimum((tp + 1) * page, s["length"][ts])
    s["chunk_off"][ts, tp + 1] = ends.int()
    s["n_chunks"].copy_((s["length"] + page - 1) // page)
    return _appended(s)


def _decode(s):
    c = s["case"]
    B, hkv, g, page = c["batch"], c["hkv"], c["hq"] // c["hkv"], c["page"]
    inside = torch.arange(page, device="cuda")
    if s["sel_idx"] is None:
        phys = s["table"][:, : s["widest"]].long().clamp_min(0)                             # [B, P]
        pos = torch.arange(s["widest"] * page, device="cuda").expand(B, 1, 1, -1)
        valid = pos < s["length"][:, None, None, None]
        K, V = (_values(s[n + "_pages"], s[n + "_scale"], phys).transpose(1, 2).reshape(B, hkv, -1, D) for n in "kv")
    else:
        idx = s["sel_idx"].long()                                                           # [B, Hkv, k]
        listed_ = torch.arange(idx.shape[2], device="cuda") < s["sel_count"][..., None]
        phys = torch.gather(s["table"][:, None].expand(-1, hkv, -1).long(), 2, idx.clamp_min(0)).clamp_min(0)
        pos = idx[..., None] * page + inside
        valid = (listed_[..., None] & (pos < s["length"][:, None, None, None])).reshape(B, hkv, 1, -1)
        head = torch.arange(hkv, device="cuda")[None, :, None]
        K, V = (s[n + "_pages"][phys, head].float() for n in "kv")                          # [B, Hkv, k, page, D]
        if s["k_scale"] is not None:
            K, V = K * s["k_scale"][phys, head][..., None, None], V * s["v_scale"][phys, head][..., None, None]
        K, V = K.reshape(B, hkv, -1, D), V.reshape(B, hkv, -1, D)
    return _attend(s, s["q"].float().reshape(B, hkv, g, D), K, V, valid)


def _attend(s, q, K, V, valid):
    z = torch.matmul(q, K.transpose(-1, -2)).mul_(s["scale"])
    z.masked_fill_(~valid, -math.inf)
    m = z.amax(-1, keepdim=True)
    p = z.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, V).div_(total)
    s["out"].copy_(o.reshape(s["out"].shape))
    s["lse"].copy_((m + total.log()).reshape(s["lse"].shape))
    return {"out": s["out"], "lse": s["lse"]}


def _prefill(s):
    c = s["case"]
    B, hkv, g, page, n = c["batch"], c["hkv"], c["hq"] // c["hkv"], c["page"], s["most_new"]
    phys = s["table"][:, : s["widest"]].long().clamp_min(0)
    K, V = (_values(s[x + "_pages"], s[x + "_scale"], phys).transpose(1, 2).reshape(B, hkv, -1, D) for x in "kv")
    i = torch.arange(n, device="cuda")
    rows = (s["starts"][:, None] + torch.minimum(i, s["n_new"][:, None] - 1)).reshape(-1)      # padded by the last row
    q = s["q"][rows].float().reshape(B, n, hkv, g, D).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * g, D)
    z = torch.matmul(q, K.transpose(-1, -2)).mul_(s["scale"]).reshape(B, hkv, n, g, -1)
    last = (s["length"] - s["n_new"])[:, None] + torch.minimum(i, s["n_new"][:, None] - 1)     # [B, n] its own position
    hidden = torch.arange(s["widest"] * page, device="cuda") > last[:, :, None]
    z.masked_fill_(hidden[:, None, :, None], -math.inf)
    m = z.amax(-1, keepdim=True)
    p = z.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(B, hkv, n * g, -1), V).reshape(B, hkv, n, g, D).div_(total)
    lse = (m + total.log()).squeeze(-1)
    pick = lambda x: x.transpose(1, 2).flatten(0, 1)[s["row_of"]].flatten(1, 2)  # noqa: E731
    s["out"].copy_(pick(o))
    s["lse"].copy_(pick(lse))
    return {"out": s["out"], "lse": s["lse"]}


# ---- the definition in 64 bits -----------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    length, n_new = _lengths(case)
    return _exact_append(case, s, length, n_new) if case["op"] == "append" else _exact_attention(case, s, length, n_new)


def _grid(x):
    """x to the nearest value of the 8-bit format (3 fraction bits, smallest step 2^-9, at most 448), ties to even."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 4).clamp_min(-9))
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _exact_append(case, s, length, n_new):
    hkv, page, rot = case["hkv"], case["page"], case["rot"]
    half = rot // 2
    lo, hi = EXPONENTS.get(case["dtype"], (0, 0))
    turned = {}
    for name in "qk":
        x = s[name].double()
        if rot:
            first = torch.arange(half, device="cuda") * (1 if case["pairs"] == "halves" else 2)
            second = first + (half if case["pairs"] == "halves" else 1)
            row = s["rope"].double()[s["pos"]]
            z = torch.complex(x[..., first], x[..., second]) * torch.complex(row[:, None, :half], row[:, None, half:])
            x = x.clone()
            x[..., first], x[..., second] = z.real, z.imag
        turned[name] = x
    turned["v"] = s["v"].double()
    got = {"q": turned["q"]}
    abstract = s["abstract"].double()
    bounds, at = s["chunk_off"].clone(), 0
    quantised = case["store"] == "e4m3"
    for name in "kv":
        got[name] = s[name + "_pages"].double()
        if quantised:
            got[name + "_scale"] = s[name + "_scale"].double()
    table = s["table"].cpu().numpy()
    for b in range(case["batch"]):
        start, end = int(length[b] - n_new[b]), int(length[b])
        for p in range(start // page, (end - 1) // page + 1):
            phys, lo_pos, hi_pos = int(table[b, p]), max(start, p * page), min(end, (p + 1) * page)
            kept = max(0, start - p * page)
            i = at + lo_pos - start
            for name in "kv":
                x = turned[name][i: i + hi_pos - lo_pos].transpose(0, 1)          # [Hkv, new, D]
                a, z = lo_pos - p * page, hi_pos - p * page
                if not quantised:
                    got[name][phys, :, a:z] = x
                    continue
                old = got[name + "_scale"][phys] if kept else torch.zeros(hkv, dtype=torch.float64, device="cuda")
                top = x.abs().amax((1, 2))
                need = torch.exp2(torch.ceil(torch.log2(top / 448.0)).clamp(lo, hi))
                now = torch.maximum(old, torch.where(top > 0, need, torch.zeros_like(need)))
                safe = torch.where(now > 0, now, torch.ones_like(now))[:, None, None]
                if kept:
                    got[name][phys, :, :kept] = _grid(got[name][phys, :, :kept] * old[:, None, None] / safe)
                got[name][phys, :, a:z] = _grid(x / safe)
                got[name + "_scale"][phys] = now
            held = got["k"][phys, :, : hi_pos - p * page] * (got["k_scale"][phys][:, None, None] if quantised else 1.0)
            abstract[b, :, p, 0], abstract[b, :, p, 1] = held.amax(1), held.amin(1)
            bounds[b, p + 1] = hi_pos
        at += end - start
    got.update(abstract=abstract, chunk_off=bounds, n_chunks=torch.from_numpy((-(-length // page)).astype(np.int32)).cuda())
    return got


def _exact_attention(case, s, length, n_new):
    """Sequence by sequence, softmax shifted by its log-sum."""
    hkv, hq, page = case["hkv"], case["hq"], case["page"]
    g = hq // hkv
    out, lse, at = [], [], 0
    for b in range(case["batch"]):
        n, m = int(length[b]), int(n_new[b])
        phys = s["table"][b, : -(-n // page)].long()
        q = s["q"][at: at + m].double()                                           # [m, Hq, D]
        at += m
        heads, sums = [], []
        for h in range(hkv):
            K, V = s["k_pages"][phys, h].double(), s["v_pages"][phys, h].double()   # [P, page, D]
            if s["k_scale"] is not None:
                K, V = K * s["k_scale"][phys, h].double()[:, None, None], V * s["v_scale"][phys, h].double()[:, None, None]
            K, V, pos = K.flatten(0, 1)[:n], V.flatten(0, 1)[:n], torch.arange(n, device="cuda")
            if case["op"] == "decode" and s["sel_idx"] is not None:
                ids = s["sel_idx"][b, h, : int(s["sel_count"][b, h])].long()
                pos = (ids[:, None] * page + torch.arange(page, device="cuda")).flatten()
                pos = pos[pos < n]
                K, V = K[pos], V[pos]
            z = torch.matmul(q[:, h * g: (h + 1) * g].transpose(0, 1).reshape(g * m, D), K.t().contiguous()) * s["scale"]
            z = z.reshape(g, m, -1)
            if case["op"] == "prefill":
                z = torch.where(pos[None, :] <= n - m + torch.arange(m, device="cuda")[:, None], z, -math.inf)
            total = torch.logsumexp(z, -1)
            heads.append(torch.matmul(torch.exp(z - total[..., None]).reshape(g * m, -1), V).reshape(g, m, D))
            sums.append(total)
        out.append(torch.cat(heads, 0).transpose(0, 1))
        lse.append(torch.cat(sums, 0).transpose(0, 1))
    return {"out": torch.cat(out, 0), "lse": torch.cat(lse, 0)}
