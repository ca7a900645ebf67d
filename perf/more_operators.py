"""The operators of a long cache that is read in part and kept in part, as they are timed: the
bounds of each page's keys, the choice of pages that a cheap score makes for every query row, the
attention over the chosen pages, decode attention that adds up the weight each page gets, and the
eviction of the pages that got the least.

A case is one call (or the few calls that always go together) as a rollout engine makes
it.  Head layouts and page sizes are those of the named workloads of
paper_2607_09207_amd.inputs, lengths follow the same laws (uniform, lognormal).  `run`
computes a case either through the library's entry points (`own`) or in plain torch
operations in 32 bits, and `exact` in 64 bits on its own.

A case fixes the multiset of lengths (`lens_seed`); the seed of a preparation fixes the
order of the sequences, the pages they occupy in the pool, and every value.
"""
import math

import numpy as np
import torch

own = False
PAGE = 16
DEV = "cuda:0"
KV_TORCH = {"bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn, "f32": torch.float32}
KV_BYTES = {"bf16": 2, "fp8": 1, "f32": 4}
KV_NAME = {"bf16": "bf16", "fp8": "fp8_e4m3fn", "f32": "f32"}


def listed():
    gqa = dict(hq=28, hkv=4, d=128, kv="bf16")
    grpo = dict(hq=12, hkv=2, d=128, kv="bf16")
    fp8 = dict(hq=40, hkv=8, d=128, kv="fp8")
    return [
        # The bounds of the page that each of 8 responses has just written to, fp8.  Latency.
        dict(fp8, name="bounds_step_fp8", kind="bounds", batch=8, whole=False, law="uniform", lo=16, hi=1024,
             max_pages=64, lens_seed=4001),
        # The bounds of whole prompts after their prefill, ragged.  Bandwidth is all of it.
        dict(gqa, name="bounds_prompts_bf16", kind="bounds", batch=64, whole=True, law="uniform", lo=500, hi=4096,
             max_pages=256, lens_seed=4002),
        # A step's choice for a few responses of a GRPO batch.  Latency.
        dict(grpo, name="select_step_small_bf16", kind="select", batch=8, rows=1, budget=32, sink=1, recent=2,
             law="uniform", lo=1000, hi=4096, max_pages=256, lens_seed=4003),
        # A step's choice over long contexts: a byte of bounds for every 32 of the cache.
        dict(gqa, name="select_long_bf16", kind="select", batch=64, rows=1, budget=128, sink=1, recent=4,
             law="uniform", lo=8192, hi=32768, max_pages=2048, lens_seed=4004),
        # Four drafted tokens of each sequence, every one with a choice of its own.
        dict(fp8, name="select_verify_fp8", kind="select", batch=16, rows=4, budget=64, sink=1, recent=2,
             law="lognormal", median=8192, sigma=0.7, lo=512, hi=16384, max_pages=1024, lens_seed=4005),
        # A few long responses over their chosen pages: few segments, each cut over many workgroups.
        dict(fp8, name="selected_stragglers_fp8", kind="selected", batch=4, rows=1, budget=48, law="uniform", lo=2048,
             hi=8192, max_pages=512, lens_seed=4006),
        # Long contexts, 2048 tokens of each read.
        dict(gqa, name="selected_long_bf16", kind="selected", batch=64, rows=1, budget=128, law="uniform", lo=1500,
             hi=16384, max_pages=1024, lens_seed=4007),
        # The largest batch: 256 sequences on an fp8 cache, 1024 tokens of each read.
        dict(fp8, name="selected_batch_fp8", kind="selected", batch=256, rows=1, budget=64, law="uniform", lo=700,
             hi=4096, max_pages=256, lens_seed=4008),
        # Weights beside the attention of a small batch.  Latency.
        dict(grpo, name="weighed_step_small_bf16", kind="weighed", batch=8, rows=1, decay=1.0, law="uniform", lo=64,
             hi=1024, max_pages=64, lens_seed=4009),
        # ... of a long-tailed batch, older weights fading: the cache is read once.
        dict(gqa, name="weighed_longtail_bf16", kind="weighed", batch=64, rows=1, decay=0.9375, law="lognormal",
             median=2048, sigma=1.0, lo=32, hi=16384, max_pages=1024, lens_seed=4010),
        # A page of new tokens for each of 8 sequences at their budget, and one page of each dropped.  Latency.
        dict(grpo, name="evict_step_small", kind="evict", batch=8, budget=64, sink=1, recent=4, new_pages=1, group=8,
             shared=16, max_pages=80, slack=64),
        # The same after 64 new tokens of each of 512 sequences that keep 2048.
        dict(grpo, name="evict_large", kind="evict", batch=512, budget=128, sink=1, recent=8, new_pages=4, group=8,
             shared=32, max_pages=256, slack=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call of these ranges."""
    while True:
        kind = rng.choice(["bounds", "select", "select", "selected", "selected", "weighed", "weighed", "evict"])
        hq, hkv = rng.choice([(28, 4), (12, 2), (40, 8), (64, 8), (8, 1), (16, 16)])
        d = rng.choice([64, 128, 128])
        kv = rng.choice(["bf16", "bf16", "fp8"])
        c = dict(kind=kind, hq=hq, hkv=hkv, d=d, kv=kv, layout=rng.choice(["head", "head", "slot"]),
                 lens_seed=rng.randrange(1 << 30), law="uniform")
        sink, recent = rng.choice([(0, 1), (1, 2), (4, 8)])
        if kind == "bounds":
            hi = _log_int(rng, 20, 4096)
            c.update(batch=_log_int(rng, 1, 256), whole=rng.random() < 0.6, lo=rng.choice([1, max(1, hi // 2)]), hi=hi)
        elif kind == "select":
            hi = _log_int(rng, 64, 32768)
            c.update(batch=_log_int(rng, 1, 128), rows=rng.choice([1, 1, 1, 3, 8]), lo=rng.choice([1, max(1, hi // 2)]),
                     hi=hi, budget=rng.choice([16, 37, 64, 128, 300]), sink=sink, recent=recent)
        elif kind == "selected":
            hi = _log_int(rng, 64, 16384)
            c.update(batch=_log_int(rng, 1, 256), rows=rng.choice([1, 1, 1, 1, 4]), lo=rng.choice([1, max(1, hi // 2)]),
                     hi=hi, budget=rng.choice([13, 32, 64, 100, 256]))
        elif kind == "weighed":
            hi = _log_int(rng, 33, 16384)
            c.update(batch=_log_int(rng, 1, 96), rows=rng.choice([1, 1, 1, 2]), lo=rng.choice([1, 16, max(1, hi // 2)]),
                     hi=hi, decay=rng.choice([1.0, 0.9375, 0.0]))
        else:
            group = rng.choice([1, 2, 4, 8])
            budget = _log_int(rng, 16, 256)
            new = rng.choice([1, 1, 2, 5])
            c.update(batch=group * _log_int(rng, 1, 512 // group), budget=budget, new_pages=new, sink=sink, recent=recent,
                     group=group, shared=rng.randint(0, budget // 2), max_pages=budget + new + rng.choice([0, 3, 100]),
                     slack=rng.choice([0, 17, 1000]))
            return c
        c["max_pages"] = int(-(-int(_lengths(c).max()) // PAGE)) + rng.choice([0, 0, 3, 64, 500])
        padded = c["batch"] * c["hi"] * hkv * d * 4.0   # of the plain form, a cache
        w = work(c)
        if w["bytes"] <= 5.4e8 and w["flops"] <= 6e9 and _pool_pages(c) * hkv * PAGE * d * KV_BYTES[kv] <= 1.5e9 and \
                (kind == "select" or padded <= 8e9):
            return c


# ------------------------------------------------------------------ sizes

def _lengths(c):
    """The multiset of sequence lengths (cached tokens), in draw order."""
    rng = np.random.default_rng(c["lens_seed"])
    if c["law"] == "uniform":
        lens = rng.integers(c["lo"], c["hi"] + 1, size=c["batch"])
    else:
        lens = np.clip(np.rint(c["median"] * np.exp(c["sigma"] * rng.standard_normal(c["batch"]))), c["lo"], c["hi"])
    return lens.astype(np.int64)


def _pages_of(lens):
    return -(-np.asarray(lens) // PAGE)


def _pool_pages(c):
    if c["kind"] == "evict":
        return c["batch"] * (c["budget"] - c["shared"] + c["new_pages"]) + c["batch"] // c["group"] * c["shared"] + c["slack"]
    return int(_pages_of(_lengths(c)).sum())


def _rows(lens, rows):
    """Query rows of each sequence (its last tokens), their offsets, and per row its sequence and position."""
    n = np.minimum(lens, rows)
    start = np.concatenate([[0], np.cumsum(n)])
    seq = np.repeat(np.arange(len(lens)), n)
    pos = (lens - n)[seq] + np.arange(int(start[-1])) - start[:-1][seq]
    return n, start, seq, pos


def work(c):
    hq, hkv, d, eb = c["hq"], c["hkv"], c["d"], KV_BYTES[c["kv"]]
    if c["kind"] == "evict":   # the counts, every row's entries and weights, and what moves (about half of a row)
        n = c["batch"] * (c["budget"] + c["new_pages"])
        return {"bytes": 4.0 * _pool_pages(c) + 8.0 * n + 4.0 * n + 16.0 * c["batch"] * c["new_pages"], "flops": 0.0}
    lens = _lengths(c)
    pages = _pages_of(lens)
    if c["kind"] == "bounds":
        tokens = lens if c["whole"] else lens - (pages - 1) * PAGE
        n = float(pages.sum()) if c["whole"] else float(len(lens))
        return {"bytes": float(tokens.sum()) * hkv * d * eb + n * hkv * (2 * d + 4) + 4.0 * n, "flops": 2.0 * float(tokens.sum()) * hkv * d}
    rows, _, seq, pos = _rows(lens, c["rows"])
    if c["kind"] == "select":
        return {"bytes": float(pages.sum()) * hkv * (2 * d + 4) + 2.0 * len(pos) * hq * d + 4.0 * len(pos) * hkv * (c["budget"] + 1),
                "flops": 4.0 * d * hq * float((pos // PAGE + 1).sum())}
    if c["kind"] == "selected":   # the rows of a sequence choose much the same pages
        tokens = np.minimum(pages, c["budget"]) * PAGE
        return {"bytes": float(tokens.sum()) * hkv * d * 2 * eb + 4.0 * len(pos) * hq * d,
                "flops": 4.0 * d * hq * float((np.minimum(pos // PAGE + 1, c["budget"]) * PAGE).sum())}
    return {"bytes": float(lens.sum()) * hkv * d * 2 * eb + 4.0 * len(pos) * hq * d + 8.0 * float(pages.sum()),
            "flops": 4.0 * d * hq * float((pos + 1).sum())}


# ------------------------------------------------------------------ inputs

def _pool(c, gen, npages):
    """One cache (K or V) of N(0, 1) values, [pages][Hkv][16][d], and its fp8 scales (the
    tile's largest magnitude at 448)."""
    shape = (npages, c["hkv"], PAGE, c["d"])
    pool = torch.empty(shape, dtype=KV_TORCH[c["kv"]], device=DEV)
    scale = torch.empty(shape[:2], dtype=torch.float32, device=DEV) if c["kv"] == "fp8" else None
    step = max(1, (1 << 27) // (c["hkv"] * PAGE * c["d"]))
    for i in range(0, npages, step):
        x = torch.randn((min(step, npages - i),) + shape[1:], device=DEV, generator=gen)
        if scale is not None:
            s = x.abs().amax(dim=(2, 3)) / 448.0
            scale[i:i + step] = s
            x = x / s[:, :, None, None]
        pool[i:i + step] = x.to(pool.dtype)
    if c.get("layout") == "slot":   # the same values, stored [pages][16][Hkv][d]
        pool = pool.transpose(1, 2).contiguous().transpose(1, 2)
    return pool, scale


def _bounds_pool(c, gen, npages):
    """Bounds of pages whose keys lie about a centre of their own: [pages][Hkv][2][d] int8, scales."""
    shape = (npages, c["hkv"], c["d"])
    centre = torch.randn(shape, device=DEV, generator=gen)
    width = torch.rand(shape, device=DEV, generator=gen) + 0.5
    x = torch.stack([centre - width, centre + width], dim=2)
    s = x.abs().amax(dim=(2, 3)) / 127.0
    return torch.round(x / s[:, :, None, None]).to(torch.int8), s


def _cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _inputs(c, seed):
    """Tensors of one call, from the case and the seed alone."""
    rng = np.random.default_rng([seed, 19])
    gen = torch.Generator(device=DEV).manual_seed(seed)
    t = {"case": c}
    npages, mp, hq, hkv, d = _pool_pages(c), c["max_pages"], c["hq"], c["hkv"], c["d"]
    ids = rng.permutation(npages).astype(np.int32)
    if c["kind"] == "evict":
        B, n, sh = c["batch"], c["budget"], c["shared"]
        table = np.zeros((B, mp), np.int32)
        groups = B // c["group"]
        table[:, :sh] = np.repeat(ids[:groups * sh].reshape(groups, sh), c["group"], axis=0)
        table[:, sh:n] = ids[groups * sh:groups * sh + B * (n - sh)].reshape(B, n - sh)
        refs = np.zeros(npages, np.int64)
        np.add.at(refs, table[:, :n], 1)
        weights = torch.zeros((B, mp), device=DEV)
        weights[:, :n] = torch.rand((B, n), device=DEV, generator=gen) ** 4 * 50
        t.update(refs=_cuda(refs), block_table=_cuda(table), weights=weights,
                 seq_lens=_cuda((n - 1) * PAGE + rng.integers(1, PAGE + 1, size=B)),
                 add=_cuda(np.full(B, PAGE * c["new_pages"])))
        return t
    lens = rng.permutation(_lengths(c))
    table = np.zeros((len(lens), mp), np.int32)
    table[np.arange(mp)[None, :] < _pages_of(lens)[:, None]] = ids
    t.update(lens=lens, block_table=_cuda(table), seq_lens=_cuda(lens), span=int(_pages_of(lens).max()))
    if c["kind"] == "bounds":
        t["k"], t["ks"] = _pool(c, gen, npages)
        t["first"] = torch.zeros(len(lens), dtype=torch.int32, device=DEV) if c["whole"] else None
        t["bounds"] = torch.zeros((npages, hkv, 2, d), dtype=torch.int8, device=DEV)
        t["bound_scale"] = torch.zeros((npages, hkv), device=DEV)
        return t
    n, start, seq, pos = _rows(lens, c["rows"])
    t.update(rows=n, start=start, seq=torch.from_numpy(seq).to(DEV), pos=torch.from_numpy(pos).to(DEV), most=int(n.max()),
             row_of=torch.from_numpy(np.arange(len(pos)) - start[:-1][seq]).to(DEV),
             q_start=_cuda(start) if c["rows"] > 1 else None)
    t["q"] = (2 * torch.randn((len(pos), hq, d), device=DEV, generator=gen)).to(torch.bfloat16)
    if c["kind"] == "select":
        t["bounds"], t["bound_scale"] = _bounds_pool(c, gen, npages)
        return t
    t["k"], t["ks"] = _pool(c, gen, npages)
    t["v"], t["vs"] = _pool(c, gen, npages)
    if c["kind"] == "weighed":
        t["weights"] = torch.rand((len(lens), mp), device=DEV, generator=gen) * 3
        return t
    # The first page, the row's own, and others at random.
    S, k = t["span"], min(c["budget"], t["span"])
    x = torch.rand((len(pos), hkv, S), device=DEV, generator=gen)
    at, last = torch.arange(S, device=DEV), (t["pos"] // PAGE)[:, None, None]
    x = torch.where((at == 0) | (at == last), 2.0, x).masked_fill(at > last, -1.0)
    chosen = x.topk(k, dim=-1).indices
    chosen = torch.where(chosen <= last, chosen, S).sort(dim=-1).values
    t["pages"] = torch.full((len(pos), hkv, c["budget"]), -1, dtype=torch.int32, device=DEV)
    t["pages"][..., :k] = torch.where(chosen < S, chosen, -1).to(torch.int32)
    t["counts"] = (t["pages"] >= 0).sum(dim=-1).to(torch.int32)
    return t


def prepare(c, seed):
    """The call's inputs; with the library, the layer's handle and its workspaces."""
    s = _inputs(c, seed)
    if own:
        from paper_2607_09207_amd import DecodeAttention
        strides = s["k"].stride()[:3] if "k" in s else None
        layer = DecodeAttention(c["hq"], c["hkv"], c["d"], len(s["seq_lens"]), c["max_pages"], "bf16", KV_NAME[c["kv"]],
                                "bf16", kv_strides=strides)
        s["layer"] = layer
        if c["kind"] == "evict":
            layer.page_workspace(len(s["refs"]), DEV)
        elif c["kind"] == "weighed":
            layer.weighed_workspace(len(s["q"]), DEV)
        else:
            layer.workspace(DEV)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _own(s)
    return {"bounds": _bounds, "select": _select, "selected": _selected, "weighed": _weighed, "evict": _evict}[s["case"]["kind"]](s)


def _own(s):
    c, layer = s["case"], s["layer"]
    if c["kind"] == "bounds":
        layer.page_bounds(s["k"], s["block_table"], s["seq_lens"], s["bounds"], s["bound_scale"], first=s["first"],
                          k_scale=s["ks"])
        return {"bounds": s["bounds"], "scale": s["bound_scale"]}
    if c["kind"] == "select":
        pages, counts = layer.select_pages(s["q"], s["bounds"], s["bound_scale"], s["block_table"], s["seq_lens"],
                                           c["budget"], sink=c["sink"], recent=c["recent"], q_start=s["q_start"])
        return {"pages": pages, "counts": counts}
    if c["kind"] == "selected":
        return layer.selected(s["q"], s["k"], s["v"], s["block_table"], s["seq_lens"], s["pages"], s["counts"],
                              q_start=s["q_start"], k_scale=s["ks"], v_scale=s["vs"])
    if c["kind"] == "weighed":
        out = layer.weighed(s["q"], s["k"], s["v"], s["block_table"], s["seq_lens"], s["weights"], decay=c["decay"],
                            q_start=s["q_start"], k_scale=s["ks"], v_scale=s["vs"])
        return {"out": out, "weights": s["weights"]}
    state = (s["refs"], s["block_table"], s["seq_lens"])
    layer.page_grow(*state, s["add"])
    dropped = layer.page_evict(*state, s["weights"], c["budget"], sink=c["sink"], recent=c["recent"])
    return {"refs": s["refs"], "table": s["block_table"], "lens": s["seq_lens"], "weights": s["weights"], "dropped": dropped}


# ------------------------------------------------------------------ the plain forms

def _bytes(x):
    return x.view(torch.uint8) if x.element_size() == 1 else x


def _page_values(s, cache, scale, page):
    """Pages [...] of a cache in 32 bits: [...][Hkv][16][d]."""
    x = _bytes(cache)[page]
    x = x.view(cache.dtype).float() if cache.element_size() == 1 else x.float()
    return x if scale is None else x * scale[page][..., None, None]


def _over_127(x):
    """The quotient, rounded once (a number as the divisor would be a product with its reciprocal)."""
    return x / torch.full_like(x, 127)


def _bounds(s):
    lens = s["seq_lens"].long()
    last = (lens - 1) // PAGE
    first = last if s["first"] is None else s["first"].long() // PAGE
    width = 1 if s["first"] is None else s["span"]
    j = (first[:, None] + torch.arange(width, device=DEV)).minimum(last[:, None])   # the last page again: the same values
    page = s["block_table"].long().gather(1, j)
    x = _page_values(s, s["k"], s["ks"], page)
    there = ((j * PAGE)[:, :, None] + torch.arange(PAGE, device=DEV) < lens[:, None, None])[:, :, None, :, None]
    hi, lo = x.masked_fill(~there, -math.inf).amax(dim=3), x.masked_fill(~there, math.inf).amin(dim=3)
    scale = _over_127(torch.maximum(hi.abs(), lo.abs()).amax(dim=-1))
    by = torch.where(scale > 0, scale, 1.0)[..., None]
    s["bounds"][page] = torch.stack([(lo / by).floor().clamp_min(-127), (hi / by).ceil().clamp_max(127)], dim=-2).to(torch.int8)
    s["bound_scale"][page] = scale
    return {"bounds": s["bounds"], "scale": s["bound_scale"]}


def _best(key, kept, seen, budget):
    """The places of `kept` and of the largest keys among `seen`, `budget` together, ascending
    (the number of places where there are fewer); ties go to the lowest."""
    S = key.shape[-1]
    key = torch.where(kept, math.inf, key).masked_fill(~seen, -math.inf)
    at = key.sort(dim=-1, descending=True, stable=True).indices[..., :budget]
    return torch.where(seen.expand_as(key).gather(-1, at), at, S).sort(dim=-1).values


def _select(s):
    c = s["case"]
    B, n, S, hkv, d = len(s["seq_lens"]), s["most"], s["span"], c["hkv"], c["d"]
    G = c["hq"] // hkv
    q = s["q"].float()
    sq = _over_127(q.abs().amax(dim=-1, keepdim=True))
    q8 = torch.where(sq > 0, (q / torch.where(sq > 0, sq, 1.0)).round(), 0.0)
    rows = torch.zeros((B, n, c["hq"], 2 * d + 1), device=DEV)
    rows[s["seq"], s["row_of"]] = torch.cat([q8.clamp_max(0), q8.clamp_min(0), sq], dim=-1)
    rows = rows.view(B, n, hkv, G, 2 * d + 1).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * G, 2 * d + 1)
    page = s["block_table"][:, :S].long()
    b = s["bounds"][page].float().view(B, S, hkv, 2 * d).permute(0, 2, 3, 1).contiguous()
    u = torch.matmul(rows[..., :-1].contiguous(), b) * rows[..., -1:]        # whole numbers below 2^24, by the row's scale
    score = u.view(B, hkv, n, G, S).amax(dim=3) * s["bound_scale"][page].permute(0, 2, 1)[:, :, None]
    score = score.permute(0, 2, 1, 3)[s["seq"], s["row_of"]]                 # [rows][Hkv][S]
    last, at = (s["pos"] // PAGE)[:, None, None], torch.arange(S, device=DEV)
    seen = at <= last
    kept = seen & ((at < c["sink"]) | (at > last - c["recent"]))
    best = _best(score, kept, seen, c["budget"])
    pages = torch.full((len(q), hkv, c["budget"]), -1, dtype=torch.int32, device=DEV)
    pages[..., :best.shape[-1]] = torch.where(best < S, best, -1).to(torch.int32)
    return {"pages": pages, "counts": (pages >= 0).sum(dim=-1).to(torch.int32)}


def _selected(s):
    c = s["case"]
    n, hkv, d, k = len(s["q"]), c["hkv"], c["d"], c["budget"]
    G = c["hq"] // hkv
    j = s["pages"].long().clamp_min(0)                                       # [rows][Hkv][budget]
    page = s["block_table"].long()[s["seq"][:, None, None], j]
    head = torch.arange(hkv, device=DEV)[None, :, None]

    def values(cache, scale):
        x = _bytes(cache)[page, head]
        x = x.view(cache.dtype).float() if cache.element_size() == 1 else x.float()
        return (x if scale is None else x * scale[page, head][..., None, None]).reshape(n, hkv, k * PAGE, d)

    q = s["q"].float().view(n, hkv, G, d)
    x = torch.matmul(q, values(s["k"], s["ks"]).transpose(-1, -2).contiguous()) / math.sqrt(d)
    token = (j * PAGE)[..., None] + torch.arange(PAGE, device=DEV)
    seen = (s["pages"] >= 0)[..., None] & (token <= s["pos"][:, None, None, None])
    p = torch.exp(x.masked_fill(~seen.view(n, hkv, 1, k * PAGE), -math.inf) - x.amax(dim=-1, keepdim=True))
    o = torch.matmul(p / p.sum(dim=-1, keepdim=True), values(s["v"], s["vs"]))
    return o.reshape(n, c["hq"], d).to(torch.bfloat16)


def _weighed(s):
    c = s["case"]
    B, n, S, hkv, d = len(s["seq_lens"]), s["most"], s["span"], c["hkv"], c["d"]
    G = c["hq"] // hkv
    page = s["block_table"][:, :S].long()

    def values(cache, scale):   # [B][Hkv][tokens][d]
        return _page_values(s, cache, scale, page).permute(0, 2, 1, 3, 4).reshape(B, hkv, S * PAGE, d)

    q = torch.zeros((B, n, c["hq"], d), device=DEV)
    q[s["seq"], s["row_of"]] = s["q"].float()
    pos = torch.full((B, n), -1, dtype=torch.int64, device=DEV).index_put_((s["seq"], s["row_of"]), s["pos"])
    q = q.view(B, n, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * G, d)
    x = torch.matmul(q, values(s["k"], s["ks"]).transpose(-1, -2).contiguous()) / math.sqrt(d)
    seen = (torch.arange(S * PAGE, device=DEV) <= pos[:, :, None])[:, None, :, None]
    x = x.view(B, hkv, n, G, S * PAGE).masked_fill(~seen, -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - torch.where(top.isfinite(), top, 0.0))
    p = p / p.sum(dim=-1, keepdim=True).clamp_min(1e-38)
    o = torch.matmul(p.view(B, hkv, n * G, S * PAGE), values(s["v"], s["vs"]))
    o = o.view(B, hkv, n, G, d).permute(0, 2, 1, 3, 4).reshape(B, n, c["hq"], d)
    got = p.view(B, -1, S, PAGE).sum(dim=(1, 3))
    w = s["weights"][:, :S]
    there = torch.arange(S, device=DEV) * PAGE < s["seq_lens"].long()[:, None]
    w.copy_(torch.where(there, w * c["decay"] + got, w))
    return {"out": o[s["seq"], s["row_of"]].to(torch.bfloat16), "weights": s["weights"]}


def _count_pages(lens):
    return (lens.long() + PAGE - 1) // PAGE


def _evict(s):
    c = s["case"]
    table, lens, w, k = s["block_table"], s["seq_lens"], s["weights"], c["budget"]
    at = torch.arange(table.shape[1], device=DEV)[None, :]
    # Room for the new tokens: the lowest free pages, in sequence order.
    have, want = _count_pages(lens), _count_pages(lens + s["add"])
    need, free = want - have, s["refs"] == 0
    ids = torch.argsort((~free).to(torch.int32), stable=True).to(torch.int32)
    s["refs"].add_((free & (free.cumsum(0) <= need.sum())).to(torch.int32))
    index = ((need.cumsum(0) - need)[:, None] + at - have[:, None]).clamp(0, len(ids) - 1)
    table.copy_(torch.where((at >= have[:, None]) & (at < want[:, None]), ids[index], table))
    lens.add_(s["add"])
    # The pages that stay.
    seen = at < want[:, None]
    best = _best(w, seen & ((at < c["sink"]) | (at >= (want - c["recent"])[:, None])), seen, k)
    S, left = table.shape[1], torch.minimum(want, torch.full_like(want, k))
    stays = torch.zeros((len(lens), S + 1), dtype=torch.bool, device=DEV).scatter_(1, best, True)[:, :S]
    s["refs"].index_add_(0, table.flatten().long(), (seen & ~stays).flatten().to(torch.int32), alpha=-1)
    take = best.clamp_max(S - 1)
    front = at[:, :best.shape[1]] < left[:, None]
    rest = torch.where(seen, 0.0, w)
    new_table, new_w = table.gather(1, take), w.gather(1, take)
    table[:, :best.shape[1]] = torch.where(front, new_table, table[:, :best.shape[1]])
    w.copy_(rest)
    w[:, :best.shape[1]] = torch.where(front, new_w, rest[:, :best.shape[1]])
    dropped = (want - left).to(torch.int32)
    lens.sub_(PAGE * dropped)
    return {"refs": s["refs"], "table": table, "lens": lens, "weights": w, "dropped": dropped}


# ------------------------------------------------------------------ what the results should be

def exact(c, seed):
    if c["kind"] in ("select", "evict"):
        return None   # whole numbers, and weights as they are
    t = _inputs(c, seed)
    hkv, d, G = c["hkv"], c["d"], c["hq"] // c["hkv"]
    table, lens = t["block_table"].cpu().numpy(), t["lens"]

    def sequence(b, cache, scale, L):   # [Hkv][L][d] in 64 bits
        pages = torch.from_numpy(table[b, :-(-L // PAGE)].astype(np.int64)).to(DEV)
        x = _bytes(cache)[pages]
        x = x.view(cache.dtype).double() if x.element_size() == 1 else x.double()
        if scale is not None:
            x = x * scale[pages].double()[:, :, None, None]
        return x.transpose(0, 1).reshape(hkv, -1, d)[:, :L]

    if c["kind"] == "bounds":
        scale = t["bound_scale"].double()
        for b, L in enumerate(lens):
            x = sequence(b, t["k"], t["ks"], int(L)).abs().amax(dim=-1)          # [Hkv][L]
            x = torch.nn.functional.pad(x, (0, -int(L) % PAGE)).view(hkv, -1, PAGE).amax(dim=-1) / 127.0
            j = slice(0 if c["whole"] else x.shape[1] - 1, x.shape[1])
            scale[torch.from_numpy(table[b, j].astype(np.int64)).to(DEV)] = x[:, j].t()
        return {"bounds": None, "scale": scale}
    out = torch.zeros(t["q"].shape, dtype=torch.float64, device=DEV)
    weights = t["weights"].double() if c["kind"] == "weighed" else None
    for b, L in enumerate(lens):
        L, r = int(L), slice(int(t["start"][b]), int(t["start"][b + 1]))
        n = r.stop - r.start
        k, v = sequence(b, t["k"], t["ks"], L), sequence(b, t["v"], t["vs"], L)
        q = t["q"][r].double().view(n, hkv, G, d).transpose(0, 1).reshape(hkv, n * G, d)
        x = (torch.matmul(q, k.transpose(1, 2).contiguous()) * d ** -0.5).view(hkv, n, G, L)
        seen = torch.arange(L, device=DEV) <= t["pos"][r, None]                   # [n][L]
        if c["kind"] == "selected":
            listed_ = torch.zeros((n, hkv, -(-L // PAGE) + 1), dtype=torch.bool, device=DEV)
            listed_.scatter_(2, torch.where(t["pages"][r] >= 0, t["pages"][r], listed_.shape[2] - 1).long(), True)
            seen = seen[:, None] & listed_[..., :-1].repeat_interleave(PAGE, dim=-1)[..., :L]
            seen = seen.transpose(0, 1)                                           # [Hkv][n][L]
        else:
            seen = seen[None]
        p = torch.softmax(x.masked_fill(~seen[:, :, None], -math.inf), dim=-1)
        out[r] = torch.matmul(p.view(hkv, n * G, L), v).view(hkv, n, G, d).transpose(0, 1).reshape(n, hkv * G, d)
        if weights is not None:
            m = -(-L // PAGE)
            got = torch.nn.functional.pad(p.sum(dim=(0, 1, 2)), (0, m * PAGE - L)).view(m, PAGE).sum(dim=1)
            weights[b, :m] = weights[b, :m] * c["decay"] + got
    return out if weights is None else {"out": out, "weights": weights}
