"""The operators around the decode attention that are timed: rotary positions, the pages of
the cache, and attention whose scores are capped, biased by distance or masked to an interval.

A case is one call (or the few calls that always go together) as a rollout engine makes
it.  Head layouts, lengths and page sizes are those of the named workloads of
paper_2607_09207_amd.inputs, lengths follow the same laws (uniform, lognormal).  `run`
computes a case either through the library's entry points (`own`) or in plain torch
operations in 32 bits (angles in 64), and `exact` in 64 bits on its own.

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
    tail = dict(law="lognormal", median=2048, sigma=1.0, lo=32, hi=16384, max_pages=1024)
    return [
        # The gradient of the rotation over a training batch of packed responses: q and k of
        # every token, a slice of the projection's output.  Bandwidth is all of it.
        dict(name="rotate_grad_bf16", kind="rotate", rows=32768, heads=32, extra=4, d=128, rot=128, pairs="half",
             dtype="bf16", inverse=True, amplitude=1.0, base=1e6, span=32768),
        # The smallest step: the new token of 8 responses into an fp8 cache.  Latency.
        dict(fp8, name="append_step_small_fp8", kind="append", batch=8, rows=1, rot=128, pairs="half", amplitude=1.0,
             base=1e4, law="uniform", lo=16, hi=1024, max_pages=64, lens_seed=3001),
        # The new token of the largest decode batch, 512 sequences.
        dict(name="append_step_large_bf16", kind="append", hq=64, hkv=8, d=128, kv="bf16", batch=512, rows=1, rot=128,
             pairs="half", amplitude=1.0, base=5e5, law="uniform", lo=16, hi=2048, max_pages=2048, lens_seed=3002),
        # Prompts into the cache, ragged, positions scaled for long contexts, half of the head rotated.
        dict(fp8, name="append_prompts_fp8", kind="append", batch=48, rows=1024, rot=64, pairs="interleaved",
             amplitude=1.1386, base=1e4, law="uniform", lo=100, hi=1024, max_pages=128, lens_seed=3003),
        # Requests that ended leave their rows, new prompts take them: 8 of 64 rows.  Latency.
        dict(grpo, name="pages_admit_small", kind="admit", batch=64, group=8, prompt=512, ended=8, law="lognormal",
             median=512, sigma=1.0, lo=1, hi=4096, max_pages=512, slack=1024, lens_seed=3004),
        # Two training iterations meet: the last responses are released and every prompt is
        # forked for its 8 responses, the partial last page of each copied in all 28 layers.
        dict(grpo, name="pages_fork_grpo", kind="fork", layers=28, prompts=32, group=8, law="uniform", lo=200, hi=1000,
             max_pages=256, lens_seed=3005),
        # Half of the responses have ended and the memory goes back: the live pages of 16
        # layers move to the front of the pool.  The largest copy.
        dict(grpo, name="pages_compact_half", kind="compact", layers=16, batch=128, group=8, prompt=512, law="lognormal",
             median=512, sigma=1.0, lo=1, hi=8192, max_pages=640, slack=64, lens_seed=3006),
        # A few long responses, scores capped.
        dict(gqa, name="scored_stragglers_cap_bf16", kind="scored", batch=4, rows=1, cap=30.0, slopes=False, window=0,
             docs=0, prefix=False, law="uniform", lo=8192, hi=16384, max_pages=1024, lens_seed=3007),
        # Long-tailed decode with a bias by distance in place of rotary positions.
        dict(gqa, name="scored_longtail_bias_bf16", kind="scored", batch=64, rows=1, cap=0.0, slopes=True, window=0,
             docs=0, prefix=False, lens_seed=3008, **tail),
        # A layer with a sliding window and a cap on an fp8 cache.
        dict(fp8, name="scored_window_cap_fp8", kind="scored", batch=128, rows=1, cap=50.0, slopes=False, window=4096,
             docs=0, prefix=False, law="lognormal", median=4096, sigma=1.0, lo=64, hi=16384, max_pages=2048,
             lens_seed=3009),
        # Prefill of packed documents, scores capped.
        dict(gqa, name="scored_documents_cap_bf16", kind="scored", batch=16, rows=1024, cap=50.0, slopes=False, window=0,
             docs=900, prefix=False, law="uniform", lo=1024, hi=4096, max_pages=256, lens_seed=3010),
        # Prefill with a prefix that every row sees, and the bias, on an fp8 cache: the largest product.
        dict(fp8, name="scored_prefix_bias_fp8", kind="scored", batch=8, rows=512, cap=0.0, slopes=True, window=0,
             docs=0, prefix=True, law="uniform", lo=300, hi=3000, max_pages=256, lens_seed=3011),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call of these ranges."""
    while True:
        kind = rng.choice(["rotate", "append", "append", "admit", "fork", "compact", "scored", "scored", "scored",
                           "prefill", "prefill"])
        hq, hkv = rng.choice([(28, 4), (12, 2), (40, 8), (64, 8), (8, 1), (16, 16)])
        d = rng.choice([64, 128, 128])
        kv = rng.choice(["bf16", "bf16", "fp8"])
        pairs = rng.choice(["half", "half", "interleaved"])
        amplitude = rng.choice([1.0, 1.0, 1.25])
        base = rng.choice([1e4, 5e5, 1e6])
        seed = rng.randrange(1 << 30)
        if kind == "rotate":
            d = rng.choice([64, 80, 128, 256])
            c = dict(kind=kind, rows=_log_int(rng, 1, 32768), heads=rng.choice([1, 8, 16, 32, 40]),
                     extra=rng.choice([0, 2, 8]), d=d, rot=rng.choice([16, d // 32 * 16, d]), pairs=pairs,
                     dtype=rng.choice(["bf16", "bf16", "f32"]), inverse=rng.random() < 0.5, amplitude=amplitude,
                     base=base, span=_log_int(rng, 1024, 1 << 20))
        else:
            layout = rng.choice(["head", "head", "slot"])
            c = dict(kind=kind, hq=hq, hkv=hkv, d=d, kv=kv, layout=layout, lens_seed=seed)
            if kind == "append":
                rows = rng.choice([1, 1, rng.randint(2, 16), 300, 1024])
                hi = max(rows, _log_int(rng, 33, 1500))
                c.update(batch=_log_int(rng, 1, 512 if rows <= 16 else 48), rows=rows, rot=rng.choice([d, d, d // 2, 16]),
                         pairs=pairs, amplitude=amplitude, base=base, law="uniform", lo=1, hi=hi)
            elif kind in ("admit", "compact"):
                group = rng.choice([1, 2, 4, 8])
                batch = group * _log_int(rng, 1, 128 // group)
                c.update(batch=batch, group=group, prompt=PAGE * _log_int(rng, 1, 64), law="lognormal",
                         median=_log_int(rng, 32, 512), sigma=1.0, lo=1, hi=_log_int(rng, 1024, 8192),
                         slack=rng.choice([0, 17, 1000]))
                if kind == "admit":
                    c["ended"] = rng.randint(1, max(1, batch // 3))
                else:
                    c["layers"] = _log_int(rng, 1, 16)
            elif kind == "fork":
                c.update(layers=_log_int(rng, 1, 28), prompts=_log_int(rng, 1, 32), group=rng.choice([2, 3, 4, 8, 16]),
                         law="uniform", lo=1, hi=_log_int(rng, 20, 2000))
            else:
                pre = kind == "prefill"
                hi = _log_int(rng, 33, 2048 if pre else 16384)
                c.update(kind="scored", batch=_log_int(rng, 1, 12 if pre else 96),
                         rows=rng.choice([64, 200, 512, 777]) if pre else rng.choice([1, 1, 1, 2, 4]),
                         cap=rng.choice([0.0, 20.0, 50.0]), slopes=rng.random() < 0.5,
                         window=rng.choice([0, 0, _log_int(rng, 1, 4096)]), docs=rng.choice([0, 0, _log_int(rng, 20, 2000)]),
                         prefix=rng.random() < 0.3, law="uniform", lo=rng.choice([1, 16, max(1, hi // 2)]), hi=hi)
            lens = _lengths(c)
            c["max_pages"] = int(-(-max(lens) // PAGE)) + rng.choice([0, 0, 3, 64, 500])
            if kind in ("fork", "compact") and _pool_pages(c) * c["layers"] * hkv * d * KV_BYTES[kv] > 1.0e8:
                continue
        w = work(c)
        if w["bytes"] <= 9e8 and w["flops"] <= 9e10:
            return c


# ------------------------------------------------------------------ sizes

def _lengths(c):
    """The multiset of sequence lengths (cached tokens, prompt included), in draw order."""
    rng = np.random.default_rng(c["lens_seed"])
    n = c["prompts"] if c["kind"] == "fork" else c["batch"]
    if c["law"] == "uniform":
        lens = rng.integers(c["lo"], c["hi"] + 1, size=n)
    else:
        lens = np.clip(np.rint(c["median"] * np.exp(c["sigma"] * rng.standard_normal(n))), c["lo"], c["hi"])
    return lens.astype(np.int64) + c.get("prompt", 0)


def _pages_of(lens):
    return -(-np.asarray(lens) // PAGE)


def _pool_pages(c):
    lens = _lengths(c)
    if c["kind"] == "fork":   # a child's partial last page is its own
        return int(_pages_of(lens).sum() + (lens % PAGE > 0).sum() * c["group"]) + 40
    if "prompt" in c:
        pp = c["prompt"] // PAGE
        return int((_pages_of(lens) - pp).sum()) + c["batch"] // c["group"] * pp + c["slack"] + \
            (c.get("ended", 0) * pp)
    return int(_pages_of(lens).sum())


def _intervals(c, lens, rng):
    """Query rows of each sequence, and per row its position, first and last visible key
    (and what gives them: the rows' first keys, the sequences' prefixes)."""
    rows = np.minimum(lens, c["rows"])
    start = np.concatenate([[0], np.cumsum(rows)])
    seq = np.repeat(np.arange(len(lens)), rows)
    pos = (lens - rows)[seq] + np.arange(int(start[-1])) - start[:-1][seq]
    key_start = prefix = None
    lo, hi = np.zeros_like(pos), pos + 1
    if c["docs"]:
        off = rng.integers(0, c["docs"], size=len(lens))[seq]
        key_start = np.maximum((pos + off) // c["docs"] * c["docs"] - off, 0)
        lo = key_start
    if c["window"]:
        lo = np.maximum(lo, pos - c["window"] + 1)
    if c["prefix"]:
        prefix = rng.integers(0, lens + 1)
        hi = np.maximum(hi, prefix[seq])
    return rows, start, seq, pos, np.maximum(lo, 0), hi, key_start, prefix


def work(c):
    if c["kind"] == "rotate":
        n = c["rows"] * c["heads"]
        e = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": 2.0 * n * c["d"] * e + 4.0 * c["rows"], "flops": 3.0 * n * c["rot"]}
    lens, eb = _lengths(c), KV_BYTES[c["kv"]]
    if c["kind"] == "append":
        n = float(np.minimum(lens, c["rows"]).sum())
        return {"bytes": n * c["d"] * (4 * c["hq"] + c["hkv"] * (4 + 2 * eb)) + 4.0 * len(lens),
                "flops": 3.0 * n * (c["hq"] + c["hkv"]) * c["rot"]}
    if c["kind"] == "scored":
        rows, start, seq, pos, lo, hi, _, _ = _intervals(c, lens, np.random.default_rng(c["lens_seed"] + 1))
        first = np.minimum.reduceat(lo, start[:-1])
        last = np.maximum.reduceat(hi, start[:-1])
        n = float((last - first).sum())
        return {"bytes": n * c["hkv"] * c["d"] * 2 * eb + 4.0 * len(pos) * c["hq"] * c["d"],
                "flops": 4.0 * c["d"] * c["hq"] * float((hi - lo).sum())}
    npages = _pool_pages(c)
    page = 2.0 * c["hkv"] * PAGE * (c["d"] * eb + (4.0 / PAGE if c["kv"] == "fp8" else 0))
    used = _pages_of(lens)
    if c["kind"] == "admit":
        n = float(used.mean()) * c["ended"]
        return {"bytes": 4.0 * npages + 12.0 * n + 16.0 * c["batch"], "flops": 0.0}
    if c["kind"] == "fork":   # children: entries read and written twice, the tails copied in every layer
        n, tails = float((lens // PAGE).sum()) * c["group"], float((lens % PAGE > 0).sum()) * c["group"]
        return {"bytes": 4.0 * npages + 20.0 * n + 2.0 * page * tails * c["layers"], "flops": 0.0}
    # Compaction: half of the rows are left, spread evenly over the pool; half of their pages move.
    n = float(used.sum()) / 2
    return {"bytes": 4.0 * npages + 8.0 * n + page * (npages - c["slack"]) / 2 * c["layers"], "flops": 0.0}


# ------------------------------------------------------------------ inputs

def _pool(c, gen, npages, layers=None):
    """One cache (K or V) of N(0, 1) values, [pages][Hkv][16][d] (every layer's one behind the
    other where `layers`), and its fp8 scales (the tile's largest magnitude at 448)."""
    shape = ((layers,) if layers else ()) + (npages, c["hkv"], PAGE, c["d"])
    pool = torch.empty(shape, dtype=KV_TORCH[c["kv"]], device=DEV)
    scale = torch.empty(shape[:-2], dtype=torch.float32, device=DEV) if c["kv"] == "fp8" else None
    flat, fscale = pool.view(-1, c["hkv"], PAGE, c["d"]), None if scale is None else scale.view(-1, c["hkv"])
    step = max(1, (1 << 27) // (c["hkv"] * PAGE * c["d"]))
    for i in range(0, len(flat), step):
        x = torch.randn((min(step, len(flat) - i),) + flat.shape[1:], device=DEV, generator=gen)
        if scale is not None:
            s = x.abs().amax(dim=(2, 3)) / 448.0
            fscale[i:i + step] = s
            x = x / s[:, :, None, None]
        flat[i:i + step] = x.to(pool.dtype)
    if c.get("layout") == "slot":   # the same values, stored [pages][16][Hkv][d]
        pool = pool.transpose(-3, -2).contiguous().transpose(-3, -2)
    return pool, scale


def frequencies(rot, base):
    """Radians a position of each pair, in 64 bits."""
    return base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)


def _table(lens, mp, pages, first=0):
    """Rows of page ids: sequence b's pages from `first` on, taken from `pages` in order."""
    table = np.zeros((len(lens), mp), np.int32)
    at = 0
    for b, n in enumerate(_pages_of(lens) - first):
        table[b, first:first + n] = pages[at:at + n]
        at += int(n)
    return table, at


def _cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _inputs(c, seed):
    """Tensors of one call, from the case and the seed alone."""
    rng = np.random.default_rng([seed, 17])
    gen = torch.Generator(device=DEV).manual_seed(seed)
    t = {"case": c}
    if c["kind"] == "rotate":
        dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        fused = torch.randn((c["rows"], c["heads"] + c["extra"], c["d"]), dtype=dt, device=DEV, generator=gen)
        t["x"] = fused[:, :c["heads"]]
        t["positions"] = _cuda(rng.integers(0, c["span"], size=c["rows"]))
        t["freqs"] = frequencies(c["rot"], c["base"])
        return t
    lens = _lengths(c)
    npages, mp, hq, hkv, d = _pool_pages(c), c["max_pages"], c["hq"], c["hkv"], c["d"]
    if c["kind"] in ("append", "scored"):
        order = rng.permutation(len(lens))
        rows, start, seq, pos, lo, hi, key_start, prefix = _intervals(
            dict(dict(docs=0, window=0, prefix=False), **c), lens, np.random.default_rng(c["lens_seed"] + 1))
        # The sequences in the seed's order, their rows with them.
        by_row = np.concatenate([np.arange(start[b], start[b + 1]) for b in order])
        lens, rows = lens[order], rows[order]
        seq, pos, lo, hi = np.repeat(np.arange(len(lens)), rows), pos[by_row], lo[by_row], hi[by_row]
        start = np.concatenate([[0], np.cumsum(rows)])
        total = int(start[-1])
        table, _ = _table(lens, mp, rng.permutation(npages))
        t.update(lens=lens, rows=rows, seq=torch.from_numpy(seq).to(DEV), pos=torch.from_numpy(pos).to(DEV),
                 row_of=torch.from_numpy(np.arange(total) - start[:-1][seq]).to(DEV), block_table=_cuda(table),
                 seq_lens=_cuda(lens), q_start=_cuda(start) if c["rows"] > 1 else None)
        t["k"], t["ks"] = _pool(c, gen, npages)
        t["v"], t["vs"] = _pool(c, gen, npages)
        # The projection's output: q, k and v of a token behind one another.
        qkv = torch.randn((total, hq + 2 * hkv, d), dtype=torch.bfloat16, device=DEV, generator=gen)
        if c["kind"] == "append":
            t["q"], t["k_new"], t["v_new"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
            t["freqs"] = frequencies(c["rot"], c["base"])
            return t
        t["q"] = (qkv[:, :hq] * 2).contiguous()
        t["lo"], t["hi"] = torch.from_numpy(lo).to(DEV), torch.from_numpy(hi).to(DEV)
        t["key_start"] = None if key_start is None else _cuda(key_start[by_row])
        t["prefix"] = None if prefix is None else _cuda(prefix[order])
        t["slopes"] = (torch.exp2(-8.0 * torch.arange(1, hq + 1, device=DEV, dtype=torch.float64) / hq).float()
                       if c["slopes"] else None)
        # What the plain form gathers: every sequence's pages from the first visible key's on.
        first = np.minimum.reduceat(lo, start[:-1]) // PAGE * PAGE
        t["first"] = torch.from_numpy(first).to(DEV)
        t["span"] = int((np.maximum.reduceat(hi, start[:-1]) - first).max())
        return t
    perm = rng.permutation(npages).astype(np.int32)
    if c["kind"] == "fork":
        P, g = c["prompts"], c["group"]
        table, at = _table(lens, mp, perm)
        full, tail = lens // PAGE, lens % PAGE > 0
        kids = np.repeat(np.arange(P), g)
        child = table[kids].copy()
        for i, p in enumerate(kids):   # the last forks are still there
            child[i, full[p]:] = 0
            if tail[p]:
                child[i, full[p]] = perm[at]
                at += 1
        all_lens = np.concatenate([lens, lens[kids]])
        table = np.concatenate([table, child])
        t["parents"], t["children"] = _cuda(kids), _cuda(P + rng.permutation(P * g))
        t["k"], t["ks"] = _pool(c, gen, npages, c["layers"])
        t["v"], t["vs"] = _pool(c, gen, npages, c["layers"])
    else:
        lens = np.concatenate([rng.permutation(x) for x in lens.reshape(-1, c["group"])])
        pp, g = c["prompt"] // PAGE, c["group"]
        table, at = _table(lens, mp, perm, pp)
        table[:, :pp] = np.repeat(perm[at:at + len(lens) // g * pp].reshape(-1, pp), g, axis=0)
        all_lens = lens
        gone = rng.permutation(len(lens))
        if c["kind"] == "admit":
            t["rows"] = _cuda(gone[: c["ended"]])
            add = np.zeros(len(lens), np.int64)
            add[gone[: c["ended"]]] = lens[gone[: c["ended"]]]
            t["add"] = _cuda(add)
        else:
            all_lens = lens.copy()
            all_lens[gone[: len(lens) // 2]] = 0
            t["k"], t["ks"] = _pool(c, gen, npages, c["layers"])
            t["v"], t["vs"] = _pool(c, gen, npages, c["layers"])
    refs = np.zeros(npages, np.int64)
    used = np.arange(mp)[None, :] < _pages_of(all_lens)[:, None]
    np.add.at(refs, table[used], 1)
    t.update(block_table=_cuda(table), seq_lens=_cuda(all_lens), refs=_cuda(refs))
    if c["kind"] == "compact":
        t["table0"], t["refs0"] = t["block_table"].clone(), t["refs"].clone()
    return t


def prepare(c, seed):
    """The call's inputs; with the library, the layer's handle, its workspaces and its caches."""
    s = _inputs(c, seed)
    if own and c["kind"] != "rotate":
        from paper_2607_09207_amd import DecodeAttention
        strides = s["k"].stride()[-4:-1] if "k" in s else None
        layer = DecodeAttention(c["hq"], c["hkv"], c["d"], len(s["seq_lens"]), c["max_pages"], "bf16", KV_NAME[c["kv"]],
                                "bf16", kv_strides=strides)
        s["layer"] = layer
        if c["kind"] in ("append", "scored"):
            layer.workspace(s["q"].device)
        else:
            layer.page_workspace(len(s["refs"]), s["refs"].device)
            if "layers" in c:
                s["caches"] = layer.caches([(s["k"][i], s["v"][i]) if s["ks"] is None else
                                            (s["k"][i], s["v"][i], s["ks"][i], s["vs"][i]) for i in range(c["layers"])])
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _own(s)
    return {"rotate": _rotate_call, "append": _append_call, "admit": _admit, "fork": _fork, "compact": _compact,
            "scored": _scored}[s["case"]["kind"]](s)


def _own(s):
    c = s["case"]
    if c["kind"] == "rotate":
        from paper_2607_09207_amd import rotate
        return rotate(s["x"], s["positions"], s["freqs"], interleaved=c["pairs"] == "interleaved",
                      amplitude=c["amplitude"], inverse=c["inverse"])
    layer = s["layer"]
    if c["kind"] == "append":
        q = layer.append_rotary(s["q"], s["k_new"], s["v_new"], s["k"], s["v"], s["block_table"], s["seq_lens"],
                                s["freqs"], q_start=s["q_start"], interleaved=c["pairs"] == "interleaved",
                                amplitude=c["amplitude"], k_scale=s["ks"], v_scale=s["vs"])
        return {"q": q, "k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"]}
    if c["kind"] == "scored":
        return layer.scored(s["q"], s["k"], s["v"], s["block_table"], s["seq_lens"], q_start=s["q_start"],
                            max_q_len=c["rows"], score_cap=c["cap"], slopes=s["slopes"], window=c["window"],
                            key_start=s["key_start"], prefix_lens=s["prefix"], k_scale=s["ks"], v_scale=s["vs"])
    state = (s["refs"], s["block_table"], s["seq_lens"])
    live = None
    if c["kind"] == "admit":
        layer.page_release(*state, s["rows"])
        layer.page_grow(*state, s["add"])
    elif c["kind"] == "fork":
        layer.page_release(*state, s["children"])
        layer.page_fork(*state, s["parents"], s["children"], s["caches"])
    else:   # the same holes again for every pass
        s["block_table"].copy_(s["table0"])
        s["refs"].copy_(s["refs0"])
        live = layer.page_compact(*state, s["caches"])
    return _page_answer(s, live)


def _page_answer(s, live=None):
    return {"refs": s["refs"], "table": s["block_table"], "lens": s["seq_lens"], "live": live, "k": s.get("k"),
            "v": s.get("v"), "ks": s.get("ks"), "vs": s.get("vs")}


# ------------------------------------------------------------------ the plain forms

def _turn(x, positions, freqs, pairs, amplitude, inverse):
    """Rows [n][heads][d] turned by their positions, in 32 bits (the angles in 64)."""
    x = x.float()
    rot = 2 * len(freqs)
    angle = positions.double()[:, None] * freqs[None, :]
    cos, sin = (angle.cos() * amplitude).float()[:, None], (angle.sin() * amplitude).float()[:, None]
    if inverse:
        sin = -sin
    if pairs == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _rotate_call(s):
    c = s["case"]
    return _turn(s["x"], s["positions"], s["freqs"], c["pairs"], c["amplitude"], c["inverse"]).to(s["x"].dtype)


def _bytes(x):
    return x.view(torch.uint8) if x.element_size() == 1 else x


def _write_rows(s, cache, scale, x):
    """New rows (32 bits) into their pages, in place.  fp8: every page's scale grows to cover
    them (its earlier rows are encoded again), a page's first row starts it."""
    pos = s["pos"]
    page = s["block_table"].long()[s["seq"], pos // PAGE]
    slot = pos % PAGE
    if scale is None:
        cache[page, :, slot] = x.to(cache.dtype)
        return
    pages, page = torch.unique(page, return_inverse=True)
    tile, scales = _bytes(cache)[pages].view(cache.dtype).float(), scale[pages]
    amax = torch.zeros_like(scales).index_reduce_(0, page, x.abs().amax(dim=2), "amax")
    first = torch.full((len(pages),), PAGE, dtype=torch.int64, device=DEV).index_reduce_(0, page, slot, "amin")
    old = torch.where((scales > 0) & scales.isfinite() & (first > 0)[:, None], scales, 0.0)
    grow = (first == 0)[:, None] | (amax > 448.0 * old)
    new = torch.where(grow, amax / 448.0, old)
    ratio = torch.where(grow & (old > 0), old / new, 0.0)
    before = torch.arange(PAGE, device=DEV)[None, :] < first[:, None]
    again = (grow[:, :, None] & before[:, None, :])[..., None]
    tile = torch.where(again, (tile * ratio[:, :, None, None]).clamp(-448, 448), tile)
    tile[page, :, slot] = torch.where(new[page][:, :, None] > 0, x / new[page][:, :, None], 0.0).clamp(-448, 448)
    _bytes(cache)[pages] = _bytes(tile.to(cache.dtype))
    scale[pages] = new


def _append_call(s):
    c = s["case"]
    turn = lambda x: _turn(x, s["pos"], s["freqs"], c["pairs"], c["amplitude"], False)   # noqa: E731
    _write_rows(s, s["k"], s["ks"], turn(s["k_new"]))
    _write_rows(s, s["v"], s["vs"], s["v_new"].float())
    return {"q": turn(s["q"]).to(torch.bfloat16), "k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"]}


def _count_pages(lens):
    return (lens.long() + PAGE - 1) // PAGE


def _release(s, rows):
    """The pages of `rows` lose one reference each; the rows are empty then."""
    rows = rows.long()
    used = torch.arange(s["block_table"].shape[1], device=DEV)[None, :] < _count_pages(s["seq_lens"][rows])[:, None]
    s["refs"].index_add_(0, s["block_table"][rows].flatten(), used.flatten().to(torch.int32), alpha=-1)
    s["seq_lens"][rows] = 0


def _take(s, need):
    """Page ids for the requests' `need`, the lowest free ones in order: [requests][most] with
    the request's pages first (beyond them, any)."""
    free = s["refs"] == 0
    ids = torch.argsort((~free).to(torch.int32), stable=True).to(torch.int32)
    s["refs"].add_((free & (free.cumsum(0) <= need.sum())).to(torch.int32))
    return ids, need.cumsum(0) - need


def _admit(s):
    _release(s, s["rows"])
    lens, table = s["seq_lens"].long(), s["block_table"]
    have, want = _count_pages(lens), _count_pages(lens + s["add"])
    ids, at = _take(s, want - have)
    j = torch.arange(table.shape[1], device=DEV)[None, :]
    index = (at[:, None] + j - have[:, None]).clamp(0, len(ids) - 1)
    table.copy_(torch.where((j >= have[:, None]) & (j < want[:, None]), ids[index], table))
    s["seq_lens"].add_(s["add"])
    return _page_answer(s)


def _copy_pages(s, src, dst):
    for name in ("k", "v"):
        x = _bytes(s[name])
        x[:, dst] = x[:, src]
    if s["ks"] is not None:
        s["ks"][:, dst] = s["ks"][:, src]
        s["vs"][:, dst] = s["vs"][:, src]


def _fork(s):
    _release(s, s["children"])
    parents, children = s["parents"].long(), s["children"].long()
    lens, table = s["seq_lens"].long()[parents], s["block_table"]
    full, tail = lens // PAGE, (lens % PAGE > 0).long()
    j = torch.arange(table.shape[1], device=DEV)[None, :]
    shared = j < full[:, None]
    s["refs"].index_add_(0, table[parents].flatten(), shared.flatten().to(torch.int32))
    ids, at = _take(s, tail)
    own_page = ids[at.clamp(max=len(ids) - 1)]
    last = (j == full[:, None]) & (tail > 0)[:, None]
    src = table[parents].gather(1, full.clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    table[children] = torch.where(shared, table[parents], torch.where(last, own_page[:, None], table[children]))
    s["seq_lens"][children] = lens.to(torch.int32)
    partial = tail > 0
    _copy_pages(s, src[partial].long(), own_page[partial].long())
    return _page_answer(s)


def _compact(s):
    s["block_table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    refs, table = s["refs"], s["block_table"]
    live = refs > 0
    n = live.sum()
    page = torch.arange(len(refs), device=DEV)
    src = page[live & (page >= n)]
    dst = page[~live & (page < n)]
    to = page.to(torch.int32)
    to[src] = dst.to(torch.int32)
    used = torch.arange(table.shape[1], device=DEV)[None, :] < _count_pages(s["seq_lens"])[:, None]
    table.copy_(torch.where(used, to[table.long()], table))
    refs[dst] = refs[src]
    refs[src] = 0
    _copy_pages(s, src, dst)
    return _page_answer(s, n.to(torch.int32).reshape(1))


def _gathered(s, cache, scale, token):
    """[B][tokens][Hkv][d] in 32 bits."""
    page = s["block_table"].long().gather(1, token // PAGE)
    x = _bytes(cache)[page, :, token % PAGE]
    x = x.view(cache.dtype).float() if cache.element_size() == 1 else x.float()
    return x if scale is None else x * scale[page][..., None]


def _scored(s):
    c = s["case"]
    B, hq, hkv, d = len(s["seq_lens"]), c["hq"], c["hkv"], c["d"]
    G, n, S = hq // hkv, int(s["rows"].max()), s["span"]
    lens = s["seq_lens"].long()
    token = s["first"][:, None] + torch.arange(S, device=DEV)
    inside = token.minimum(lens[:, None] - 1)
    k = _gathered(s, s["k"], s["ks"], inside).permute(0, 2, 3, 1).contiguous()     # [B][Hkv][d][S]
    v = _gathered(s, s["v"], s["vs"], inside).permute(0, 2, 1, 3).contiguous()     # [B][Hkv][S][d]
    q = torch.zeros((B, n, hq, d), device=DEV)
    q[s["seq"], s["row_of"]] = s["q"].float()
    pad = lambda x: torch.zeros((B, n), dtype=torch.int64, device=DEV).index_put_((s["seq"], s["row_of"]), x)   # noqa: E731
    pos, lo, hi = pad(s["pos"]), pad(s["lo"]), pad(s["hi"])
    q = q.view(B, n, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * G, d)
    x = (torch.matmul(q, k) / math.sqrt(d)).view(B, hkv, n, G, S)
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    at = token[:, None]
    if s["slopes"] is not None:
        far = (pos[:, :, None] - at).abs().float()
        x = x - s["slopes"].view(1, hkv, 1, G, 1) * far[:, None, :, None, :]
    seen = ((at >= lo[:, :, None]) & (at < hi[:, :, None]))[:, None, :, None, :]
    x = x.masked_fill(~seen, -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - torch.where(top.isfinite(), top, 0.0))
    p = p / p.sum(dim=-1, keepdim=True).clamp_min(1e-38)
    o = torch.matmul(p.view(B, hkv, n * G, S), v).view(B, hkv, n, G, d).permute(0, 2, 1, 3, 4).reshape(B, n, hq, d)
    return o[s["seq"], s["row_of"]].to(torch.bfloat16)


# ------------------------------------------------------------------ what the results should be

def _turned64(x, positions, c, inverse):
    """The rotation as a complex product, in 64 bits."""
    rot = c["rot"]
    f = float(c["base"]) ** (-torch.arange(rot // 2, dtype=torch.float64, device=DEV) * 2 / rot)
    w = torch.polar(torch.full_like(f, c["amplitude"])[None, :].expand(len(positions), -1).contiguous(),
                    positions.double()[:, None] * f * (-1.0 if inverse else 1.0))[:, None]
    x = x.double()
    head = x[..., :rot]
    pair = head.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if c["pairs"] == "half" else head.unflatten(-1, (-1, 2))
    z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * w)
    z = z.transpose(-1, -2).flatten(-2) if c["pairs"] == "half" else z.flatten(-2)
    return torch.cat([z, x[..., rot:]], dim=-1)


def _cache64(t, cache, scale, x):
    """The pool after the rows x (64 bits) were written, page by page."""
    out = cache.double() if cache.element_size() > 1 else cache.float().double()
    sc = None if scale is None else scale.double()
    table = t["block_table"].cpu().numpy()
    at = 0
    for b, (L, n) in enumerate(zip(t["lens"], t["rows"])):
        p = int(L - n)
        while p < L:
            m = min(PAGE - p % PAGE, int(L) - p)
            page, s0 = int(table[b, p // PAGE]), p % PAGE
            r = x[at:at + m].transpose(0, 1)   # [Hkv][m][d]
            if scale is None:
                out[page, :, s0:s0 + m] = r
            else:
                amax = r.abs().amax(dim=(1, 2))
                old = sc[page] if s0 else torch.zeros_like(amax)
                new = torch.where((amax > 448.0 * old) if s0 else torch.ones_like(amax, dtype=torch.bool), amax / 448.0, old)
                if s0:
                    out[page, :, :s0] *= torch.where(new > old, old / new, 1.0)[:, None, None]
                out[page, :, s0:s0 + m] = r / new[:, None, None]
                sc[page] = new
            p += m
            at += m
    if scale is not None:   # what E4M3 can hold
        out = out.float().clamp(-448, 448).to(torch.float8_e4m3fn).double()
    return out, sc


def exact(c, seed):
    if c["kind"] in ("admit", "fork", "compact"):
        return None   # page ids, and pages as they are
    t = _inputs(c, seed)
    if c["kind"] == "rotate":
        return _turned64(t["x"], t["positions"], c, c["inverse"])
    if c["kind"] == "append":
        k, ks = _cache64(t, t["k"], t["ks"], _turned64(t["k_new"], t["pos"], c, False))
        v, vs = _cache64(t, t["v"], t["vs"], t["v_new"].double())
        return {"q": _turned64(t["q"], t["pos"], c, False), "k": k, "v": v, "ks": ks, "vs": vs}
    G, d = c["hq"] // c["hkv"], c["d"]
    out = torch.zeros(t["q"].shape, dtype=torch.float64, device=DEV)
    pos, lo, hi = (t[x] for x in ("pos", "lo", "hi"))
    at = 0
    for b, (L, n) in enumerate(zip(t["lens"], t["rows"])):
        L, n = int(L), int(n)
        pages = t["block_table"][b, :-(-L // PAGE)].long()
        for g in range(c["hkv"]):
            k, v = (_bytes(x)[pages, g].view(x.dtype).double() if x.element_size() == 1 else x[pages, g].double()
                    for x in (t["k"], t["v"]))
            if t["ks"] is not None:
                k, v = k * t["ks"][pages, g].double()[:, None, None], v * t["vs"][pages, g].double()[:, None, None]
            k, v = k.reshape(-1, d)[:L], v.reshape(-1, d)[:L]
            r = slice(at, at + n)
            q = t["q"][r, g * G:(g + 1) * G].double().reshape(n * G, d)
            x = (torch.matmul(q, k.t().contiguous()) * d ** -0.5).view(n, G, L)
            if c["cap"]:
                x = torch.tanh(x / c["cap"]) * c["cap"]
            key = torch.arange(L, device=DEV)
            if t["slopes"] is not None:
                x = x - t["slopes"][g * G:(g + 1) * G].double()[None, :, None] * (pos[r, None] - key).abs().double()[:, None]
            x = x.masked_fill(((key < lo[r, None]) | (key >= hi[r, None]))[:, None], -math.inf)
            p = torch.softmax(x, dim=-1).nan_to_num(0.0)
            out[r, g * G:(g + 1) * G] = torch.matmul(p.view(n * G, L), v).view(n, G, d)
        at += n
    return out
