"""Attention with modified scores on the GPU (DecodeAttention.scored) against float64.

Tolerance of an output o = sum_t p_t v_t, with A = sum_t p_t |v_t|: every p_t is off by a
factor that has
  - the error of its score: the product of d terms accumulated in fp32, d 2^-24 of
    |q| |k| scale, the cap's 2^-21 of the cap (its tanh is 2^-22 off), the bias's 2^-22 of
    itself, and 2^-21 of the score for the log2 units; twice, for the maximum's too;
  - the exponential's 2^-21, the sum's n 2^-24 (n terms of one sign) and the product's n 2^-24;
  - its rounding: a bf16 value and a bf16 remainder, 2^-16, on the decode stream, one bf16
    value, 2^-8, in the multi-token kernel.
A bf16 output adds half a step, 2^-8 |o|.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

PAGE = 16


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_09207_amd import _abi
    _abi.load()
    return torch


class Case:
    def __init__(self, torch, kv, hq, hkv, d, lens, rows=None, layout="head", seed=0, out="f32", ranges=0, max_batch=None,
                 extra_pages=0, head_map=None):
        from paper_2607_09207_amd import DecodeAttention
        self.torch, self.kv, self.hq, self.hkv, self.d = torch, kv, hq, hkv, d
        rng = np.random.default_rng(seed)
        g = torch.Generator("cuda").manual_seed(seed)
        self.lens = np.asarray(lens, np.int64)
        self.rows = np.ones(len(lens), np.int64) if rows is None else np.asarray(rows, np.int64)
        used = -(-self.lens // PAGE)
        mp = int(max(1, used.max() if len(used) else 1)) + extra_pages
        npages = int(used.sum()) + 2
        perm = rng.permutation(npages)
        self.table = np.full((len(lens), mp), -1, np.int32)
        at = 0
        for b, u in enumerate(used):
            self.table[b, :u] = perm[at:at + u]
            at += u
        self.start = np.concatenate([[0], np.cumsum(self.rows)])
        n = int(self.start[-1]) if rows is not None else len(lens)
        self.q = (torch.randn((n, hq, d), device="cuda", generator=g) * 2).bfloat16()
        shape = (npages, hkv, PAGE, d) if layout == "head" else (npages, PAGE, hkv, d)
        view = (lambda t: t) if layout == "head" else (lambda t: t.transpose(1, 2))

        def pool():
            x = torch.randn(shape, device="cuda", generator=g)
            if kv == "bf16":
                return view(x.bfloat16()), None
            s = torch.rand((npages, hkv), device="cuda", generator=g) * 0.02 + 0.005
            sx = s[:, :, None, None] if layout == "head" else s[:, None, :, None]
            return view((x / sx).clamp(-448, 448).to(torch.float8_e4m3fn)), s
        (self.k, self.ks), (self.v, self.vs) = pool(), pool()
        # Slots past a sequence's end, and pages nobody uses, hold NaN.
        nan = {"bf16": 0x7FC0, "fp8": 0x7F}[kv]
        raw = torch.int16 if kv == "bf16" else torch.uint8
        spare = np.ones((npages, PAGE), bool)
        for b, L in enumerate(self.lens):
            for j in range(used[b]):
                spare[self.table[b, j], :min(PAGE, L - j * PAGE)] = False
        for t in (self.k, self.v):
            t.view(raw).transpose(1, 2)[torch.from_numpy(spare).cuda()] = nan
        self.block_table = torch.from_numpy(self.table).cuda()
        self.seq_lens = torch.from_numpy(self.lens.astype(np.int32)).cuda()
        self.q_start = None if rows is None else torch.from_numpy(self.start.astype(np.int32)).cuda()
        self.head_map = list(range(hq)) if head_map is None else head_map
        self.kv_of = [h // (hq // hkv) for h in range(hq)] if head_map is None else head_map
        self.layer = DecodeAttention(hq, hkv, d, max_batch or max(len(lens), 1), mp, "bf16",
                                     {"bf16": "bf16", "fp8": "fp8_e4m3fn"}[kv], out, kv_head_of_q=None if head_map is None else head_map,
                                     kv_strides=self.k.stride()[:3], num_work_ranges=ranges)
        self.out_bf16 = out == "bf16"

    def dense(self, b):
        """K, V of sequence b, [L][Hkv][d] in float64."""
        torch, L = self.torch, int(self.lens[b])
        pages = torch.from_numpy(self.table[b, :-(-L // PAGE)].astype(np.int64)).cuda()
        out = []
        for t, s in ((self.k, self.ks), (self.v, self.vs)):
            raw = torch.int16 if self.kv == "bf16" else torch.uint8
            x = t.view(raw)[pages].view(t.dtype).float().double()
            if s is not None:
                x = x * s[pages].double()[:, :, None, None]
            out.append(x.permute(0, 2, 1, 3).reshape(-1, self.hkv, self.d)[:L])
        return out

    def want(self, mod, few):
        """(outputs, tolerances) in float64.  few: the decode stream's rounding."""
        torch, G, d = self.torch, self.hq // self.hkv, self.d
        n = self.q.shape[0]
        o = torch.zeros((n, self.hq, d), dtype=torch.float64, device="cuda")
        tol = torch.zeros_like(o)
        cap, slopes, window = mod.get("score_cap", 0.0), mod.get("slopes"), mod.get("window", 0)
        key_start, prefix = mod.get("key_start"), mod.get("prefix_lens")
        kv_of = torch.tensor(self.kv_of, device="cuda")
        for b in range(len(self.lens)):
            L, m = int(self.lens[b]), int(self.rows[b])
            if L == 0 or m == 0:
                continue
            r = slice(int(self.start[b]), int(self.start[b]) + m) if self.q_start is not None else slice(b, b + 1)
            k, v = self.dense(b)
            k, v = k[:, kv_of].transpose(0, 1).contiguous(), v[:, kv_of].transpose(0, 1).contiguous()   # [Hq][L][d]
            q = self.q[r].double().transpose(0, 1).contiguous()                                        # [Hq][m][d]
            pos = (L - m + torch.arange(m, device="cuda"))[:, None]
            t = torch.arange(L, device="cuda")[None, :]
            lo, hi = torch.zeros_like(pos), pos + 1
            if key_start is not None:
                lo = torch.maximum(lo, key_start[r].long()[:, None])
            if window:
                lo = torch.maximum(lo, pos - window + 1)
            if prefix is not None:
                hi = torch.maximum(hi, prefix[b].long().clamp(max=L))
            seen = ((t >= lo) & (t < hi) & (pos >= 0))[None]
            kf = torch.where(k.isfinite(), k, 0.0)
            s = torch.matmul(q, kf.transpose(1, 2).contiguous()) / math.sqrt(d)
            odd = ~k.isfinite().all(-1)[:, None, :] & seen
            big = (q.norm(dim=-1)[:, :, None] * kf.norm(dim=-1)[:, None, :] / math.sqrt(d))
            err = d * 2.0 ** -24 * big + 2.0 ** -21 * s.abs()
            if cap:
                s = cap * torch.tanh(s / cap)
                err = err + 2.0 ** -21 * cap
            if slopes is not None:
                bias = slopes.double()[:, None, None] * (pos - t).abs().double()[None]
                s = s - bias
                err = err + 2.0 ** -22 * bias.abs()
            s = s.masked_fill(~seen, -math.inf)
            p = torch.softmax(s, dim=-1)
            none = ~seen.any(-1, keepdim=True)
            p = torch.where(none.expand_as(p), 0.0, p)
            err = torch.where(seen, err, 0.0).amax(-1, keepdim=True)
            vf = torch.where(v.isfinite(), v, 0.0)
            x = torch.matmul(p, vf)
            for is_odd, value in ((v == math.inf, math.inf), (v == -math.inf, -math.inf), (v.isnan(), math.nan)):
                if is_odd.any():
                    hit = torch.matmul(seen.expand_as(p).double(), is_odd.double()) > 0
                    x = torch.where(hit, x + value, x)
            x = torch.where(odd.any(-1, keepdim=True).expand_as(x), math.nan, x)
            a = torch.matmul(p, vf.abs())
            f = 2 * err + 2.0 ** -20 + 2 * L * 2.0 ** -24 + (2.0 ** -16 if few else 2.0 ** -8)
            o[r], tol[r] = x.transpose(0, 1), (a * f).transpose(0, 1)
        return o, tol

    def run(self, mod, **kw):
        return self.layer.scored(self.q, self.k, self.v, self.block_table, self.seq_lens, q_start=self.q_start,
                                 k_scale=self.ks, v_scale=self.vs, **mod, **kw)

    def check(self, mod, few, what, **kw):
        torch = self.torch
        print(what, {k: (v if not hasattr(v, "shape") else "tensor") for k, v in mod.items()}, flush=True)
        got = self.run(mod, **kw).double()
        want, tol = self.want(mod, few)
        if self.out_bf16:
            tol = tol * 1.01 + 2.0 ** -8 * (want.abs() + tol)
        fin = want.isfinite()
        assert torch.equal(fin, got.isfinite()), f"{what}: {int((fin != got.isfinite()).sum())} infinities or NaN misplaced"
        assert torch.equal(want.isnan(), got.isnan()) and torch.equal(want == math.inf, got == math.inf), f"{what}: odd values differ"
        bad = fin & ~((got - want).abs() <= tol + 1e-30)
        assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, first {bad.nonzero()[0].tolist()}, "
                               f"worst {float(((got - want).abs() / (tol + 1e-30))[bad].max()):.3g} times the tolerance")
        return got

    def mods(self, seed):
        """Modifications, alone and together."""
        torch, rng = self.torch, np.random.default_rng(seed)
        n = self.q.shape[0]
        slopes = torch.exp2(-8.0 * torch.arange(1, self.hq + 1, device="cuda") / self.hq)
        longest = int(self.lens.max()) if len(self.lens) else 1
        starts = torch.from_numpy(rng.integers(-3, longest + 2, size=n).astype(np.int32)).cuda()
        prefix = torch.from_numpy(rng.integers(-2, longest + 20, size=len(self.lens)).astype(np.int32)).cuda()
        doc = torch.from_numpy((np.concatenate([np.maximum(L - m + np.arange(m), 0) // 37 * 37 for L, m in zip(self.lens, self.rows)])
                                if self.q_start is not None else np.maximum(self.lens - 1, 0) // 37 * 37).astype(np.int32)).cuda()
        return [dict(), dict(score_cap=20.0), dict(slopes=slopes), dict(window=1), dict(window=16), dict(window=33),
                dict(key_start=starts), dict(prefix_lens=prefix), dict(key_start=doc, score_cap=5.0),
                dict(window=50, slopes=-slopes, score_cap=1000.0),
                dict(score_cap=50.0, slopes=slopes, window=100, key_start=doc, prefix_lens=prefix)]


HEADS = [(8, 2), (16, 16), (28, 4), (16, 1), (40, 8)]
ONE = [("short", [1, 16, 17, 0, 5, 33, 64, 15, 250], 0), ("long", [3000, 1, 700, 0, 129], 0), ("cut", [900, 0, 77, 400], 23),
       ("many", list(range(0, 600, 23)) * 2, 0)]


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name,lens,ranges", ONE, ids=[x[0] for x in ONE])
def test_one_row(torch, kv, d, name, lens, ranges):
    for i, (hq, hkv) in enumerate(HEADS):
        c = Case(torch, kv, hq, hkv, d, lens, seed=i, ranges=ranges, layout=["head", "slot"][i % 2], out=["f32", "bf16"][i // 2 % 2])
        for mod in c.mods(i):
            c.check(mod, True, f"one row {kv} {hq}/{hkv} d{d} {name}")
        assert c.layer.read_flags(device=c.q.device) == 0


def test_one_row_large_batch(torch):
    """More sequences than two workgroups a CU take, and empty ones among them."""
    lens = np.random.default_rng(0).integers(0, 90, size=1500)
    for kv, d in (("fp8", 64), ("bf16", 64), ("bf16", 128)):
        c = Case(torch, kv, 8, 1, d, lens, seed=3)
        for mod in c.mods(1)[1::3]:
            c.check(mod, True, f"batch of 1500 {kv} d{d}")


ROWS = [([40, 5, 0, 300], [3, 5, 0, 4]), ([1, 17, 64], [1, 1, 1]), ([700, 33, 16], [16, 10, 16]), ([2000], [2]),
        ([100] * 30, [4] * 30)]


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", range(len(ROWS)))
def test_few_rows(torch, kv, d, case):
    """The decode stream with several rows: one and two tiles a segment, several chunks."""
    lens, rows = ROWS[case]
    for i, (hq, hkv) in enumerate(HEADS):
        if max(rows) * hq // hkv > 64:
            continue
        c = Case(torch, kv, hq, hkv, d, lens, rows, seed=i, ranges=[0, 0, 11][i % 3], layout=["slot", "head"][i % 2])
        for mod in c.mods(i):
            c.check(mod, True, f"few rows {kv} {hq}/{hkv} d{d} {rows}", max_q_len=max(rows))
        assert c.layer.read_flags(device=c.q.device) == 0


MANY = [([40], [40]), ([300, 70], [33, 70]), ([500, 64, 0, 200, 1], [100, 64, 0, 17, 1]), ([130] * 20, [130] * 20),
        ([1000, 900], [200, 5]), ([200] * 70, [9] * 70)]


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", range(len(MANY)))
def test_many_rows(torch, kv, d, case):
    """The multi-token kernel: 128 rows a workgroup, and 32 with the keys split."""
    lens, rows = MANY[case]
    for i, (hq, hkv) in enumerate(HEADS):
        c = Case(torch, kv, hq, hkv, d, lens, rows, seed=i, layout=["slot", "head"][i % 2], out=["bf16", "f32"][i % 2])
        for mod in c.mods(i):
            c.check(mod, False, f"many rows {kv} {hq}/{hkv} d{d} case {case}")
        assert c.layer.read_flags(device=c.q.device) == 0


def poison(c, b, t0, t1, what):
    """Keys t0 .. t1 of sequence b get odd values."""
    torch = c.torch
    nan, inf, ninf = ((0x7FC0, 0x7F80, 0xFF80 - 65536) if c.kv == "bf16" else (0x7F, 0xFF, 0x7F))
    raw = torch.int16 if c.kv == "bf16" else torch.uint8
    for t in range(t0, t1):
        p, s = int(c.table[b, t // PAGE]), t % PAGE
        if "k" in what:
            c.k.view(raw)[p, :, s, t % c.d] = nan
        if "v" in what:
            c.v.view(raw)[p, :, s, (3 * t) % c.d] = inf
            c.v.view(raw)[p, :, s, (5 * t + 1) % c.d] = ninf
        if "n" in what:
            c.v.view(raw)[p, :, s, (7 * t + 2) % c.d] = nan


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
def test_odd_values_in_masked_places(torch, kv, d):
    """A key that a row does not see has no part in it; one it sees does."""
    # One row: everything below the window, in the first page that is read too.
    c = Case(torch, kv, 8, 2, d, [100, 37, 300], seed=1)
    for b, L in enumerate([100, 37, 300]):
        poison(c, b, 0, L - 21, "kvn")
    c.check(dict(window=21), True, "one row, odd values below the window")
    poison(c, 2, 290, 292, "v")
    c.check(dict(window=21), True, "one row, odd values in it")
    # Rows of one tile in two documents: the first one's keys are odd.
    for few, hq, hkv, lens, rows in ((True, 8, 2, [40, 90], [8, 6]), (True, 12, 2, [40, 90], [8, 6]),
                                     (False, 8, 2, [140, 90], [50, 60]), (False, 28, 4, [300] * 9, [290] * 9)):
        for what in ("v", "vn", "k"):
            c = Case(torch, kv, hq, hkv, d, lens, rows, seed=2)
            start = []
            for b, (L, m) in enumerate(zip(lens, rows)):
                cut = L - m // 2
                poison(c, b, max(0, cut - 19), cut - 1, what)
                start += [0 if L - m + i < cut else cut for i in range(m)]
            mod = dict(key_start=torch.tensor(start, dtype=torch.int32, device="cuda"), score_cap=30.0)
            c.check(mod, few, f"documents, odd {what}", max_q_len=max(rows) if few else 0)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_odd_values_that_weigh_nothing(torch, kv):
    """Rows of one workgroup of which some see an infinity, with a weight that fp32 holds as 0,
    and the others do not: the same result every time, and infinite in the rows that see it."""
    for hq, hkv, lens, rows in ((8, 2, [340, 300], [100, 60]), (28, 4, [700] * 9, [290] * 9), (8, 1, [500], [40])):
        c = Case(torch, kv, hq, hkv, 128, lens, rows, seed=3)
        start = []
        for b, (L, m) in enumerate(zip(lens, rows)):
            at = 30 + 3 * b
            poison(c, b, at, at + 2, "v")
            # Every third row begins behind them (the first keys weigh 2^-577 and less in all of them).
            start += [at + 2 if i % 3 == 2 else 0 for i in range(m)]
        mod = dict(key_start=torch.tensor(start, dtype=torch.int32, device="cuda"), slopes=torch.full((hq,), 4.0, device="cuda"))
        first = c.check(mod, False, f"odd values of no weight {kv} {hq}/{hkv}")
        for _ in range(5):
            assert torch.equal(c.run(mod).double().nan_to_num(7.0), first.nan_to_num(7.0))


@pytest.mark.parametrize("rows,kw", [(None, {}), ([4, 3, 5], dict(max_q_len=5)), ([90, 70, 60], {})])
def test_pages_of_zeros(torch, rows, kw):
    """fp8 pages whose V scale is 0: their keys count, with values of 0."""
    c = Case(torch, "fp8", 8, 2, 128, [300, 90, 77], rows, seed=4)
    for b, j in ((0, 0), (0, 7), (0, 18), (1, 5), (2, 0), (2, 1), (2, 2), (2, 3), (2, 4)):
        c.vs[int(c.table[b, j])] = 0.0
    for mod in (dict(), dict(score_cap=10.0), dict(window=40)):
        got = c.check(mod, rows is None or max(rows) < 16, "zeros", **kw)
        assert not got[2 if rows is None else slice(int(c.start[2]), None)].any()


@pytest.mark.parametrize("rows,kw", [(None, {}), ([4, 3, 5], dict(max_q_len=5)), ([90, 70, 60], {}), ([290, 80, 70], {})])
def test_scales_far_apart(torch, rows, kw):
    """fp8 pages of one sequence whose V scales differ by up to 2^180: a key's weight in the sum
    does not depend on its page's scale."""
    for d, (hq, hkv) in ((64, (8, 2)), (128, (28, 4))):
        c = Case(torch, "fp8", hq, hkv, d, [300, 90, 77], rows, seed=4)
        g = torch.Generator("cuda").manual_seed(7)
        c.vs.copy_(torch.exp2(180 * torch.rand(c.vs.shape, device="cuda", generator=g) - 90))
        few = rows is None or max(rows) < 16
        for q in (c.q, torch.zeros_like(c.q)):   # (and all weights alike)
            c.q = q
            for mod in (dict(), dict(score_cap=10.0), dict(score_cap=300.0), dict(window=40)):
                c.check(mod, few, f"scales far apart {d} {rows}", **kw)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_pages_below_the_window_are_not_read(torch, kv):
    for rows, few in ((None, True), ([3, 4], True), ([40, 30], False)):
        c = Case(torch, kv, 8, 2, 128, [700, 333], rows, seed=5)
        m = 0 if rows is None else max(rows)
        for b, L in enumerate([700, 333]):
            first = (L - (1 if rows is None else rows[b]) - 64 + 1) // PAGE
            c.block_table[b, :first] = 10 ** 9
        c.check(dict(window=64), few, "pages below the window", max_q_len=m if few and m else 0)
        assert c.layer.read_flags(device=c.q.device) == 0


def test_head_map_and_empty_calls(torch):
    c = Case(torch, "bf16", 8, 4, 64, [50, 200], seed=6, head_map=[3, 1, 0, 2, 2, 0, 1, 3])
    for mod in c.mods(0):
        c.check(mod, True, "head map")
    c = Case(torch, "bf16", 8, 4, 64, [50, 200], [20, 100], seed=6, head_map=[3, 1, 0, 2, 2, 0, 1, 3])
    for mod in c.mods(0):
        c.check(mod, False, "head map, many rows")
    c = Case(torch, "bf16", 8, 2, 64, [0, 0], seed=7)
    assert not c.run(dict(window=5, slopes=torch.ones(8, device="cuda"))).any()
    e = torch.empty((0, 8, 64), dtype=torch.bfloat16, device="cuda")
    assert c.layer.scored(e, c.k, c.v, c.block_table[:0], c.seq_lens[:0], window=3).shape == (0, 8, 64)


def test_plain_scores_are_run(torch):
    """Without modifications: the results of the plain calls, within their own tolerance."""
    c = Case(torch, "bf16", 28, 4, 128, [900, 33, 0, 2500], seed=8)
    a = c.run({}).double()
    b = c.layer(c.q, c.k, c.v, c.block_table, c.seq_lens).double()
    _, tol = c.want({}, False)
    assert ((a - b).abs() <= 2 * tol + 1e-30).all()


def test_bad_pages_and_lengths(torch):
    c = Case(torch, "bf16", 8, 2, 64, [100, 50], seed=9)
    good = c.run(dict(window=40))
    c.block_table[0, 5] = c.k.shape[0]
    out = c.run(dict(window=40))
    assert torch.equal(out[1], good[1]) and out.isfinite().all()
    assert c.layer.read_flags(device=c.q.device) == 1
    c.seq_lens[0] = -4
    c.run(dict(window=40))
    assert c.layer.read_flags(device=c.q.device) == 3
    c = Case(torch, "bf16", 8, 2, 64, [10, 50], [20, 30], seed=9)   # more rows than tokens
    o = c.run(dict(score_cap=9.0, prefix_lens=torch.tensor([10, 3], dtype=torch.int32, device="cuda")))
    assert not o[:10].any() and o[10:].abs().sum(-1).all()
    assert c.layer.read_flags(device=c.q.device) == 2


def test_refusals(torch):
    from paper_2607_09207_amd import DecodeAttention, RldaError
    c = Case(torch, "bf16", 8, 2, 64, [100, 50], seed=9)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")   # noqa: E731
    for bad in (dict(score_cap=-1.0), dict(score_cap=float("nan")), dict(score_cap=float("inf")), dict(score_cap=1e-5), dict(window=-1),
                dict(slopes=torch.ones(7, device="cuda")), dict(slopes=torch.ones(8, device="cuda").double()), dict(key_start=i32(3)),
                dict(key_start=i32(2).cpu()), dict(prefix_lens=i32(1)), dict(prefix_lens=i32(4)[::2])):
        with pytest.raises(RldaError):
            c.run(bad)
            print("taken:", bad)
    with pytest.raises(RldaError):
        c.layer.scored(c.q[:1], c.k, c.v, c.block_table, c.seq_lens)
    f = DecodeAttention(2, 2, 64, 2, 8, "f32", "f32", "f32")
    k = torch.zeros((4, 2, 16, 64), device="cuda")
    with pytest.raises(RldaError):
        f.scored(torch.zeros((2, 2, 64), device="cuda"), k, k.clone(), i32(16).view(2, 8), i32(2), window=4)


def test_stream_and_graph(torch):
    """On another stream, and captured and replayed with eager calls between."""
    for rows, kw in ((None, {}), ([4, 2, 1], dict(max_q_len=4)), ([60, 2, 7], {})):
        c = Case(torch, "fp8", 12, 2, 128, [900, 33, 70], rows, seed=5)
        mod = c.mods(3)[-1]
        want = c.run(mod, **kw)
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        got = c.run(mod, stream=st, **kw)
        torch.cuda.current_stream().wait_stream(st)
        assert torch.equal(got, want)
        out = torch.empty_like(want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.run(mod, out=out, **kw)
        for _ in range(3):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            assert torch.equal(c.run(mod, **kw), want)


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
def test_caps_out_of_range(torch, native):
    """A cap that fp32 holds as 0 is refused as any other below the range, and does not mean none."""
    from paper_2607_09207_amd import RldaError, _abi
    c = Case(torch, "bf16", 8, 2, 64, [90, 33])
    c.layer.workspace(c.q.device)
    if not native:
        c.layer._fast = _abi.LEFT_TO_PYTHON
    for cap in (1e-50, -1e-50, 1e-46, 1e-30, 2.0 ** -11, -1.0, math.nan, math.inf, 1e300, 2.0 ** 31):
        with pytest.raises(RldaError):
            c.run(dict(score_cap=cap))
    assert torch.equal(c.run(dict(score_cap=0)), c.run(dict(score_cap=-0.0)))
