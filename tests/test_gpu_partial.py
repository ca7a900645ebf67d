"""A cache read in part and kept in part (page_bounds, select_pages, selected, weighed, page_evict)
on the GPU.

Bounds, choices and evictions are compared exactly: bounds are quotients of fp32 numbers rounded
to whole ones (one IEEE division and a floor or ceiling on both sides), a choice's scores are
whole numbers below 2^24 times two fp32 factors in one order.

Tolerance of an attention output o = sum_t p_t v_t, with A = sum_t p_t |v_t|: every p_t is off by a
factor that has
  - the error of its score: the product of d terms accumulated in fp32, d 2^-24 of |q| |k| scale,
    and 2^-21 of the score for the log2 units; twice, for the maximum's too;
  - the exponential's 2^-21, the sum's n 2^-24 (n terms of one sign) and the product's n 2^-24;
  - its rounding, to a bf16 value and a bf16 remainder, 2^-16 (f32 caches: none).
A bf16 output adds half a step, 2^-8 |o|.  A page's weight has the scores' errors, the
exponentials', twice the sums', and half a step, 2^-24, of the two logarithms (times ln 2), of
the additions over the rows and heads (one of each, all of one sign) and of the update (two).
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

PAGE = 16
NAN = {"bf16": 0x7FC0, "fp8": 0x7F, "f32": 0x7FC00000}


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_09207_amd import _abi
    _abi.load()
    return torch


def raw_type(torch, kv):
    return {"bf16": torch.int16, "fp8": torch.uint8, "f32": torch.int32}[kv]


class Case:
    """Sequences on a pool of their own; slots past their ends, and pages nobody uses, hold NaN."""

    def __init__(self, torch, kv, hq, hkv, d, lens, rows=None, layout="head", seed=0, out="f32", ranges=0, max_batch=None,
                 extra_pages=0, head_map=None, spare=2):
        from paper_2607_09207_amd import DecodeAttention
        self.torch, self.kv, self.hq, self.hkv, self.d, self.G = torch, kv, hq, hkv, d, hq // hkv
        rng = np.random.default_rng(seed)
        g = self.gen = torch.Generator("cuda").manual_seed(seed)
        self.lens = np.asarray(lens, np.int64)
        self.rows = np.ones(len(lens), np.int64) if rows is None else np.asarray(rows, np.int64)
        self.start = np.concatenate([[0], np.cumsum(self.rows)])
        self.used = -(-self.lens // PAGE)
        self.mp = int(max(1, self.used.max() if len(lens) else 1)) + extra_pages
        self.npages = int(self.used.sum()) + spare
        perm = rng.permutation(self.npages)
        self.table = np.full((len(lens), self.mp), -1, np.int32)
        at = 0
        for b, u in enumerate(self.used):
            self.table[b, :u] = perm[at:at + u]
            at += u
        qd = torch.float32 if kv == "f32" else torch.bfloat16
        self.q = (torch.randn((int(self.start[-1]), hq, d), device="cuda", generator=g) * 2).to(qd)
        shape = (self.npages, hkv, PAGE, d) if layout == "head" else (self.npages, PAGE, hkv, d)
        view = (lambda t: t) if layout == "head" else (lambda t: t.transpose(1, 2))

        def pool():
            x = torch.randn(shape, device="cuda", generator=g)
            if kv != "fp8":
                return view(x.to(qd)), None
            s = torch.rand((self.npages, hkv), device="cuda", generator=g) * 0.02 + 0.005
            sx = s[:, :, None, None] if layout == "head" else s[:, None, :, None]
            return view((x / sx).clamp(-448, 448).to(torch.float8_e4m3fn)), s
        (self.k, self.ks), (self.v, self.vs) = pool(), pool()
        spare = np.ones((self.npages, PAGE), bool)
        for b, L in enumerate(self.lens):
            for j in range(self.used[b]):
                spare[self.table[b, j], :min(PAGE, L - j * PAGE)] = False
        for t in (self.k, self.v):
            t.view(raw_type(torch, kv)).transpose(1, 2)[torch.from_numpy(spare).cuda()] = NAN[kv]
        self.block_table = torch.from_numpy(self.table).cuda()
        self.seq_lens = torch.from_numpy(self.lens.astype(np.int32)).cuda()
        self.q_start = None if rows is None else torch.from_numpy(self.start.astype(np.int32)).cuda()
        self.kv_of = [h // self.G for h in range(hq)] if head_map is None else head_map
        self.layer = DecodeAttention(hq, hkv, d, max_batch or max(len(lens), 1), self.mp, qd,
                                     {"bf16": "bf16", "fp8": "fp8_e4m3fn", "f32": "f32"}[kv], out, kv_head_of_q=head_map,
                                     kv_strides=self.k.stride()[:3], num_work_ranges=ranges)
        self.bounds = torch.full((self.npages, hkv, 2, d), 55, dtype=torch.int8, device="cuda")
        self.bscale = torch.full((self.npages, hkv), -3.0, device="cuda")

    def cache(self):
        return self.k, self.v, self.block_table, self.seq_lens

    def scales(self):
        return dict(k_scale=self.ks, v_scale=self.vs)

    def make_bounds(self, first=None, **kw):
        self.layer.page_bounds(self.k, self.block_table, self.seq_lens, self.bounds, self.bscale, first=first,
                               k_scale=self.ks, **kw)

    def all_bounds(self):
        self.make_bounds(first=self.torch.zeros(len(self.lens), dtype=self.torch.int32, device="cuda"))

    def values(self, t, s, page):
        """Page `page` of a cache, [Hkv][16][d] in fp32."""
        x = t[page].contiguous()
        x = x.view(raw_type(self.torch, self.kv)).view(t.dtype).float()
        return x if s is None else x * s[page][:, None, None]

    def select(self, budget, **kw):
        return self.layer.select_pages(self.q, self.bounds, self.bscale, self.block_table, self.seq_lens, budget,
                                       q_start=self.q_start, **kw)

    def attend(self, pages, counts, **kw):
        return self.layer.selected(self.q, *self.cache(), pages, counts, q_start=self.q_start, **self.scales(), **kw)

    def weigh(self, weights, **kw):
        return self.layer.weighed(self.q, *self.cache(), weights, q_start=self.q_start, **self.scales(), **kw)

    def row_list(self):
        """(row, sequence, tokens it sees)."""
        return [(int(self.start[b]) + i, b, int(L) - int(n) + i + 1) for b, (L, n) in enumerate(zip(self.lens, self.rows))
                for i in range(int(n))]

    def flags(self, ws=None):
        self.torch.cuda.synchronize()
        return self.layer.read_flags(device="cuda:0") if ws is None else self.layer.read_flags(workspace=ws)

    # The attention of every row over the keys in keys[row][g], in float64: outputs, their tolerances,
    # and per row the probabilities [Hq][tokens] with their factors of error.
    def want(self, keys):
        torch, d = self.torch, self.d
        n = self.q.shape[0]
        o = torch.zeros((n, self.hq, d), dtype=torch.float64, device="cuda")
        tol, parts = torch.zeros_like(o), {}
        for r, b, L in self.row_list():
            if L <= 0:
                continue
            pages = [self.values(self.k, self.ks, int(p)) for p in self.table[b, :-(-L // PAGE)]]
            k = torch.cat(pages, dim=1)[:, :L].double()
            v = torch.cat([self.values(self.v, self.vs, int(p)) for p in self.table[b, :-(-L // PAGE)]], dim=1)[:, :L].double()
            kv = torch.tensor(self.kv_of, device="cuda")
            k, v, q = k[kv].contiguous(), v[kv].contiguous(), self.q[r].double()       # [Hq][L][d], [Hq][d]
            x = (k * q[:, None]).sum(-1) / math.sqrt(d)
            seen = torch.zeros((self.hq, L), device="cuda", dtype=torch.float64)      # how often a key counts
            for h in range(self.hq):
                for j in keys(r, self.kv_of[h], L):
                    seen[h, j * PAGE:(j + 1) * PAGE] += 1
            err = d * 2.0 ** -24 * q.norm(dim=-1)[:, None] * k.norm(dim=-1) / math.sqrt(d) + 2.0 ** -21 * x.abs()
            err = torch.where(seen > 0, err, 0.0).amax(-1, keepdim=True)
            x = x.masked_fill(seen == 0, -math.inf)
            top = x.amax(-1, keepdim=True)
            top = torch.where(top.isfinite(), top, 0.0)
            e = torch.exp(x - top) * seen
            z = e.sum(-1, keepdim=True)
            p = torch.where(z > 0, e / z.clamp_min(1e-300), 0.0)
            o[r] = (p[:, :, None] * v).sum(1)
            a = (p[:, :, None] * v.abs()).sum(1)
            f = 2 * err + 2.0 ** -20 + 2 * L * 2.0 ** -24
            tol[r] = a * (f + (0.0 if self.kv == "f32" else 2.0 ** -16))
            logs = (top.abs() / math.log(2) + (L + 1.0) ** 0.5) * 2.0 ** -23      # |log2 of sums| of 1 to L terms, and of pages
            small = torch.log2(p.clamp_min(1e-38)).abs() * 2.0 ** -23
            parts[r] = (p, f + logs + small)
        return o, tol, parts

    def check(self, got, o, tol, out="f32"):
        if out == "bf16":
            tol = tol + 2.0 ** -8 * o.abs()
        bad = ~((got.double() - o).abs() <= tol + 1e-30)
        assert not bad.any(), (int(bad.sum()), float(((got.double() - o).abs() / (tol + 1e-30))[bad].max()))


LAYOUTS = [("bf16", 28, 4, 128), ("fp8", 40, 8, 128), ("bf16", 12, 2, 64), ("fp8", 16, 1, 64), ("bf16", 3, 3, 128),
           ("f32", 4, 4, 128), ("f32", 4, 2, 64)]


# ---------------------------------------------------------------- bounds

def over_127(x):
    """The quotient, rounded once (a number as the divisor would be a product with its reciprocal)."""
    return x / x.new_full(x.shape, 127)


def plain_bounds(torch, x):
    """x [Hkv][tokens][d] fp32: (bounds [Hkv][2][d], scale [Hkv])."""
    if not bool(x.isfinite().all()):
        odd = ~x.isfinite().flatten(1).all(-1)
    else:
        odd = torch.zeros(x.shape[0], dtype=torch.bool, device=x.device)
    y = torch.where(odd[:, None, None], 0.0, x)
    s = over_127(y.abs().amax(dim=(1, 2)))
    by = torch.where(s > 0, s, 1.0)[:, None]
    zero = (s == 0)[:, None]
    lo = torch.where(zero, 0.0, (y.amin(1) / by).floor().clamp(-127, 127))
    hi = torch.where(zero, 0.0, (y.amax(1) / by).ceil().clamp(-127, 127))
    return torch.stack([lo, hi], 1).to(torch.int8), torch.where(odd, math.inf, s)


def expect_bounds(c, first, b0, s0):
    want, scale = b0.clone(), s0.clone()
    for b, L in enumerate(c.lens):
        L = int(L)
        if L == 0:
            continue
        j0 = (L - 1) // PAGE if first is None else first[b] // PAGE
        for j in range(j0, -(-L // PAGE)):
            page = int(c.table[b, j])
            x = c.values(c.k, c.ks, page)[:, :min(PAGE, L - j * PAGE)]
            want[page], scale[page] = plain_bounds(c.torch, x)
    return want, scale


@pytest.mark.parametrize("layout", ["head", "slot"])
@pytest.mark.parametrize("kv,hq,hkv,d", LAYOUTS)
def test_bounds(torch, kv, hq, hkv, d, layout):
    c = Case(torch, kv, hq, hkv, d, [1, 0, 15, 16, 17, 250, 33, 700], layout=layout, seed=d + hq)
    for first in (None, [0] * 8, [1, 0, 3, 16, 16, 100, 32, 511]):
        b0, s0 = c.bounds.clone(), c.bscale.clone()
        c.make_bounds(None if first is None else torch.tensor(first, dtype=torch.int32, device="cuda"))
        want, scale = expect_bounds(c, first, b0, s0)
        torch.cuda.synchronize()
        assert torch.equal(c.bounds, want) and torch.equal(c.bscale, scale), first
    # s lo <= k <= s hi, up to the roundings of s and of a quotient below 128.
    for b, L in enumerate(c.lens):
        for j in range(c.used[b]):
            page = int(c.table[b, j])
            x = c.values(c.k, c.ks, page)[:, :min(PAGE, int(L) - j * PAGE)].double()
            s = c.bscale[page].double()[:, None]
            lo, hi = c.bounds[page, :, 0].double() * s, c.bounds[page, :, 1].double() * s
            slack = 128 * 2.0 ** -22 * s
            assert (x.amin(1) >= lo - slack).all() and (x.amax(1) <= hi + slack).all()
    assert c.flags() == 0


@pytest.mark.parametrize("kv,hq,hkv,d", [("bf16", 8, 2, 128), ("fp8", 8, 2, 64), ("f32", 2, 2, 64)])
def test_bounds_of_odd_keys(torch, kv, hq, hkv, d):
    """Zeros, the type's largest values, infinities and NaN; an fp8 page's scale that is negative,
    0, infinite."""
    c = Case(torch, kv, hq, hkv, d, [PAGE * 6], seed=3)
    t = [int(x) for x in c.table[0]]
    c.k[t[0]] = 0
    c.k.view(raw_type(torch, kv))[t[1], 0, 5, 7] = NAN[kv]
    if kv != "fp8":
        c.k[t[2], 1, 3, 0] = math.inf
        c.k[t[3], 0, 0, 1] = -math.inf
        c.k[t[4], 0, 2, 2] = torch.finfo(c.k.dtype).max
        c.k[t[4], 0, 2, 3] = -torch.finfo(c.k.dtype).max
        c.k[t[5], 0] = -0.0
        c.k[t[2], 0] = c.k[t[2], 0] * 1e-38 * 1e-5   # quotients far beyond 127, one sign alone in some elements
        c.k[t[5], 1] = -c.k[t[5], 1].abs() * 1e-38 * 1e-4
    else:
        c.ks[t[2], 0], c.ks[t[3], 0], c.ks[t[4], 1], c.ks[t[5], 0] = -0.01, 0.0, math.inf, 1e38
        c.ks[t[2], 1], c.ks[t[5], 1] = 2e-45, -3e-45
    c.all_bounds()
    want, scale = expect_bounds(c, [0], c.bounds, c.bscale)
    torch.cuda.synchronize()
    assert torch.equal(c.bscale, scale) and torch.equal(c.bounds, want)
    assert c.bscale[t[1], 0] == math.inf and c.bscale[t[1], 1] < math.inf and c.flags() == 0


def test_bounds_of_wrong_tables(torch):
    c = Case(torch, "bf16", 8, 2, 64, [40, 50, 60], seed=4)
    c.block_table[0, 1], c.block_table[1, 3] = -7, c.npages
    c.seq_lens[2] = PAGE * c.mp + 1
    b0 = c.bounds.clone()
    c.all_bounds()
    assert c.flags() == 3
    for page in c.table[2][:4]:
        assert torch.equal(c.bounds[int(page)], b0[int(page)])
    c = Case(torch, "bf16", 8, 2, 64, [40, 50, 60], seed=4)
    c.make_bounds(torch.tensor([-1, 51, 60], dtype=torch.int32, device="cuda"))
    assert c.flags() == 2


# ---------------------------------------------------------------- choice

def plain_choice(c, budget, sink, recent):
    """Pages of every (row, KV head), in Python floats and fp32 factors."""
    torch, d = c.torch, c.d
    pages = np.full((c.q.shape[0], c.hkv, budget), -1, np.int32)
    counts = np.zeros((c.q.shape[0], c.hkv), np.int32)
    q = c.q.float()
    fine = q.isfinite().all(-1, keepdim=True)
    q = torch.where(fine, q, 0.0)
    sq = over_127(q.abs().amax(-1, keepdim=True))
    q8 = torch.where(sq > 0, (q / torch.where(sq > 0, sq, 1.0)).round().clamp(-127, 127), 0.0).double()
    for r, b, L in c.row_list():
        n = max(-(-L // PAGE), 0)
        page = torch.from_numpy(c.block_table[b, :n].cpu().numpy().astype(np.int64)).cuda()
        there = (page >= 0) & (page < c.npages)
        page = torch.where(there, page, 0)
        for g in range(c.hkv):
            heads = [h for h in range(c.hq) if c.kv_of[h] == g]
            lo, hi = c.bounds[page, g, 0].double(), c.bounds[page, g, 1].double()     # [n][d]
            s = c.bscale[page, g]
            u = torch.stack([(torch.maximum(q8[r, h] * lo, q8[r, h] * hi)).sum(-1).float() * sq[r, h] for h in heads]).amax(0)
            x = torch.where(s.isfinite(), u * s, math.inf)
            x = torch.where(there, x, -math.inf).cpu().numpy()
            kept = [j for j in range(n) if j < sink or j >= n - recent]
            rest = sorted((j for j in range(n) if j not in set(kept)), key=lambda j: (-x[j], j))
            got = sorted(kept + rest[:max(budget - len(kept), 0)]) if n > budget else list(range(n))
            pages[r, g, :len(got)] = got
            counts[r, g] = len(got)
    return pages, counts


@pytest.mark.parametrize("budget,sink,recent", [(1, 0, 1), (4, 1, 2), (16, 4, 4), (16, 8, 8), (40, 0, 1), (100, 1, 1)])
@pytest.mark.parametrize("kv,hq,hkv,d", LAYOUTS)
def test_choice(torch, kv, hq, hkv, d, budget, sink, recent):
    c = Case(torch, kv, hq, hkv, d, [1, 0, 16, 17, 250, 64, 1000, 790], seed=budget + d)
    c.all_bounds()
    pages, counts = c.select(budget, sink=sink, recent=recent)
    want_pages, want_counts = plain_choice(c, budget, sink, recent)
    torch.cuda.synchronize()
    assert np.array_equal(counts.cpu().numpy(), want_counts)
    assert np.array_equal(pages.cpu().numpy(), want_pages)
    assert c.flags() == 0


@pytest.mark.parametrize("kv,hq,hkv,d", [("bf16", 28, 4, 128), ("fp8", 8, 1, 64), ("f32", 4, 4, 64)])
def test_choice_of_several_rows(torch, kv, hq, hkv, d):
    rows = [3, 0, 1, 5, 17, 0, 40, 2]
    c = Case(torch, kv, hq, hkv, d, [300, 0, 1, 5, 400, 31, 700, 33], rows, seed=7, max_batch=300)
    c.all_bounds()
    pages, counts = c.select(12, sink=1, recent=2)
    want_pages, want_counts = plain_choice(c, 12, 1, 2)
    torch.cuda.synchronize()
    assert np.array_equal(counts.cpu().numpy(), want_counts) and np.array_equal(pages.cpu().numpy(), want_pages)
    assert c.flags() == 0


@pytest.mark.parametrize("n,max_pages,rows,hkv", [(5000, 5000, 1, 1), (700, 9000, 1, 1), (2600, 2600, 3, 1), (20000, 32768, 1, 1),
                                                  (1500, 1500, 20, 8), (2600, 2600, 18, 8), (5000, 5000, 17, 8), (300, 9000, 17, 8)])
def test_choice_of_long_rows(torch, n, max_pages, rows, hkv):
    """Cut over several workgroups, or several rows to one; tables beyond what the small form holds."""
    c = Case(torch, "bf16", 4 * hkv, hkv, 64, [PAGE * n - 3, 900], [rows, rows], seed=n, extra_pages=max_pages - n)
    g = torch.Generator("cuda").manual_seed(1)
    c.bounds.copy_(torch.randint(-127, 128, c.bounds.shape, device="cuda", generator=g, dtype=torch.int8).sort(dim=2).values)
    c.bscale.copy_(torch.rand(c.bscale.shape, device="cuda", generator=g))
    for budget in (64, 1000):
        pages, counts = c.select(budget, sink=2, recent=3)
        want_pages, want_counts = plain_choice(c, budget, 2, 3)
        torch.cuda.synchronize()
        assert np.array_equal(counts.cpu().numpy(), want_counts) and np.array_equal(pages.cpu().numpy(), want_pages)
    assert c.flags() == 0


@pytest.mark.parametrize("outliers", [0, 3], ids=["even", "outliers"])
@pytest.mark.parametrize("kv,hq,hkv,d", LAYOUTS)
def test_choice_against_the_score_of_unrounded_queries(torch, kv, hq, hkv, d, outliers):
    """The definition that the 8-bit query stands for, in float64: S = max_i s sum_d max(q_d lo_d, q_d hi_d)
    is no less than q . k of any of the page's keys, and no page that is left out beats a chosen one
    by more than the roundings allow.
      Bounds: s lo <= k <= s hi up to 128 2^-22 s (test_bounds), so S >= q . k - 128 2^-22 s sum |q_d|.
      Choice: rint(q / sq) is within 1/2 of the fp32 quotient, and that within 127 2^-24 of q / sq; with m_d
    = max(|lo_d|, |hi_d|) a head's score is off by E = s sq (1/2 + 2^-16) sum m_d and by two fp32
    products, 2^-22 of it.  So for a page a that is chosen and b that is not, S_a + E_a >= S_b - E_b."""
    c = Case(torch, kv, hq, hkv, d, [1500, 16, 900, 2000], [2, 1, 3, 1], seed=36)
    if outliers:   # a few channels of much larger keys, as caches have: they coarsen the others' bounds
        for t in (c.k,):
            big = torch.randperm(d, device="cuda", generator=c.gen)[:outliers]
            if kv == "fp8":
                x = t.float()
                x[..., [i for i in range(d) if i not in set(big.tolist())]] /= 24
                t.copy_(x.to(t.dtype))
            else:
                t[..., big] *= 24
    c.all_bounds()
    budget = 12
    pages, counts = c.select(budget, sink=1, recent=2)
    chosen = pages.cpu().numpy()
    cut = 0
    for r, b, L in c.row_list():
        n = -(-L // PAGE)
        page = torch.from_numpy(c.table[b, :n].astype(np.int64)).cuda()
        for g in range(hkv):
            q = c.q[r, [h for h in range(hq) if c.kv_of[h] == g]].double()                     # [G][d]
            lo, hi = c.bounds[page, g, 0].double(), c.bounds[page, g, 1].double()              # [n][d]
            s = c.bscale[page, g].double()
            score = s * torch.maximum(q[:, None] * lo, q[:, None] * hi).sum(-1)                # [G][n]
            for j in range(n):
                k = c.values(c.k, c.ks, int(page[j]))[g, :min(PAGE, L - j * PAGE)].double()    # [tokens][d]
                most = (q[:, None] * k).sum(-1).amax(-1)
                assert bool((score[:, j] >= most - 128 * 2.0 ** -22 * s[j] * q.abs().sum(-1)).all())
            if n <= budget:
                continue
            cut += 1
            sq = q.abs().amax(-1, keepdim=True) / 127
            m = torch.maximum(lo.abs(), hi.abs()).sum(-1)
            err = s * sq * (0.5 + 2.0 ** -16) * m
            err = (err + 2.0 ** -22 * (score.abs() + err)).amax(0)
            x, took = score.amax(0), torch.zeros(n, dtype=torch.bool, device="cuda")
            took[torch.from_numpy(chosen[r, g].astype(np.int64)).cuda()] = True
            rest = torch.arange(n, device="cuda")
            rest = (rest >= 1) & (rest < n - 2)
            worst, best = (x + err)[rest & took].amin(), (x - err)[rest & ~took].amax()
            assert bool(worst >= best), (r, g, float(worst), float(best))
    assert cut > 0 and c.flags() == 0


def test_choice_with_ties_and_odd_values(torch):
    """Equal scores go to the lower page, zeros of both signs are equal; pages that are not
    finite come first, pages outside the pool last; a query that is not finite says nothing."""
    c = Case(torch, "bf16", 8, 2, 64, [PAGE * 50, PAGE * 50, PAGE * 50, PAGE * 50], seed=9)
    c.all_bounds()
    same = c.table[0, 5:40:3]
    c.bounds[torch.from_numpy(same.astype(np.int64)).cuda()] = c.bounds[int(same[0])].clone()
    c.bscale[torch.from_numpy(same.astype(np.int64)).cuda()] = c.bscale[int(same[0])].clone()
    c.bounds[torch.from_numpy(c.table[1].astype(np.int64)).cuda()] = 0           # scores of 0 and -0
    c.bscale[int(c.table[2, 20]), 0] = math.inf
    c.bscale[int(c.table[2, 31]), 0] = math.nan
    c.q[2, 0, 3], c.q[3, 5, 0] = math.nan, math.inf
    c.block_table[3, 7] = c.npages
    c.block_table[3, 8] = -1
    for budget in (8, 13, 20, 49):
        pages, counts = c.select(budget, sink=1, recent=2)
        want_pages, want_counts = plain_choice(c, budget, 1, 2)
        torch.cuda.synchronize()
        assert np.array_equal(counts.cpu().numpy(), want_counts) and np.array_equal(pages.cpu().numpy(), want_pages)
    assert {20, 31} <= set(c.select(5, sink=0, recent=1)[0][2, 0].tolist())
    assert c.flags() == 1


def test_choice_by_tiny_queries(torch):
    """Queries whose scale is subnormal: their quotients end at 127."""
    c = Case(torch, "f32", 2, 2, 64, [PAGE * 60, PAGE * 70], seed=30)
    c.all_bounds()
    c.q[0] = torch.randint(-190, 191, c.q[0].shape, device="cuda").float() * 2.0 ** -149
    c.q[1, 0] = 0.0
    pages, counts = c.select(9)
    want_pages, want_counts = plain_choice(c, 9, 1, 1)
    assert np.array_equal(counts.cpu().numpy(), want_counts) and np.array_equal(pages.cpu().numpy(), want_pages)


def test_choice_head_map_and_outputs(torch):
    head_map = [2, 0, 1, 1, 0, 2, 2, 0, 1]
    c = Case(torch, "bf16", 9, 3, 128, [900, 40], seed=10, head_map=head_map)
    c.all_bounds()
    out = (torch.full((2, 3, 7), 99, dtype=torch.int32, device="cuda"), torch.full((2, 3), 99, dtype=torch.int32, device="cuda"))
    got = c.select(7, sink=1, recent=1, out=out)
    want_pages, want_counts = plain_choice(c, 7, 1, 1)
    assert got[0] is out[0] and got[1] is out[1]
    assert np.array_equal(out[0].cpu().numpy(), want_pages) and np.array_equal(out[1].cpu().numpy(), want_counts)
    o, tol, _ = c.want(lambda r, g, L: want_pages[r, g, :want_counts[r, g]])
    c.check(c.attend(*out), o, tol)
    o, tol, parts = c.want(lambda r, g, L: range(-(-L // PAGE)))
    w0 = torch.zeros((2, c.mp), device="cuda")
    w = w0.clone()
    c.check(c.weigh(w), o, tol)
    want, wtol = expect_weights(c, parts, w0, 1.0)
    assert bool(((w.double() - want).abs() <= wtol + 1e-30).all())


def test_rows_of_no_sequence(torch):
    """Rows before the first and behind the last sequence's, and of a sequence whose offsets
    disagree, are left as they were, by the choice and by both attentions."""
    c = Case(torch, "bf16", 8, 2, 64, [100, 50, 80], [2, 3, 4], seed=11)
    c.all_bounds()
    c.q = torch.cat([c.q, c.q])[:14].contiguous()
    for starts, live, flags in (([2, 4, 7, 11], set(range(2, 11)), 0), ([0, 2, 20, 11], {0, 1}, 2), ([-3, 2, 5, 9], set(range(2, 9)), 2)):
        qs = torch.tensor(starts, dtype=torch.int32, device="cuda")
        out = (torch.full((14, 2, 4), 99, dtype=torch.int32, device="cuda"), torch.full((14, 2), 99, dtype=torch.int32, device="cuda"))
        c.q_start = qs
        c.select(4, out=out)
        assert c.flags() == flags
        written = {r for r in range(14) if bool((out[1][r] != 99).all())}
        assert written == live and all(bool((out[0][r] == 99).all()) for r in range(14) if r not in live), starts
        lists = out[0].clamp(-1, 3), out[1].clamp(0, 4)
        o = torch.full((14, 8, 64), 7.0, device="cuda")
        c.attend(*lists, out=o)
        assert {r for r in range(14) if not bool((o[r] == 7).all())} == live
        w = torch.zeros((3, c.mp), device="cuda")
        o.fill_(7.0)
        ws = torch.zeros(c.layer.weighed_workspace(14, "cuda").numel(), dtype=torch.uint8, device="cuda")
        c.weigh(w, out=o, workspace=ws)
        assert {r for r in range(14) if not bool((o[r] == 7).all())} == live and c.flags(ws) == flags
        c.layer._ws.clear()
    # More rows than tokens: those before token 0 choose nothing and give zeros.
    c = Case(torch, "bf16", 8, 2, 64, [2, 50], [5, 1], seed=12)
    c.all_bounds()
    pages, counts = c.select(4)
    assert counts[:, 0].tolist() == [0, 0, 0, 1, 1, 4] and bool((pages[:3] == -1).all()) and c.flags() == 2
    o = c.attend(pages, counts)
    assert bool((o[:3] == 0).all()) and bool((o[3:] != 0).any(-1).all())


def owners(starts, n):
    """The sequence of every row (-1: none): the one that a search of 64 entries a step ends at, if its
    offsets agree and the row lies between them."""
    got = []
    for r in range(n):
        lo, hi = 0, len(starts)
        while lo < hi:
            step = -(-(hi - lo) // 64)
            lo += step * sum(starts[at] <= r for at in range(lo + step - 1, min(hi, lo + 64 * step), step))
            hi = min(hi, lo + step - 1)
        got.append(lo - 1 if 0 < lo < len(starts) and 0 <= starts[lo - 1] <= r < starts[lo] <= n else -1)
    return got


CLAIMED = [[0, 5, 3, 9], [0, 5, 0, 9], [0, 9, 2, 4, 9], [0, 8, 3, 7], [2, 4, 7, 11], [0, 2, 20, 11], [-3, 2, 5, 9], [70, 40, 5],
           [600, 520, 300]]
CLAIMED_IDS = ["overlap", "whole", "inside", "hole", "between", "beyond", "before", "70", "600"]


def claimed_case(torch, starts, kv):
    """Offsets of which some run backwards, so that two sequences claim the same rows, or leave the
    call's rows: the rows as they are taken (owners), those of no sequence, and the flags."""
    n = 12
    if starts[0] > 60:   # one row a sequence, but the entry of one goes back
        n, (batch, b, to) = starts[0], starts
        starts = list(range(batch + 1))
        starts[b] = to
    B = len(starts) - 1
    rng = np.random.default_rng(B)
    lens = [400, 50, 90, 130] if B < 5 else list(rng.integers(40, 100, size=B))
    c = Case(torch, kv, 4, 2, 64, lens[:B], [n] + [0] * (B - 1), seed=33, extra_pages=1)
    own = owners(starts, n)
    c.q_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    c.rows = np.bincount([b for b in own if b >= 0], minlength=B)
    rows = [(r, b, int(c.lens[b]) - (starts[b + 1] - 1 - r)) for r, b in enumerate(own) if b >= 0]
    c.row_list = lambda: rows
    c.all_bounds()
    agree = all(0 <= a <= b <= n for a, b in zip(starts, starts[1:]))
    return c, [r for r, b in enumerate(own) if b >= 0], [r for r, b in enumerate(own) if b < 0], 0 if agree else 2


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("starts", CLAIMED, ids=CLAIMED_IDS)
def test_choice_of_rows_that_two_sequences_claim(torch, starts, kv):
    """The choice and the attention over it take a row as the same sequence's, and say so."""
    c, mine, free, flags = claimed_case(torch, starts, kv)
    n = len(c.q)
    out = (torch.full((n, 2, 3), 99, dtype=torch.int32, device="cuda"), torch.full((n, 2), 99, dtype=torch.int32, device="cuda"))
    c.select(3, out=out)
    assert c.flags() == flags
    c.layer._ws.clear()   # (flags stay)
    pages, counts = plain_choice(c, 3, 1, 1)
    assert np.array_equal(out[0].cpu().numpy()[mine], pages[mine]) and np.array_equal(out[1].cpu().numpy()[mine], counts[mine])
    assert bool((out[0][free] == 99).all()) and bool((out[1][free] == 99).all())
    o, tol, _ = c.want(lambda r, g, L: pages[r, g, :counts[r, g]])
    got = torch.full((n, 4, 64), 7.0, device="cuda")
    c.attend(torch.from_numpy(pages).cuda(), torch.from_numpy(counts).cuda(), out=got)
    assert c.flags() == flags and bool((got[free] == 7).all())
    c.check(got[mine], o[mine], tol[mine])


# ---------------------------------------------------------------- attention over the chosen pages

def random_lists(c, budget, seed, full=False):
    rng = np.random.default_rng(seed)
    pages = rng.integers(-5, 1000, size=(c.q.shape[0], c.hkv, budget)).astype(np.int32)   # beyond the counts: anything
    counts = np.zeros((c.q.shape[0], c.hkv), np.int32)
    for r, _, L in c.row_list():
        n = max(-(-L // PAGE), 0)
        for g in range(c.hkv):
            m = min(n, budget) if full else int(rng.integers(0, min(n, budget) + 1))
            pages[r, g, :m] = rng.permutation(n)[:m] if rng.random() < 0.5 else np.sort(rng.permutation(n)[:m])
            counts[r, g] = m
    return pages, counts


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("ranges", [0, 7, 300])
@pytest.mark.parametrize("kv,hq,hkv,d", LAYOUTS)
def test_selected(torch, kv, hq, hkv, d, ranges, out):
    if kv == "f32" and out == "bf16":
        pytest.skip("f32 layers give f32")
    c = Case(torch, kv, hq, hkv, d, [1, 0, 16, 17, 250, 1500, 33, 640], seed=hq + d, out=out, ranges=ranges)
    for budget, full in ((1, True), (9, False), (40, False), (120, True)):
        pages, counts = random_lists(c, budget, budget, full)
        got = c.attend(torch.from_numpy(pages).cuda(), torch.from_numpy(counts).cuda())
        o, tol, _ = c.want(lambda r, g, L: pages[r, g, :counts[r, g]])
        torch.cuda.synchronize()
        c.check(got, o, tol, out)
    assert c.flags() == 0


@pytest.mark.parametrize("kv,hq,hkv,d,layout", [("bf16", 28, 4, 128, "slot"), ("fp8", 40, 8, 64, "head"), ("f32", 2, 1, 64, "slot")])
def test_selected_of_several_rows(torch, kv, hq, hkv, d, layout):
    rows = [3, 0, 1, 5, 17, 0, 30, 2]
    c = Case(torch, kv, hq, hkv, d, [300, 0, 1, 5, 400, 31, 700, 33], rows, seed=7, layout=layout, max_batch=9)
    pages, counts = random_lists(c, 11, 3)
    got = c.attend(torch.from_numpy(pages).cuda(), torch.from_numpy(counts).cuda())
    o, tol, _ = c.want(lambda r, g, L: pages[r, g, :counts[r, g]])
    torch.cuda.synchronize()
    c.check(got, o, tol)
    assert c.flags() == 0


def test_selected_many_rows(torch):
    """As many rows as a call may have, of two sequences."""
    c = Case(torch, "bf16", 4, 2, 64, [2500, 2000], [2300, 1796], seed=8)
    pages, counts = random_lists(c, 3, 4)
    got = c.attend(torch.from_numpy(pages).cuda(), torch.from_numpy(counts).cuda())
    torch.cuda.synchronize()
    full = c.attend(torch.from_numpy(pages).cuda(), torch.from_numpy(counts).cuda())
    assert torch.equal(got, full)
    keep = np.random.default_rng(0).permutation(4096)[:60]
    rows = [x for x in c.row_list() if x[0] in set(keep.tolist())]
    c.row_list = lambda: rows
    o, tol, _ = c.want(lambda r, g, L: pages[r, g, :counts[r, g]])
    pick = torch.tensor(sorted(keep.tolist()), device="cuda")
    c.check(got[pick], o[pick], tol[pick])
    assert c.flags() == 0


def test_selected_everything_is_the_plain_attention(torch):
    for kv, hq, hkv, d in LAYOUTS:
        c = Case(torch, kv, hq, hkv, d, [1, 0, 100, 700, 3000], seed=5)
        n = int(c.used.max())
        pages = torch.arange(n, dtype=torch.int32, device="cuda").expand(5, hkv, n).contiguous()
        counts = torch.from_numpy(np.repeat(c.used[:, None], hkv, 1).astype(np.int32)).cuda()
        plain = c.layer(c.q, *c.cache(), **c.scales())
        o, tol, _ = c.want(lambda r, g, L: range(-(-L // PAGE)))
        got = c.attend(pages, counts)
        c.check(got, o, tol)
        # The plain call rounds probabilities to one bf16 value where its streams are short: 2^-8
        # of A, and |o| <= A <= max |v|.
        assert bool(((got - plain).abs() <= 2.0 ** -8 * float(c.v.float().nan_to_num().abs().max() if c.vs is None else 4 * 448 * c.vs.max())
                     + tol).all())


def test_selected_twice_the_same_page_and_bad_entries(torch):
    c = Case(torch, "bf16", 8, 2, 64, [200, 200, 200, 200], seed=6)
    pages = torch.tensor([[3, 3, 7, 1], [0, 1, 2, 3], [5, -1, 6, 0], [2, 13, 4, 1 << 30]], dtype=torch.int32, device="cuda")
    pages = pages[:, None].expand(4, 2, 4).contiguous()
    counts = torch.tensor([4, -5, 4, 1 << 20], dtype=torch.int32, device="cuda")[:, None].expand(4, 2).contiguous()
    got = c.attend(pages, counts)
    seen = {0: [3, 3, 7, 1], 1: [], 2: [5, 6, 0], 3: [2, 4]}
    o, tol, _ = c.want(lambda r, g, L: seen[r])
    c.check(got, o, tol)
    assert c.flags() == 1 and bool((got[1] == 0).all())


@pytest.mark.parametrize("ranges", [0, 3])
@pytest.mark.parametrize("bad", [-1, -2 ** 31, 2 ** 31 - 1])
def test_listed_pages_outside_the_pool(torch, bad, ranges):
    c = Case(torch, "bf16", 8, 2, 64, [200, 330], seed=31, ranges=ranges)
    pages = torch.tensor([[3, 7, 1], [0, 5, 2]], dtype=torch.int32, device="cuda")[:, None].expand(2, 2, 3).contiguous()
    counts = torch.tensor([2, 3], dtype=torch.int32, device="cuda")[:, None].expand(2, 2).contiguous()
    c.block_table[0, 1] = bad     # beyond the count
    c.attend(pages, counts)
    assert c.flags() == 0
    c.block_table[1, 5] = bad
    got = c.attend(pages, counts)
    assert c.flags() == 1
    o, tol, _ = c.want(lambda r, g, L: [[3, 7], [0, 2]][r])
    c.check(got, o, tol)


def test_selected_keys_that_are_not_listed_have_no_part(torch):
    """NaN and infinities in every other page, and behind a row's own position."""
    for kv in ("bf16", "fp8", "f32"):
        c = Case(torch, kv, 4, 2, 64, [330, 150], [3, 2], seed=13)
        pages, counts = random_lists(c, 6, 1)
        free = next(x for x in range(c.npages - 1, -1, -1) if x not in set(c.table.flatten().tolist()))
        for t in (c.k, c.v, c.ks, c.vs):   # page 0 is nobody's
            if t is not None:
                t.view(raw_type(torch, kv) if t.dim() == 4 else t.dtype)[free] = \
                    t.view(raw_type(torch, kv) if t.dim() == 4 else t.dtype)[0].clone()
        c.table[c.table == 0] = free
        c.block_table.copy_(torch.from_numpy(c.table))
        for t in (c.ks, c.vs):
            if t is not None:
                t[0] = math.nan
        listed = {(b, int(j)) for r, b, _ in c.row_list() for g in range(2) for j in pages[r, g, :counts[r, g]]}
        for b in range(2):
            for j in range(c.used[b]):
                if (b, j) not in listed:
                    for t in (c.k, c.v):
                        t.view(raw_type(torch, kv))[int(c.table[b, j])] = NAN[kv]
                    for t in (c.ks, c.vs):
                        if t is not None:
                            t[int(c.table[b, j])] = math.nan
        got = c.attend(torch.from_numpy(pages).cuda(), torch.from_numpy(counts).cuda())
        assert bool(got.isfinite().all())
        # The last token of each sequence is seen by its last row alone.
        for b in range(2):
            L = int(c.lens[b])
            for t in (c.k, c.v):
                t.view(raw_type(torch, kv))[int(c.table[b, (L - 1) // PAGE]), :, (L - 1) % PAGE] = NAN[kv]
        again = c.attend(torch.from_numpy(pages).cuda(), torch.from_numpy(counts).cuda())
        for r, b, L in c.row_list():
            if L < c.lens[b]:
                assert torch.equal(again[r], got[r])


# ---------------------------------------------------------------- weights

def expect_weights(c, parts, w0, decay):
    torch = c.torch
    want, tol = w0.double().clone(), torch.zeros(w0.shape, dtype=torch.float64, device="cuda")
    for b in range(len(c.lens)):
        n = int(c.used[b])
        if n == 0 or c.rows[b] == 0:
            continue
        got = torch.zeros(n, dtype=torch.float64, device="cuda")
        off = torch.zeros_like(got)
        for r, bb, L in c.row_list():
            if bb != b or L <= 0:
                continue
            p, f = parts[r]
            pad = lambda x: torch.nn.functional.pad(x.sum(0), (0, n * PAGE - L)).view(n, PAGE).sum(1)   # noqa: E731
            got += pad(p)
            off += pad(p * f)
        want[b, :n] = (w0[b, :n].double() * decay if decay else 0.0) + got
        tol[b, :n] = off + (int(c.rows[b]) * c.hq + 2) * 2.0 ** -24 * want[b, :n]
    return want, tol


@pytest.mark.parametrize("ranges", [0, 5, 200])
@pytest.mark.parametrize("kv,hq,hkv,d", LAYOUTS)
def test_weighed(torch, kv, hq, hkv, d, ranges):
    c = Case(torch, kv, hq, hkv, d, [1, 0, 16, 17, 250, 1500, 33, 640], seed=hq, ranges=ranges, extra_pages=3)
    o, tol, parts = c.want(lambda r, g, L: range(-(-L // PAGE)))
    for decay in (1.0, 0.9, 0.0):
        w0 = torch.rand((8, c.mp), device="cuda", generator=c.gen)
        if decay == 0.0:
            w0[:] = math.nan   # not read
        w = w0.clone()
        got = c.weigh(w, decay=decay)
        torch.cuda.synchronize()
        c.check(got, o, tol)
        want, wtol = expect_weights(c, parts, w0, decay)
        for b in range(8):
            n = int(c.used[b])
            assert torch.equal(w[b, n:].isnan(), w0[b, n:].isnan()) and torch.equal(w[b, n:].nan_to_num(), w0[b, n:].nan_to_num())
            bad = ~((w[b, :n].double() - want[b, :n]).abs() <= wtol[b, :n] + 1e-30)
            assert not bad.any(), (b, float(((w[b, :n] - want[b, :n]).abs() / wtol[b, :n]).max()))
    assert c.flags(c.layer.weighed_workspace(8, "cuda")) == 0


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("starts", CLAIMED, ids=CLAIMED_IDS)
def test_weights_of_rows_that_two_sequences_claim(torch, starts, kv):
    """Weights of the rows as the attention takes them: a sequence without rows of its own keeps its
    weights, and nothing that an earlier call left in the workspace gets into any."""
    c, mine, free, flags = claimed_case(torch, starts, kv)
    n = len(c.q)
    o, tol, parts = c.want(lambda r, g, L: range(-(-L // PAGE)))
    ws = c.layer.weighed_workspace(n, "cuda")
    at = -ws.data_ptr() % 256 + c.layer.workspace_bytes
    ws[at:at + (ws.numel() - at) // 4 * 4].view(torch.float32).fill_(100.0)   # what an earlier call may leave
    w0 = torch.rand((len(c.lens), c.mp), device="cuda", generator=c.gen)
    w = w0.clone()
    got = torch.full((n, 4, 64), 7.0, device="cuda")
    c.weigh(w, decay=0.5, out=got)
    assert c.flags(ws) == flags and bool((got[free] == 7).all())
    c.check(got[mine], o[mine], tol[mine])
    want, wtol = expect_weights(c, parts, w0, 0.5)
    for b in range(len(c.lens)):
        assert bool(((w[b].double() - want[b]).abs() <= wtol[b] + 1e-30).all()), (b, w[b].tolist(), want[b].tolist())


@pytest.mark.parametrize("kv,hq,hkv,d", [("bf16", 28, 4, 128), ("fp8", 8, 1, 64), ("f32", 4, 4, 64)])
def test_weighed_several_rows(torch, kv, hq, hkv, d):
    rows = [3, 0, 1, 5, 17, 0, 30, 2]
    c = Case(torch, kv, hq, hkv, d, [300, 0, 1, 5, 400, 31, 700, 33], rows, seed=17, max_batch=9)
    o, tol, parts = c.want(lambda r, g, L: range(-(-L // PAGE)))
    w0 = torch.rand((8, c.mp), device="cuda", generator=c.gen)
    w = w0.clone()
    got = c.weigh(w, decay=0.5)
    torch.cuda.synchronize()
    c.check(got, o, tol)
    want, wtol = expect_weights(c, parts, w0, 0.5)
    assert bool(((w.double() - want).abs() <= wtol + 1e-30).all())
    assert torch.equal(w[1], w0[1]) and torch.equal(w[5], w0[5])   # no rows, no change
    # A sequence whose weights add up to its rows' heads.
    w.zero_()
    c.weigh(w)
    total = w.double().sum(1).cpu().numpy()
    assert np.allclose(total, np.where(c.lens > 0, c.rows * hq, 0), rtol=1e-5)


def test_weighed_of_keys_that_are_not_finite(torch):
    """An infinite score takes the row's whole softmax to NaN, as in plain attention; other
    sequences' weights stay clean."""
    c = Case(torch, "bf16", 4, 2, 64, [100, 100], seed=18)
    c.k[int(c.table[0, 2]), 0, 3, 5] = math.nan
    w = torch.zeros((2, c.mp), device="cuda")
    got = c.weigh(w)
    plain = c.layer(c.q, *c.cache())
    assert torch.equal(got.isnan(), plain.isnan()) and bool(w[1].isfinite().all())
    assert abs(float(w[1].sum()) - 4) < 1e-4


def test_weighed_repeats_to_the_bit(torch):
    c = Case(torch, "fp8", 40, 8, 128, [3000, 70, 1200, 5], seed=19)
    runs = []
    for _ in range(4):
        w = torch.zeros((4, c.mp), device="cuda")
        runs.append((c.weigh(w).clone(), w))
    assert all(torch.equal(a, runs[0][0]) and torch.equal(b, runs[0][1]) for a, b in runs)


# ---------------------------------------------------------------- eviction

class Pool:
    def __init__(self, torch, pages, mp=64, spare=5, seed=0, shared=0):
        from paper_2607_09207_amd import DecodeAttention
        rng = np.random.default_rng(seed)
        B = len(pages)
        self.torch = torch
        self.lens = np.array([0 if n == 0 else (n - 1) * PAGE + rng.integers(1, PAGE + 1) for n in pages], np.int32)
        self.np = shared + sum(max(n - shared, 0) for n in pages) + spare
        perm = rng.permutation(self.np)
        self.table = np.full((B, mp), -1, np.int32)
        at = shared
        for b, n in enumerate(pages):
            self.table[b, :min(n, shared)] = perm[:min(n, shared)]
            own = max(n - shared, 0)
            self.table[b, shared:shared + own] = perm[at:at + own]
            at += own
        self.refs = np.zeros(self.np, np.int32)
        for b, n in enumerate(pages):
            np.add.at(self.refs, self.table[b, :n], 1)
        self.w = (rng.random((B, mp)) * 10).astype(np.float32)
        self.layer = DecodeAttention(8, 2, 64, B, mp)
        self.dev = [torch.from_numpy(x.copy()).cuda() for x in (self.refs, self.table, self.lens, self.w)]

    def evict(self, budget, **kw):
        refs, table, lens, w = self.dev
        return self.layer.page_evict(refs, table, lens, w, budget, **kw)

    def expect(self, budget, sink=1, recent=1):
        refs, table, lens, w = (x.copy() for x in (self.refs, self.table, self.lens, self.w))
        dropped = np.zeros(len(lens), np.int32)
        for b, L in enumerate(lens):
            n = -(-int(L) // PAGE)
            if n <= budget:
                continue
            key = np.where(np.isnan(w[b]), np.inf, w[b])
            rest = sorted(range(sink, n - recent), key=lambda j: (-key[j], not np.isnan(w[b, j]), j))
            keep = sorted(list(range(sink)) + rest[:budget - sink - recent] + list(range(n - recent, n)))
            for j in set(range(n)) - set(keep):
                refs[table[b, j]] -= 1
            table[b, :budget], w[b, :budget] = table[b, keep], w[b, keep]
            w[b, budget:n] = 0
            lens[b] -= PAGE * (n - budget)
            dropped[b] = n - budget
        return refs, table, lens, w, dropped

    def check(self, dropped, want):
        self.torch.cuda.synchronize()
        for name, a, b in zip(("refs", "table", "lens", "weights", "dropped"), self.dev + [dropped], want):
            assert np.array_equal(a.cpu().numpy(), b, equal_nan=name == "weights"), name


@pytest.mark.parametrize("budget,sink,recent", [(1, 0, 1), (8, 1, 2), (8, 4, 4), (20, 0, 1), (63, 2, 3)])
def test_evict(torch, budget, sink, recent):
    for seed, shared in ((0, 0), (1, 6), (2, 30)):
        s = Pool(torch, [0, 1, 7, 8, 9, 20, 21, 64, 40, 33], seed=seed, shared=shared)
        want = s.expect(budget, sink, recent)
        s.check(s.evict(budget, sink=sink, recent=recent), want)
        assert s.layer.page_flags(s.np, "cuda") == 0


@pytest.mark.parametrize("n,mp", [(1500, 1500), (700, 9000), (12000, 32768)])
def test_evict_long_rows(torch, n, mp):
    s = Pool(torch, [n, 3, n - 1], mp=mp, seed=5)
    s.w[0] = np.round(s.w[0])   # many equal ones
    s.dev[3].copy_(torch.from_numpy(s.w))
    for budget in (600, 513):
        want = s.expect(budget, 4, 100)
        s.check(s.evict(budget, sink=4, recent=100), want)
        s.refs, s.table, s.lens, s.w = want[:4]


def test_evict_odd_weights(torch):
    """Ties to the lower page, zeros of both signs alike, NaN and infinities heaviest."""
    s = Pool(torch, [40, 40, 40], seed=6)
    s.w[0] = 0.0
    s.w[0, ::2] = -0.0
    s.w[1, 5], s.w[1, 9], s.w[1, 11], s.w[1, 30] = math.nan, math.inf, -math.inf, math.nan
    s.w[2] = -s.w[2]
    s.dev[3].copy_(torch.from_numpy(s.w))
    want = s.expect(10, 1, 2)
    s.check(s.evict(10, sink=1, recent=2), want)


def test_evict_wrong_state(torch):
    """A length out of range leaves its row; dropped ids outside the pool, and pages that nobody
    holds, are flagged and change no count."""
    s = Pool(torch, [20, 20, 20], mp=20, seed=7)
    s.lens[0] = 20 * PAGE + 1
    s.w[1, :10], s.w[2, :10] = 0, 0   # of these go: all but the first
    s.table[1, 3] = s.np + 5
    s.table[2, 4] = -1
    s.refs[s.table[1, 2]] = 0
    for i, x in enumerate((s.refs, s.table, s.lens, s.w)):
        s.dev[i].copy_(torch.from_numpy(x))
    keep = s.refs.copy()
    dropped = s.evict(11, sink=1, recent=10)
    torch.cuda.synchronize()
    assert dropped.tolist() == [0, 9, 9] and s.layer.page_flags(s.np, "cuda") == 3
    for b in (1, 2):
        for j in range(1, 10):
            if 0 <= s.table[b, j] < s.np and keep[s.table[b, j]] > 0:
                keep[s.table[b, j]] -= 1
    assert np.array_equal(s.dev[0].cpu().numpy(), keep)
    assert np.array_equal(s.dev[1].cpu().numpy()[0], s.table[0]) and s.dev[2].tolist()[0] == 20 * PAGE + 1


def test_growth_and_eviction_in_a_pool_that_runs_dry(torch):
    """A shared page that some rows drop stays taken, so a pool with room for one page a row runs
    short: rows that get none keep what they have, and are not evicted."""
    s = Pool(torch, [12] * 24, mp=16, spare=30, seed=12, shared=8)
    add = torch.full((24,), PAGE, dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(13)
    short = 0
    for _ in range(8):
        s.w[:, :12] = rng.random((24, 12))   # other pages go from every row
        s.dev[3].copy_(torch.from_numpy(s.w))
        free = list(np.flatnonzero(s.refs == 0))
        served = np.arange(24) < len(free)   # a page of tokens more needs a page
        for b in np.flatnonzero(served):
            s.refs[free[b]], s.table[b, -(-int(s.lens[b]) // PAGE)] = 1, free[b]
            s.lens[b] += PAGE
        short += int((~served).sum())
        s.layer.page_grow(*s.dev[:3], add)
        want = s.expect(12, 2, 2)
        s.check(s.evict(12, sink=2, recent=2), want)
        assert np.array_equal(want[4], served.astype(np.int32))
        assert s.layer.page_flags(s.np, "cuda") == (0 if served.all() else 16)   # (read and cleared)
        s.refs, s.table, s.lens, s.w = want[:4]
    assert short > 0


# ---------------------------------------------------------------- refusals

def test_refusals(torch):
    from paper_2607_09207_amd import RldaError
    c = Case(torch, "fp8", 8, 2, 64, [100, 50], seed=20)
    c.all_bounds()
    pages, counts = c.select(4)
    w = torch.zeros((2, c.mp), device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    L = c.layer
    bounds = lambda **kw: L.page_bounds(**dict(dict(k_cache=c.k, block_table=c.block_table, seq_lens=c.seq_lens, bounds=c.bounds,   # noqa: E731
                                                    bound_scale=c.bscale, k_scale=c.ks), **kw))
    choose = lambda **kw: L.select_pages(**dict(dict(q=c.q, bounds=c.bounds, bound_scale=c.bscale, block_table=c.block_table,   # noqa: E731
                                                     seq_lens=c.seq_lens, budget=4), **kw))
    attend = lambda **kw: L.selected(**dict(dict(q=c.q, k_cache=c.k, v_cache=c.v, block_table=c.block_table, seq_lens=c.seq_lens,   # noqa: E731
                                                 pages=pages, counts=counts, **c.scales()), **kw))
    weigh = lambda **kw: L.weighed(**dict(dict(q=c.q, k_cache=c.k, v_cache=c.v, block_table=c.block_table, seq_lens=c.seq_lens,   # noqa: E731
                                               weights=w, **c.scales()), **kw))
    short = torch.zeros((2,), **i32)
    for call, kws in (
            (bounds, [dict(k_scale=None), dict(bounds=None), dict(bounds=c.bounds[:-1]), dict(bounds=c.bounds.to(torch.uint8)),
                      dict(bounds=c.bounds[:, :, :, :32]), dict(bound_scale=c.bscale.double()), dict(bound_scale=c.bscale.t()),
                      dict(first=torch.zeros(3, **i32)), dict(first=torch.zeros(2, device="cuda")), dict(k_cache=c.k.cpu()),
                      dict(seq_lens=c.seq_lens.long()), dict(workspace=torch.zeros(100, dtype=torch.uint8, device="cuda"))]),
            (choose, [dict(budget=0), dict(budget=1, sink=1, recent=1), dict(sink=-1), dict(recent=0), dict(budget=4.5), dict(budget=2 ** 31),
                      dict(q=c.q.float()), dict(q=c.q[:1]), dict(q=c.q.detach().requires_grad_()), dict(q=c.q.cpu()), dict(bounds=None),
                      dict(bound_scale=None), dict(out=(pages,)), dict(out=(pages[:1], counts)), dict(q_start=torch.zeros((2, 2), **i32)),
                      dict(q_start=torch.zeros(0, **i32))]),
            (attend, [dict(pages=None), dict(counts=None), dict(pages=pages[:1]), dict(pages=pages.long()), dict(counts=counts[:, :1]),
                      dict(counts=short), dict(q=c.q.detach().requires_grad_()), dict(k_cache=None), dict(k_scale=None),
                      dict(out=torch.zeros(2, 8, 64, device="cuda", dtype=torch.bfloat16)), dict(pages=pages[:, :, :0])]),
            (weigh, [dict(weights=None), dict(weights=w[:1]), dict(weights=w.double()), dict(decay=-0.1), dict(decay=1.5),
                     dict(decay=math.nan), dict(weights=w.clone().requires_grad_()), dict(q=c.q.detach().requires_grad_()),
                     dict(workspace=L.workspace("cuda"))])):
        for kw in kws:
            with pytest.raises(RldaError):
                call(**kw)
                print(kw)
    s = Pool(torch, [9, 3], mp=16)
    refs, table, lens, weights = s.dev
    for a, kw in (((refs, table, lens, weights, 0), {}), ((refs, table, lens, weights, 4), dict(recent=0)),
                  ((refs, table, lens, weights[:1], 4), {}), ((refs, table, lens, None, 4), {}),
                  ((refs, table, lens, weights, 4), dict(dropped=torch.zeros(3, **i32))), ((refs, table, lens, weights, "4"), {}),
                  ((refs, table, lens, weights.clone().requires_grad_(), 4), {})):
        with pytest.raises(RldaError):
            s.layer.page_evict(*a, **kw)
    torch.cuda.synchronize()
    assert c.flags() == 0 and np.array_equal(table.cpu().numpy(), s.table)
    # Empty calls.
    e = Case(torch, "bf16", 8, 2, 64, [], max_batch=3)
    e.make_bounds()
    assert e.select(4)[0].shape == (0, 2, 4)
    assert e.attend(torch.zeros((0, 2, 4), **i32), torch.zeros((0, 2), **i32)).shape == (0, 8, 64)
    assert e.weigh(torch.zeros((0, e.mp), device="cuda")).shape == (0, 8, 64)


# ---------------------------------------------------------------- calls as they are used

@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
def test_native_and_python_paths_agree(torch, native):
    from paper_2607_09207_amd import _abi
    got = []
    for left in (True, False):
        c = Case(torch, "fp8", 8, 2, 64, [100, 500, 33], seed=21)
        c.layer.workspace("cuda")
        c.layer.weighed_workspace(3, "cuda")
        if left != native:
            c.layer._fast = _abi.LEFT_TO_PYTHON
        c.all_bounds()
        pages, counts = c.select(6)
        w = torch.zeros((3, c.mp), device="cuda")
        v = w._version
        got.append((c.bounds, c.bscale, pages, counts, c.attend(pages, counts), c.weigh(w), w))
        assert w._version == v + 1
        s = Pool(torch, [20, 9, 30], seed=1)
        s.layer.page_workspace(s.np, "cuda")
        if left != native:
            s.layer._fast = _abi.LEFT_TO_PYTHON
        got[-1] += (s.evict(8),) + tuple(s.dev)
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_graph(torch):
    """A step of all of them captured once and replayed, with eager calls of other sizes on the same
    workspaces between, gives what eager calls give."""
    c = Case(torch, "bf16", 28, 4, 128, [900, 2000, 64], seed=22, ranges=0)
    L = c.layer
    refs = torch.ones(c.npages, dtype=torch.int32, device="cuda")
    w = torch.zeros((3, c.mp), device="cuda")
    keep = [t.clone() for t in (c.block_table, c.seq_lens, refs)]

    def step():
        c.make_bounds()
        pages, counts = c.select(16, recent=2)
        o = c.attend(pages, counts)
        o2 = c.weigh(w, decay=0.5)
        dropped = L.page_evict(refs, c.block_table, c.seq_lens, w, 100, recent=2)
        return pages, counts, o, o2, dropped, w, refs, c.block_table, c.seq_lens

    def reset(i):
        for t, x in zip((c.block_table, c.seq_lens, refs), keep):
            t.copy_(x)
        w.zero_()
        c.q.copy_(torch.randn(c.q.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(i)))

    c.all_bounds()
    L.workspace("cuda"), L.weighed_workspace(3, "cuda"), L.page_workspace(c.npages, "cuda")
    reset(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    reset(0)
    with torch.cuda.graph(graph):
        held = step()
    for i in range(1, 6):
        reset(i)
        want = [t.clone() for t in step()]
        reset(i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b), i
        c.weigh(torch.zeros_like(w))
    assert c.flags() == 0


def test_two_graphs_on_one_workspace(torch):
    """Captured one after the other, replayed in turn with eager calls between."""
    c = Case(torch, "fp8", 8, 2, 64, [3000, 40, 700], seed=29)
    c.all_bounds()
    L = c.layer
    L.workspace("cuda"), L.weighed_workspace(3, "cuda")
    w = [torch.zeros((3, c.mp), device="cuda") for _ in range(2)]
    qs = [c.q, (c.q.float() * -0.7 + 0.1).to(c.q.dtype)]

    def step(i):
        pages, counts = L.select_pages(qs[i], c.bounds, c.bscale, c.block_table, c.seq_lens, 10 + 30 * i)
        return (pages, counts, L.selected(qs[i], *c.cache(), pages, counts, **c.scales()),
                L.weighed(qs[i], *c.cache(), w[i], decay=0.0, **c.scales()), w[i])

    want = [[t.clone() for t in step(i)] for i in range(2)]
    for x in want:   # (weights past a sequence's pages stay as they are: 77, below)
        x[4][torch.arange(c.mp, device="cuda")[None, :] * PAGE >= c.seq_lens[:, None]] = 77
    torch.cuda.synchronize()
    graphs, held = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for i in range(2):
        with torch.cuda.graph(graphs[i]):
            held.append(step(i))
    for turn in range(6):
        for t in held[0] + held[1]:
            t.fill_(77)
        torch.cuda.synchronize()
        graphs[turn % 2].replay()
        graphs[1 - turn % 2].replay()
        c.attend(want[0][0], want[0][1])
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(a, b) for a, b in zip(held[i], want[i])), (turn, i)
    assert c.flags() == 0


def test_events_bracket_the_kernels(torch):
    c = Case(torch, "bf16", 8, 2, 64, [900, 64], seed=28)
    c.all_bounds()
    pages, counts = c.select(6)
    w = torch.zeros((2, c.mp), device="cuda")
    want = c.attend(pages, counts), c.weigh(w)
    for call, o in ((lambda e: c.attend(pages, counts, events=e), want[0]), (lambda e: c.weigh(w, events=e), want[1])):
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        got = call(ev)
        torch.cuda.synchronize()
        assert torch.equal(got, o) and 0 < ev[0].elapsed_time(ev[1]) < 1000


def test_other_streams(torch):
    c = Case(torch, "fp8", 40, 8, 128, [900, 2000, 64], seed=23)
    c.all_bounds()
    c.layer.weighed_workspace(3, "cuda")
    pages, counts = c.select(16)
    want = c.attend(pages, counts)
    w0 = torch.zeros((3, c.mp), device="cuda")
    c.weigh(w0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    w = torch.zeros((3, c.mp), device="cuda")
    torch.cuda.synchronize()
    p, n = c.select(16, stream=side)
    o = c.attend(p, n, stream=side)
    c.weigh(w, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(p, pages) and torch.equal(n, counts) and torch.equal(o, want) and torch.equal(w, w0)


def test_a_rollout_that_reads_and_keeps_a_part(torch):
    """Steps of growth, append with positions, bounds, choice, attention over it, weights and
    eviction, each against its own plain form on the state as it then is; shared prompt pages go
    back to the pool when their last holder drops them."""
    from paper_2607_09207_amd import DecodeAttention, rotary_frequencies
    torch.manual_seed(0)
    B, hq, hkv, d, mp, npages, budget = 6, 8, 2, 64, 24, 160, 10
    layer = DecodeAttention(hq, hkv, d, B, mp, "bf16", "bf16", "f32")
    freqs, _ = rotary_frequencies(d)
    k = torch.zeros((npages, hkv, PAGE, d), device="cuda", dtype=torch.bfloat16)
    v = torch.zeros_like(k)
    refs = torch.zeros(npages, dtype=torch.int32, device="cuda")
    table = torch.zeros((B, mp), dtype=torch.int32, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    bounds = torch.zeros((npages, hkv, 2, d), dtype=torch.int8, device="cuda")
    bscale = torch.zeros((npages, hkv), device="cuda")
    w = torch.zeros((B, mp), device="cuda")
    gone = torch.zeros(B, dtype=torch.int32, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    caches = layer.caches([(k, v)])
    # One prompt of 100 tokens, forked for the others.
    layer.page_grow(refs, table, lens, torch.tensor([100] + [0] * (B - 1), **i32))
    rows = lambda n, h: torch.randn((n, h, d), device="cuda", dtype=torch.bfloat16)   # noqa: E731
    starts = torch.tensor([0, 100] + [100] * (B - 1), **i32)
    layer.append_rotary(rows(100, hq), rows(100, hkv), rows(100, hkv), k, v, table, lens, freqs, q_start=starts)
    layer.page_bounds(k, table, lens, bounds, bscale, first=torch.zeros(B, **i32))
    layer.page_fork(refs, table, lens, torch.zeros(B - 1, **i32), torch.arange(1, B, **i32), caches)

    def kept_values(b, L):
        pages = table[b, :-(-L // PAGE)].long()
        return [t[pages].transpose(1, 2).reshape(-1, hkv, d)[:L].double() for t in (k, v)]

    for step in range(60):
        layer.page_grow(refs, table, lens, torch.full((B,), 3 if step % 2 else 1, **i32))
        n = 3 if step % 2 else 1
        starts = torch.arange(0, B * n + 1, n, **i32)
        pos = (lens + PAGE * gone).repeat_interleave(n) - n + torch.arange(n, **i32).repeat(B)
        q = layer.append_rotary(rows(B * n, hq), rows(B * n, hkv), rows(B * n, hkv), k, v, table, lens, freqs, q_start=starts,
                                positions=pos.to(torch.int32))
        layer.page_bounds(k, table, lens, bounds, bscale, first=lens - n)
        pages, counts = layer.select_pages(q, bounds, bscale, table, lens, 5, sink=1, recent=2, q_start=starts)
        part = layer.selected(q, k, v, table, lens, pages, counts, q_start=starts)
        whole = layer.weighed(q, k, v, table, lens, w, decay=0.9375, q_start=starts)
        before = lens.clone()
        if step % 10 == 3:
            for r in range(B * n):
                b, L = r // n, int(lens[r // n]) - n + r % n + 1
                kk, vv = kept_values(b, L)
                for h in range(hq):
                    g = h // (hq // hkv)
                    x = kk[:, g] @ q[r, h].double() / math.sqrt(d)
                    p = torch.softmax(x, 0)
                    a = float((p[:, None] * vv[:, g].abs()).sum(0).max())
                    tol = a * (2.0 ** -16 + 2 * (d * 2.0 ** -24 * float(q[r, h].double().norm() * kk[:, g].norm(dim=-1).max()) / 8 +
                                                2.0 ** -21 * float(x.abs().max())) + 2.0 ** -20 + 2 * L * 2.0 ** -24)
                    assert float((whole[r, h].double() - p @ vv[:, g]).abs().max()) <= tol
                    seen = torch.zeros(L, dtype=torch.bool, device="cuda")
                    for j in pages[r, g, :int(counts[r, g])].tolist():
                        seen[j * PAGE:(j + 1) * PAGE] = True
                    p = torch.softmax(x.masked_fill(~seen, -math.inf), 0)
                    assert float((part[r, h].double() - p @ vv[:, g]).abs().max()) <= tol * float(
                        (p[:, None] * vv[:, g].abs()).sum(0).max()) / a + 1e-12
        gone += layer.page_evict(refs, table, lens, w, budget, sink=1, recent=3)
        assert int(lens.max()) <= budget * PAGE and torch.equal((before - lens) % PAGE, torch.zeros_like(lens))
        held = torch.zeros(npages, **i32)
        for b in range(B):
            m = -(-int(lens[b]) // PAGE)
            held.index_add_(0, table[b, :m], torch.ones(m, **i32))
        assert torch.equal(held, refs), step
    assert int(gone.min()) > 0 and layer.read_flags(device="cuda") == 0 and layer.page_flags(npages, "cuda") == 0


# ---------------------------------------------------------------- memory: streams, far offsets

def stream_calls(torch):
    """name -> call(stream), the same result every time, as test_gpu_stream_memory takes them."""
    c = Case(torch, "bf16", 8, 2, 64, [900, 330, 700], [3, 2, 4], seed=24)
    c.all_bounds()
    s = Pool(torch, [9, 5, 7], seed=2)
    pages, counts = c.select(6)
    w = torch.zeros((3, c.mp), device="cuda")
    c.layer.weighed_workspace(9, "cuda")
    s.layer.page_workspace(s.np, "cuda")
    torch.cuda.synchronize()
    return {"select_pages": lambda st: c.select(6, stream=st)[0], "counts": lambda st: c.select(6, stream=st)[1],
            "selected": lambda st: c.attend(pages, counts, stream=st), "weighed": lambda st: c.weigh(w, stream=st),
            "page_evict": lambda st: s.evict(9, stream=st)}, [c.layer, s.layer]


@pytest.mark.parametrize("raw", [False, True], ids=["stream", "handle"])
@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
@pytest.mark.parametrize("name", ["select_pages", "counts", "selected", "weighed", "page_evict"])
def test_results_on_another_stream(torch, name, native, raw, monkeypatch):
    import test_gpu_stream_memory as memory
    monkeypatch.setattr(memory, "make_calls", stream_calls)
    memory.test_results_on_another_stream(torch, name, native, raw, monkeypatch)


def test_two_calls_at_once(torch):
    """On two streams, each with workspaces of its own."""
    c = Case(torch, "fp8", 40, 8, 128, [6000, 2000, 64, 7000], seed=25)
    c.all_bounds()
    pages, counts = c.select(40)
    w = torch.zeros((4, c.mp), device="cuda")
    want = [c.attend(pages, counts), c.weigh(w), w]
    n = c.layer.weighed_workspace(4, "cuda").numel()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    sums = [torch.zeros((4, c.mp), device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(8):
        for st, ws, sm in zip(streams, spaces, sums):
            with torch.cuda.stream(st):
                sm.zero_()
                p, k = c.select(40, workspace=ws)
                got.append((p, k, c.attend(p, k, workspace=ws), c.weigh(sm, workspace=ws), sm.clone()))
    torch.cuda.synchronize()
    for p, k, o, o2, sm in got:
        assert torch.equal(p, pages) and torch.equal(k, counts) and torch.equal(o, want[0]) and torch.equal(o2, want[1]) and \
            torch.equal(sm, want[2])
    assert all(c.flags(ws) == 0 for ws in spaces)


def far_copy(torch, c, ids, npages):
    """The case's pages at other ids of a pool of `npages`: (cache tensors, table)."""
    out = []
    for t, s in ((c.k, c.ks), (c.v, c.vs)):
        x = torch.empty((npages,) + t.shape[1:], dtype=t.dtype, device="cuda")
        sc = None if s is None else torch.empty((npages,) + s.shape[1:], device="cuda")
        x.view(raw_type(torch, c.kv))[ids] = t.view(raw_type(torch, c.kv))
        if sc is not None:
            sc[ids] = s
        out.append((x, sc))
    table = torch.where(c.block_table >= 0, ids[c.block_table.clamp_min(0).long()].to(torch.int32), -1)
    return out, table


@pytest.mark.parametrize("kv,hkv,d,npages", [("bf16", 8, 128, 140000), ("fp8", 1, 64, 17200000)])
def test_pages_past_32_bits(torch, kv, hkv, d, npages):
    """Caches of more than 4 GiB; for the fp8 one, bounds of more than 2 GiB too."""
    c = Case(torch, kv, 2 * hkv, hkv, d, [600, 64, 1000], seed=26)
    c.all_bounds()
    pages, counts = c.select(12)
    want, w0 = c.attend(pages, counts), torch.zeros((3, c.mp), device="cuda")
    want2 = c.weigh(w0)
    ids = torch.cat([torch.arange(npages - c.npages // 2, npages), torch.arange(npages // 2, npages // 2 + c.npages - c.npages // 2)]).cuda()
    ids = ids[torch.randperm(c.npages, device="cuda")]
    ((k, ks), (v, vs)), table = far_copy(torch, c, ids, npages)
    bounds = torch.empty((npages, hkv, 2, d), dtype=torch.int8, device="cuda")
    bscale = torch.empty((npages, hkv), device="cuda")
    L, w = c.layer, torch.zeros((3, c.mp), device="cuda")
    L.page_bounds(k, table, c.seq_lens, bounds, bscale, first=torch.zeros(3, dtype=torch.int32, device="cuda"), k_scale=ks)
    p, n = L.select_pages(c.q, bounds, bscale, table, c.seq_lens, 12)
    o = L.selected(c.q, k, v, table, c.seq_lens, p, n, k_scale=ks, v_scale=vs)
    o2 = L.weighed(c.q, k, v, table, c.seq_lens, w, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    used = torch.unique(c.block_table[c.block_table >= 0]).long()
    assert torch.equal(bounds[ids[used]], c.bounds[used]) and torch.equal(bscale[ids[used]], c.bscale[used])
    assert torch.equal(p, pages) and torch.equal(n, counts) and torch.equal(o, want) and torch.equal(o2, want2) and torch.equal(w, w0)
    assert c.flags() == 0


def test_weights_past_32_bits(torch):
    """Rows of 40 million pages: what is kept of every page takes more than 2^31 values."""
    from paper_2607_09207_amd import DecodeAttention
    c = Case(torch, "bf16", 16, 1, 64, [700, 33, 400, 900], seed=27)
    w0 = torch.zeros((4, c.mp), device="cuda")
    want = c.weigh(w0)
    mp = 40_000_000
    L = DecodeAttention(16, 1, 64, 4, mp, "bf16", "bf16", "f32")
    table = torch.full((4, mp), -1, dtype=torch.int32, device="cuda")
    table[:, :c.mp] = c.block_table
    w = torch.zeros((4, mp), device="cuda")
    got = L.weighed(c.q, c.k, c.v, table, c.seq_lens, w)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(w[:, :c.mp], w0) and not bool(w[:, c.mp:].any())
    assert L.read_flags(workspace=L.weighed_workspace(4, "cuda")) == 0


def test_flags_of_weights_survive_growth(torch):
    """What calls with weights raised is found where the layer keeps it, also in a workspace that they
    outgrew: what it held before the growth, and what comes after, as from a graph captured before."""
    from paper_2607_09207_amd import RldaError
    c = Case(torch, "bf16", 8, 2, 64, [100, 50, 80], [2, 3, 4], seed=34)
    L, w = c.layer, torch.zeros((3, c.mp), device="cuda")
    with pytest.raises(RldaError, match="weighed_flags"):
        L.weighed_flags("cuda")
    first = L.weighed_workspace(9, "cuda")
    c.weigh(w)
    assert L.weighed_flags("cuda") == 0
    c.block_table[1, 1] = c.npages
    c.weigh(w)
    assert L.weighed_flags("cuda") == 1
    c.block_table[1, 1] = int(c.table[1, 1])
    second = L.weighed_workspace(40, "cuda")
    c.weigh(w)
    assert second is not first and L.weighed_flags(None, workspace=second) == 0
    assert L.weighed_flags("cuda:0") == 1
    c.seq_lens[2] = 2   # fewer tokens than rows
    c.weigh(w, workspace=first)
    assert L.weighed_flags("cuda", stream=torch.cuda.current_stream().cuda_stream) == 3
    assert L.weighed_flags(None, workspace=second) == 0 and L.read_flags(device="cuda") == 0
    c.weigh(w)
    assert L.weighed_flags("cuda", workspace=second) == 2


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
def test_what_is_written_is_marked(torch, native):
    """A backward pass that saved a tensor before a call wrote to it is to notice: every tensor that the
    caller gives to be written has another version afterwards."""
    from paper_2607_09207_amd import _abi
    c = Case(torch, "bf16", 8, 2, 64, [100, 50, 80], seed=35)
    L, w = c.layer, torch.zeros((3, c.mp), device="cuda")
    s = Pool(torch, [20, 9, 30], seed=1)
    L.workspace("cuda"), L.weighed_workspace(3, "cuda"), s.layer.page_workspace(s.np, "cuda")
    if not native:
        L._fast = s.layer._fast = _abi.LEFT_TO_PYTHON
    i32 = dict(dtype=torch.int32, device="cuda")
    pages, counts, dropped = torch.zeros((3, 2, 4), **i32), torch.zeros((3, 2), **i32), torch.zeros(3, **i32)
    out = torch.zeros((3, 8, 64), device="cuda")
    for call, written in ((c.make_bounds, [c.bounds, c.bscale]), (lambda: c.select(4, out=(pages, counts)), [pages, counts]),
                          (lambda: c.select(4, out=(None, counts)), [counts]), (lambda: c.attend(pages, counts, out=out), [out]),
                          (lambda: c.weigh(w, out=out), [out, w]), (lambda: s.evict(8, dropped=dropped), [s.dev[3], dropped])):
        before = [t._version for t in written]
        call()
        assert [t._version for t in written] == [v + 1 for v in before]
    x = torch.ones(c.bscale.shape, device="cuda", requires_grad=True)
    y = (x * c.bscale).sum()
    c.make_bounds()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    with torch.inference_mode():   # tensors without versions
        c.bounds, c.bscale, out = torch.zeros_like(c.bounds), torch.zeros_like(c.bscale), torch.zeros_like(out)
        c.make_bounds()
        c.attend(pages, counts, out=out)
