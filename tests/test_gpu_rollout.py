"""The page operations, rotary appends and modified scores together, as a rollout uses them:
prompts take pages, are written and attended to; every prompt is forked for its responses;
the responses grow a token a step; some end, others take their rows; the pool is compacted.
Two layers share the page ids.

What is checked after every step: the counts and the table against the page manager in
plain Python (test_gpu_pages.Model), and, with each sequence's own K and V rows kept beside
(in 64 bits, from the rows as they were given), the caches' contents and the attention's
results.

Tolerances.  The stored rows as in test_gpu_rotary (a bf16 rounding, or half an E4M3 step of
the page's scale, which grows: a re-encoded row is off by half a step of every scale it
had, so 16 rewrites at most; the values here are normal, and the sum of halved steps is
bounded by twice the last one where scales grow by halves; they are compared with two
steps).  The attention is compared with the one over the caches' contents, as in
test_gpu_scored.
"""
import math

import numpy as np
import pytest

from test_gpu_pages import Model, pages_of
from test_gpu_rotary import turned

pytestmark = pytest.mark.gpu
PAGE = 16


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


class Rollout:
    HQ, HKV, D, ROT, ROWS, MP, LAYERS = 8, 2, 64, 32, 14, 20, 2

    def __init__(self, torch, kv):
        from paper_2607_09207_amd import DecodeAttention, rotary_frequencies
        self.torch, self.kv, self.npages = torch, kv, 120
        self.layer = DecodeAttention(self.HQ, self.HKV, self.D, self.ROWS, self.MP, "bf16", {"bf16": "bf16", "fp8": "fp8_e4m3fn"}[kv], "f32")
        shape = (self.npages, self.HKV, PAGE, self.D)
        dt = torch.bfloat16 if kv == "bf16" else torch.float8_e4m3fn
        self.pools = [tuple(torch.zeros(shape, device="cuda").to(dt) for _ in range(2)) +
                      (tuple(torch.zeros(shape[:2], device="cuda") for _ in range(2)) if kv == "fp8" else ()) for _ in range(self.LAYERS)]
        self.caches = self.layer.caches(self.pools)
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")   # noqa: E731
        self.refs, self.table, self.lens = i32(self.npages), i32(self.ROWS, self.MP), i32(self.ROWS)
        self.model = Model(self.refs.cpu().numpy(), self.table.cpu().numpy(), self.lens.cpu().numpy())
        self.freqs, _ = rotary_frequencies(self.ROT, 1e4)
        self.rows = [[[] for _ in range(self.LAYERS)] for _ in range(self.ROWS)]   # [(k, v)] of every token, as given
        self.gen = torch.Generator("cuda").manual_seed(1)
        self.mod = dict(score_cap=20.0, slopes=torch.exp2(-1.0 - torch.arange(self.HQ, device="cuda")), window=100)

    def state(self):
        return self.refs, self.table, self.lens

    def cuda(self, x):
        return self.torch.tensor(x, dtype=self.torch.int32, device="cuda")

    def step(self, n):
        """n[b] new tokens of every row: room, K and V into every layer, attention."""
        torch, L = self.torch, self.layer
        L.page_grow(*self.state(), self.cuda(n))
        self.model.grow(np.array(n))
        total = sum(n)
        start = self.cuda(np.concatenate([[0], np.cumsum(n)]).tolist())
        one = all(x <= 1 for x in n) and sum(n) == self.ROWS
        for i, pool in enumerate(self.pools):
            fused = torch.randn((total, self.HQ + 2 * self.HKV, self.D), device="cuda", generator=self.gen).bfloat16()
            q, k, v = fused[:, :self.HQ], fused[:, self.HQ:self.HQ + self.HKV], fused[:, self.HQ + self.HKV:]
            ks, vs = pool[2:] if self.kv == "fp8" else (None, None)
            kw = dict(q_start=None if one else start, k_scale=ks, v_scale=vs)
            q = L.append_rotary(q, k, v, pool[0], pool[1], self.table, self.lens, self.freqs, **kw)
            o = L.scored(q, pool[0], pool[1], self.table, self.lens, max_q_len=max(n), **kw, **self.mod)
            at = 0
            for b, m in enumerate(n):
                self.rows[b][i] += list(zip(k[at:at + m].float().cpu().numpy(), v[at:at + m].float().cpu().numpy()))
                at += m
            self.check_layer(i, n, q, o)
        self.check_state("step")

    def check_state(self, what):
        for name, got, want in (("refs", self.refs, self.model.refs), ("table", self.table, self.model.table), ("lens", self.lens, self.model.lens)):
            assert np.array_equal(got.cpu().numpy(), want), f"{what}: {name}"
        assert self.layer.page_flags(self.npages, self.refs.device) == 0 and self.layer.read_flags(device=self.refs.device) == 0

    def content(self, i, b):
        """K and V of row b in layer i, [tokens][Hkv][d], and their E4M3 steps."""
        n = int(self.model.lens[b])
        pages = self.torch.from_numpy(self.model.table[b, :pages_of(n)].astype(np.int64)).cuda()
        out = []
        for j in range(2):
            x = self.pools[i][j].view(self.torch.uint8 if self.kv == "fp8" else self.torch.bfloat16)[pages].view(self.pools[i][j].dtype).double()
            s = self.pools[i][2 + j][pages].double()[:, :, None, None] if self.kv == "fp8" else self.torch.zeros_like(x[..., :1, :1])
            x = x * s if self.kv == "fp8" else x
            tidy = lambda t: t.permute(0, 2, 1, 3).reshape(-1, self.HKV, t.shape[-1])[:n]   # noqa: E731
            out.append((tidy(x), tidy(s.expand_as(x))))
        return out

    def check_cache(self, what):
        """Every row's K and V are what was written, turned by its tokens."""
        f = self.freqs.cpu().numpy()
        for i in range(self.LAYERS):
            for b in range(self.ROWS):
                n = int(self.model.lens[b])
                assert len(self.rows[b][i]) == n
                if not n:
                    continue
                (k, sk), (v, sv) = self.content(i, b)
                k0 = np.stack([r[0] for r in self.rows[b][i]])
                want, tol = turned(k0, np.arange(n), f, False, 1.0, False)
                for got, x, t, s in ((k, want, tol, sk), (v, np.stack([r[1] for r in self.rows[b][i]]).astype(np.float64), 0.0, sv)):
                    got, s = got.cpu().numpy(), s.cpu().numpy()
                    room = 2.0 ** -8 * np.abs(x) + t if self.kv == "bf16" else 2 * np.maximum(2.0 ** -3 * np.abs(x), 2.0 ** -9 * s) + t
                    assert (np.abs(got - x) <= room + 1e-12).all(), f"{what}: layer {i} row {b}"

    def check_layer(self, i, n, q, o):
        torch, at = self.torch, 0
        G = self.HQ // self.HKV
        cap, slopes, window = self.mod["score_cap"], self.mod["slopes"].double(), self.mod["window"]
        for b, m in enumerate(n):
            if m == 0:
                continue
            L = int(self.model.lens[b])
            (k, _), (v, _) = self.content(i, b)
            k, v = (x.repeat_interleave(G, 1).transpose(0, 1).contiguous() for x in (k, v))
            qq = q[at:at + m].double().transpose(0, 1).contiguous()
            s = torch.matmul(qq, k.transpose(1, 2).contiguous()) / math.sqrt(self.D)
            big = qq.norm(dim=-1).amax() * k.norm(dim=-1).amax() / math.sqrt(self.D)
            s = cap * torch.tanh(s / cap)
            pos = (L - m + torch.arange(m, device="cuda"))[:, None]
            t = torch.arange(L, device="cuda")[None]
            s = s - slopes[:, None, None] * (pos - t).abs().double()
            s = s.masked_fill(((t > pos) | (t <= pos - window))[None], -math.inf)
            p = torch.softmax(s, dim=-1)
            want, a = torch.matmul(p, v), torch.matmul(p, v.abs())
            err = self.D * 2.0 ** -24 * big + 2.0 ** -21 * (cap + s[s.isfinite()].abs().amax()) + 2.0 ** -22 * L
            f = 2 * err + 2.0 ** -20 + 2 * L * 2.0 ** -24 + 2.0 ** -8
            got = o[at:at + m].double().transpose(0, 1)
            assert ((got - want).abs() <= a * f + 1e-30).all(), f"layer {i} row {b}"
            at += m

    def fork(self, parents, kids):
        self.layer.page_fork(*self.state(), self.cuda(parents), self.cuda(kids), self.caches)
        self.model.fork(parents, kids)
        for a, c in zip(parents, kids):
            self.rows[c] = [list(x) for x in self.rows[a]]

    def release(self, rows):
        self.layer.page_release(*self.state(), self.cuda(rows))
        self.model.release(rows)
        for r in rows:
            self.rows[r] = [[] for _ in range(self.LAYERS)]

    def compact(self):
        live = self.layer.page_compact(*self.state(), self.caches)
        assert int(live) == self.model.compact()
        self.check_state("compact")


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_rollout(torch, kv):
    r = Rollout(torch, kv)
    none = [0] * r.ROWS

    def at(**rows):
        n = list(none)
        for k, v in rows.items():
            n[int(k[1:])] = v
        return n
    print("prompts", flush=True)
    r.step(at(r0=37, r1=64, r2=1))
    r.step(at(r0=20, r2=130))   # a second chunk
    r.check_cache("prompts")
    print("fork", flush=True)
    r.fork([0, 0, 0, 1, 1, 2, 2], [3, 4, 5, 6, 7, 8, 9])
    r.check_state("fork")
    r.check_cache("fork")
    print("responses", flush=True)
    for k in range(18):
        r.step([0 if b < 3 or b > 9 else 1 for b in range(r.ROWS)])
    r.step(at(r3=4, r4=4, r6=2, r8=3))   # a few tokens at once
    r.check_cache("responses")
    print("some end, others begin", flush=True)
    r.release([0, 4, 7])
    r.check_state("release")
    r.step(at(r0=50, r10=9, r11=16, r12=1, r13=33))
    r.compact()
    r.check_cache("compaction")
    for k in range(3):
        r.step([1 if b not in (4, 7) else 0 for b in range(r.ROWS)])
    print("every row", flush=True)
    r.step(at(r4=3, r7=2))
    for k in range(17):
        r.step([1] * r.ROWS)   # the form without q_start
    r.check_cache("every row")
    r.release(list(range(r.ROWS)))
    assert int(r.refs.sum()) == 0
    r.compact()
