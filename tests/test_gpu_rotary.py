"""Rotary positions on the GPU: rows alone (rotate) and on their way into the paged cache
(append_rotary), against the rotation in 64 bits.

Tolerances.  With c, s the cosine and sine rounded to fp32 (2^-24 relative each), the
product y s rounded, and one rounding of x c - y s:
    |error| <= 2^-24 (2 |x c| + 3 |y s|) (A inside c and s),
and where the result is bf16 half a step of it, 2^-8 |a'|, more.  The angle is reduced in 64
bits: at 2^20 positions three roundings of 2^-53 of at most 2^18 turns, 2^-34 turns, which
3 2^-34 2 pi < 2^-29 of |x| + |y| covers.  E4M3: half a step is 2^-4 of the value, or 2^-10
of the scale below the normal range.
"""
import math

import numpy as np
import pytest

from oracle.append import e4m3_decode, e4m3_encode

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


def say(*a):
    print(*a, flush=True)


def np64(t):
    with np.errstate(invalid="ignore"):   # rows that nobody writes may hold anything
        return _np64(t)


def _np64(t):
    return t.detach().float().cpu().numpy().astype(np.float64) if t.element_size() < 8 else t.detach().cpu().numpy()


def turned(x, pos, freqs, interleaved, amplitude, inverse):
    """(x [n][heads][d] turned, in 64 bits; the bound on an fp32 result's error)."""
    x = x.astype(np.float64)
    half = len(freqs)
    t = pos.astype(np.float64)[:, None] * freqs[None, :] * (-1.0 if inverse else 1.0)
    c, s = amplitude * np.cos(t)[:, None], amplitude * np.sin(t)[:, None]
    out, tol = x.copy(), np.zeros_like(x)
    ia = np.arange(half) * 2 if interleaved else np.arange(half)
    ib = ia + 1 if interleaved else ia + half
    a, b = x[..., ia], x[..., ib]
    out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
    far = 2.0 ** -29 * amplitude * (np.abs(a) + np.abs(b))
    tol[..., ia] = 2.0 ** -24 * (2 * np.abs(a * c) + 3 * np.abs(b * s)) * 1.001 + far
    tol[..., ib] = 2.0 ** -24 * (2 * np.abs(b * c) + 3 * np.abs(a * s)) * 1.001 + far
    return out, tol


def within(got, want, tol, bf16, what):
    if bf16:
        tol = tol * 1.01 + 2.0 ** -8 * (np.abs(want) + tol)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(got - want)[bad])}"


# ------------------------------------------------------------------ rows alone

SHAPES = [(1, 1, 32, 16), (1, 8, 64, 64), (17, 3, 80, 80), (16, 5, 128, 128), (33, 7, 128, 32), (5, 256, 32, 32),
          (100, 2, 256, 256), (257, 12, 40, 16), (2, 9, 256, 16), (1000, 36, 128, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_rotate(torch, shape, interleaved, dtype):
    from paper_2607_09207_amd import rotary_frequencies, rotate
    n, heads, d, rot = shape
    say("rotate", shape, interleaved, dtype)
    g = torch.Generator("cuda").manual_seed(n * 7 + heads)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    fused = torch.randn((n, heads + 3, d), device="cuda", generator=g).to(dt)
    x = fused[:, 1:heads + 1]
    pos = torch.randint(-5, 1 << 20, (n,), device="cuda", generator=g, dtype=torch.int32)
    freqs, _ = rotary_frequencies(rot, 1e4)
    for amplitude, inverse in ((1.0, False), (1.25, True)):
        got = rotate(x, pos, freqs, interleaved=interleaved, amplitude=amplitude, inverse=inverse)
        want, tol = turned(np64(x), pos.cpu().numpy(), freqs.cpu().numpy(), interleaved, amplitude, inverse)
        within(np64(got), want, tol, dtype == "bf16", "rotate")
        assert torch.equal(got[..., rot:], x[..., rot:])
    # In place, on a slice, and into a [heads][n] buffer: the same bits, the neighbours left alone.
    back = fused.clone()
    want = rotate(x, pos, freqs, interleaved=interleaved)
    y = back[:, 1:heads + 1]
    assert rotate(y, pos, freqs, interleaved=interleaved, out=y) is y
    assert torch.equal(y, want) and torch.equal(back[:, 0], fused[:, 0]) and torch.equal(back[:, heads + 1:], fused[:, heads + 1:])
    other = torch.zeros((heads, n, d), device="cuda", dtype=dt).transpose(0, 1)
    assert torch.equal(rotate(x, pos, freqs, interleaved=interleaved, out=other), want)


@pytest.mark.parametrize("n", [17000, 40000, 70000, 140001])
def test_rotate_windows(torch, n):
    """Enough rows for windows of 2, 4, 8 and 16, and (the last) for reading past the caches."""
    from paper_2607_09207_amd import rotary_frequencies, rotate
    heads = 1 if n < 140000 else 9
    x = torch.randn((n, heads, 64), device="cuda").bfloat16()
    pos = torch.randint(0, 1 << 20, (n,), device="cuda", dtype=torch.int32)
    freqs, _ = rotary_frequencies(32)
    got = rotate(x, pos, freqs)
    pick = torch.cat([torch.arange(40), torch.arange(n - 40, n), torch.randint(0, n, (3000,))]).cuda()
    want, tol = turned(np64(x[pick]), pos[pick].cpu().numpy(), freqs.cpu().numpy(), False, 1.0, False)
    within(np64(got[pick]), want, tol, True, "rotate")
    part = rotate(x[5:1000], pos[5:1000], freqs)   # the same rows in other windows
    assert torch.equal(part, got[5:1000])


def test_append_rotary_large_windows(torch):
    """140,000 rows in a bf16 cache: windows of 16."""
    from paper_2607_09207_amd import rotary_frequencies
    rng = np.random.default_rng(1)
    rows = rng.integers(1, 5000, size=60)
    c = Case(torch, "bf16", 1, 1, 64, rows + rng.integers(0, 30, size=60), rows, seed=3)
    assert c.q.shape[0] > 16 * 8192
    freqs, _ = rotary_frequencies(64)
    q = c.run(freqs)
    pos = torch.cat([torch.arange(L - m, L) for L, m in zip(c.lens.tolist(), c.rows.tolist())])
    want, tol = turned(np64(c.q), pos.numpy(), freqs.cpu().numpy(), False, 1.0, False)
    within(np64(q), want, tol, True, "q")
    seq = np.repeat(np.arange(60), c.rows)
    page, slot = c.table[seq, pos.numpy() // PAGE], pos.numpy() % PAGE
    want, tol = turned(np64(c.k_new), pos.numpy(), freqs.cpu().numpy(), False, 1.0, False)
    within(np64(c.k)[page, :, slot], want, tol, True, "k")
    assert np.array_equal(np64(c.v)[page, :, slot], np64(c.v_new))


def test_rotate_broadcast_and_empty(torch):
    from paper_2607_09207_amd import rotary_frequencies, rotate
    freqs, _ = rotary_frequencies(64)
    one = torch.randn((1, 1, 64), device="cuda")
    pos = torch.arange(20, device="cuda", dtype=torch.int32)
    got = rotate(one.expand(20, 4, 64), pos, freqs)
    assert torch.equal(got, rotate(one.expand(20, 4, 64).contiguous(), pos, freqs))
    assert rotate(torch.empty((0, 4, 64), device="cuda"), pos[:0], freqs).shape == (0, 4, 64)
    assert rotate(torch.empty((3, 0, 64), device="cuda"), pos[:3], freqs).shape == (3, 0, 64)


def test_rotate_infinities_stay_in_their_pair(torch):
    from paper_2607_09207_amd import rotary_frequencies, rotate
    freqs, _ = rotary_frequencies(64)
    x = torch.randn((3, 2, 128), device="cuda")
    y = x.clone()
    y[1, 1, 5], y[1, 1, 100] = float("inf"), float("nan")
    pos = torch.tensor([0, 7, 9], device="cuda", dtype=torch.int32)
    a, b = rotate(x, pos, freqs), rotate(y, pos, freqs)
    hit = torch.zeros_like(x, dtype=torch.bool)
    hit[1, 1, [5, 37, 100]] = True
    assert torch.equal(a[~hit], b[~hit]) and not b[hit].isfinite().any()


@pytest.mark.parametrize("interleaved", [False, True])
def test_inverse_is_the_gradient(torch, interleaved):
    """<w, R x> = <R' w, x>, and R' w against differences of <w, R x> (linear in x: a step
    of any size; fp32 results, so the difference carries their error)."""
    from paper_2607_09207_amd import rotary_frequencies, rotate
    freqs, _ = rotary_frequencies(32, 1e3)
    n, h, d = 9, 2, 64
    g = torch.Generator("cuda").manual_seed(3)
    x, w = (torch.randn((n, h, d), device="cuda", generator=g) for _ in range(2))
    pos = torch.randint(0, 5000, (n,), device="cuda", generator=g, dtype=torch.int32)
    kw = dict(interleaved=interleaved, amplitude=1.5)
    grad = rotate(w, pos, freqs, inverse=True, **kw)
    want, tol = turned(np64(w), pos.cpu().numpy(), freqs.cpu().numpy(), interleaved, 1.5, True)
    within(np64(grad), want, tol, False, "gradient")
    base = rotate(x, pos, freqs, **kw).double()
    for i in range(0, d, 5):
        step = x.clone()
        step[..., i] += 1.0
        diff = ((rotate(step, pos, freqs, **kw).double() - base) * w.double()).sum(-1)
        # Two results of two elements, each within 5 2^-24 A max|.| of its value, times w.
        room = 4 * 5 * 2.0 ** -24 * 1.5 * (x.abs().amax() + 1) * w.abs().amax()
        assert (diff - grad[..., i].double()).abs().max() <= room


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_autograd(torch, dtype):
    """x.grad is the inverse rotation of the gradient, through a slice, a broadcast, and twice."""
    from paper_2607_09207_amd import RldaError, rotary_frequencies, rotate
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    freqs, _ = rotary_frequencies(64)
    fused = torch.randn((50, 6, 128), device="cuda").to(dt).requires_grad_()
    pos = torch.randint(0, 3000, (50,), device="cuda", dtype=torch.int32)
    w = torch.randn((50, 4, 128), device="cuda").to(dt)
    y = rotate(fused[:, 1:5], pos, freqs, amplitude=1.25)
    assert torch.equal(y.detach(), rotate(fused.detach()[:, 1:5], pos, freqs, amplitude=1.25))
    (g,) = torch.autograd.grad(y, fused, w, retain_graph=True)
    assert torch.equal(g[:, 1:5], rotate(w, pos, freqs, amplitude=1.25, inverse=True)) and not g[:, 0].any() and not g[:, 5].any()
    (g,) = torch.autograd.grad(y.sum(), fused)   # a broadcast gradient
    assert torch.equal(g[:, 1:5], rotate(torch.ones_like(w), pos, freqs, amplitude=1.25, inverse=True))
    one = torch.randn((1, 1, 128), device="cuda").to(dt).requires_grad_()
    rotate(one.expand(50, 4, 128), pos, freqs).backward(w)
    want = rotate(w, pos, freqs, inverse=True)
    assert torch.equal(one.grad, want.sum((0, 1), keepdim=True, dtype=want.dtype))
    v = w.clone().requires_grad_()
    (g,) = torch.autograd.grad(rotate(fused[:, 1:5], pos, freqs), fused, v, create_graph=True)
    (g2,) = torch.autograd.grad((g[:, 1:5] * w).sum(), v)
    assert torch.equal(g2, rotate(w, pos, freqs))
    with pytest.raises(RldaError):
        rotate(fused[:, 1:5], pos, freqs, out=w)
    with torch.no_grad():
        assert not rotate(fused[:, 1:5], pos, freqs).requires_grad


def test_autograd_refusals_and_versions(torch):
    """What would go without a gradient is refused; a saved tensor turned in place is noticed."""
    from paper_2607_09207_amd import RldaError, rotary_frequencies, rotate
    freqs, _ = rotary_frequencies(64)
    x = torch.randn((5, 2, 64), device="cuda")
    pos = torch.arange(5, device="cuda", dtype=torch.int32)
    grads = x.clone().requires_grad_()
    with pytest.raises(RldaError):
        rotate(x, pos, freqs, out=grads)
    with pytest.raises(RldaError):
        rotate(x, pos, freqs.clone().requires_grad_())
    with torch.no_grad():
        assert rotate(x, pos, freqs, out=grads) is grads
    w = torch.ones_like(x).requires_grad_()
    y = w * x
    assert torch.equal(rotate(x, pos, freqs, out=x), grads)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    with torch.inference_mode():
        z = x + 1
        assert rotate(z, pos, freqs, out=z) is z


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
def test_forward_mode(torch, native, monkeypatch):
    """A dual tensor's tangent is turned as its value is (the rotation is linear), also where it
    requires grad; a tangent that would be lost is refused."""
    import torch.autograd.forward_ad as fwd

    from paper_2607_09207_amd import RldaError, _abi, rotary_frequencies, rotate
    if not native:
        monkeypatch.setattr(_abi, "fastcall", lambda: None)
    freqs, _ = rotary_frequencies(64)
    x, t = (torch.randn((5, 2, 64), device="cuda") for _ in range(2))
    pos = torch.arange(5, device="cuda", dtype=torch.int32)
    kw = dict(interleaved=True, amplitude=1.5)
    y, ty = rotate(x, pos, freqs, **kw), rotate(t, pos, freqs, **kw)
    leaf = x.clone().requires_grad_()
    with fwd.dual_level():
        for v in (x, leaf):
            got = fwd.unpack_dual(rotate(fwd.make_dual(v, t), pos, freqs, **kw))
            assert torch.equal(got.primal, y) and torch.equal(got.tangent, ty)
        assert torch.equal(torch.autograd.grad(got.primal, leaf, t)[0], rotate(t, pos, freqs, inverse=True, **kw))
        # (a tangent of any layout, and the tangent of the inverse)
        wide = torch.randn((2, 64, 5), device="cuda").permute(2, 0, 1)
        got = fwd.unpack_dual(rotate(fwd.make_dual(x, wide), pos, freqs, inverse=True)).tangent
        assert torch.equal(got, rotate(wide.contiguous(), pos, freqs, inverse=True))
        dual = fwd.make_dual(x, t)
        for bad in (lambda: rotate(dual, pos, freqs, out=torch.empty_like(x)), lambda: rotate(x, pos, freqs, out=dual),
                    lambda: rotate(dual, pos, freqs, stream=torch.cuda.current_stream()),
                    lambda: rotate(x, pos, fwd.make_dual(freqs, freqs))):
            with pytest.raises(RldaError):
                bad()
        assert fwd.unpack_dual(rotate(x, pos, freqs)).tangent is None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_that_begin_anywhere(torch, dtype):
    """A gradient that is a contiguous piece of another one (of a concatenation) is not aligned
    as rows have to be; a tangent neither."""
    import torch.autograd.forward_ad as fwd

    from paper_2607_09207_amd import rotary_frequencies, rotate
    freqs, _ = rotary_frequencies(32)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.randn((5, 2, 32), device="cuda").to(dt).requires_grad_()
    pos = torch.arange(5, device="cuda", dtype=torch.int32)
    head = torch.zeros(3, device="cuda", dtype=dt, requires_grad=True)
    w = torch.randn(3 + x.numel(), device="cuda").to(dt)
    y = torch.cat([head, rotate(x, pos, freqs).flatten()])
    piece = w[3:].view(5, 2, 32)
    assert piece.data_ptr() % 16 != 0
    y.backward(w)
    assert torch.equal(x.grad, rotate(piece.clone(), pos, freqs, inverse=True)) and torch.equal(head.grad, w[:3])
    with fwd.dual_level():
        got = fwd.unpack_dual(rotate(fwd.make_dual(x.detach(), piece), pos, freqs)).tangent
        assert torch.equal(got, rotate(piece.clone(), pos, freqs))


def test_single_rows_of_any_stride(torch):
    """One row, or one head, of a buffer whose other stride is no multiple of 16 bytes."""
    from paper_2607_09207_amd import rotary_frequencies, rotate
    freqs, _ = rotary_frequencies(64)
    pos = torch.full((1,), 77, device="cuda", dtype=torch.int32)
    x = torch.randn(1, 2 * 64 + 3, device="cuda").to(torch.bfloat16)[:, :128].view(1, 2, 64)
    x = x.as_strided((1, 2, 64), (131, 64, 1))
    assert torch.equal(rotate(x, pos, freqs), rotate(x.clone(memory_format=torch.contiguous_format), pos, freqs))
    y = torch.randn((3, 1, 64), device="cuda").as_strided((3, 1, 64), (64, 7, 1))
    assert torch.equal(rotate(y, pos.expand(3).contiguous(), freqs), rotate(y.contiguous().view(3, 1, 64), pos.expand(3).contiguous(), freqs))


def test_captured_backward(torch):
    """Forward and backward in one graph, replayed, with eager work between."""
    from paper_2607_09207_amd import rotary_frequencies, rotate
    freqs, amp = rotary_frequencies(128)
    x = torch.randn((40, 3, 128), device="cuda").to(torch.bfloat16).requires_grad_()
    w = torch.randn((40, 3, 128), device="cuda").to(torch.bfloat16)
    pos = torch.randint(0, 9000, (40,), device="cuda", dtype=torch.int32)

    def step():
        y = rotate(x, pos, freqs, interleaved=True)
        return y.detach(), torch.autograd.grad(y, x, w)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, g = step()
    for i in range(3):
        with torch.no_grad():
            x.copy_(torch.randn((40, 3, 128), device="cuda"))
        w.copy_(torch.randn((40, 3, 128), device="cuda"))
        pos.add_(1000 * i)
        y.zero_(), g.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want, grad = step()
        assert torch.equal(y, want) and torch.equal(g, grad)


# ------------------------------------------------------------------ rows into the cache

KV = {"f32": ("f32", 4), "bf16": ("bf16", 2), "fp8": ("fp8_e4m3fn", 1)}


class Case:
    """lens: lengths; rows: new tokens of each (None: one each, without q_start)."""

    def __init__(self, torch, kv, hq, hkv, d, lens, rows, layout="head", seed=0, extra=3, lead=0, behind=0):
        from paper_2607_09207_amd import DecodeAttention
        rng = np.random.default_rng(seed)
        g = torch.Generator("cuda").manual_seed(seed)
        self.lens, self.rows = np.asarray(lens), np.ones(len(lens), int) if rows is None else np.asarray(rows)
        self.kv, self.hq, self.hkv, self.d, self.lead = kv, hq, hkv, d, lead
        used = -(-np.maximum(self.lens, 0) // PAGE)
        mp = int(used.max()) + 2
        self.npages = int(used.sum()) + extra
        perm = rng.permutation(self.npages)
        self.table = np.full((len(lens), mp), -1, np.int32)
        at = 0
        for b, u in enumerate(used):
            self.table[b, :u] = perm[at:at + u]
            at += u
        self.start = lead + np.concatenate([[0], np.cumsum(self.rows)])
        n = int(self.start[-1]) + behind
        if rows is None:
            n = len(lens)
        dt = torch.float32 if kv == "f32" else torch.bfloat16
        fused = torch.randn((n, hq + 2 * hkv + 1, d), device="cuda", generator=g).to(dt)
        self.q, self.k_new, self.v_new = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv + 1:]
        shape = (self.npages, hkv, PAGE, d) if layout == "head" else (self.npages, PAGE, hkv, d)
        view = (lambda t: t) if layout == "head" else (lambda t: t.transpose(1, 2))

        def pool():
            if kv != "fp8":
                return view(torch.randn(shape, device="cuda", generator=g).to(dt)), None
            raw = torch.randint(0, 256, shape, device="cuda", generator=g, dtype=torch.uint8)
            raw[(raw & 0x7F) == 0x7F] = 0
            return view(raw.view(torch.float8_e4m3fn)), torch.rand((self.npages, hkv), device="cuda", generator=g) * 0.01
        (self.k, self.ks), (self.v, self.vs) = pool(), pool()
        self.block_table = torch.from_numpy(self.table).cuda()
        self.seq_lens = torch.from_numpy(self.lens.astype(np.int32)).cuda()
        self.q_start = None if rows is None else torch.from_numpy(self.start.astype(np.int32)).cuda()
        self.layer = DecodeAttention(hq, hkv, d, len(lens), mp, "f32" if kv == "f32" else "bf16", KV[kv][0],
                                     "f32", kv_strides=self.k.stride()[:3])

    def run(self, freqs, **kw):
        return self.layer.append_rotary(self.q, self.k_new, self.v_new, self.k, self.v, self.block_table, self.seq_lens,
                                        freqs, q_start=self.q_start, k_scale=self.ks, v_scale=self.vs, **kw)

    def tokens(self):
        """(row, sequence, token) of every written row."""
        for b, (L, n) in enumerate(zip(self.lens, self.rows)):
            for i in range(n):
                if 0 <= L - n + i and (self.q_start is not None or L > 0):
                    yield int(self.start[b]) + i if self.q_start is not None else b, b, int(L - n + i)


def raw(t):
    import torch
    t = t.contiguous()
    return (t.view(torch.uint8) if t.element_size() == 1 else t.view(torch.int16) if t.element_size() == 2 else
            t.view(torch.int32)).cpu().numpy()


def check(torch, c, freqs, before, q, interleaved, amplitude, positions=None):
    """c's caches after a run, from their state `before` (k, v, ks, vs) and the rows."""
    f = freqs.cpu().numpy()
    written = list(c.tokens())
    rows = np.array([r for r, _, _ in written], int)
    pos = np.array([t for _, _, t in written]) if positions is None else positions.cpu().numpy()[rows]
    bf16 = c.kv != "f32"
    if len(rows):
        want, tol = turned(np64(c.q)[rows], pos, f, interleaved, amplitude, False)
        within(np64(q)[rows], want, tol, bf16, "q")
    page = np.array([c.table[b, t // PAGE] for _, b, t in written], int)
    slot = np.array([t % PAGE for _, _, t in written], int)
    for name, turns in (("k", True), ("v", False)):
        new, now, old = np64(getattr(c, name + "_new")), getattr(c, name), before[name]
        want, tol = (turned(new[rows], pos, f, interleaved, amplitude, False) if turns and len(rows)
                     else (new[rows], np.zeros_like(new[rows])))
        if c.kv != "fp8":
            keep = np.ones((c.npages, PAGE), bool)
            keep[page, slot] = False
            a, b = raw(now).transpose(0, 2, 1, 3), raw(old).transpose(0, 2, 1, 3)
            assert np.array_equal(a[keep], b[keep]), f"{name}: other slots changed"
            got = np64(now).transpose(0, 2, 1, 3)[page, slot]
            if turns:
                within(got, want, tol, bf16, name)
            else:
                assert np.array_equal(got, want), name
            continue
        a, b = raw(now), raw(old)
        sa, sb = getattr(c, name + "s").cpu().numpy(), before[name + "s"].cpu().numpy()
        touched = set(page.tolist())
        rest = np.array([p for p in range(c.npages) if p not in touched], int)
        assert np.array_equal(a[rest], b[rest]) and np.array_equal(sa[rest], sb[rest]), f"{name}: other pages changed"
        for p in touched:
            mine = np.flatnonzero(page == p)
            mine = mine[np.argsort(slot[mine])]
            s0, s1 = int(slot[mine[0]]), int(slot[mine[-1]])
            assert s1 - s0 + 1 == len(mine)
            assert np.array_equal(a[p, :, s1 + 1:], b[p, :, s1 + 1:]), f"{name}: slots behind the rows changed"
            for g in range(c.hkv):
                x = want[mine, g]
                amax = np.float32(np.abs(x).max())
                old_s = np.float32(sb[p, g]) if s0 else np.float32(0)
                if not (old_s > 0 and np.isfinite(old_s)):
                    old_s = np.float32(0)
                limit, s_new = np.float32(448) * old_s, sa[p, g]
                # (The turned rows' amax is known to within their tolerance.)
                near = turns and abs(float(amax) - float(limit)) <= 1e-5 * float(amax)
                grew = s0 == 0 or amax > limit
                if not near:
                    expect = np.float32(amax / np.float32(448)) if grew else old_s
                    if turns:
                        assert abs(float(s_new) - float(expect)) <= 1e-6 * float(expect), (name, p, g)
                    else:
                        assert s_new == expect, (name, p, g, s_new, expect)
                    if s0:
                        e = b[p, g, :s0]
                        if grew:
                            ratio = np.float32(old_s / s_new) if old_s > 0 else np.float32(0)
                            e = e4m3_encode((e4m3_decode(e).astype(np.float32) * ratio).astype(np.float32)) if old_s > 0 else e * 0
                        assert np.array_equal(a[p, g, :s0], e), f"{name}: earlier rows"
                code = a[p, g, s0:s1 + 1]
                if turns:
                    got = e4m3_decode(code) * float(s_new)
                    room = np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * float(s_new)) * 1.0001 + tol[mine, g] + 1e-6 * np.abs(x)
                    assert (np.abs(got - x) <= room).all(), (name, p, g, np.max(np.abs(got - x) - room))
                else:
                    # Rows that set the scale: 448 x / amax (448 x is exact), else x / scale.
                    f = x.astype(np.float32)
                    e = e4m3_encode(np.float32(448) * f / amax if grew else f / s_new) if s_new > 0 else np.zeros_like(code)
                    assert np.array_equal(code, e), (name, p, g)


LENS1 = [1, 16, 17, 0, 33, 200, 2, 31, 32, 48, 1, 15, 1000]
CHUNKS = [([5], [5]), ([16], [16]), ([17], [17]), ([40], [7]), ([40], [31]), ([100, 3, 64], [33, 3, 64]),
          ([20, 0, 50, 7, 300], [1, 0, 50, 0, 47]), ([1] * 40, [1] * 40), ([95, 18, 130], [80, 2, 115]), ([600], [555])]


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", ["one"] + list(range(len(CHUNKS))), ids=str)
def test_append_rotary(torch, kv, d, rows):
    from paper_2607_09207_amd import rotary_frequencies
    lens, n = (LENS1, None) if rows == "one" else CHUNKS[rows]
    hq, hkv = (2, 2) if kv == "f32" else (12, 2)
    if kv == "f32" and d == 128:
        hq, hkv = 2, 2
    for k, (rot, il, amp, layout) in enumerate([(d, False, 1.0, "head"), (d // 2, True, 1.1386, "slot"), (16, False, 1.0, "slot"),
                                                (48, False, 0.5, "head"), (16, True, 1.0, "head")]):
        say("append_rotary", kv, d, rows, rot, il, layout)
        c = Case(torch, kv, hq, hkv, d, lens, n, layout, seed=k + 10)
        freqs, _ = rotary_frequencies(rot, 1e4)
        before = {x: None if getattr(c, x) is None else getattr(c, x).clone() for x in ("k", "v", "ks", "vs")}
        q = c.run(freqs, interleaved=il, amplitude=amp)
        check(torch, c, freqs, before, q, il, amp)
        assert c.layer.read_flags(device=c.q.device) == 0


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("n", [2100, 4300, 9000, 17000])
def test_append_rotary_windows(torch, kv, n):
    """Enough rows for windows of 2, 4, 8 and 16, cut into sequences of any length."""
    from paper_2607_09207_amd import rotary_frequencies
    rng = np.random.default_rng(n)
    rows = []
    while sum(rows) < n:
        rows.append(int(rng.choice([0, 1, 2, 15, 16, 17, 40, 333, 900])))
    lens = [m + int(rng.integers(0, 40)) for m in rows]
    say("windows", kv, n, len(rows))
    c = Case(torch, kv, 4, 2, 64, lens, rows, seed=n, lead=1, behind=2)
    freqs, _ = rotary_frequencies([64, 32, 48, 16][n % 4], 1e4)
    before = {x: None if getattr(c, x) is None else getattr(c, x).clone() for x in ("k", "v", "ks", "vs")}
    q = c.run(freqs)
    check(torch, c, freqs, before, q, False, 1.0)
    assert c.layer.read_flags(device=c.q.device) == 0


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_append_rotary_between_empty_sequences(torch, kv):
    """Rows of neighbours with runs of sequences that bring none between them, shorter and
    longer than a wave; and what such runs cost: next to nothing."""
    from paper_2607_09207_amd import rotary_frequencies
    freqs, _ = rotary_frequencies(64, 1e4)
    for gaps in ([0, 1, 62, 63, 64, 65, 3], [200, 64, 0, 0, 127, 128, 129, 1000], [5, 3000, 1]):
        rows = []
        for i, gap in enumerate(gaps):
            rows += [0] * gap + [[1, 2, 17, 1][i % 4]]
        rows += [0] * gaps[0]
        lens = [m and m + i % 23 for i, m in enumerate(rows)]
        say("empty sequences", kv, gaps)
        c = Case(torch, kv, 4, 2, 64, lens, rows, seed=len(rows), lead=2, behind=1)
        before = {x: None if getattr(c, x) is None else getattr(c, x).clone() for x in ("k", "v", "ks", "vs")}
        check(torch, c, freqs, before, c.run(freqs), False, 1.0)
        assert c.layer.read_flags(device=c.q.device) == 0

    def us(rows):
        c = Case(torch, kv, 4, 2, 64, [40 if m else 0 for m in rows], rows, seed=1)
        best = math.inf
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            for _ in range(20):
                c.run(freqs)
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b) * 50)
        return best
    alone, among = us([1] * 8), us(([0] * 1000 + [1]) * 8)
    say("8 rows", kv, alone, "us, with 8000 empty sequences among them", among)
    assert among < 10 * alone   # (one after the other they took 94 times as long)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_rows_of_nobody_stay(torch, kv):
    """q_start that begins after row 0 and ends before the last row; given positions; q in place."""
    from paper_2607_09207_amd import rotary_frequencies
    c = Case(torch, kv, 8, 2, 64, [40, 30], [20, 9], seed=4, lead=3, behind=5)
    freqs, _ = rotary_frequencies(64)
    before = {x: None if getattr(c, x) is None else getattr(c, x).clone() for x in ("k", "v", "ks", "vs")}
    pos = torch.randint(0, 9999, (c.q.shape[0],), device="cuda", dtype=torch.int32)
    q0 = c.q.clone()
    out = torch.full_like(q0, 7.0)
    assert c.run(freqs, positions=pos, out=out) is out
    check(torch, c, freqs, before, out, False, 1.0, pos)
    assert (out[:3] == 7).all() and (out[-5:] == 7).all()
    again = c.run(freqs, positions=pos, out=c.q)
    assert torch.equal(again[3:-5], out[3:-5]) and torch.equal(again[:3], q0[:3]) and torch.equal(again[-5:], q0[-5:])
    assert c.layer.read_flags(device=c.q.device) == 0


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_one_token_is_append(torch, kv):
    """At position 0 nothing turns: the caches and scales append leaves, bit for bit, but for
    fp8 values halfway between two codes (append rounds value / scale in between)."""
    from paper_2607_09207_amd import rotary_frequencies
    a, b = (Case(torch, kv, 12, 2, 128, LENS1, None, seed=9) for _ in range(2))
    freqs, _ = rotary_frequencies(128)
    zero = torch.zeros(len(LENS1), dtype=torch.int32, device="cuda")
    q = a.run(freqs, positions=zero)
    b.layer.append(b.k_new.contiguous(), b.v_new.contiguous(), b.k, b.v, b.block_table, b.seq_lens, k_scale=b.ks, v_scale=b.vs)
    live = torch.tensor([x > 0 for x in LENS1], device="cuda")
    assert torch.equal(q[live], a.q[live])
    if kv == "fp8":
        assert torch.equal(a.ks, b.ks) and torch.equal(a.vs, b.vs)
    for x in ("k", "v"):
        ra, rb = raw(getattr(a, x)), raw(getattr(b, x))
        if kv == "bf16":
            assert np.array_equal(ra, rb), x
            continue
        for p, g, s, e in np.argwhere(ra != rb):
            seq, tok = next((i, t) for _, i, t in a.tokens() if a.table[i, t // PAGE] == p)
            row = np64(getattr(a, x + "_new"))[seq, g]
            assert s == tok % PAGE, "an earlier row differs"
            mid = (e4m3_decode(ra[p, g, s, e]) + e4m3_decode(rb[p, g, s, e])) / 2
            assert abs(int(ra[p, g, s, e]) - int(rb[p, g, s, e])) == 1
            assert abs(row[e] * 448 / np.abs(row).max() - mid) <= 2.0 ** -22 * abs(mid), "not halfway between two codes"


@pytest.mark.parametrize("rows", [None, [7, 20, 3]], ids=["one", "chunks"])
def test_large_rows_in_fp8(torch, rows):
    """Rows near the largest bf16 value, and (of V) beside an infinity: E4M3(448 value / amax) or
    E4M3(value / scale), as the quotients are in 64 bits (448 value overflows in 32)."""
    from paper_2607_09207_amd import rotary_frequencies
    freqs, _ = rotary_frequencies(64)
    for big in (7e35, 8e35, 1e37, 3.3e38):
        say("large rows", rows, big)
        c = Case(torch, "fp8", 4, 2, 64, [40, 20, 35], rows, seed=6)
        n = c.q.shape[0]
        # Magnitudes from the largest down to 2^-20 of it: codes of every size.
        g = torch.Generator("cuda").manual_seed(1)
        for t in (c.k_new, c.v_new):
            size = torch.exp2(-20 * torch.rand(t.shape, device="cuda", generator=g))
            t.copy_(torch.where(torch.rand(t.shape, device="cuda", generator=g) < 0.5, -big, big) * size)
            t[..., 5] = big
        c.v_new[n - 1, 1, 9] = float("inf")
        old = {x: getattr(c, x + "s").clone().cpu().numpy() for x in "kv"}
        c.run(freqs, positions=torch.zeros(n, dtype=torch.int32, device="cuda"))
        rows_of = {}
        for r, b, t in c.tokens():
            rows_of.setdefault(int(c.table[b, t // PAGE]), []).append((t % PAGE, r))
        for name in "kv":
            new, code = np64(getattr(c, name + "_new")), raw(getattr(c, name))
            scale = getattr(c, name + "s").cpu().numpy().astype(np.float64)
            for p, of in rows_of.items():
                for g in range(c.hkv):
                    x = np.stack([new[r, g] for _, r in of])
                    amax = np.abs(x).max()
                    assert of[0][0] == 0 or amax > 448 * float(old[name][p, g])   # they set the scale
                    assert scale[p, g] == np.float32(amax) / np.float32(448) if np.isfinite(amax) else np.isinf(scale[p, g])
                    got = np.stack([code[p, g, s] for s, _ in of])
                    if np.isfinite(amax):
                        assert np.array_equal(got, e4m3_encode(448.0 * x / amax)), (name, p, g)
                    else:
                        assert np.array_equal((got & 0x7F) == 0x7F, np.isinf(x)) and not (got[np.isfinite(x)] & 0x7F).any()


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_bad_rows_are_flagged_and_skipped(torch, kv):
    from paper_2607_09207_amd import rotary_frequencies
    freqs, _ = rotary_frequencies(64)
    # A page id outside the pool: its token's q alone is written.
    c = Case(torch, kv, 4, 2, 64, [20, 40, 33], [20, 5, 33], seed=1)
    c.block_table[0, 1] = c.npages
    c.block_table[2, 0] = -1
    before = {x: None if getattr(c, x) is None else getattr(c, x).clone() for x in ("k", "v", "ks", "vs")}
    q = c.run(freqs)
    want, tol = turned(np64(c.q), np.concatenate([np.arange(20), np.arange(35, 40), np.arange(33)]), freqs.cpu().numpy(), False, 1.0, False)
    within(np64(q), want, tol, True, "q")
    page1, page2 = int(c.table[0, 1]), int(c.table[2, 0])
    for x in ("k", "v"):
        for p in (page1, page2):
            assert np.array_equal(raw(getattr(c, x))[p], raw(before[x])[p])
    assert c.layer.read_flags(device=c.q.device) == 1
    # Lengths out of range, offsets that run backwards, more rows than tokens.
    c = Case(torch, kv, 4, 2, 64, [20, 40, 33, 18], [4, 5, 6, 7], seed=2)
    c.seq_lens[1] = 10 ** 6
    c.seq_lens[2] = 4
    out = torch.full_like(c.q.contiguous(), 3.0)
    c.run(freqs, out=out)
    assert (out[4:9] == 3).all() and (out[9:11] == 3).all() and not (out[:4] == 3).all() and not (out[11:15] == 3).all()
    assert c.layer.read_flags(device=c.q.device) == 2
    c = Case(torch, kv, 4, 2, 64, [20, 40, 33], [4, 5, 6], seed=2)
    c.q_start[1] = 10 ** 6
    c.run(freqs)
    assert c.layer.read_flags(device=c.q.device) & 2


def test_refusals(torch):
    from paper_2607_09207_amd import RldaError, rotary_frequencies, rotate
    freqs, _ = rotary_frequencies(64)
    x = torch.randn((4, 2, 64), device="cuda")
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    bad = [lambda: rotate(x.half(), pos, freqs), lambda: rotate(x.cpu(), pos, freqs), lambda: rotate(x, pos.long(), freqs),
           lambda: rotate(x, pos[:3], freqs), lambda: rotate(x, pos, freqs.float()), lambda: rotate(x, pos, freqs[:5]),
           lambda: rotate(x, pos, torch.cat([freqs, freqs])), lambda: rotate(x[..., ::2], pos, freqs[:16]),
           lambda: rotate(x[..., 1:], pos, freqs[:16]), lambda: rotate(x, pos, freqs, out=x.bfloat16()),
           lambda: rotate(x, pos, freqs, out=x[:1].expand(4, 2, 64)), lambda: rotate(x, pos, freqs, amplitude=float("nan")),
           lambda: rotate(torch.randn((4, 300, 64), device="cuda"), pos, freqs),
           lambda: rotate(torch.randn((4, 2, 24), device="cuda"), pos, freqs[:8])]
    for i, f in enumerate(bad):
        with pytest.raises(RldaError):
            f()
            print("taken:", i)
    c = Case(torch, "bf16", 4, 2, 64, [20, 5], None)
    kw = dict(k_scale=None, v_scale=None)
    args = (c.q, c.k_new, c.v_new, c.k, c.v, c.block_table, c.seq_lens, freqs)
    for at, wrong in ((0, c.q[:1]), (1, c.k_new.float()), (2, c.v_new[..., :32]), (3, c.k.float()), (4, c.k), (5, c.block_table[:1]),
                      (6, c.seq_lens.long()), (7, freqs.float())):
        with pytest.raises(RldaError):
            c.layer.append_rotary(*args[:at], wrong, *args[at + 1:], **kw)
    with pytest.raises(RldaError):
        c.layer.append_rotary(*args, q_start=torch.zeros(5, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
@pytest.mark.parametrize("rows", [None, [3, 2]], ids=["one", "chunks"])
def test_append_rotary_derivatives_and_versions(torch, rows, native):
    """Rows whose gradient or tangent would be lost are refused, before anything is written; a
    saved tensor turned in place is noticed."""
    import torch.autograd.forward_ad as fwd

    from paper_2607_09207_amd import RldaError, _abi, rotary_frequencies
    freqs, _ = rotary_frequencies(64)
    c = Case(torch, "bf16", 4, 2, 64, [20, 35], rows, seed=3)
    c.layer.workspace(c.q.device)
    if not native:
        c.layer._fast = _abi.LEFT_TO_PYTHON
    k, v = c.k.clone(), c.v.clone()
    for name in ("q", "k_new", "v_new"):
        plain = getattr(c, name)
        setattr(c, name, plain.clone().requires_grad_())
        with pytest.raises(RldaError, match=f"{name} gets no gradient"):
            c.run(freqs)
        with fwd.dual_level():
            setattr(c, name, fwd.make_dual(plain.clone(), torch.ones_like(plain)))
            with pytest.raises(RldaError, match=f"{name} gets no gradient"):
                c.run(freqs)
        setattr(c, name, plain)
    leaf = torch.empty_like(c.q).requires_grad_()
    with pytest.raises(RldaError, match="out gets no gradient"):
        c.run(freqs, out=leaf)
    assert torch.equal(c.k, k) and torch.equal(c.v, v)
    want = c.run(freqs)
    with torch.no_grad():   # no derivatives are asked for here
        c.q = c.q.clone().requires_grad_()
        assert torch.equal(c.run(freqs), want) and c.run(freqs, out=leaf) is leaf and torch.equal(leaf, want)
    c.q = c.q.detach()
    w = torch.ones_like(c.q).requires_grad_()
    y = w * c.q
    assert torch.equal(c.run(freqs, out=c.q), want)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    with torch.inference_mode():
        z = want + 1
        c.q = z
        assert c.run(freqs, out=z) is z


def test_other_stream_and_graph(torch):
    """A call on another stream, and one captured and replayed, with eager work between."""
    from paper_2607_09207_amd import rotary_frequencies
    freqs, _ = rotary_frequencies(128)
    a, b, g = (Case(torch, "fp8", 12, 2, 128, [100, 33, 7], [60, 2, 7], seed=5) for _ in range(3))
    qa = a.run(freqs)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    qb = b.run(freqs, stream=st)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(qa, qb) and np.array_equal(raw(a.k), raw(b.k)) and torch.equal(a.ks, b.ks)
    g.layer.workspace(g.q.device)
    out = torch.empty_like(qa)
    k0, ks0 = g.k.clone(), g.ks.clone()
    v0, vs0 = g.v.clone(), g.vs.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.run(freqs, out=out)
    for _ in range(3):
        g.k.copy_(k0), g.ks.copy_(ks0), g.v.copy_(v0), g.vs.copy_(vs0)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, qa) and np.array_equal(raw(a.k), raw(g.k)) and np.array_equal(raw(a.v), raw(g.v))
        assert torch.equal(a.vs, g.vs)
