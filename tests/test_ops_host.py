"""Refusals of the rotary, page and modified-score entry points that need no GPU: every check
comes before any HIP call, so all of this runs on the CPU, with addresses that nothing
reads.  And the frequencies, which are host arithmetic."""
import ctypes
import math

import pytest

from paper_2607_09207_amd import _abi
from test_abi_host import cfg, create, lib  # noqa: F401  (the fixture)

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -4
P = 1 << 20   # an aligned address


@pytest.fixture(scope="module")
def handles(lib):  # noqa: F811
    made = {kv: create(lib, cfg(num_q_heads=8, num_kv_heads=2, max_batch=16, max_pages_per_seq=8, kv_dtype=code))
            for kv, code in (("bf16", _abi.RLDA_BF16), ("fp8", _abi.RLDA_FP8_E4M3FN))}
    made["f32"] = create(lib, cfg(num_q_heads=2, num_kv_heads=2, max_batch=16, max_pages_per_seq=8, head_dim=64, q_dtype=0, kv_dtype=0,
                                  out_dtype=0))
    assert all(st == 0 for st, _ in made.values())
    yield {k: h for k, (_, h) in made.items()}
    for _, h in made.values():
        lib.rl_decode_attn_destroy(h)


def rows(data=P, r=1024, h=128):
    return _abi.Rows(data, r, h)


def rotary(**kw):
    a = dict(freqs=P, rot_dim=128, interleaved=0, amplitude=1.0, inverse=0)
    a.update(kw)
    return _abi.Rotary(*[a[k] for k, _ in _abi.Rotary._fields_])


def rotate(lib, **kw):  # noqa: F811
    a = dict(dtype=1, rows=4, heads=8, d=128, x=rows(), pos=P, rot=rotary(), out=rows(), stream=None)
    a.update(kw)
    ref = lambda s: None if s is None else ctypes.byref(s)   # noqa: E731
    return lib.rl_decode_attn_rotate(a["dtype"], a["rows"], a["heads"], a["d"], ref(a["x"]), a["pos"], ref(a["rot"]), ref(a["out"]),
                                     a["stream"])


def test_rotate_refuses(lib):  # noqa: F811
    inf, nan = float("inf"), float("nan")
    for kw in (dict(dtype=7), dict(rows=-1), dict(heads=-1), dict(x=None), dict(out=None), dict(rot=None), dict(pos=None), dict(pos=P + 2),
               dict(x=rows(P + 8)), dict(x=rows(r=1025)), dict(x=rows(h=4)), dict(x=rows(r=-1024)), dict(out=rows(P + 2)),
               dict(out=rows(r=0)), dict(out=rows(r=512)), dict(out=rows(h=64)), dict(out=rows(r=128, h=128)), dict(x=rows(None)),
               dict(rot=rotary(freqs=None)), dict(rot=rotary(freqs=P + 4)), dict(rot=rotary(rot_dim=0)), dict(rot=rotary(rot_dim=24)),
               dict(rot=rotary(rot_dim=144)), dict(rot=rotary(rot_dim=-16)), dict(rot=rotary(amplitude=inf)),
               dict(rot=rotary(amplitude=nan)), dict(dtype=0, x=rows(h=130))):
        assert rotate(lib, **kw) == INVALID, kw
    for kw in (dict(dtype=2), dict(heads=257), dict(d=24), dict(d=264), dict(d=132), dict(rows=2 ** 31 - 1)):
        assert rotate(lib, **kw) == UNSUPPORTED, kw
    assert rotate(lib, rows=0) == 0 and rotate(lib, heads=0) == 0 and rotate(lib, rows=0, x=None, pos=None, out=None) == 0


def append(lib, handle, **kw):  # noqa: F811
    n = ctypes.c_size_t()
    lib.rl_decode_attn_workspace_size(handle, ctypes.byref(n))
    a = dict(h=handle, batch=4, pages=10, total=4, rot=rotary(rot_dim=64), q=rows(), k=rows(), v=rows(), q_start=None, pos=None, kc=P, vc=2 * P,
             ks=P, vs=2 * P, table=P, lens=P, out=rows(), ws=P, bytes=n.value, stream=None)
    a.update(kw)
    ref = lambda s: None if s is None else ctypes.byref(s)   # noqa: E731
    return lib.rl_decode_attn_append_rotary(a["h"], a["batch"], a["pages"], a["total"], ref(a["rot"]), ref(a["q"]), ref(a["k"]), ref(a["v"]),
                                            a["q_start"], a["pos"], a["kc"], a["vc"], a["ks"], a["vs"], a["table"], a["lens"],
                                            ref(a["out"]), a["ws"], a["bytes"], a["stream"])


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_append_rotary_refuses(lib, handles, kv):  # noqa: F811
    h = handles[kv]
    bad = [dict(h=None), dict(batch=-1), dict(batch=17, total=17), dict(pages=-1), dict(total=-1), dict(total=3), dict(rot=None),
           dict(rot=rotary(rot_dim=144)), dict(q=None), dict(k=rows(P + 4)), dict(v=rows(h=2)), dict(out=rows(r=0)), dict(out=None),
           dict(table=None), dict(lens=None), dict(table=P + 1), dict(lens=P + 2), dict(q_start=P + 2), dict(pos=P + 1), dict(kc=None),
           dict(vc=None), dict(kc=P, vc=P), dict(kc=P + 8)]
    if kv == "fp8":
        bad += [dict(ks=None), dict(vs=None), dict(ks=P, vs=P), dict(vs=P + 2)]
    for kw in bad:
        assert append(lib, h, **kw) == INVALID, kw
    for kw in (dict(ws=None), dict(ws=P + 128), dict(bytes=0)):
        assert append(lib, h, **kw) == WORKSPACE, kw
    assert append(lib, h, batch=0, total=0) == 0 and append(lib, h, batch=0, total=0, q=None, table=None, ws=None) == 0
    assert append(lib, h, total=0, q_start=P) == 0
    assert append(lib, h, total=2 ** 31 - 1, q_start=P) == UNSUPPORTED


def page_bytes(lib, h, pages):  # noqa: F811
    n = ctypes.c_size_t()
    assert lib.rl_decode_attn_page_workspace_size(h, pages, ctypes.byref(n)) == 0
    return n.value


def test_page_workspace(lib, handles):  # noqa: F811
    h = handles["bf16"]
    n = ctypes.c_size_t()
    f = lib.rl_decode_attn_page_workspace_size
    assert f(None, 5, ctypes.byref(n)) == INVALID and f(h, -1, ctypes.byref(n)) == INVALID and f(h, 5, None) == INVALID
    sizes = [page_bytes(lib, h, p) for p in (0, 1, 100, 131072, 131073, 10 ** 6, 2 ** 31 - 1)]
    assert all(s % 256 == 0 for s in sizes) and sizes == sorted(sizes)


def test_page_operations_refuse(lib, handles):  # noqa: F811
    h = handles["fp8"]
    ws = page_bytes(lib, h, 10)
    caches = (_abi.Cache * 2)(_abi.Cache(P, P, P, P), _abi.Cache(P, P, P, P))
    state = dict(h=h, batch=4, pages=10, refs=P, table=P, lens=P)
    end = dict(ws=P, bytes=ws, stream=None)
    ops = {
        "grow": (lib.rl_decode_attn_page_grow, dict(state, add=P, **end), [dict(add=P + 2)], [dict(batch=0, table=None, lens=None)]),
        "release": (lib.rl_decode_attn_page_release, dict(state, count=2, rows=P, **end), [dict(count=-1), dict(rows=None), dict(rows=P + 1)],
                    [dict(count=0), dict(count=0, rows=None)]),
        "fork": (lib.rl_decode_attn_page_fork, dict(state, count=2, parents=P, children=P, n=2, caches=caches, **end),
                 [dict(count=-1), dict(count=17), dict(parents=None), dict(children=None), dict(children=P + 2), dict(n=-1), dict(caches=None)],
                 [dict(count=0), dict(count=0, parents=None, children=None, n=0, caches=None)]),
        "compact": (lib.rl_decode_attn_page_compact, dict(state, n=2, caches=caches, live=P, **end),
                    [dict(live=None), dict(live=P + 1), dict(n=-1), dict(caches=None)], []),
    }
    for name, (f, base, bad, good) in ops.items():
        call = lambda **kw: f(*{**base, **kw}.values())   # noqa: E731
        for kw in [dict(h=None), dict(batch=-1), dict(batch=17), dict(pages=-1), dict(refs=None), dict(refs=P + 2), dict(table=None),
                   dict(table=P + 1), dict(lens=None), dict(lens=P + 3)] + bad:
            assert call(**kw) == INVALID, (name, kw)
        for kw in (dict(ws=None), dict(ws=P + 64), dict(bytes=ws - 1), dict(pages=10 ** 6)):
            assert call(**kw) == WORKSPACE, (name, kw)
        for kw in good:
            assert call(**kw) == 0, (name, kw)
        if "caches" in base:
            for c in (_abi.Cache(None, P, P, P), _abi.Cache(P, P + 8, P, P), _abi.Cache(P, P, None, P), _abi.Cache(P, P, P, P + 2)):
                assert call(caches=(_abi.Cache * 2)(_abi.Cache(P, P, P, P), c)) == INVALID
    copy = lib.rl_decode_attn_page_copy
    ok = dict(h=h, pages=10, count=2, src=P, dst=P, n=2, caches=caches, **end)
    call = lambda **kw: copy(*{**ok, **kw}.values())   # noqa: E731
    for kw in (dict(h=None), dict(pages=-1), dict(count=-1), dict(src=None), dict(dst=None), dict(src=P + 2), dict(n=-1), dict(caches=None)):
        assert call(**kw) == INVALID, kw
    assert call(ws=None) == WORKSPACE and call(count=0) == 0 and call(n=0, caches=None) == 0
    assert call(count=2 ** 30) == UNSUPPORTED


def scored(lib, handle, **kw):  # noqa: F811
    n = ctypes.c_size_t()
    lib.rl_decode_attn_workspace_size(handle, ctypes.byref(n))
    sc = dict(score_cap=0.0, window=0, slopes=None, key_start=None, prefix_lens=None)
    sc.update({k: kw.pop(k) for k in list(kw) if k in sc})
    a = dict(h=handle, sc=_abi.Scores(*[sc[k] for k, _ in _abi.Scores._fields_]), batch=4, pages=10, total=4, max_q=0, q=P, k=P, v=P, ks=P, vs=P,
             table=P, lens=P, q_start=None, out=P, ws=P, bytes=n.value, stream=None, e0=None, e1=None)
    a.update(kw)
    v = list(a.values())
    v[1] = None if v[1] is None else ctypes.byref(v[1])
    return lib.rl_decode_attn_run_scored(*v)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_scored_refuses(lib, handles, kv):  # noqa: F811
    h = handles[kv]
    inf, nan = float("inf"), float("nan")
    both = [dict(h=None), dict(sc=None), dict(score_cap=-1.0), dict(score_cap=nan), dict(score_cap=inf), dict(score_cap=2.0 ** -11),
            dict(score_cap=2.0 ** 31), dict(window=-1), dict(slopes=P + 2), dict(key_start=P + 1), dict(prefix_lens=P + 3), dict(e0=P),
            dict(e1=P), dict(batch=-1), dict(batch=17, total=17), dict(pages=-1), dict(q=None), dict(q=P + 8), dict(k=None), dict(v=P + 4),
            dict(table=None), dict(lens=P + 1), dict(out=None)]
    if kv == "fp8":
        both += [dict(ks=None), dict(vs=P + 2)]
    for kw in both:
        assert scored(lib, h, **kw) == INVALID, kw
        assert scored(lib, h, **dict(kw, q_start=P)) == INVALID, kw
    for kw in (dict(total=3), dict(total=5), dict(q_start=P, total=-1), dict(q_start=P, max_q=-1), dict(q_start=P + 2)):
        assert scored(lib, h, **kw) == INVALID, kw
    for kw in (dict(ws=None), dict(ws=P + 1), dict(bytes=0)):
        assert scored(lib, h, **kw) == WORKSPACE and scored(lib, h, q_start=P, **kw) == WORKSPACE
    assert scored(lib, h, batch=0, total=0) == 0 and scored(lib, h, q_start=P, total=0) == 0
    assert scored(lib, handles["f32"]) == UNSUPPORTED
    assert scored(lib, h, q_start=P, total=2 ** 31 - 1) == UNSUPPORTED


def test_python_refuses_host_tensors():
    import torch

    from paper_2607_09207_amd import DecodeAttention, RldaError, rotary_frequencies, rotate
    h = DecodeAttention(8, 2, 128, 4, 8, "bf16", "bf16", "bf16")
    q = torch.zeros((2, 8, 128), dtype=torch.bfloat16)
    kn = torch.zeros((2, 2, 128), dtype=torch.bfloat16)
    k = torch.zeros((5, 2, 16, 128), dtype=torch.bfloat16)
    bt, sl, refs = torch.zeros((2, 8), dtype=torch.int32), torch.ones(2, dtype=torch.int32), torch.zeros(5, dtype=torch.int32)
    f, _ = rotary_frequencies(128, device="cpu")
    one = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: rotate(q, sl, f), lambda: h.append_rotary(q, kn, kn, k, k.clone(), bt, sl, f), lambda: h.scored(q, k, k, bt, sl),
                 lambda: h.page_grow(refs, bt, sl), lambda: h.page_release(refs, bt, sl, one), lambda: h.page_fork(refs, bt, sl, one, one),
                 lambda: h.page_compact(refs, bt, sl), lambda: h.page_copy(one, one, [(k, k)]), lambda: h.caches([(k, k)])):
        with pytest.raises(RldaError, match="must be on|a GPU"):
            call()


def test_a_set_of_another_layer():
    """A set holds addresses: a layer whose pages differ refuses it (here before it looks at
    the lists, so without a GPU)."""
    import torch

    from paper_2607_09207_amd import DecodeAttention, RldaError
    from paper_2607_09207_amd.cache_ops import CacheSet
    bf16 = DecodeAttention(8, 2, 128, 4, 8, "bf16", "bf16", "bf16")
    same = DecodeAttention(4, 2, 128, 9, 3, "bf16", "bf16", "f32")
    k = torch.zeros((5, 2, 16, 128), dtype=torch.bfloat16)
    cs = CacheSet([(k, k)], (_abi.Cache * 1)(), 5, k.device, bf16._geometry)
    one = torch.zeros(1, dtype=torch.int32)
    for other in (DecodeAttention(8, 2, 128, 4, 8, "bf16", "fp8_e4m3fn", "bf16"), DecodeAttention(8, 4, 128, 4, 8),
                  DecodeAttention(8, 2, 64, 4, 8), DecodeAttention(8, 2, 128, 4, 8, kv_strides=(4096, 128, 256))):
        with pytest.raises(RldaError, match="caches are of"):
            other.page_copy(one, one, cs)
        with pytest.raises(RldaError, match="caches are of"):
            other._check_set("page_fork", cs)
    assert same._check_set("page_fork", cs) is cs


def test_frequencies():
    import torch

    from paper_2607_09207_amd import rotary_frequencies as F
    f, a = F(64, 1e4, device="cpu")
    assert f.dtype == torch.float64 and a == 1.0 and f.shape == (32,)
    for j in range(32):
        assert f[j] == pytest.approx(1e4 ** (-2 * j / 64), rel=1e-14)
    g, a = F(64, 1e4, {"type": "linear", "factor": 4.0}, "cpu")
    assert a == 1.0 and torch.allclose(g * 4, f, rtol=1e-14)
    g, a = F(64, 1e4, {"type": "base", "factor": 8.0}, "cpu")
    assert a == 1.0 and g[0] == 1.0 and g[-1] * 8 == pytest.approx(float(f[-1]), rel=1e-12) and (g[1:] < f[1:]).all()
    how = {"type": "ramp", "factor": 16.0, "context": 4096, "fast": 32, "slow": 1}
    g, a = F(64, 1e4, how, "cpu")
    assert a == pytest.approx(0.1 * math.log(16) + 1)
    turns = 4096 * f / (2 * math.pi)
    j = torch.arange(32)
    lo = math.floor(32 * math.log(4096 / (2 * math.pi * 32)) / math.log(1e4))
    hi = math.ceil(32 * math.log(4096 / (2 * math.pi)) / math.log(1e4))
    assert torch.equal(g[j <= lo], f[j <= lo]) and torch.allclose(g[j >= hi] * 16, f[j >= hi], rtol=1e-14)
    assert (turns[:lo] > 32).all() and (turns[hi + 1:] < 1).all()
    mid = (j > lo) & (j < hi)
    assert mid.any() and (g[mid] < f[mid]).all() and (g[mid] * 16 > f[mid]).all() and (g[1:] < g[:-1]).all()
    assert F(64, 1e4, dict(how, amplitude=1.0), "cpu")[1] == 1.0
    assert F(2, 1e4, device="cpu")[0].tolist() == [1.0]
    for bad in (lambda: F(0), lambda: F(7), lambda: F(64, 1.0), lambda: F(64, 1e4, {"type": "else", "factor": 2}),
                lambda: F(64, 1e4, {"type": "linear", "factor": 0}), lambda: F(64, 1e4, dict(how, fast=1, slow=2)),
                lambda: F(64, 1e4, dict(how, context=0))):
        with pytest.raises(ValueError):
            bad()


def test_ramp_of_short_contexts():
    """A pair that turns `slow` times or less over the context is slowed down, the first one too."""
    import torch

    from paper_2607_09207_amd import rotary_frequencies as F
    f, _ = F(64, 1e4, device="cpu")
    for n in (1, 6, 6.28, 7, 30, 200):
        g, _ = F(64, 1e4, {"type": "ramp", "factor": 16.0, "context": n, "fast": 32, "slow": 1}, "cpu")
        turns = n * f / (2 * math.pi)
        slow = turns <= 1
        at = 32 * math.log(n / (2 * math.pi)) / math.log(1e4)   # the pair that turns once
        slow &= torch.arange(32) >= math.ceil(at)
        assert slow.any() and torch.allclose(g[slow] * 16, f[slow], rtol=1e-14)
        assert (g <= f).all() and (g * 16 >= f * (1 - 1e-14)).all() and (g[1:] < g[:-1]).all()


def test_sizes_beyond_a_launch(lib, handles):  # noqa: F811
    """What one launch cannot hold is refused before it."""
    assert rotate(lib, rows=2 ** 27 + 1) == UNSUPPORTED
    h = handles["bf16"]
    assert append(lib, h, total=2 ** 27 + 1, q_start=P) == UNSUPPORTED
    # 2^23 windows of two workgroups (rows and pages) and more.
    assert append(lib, handles["fp8"], total=2 ** 27, q_start=P) == UNSUPPORTED
    ws = page_bytes(lib, h, 10)
    assert lib.rl_decode_attn_page_release(h, 4, 10, P, P, P, 2 ** 23 + 1, P, P, ws, None) == UNSUPPORTED


def test_scored_rows_of_large_batches(lib):  # noqa: F811
    st, h = create(lib, cfg(num_q_heads=8, num_kv_heads=2, max_batch=8192, max_pages_per_seq=8, kv_dtype=_abi.RLDA_BF16))
    assert st == 0
    for mq in (0, 1, 4, 100):
        assert scored(lib, h, batch=4097, total=4097, q_start=P, max_q=mq) == UNSUPPORTED
    lib.rl_decode_attn_destroy(h)
