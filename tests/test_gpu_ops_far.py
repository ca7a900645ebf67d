"""Rotary appends, page operations and modified scores where offsets pass 32 bits, and with
workspaces that captured graphs share.

The far calls are the near ones with their pages at the end of a pool of more than 2^31
elements and 2^32 bytes, so results are compared bit for bit with those of a small pool.
"""
import numpy as np
import pytest

from test_gpu_rotary import Case as RotaryCase
from test_gpu_rotary import raw
from test_gpu_scored import Case as ScoredCase

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_09207_amd import _abi
    _abi.load()
    return torch


def far(torch, t, pages):
    """A pool of `pages` whose last ones hold t; the others are not written."""
    out = torch.empty((pages,) + tuple(t.shape[1:]), dtype=t.dtype, device=t.device)
    out[pages - len(t):] = t
    return out


def pages_past_32_bits(t):
    per = t[0].numel()
    return max(2 ** 31 // per, 2 ** 32 // (per * t.element_size())) + 2 * len(t)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("rows,kw", [(None, {}), ([4, 2, 1], dict(max_q_len=4)), ([300, 2, 70], {})])
def test_scored_far_pages(torch, kv, rows, kw):
    c = ScoredCase(torch, kv, 16, 4, 128, [900, 33, 70], rows, seed=2)
    mod = c.mods(3)[-1]
    want = c.run(mod, **kw)
    n = pages_past_32_bits(c.k)
    off = n - len(c.k)
    k, v = far(torch, c.k, n), far(torch, c.v, n)
    ks, vs = (None, None) if c.ks is None else (far(torch, c.ks, n), far(torch, c.vs, n))
    table = torch.where(c.block_table >= 0, c.block_table + off, c.block_table)
    got = c.layer.scored(c.q, k, v, table, c.seq_lens, q_start=c.q_start, k_scale=ks, v_scale=vs, **mod, **kw)
    assert torch.equal(got, want) and got.isfinite().all()
    assert c.layer.read_flags(device=c.q.device) == 0


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_append_far_pages(torch, kv):
    from paper_2607_09207_amd import rotary_frequencies
    freqs, _ = rotary_frequencies(128)
    c = RotaryCase(torch, kv, 4 if kv == "f32" else 8, 4, 128, [100, 33, 7], [60, 2, 7], seed=5)
    n = pages_past_32_bits(c.k)
    off = n - len(c.k)
    k, v = far(torch, c.k, n), far(torch, c.v, n)
    ks, vs = (None, None) if c.ks is None else (far(torch, c.ks, n), far(torch, c.vs, n))
    table = torch.where(c.block_table >= 0, c.block_table + off, c.block_table)
    want = c.run(freqs)
    got = c.layer.append_rotary(c.q, c.k_new, c.v_new, k, v, table, c.seq_lens, freqs, q_start=c.q_start, k_scale=ks, v_scale=vs)
    assert torch.equal(got, want)
    assert np.array_equal(raw(k[off:]), raw(c.k)) and np.array_equal(raw(v[off:]), raw(c.v))
    if ks is not None:
        assert torch.equal(ks[off:], c.ks) and torch.equal(vs[off:], c.vs)


def test_page_contents_far(torch):
    """Copies, forks and moves between the ends of a pool."""
    from paper_2607_09207_amd import DecodeAttention
    n = 2 ** 31 // (4 * 16 * 128) + 100
    layer = DecodeAttention(4, 4, 128, 4, 8, "bf16", "bf16", "bf16")
    k, v = (torch.empty((n, 4, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    for j in (0, 1, 2, n - 2, n - 1):
        k[j], v[j] = j % 251, j % 241 + 1000
    is_page = lambda at, j: bool((k[at] == j % 251).all() and (v[at] == j % 241 + 1000).all())   # noqa: E731
    layer.page_copy(i32([0, n - 1]), i32([n - 3, 3]), [(k, v)])
    assert is_page(n - 3, 0) and is_page(3, n - 1)
    # Every page but n - 5 is taken: the fork's copy of page n - 1 goes there.
    refs = torch.ones(n, dtype=torch.int32, device="cuda")
    refs[n - 5] = 0
    table, lens = i32([[n - 2, n - 1] + [0] * 6, [0] * 8]), i32([20, 0])
    layer.page_fork(refs, table, lens, i32([0]), i32([1]), [(k, v)])
    assert table[1, :2].tolist() == [n - 2, n - 5] and lens.tolist() == [20, 20] and is_page(n - 5, n - 1)
    assert refs[n - 2] == 2 and refs[n - 5] == 1
    # Three pages are live, and move to the front.
    refs.zero_()
    refs[n - 5], refs[n - 2], refs[n - 1] = 1, 2, 1
    live = layer.page_compact(refs, table, lens, [(k, v)])
    assert live.item() == 3 and refs[:4].tolist() == [1, 2, 1, 0] and int(refs.sum()) == 4
    assert table[:, :2].tolist() == [[1, 2], [1, 0]] and is_page(0, n - 1) and is_page(1, n - 2) and is_page(2, n - 1)
    assert layer.page_flags(n, k.device) == 0


def test_rotate_far_rows(torch):
    """Rows past 2^31 elements and 2^32 bytes of x and out: the same as in a call of their own."""
    from paper_2607_09207_amd import rotary_frequencies, rotate
    freqs, _ = rotary_frequencies(128)
    n = 2 ** 31 // (256 * 128) + 40
    x = torch.zeros((n, 256, 128), dtype=torch.bfloat16, device="cuda")
    x[-50:].normal_()
    x[:10].normal_()
    pos = torch.randint(0, 10000, (n,), device="cuda", dtype=torch.int32)
    y = rotate(x, pos, freqs)
    assert torch.equal(y[-50:], rotate(x[-50:], pos[-50:], freqs)) and torch.equal(y[:10], rotate(x[:10], pos[:10], freqs))
    assert not y[10:-50].any()


def test_two_graphs_one_workspace(torch):
    """Two graphs of different calls on one layer's workspaces, replayed in turn with eager
    calls between: appends and scored attention, and the page operations."""
    from paper_2607_09207_amd import rotary_frequencies
    freqs, _ = rotary_frequencies(128)
    a = ScoredCase(torch, "fp8", 12, 2, 128, [900, 33, 70, 1500], seed=5, ranges=64)
    b = ScoredCase(torch, "fp8", 12, 2, 128, [1500, 900, 2, 70], [4, 1, 2, 3], seed=6, ranges=64)
    b.layer = a.layer
    mods = a.mods(1)[-1], b.mods(2)[-1]
    layer = a.layer
    dev = a.q.device
    mp = layer.config.max_pages_per_seq
    assert b.block_table.shape[1] == mp
    kws = {}, dict(max_q_len=4)
    want = [c.run(m, **kw) for c, m, kw in zip((a, b), mods, kws)]
    turned = [layer.append_rotary(c.q, c.q[:, :2], c.q[:, 2:4], c.k.clone(), c.v.clone(), c.block_table, c.seq_lens, freqs,
                                  q_start=c.q_start, k_scale=c.ks.clone(), v_scale=c.vs.clone()) for c in (a, b)]
    copies = [(c.k.clone(), c.v.clone(), c.ks.clone(), c.vs.clone()) for c in (a, b)]
    n = 300
    layer.page_workspace(n, dev)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    states = [(torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros((2, mp), dtype=torch.int32, device="cuda"), i32([0, 0]), i32(add))
              for add in ([100, 40], [1, 700])]
    outs, rots, graphs = [torch.empty_like(w) for w in want], [torch.empty_like(t) for t in turned], []
    for i, (c, m, kw) in enumerate(zip((a, b), mods, kws)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.run(m, out=outs[i], **kw)
            k, v, ks, vs = copies[i]
            layer.append_rotary(c.q, c.q[:, :2], c.q[:, 2:4], k, v, c.block_table, c.seq_lens, freqs, q_start=c.q_start, k_scale=ks,
                                v_scale=vs, out=rots[i])
            refs, table, lens, add = states[i]
            layer.page_grow(refs, table, lens, add)
        graphs.append(g)
    for step in range(1, 4):
        for i, c in enumerate((a, b)):
            outs[i].zero_(), rots[i].zero_()
            graphs[i].replay()
            assert torch.equal(c.run(mods[i], **kws[i]), want[i])
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want[i]) and torch.equal(rots[i], turned[i])
            refs, table, lens, add = states[i]
            grown = [step * x if step * x <= mp * 16 else None for x in add.tolist()]
            if None not in grown:
                assert lens.tolist() == grown and int(refs.sum()) == sum(-(-x // 16) for x in grown)
    assert layer.read_flags(device=dev) == 0


def test_extreme_slopes(torch):
    """Slopes up to 2^64 of both signs: each row's nearest or farthest key alone has a part."""
    c = ScoredCase(torch, "bf16", 8, 2, 64, [200, 33, 16, 1])
    slopes = torch.tensor([2.0 ** 64, -2.0 ** 64, 2.0 ** 40, -2.0 ** 40] * 2, device="cuda")
    for rows, few in ((None, True), ([30, 33, 1, 1], False)):
        c = ScoredCase(torch, "bf16", 8, 2, 64, [200, 33, 16, 1], rows)
        got = c.run(dict(slopes=slopes))
        for b, L in enumerate(c.lens):
            _, v = c.dense(b)
            for i in range(int(c.rows[b])):
                pos = int(L) - int(c.rows[b]) + i
                r = int(c.start[b]) + i if rows is not None else b
                for h in range(8):
                    key = pos if h % 2 == 0 else 0
                    assert torch.equal(got[r, h].double(), v[key, h // 4]), (b, i, h)
