"""Refusals of the entry points for a cache that is read and kept in part, without a GPU: every
check comes before any HIP call, so all of this runs on the CPU, with addresses that nothing
reads.  And the sizes of their workspace."""
import ctypes

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
    made["long"] = create(lib, cfg(num_q_heads=8, num_kv_heads=2, max_batch=16, max_pages_per_seq=32769))
    made["wide"] = create(lib, cfg(num_q_heads=8, num_kv_heads=8, max_batch=16, max_pages_per_seq=1 << 20))
    assert all(st == 0 for st, _ in made.values())
    yield {k: h for k, (_, h) in made.items()}
    for _, h in made.values():
        lib.rl_decode_attn_destroy(h)


def run_bytes(lib, h):  # noqa: F811
    n = ctypes.c_size_t()
    assert lib.rl_decode_attn_workspace_size(h, ctypes.byref(n)) == 0
    return n.value


def weighed_bytes(lib, h, rows):  # noqa: F811
    n = ctypes.c_size_t()
    assert lib.rl_decode_attn_weighed_workspace_size(h, rows, ctypes.byref(n)) == 0
    return n.value


def page_bytes(lib, h, pages):  # noqa: F811
    n = ctypes.c_size_t()
    assert lib.rl_decode_attn_page_workspace_size(h, pages, ctypes.byref(n)) == 0
    return n.value


def check(call, base, invalid, unsupported=(), ok=()):
    for kws, want in ((invalid, INVALID), (unsupported, UNSUPPORTED), ([dict(ws=None), dict(ws=P + 128), dict(bytes=0),
                                                                       dict(bytes=base["bytes"] - 1)], WORKSPACE), (ok, 0)):
        for kw in kws:
            assert call(*dict(base, **kw).values()) == want, (kw, want)


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_page_bounds_refuses(lib, handles, kv):  # noqa: F811
    h = handles[kv]
    base = dict(h=h, batch=4, pages=10, k=P, ks=P, table=P, lens=P, first=P, bounds=P, scale=P, ws=P, bytes=run_bytes(lib, h), stream=None)
    bad = [dict(h=None), dict(batch=-1), dict(batch=17), dict(pages=-1), dict(k=None), dict(k=P + 8), dict(table=None), dict(lens=None),
           dict(table=P + 2), dict(lens=P + 1), dict(first=P + 2), dict(bounds=None), dict(bounds=P + 8), dict(scale=None), dict(scale=P + 1)]
    if kv == "fp8":
        bad += [dict(ks=None), dict(ks=P + 2)]
    check(lib.rl_decode_attn_page_bounds, base, bad, ok=[dict(batch=0), dict(batch=0, k=None, table=None, bounds=None, ws=None)])


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_select_pages_refuses(lib, handles, kv):  # noqa: F811
    h = handles[kv]
    base = dict(h=h, batch=4, pages=10, total=4, budget=6, sink=1, recent=2, q=P, bounds=P, scale=P, table=P, lens=P, q_start=None,
                out=P, counts=P, ws=P, bytes=run_bytes(lib, h), stream=None)
    bad = [dict(h=None), dict(batch=-1), dict(batch=17, total=17), dict(pages=-1), dict(total=-1), dict(total=3), dict(budget=0), dict(budget=2),
           dict(sink=-1), dict(recent=0), dict(recent=-5), dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1), dict(q=None), dict(q=P + 4),
           dict(bounds=None), dict(bounds=P + 4), dict(scale=None), dict(scale=P + 2), dict(table=None), dict(lens=None), dict(table=P + 1),
           dict(lens=P + 2), dict(q_start=P + 2, total=9), dict(out=None), dict(counts=None), dict(out=P + 2), dict(counts=P + 1)]
    check(lib.rl_decode_attn_select_pages, base, bad, [dict(h=handles["long"], bytes=run_bytes(lib, handles["long"])),
                                                       dict(total=2 ** 31 - 1, q_start=P), dict(budget=2 ** 24 + 1), dict(budget=2 ** 31 - 1)],
          [dict(batch=0, total=0), dict(batch=0, total=0, q=None, bounds=None, table=None, out=None, ws=None), dict(total=0, q_start=P)])


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_run_selected_refuses(lib, handles, kv):  # noqa: F811
    h, w = handles[kv], handles["wide"]
    base = dict(h=h, batch=4, pages=10, total=4, budget=6, list=P, counts=P, q=P, k=P, v=P, ks=P, vs=P, table=P, lens=P, q_start=None, out=P,
                ws=P, bytes=run_bytes(lib, h), stream=None, e0=None, e1=None)
    bad = [dict(h=None), dict(batch=-1), dict(batch=17, total=17), dict(pages=-1), dict(total=-1), dict(total=3), dict(budget=0),
           dict(budget=-4), dict(list=None), dict(counts=None), dict(list=P + 2), dict(counts=P + 1), dict(q=None), dict(q=P + 8), dict(k=None),
           dict(v=None), dict(k=P + 8), dict(v=P + 4), dict(table=None), dict(lens=None), dict(table=P + 1), dict(lens=P + 2),
           dict(q_start=P + 2), dict(out=None), dict(out=P + 4), dict(e0=P), dict(e1=P)]
    if kv == "fp8":
        bad += [dict(ks=None), dict(vs=None), dict(ks=P + 2)]
    check(lib.rl_decode_attn_run_selected, base, bad,
          [dict(total=4097, q_start=P), dict(total=2 ** 31 - 1, q_start=P),
           dict(h=w, budget=1 << 20, total=300, q_start=P, bytes=run_bytes(lib, w))],
          [dict(batch=0, total=0), dict(batch=0, total=0, q=None, k=None, table=None, list=None, ws=None), dict(total=0, q_start=P)])


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_run_weighed_refuses(lib, handles, kv):  # noqa: F811
    h, w = handles[kv], handles["wide"]
    base = dict(h=h, batch=4, pages=10, total=4, weights=P, decay=0.5, q=P, k=P, v=P, ks=P, vs=P, table=P, lens=P, q_start=None, out=P, ws=P,
                bytes=weighed_bytes(lib, h, 4), stream=None, e0=None, e1=None)
    bad = [dict(h=None), dict(batch=-1), dict(batch=17, total=17), dict(pages=-1), dict(total=-1), dict(total=3), dict(weights=None),
           dict(weights=P + 2), dict(decay=-0.001), dict(decay=1.001), dict(decay=float("nan")), dict(q=None), dict(k=None), dict(v=P + 8),
           dict(table=None), dict(lens=P + 1), dict(out=None), dict(out=P + 8), dict(e0=P), dict(e1=P)]
    if kv == "fp8":
        bad += [dict(ks=None), dict(vs=P + 2)]
    check(lib.rl_decode_attn_run_weighed, base, bad, [dict(total=4097, q_start=P), dict(h=w, total=300, q_start=P)],
          [dict(batch=0, total=0), dict(batch=0, total=0, weights=None, q=None, ws=None), dict(total=0, q_start=P), dict(batch=0, total=0, decay=1.0)])
    assert lib.rl_decode_attn_run_weighed(*dict(base, bytes=run_bytes(lib, h)).values()) == WORKSPACE


def test_weighed_workspace_size(lib, handles):  # noqa: F811
    n = ctypes.c_size_t()
    f = lib.rl_decode_attn_weighed_workspace_size
    h = handles["bf16"]
    assert f(None, 4, ctypes.byref(n)) == INVALID and f(h, -1, ctypes.byref(n)) == INVALID and f(h, 4, None) == INVALID
    assert f(h, 4097, ctypes.byref(n)) == UNSUPPORTED
    sizes = [weighed_bytes(lib, h, r) for r in (0, 1, 2, 100, 4096)]
    assert all(s % 256 == 0 for s in sizes) and sizes == sorted(sizes) and sizes[0] >= run_bytes(lib, h)
    assert sizes[4] >= run_bytes(lib, h) + 4096 * 8 * 9 * 4   # every row's pages, and its own


def test_page_evict_refuses(lib, handles):  # noqa: F811
    h = handles["bf16"]
    base = dict(h=h, batch=4, pages=10, refs=P, table=P, lens=P, weights=P, budget=6, sink=1, recent=2, dropped=P, ws=P,
                bytes=page_bytes(lib, h, 10), stream=None)
    bad = [dict(h=None), dict(batch=-1), dict(batch=17), dict(pages=-1), dict(refs=None), dict(table=None), dict(lens=None), dict(refs=P + 1),
           dict(table=P + 2), dict(lens=P + 1), dict(weights=None), dict(weights=P + 2), dict(dropped=None), dict(dropped=P + 1), dict(budget=0),
           dict(budget=2), dict(sink=-1), dict(recent=0), dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1)]
    check(lib.rl_decode_attn_page_evict, base, bad, [dict(h=handles["long"], bytes=page_bytes(lib, handles["long"], 10))],
          [dict(batch=0), dict(batch=0, weights=None, dropped=None, table=None, lens=None)])


def test_rising_rows_make_few_workspaces(monkeypatch):
    """What a layer keeps of the weights' workspaces, live and outgrown, is a small multiple of the
    largest call's, however the calls' rows rise; the first one is made to measure."""
    import torch

    from paper_2607_09207_amd import DecodeAttention
    layer = DecodeAttention(8, 2, 128, 16, 64, "bf16", "bf16", "f32")
    made = []

    def zeroed(nbytes, device):
        made.append(nbytes)
        return torch.empty(nbytes, dtype=torch.uint8)

    monkeypatch.setattr(layer, "_zeroed", zeroed)
    size = lambda rows: weighed_bytes(layer._lib, layer._h, rows) + 256   # noqa: E731
    for rows in range(30, 700):
        ws = layer.weighed_workspace(rows, "cuda:0")
        assert ws.numel() >= size(rows) and layer.weighed_workspace(rows - 7, "cuda:0") is ws
    plain = size(0)   # of which a call without rows has one
    assert made[0] == size(30) and len(made) <= 6 and sum(n - plain for n in made) <= 4 * (size(699) - plain)
    assert layer.weighed_workspace(4096, "cuda:0").numel() == size(4096)
    layer.weighed_workspace(3, "cuda:1")   # another device's: to measure again
    assert made[-1] == size(3)
    made.clear()
    for rows in (2100, 2200, 4096):   # never beyond what a call may have
        layer.weighed_workspace(rows, "cuda:2")
    assert made == [size(2100), size(4096)]


def test_flags_of_weights_need_a_workspace():
    from paper_2607_09207_amd import DecodeAttention, RldaError
    layer = DecodeAttention(8, 2, 128, 16, 64, "bf16", "bf16", "f32")
    with pytest.raises(RldaError, match="weighed_flags"):
        layer.weighed_flags("cuda:0")
