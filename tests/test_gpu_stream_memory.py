"""Results that a call on another stream allocates for itself: their memory is neither in use
by what is queued on the current stream, nor given out again while the current stream still
reads it.  Work that holds the current stream back makes that visible where the two streams
run beside each other (streams may share a queue of the GPU: it is printed).
"""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_09207_amd import _abi
    _abi.load()
    return torch


def make_calls(torch):
    """name -> call(stream), the same result every time."""
    from paper_2607_09207_amd import rotary_frequencies, rotate
    from test_gpu_pages import State
    from test_gpu_rotary import Case as Rotary
    from test_gpu_scored import Case as Scored
    freqs, _ = rotary_frequencies(64)
    one = Scored(torch, "bf16", 8, 2, 64, [90, 33, 70], None, seed=1)
    few = Scored(torch, "bf16", 8, 2, 64, [90, 33, 70], [3, 2, 4], seed=1)
    app = Rotary(torch, "bf16", 8, 2, 64, [90, 33, 70], [3, 2, 4], seed=1)
    state = State(torch, 60, [45, 64, 0], 40, layers=1, seed=1)
    x = torch.randn((40, 5, 64), device="cuda")
    pos = torch.arange(40, device="cuda", dtype=torch.int32)
    for c in (one, few, app):
        c.layer.workspace(c.q.device, grouped=True)
    state.layer.page_workspace(60, state.refs.device)
    args = lambda c: (c.q, c.k, c.v, c.block_table, c.seq_lens)   # noqa: E731
    pp = torch.zeros(3, dtype=torch.int32, device="cuda")
    cap = few.mods(0)[1]
    calls = {
        "run": lambda s: one.layer(*args(one), stream=s),
        "grouped": lambda s: one.layer(*args(one), group_size=1, prefix_pages=pp, stream=s),
        "noalloc": lambda s: one.layer.run_noalloc(*args(one), stream=s),
        "multi": lambda s: few.layer.multi(*args(few), few.q_start, stream=s),
        "scored": lambda s: few.run(cap, stream=s),
        "append_rotary": lambda s: app.run(freqs, stream=s),
        "rotate": lambda s: rotate(x, pos, freqs, stream=s),
        "page_compact": lambda s: state.layer.page_compact(*state.args(), state.caches, stream=s),
    }
    layers = [one.layer, few.layer, app.layer, state.layer]
    return calls, layers


NAMES = ["run", "grouped", "noalloc", "multi", "scored", "append_rotary", "rotate", "page_compact"]


@pytest.mark.parametrize("raw", [False, True], ids=["stream", "handle"])
@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
@pytest.mark.parametrize("name", NAMES)
def test_results_on_another_stream(torch, name, native, raw, monkeypatch):
    from paper_2607_09207_amd import _abi
    calls, layers = make_calls(torch)
    if not native:
        for layer in layers:
            layer._fast = _abi.LEFT_TO_PYTHON
        monkeypatch.setattr(_abi, "fastcall", lambda: None)
    call = calls[name]
    current, side = torch.cuda.current_stream(), torch.cuda.Stream()
    on = side.cuda_stream if raw else side
    want = call(None).clone()
    torch.cuda.synchronize()
    assert torch.equal(call(current.cuda_stream if raw else current), want)
    call(on)   # (the other stream has memory enough of its own from here on: taking more may wait for the GPU)
    with torch.cuda.stream(side):
        junk = [torch.full_like(want, 3) for _ in range(40)]
    torch.cuda.synchronize()
    del junk
    # 1. Memory that the current stream is about to write to, freed on the host already.
    busy = [torch.empty_like(want) for _ in range(8)]
    torch.cuda._sleep(20_000_000)
    for t in busy:
        t.fill_(7)
    del busy, t
    got = call(on)
    side.synchronize()
    print("held back:", not current.query(), flush=True)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    # 2. A result that the current stream reads later, freed on the host already.
    keep = torch.empty_like(want)
    current.wait_stream(side)
    torch.cuda._sleep(20_000_000)
    keep.copy_(got)
    del got
    with torch.cuda.stream(side):
        junk = [torch.full_like(want, 3) for _ in range(8)]
    side.synchronize()
    print("held back:", not current.query(), flush=True)
    torch.cuda.synchronize()
    assert torch.equal(keep, want) and len(junk) == 8


def test_the_default_stream_by_its_handle(torch):
    """0 is the default stream, whatever the current one is."""
    calls, _ = make_calls(torch)
    with torch.cuda.stream(torch.cuda.Stream()):
        for name in NAMES:
            a, b = calls[name](0), calls[name](torch.cuda.default_stream())
            torch.cuda.synchronize()
            assert torch.equal(a, b), name


def test_workspaces_are_zero_for_every_stream(torch):
    """A workspace is handed out with its zeros in it, whatever its maker's stream has queued."""
    from paper_2607_09207_amd import DecodeAttention
    layer = DecodeAttention(8, 2, 64, 4, 8)
    dev = torch.device("cuda:0")
    for make in (lambda: layer.workspace(dev), lambda: layer.workspace(dev, grouped=True), lambda: layer.page_workspace(50, dev)):
        torch.cuda._sleep(20_000_000)
        ws = make()
        assert torch.cuda.current_stream().query()
        with torch.cuda.stream(torch.cuda.Stream()):
            assert not ws.any()


def test_a_graph_keeps_its_workspace(torch):
    """A graph captured on the plain workspace, replayed after grouped calls took a larger one."""
    from test_gpu_scored import Case
    c = Case(torch, "bf16", 8, 2, 64, [5000, 33, 3000], None, seed=1)
    want = c.layer(c.q, c.k, c.v, c.block_table, c.seq_lens)
    old = c.layer.workspace(c.q.device)
    size, at = old.numel(), old.data_ptr()
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.layer(c.q, c.k, c.v, c.block_table, c.seq_lens, out=out)
    del old
    pp = torch.zeros(3, dtype=torch.int32, device="cuda")
    c.layer(c.q, c.k, c.v, c.block_table, c.seq_lens, group_size=1, prefix_pages=pp)
    assert c.layer.workspace(c.q.device).numel() > size
    junk = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert all(t.data_ptr() != at for t in junk)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all((t == 255).all() for t in junk)


def test_no_workspace_is_made_in_a_capture(torch):
    from paper_2607_09207_amd import RldaError
    calls, layers = make_calls(torch)
    for layer in layers:
        layer._ws.clear()
        layer._page_ws.clear()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for name in ("run", "grouped", "multi", "scored", "append_rotary", "page_compact"):
            with pytest.raises(RldaError, match="workspace"):
                calls[name](None)
    for name in NAMES:
        calls[name](None)
    torch.cuda.synchronize()
    assert all(layer.read_flags(device="cuda:0") == 0 for layer in layers)
