"""The newer calls by the native path and by the Python path of the binding: the native one
takes ordinary calls, leaves the others, and both give the same bits."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


class Watch:
    """A layer's native path that counts what it takes."""

    def __init__(self, native):
        self.native, self.taken, self.asked = native, 0, 0

    def __getattr__(self, name):
        f = getattr(self.native, name)

        def call(*a):
            got = f(*a)
            self.asked += 1
            self.taken += got is not None
            return got
        return call


def both(layer, f):
    """f() by the native path and by the Python path; whether the native path took it."""
    from paper_2607_09207_amd import _abi
    native = layer._fast
    watch = layer._fast = Watch(native)
    try:
        a = f()
        layer._fast = _abi.LEFT_TO_PYTHON
        b = f()
    finally:
        layer._fast = native
    return a, b, watch


def test_scored_and_append_rotary(torch):
    from test_gpu_rotary import Case as RotaryCase
    from test_gpu_scored import Case as ScoredCase
    from paper_2607_09207_amd import rotary_frequencies
    freqs, _ = rotary_frequencies(64)
    for rows in (None, [3, 2, 4], [30, 2, 40]):
        c = ScoredCase(torch, "fp8", 8, 2, 64, [90, 33, 70], rows, seed=1)
        c.layer.workspace(c.q.device)
        mod = c.mods(0)[-1]
        for kw in (dict(), dict(max_q_len=max(rows) if rows and max(rows) <= 16 else 0), dict(num_pages=c.k.shape[0] - 1)):
            a, b, w = both(c.layer, lambda: c.run(mod, **kw))
            assert w.taken == w.asked == 1 and torch.equal(a, b)
        out = torch.empty_like(a)
        a, b, w = both(c.layer, lambda: c.run(mod, out=out, stream=torch.cuda.current_stream()))
        assert w.taken == 1 and a is out and b is out
        _, _, w = both(c.layer, lambda: c.run(mod, stream=torch.cuda.current_stream()))   # a fresh output on a given stream
        assert w.taken == 0
        r = RotaryCase(torch, "fp8", 8, 2, 64, [90, 33, 70], rows, seed=1)
        r.layer.workspace(r.q.device)
        state = [x.clone() for x in (r.k, r.v, r.ks, r.vs)]
        got = []

        def run():
            for x, y in zip((r.k, r.v, r.ks, r.vs), state):
                x.copy_(y)
            q = r.run(freqs, interleaved=True, amplitude=1.5)
            got.append([x.view(torch.uint8).clone() for x in (r.k, r.v)] + [r.ks.clone(), r.vs.clone()])
            return q
        a, b, w = both(r.layer, run)
        live = slice(None)
        assert w.taken == 1 and torch.equal(a[live], b[live]) and all(torch.equal(x, y) for x, y in zip(*got))


def test_rotate(torch, monkeypatch):
    from paper_2607_09207_amd import _abi, rotary_frequencies, rotate
    freqs, _ = rotary_frequencies(32)
    x = torch.randn((40, 5, 64), device="cuda").bfloat16()
    pos = torch.arange(40, device="cuda", dtype=torch.int32)
    a = rotate(x[:, 1:], pos, freqs, interleaved=True, amplitude=2, inverse=True)
    monkeypatch.setattr(_abi, "fastcall", lambda: None)
    assert torch.equal(a, rotate(x[:, 1:], pos, freqs, interleaved=True, amplitude=2, inverse=True))


def test_pages(torch):
    from test_gpu_pages import State
    runs = []
    for native in (True, False):
        from paper_2607_09207_amd import _abi
        s = State(torch, 300, [45, 64, 0, 0, 0, 100], 40, layers=2, seed=1)
        s.layer.page_workspace(300, "cuda:0")
        w = s.layer._fast = Watch(s.layer._fast) if native else _abi.LEFT_TO_PYTHON
        s.layer.page_fork(*s.args(), s.cuda([0, 1]), s.cuda([2, 3]), s.caches)
        s.layer.page_grow(*s.args(), s.cuda([0, 0, 3, 40, 5, 0]))
        s.layer.page_grow(*s.args())
        s.layer.page_release(*s.args(), s.cuda([5, 0]))
        live = s.layer.page_compact(*s.args(), s.caches)
        runs.append([x.clone() for x in s.args()] + [live] + [t.view(torch.int16) for one in s.tensors for t in one])
        assert not native or w.taken == w.asked == 5
    assert all(torch.equal(a, b) for a, b in zip(*runs))
