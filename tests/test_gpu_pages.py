"""The page operations on the GPU against a page manager in plain Python: counts, tables,
lengths and caches have to be equal."""
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


def pages_of(n):
    return -(-int(n) // PAGE)


class Model:
    """The documented rules, one request after the other, on host arrays."""

    def __init__(self, refs, table, lens, pools=()):
        self.refs, self.table, self.lens = refs.copy(), table.copy(), lens.copy()
        self.pools, self.flags = [p.copy() for p in pools], 0
        self.cap = table.shape[1] * PAGE

    def free(self):
        return np.flatnonzero(self.refs == 0)

    def grow(self, add=None):
        free, at, out = self.free(), 0, False
        for b in range(len(self.lens)):
            L, a = int(self.lens[b]), 1 if add is None else int(add[b])
            if L < 0 or L > self.cap or a < 0 or L + a > self.cap:
                self.flags |= 2
                continue
            need = pages_of(L + a) - pages_of(L)
            out = out or (need > 0 and at + need > len(free))
            if need > 0 and out:
                self.flags |= 16
                continue
            for j in range(need):
                self.table[b, pages_of(L) + j] = free[at + j]
                self.refs[free[at + j]] = 1
            at += need
            self.lens[b] = L + a

    def release(self, rows):
        for r in rows:
            if not 0 <= r < len(self.lens) or not 0 <= self.lens[r] <= self.cap:
                self.flags |= 2
                continue
            for p in self.table[r, :pages_of(self.lens[r])]:
                if 0 <= p < len(self.refs) and self.refs[p] > 0:
                    self.refs[p] -= 1
                else:
                    self.flags |= 1
            self.lens[r] = 0

    def fork(self, parents, children):
        lens0, table0, free, at, named = self.lens.copy(), self.table.copy(), self.free(), 0, set()
        for a, c in zip(parents, children):
            if not (0 <= a < len(lens0) and 0 <= c < len(lens0)) or a == c:
                self.flags |= 2
                continue
            first = c not in named
            named.add(c)
            L = int(lens0[a])
            if L < 0 or L > self.cap or lens0[c] != 0 or not first:
                self.flags |= 2
                continue
            full = L // PAGE
            if L % PAGE:
                if at >= len(free):
                    self.flags |= 16
                    at += 1
                    continue
                src, dst = table0[a, full], free[at]
                at += 1
                self.table[c, full] = dst
                self.refs[dst] = 1
                for p in self.pools:
                    p[dst] = p[src]
            self.table[c, :full] = table0[a, :full]
            np.add.at(self.refs, table0[a, :full], 1)
            self.lens[c] = L

    def compact(self):
        n = int((self.refs > 0).sum())
        src = np.flatnonzero((self.refs > 0) & (np.arange(len(self.refs)) >= n))
        dst = np.flatnonzero((self.refs == 0) & (np.arange(len(self.refs)) < n))
        to = np.arange(len(self.refs))
        to[src] = dst
        for b, L in enumerate(self.lens):
            for j in range(pages_of(L)):
                self.table[b, j] = to[self.table[b, j]]
        self.refs[dst] = self.refs[src]
        self.refs[src] = 0
        for p in self.pools:
            p[dst] = p[src]
        return n


class State:
    """A pool of `npages` with rows of `lens` tokens on random pages, on the GPU and in a Model."""

    def __init__(self, torch, npages, lens, mp, kv="bf16", hkv=2, d=64, layers=2, layout="head", seed=0, max_batch=None):
        from paper_2607_09207_amd import DecodeAttention
        rng = np.random.default_rng(seed)
        self.torch, lens = torch, np.asarray(lens, np.int32)
        used = [pages_of(x) for x in lens]
        perm = rng.permutation(npages)
        assert sum(used) <= npages
        table = rng.integers(-9, npages + 9, size=(len(lens), mp)).astype(np.int32)
        refs = np.zeros(npages, np.int32)
        at = 0
        for b, u in enumerate(used):
            table[b, :u] = perm[at:at + u]
            at += u
        refs[perm[:at]] = 1
        dt = {"bf16": torch.int16, "fp8": torch.uint8, "f32": torch.int32}[kv]
        as_t = {"bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn, "f32": torch.float32}[kv]
        g = torch.Generator("cuda").manual_seed(seed)
        self.raw, tensors, pools = [], [], []
        for _ in range(layers):
            one = []
            for _ in range(2):
                shape = {"head": (npages, hkv, PAGE, d), "slot": (npages, PAGE, hkv, d), "apart": (npages, 2, hkv, PAGE, d + 16)}[layout]
                x = torch.randint(-2 ** 15 if kv != "fp8" else 0, 2 ** 15 if kv != "fp8" else 256, shape, device="cuda", generator=g).to(dt)
                y = x if layout == "head" else x.transpose(1, 2) if layout == "slot" else x[:, 0, :, :, :d]
                self.raw.append(x)
                one.append(y.view(as_t) if layout != "apart" else y.view(as_t))
                pools.append(y.cpu().numpy())
            if kv == "fp8":
                for _ in range(2):
                    one.append(torch.rand((npages, hkv), device="cuda", generator=g))
                    self.raw.append(one[-1])
                    pools.append(one[-1].cpu().numpy())
            tensors.append(tuple(one))
        self.tensors = tensors
        strides = tensors[0][0].stride()[:3] if tensors else None
        self.layer = DecodeAttention(hkv, hkv, d, max_batch or max(len(lens), 1), mp, "f32" if kv == "f32" else "bf16",
                                     {"bf16": "bf16", "fp8": "fp8_e4m3fn", "f32": "f32"}[kv], "f32", kv_strides=strides)
        self.caches = self.layer.caches(tensors)
        self.refs, self.table, self.lens = (torch.from_numpy(x).cuda() for x in (refs, table, lens))
        self.model = Model(refs, table, lens, pools)

    def args(self):
        return self.refs, self.table, self.lens

    def cuda(self, x):
        return self.torch.from_numpy(np.asarray(x, np.int32)).cuda()

    def check(self, what):
        m = self.model
        for name, got, want in (("refs", self.refs, m.refs), ("table", self.table, m.table), ("lens", self.lens, m.lens)):
            got = got.cpu().numpy()
            bad = np.argwhere(got != want)
            assert len(bad) == 0, f"{what}: {name} differs at {bad[:4].tolist()}: {got[tuple(bad[0])]}, not {want[tuple(bad[0])]}"
        flat = [t for one in self.tensors for t in one]
        for i, (t, p) in enumerate(zip(flat, m.pools)):
            if t.dtype != self.torch.float32 or t.dim() == 4:
                t = t.view({1: self.torch.uint8, 2: self.torch.int16, 4: self.torch.int32}[t.element_size()])
            assert np.array_equal(t.cpu().numpy(), p), f"{what}: cache {i}"
        flags = self.layer.page_flags(len(self.refs), self.refs.device)
        assert flags == m.flags, f"{what}: flags {flags}, not {m.flags}"


LAYOUTS = [("bf16", "head", 2, 64), ("fp8", "slot", 8, 128), ("f32", "head", 1, 64), ("bf16", "apart", 3, 128), ("fp8", "head", 5, 64)]


@pytest.mark.parametrize("npages,batch", [(64, 1), (65, 7), (500, 64), (3000, 300), (140000, 40), (131072, 3), (131073, 3), (20000, 8192)])
def test_grow(torch, npages, batch):
    rng = np.random.default_rng(npages)
    mp = 40
    lens = rng.integers(0, min(500, max(1, npages // batch // 2 * PAGE)) + 1, size=batch)
    s = State(torch, npages, lens, mp, layers=0, seed=npages)
    print("grow", npages, batch, flush=True)
    for k in range(4):
        add = None if k == 0 else np.where(rng.random(batch) < 0.3, 0, rng.integers(0, 100, size=batch)).astype(np.int32)
        s.layer.page_grow(*s.args(), None if add is None else s.cuda(add))
        s.model.grow(add)
        s.check(f"grow {k}")


def test_grow_runs_out(torch):
    """Served in order until pages run out; requests for none still are; odd requests stay."""
    s = State(torch, 20, [16, 16, 5, 0, 32, 16, 15, 16], 6, layers=0, seed=1)
    for add in ([16, 33, 11, 96, 1, 1, 1, 0], [1, 0, 0, 80, 64, 0, 1, 0], [0, -1, 2000000000, 0, 0, 97, 1, 16]):
        s.layer.page_grow(*s.args(), s.cuda(add))
        s.model.grow(np.array(add))
        s.check(f"grow {add}")
    s.lens[2], s.model.lens[2] = -5, -5
    s.lens[3], s.model.lens[3] = 10 ** 6, 10 ** 6
    s.layer.page_grow(*s.args())
    s.model.grow()
    s.check("grow of odd lengths")


def test_release(torch):
    s = State(torch, 300, [0, 1, 16, 17, 640, 33, 250], 40, layers=0, seed=2)
    for rows in ([4], [1, 1, 6, 1], [], [0, 2, 3, 5]):
        s.layer.page_release(*s.args(), s.cuda(rows))
        s.model.release(rows)
        s.check(f"release {rows}")
    # Rows out of range, an odd length, a page out of the pool, and pages nobody holds.
    s = State(torch, 300, [40, 41, 42, 43], 40, layers=0, seed=3)
    s.lens[1], s.model.lens[1] = 10 ** 7, 10 ** 7
    s.table[2, 1], s.model.table[2, 1] = 300, 300
    p = int(s.table[3, 0])
    s.refs[p], s.model.refs[p] = 0, 0
    rows = [-1, 4, 1, 2, 3, 1 << 30]
    s.layer.page_release(*s.args(), s.cuda(rows))
    s.model.release(rows)
    s.check("release of what is not there")


@pytest.mark.parametrize("kv,layout,hkv,d", LAYOUTS)
def test_fork(torch, kv, layout, hkv, d):
    lens = [40, 0, 32, 0, 0, 5, 0, 0, 0, 0, 16, 0, 639, 0]
    s = State(torch, 120, lens, 40, kv, hkv, d, 3, layout, seed=4)
    print("fork", kv, layout, flush=True)
    parents, children = [0, 0, 2, 12, 5, 10], [3, 1, 4, 6, 13, 7]
    s.layer.page_fork(*s.args(), s.cuda(parents), s.cuda(children), s.caches)
    s.model.fork(parents, children)
    s.check("fork")
    # A child of a child, an empty parent; then refusals: a live child, one named twice, itself, out of range.
    parents, children = [3, 9, 0, 0, 2, 2, 8, 8, 99, 1, -1], [8, 11, 5, 9, 9, 2, 8, 200, 0, -3, 11]
    s.layer.page_fork(*s.args(), s.cuda(parents), s.cuda(children), s.caches)
    s.model.fork(parents, children)
    s.check("fork again")
    s.layer.page_release(*s.args(), s.cuda(range(14)))
    s.model.release(range(14))
    s.check("release of all")
    assert int(s.refs.sum()) == 0


def test_fork_runs_out_and_without_caches(torch):
    s = State(torch, 6, [17, 33, 0, 0, 0, 0], 40, layers=0, seed=5)
    s.layer.page_fork(*s.args(), s.cuda([0, 1, 0, 1]), s.cuda([2, 3, 4, 5]))
    s.model.fork([0, 1, 0, 1], [2, 3, 4, 5])
    s.check("fork")
    assert s.model.flags == 16
    # Every page full: nothing to copy, nothing to take.
    s = State(torch, 2, [32, 0, 0], 40, layers=1, seed=6)
    s.layer.page_fork(*s.args(), s.cuda([0, 0]), s.cuda([1, 2]), s.caches)
    s.model.fork([0, 0], [1, 2])
    s.check("fork of full pages")


def test_fork_many_and_more_caches_than_a_launch_takes(torch):
    s = State(torch, 2000, [200, 37] + [0] * 900, 40, layers=70, d=64, hkv=1, seed=7)
    parents = [k % 2 for k in range(900)]
    children = (2 + np.random.default_rng(1).permutation(900)).tolist()
    s.layer.page_fork(*s.args(), s.cuda(parents), s.cuda(children), s.caches)
    s.model.fork(parents, children)
    s.check("fork of 900")


@pytest.mark.parametrize("kv,layout,hkv,d", LAYOUTS)
@pytest.mark.parametrize("npages", [64, 700, 4097])
def test_compact(torch, kv, layout, hkv, d, npages):
    rng = np.random.default_rng(npages)
    batch = 30
    lens = rng.integers(0, npages // batch * PAGE + 1, size=batch)
    lens[:4] = [1, 0, 16, 17]
    s = State(torch, npages, lens, 300, kv, hkv, d, 2, layout, seed=npages)
    print("compact", kv, layout, npages, flush=True)
    kids = [b for b in range(batch) if lens[b] == 0]
    s.layer.page_release(*s.args(), s.cuda([b for b in range(4, batch) if b % 3 == 0]))
    s.model.release([b for b in range(4, batch) if b % 3 == 0])
    if kids:
        s.layer.page_fork(*s.args(), s.cuda([3]), s.cuda(kids[:1]), s.caches)
        s.model.fork([3], kids[:1])
    for k in range(2):
        live = s.layer.page_compact(*s.args(), s.caches)
        n = s.model.compact()
        assert int(live) == n
        s.check(f"compact {k}")
    assert (s.refs[:n] > 0).all() and int(s.refs[n:].sum()) == 0


@pytest.mark.parametrize("npages", [131072, 131073, 200000])
def test_compact_large_pools(torch, npages):
    s = State(torch, npages, [300] * 60, 40, layers=1, d=64, hkv=1, seed=8)
    s.layer.page_release(*s.args(), s.cuda(range(0, 60, 2)))
    s.model.release(range(0, 60, 2))
    live = s.layer.page_compact(*s.args(), s.caches)
    assert int(live) == s.model.compact()
    s.check("compact")


def test_compact_full_and_empty(torch):
    s = State(torch, 128, [64 * PAGE, 64 * PAGE], 64, layers=1, seed=9)
    assert int(s.layer.page_compact(*s.args(), s.caches)) == 128
    s.check("a full pool")
    s.layer.page_release(*s.args(), s.cuda([0, 1]))
    s.model.release([0, 1])
    assert int(s.layer.page_compact(*s.args(), s.caches)) == 0
    s.check("an empty pool")


def test_compact_odd_tables(torch):
    """Entries out of the pool or on pages nobody counts stay, and are flagged."""
    s = State(torch, 100, [320, 320], 40, layers=1, seed=10)
    n = 40
    s.table[0, 3] = 5000
    s.table[0, 4] = -7
    p = int(s.table[1, :20].max())
    before = s.table.clone()
    s.refs[p] = 0
    s.layer.page_compact(*s.args(), s.caches)
    assert int(s.table[0, 3]) == 5000 and int(s.table[0, 4]) == -7
    at = (before == p).nonzero()[0].tolist()
    if p >= n - 1:
        assert int(s.table[at[0], at[1]]) == p
    assert s.layer.page_flags(100, s.refs.device) == 1
    s.lens[0] = 10 ** 7
    s.layer.page_compact(*s.args(), s.caches)
    assert s.layer.page_flags(100, s.refs.device) == 3


@pytest.mark.parametrize("npages", [100, 131072 + 700])
def test_compact_flags_every_uncounted_page(torch, npages):
    """An entry whose page nothing counts stays and is flagged, wherever its page is: below the
    live pages' number (another page moves into it) or above."""
    for above in (False, True):
        s = State(torch, npages, [320, 320], 40, layers=1, kv="fp8", hkv=1, seed=10)
        # Two pages at the front and the last one are held by row 1, whatever their numbers were.
        lo, hi = 2, npages - 1
        for b, j, page in ((1, 0, lo), (1, 1, hi)):
            old = int(s.table[b, j])
            where = (s.table[:, :20] == page).nonzero()
            if len(where):
                s.table[where[0, 0], where[0, 1]] = old
            else:
                s.refs[old] = 0
            s.table[b, j] = page
            s.refs[page] = 1
        page, j = (hi, 1) if above else (lo, 0)
        s.refs[page] = 0
        n = int(s.layer.page_compact(*s.args(), s.caches))
        assert n == 39 and int(s.refs[:n].min()) == 1 and int(s.refs.sum()) == 39
        assert int(s.table[1, j]) == page
        assert s.layer.page_flags(npages, s.refs.device) == 1, above


@pytest.mark.parametrize("kv,layout,hkv,d", LAYOUTS)
def test_copy(torch, kv, layout, hkv, d):
    s = State(torch, 60, [5], 40, kv, hkv, d, 2, layout, seed=11)
    src, dst = [3, 7, 3, 9, 11], [20, 21, 22, 59, 11]
    s.layer.page_copy(s.cuda(src), s.cuda(dst), s.caches)
    for p in s.model.pools:
        p[dst] = p[src]
    s.check("copy")
    s.layer.page_copy(s.cuda([1, -1, 60, 2]), s.cuda([60, 5, 6, 40]), s.caches)
    for p in s.model.pools:
        p[40] = p[2]
    s.model.flags = 1
    s.check("copy of pages out of the pool")


def test_copy_more_pairs_than_workgroups(torch):
    """A list longer than the copies' grid: mostly pages outside the pool, copies at its end."""
    from paper_2607_09207_amd import DecodeAttention
    layer = DecodeAttention(1, 1, 64, 4, 8, "bf16", "bf16", "bf16")
    n = (1 << 20) + 1000
    k = torch.randint(-9, 9, (1000, 1, 16, 64), device="cuda").to(torch.bfloat16)
    v = k + 1
    src = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    dst = torch.arange(n, dtype=torch.int32, device="cuda")
    src[-400:] = torch.arange(0, 400, dtype=torch.int32, device="cuda")
    dst[-400:] = torch.arange(500, 900, dtype=torch.int32, device="cuda")
    want = k.clone()
    want[500:900] = k[:400]
    layer.page_copy(src, dst, [(k, v)])
    assert torch.equal(k, want) and torch.equal(v, want + 1)
    assert layer.page_flags(1000, k.device) == 1


def test_refusals(torch):
    from paper_2607_09207_amd import RldaError
    s = State(torch, 50, [20, 30], 40, layers=1)
    refs, table, lens = s.args()
    one = s.cuda([0])
    L = s.layer
    bad = [lambda: L.page_grow(refs.long(), table, lens), lambda: L.page_grow(refs.cpu(), table, lens),
           lambda: L.page_grow(refs, table[:1], lens), lambda: L.page_grow(refs, table, lens[:1]),
           lambda: L.page_grow(refs, table, lens, one), lambda: L.page_release(refs, table, lens, one.long()),
           lambda: L.page_release(refs, table, lens, one.cpu()), lambda: L.page_release(refs, table, lens, s.cuda([[0]])),
           lambda: L.page_fork(refs, table, lens, one, s.cuda([0, 1]), s.caches),
           lambda: L.page_fork(s.cuda([0] * 51), table, lens, one, one, s.caches),
           lambda: L.page_fork(refs, table, lens, s.cuda([0] * 3), s.cuda([1] * 3), s.caches),
           lambda: L.page_compact(refs, table, lens, s.caches, live=one.long()),
           lambda: L.page_copy(one, one[:0], s.caches), lambda: L.page_copy(one, one, []),
           lambda: L.page_grow(refs, table, lens, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda")),
           lambda: L.caches([(s.tensors[0][0],)]), lambda: L.caches([(s.tensors[0][0].float(), s.tensors[0][1])])]
    for i, f in enumerate(bad):
        with pytest.raises(RldaError):
            f()
            print("taken:", i)
    s.check("refusals")


def test_a_set_of_another_layer(torch):
    """A set is taken by a layer with caches of the same geometry, by both call paths, and
    refused by any other, before anything is launched."""
    from paper_2607_09207_amd import DecodeAttention, RldaError, _abi
    s = State(torch, 50, [20, 30, 0], 40, "bf16", 2, 64, layers=2)
    like = DecodeAttention(8, 2, 64, 3, 40, "bf16", "bf16", "bf16")
    others = [DecodeAttention(8, 2, 64, 3, 40, "bf16", "fp8_e4m3fn", "f32"), DecodeAttention(8, 4, 64, 3, 40),
              DecodeAttention(8, 2, 128, 3, 40), DecodeAttention(8, 2, 64, 3, 40, kv_strides=(2048, 64, 128))]
    one = s.cuda([1])
    for layer in others:
        for fast in (layer._fast, _abi.LEFT_TO_PYTHON):
            layer.page_workspace(50, "cuda:0")
            layer._fast = fast
            for call in (lambda: layer.page_fork(*s.args(), one, s.cuda([2]), s.caches),
                         lambda: layer.page_compact(*s.args(), s.caches), lambda: layer.page_copy(one, s.cuda([2]), s.caches)):
                with pytest.raises(RldaError, match="caches are of"):
                    call()
        layer.page_compact(*s.args(), s.layer.caches([]), live=s.cuda([0]))   # of none: any layer's
    s2 = State(torch, 50, [20, 30, 0], 40, "bf16", 2, 64, layers=2)
    like.page_fork(*s2.args(), one, s2.cuda([2]), s2.caches)
    s2.model.fork([1], [2])
    s2.layer = like   # whose flags they are
    s2.check("another layer of the same geometry")


def test_devices_without_an_index(torch):
    """"cuda" is the current device: the same workspaces, and the same flags."""
    from paper_2607_09207_amd import RldaError
    s = State(torch, 10, [20, 30], 40, layers=1)
    layer = s.layer
    for none in ((10, "cuda"), (10, "cuda:0")):   # no operation yet
        with pytest.raises(RldaError, match="no page operation"):
            layer.page_flags(*none)
    ws = layer.page_workspace(10, "cuda")
    s.layer.page_grow(*s.args(), s.cuda([600, 0]))
    for device in ("cuda", "cuda:0", torch.device("cuda"), 0, None):
        assert layer.page_flags(10, device) == 16
        assert layer.page_workspace(10, device) is ws
    with pytest.raises(RldaError, match="no page operation"):
        layer.page_flags(11, "cuda")
    assert len(layer._page_ws) == 1
    own = layer.workspace("cuda")
    own[own.data_ptr() % 256 and 256 - own.data_ptr() % 256] = 8
    for device in ("cuda", "cuda:0", torch.device("cuda"), 0, None):
        assert layer.workspace(device) is own and layer.read_flags(device=device) == 8


def test_graph_and_streams(torch):
    """Release, fork and grow captured into one graph and replayed; the same on another stream."""
    def steps(s, stream=None):
        s.layer.page_release(*s.args(), s.kids, stream=stream)
        s.layer.page_fork(*s.args(), s.par, s.kids, s.caches, stream=stream)
        s.layer.page_grow(*s.args(), s.add, stream=stream)

    def model(s):
        s.model.release(s.kids.tolist())
        s.model.fork(s.par.tolist(), s.kids.tolist())
        s.model.grow(s.add.tolist())

    def make(seed):
        s = State(torch, 400, [45, 64, 0, 0, 0, 0], 40, layers=2, seed=seed)
        s.par, s.kids, s.add = s.cuda([0, 1, 0]), s.cuda([2, 3, 4]), s.cuda([0, 0, 3, 40, 5, 0])
        return s
    s = make(1)
    s.layer.page_workspace(400, "cuda:0")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps(s)
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        model(s)
        s.check(f"replay {k}")
        steps(s)
        model(s)
        s.check(f"eager {k}")
    s = make(2)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    steps(s, st)
    torch.cuda.current_stream().wait_stream(st)
    model(s)
    s.check("another stream")
