"""What a layer does with its cache besides attention: rows with rotary positions into it,
and its pages (csrc/rlda_rotary.hip, csrc/rlda_pages.hip).  Methods of DecodeAttention.
"""
from __future__ import annotations

import ctypes
from typing import Optional

from . import _abi
from .rotary import check_freqs, check_rows, derived, device_of, empty_on, mark_written, on_device, raw_stream, rotary_of, rows_of


class CacheSet:
    """The caches of the layers that share one pool's page ids, checked once
    (DecodeAttention.caches), for layers whose caches are of the same `geometry`."""

    def __init__(self, tensors, array, num_pages, device, geometry):
        self.tensors, self.array, self.num_pages, self.device = tensors, array, num_pages, device
        self.geometry = geometry
        # As the native call path takes it: number, address, pages, device.
        self.native = (len(tensors), ctypes.addressof(array), num_pages, None if device is None else device.index)

    def __len__(self):
        return len(self.tensors)


class CacheOps:
    def _check_set(self, what, caches):
        """The page operations copy by their own layer's page size and strides."""
        if len(caches) and caches.geometry != self._geometry:
            self._fail(what, f"the caches are of (dtype, KV heads, page size, head_dim, strides) {caches.geometry}, "
                             f"the layer's of {self._geometry}")
        return caches

    # ---------------------------------------------------------------- rotary positions

    def append_rotary(self, q, k_new, v_new, k_cache, v_cache, block_table, seq_lens, freqs, *, q_start=None,
                      positions=None, interleaved: bool = False, amplitude: float = 1.0, k_scale=None, v_scale=None,
                      out=None, workspace=None, stream=None, num_pages: Optional[int] = None):
        """Turn q [n][Hq][d] and k_new [n][Hkv][d] by their rows' positions, write k_new and
        v_new into the caches, and return the turned q (rl_decode_attn_append_rotary).  One
        row a sequence (token seq_lens[b] - 1), or, with q_start [batch + 1], its last
        q_start[b+1] - q_start[b] tokens.  positions [n] (int32) replaces the rows' tokens as
        what they are turned by.  q, k_new and v_new may be strided (slices of a fused
        projection); out: a tensor for q (q itself: in place).  No gradient goes through the
        cache: rows that require grad, or have a tangent, are refused."""
        what = "rl_decode_attn_append_rotary"
        got = self._fast.append_rotary(q, k_cache, v_cache, block_table, seq_lens, k_scale, v_scale, stream, num_pages, out,
                                       workspace, k_new, v_new, freqs, q_start, positions, interleaved, amplitude)
        if got is not None:
            return self._answer(got, what)
        import torch
        fail = lambda msg: self._fail(what, msg)   # noqa: E731
        cfg = self.config
        if not q.is_cuda:
            fail(f"q must be on a GPU, got {q.device}")
        dev, n, d = q.device, int(q.shape[0]), cfg.head_dim
        qd = _abi.torch_dtype(cfg.q_dtype)
        check_rows(fail, "q", q, qd, (n, cfg.num_q_heads, d), dev)
        check_rows(fail, "k_new", k_new, qd, (n, cfg.num_kv_heads, d), dev)
        check_rows(fail, "v_new", v_new, qd, (n, cfg.num_kv_heads, d), dev)
        for name, t in (("q", q), ("k_new", k_new), ("v_new", v_new), ("out", out)):
            if t is not None and derived(t):
                fail(f"{name} gets no gradient here: detach it (rotate has one)")
        check_freqs(fail, freqs, d, dev)
        batch = n
        if q_start is not None:
            batch = int(q_start.shape[0]) - 1 if q_start.dim() == 1 else -1
            self._tensor(what, "q_start", q_start, torch.int32, (batch + 1,), dev)
        if batch < 0:
            fail("q_start must hold batch + 1 offsets")
        if positions is not None:
            self._tensor(what, "positions", positions, torch.int32, (n,), dev)
        npages = int(k_cache.shape[0]) if num_pages is None else int(num_pages)
        self._check_table(what, block_table, seq_lens, batch, dev)
        self._check_cache(what, k_cache, v_cache, k_scale, v_scale, npages, dev)
        with on_device(dev):
            if out is None:
                out = empty_on((n, cfg.num_q_heads, d), qd, dev, stream)
            else:
                check_rows(fail, "out", out, qd, (n, cfg.num_q_heads, d), dev)
                mark_written(out)
            ws = workspace if workspace is not None else self.workspace(dev)
            self._check_workspace(what, ws, dev)
            wp = self._aligned_ptr(ws)
            ptr = lambda t: None if t is None else t.data_ptr()   # noqa: E731
            ref = ctypes.byref
            _abi.check(self._lib.rl_decode_attn_append_rotary(
                self._h, batch, npages, n, ref(rotary_of(freqs, interleaved, amplitude)), ref(rows_of(q)),
                ref(rows_of(k_new)), ref(rows_of(v_new)), ptr(q_start), ptr(positions), ptr(k_cache), ptr(v_cache),
                ptr(k_scale), ptr(v_scale), ptr(block_table), ptr(seq_lens), ref(rows_of(out)), wp,
                ws.numel() - (wp - ws.data_ptr()), raw_stream(dev, stream)), what)
        return out

    def _zeroed(self, nbytes, device):
        """Zeroed device memory for calls on any stream: the fill is waited for."""
        import torch
        if torch.cuda.is_current_stream_capturing():
            self._fail("workspace", "none is made during a graph's capture, which would clear it, with its flags, in "
                                    "every replay: call workspace() or page_workspace() before")
        ws = torch.zeros(nbytes, dtype=torch.uint8, device=device)
        torch.cuda.current_stream(ws.device).synchronize()
        return ws

    # ---------------------------------------------------------------- pages

    def page_workspace(self, num_pages: int, device, stream=None):
        """Workspace of the page operations on a pool of `num_pages`, allocated (and zeroed)
        once.  Calls that may overlap need separate ones (`workspace=`); a call to be
        captured into a graph finds it made before.  (`stream` makes no difference: it is
        zero for every stream.)"""
        device = device_of(device)
        key = (str(device), int(num_pages))
        ws = self._page_ws.get(key)
        if ws is None:
            n = ctypes.c_size_t()
            _abi.check(self._lib.rl_decode_attn_page_workspace_size(self._h, int(num_pages), ctypes.byref(n)),
                       "rl_decode_attn_page_workspace_size")
            ws = self._page_ws[key] = self._zeroed(n.value + 256, device)
        return ws

    def caches(self, layers, num_pages: Optional[int] = None):
        """The caches of the layers that share one pool's page ids, as the page operations
        take them: [(k_cache, v_cache), ...], or (k_cache, v_cache, k_scale, v_scale) for
        fp8.  Checked here once; the set keeps the tensors.  Every layer whose caches have
        the same dtype, heads and strides takes the set; layers with others need a pool (counts,
        table and page ids) of their own."""
        what = "caches"
        layers = [tuple(x) for x in layers]
        fp8 = self.config.kv_dtype == _abi.RLDA_FP8_E4M3FN
        for x in layers:
            if len(x) != (4 if fp8 else 2):
                self._fail(what, "a cache is (k_cache, v_cache), with (.., k_scale, v_scale) for fp8")
        if not layers:
            return CacheSet([], (_abi.Cache * 1)(), None, None, self._geometry)
        dev = layers[0][0].device
        if num_pages is None:
            num_pages = int(layers[0][0].shape[0])
        array = (_abi.Cache * len(layers))()
        for i, x in enumerate(layers):
            k, v, ks, vs = x if fp8 else x + (None, None)
            self._check_cache(what, k, v, ks, vs, num_pages, dev)
            array[i] = _abi.Cache(k.data_ptr(), v.data_ptr(), ks.data_ptr() if fp8 else None, vs.data_ptr() if fp8 else None)
        return CacheSet(layers, array, num_pages, dev, self._geometry)

    def _page_call(self, what, refs, block_table, seq_lens, caches, workspace, stream):
        """Checks that the page operations share; (device, batch, pages, caches, workspace)."""
        import torch
        if refs is None or not refs.is_cuda:
            self._fail(what, "refs must be on a GPU")
        dev, npages = refs.device, int(refs.shape[0]) if refs.dim() == 1 else -1
        self._tensor(what, "refs", refs, torch.int32, (npages,), dev)
        batch = int(seq_lens.shape[0]) if seq_lens is not None and seq_lens.dim() == 1 else -1
        self._check_table(what, block_table, seq_lens, batch, dev)
        if caches is not None and not isinstance(caches, CacheSet):
            caches = self.caches(caches, npages)
        if caches is not None:
            self._check_set(what, caches)
        if caches is not None and len(caches) and (caches.device != dev or caches.num_pages < npages):
            self._fail(what, f"the caches hold {caches.num_pages} pages on {caches.device}, refs {npages} on {dev}")
        return dev, batch, npages, caches

    def _page_ws_args(self, what, npages, dev, workspace, stream):
        ws = workspace if workspace is not None else self.page_workspace(npages, dev)
        self._check_workspace(what, ws, dev)
        wp = self._aligned_ptr(ws)
        return wp, ws.numel() - (wp - ws.data_ptr()), raw_stream(dev, stream)

    def _rows_list(self, what, name, t, dev):
        import torch
        if t is None or t.dim() != 1:
            self._fail(what, f"{name} must be a vector")
        self._tensor(what, name, t, torch.int32, (int(t.shape[0]),), dev)
        return int(t.shape[0])

    def page_grow(self, refs, block_table, seq_lens, add=None, *, workspace=None, stream=None):
        """Room for add[b] more tokens of every sequence (None: one each): seq_lens grows, new
        pages are the lowest-numbered ones with refs 0 (rl_decode_attn_page_grow)."""
        what = "rl_decode_attn_page_grow"
        got = self._fast.page_grow(refs, block_table, seq_lens, add, workspace, stream)
        if got is not None:
            return _abi.check(got, what)
        import torch
        dev, batch, npages, _ = self._page_call(what, refs, block_table, seq_lens, None, workspace, stream)
        if add is not None:
            self._tensor(what, "add", add, torch.int32, (batch,), dev)
        with on_device(dev):
            args = self._page_ws_args(what, npages, dev, workspace, stream)
            _abi.check(self._lib.rl_decode_attn_page_grow(
                self._h, batch, npages, refs.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(),
                None if add is None else add.data_ptr(), *args), what)

    def page_release(self, refs, block_table, seq_lens, rows, *, workspace=None, stream=None):
        """Rows (int32 list on the device) give up their pages; their lengths become 0
        (rl_decode_attn_page_release)."""
        what = "rl_decode_attn_page_release"
        got = self._fast.page_release(refs, block_table, seq_lens, rows, workspace, stream)
        if got is not None:
            return _abi.check(got, what)
        dev, batch, npages, _ = self._page_call(what, refs, block_table, seq_lens, None, workspace, stream)
        n = self._rows_list(what, "rows", rows, dev)
        with on_device(dev):
            args = self._page_ws_args(what, npages, dev, workspace, stream)
            _abi.check(self._lib.rl_decode_attn_page_release(
                self._h, batch, npages, refs.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(), n, rows.data_ptr(),
                *args), what)

    def page_fork(self, refs, block_table, seq_lens, parents, children, caches=(), *, workspace=None, stream=None):
        """Empty rows `children` become copies of rows `parents`: full pages shared, the partial
        last page copied in every cache (rl_decode_attn_page_fork)."""
        what = "rl_decode_attn_page_fork"
        if isinstance(caches, CacheSet) and caches.geometry == self._geometry:
            got = self._fast.page_fork(refs, block_table, seq_lens, parents, children, *caches.native, workspace, stream)
            if got is not None:
                return _abi.check(got, what)
        dev, batch, npages, cs = self._page_call(what, refs, block_table, seq_lens, caches, workspace, stream)
        n = self._rows_list(what, "parents", parents, dev)
        if self._rows_list(what, "children", children, dev) != n:
            self._fail(what, "parents and children must be as many")
        with on_device(dev):
            args = self._page_ws_args(what, npages, dev, workspace, stream)
            _abi.check(self._lib.rl_decode_attn_page_fork(
                self._h, batch, npages, refs.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(), n,
                parents.data_ptr(), children.data_ptr(), len(cs), cs.array, *args), what)

    def page_compact(self, refs, block_table, seq_lens, caches=(), *, live=None, workspace=None, stream=None):
        """The live pages move to the front of the pool in every cache; the table and refs
        follow (rl_decode_attn_page_compact).  Returns their number, an int32 tensor of one."""
        what = "rl_decode_attn_page_compact"
        if isinstance(caches, CacheSet) and caches.geometry == self._geometry:
            got = self._fast.page_compact(refs, block_table, seq_lens, *caches.native, live, workspace, stream)
            if got is not None:
                return self._answer(got, what)
        import torch
        dev, batch, npages, cs = self._page_call(what, refs, block_table, seq_lens, caches, workspace, stream)
        with on_device(dev):
            if live is None:
                live = empty_on((1,), torch.int32, dev, stream)
            self._tensor(what, "live", live, torch.int32, (1,), dev)
            args = self._page_ws_args(what, npages, dev, workspace, stream)
            _abi.check(self._lib.rl_decode_attn_page_compact(
                self._h, batch, npages, refs.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(), len(cs), cs.array,
                live.data_ptr(), *args), what)
        return live

    def page_copy(self, src, dst, caches, *, workspace=None, stream=None):
        """Page src[i] over page dst[i] in every cache (rl_decode_attn_page_copy)."""
        what = "rl_decode_attn_page_copy"
        cs = self._check_set(what, caches) if isinstance(caches, CacheSet) else self.caches(caches)
        if not len(cs):
            self._fail(what, "caches is empty")
        n = self._rows_list(what, "src", src, cs.device)
        if self._rows_list(what, "dst", dst, cs.device) != n:
            self._fail(what, "src and dst must be as many")
        with on_device(cs.device):
            args = self._page_ws_args(what, cs.num_pages, cs.device, workspace, stream)
            _abi.check(self._lib.rl_decode_attn_page_copy(
                self._h, cs.num_pages, n, src.data_ptr(), dst.data_ptr(), len(cs), cs.array, *args), what)

    def page_flags(self, num_pages: int, device, workspace=None, stream=None) -> int:
        """The flags the page operations raised on a pool of `num_pages` (waits for the stream)."""
        ws = workspace
        if ws is None:
            device = device_of(device)
            ws = self._page_ws.get((str(device), int(num_pages)))
            if ws is None:
                self._fail("page_flags", f"no page operation had a workspace for {num_pages} pages on {device}")
        return self.read_flags(workspace=ws, stream=stream)
