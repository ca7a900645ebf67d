"""A long cache that is read in part and kept in part (csrc/rlda_select.hip, csrc/rlda_listed.hip):
bounds of every page's keys, the choice of pages by them, attention over the chosen pages,
attention with the weight that every page gets, and eviction.  Methods of DecodeAttention.
"""
from __future__ import annotations

import ctypes
from typing import Optional

from . import _abi
from .rotary import derived, device_of, empty_on, mark_written, on_device, raw_stream

_ptr = lambda t: None if t is None else t.data_ptr()   # noqa: E731
_MAX_ROWS = 4096   # query rows of a call


class PartialCache:
    def _row_call(self, what, q, q_start):
        """(device, rows, batch) of a call whose rows are q [rows][Hq][d], one a sequence or by q_start."""
        import torch
        cfg = self.config
        if q is None or not q.is_cuda:
            self._fail(what, f"q must be on a GPU, got {None if q is None else q.device}")
        if q.dim() != 3:
            self._fail(what, f"q must be [rows, {cfg.num_q_heads}, {cfg.head_dim}], got {tuple(q.shape)}")
        if derived(q):
            self._fail(what, "q gets no gradient here: detach it")
        dev, total = q.device, int(q.shape[0])
        batch = total
        if q_start is not None:
            batch = int(q_start.shape[0]) - 1 if q_start.dim() == 1 else -1
            self._tensor(what, "q_start", q_start, torch.int32, (batch + 1,), dev)
        if batch < 0:
            self._fail(what, "q_start must hold batch + 1 offsets")
        self._tensor(what, "q", q, _abi.torch_dtype(cfg.q_dtype), (total, cfg.num_q_heads, cfg.head_dim), dev)
        return dev, total, batch

    def _check_bounds(self, what, bounds, bound_scale, npages, dev):
        import torch
        cfg = self.config
        for name, t, tail in (("bounds", bounds, (cfg.num_kv_heads, 2, cfg.head_dim)), ("bound_scale", bound_scale, (cfg.num_kv_heads,))):
            if t is None or t.dim() != 1 + len(tail) or t.shape[0] < npages:
                self._fail(what, f"{name} must be [>= {npages}, {', '.join(map(str, tail))}], "
                                 f"got {None if t is None else tuple(t.shape)}")
            self._tensor(what, name, t, torch.int8 if name == "bounds" else torch.float32, (int(t.shape[0]),) + tail, dev)

    def _host_int(self, what, name, x):
        import operator
        try:
            x = operator.index(x)
        except TypeError:
            self._fail(what, f"{name} must be an integer, got {x!r}")
        if not -2 ** 31 <= x < 2 ** 31:
            self._fail(what, f"{name} {x} does not fit 32 bits")
        return x

    def _ws_args(self, what, ws, dev, stream):
        self._check_workspace(what, ws, dev)
        wp = self._aligned_ptr(ws)
        return wp, ws.numel() - (wp - ws.data_ptr()), raw_stream(dev, stream)

    # ---------------------------------------------------------------- read in part

    def page_bounds(self, k_cache, block_table, seq_lens, bounds, bound_scale, *, first=None, k_scale=None, workspace=None,
                    stream=None, num_pages: Optional[int] = None):
        """Bounds of the keys of every sequence's pages from that of token first[b] (int32
        [batch]) on, or of its last page, into bounds (int8 [pages][Hkv][2][d]) and bound_scale
        (fp32 [pages][Hkv]) (rl_decode_attn_page_bounds).  Called after an append, and again for
        pages whose contents were moved."""
        what = "rl_decode_attn_page_bounds"
        got = self._fast.page_bounds(k_cache, block_table, seq_lens, k_scale, stream, num_pages, workspace, bounds, bound_scale,
                                     first)
        if got is not None:
            return _abi.check(got, what)
        import torch
        if k_cache is None or not k_cache.is_cuda:
            self._fail(what, f"k_cache must be on a GPU, got {None if k_cache is None else k_cache.device}")
        dev = k_cache.device
        npages = int(k_cache.shape[0]) if num_pages is None else int(num_pages)
        batch = int(seq_lens.shape[0]) if seq_lens is not None and seq_lens.dim() == 1 else -1
        self._check_table(what, block_table, seq_lens, batch, dev)
        self._check_cache(what, k_cache, k_cache, k_scale, k_scale, npages, dev)
        self._check_bounds(what, bounds, bound_scale, npages, dev)
        if first is not None:
            self._tensor(what, "first", first, torch.int32, (batch,), dev)
        with on_device(dev):
            ws = workspace if workspace is not None else self.workspace(dev)
            args = self._ws_args(what, ws, dev, stream)
            _abi.check(self._lib.rl_decode_attn_page_bounds(
                self._h, batch, npages, k_cache.data_ptr(), _ptr(k_scale), block_table.data_ptr(), seq_lens.data_ptr(),
                _ptr(first), bounds.data_ptr(), bound_scale.data_ptr(), *args), what)
        mark_written(bounds)
        mark_written(bound_scale)

    def select_pages(self, q, bounds, bound_scale, block_table, seq_lens, budget: int, *, sink: int = 1, recent: int = 1,
                     q_start=None, out=None, workspace=None, stream=None, num_pages: Optional[int] = None):
        """(pages int32 [rows][Hkv][budget], counts int32 [rows][Hkv]): of the pages that each
        query row sees, the first `sink`, the last `recent` and the best others by the bounds of
        their keys, `budget` together, ascending, then -1 (rl_decode_attn_select_pages).  One
        row a sequence or, with q_start, its last tokens.  out: (pages, counts) to write to."""
        what = "rl_decode_attn_select_pages"
        given = (None, None) if out is None else out
        if len(given) != 2:
            self._fail(what, "out must be (pages, counts)")
        got = self._fast.select_pages(q, bounds, bound_scale, block_table, seq_lens, stream, num_pages, *given, workspace,
                                      q_start, budget, sink, recent)
        if got is not None:
            return self._answer(got, what)
        import torch
        dev, total, batch = self._row_call(what, q, q_start)
        cfg = self.config
        budget, sink, recent = (self._host_int(what, n, x) for n, x in (("budget", budget), ("sink", sink), ("recent", recent)))
        if not (sink >= 0 and recent >= 1 and sink + recent <= budget):
            self._fail(what, f"budget {budget} must hold sink {sink} (>= 0) and recent {recent} (>= 1) pages")
        if bounds is None or bounds.dim() != 4:
            self._fail(what, f"bounds must be [pages, {cfg.num_kv_heads}, 2, {cfg.head_dim}]")
        npages = int(bounds.shape[0]) if num_pages is None else int(num_pages)
        self._check_table(what, block_table, seq_lens, batch, dev)
        self._check_bounds(what, bounds, bound_scale, npages, dev)
        with on_device(dev):
            pages, counts = given
            if pages is None:
                pages = empty_on((total, cfg.num_kv_heads, budget), torch.int32, dev, stream)
            if counts is None:
                counts = empty_on((total, cfg.num_kv_heads), torch.int32, dev, stream)
            self._tensor(what, "pages", pages, torch.int32, (total, cfg.num_kv_heads, budget), dev)
            self._tensor(what, "counts", counts, torch.int32, (total, cfg.num_kv_heads), dev)
            ws = workspace if workspace is not None else self.workspace(dev)
            args = self._ws_args(what, ws, dev, stream)
            _abi.check(self._lib.rl_decode_attn_select_pages(
                self._h, batch, npages, total, budget, sink, recent, q.data_ptr(), bounds.data_ptr(), bound_scale.data_ptr(),
                block_table.data_ptr(), seq_lens.data_ptr(), _ptr(q_start), pages.data_ptr(), counts.data_ptr(), *args), what)
        for t in given:
            if t is not None:
                mark_written(t)
        return pages, counts

    def selected(self, q, k_cache, v_cache, block_table, seq_lens, pages, counts, *, q_start=None, k_scale=None, v_scale=None,
                 out=None, workspace=None, stream=None, num_pages: Optional[int] = None, events=None):
        """Attention of every (row, KV head) over the pages it lists: pages int32
        [rows][Hkv][budget], the first counts[row][g] of them (rl_decode_attn_run_selected).  One
        row a sequence or, with q_start, its last tokens, each up to its own position."""
        what = "rl_decode_attn_run_selected"
        if events is None:
            got = self._fast.selected(q, k_cache, v_cache, block_table, seq_lens, k_scale, v_scale, stream, num_pages, out,
                                      workspace, q_start, pages, counts)
            if got is not None:
                return self._answer(got, what)
        import torch
        dev, total, batch = self._row_call(what, q, q_start)
        cfg = self.config
        if pages is None or pages.dim() != 3:
            self._fail(what, f"pages must be [rows, {cfg.num_kv_heads}, budget]")
        budget = int(pages.shape[2])
        self._tensor(what, "pages", pages, torch.int32, (total, cfg.num_kv_heads, budget), dev)
        self._tensor(what, "counts", counts, torch.int32, (total, cfg.num_kv_heads), dev)
        return self._attend(what, q, k_cache, v_cache, block_table, seq_lens, q_start, k_scale, v_scale, out, stream, num_pages,
                            events, batch, workspace if workspace is not None else self.workspace(dev),
                            self._lib.rl_decode_attn_run_selected, (budget, pages.data_ptr(), counts.data_ptr()))

    def _attend(self, what, q, k_cache, v_cache, block_table, seq_lens, q_start, k_scale, v_scale, out, stream, num_pages, events,
                batch, ws, call, own_args):
        cfg, dev, total = self.config, q.device, int(q.shape[0])
        if k_cache is None:
            self._fail(what, "k_cache is required")
        npages = int(k_cache.shape[0]) if num_pages is None else int(num_pages)
        self._check_table(what, block_table, seq_lens, batch, dev)
        self._check_cache(what, k_cache, v_cache, k_scale, v_scale, npages, dev)
        shape, dtype = (total, cfg.num_q_heads, cfg.head_dim), _abi.torch_dtype(cfg.out_dtype)
        if out is not None:
            self._tensor(what, "out", out, dtype, shape, dev)
        with on_device(dev):
            if out is None:
                out = empty_on(shape, dtype, dev, stream)
            else:
                mark_written(out)
            wp, room, raw = self._ws_args(what, ws, dev, stream)
            e0, e1 = (None, None) if events is None else tuple(self._event_handle(e) for e in events)
            _abi.check(call(self._h, batch, npages, total, *own_args, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                            _ptr(k_scale), _ptr(v_scale), block_table.data_ptr(), seq_lens.data_ptr(), _ptr(q_start),
                            out.data_ptr(), wp, room, raw, e0, e1), what)
        return out

    # ---------------------------------------------------------------- kept in part

    def weighed_workspace(self, rows: int, device):
        """Workspace of weighed() for up to `rows` query rows, allocated (and zeroed) once and grown
        where a call has more, to twice the rows at least: those it outgrew are kept, and
        together have less than twice its rows.  Calls that may overlap need separate ones
        (`workspace=`); a call to be captured into a graph finds it made before."""
        device = device_of(device)
        key = str(device)
        need = self._weighed_bytes(rows)
        ws = self._weighed_ws.get(key)
        if ws is None or ws.numel() < need:
            grown = int(rows)
            if ws is not None:
                grown = max(grown, min(2 * self._weighed_rows[key], _MAX_ROWS))
            new = self._zeroed(self._weighed_bytes(grown), device)
            if ws is not None:
                self._weighed_old.setdefault(key, []).append(ws)   # a graph, or a call that still runs, may use it
            ws = self._weighed_ws[key] = new
            self._weighed_rows[key] = grown
        return ws

    def weighed_flags(self, device, workspace=None, stream=None) -> int:
        """The flags that calls of weighed() raised on the device, in workspaces that later calls
        outgrew as well (waits for the stream)."""
        if workspace is not None:
            return self.read_flags(workspace=workspace, stream=stream)
        key = str(device_of(device))
        if key not in self._weighed_ws:
            self._fail("weighed_flags", f"no call with weights had a workspace on {key}")
        flags = 0
        for ws in [self._weighed_ws[key], *self._weighed_old.get(key, ())]:
            flags |= self.read_flags(workspace=ws, stream=stream)
        return flags

    def _weighed_bytes(self, rows):
        n = ctypes.c_size_t()
        _abi.check(self._lib.rl_decode_attn_weighed_workspace_size(self._h, int(rows), ctypes.byref(n)),
                   "rl_decode_attn_weighed_workspace_size")
        return n.value + 256

    def weighed(self, q, k_cache, v_cache, block_table, seq_lens, weights, *, decay: float = 1.0, q_start=None, k_scale=None,
                v_scale=None, out=None, workspace=None, stream=None, num_pages: Optional[int] = None, events=None):
        """The layer's attention, one row a sequence or (q_start) its last tokens, and
        weights[b][j] <- decay weights[b][j] + the probabilities that go to page j of sequence b, of
        all its rows and query heads (rl_decode_attn_run_weighed).  weights: fp32
        [batch][max_pages_per_seq], zero where a sequence begins."""
        what = "rl_decode_attn_run_weighed"
        if events is None:
            got = self._fast.weighed(q, k_cache, v_cache, block_table, seq_lens, k_scale, v_scale, stream, num_pages, out,
                                     workspace, q_start, weights, decay)
            if got is not None:
                return self._answer(got, what)
        import torch
        dev, total, batch = self._row_call(what, q, q_start)
        self._tensor(what, "weights", weights, torch.float32, (batch, self.config.max_pages_per_seq), dev)
        if derived(weights):
            self._fail(what, "weights get no gradient here: detach them")
        decay = float(decay)
        if not 0.0 <= decay <= 1.0:
            self._fail(what, f"decay {decay} must be in [0, 1]")
        ws = workspace if workspace is not None else self.weighed_workspace(total, dev)
        out = self._attend(what, q, k_cache, v_cache, block_table, seq_lens, q_start, k_scale, v_scale, out, stream, num_pages,
                           events, batch, ws, self._lib.rl_decode_attn_run_weighed, (weights.data_ptr(), decay))
        mark_written(weights)
        return out

    def page_evict(self, refs, block_table, seq_lens, weights, budget: int, *, sink: int = 1, recent: int = 1, dropped=None,
                   workspace=None, stream=None):
        """Every sequence of more than `budget` pages keeps its first `sink`, its last `recent` and the
        heaviest others by weights (fp32 [batch][max_pages_per_seq]); table row, weights and
        length follow, and the pages that nobody else has are free
        (rl_decode_attn_page_evict).  Returns the pages dropped of each sequence, int32 [batch]."""
        what = "rl_decode_attn_page_evict"
        got = self._fast.page_evict(refs, block_table, seq_lens, weights, budget, sink, recent, dropped, workspace, stream)
        if got is not None:
            return self._answer(got, what)
        import torch
        budget, sink, recent = (self._host_int(what, n, x) for n, x in (("budget", budget), ("sink", sink), ("recent", recent)))
        if not (sink >= 0 and recent >= 1 and sink + recent <= budget):
            self._fail(what, f"budget {budget} must hold sink {sink} (>= 0) and recent {recent} (>= 1) pages")
        dev, batch, npages, _ = self._page_call(what, refs, block_table, seq_lens, None, workspace, stream)
        self._tensor(what, "weights", weights, torch.float32, (batch, self.config.max_pages_per_seq), dev)
        if derived(weights):
            self._fail(what, "weights get no gradient here: detach them")
        with on_device(dev):
            made = dropped is None
            if made:
                dropped = empty_on((batch,), torch.int32, dev, stream)
            self._tensor(what, "dropped", dropped, torch.int32, (batch,), dev)
            args = self._page_ws_args(what, npages, dev, workspace, stream)
            _abi.check(self._lib.rl_decode_attn_page_evict(
                self._h, batch, npages, refs.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(), weights.data_ptr(), budget,
                sink, recent, dropped.data_ptr(), *args), what)
        if not made:
            mark_written(dropped)
        mark_written(weights)
        return dropped
