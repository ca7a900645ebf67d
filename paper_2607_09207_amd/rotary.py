"""Rotary positions: turning rows by their positions, and the frequencies for it.

The arithmetic runs in the library's kernels (csrc/rlda_rotary.hip); the frequencies are a
small table of float64 values, laid out once.
"""
from __future__ import annotations

import ctypes
import math

from . import _abi

__all__ = ["rotate", "rotary_frequencies"]


def rotary_frequencies(rot_dim: int, base: float = 10000.0, scaling=None, device="cuda"):
    """(freqs, amplitude): radians a position of the rot_dim / 2 pairs (float64, on `device`),
    f_j = base ** (-2 j / rot_dim), and the factor of the turned values.

    scaling, for contexts longer than the one trained on:
      None
      {"type": "linear", "factor": s}                     positions divided by s
      {"type": "base", "factor": s}                       the base raised so that the slowest pair turns 1 / s as far
      {"type": "ramp", "factor": s, "context": n, "fast": 32, "slow": 1}
            a pair that turns `fast` times or more over the trained context n keeps its
            frequency, one that turns `slow` times or less has it divided by s, with a
            linear ramp in the pair's index between them; the amplitude is
            0.1 ln(s) + 1 ("amplitude" overrides it)
    """
    import torch
    rot_dim = int(rot_dim)
    if rot_dim < 2 or rot_dim % 2:
        raise ValueError(f"rot_dim must be even and positive, got {rot_dim}")
    if not base > 1.0:
        raise ValueError(f"base must exceed 1, got {base}")
    kind = None if scaling is None else scaling.get("type")
    if kind not in (None, "linear", "base", "ramp"):
        raise ValueError(f"unknown scaling {kind!r}")
    s = 1.0 if scaling is None else float(scaling["factor"])
    if not s > 0.0:
        raise ValueError(f"factor must be positive, got {s}")
    base, amplitude = float(base), 1.0
    if kind == "base" and rot_dim > 2:
        base *= s ** (rot_dim / (rot_dim - 2))
    j = torch.arange(rot_dim // 2, dtype=torch.float64)
    freqs = base ** (-2.0 * j / rot_dim)
    if kind == "linear":
        freqs = freqs / s
    elif kind == "ramp":
        fast, slow, n = float(scaling.get("fast", 32)), float(scaling.get("slow", 1)), float(scaling["context"])
        if not (fast > slow > 0 and n > 0):
            raise ValueError("ramp needs fast > slow > 0 and a positive context")
        # The pair that turns r times over the context: n base^(-2j/rot) = 2 pi r.
        pair = lambda r: rot_dim * math.log(n / (2 * math.pi * r)) / (2 * math.log(base))   # noqa: E731
        lo = max(math.floor(pair(fast)), 0)
        hi = min(math.ceil(pair(slow)), rot_dim - 1)
        keep = 1.0 - ((j - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
        keep[j >= hi] = 0.0   # (over a short context even the first pair: lo and hi coincide)
        freqs = freqs * keep + freqs / s * (1.0 - keep)
        amplitude = float(scaling.get("amplitude", 0.1 * math.log(s) + 1.0 if s > 1.0 else 1.0))
    return freqs.to(device), amplitude


def rows_of(t):
    """Rows [n][heads][d] as the C ABI takes them (d contiguous, or of one element)."""
    return _abi.Rows(t.data_ptr(), t.stride(0) if t.shape[0] > 1 else 0, t.stride(1) if t.shape[1] > 1 else 0)


def rotary_of(freqs, interleaved, amplitude, inverse=False):
    return _abi.Rotary(freqs.data_ptr(), 2 * freqs.shape[0], int(bool(interleaved)), float(amplitude), int(bool(inverse)))


def check_rows(fail, name, t, dtype, shape, device):
    if t is None:
        fail(f"{name} is required")
    if not t.is_cuda or t.device != device:
        fail(f"{name} must be on {device}, got {t.device}")
    if t.dtype != dtype:
        fail(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 3 or tuple(t.shape) != tuple(shape):
        fail(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.shape[2] > 1 and t.stride(2) != 1:
        fail(f"{name} needs its last dimension contiguous")
    per = 16 // t.element_size()
    if t.numel() and (t.data_ptr() % 16 or any(t.stride(i) % per for i in (0, 1) if t.shape[i] > 1)):
        fail(f"{name} needs 16-byte aligned rows (strides {tuple(t.stride())})")


def check_freqs(fail, freqs, d, device):
    import torch
    if freqs is None or not freqs.is_cuda or freqs.device != device:
        fail(f"freqs must be on {device}")
    if derived(freqs):
        fail("freqs gets no gradient: detach it")
    if freqs.dtype != torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous():
        fail("freqs must be a contiguous float64 vector")
    if not 16 <= 2 * freqs.shape[0] <= d or freqs.shape[0] % 8:
        fail(f"freqs turns {2 * freqs.shape[0]} elements: a multiple of 16 up to head_dim {d} is supported")


def derived(t):
    """Whether t's derivatives are asked for: backwards, or (a dual tensor, of which requires_grad
    says nothing) forwards."""
    import torch
    from torch.autograd import forward_ad
    return (t.requires_grad and torch.is_grad_enabled()) or forward_ad.unpack_dual(t).tangent is not None


def mark_written(t):
    """A backward pass that saved t is to notice that it was written."""
    import torch
    if not t.is_inference():
        torch.autograd.graph.increment_version(t)


def device_of(device):
    """The device meant, with its index: "cuda" (and None) is the current one."""
    import torch
    d = torch.device("cuda" if device is None else device)
    return torch.device("cuda", torch.cuda.current_device()) if d.type == "cuda" and d.index is None else d


def on_device(device):
    """A context in which `device` is the current one (nothing where it is already)."""
    import contextlib

    import torch
    return contextlib.nullcontext() if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def raw_stream(device, stream):
    import torch
    if stream is None:
        return torch.cuda.current_stream(device).cuda_stream
    return getattr(stream, "cuda_stream", stream)


def empty_on(shape, dtype, device, stream):
    """A tensor that a call on `stream` (None: the current one) writes and the caller then has.
    Memory of that stream's own: memory of the current stream's might still be in use by what
    is queued there.  And it is not given out again before what is then queued on the
    current stream, where the caller is taken to read it, is done."""
    import torch
    current = torch.cuda.current_stream(device)
    if stream is None or raw_stream(device, stream) == current.cuda_stream:
        return torch.empty(shape, dtype=dtype, device=device)
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(current)
    return t


def _laid_out(t):
    """A gradient or tangent as rotate takes it: it may come broadcast, in any layout, or as a
    contiguous piece of another tensor that begins anywhere in it."""
    import torch
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone(memory_format=torch.contiguous_format)


_turn = None


def _function():
    """The rotation for autograd: its backward is the rotation by the transpose, and its
    forward-mode derivative, as it is linear, itself."""
    global _turn
    if _turn is None:
        import torch

        class Turn(torch.autograd.Function):
            @staticmethod
            def forward(ctx, x, positions, freqs, interleaved, amplitude, inverse):
                ctx.save_for_backward(positions, freqs)
                ctx.save_for_forward(positions, freqs)
                ctx.how = interleaved, amplitude, inverse
                return _rotate(x, positions, freqs, interleaved, amplitude, inverse, None, None)

            @staticmethod
            def backward(ctx, grad):
                positions, freqs = ctx.saved_tensors
                interleaved, amplitude, inverse = ctx.how
                return rotate(_laid_out(grad), positions, freqs, interleaved=interleaved, amplitude=amplitude,
                              inverse=not inverse), None, None, None, None, None

            @staticmethod
            def jvp(ctx, tangent, *_):
                positions, freqs = ctx.saved_tensors
                interleaved, amplitude, inverse = ctx.how
                return rotate(_laid_out(tangent), positions, freqs, interleaved=interleaved, amplitude=amplitude,
                              inverse=inverse)

        _turn = Turn
    return _turn


def rotate(x, positions, freqs, *, interleaved: bool = False, amplitude: float = 1.0, inverse: bool = False, out=None,
           stream=None):
    """Rows x [n][heads][head_dim] (bf16 or fp32; any row and head strides that keep rows
    16-byte aligned, e.g. a slice of a fused projection) turned by positions [n] (int32), pair j
    by positions * freqs[j] radians (rl_decode_attn_rotate).  freqs: float64 [rot_dim / 2]
    (rotary_frequencies); elements past rot_dim pass.  inverse=True turns by the transpose:
    what takes a gradient back (an x that requires grad, or has a tangent, has its derivative
    done by autograd; `out` is refused then).  Returns `out` (x itself for in place), or a new tensor."""
    native = _abi.fastcall()
    if native is not None:
        got = native.rotate(x, positions, freqs, interleaved, amplitude, inverse, out, stream)
        if got is not None:
            if type(got) is int:
                _abi.check(got, _WHAT)
            return got
    if out is not None and derived(out):
        _refuse("out requires grad")
    if derived(x):
        if out is not None or stream is not None:
            _refuse("an x that requires grad is turned into a new tensor, on the current stream")
        _check_type(x)
        return _function().apply(x, positions, freqs, interleaved, amplitude, inverse)
    return _rotate(x, positions, freqs, interleaved, amplitude, inverse, out, stream)


_WHAT = "rl_decode_attn_rotate"


def _refuse(msg):
    raise _abi.RldaError(-1, f"{_WHAT}: {msg}")


def _check_type(x):
    import torch
    if not x.is_cuda:
        _refuse(f"x must be on a GPU, got {x.device}")
    if x.dtype not in (torch.bfloat16, torch.float32):
        _refuse(f"x must be bfloat16 or float32, got {x.dtype}")


def _rotate(x, positions, freqs, interleaved, amplitude, inverse, out, stream):
    """rotate() without derivatives."""
    import torch
    fail = _refuse
    _check_type(x)
    dev = x.device
    shape = tuple(x.shape)
    check_rows(fail, "x", x, x.dtype, shape, dev)
    check_freqs(fail, freqs, shape[2], dev)
    if positions is None or positions.device != dev or positions.dtype != torch.int32 or \
            tuple(positions.shape) != (shape[0],) or not positions.is_contiguous():
        fail(f"positions must be a contiguous int32 tensor of {shape[0]} on {dev}")
    with on_device(dev):
        if out is None:
            out = empty_on(shape, x.dtype, dev, stream)
        else:
            check_rows(fail, "out", out, x.dtype, shape, dev)
            mark_written(out)
        xr, outr, rot = rows_of(x), rows_of(out), rotary_of(freqs, interleaved, amplitude, inverse)
        _abi.check(_abi.load().rl_decode_attn_rotate(
            _abi.RLDA_F32 if x.dtype == torch.float32 else _abi.RLDA_BF16, shape[0], shape[1], shape[2], ctypes.byref(xr),
            positions.data_ptr(), ctypes.byref(rot), ctypes.byref(outr), raw_stream(dev, stream)), _WHAT)
    return out
