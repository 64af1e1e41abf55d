"""Rotary positions through the library's kernel: plain, partial, interleaved, scaled for long contexts.

`frequencies` states the scalings; `Rope` keeps the angles on the device and turns tensors by them.
Argument marshalling only: the arithmetic runs in the library's CUDA kernel, and there is no fallback.
"""
from __future__ import annotations

import ctypes
import math

import torch

from .binding import BF16, F32, _check, _raw_stream, check_stream, load_library, on_stream


def frequencies(dim: int, base: float = 10000.0, scaling=None):
    """(angles per position of the dim/2 pairs, gain).  scaling:
    None                         base^(-2i/dim)
    ("linear", s)                positions divided by s
    ("ntk", s)                   base times s^(dim/(dim-2)): the slowest pair turns s times slower, the fastest as before
    ("yarn", s, length[, fast, slow])   by parts (YaRN, arXiv 2309.00071): pairs that make more than `fast` turns over the
                                 original `length` keep their angle, those below `slow` turn s times slower, a
                                 ramp between; gain 0.1 ln(s) + 1
    """
    dim = int(dim)
    if dim < 2 or dim % 2:
        raise ValueError(f"the rotated part of a head has an even number of elements, got {dim}")
    if not base > 0:
        raise ValueError("base must be positive")
    kind, factor = (None, 1.0) if scaling is None else (scaling[0], float(scaling[1]))
    if not factor >= 1.0:
        raise ValueError("a scaling factor is at least 1")
    if kind == "ntk":
        if dim == 2:
            raise ValueError("ntk scaling needs more than one pair")
        base = base * factor ** (dim / (dim - 2))
    f = [base ** (-2 * i / dim) for i in range(dim // 2)]
    if kind in (None, "ntk"):
        return f, 1.0
    if kind == "linear":
        return [x / factor for x in f], 1.0
    if kind != "yarn":
        raise ValueError(f"unknown scaling {kind!r}")
    length = float(scaling[2])
    fast, slow = (float(x) for x in scaling[3:5]) if len(scaling) > 3 else (32.0, 1.0)
    pair_of = lambda turns: dim * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
    lo, hi = max(math.floor(pair_of(fast)), 0), min(math.ceil(pair_of(slow)), dim - 1)
    ramp = [min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0) for i in range(dim // 2)]
    return [x * (1 - r) + x / factor * r for x, r in zip(f, ramp)], 0.1 * math.log(factor) + 1.0


class _Shape(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("batch", ctypes.c_int), ("len", ctypes.c_int), ("heads", ctypes.c_int), ("head_dim", ctypes.c_int)]


class Rope:
    """Turns the first `dim` elements of every head.  interleaved: pairs are (2i, 2i+1) instead of (i, i + dim/2).
    base, scaling: see frequencies; or pass the angles themselves as `angles` (dim/2 values) and a `gain`."""

    def __init__(self, dim: int, base: float = 10000.0, interleaved: bool = False, scaling=None, angles=None, gain: float = 1.0):
        self._ctx = ctypes.c_void_p()
        self._lib = load_library()
        if angles is None:
            angles, gain = frequencies(dim, base, scaling)
        angles = [float(a) for a in angles]
        if len(angles) * 2 != int(dim):
            raise ValueError(f"{dim} elements need {int(dim) // 2} angles, got {len(angles)}")
        self.dim, self.interleaved, self.angles, self.gain = int(dim), bool(interleaved), angles, float(gain)
        _check(self._lib.adacons_rope_create(ctypes.byref(self._ctx), self.dim, (ctypes.c_double * len(angles))(*angles), self.gain, int(self.interleaved)),
               "adacons_rope_create")
        self.device = torch.cuda.current_device()        # where the angles are
        self._checked = {}

    def close(self) -> None:
        if getattr(self, "_ctx", None) is not None and self._ctx.value:
            self._lib.adacons_rope_destroy(self._ctx)
            self._ctx = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def apply(self, x, positions=None, out=None, inverse: bool = False, first: int = 0, stream=None):
        """x turned, (batch, token, head, element) in float32 or bfloat16 with unit stride along the elements;
        positions: int32 (batch, token), or None: token s is at position first + s.  out: a new tensor
        unless given; x itself is allowed, no other overlap.  inverse: the gradient's turn, by the negative angles."""
        device = x.get_device()
        if stream is not None and x.is_cuda:
            check_stream(stream, device)
            if stream.cuda_stream != _raw_stream(None, device):
                return on_stream(stream, device, (out,), lambda: (self.apply(x, positions, out, inverse, first),))[0]
        sig = (x.dtype, x.shape, x.stride(), device, None if out is None else (out.dtype, out.shape, out.stride(), out.get_device(), out.data_ptr() == x.data_ptr()),
               None if positions is None else (positions.dtype, positions.shape, positions.stride(), positions.get_device()))
        args = self._checked.get(sig)
        if out is None:
            out = torch.empty_like(x, memory_format=torch.contiguous_format)
        if args is None:
            check_rope(self.dim, x, positions, out, device=self.device)
            B, S, H, D = x.shape
            i64 = ctypes.c_int64 * 3
            if len(self._checked) >= 1024:       # a program with ever new lengths
                self._checked.clear()
            args = self._checked[sig] = (_Shape(F32 if x.dtype == torch.float32 else BF16, B, S, H, D), i64(*x.stride()[:3]), i64(*out.stride()[:3]))
        _check(self._lib.adacons_rope_apply(self._ctx, ctypes.byref(args[0]), x.data_ptr(), args[1], out.data_ptr(), args[2],
                                            None if positions is None else positions.data_ptr(), int(first), int(bool(inverse)), _raw_stream(stream, device)),
               "adacons_rope_apply")
        return out

    def __call__(self, x, positions=None, first: int = 0):
        """apply as a differentiable function of x."""
        return _Turn.apply(x, self, positions, first, False)


def check_rope(dim: int, x, positions, out, want_cuda: bool = True, device=None) -> None:
    """Raise ValueError unless x and out are alike, four-dimensional, of a type the kernel has, on the device of
    index `device` if given, and positions fit."""
    if x.dim() != 4:
        raise ValueError("x must have four dimensions: batch, token, head, element")
    if x.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"rotary positions take float32 and bfloat16, got {x.dtype}")
    if x.shape[3] < dim:
        raise ValueError(f"heads of {x.shape[3]} elements are smaller than the rotated part, {dim}")
    if out.dtype != x.dtype or out.shape != x.shape or out.device != x.device:
        raise ValueError("out must have x's type, shape and device")
    for name, t in (("x", x), ("out", out)):
        if t.stride(3) != 1:
            raise ValueError(f"{name} must have unit stride along the elements of a head")
        if want_cuda and not t.is_cuda:
            raise ValueError(f"{name} must be a CUDA tensor")
    if device is not None and x.get_device() != device:
        raise ValueError(f"x is on device {x.get_device()}, the angles are on device {device}")
    if any(n > 1 and s == 0 for n, s in zip(out.shape, out.stride())):
        raise ValueError("out must not be a broadcast view")
    if x.numel() > 0 and out.data_ptr() == x.data_ptr() and out.stride() != x.stride():      # tensors without elements may all be at address 0
        raise ValueError("in place, out must be x itself")
    if positions is not None and (positions.dtype != torch.int32 or tuple(positions.shape) != tuple(x.shape[:2]) or not positions.is_contiguous() or positions.device != x.device):
        raise ValueError(f"positions must be a contiguous int32 tensor of shape {tuple(x.shape[:2])} on x's device")


class _Turn(torch.autograd.Function):
    """The turn, or the turn back.  It is linear: its gradient is the other of the two, as often as one differentiates."""

    @staticmethod
    def forward(ctx, x, rope, positions, first, inverse):
        ctx.rope, ctx.first, ctx.inverse = rope, first, inverse
        ctx.save_for_backward(*([] if positions is None else [positions]))
        return rope.apply(x, positions, inverse=inverse, first=first)

    @staticmethod
    def backward(ctx, dy):
        pos = ctx.saved_tensors[0] if ctx.saved_tensors else None
        dy = dy if dy.stride(3) == 1 else dy.clone(memory_format=torch.contiguous_format)
        if torch.is_grad_enabled():         # a graph of the gradient is recorded
            dx = _Turn.apply(dy, ctx.rope, pos, ctx.first, not ctx.inverse)
        else:
            dx = ctx.rope.apply(dy, pos, inverse=not ctx.inverse, first=ctx.first)
        return dx, None, None, None, None
