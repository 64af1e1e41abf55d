"""Orthogonalised updates: Newton-Schulz products on the matrices of a flat vector.

The aggregated direction is one flat vector.  `Orthogonalizer` takes the weight matrices in it, each
where it lies, and replaces every one by the nearest thing to its orthogonal polar factor that a few
polynomial products give (the step of the Muon optimiser).  Argument marshalling only: the arithmetic
runs in the library's CUDA kernels, and there is no fallback.
"""
from __future__ import annotations

import ctypes

import torch

from .binding import BF16, F32, _check, _raw_stream, check_stream, load_library

# enum adacons_orth_info
INFO_BYTES, INFO_LAUNCHES = 0, 1
#: a, b, c of x <- a x + b x^3 + c x^5: steep at zero, between 0.7 and 1.2 after five steps for singular values above 0.01
COEFFS = (3.4445, -4.7750, 2.0315)


class Orthogonalizer:
    """The plan for one layout of matrices in a vector of `d` elements of `dtype` ("f32"/"bf16").

    shapes   [(rows, cols), ...]; offsets: the element each matrix starts at (default: one after
             the other from 0); d: the vector's length (default: where the last matrix ends).
    steps    polynomial steps; coeffs: one (a, b, c) for all of them or a list of `steps` triples.
    scaling  False, or True: every matrix's result times sqrt(max(1, rows / cols)).
    """

    def __init__(self, shapes, dtype: str = "bf16", offsets=None, d: int | None = None, steps: int = 5, coeffs=COEFFS,
                 eps: float = 1e-7, scaling: bool = False):
        self._ctx = ctypes.c_void_p()
        self._lib = load_library()
        shapes = [(int(m), int(n)) for m, n in shapes]
        if not shapes:
            raise ValueError("at least one matrix is needed")
        if offsets is None:
            offsets, at = [], 0
            for m, n in shapes:
                offsets.append(at)
                at += m * n
        offsets = [int(o) for o in offsets]
        if len(offsets) != len(shapes):
            raise ValueError(f"{len(shapes)} matrices need as many offsets, got {len(offsets)}")
        if d is None:
            d = max(o + m * n for o, (m, n) in zip(offsets, shapes))
        triples = [tuple(float(x) for x in t) for t in (coeffs if hasattr(coeffs[0], "__len__") else [coeffs] * int(steps))]
        if len(triples) != int(steps) or any(len(t) != 3 for t in triples):
            raise ValueError("coeffs must be one (a, b, c) or one triple per step")
        self.shapes, self.offsets, self.d, self.dtype, self.steps = shapes, offsets, int(d), dtype, int(steps)
        n = len(shapes)
        i64 = ctypes.c_int64 * n
        flat = (ctypes.c_double * (3 * len(triples)))(*[x for t in triples for x in t])
        _check(self._lib.adacons_orth_create(ctypes.byref(self._ctx), {"f32": F32, "bf16": BF16}[dtype], self.d, n, i64(*[m for m, _ in shapes]),
                                             i64(*[k for _, k in shapes]), i64(*offsets), int(bool(scaling)), int(steps), flat, float(eps)),
               "adacons_orth_create")
        self.device = torch.cuda.current_device()        # where the plan's memory is
        self._checked = None

    def close(self) -> None:
        if getattr(self, "_ctx", None) is not None and self._ctx.value:
            self._lib.adacons_orth_destroy(self._ctx)
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

    def apply(self, update, out, stream=None) -> None:
        """out[matrix] = orthogonalised update[matrix] for every matrix; the rest of `out` stays as it is.
        Flat CUDA tensors of d elements; `out` may be `update`, otherwise they must not share memory."""
        device = update.get_device()
        sig = (update.dtype, update.shape, update.stride(), device, out.dtype, out.shape, out.stride(), out.get_device())
        if sig != self._checked:
            check_vectors(self.d, self.dtype, update, out, device=self.device)
            self._checked = sig
        if stream is not None:
            check_stream(stream, device)
        _check(self._lib.adacons_orth_apply(self._ctx, update.data_ptr(), out.data_ptr(), _raw_stream(stream, device)), "adacons_orth_apply")

    def selftest_bounded_wait(self, update, out, stream=None) -> None:
        """apply with a tile that nobody computes: its waits run out (2 s each) and status() says so.  `out` is invalid."""
        check_vectors(self.d, self.dtype, update, out, device=self.device)
        _check(self._lib.adacons_selftest_orth(self._ctx, update.data_ptr(), out.data_ptr(), _raw_stream(stream, self.device)), "adacons_selftest_orth")

    def status(self, stream=None) -> int:
        """The ADACONS_FLAG_TIMEOUT bit since the last call (0: all waits ended)."""
        v = ctypes.c_uint32()
        _check(self._lib.adacons_orth_get_status(self._ctx, ctypes.byref(v), _raw_stream(stream, self.device)), "adacons_orth_get_status")
        return v.value

    def info(self, key: int) -> int:
        v = ctypes.c_int64()
        _check(self._lib.adacons_orth_get_info(self._ctx, key, ctypes.byref(v)), "adacons_orth_get_info")
        return v.value


def check_vectors(d: int, dtype: str, update, out, want_cuda: bool = True, device=None) -> None:
    """Raise ValueError unless both are contiguous vectors of d elements of `dtype` on one (CUDA) device, the one of
    index `device` if given."""
    tdt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    for name, t in (("update", update), ("out", out)):
        if t.dtype != tdt:
            raise ValueError(f"{name} must be {tdt}, got {t.dtype}")
        if t.dim() != 1 or t.shape[0] != d:
            raise ValueError(f"{name} must have shape ({d},), got {tuple(t.shape)}")
        if d > 1 and t.stride(0) != 1:
            raise ValueError(f"{name} must be contiguous")
        if want_cuda and not t.is_cuda:
            raise ValueError(f"{name} must be a CUDA tensor")
    if update.device != out.device:
        raise ValueError("update and out must be on the same device")
    if device is not None and update.get_device() != device:
        raise ValueError(f"update and out are on device {update.get_device()}, the plan was made on device {device}")
