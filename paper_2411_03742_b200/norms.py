"""Norms before and after a block, its gate and the residual addition through the library's kernels.

A transformer's block ends in  x' = x + scale act(gate) rms(f) post  and the next one begins with
h = rms(x') pre: `residual_norm_forward` makes both in one pass over the rows, `residual_norm_backward`
their gradients, and `residual_norm` is the two of them as one differentiable torch operation.  Argument
marshalling only: the arithmetic runs in the library's CUDA kernels, and there is no fallback.
"""
from __future__ import annotations

import ctypes
import math

import torch

from .attention import F16
from .binding import BF16, F32, _check, _raw_stream, load_library
from .calls import Plans, address, elsewhere, here, layout, starts_with

MAX_DIM = 16384
_CODES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
_NONE, _CHANNEL, _SEQUENCE, _TOKEN = range(4)       # ADACONS_NORM_GATE_
_BY = {None: 0, "sigmoid": 1, "tanh": 2}            # ADACONS_NORM_BY_


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


class _Shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("stream_dtype", "dtype", "batch", "len", "dim", "gate", "gate_by", "gate_dtype", "post_dtype", "pre_dtype")] + \
               [("scale", ctypes.c_float), ("eps", ctypes.c_float)]


class _Plan:
    """Shape and row blocks of one layout, and references to them for the call."""

    def __init__(self, shape, rows):
        self.shape, self.shape_ref = shape, ctypes.byref(shape)
        self.blocks = [_Rows(None, *strides) for strides in rows]
        self.refs = [ctypes.byref(b) for b in self.blocks]
        self.workspace = 0


_plans, _back_plans = Plans(), Plans()


def _gate_kind(x, gate) -> int:
    if gate is None:
        return _NONE
    if gate.dim() == 1:
        return _CHANNEL
    return _TOKEN if gate.dim() == x.dim() else _SEQUENCE


def check_norm(x, f=None, gate=None, post=None, pre=None, gate_by=None, scale: float = 1.0, eps: float = 1e-6, dtype=None, like_x=(), like_f=(), like_gate=(), like_post=(),
               like_pre=(), rows=None, want_cuda: bool = True) -> None:
    """Raise ValueError unless x is (token, dim) or (batch, token, dim), f (and what is shaped like it) fits it, the gate is (dim,),
    (batch, dim) or of x's shape, the gains are (dim,), all of types that the kernels have and on one device; the like_*: (name, tensor or None) that
    must be as x, as the block's output, as the gate and as the gains; rows: the forward pass's, fp32."""
    if x.dim() not in (2, 3):
        raise ValueError("x must have two or three dimensions: token, element or batch, token, element")
    D = x.shape[-1]
    if not 1 <= D <= MAX_DIM:
        raise ValueError(f"rows have 1 to {MAX_DIM} elements, got {D}")
    block = f.dtype if f is not None else dtype if dtype is not None else x.dtype
    for t in (x.dtype, block):
        if t not in _CODES:
            raise ValueError(f"norms take float32, bfloat16 and float16, got {t}")
    if dtype is not None and dtype != block:
        raise ValueError(f"the normed rows are of f's type, {block}")
    if x.dtype not in (block, torch.float32):
        raise ValueError(f"x must be {block} or float32, got {x.dtype}")
    if f is None and (gate is not None or post is not None):
        raise ValueError("a gate and a gain behind the block need the block's output f")
    if f is None and pre is None:
        raise ValueError("nothing to do without f and without pre")
    if gate_by not in _BY:
        raise ValueError(f"gate_by must be None, 'sigmoid' or 'tanh', got {gate_by!r}")
    if gate is None and gate_by is not None:
        raise ValueError("gate_by without a gate")
    if not math.isfinite(scale):
        raise ValueError("scale must be finite")
    if not (eps > 0 and math.isfinite(eps)):
        raise ValueError("eps must be positive")
    same = [("x", x, x.shape, (x.dtype,))] + [(n, t, x.shape, (x.dtype,)) for n, t in like_x if t is not None]
    if f is not None:
        same.append(("f", f, x.shape, (block,)))
    same += [(n, t, x.shape, (block,)) for n, t in like_f if t is not None]
    if gate is not None:
        shapes = {1: (D,), 2: (x.shape[0], D), 3: tuple(x.shape)}
        shape = shapes.get(gate.dim()) if gate.dim() <= x.dim() else None
        if shape is None or tuple(gate.shape) != tuple(shape):
            raise ValueError(f"the gate must have shape {(D,)}{f', {(x.shape[0], D)}' if x.dim() == 3 else ''} or {tuple(x.shape)}, got {tuple(gate.shape)}")
        same += [("gate", gate, gate.shape, (block, torch.float32))] + [(n, t, gate.shape, (gate.dtype,)) for n, t in like_gate if t is not None]
    for name, t, like in (("post", post, like_post), ("pre", pre, like_pre)):
        if t is not None:
            same += [(name, t, (D,), (block, torch.float32))] + [(n, o, (D,), (t.dtype,)) for n, o in like if o is not None]
    for name, t, shape, types in same:
        if t.dtype not in types or tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} must be {' or '.join(map(str, types))} of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
        if t.device != x.device or (want_cuda and not t.is_cuda):
            raise ValueError(f"{name} must be a CUDA tensor on x's device")
        if D > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name} must have unit stride along a row")
    for name, t in (*like_x, *like_f, *like_gate):
        if t is not None and any(n > 1 and s == 0 for n, s in zip(t.shape, t.stride())):
            raise ValueError(f"{name} must not be a broadcast view")
    if rows is not None and (rows.dtype != torch.float32 or tuple(rows.shape) != (2, *x.shape[:-1]) or not rows.is_contiguous() or rows.device != x.device):
        raise ValueError(f"rows must be a contiguous float32 tensor of shape {(2, *x.shape[:-1])} on x's device")
    if math.prod(x.shape[:-1]) > 2 ** 31 - 1:
        raise ValueError("at most 2^31 - 1 tokens")


def _strides(t, kind=_TOKEN):
    """(batch, row) strides of a tensor of rows; a gate's go by its kind."""
    if t is None or kind in (_NONE, _CHANNEL):
        return 0, 0
    if kind == _SEQUENCE:
        return t.stride(0), 0
    return (0, t.stride(0)) if t.dim() == 2 else (t.stride(0), t.stride(1))


def _shape(x, block, gate, kind, post, pre, gate_by, scale, eps):
    batch, length = (1, x.shape[0]) if x.dim() == 2 else x.shape[:2]
    code = _CODES[block]
    return _Shape(_CODES[x.dtype], code, batch, length, x.shape[-1], kind, _BY[gate_by], code if gate is None else _CODES[gate.dtype],
                  code if post is None else _CODES[post.dtype], code if pre is None else _CODES[pre.dtype], scale, eps)


def _kind(x, gate):
    kind = _gate_kind(x, gate)
    return _TOKEN if kind == _SEQUENCE and x.shape[1] == 1 else kind        # sequences of one token: nothing to sum up


def _gate_strides(x, gate, kind):
    return (gate.stride(0), 0) if kind == _TOKEN and gate.dim() < x.dim() else _strides(gate, kind)


def residual_norm_forward(x, f=None, *, gate=None, gate_by=None, post=None, scale: float = 1.0, pre=None, eps: float = 1e-6, dtype=None, out=None, normed=None, rows=None,
                          stream=None):
    """(out, normed, rows) with  out = x + scale act(gate) n post,  n = f / sqrt(mean f^2 + eps)  (f itself without `post`), and
    normed = out / sqrt(mean out^2 + eps) pre  (None without `pre`).

    x: (batch, token, dim) or (token, dim); f: the block's output, of a 16-bit type or float32; x may be float32 beside a 16-bit f.
    Without f, out is x itself and normed its norm, of type `dtype` (x's by default).
    gate: one row (dim,), one for each sequence (batch, dim) or one for each token (x's shape); gate_by: act, None (the gate as it
    is), "sigmoid" or "tanh".  gate, post and pre are float32 or of f's type.
    rows: the factors of both norms, fp32 (2, batch, token), 0 where there is no such norm; the gradient wants them.
    out (which may be x), normed and rows are made here unless given.  stream: where the kernel goes (the current one by
    default); the caller orders it behind whatever makes the inputs, and its own use of the results behind it."""
    scale, eps = float(scale), float(eps)
    sig = (layout(x), layout(f), layout(gate), gate_by, layout(post), scale, layout(pre), eps, dtype, layout(out), layout(normed), layout(rows))
    plan = _plans.known.get(sig)
    if plan is None:
        check_norm(x, f, gate, post, pre, gate_by, scale, eps, dtype, like_x=[("out", out)], like_f=[("normed", normed)], rows=rows)
        if normed is not None and pre is None:
            raise ValueError("normed without pre")
    device = sig[0][3]
    if not here(device, stream):
        results = elsewhere(device, stream, (x if f is None and out is None else out, True if pre is None else normed, rows), lambda: residual_norm_forward(
            x, f, gate=gate, gate_by=gate_by, post=post, scale=scale, pre=pre, eps=eps, dtype=dtype, out=out, normed=normed, rows=rows))
        if results is not None:
            return results
    if out is not None or normed is not None or rows is not None:
        _check_places(x, f, gate, post, pre, out, normed, rows)
    if f is None:
        out = x
    elif out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    if pre is not None and normed is None:
        normed = x.new_empty(x.shape, dtype=dtype or x.dtype) if f is None else torch.empty_like(f, memory_format=torch.contiguous_format)
    if plan is None:
        kind = _kind(x, gate)
        plan = _plans.remember(sig, _Plan(_shape(x, f.dtype if f is not None else dtype or x.dtype, gate, kind, post, pre, gate_by, scale, eps),
                                          [_strides(x), _strides(f), _gate_strides(x, gate, kind), _strides(out), _strides(normed)]))
        plan.rows = (2, *x.shape[:-1])
        plan.call = load_library().adacons_norm_forward
    if rows is None:
        rows = x.new_empty(plan.rows, dtype=torch.float32)
    b = plan.blocks
    b[0].data = x.data_ptr()
    if f is not None:
        b[1].data, b[3].data = f.data_ptr(), out.data_ptr()
        if gate is not None:
            b[2].data = gate.data_ptr()
    if normed is not None:
        b[4].data = normed.data_ptr()
    r = plan.refs
    _check(plan.call(plan.shape_ref, r[0], r[1], r[2], None if post is None else post.data_ptr(), None if pre is None else pre.data_ptr(), r[3], r[4], rows.data_ptr(),
                     _raw_stream(None, device)), "adacons_norm_forward")
    return out, normed, rows


def _check_places(x, f, gate, post, pre, out, normed, rows):
    """Results that were given: out may be x, and is without f."""
    if f is None and out is not None and (out.data_ptr() != x.data_ptr() or out.stride() != x.stride()):
        raise ValueError("without f, out is x: none can be given")
    if f is not None and out is not None and starts_with(out, (x,)) and out.stride() != x.stride():
        raise ValueError("in place, out must be x itself")
    if starts_with(normed, (x, f, gate, post, pre, out)) or (f is not None and starts_with(out, (f, gate, post, pre))) or starts_with(rows, (x, f, gate, post, pre, out, normed)):
        raise ValueError("out may be x; no other result may share memory with what is read or with another result")


def residual_norm_backward(dout, dnormed, out, f, rows, *, gate=None, gate_by=None, post=None, scale: float = 1.0, pre=None, eps: float = 1e-6, dx=None, df=None, dgate=None,
                           dpost=None, dpre=None, workspace=None, stream=None):
    """(dx, df, dgate, dpost, dpre) of residual_norm_forward with the same arguments, from its out and rows and the gradients dout and
    dnormed (either may be None: zeros); None where there is no such input.  Every gradient has its tensor's type; sums over tokens are
    taken in fp32 and in a fixed order.  eps is not looked at: the factors are in rows.
    dx (which may be dout), df, dgate, dpost and dpre are made here unless given, as is the workspace (a uint8 tensor of workspace_bytes)."""
    scale, eps = float(scale), float(eps)
    given = (dx, df, dgate, dpost, dpre)
    sig = (layout(dout), layout(dnormed), layout(out), layout(f), layout(rows), layout(gate), gate_by, layout(post), scale, layout(pre), eps, layout(dx), layout(df), layout(dgate),
           layout(dpost), layout(dpre))
    plan = _back_plans.known.get(sig)
    if plan is None:
        block = f.dtype if f is not None else dnormed.dtype if dnormed is not None else out.dtype
        check_norm(out, f, gate, post, pre, gate_by, scale, eps, block, like_x=[("dx", dx)], like_f=[("df", df)], like_gate=[("dgate", dgate)], like_post=[("dpost", dpost)],
                   like_pre=[("dpre", dpre)], rows=rows)
        for name, t, dtype in (("dout", dout, out.dtype), ("dnormed", dnormed, block)):
            if t is not None and (t.dtype != dtype or t.shape != out.shape or t.device != out.device or (out.shape[-1] > 1 and t.stride(-1) != 1)):
                raise ValueError(f"{name} must be {dtype} of shape {tuple(out.shape)} on out's device with unit stride along a row, got {t.dtype} {tuple(t.shape)}")
        if dnormed is not None and pre is None:
            raise ValueError("dnormed without pre")
        for name, t, of in (("df", df, f), ("dgate", dgate, gate), ("dpost", dpost, post), ("dpre", dpre, pre)):
            if t is not None and of is None:
                raise ValueError(f"{name}: there is nothing that it is the gradient of")
    device = sig[2][3]
    if not here(device, stream):
        results = elsewhere(device, stream, tuple(True if of is None else t for t, of in zip(given, (out, f, gate, post, pre))), lambda: residual_norm_backward(
            dout, dnormed, out, f, rows, gate=gate, gate_by=gate_by, post=post, scale=scale, pre=pre, eps=eps, dx=dx, df=df, dgate=dgate, dpost=dpost, dpre=dpre, workspace=workspace))
        if results is not None:
            return results
    if any(t is not None for t in given):
        reads = (dnormed, out, f, gate, post, pre, rows)
        if dx is not None and dout is not None and starts_with(dx, (dout,)) and dx.stride() != dout.stride():
            raise ValueError("in place, dx must be dout itself")
        if any(starts_with(t, (*reads, *given[:k], *([dout] if k else []))) for k, t in enumerate(given)):
            raise ValueError("dx may be dout; no other result may share memory with what is read or with another result")
    dx = torch.empty_like(out, memory_format=torch.contiguous_format) if dx is None else dx
    if f is not None and df is None:
        df = torch.empty_like(f, memory_format=torch.contiguous_format)
    if gate is not None and dgate is None:
        dgate = torch.empty_like(gate, memory_format=torch.contiguous_format)
    if post is not None and dpost is None:
        dpost = torch.empty_like(post, memory_format=torch.contiguous_format)
    if pre is not None and dpre is None:
        dpre = torch.empty_like(pre, memory_format=torch.contiguous_format)
    if plan is None:
        kind = _kind(out, gate)
        plan = _Plan(_shape(out, block, gate, kind, post, pre, gate_by, scale, eps),
                     [_strides(dout), _strides(dnormed), _strides(out), _strides(f), _gate_strides(out, gate, kind), _strides(dx), _strides(df), _gate_strides(out, dgate, kind)])
        plan.call = load_library().adacons_norm_backward
        if post is not None or pre is not None or kind in (_CHANNEL, _SEQUENCE):
            n = ctypes.c_int64()
            _check(load_library().adacons_norm_workspace_bytes(plan.shape_ref, ctypes.byref(n)), "adacons_norm_workspace_bytes")
            plan.workspace = n.value
        _back_plans.remember(sig, plan)
    if workspace is None:
        if plan.workspace:
            workspace = rows.new_empty(plan.workspace // 4)
    elif workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous on out's device")
    for b, t in zip(plan.blocks, (dout, dnormed, out, f, gate, dx, df, dgate)):
        b.data = None if t is None else t.data_ptr()
    r = plan.refs
    _check(plan.call(plan.shape_ref, r[0], r[1], r[2], r[3], r[4], address(post), address(pre), rows.data_ptr(), r[5], r[6], r[7], address(dpost), address(dpre),
                     address(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(), _raw_stream(None, device)), "adacons_norm_backward")
    return dx, df, dgate, dpost, dpre


def residual_norm(x, f=None, *, gate=None, gate_by=None, post=None, scale: float = 1.0, pre=None, eps: float = 1e-6, dtype=None):
    """(out, normed) of residual_norm_forward as functions of x, f, the gate and the gains that can be differentiated once.  Not of the
    scale: a learned one belongs into the gate.  normed is None without `pre`.  What does not lie as the passes want it, along rows (transposed, broadcast), is copied."""
    if getattr(scale, "requires_grad", False):
        raise ValueError("the residual addition has no gradient for its scale: make it a gate")
    out, normed = _Residual.apply(*(_along(t) for t in (x, f, gate, post, pre)), gate_by, float(scale), float(eps), dtype)
    return (x if f is None else out), normed


def _along(t):
    """t, or a copy of it where its last dimension has not unit stride."""
    return t if t is None or t.dim() == 0 or t.shape[-1] <= 1 or t.stride(-1) == 1 else t.contiguous()


class _Residual(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, f, gate, post, pre, gate_by, scale, eps, dtype):
        out, normed, rows = residual_norm_forward(x, f, gate=gate, gate_by=gate_by, post=post, scale=scale, pre=pre, eps=eps, dtype=dtype)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(out, f, rows, gate, post, pre)
        ctx.how = {"gate_by": gate_by, "scale": scale, "eps": eps}
        return (None if f is None else out), normed

    @staticmethod
    def backward(ctx, dout, dnormed):
        out, f, rows, gate, post, pre = ctx.saved_tensors
        compute = _Gradient.apply if torch.is_grad_enabled() else _Gradient.compute
        if dout is None and dnormed is None:
            return (None,) * 9
        dx, df, dgate, dpost, dpre = compute(_along(dout), _along(dnormed), out.detach(), f, rows, gate, post, pre, ctx.how)
        return dx, df, dgate, dpost, dpre, None, None, None, None


class _Gradient(torch.autograd.Function):
    """The gradient where a graph of it is recorded: differentiating it again is an error (taken for a constant, it would silently leave
    terms out of a second derivative)."""

    @staticmethod
    def compute(dout, dnormed, out, f, rows, gate, post, pre, how):
        return residual_norm_backward(dout, dnormed, out, f, rows, gate=gate, post=post, pre=pre, **how)

    @staticmethod
    def forward(ctx, *args):
        return _Gradient.compute(*args)

    @staticmethod
    def backward(ctx, *grads):
        raise NotImplementedError("the residual addition can be differentiated once: its gradient has no gradient of its own")
