"""The gated feed-forward block and its gradient through the library's kernels.

    gate = x w_gate^T,  up = x w_up^T,  y = (act(gate) up) w_down^T

`feedforward_forward` and `feedforward_backward` marshal arguments only; `gated_feedforward` is the two of them as one
differentiable torch operation.  Weights lie as torch's linear layers keep them, (out, in).  There is no fallback.
"""
from __future__ import annotations

import ctypes

import torch

from .attention import F16
from .binding import BF16, _check, _raw_stream, _stream_handle, load_library
from .calls import Plans, address, elsewhere, here, layout, starts_with

#: the activations, in the order of the C header's ADACONS_FFN_ values
ACTS = ("silu", "gelu", "gelu_tanh", "relu")


class _Matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64)]


class _Shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("dtype", "tokens", "dim", "hidden", "act")]


class _Plan:
    """Shape and matrix blocks of one layout, and references to them for the call."""

    def __init__(self, x, w_gate, act, matrices, backward):
        self.shape = _Shape(BF16 if x.dtype == torch.bfloat16 else F16, x.shape[0], x.shape[1], w_gate.shape[0], ACTS.index(act))
        self.shape_ref = ctypes.byref(self.shape)
        self.blocks = [_Matrix(None, 0 if t is None else t.stride(0)) for t in matrices]
        self.refs = [ctypes.byref(b) for b in self.blocks]
        n = ctypes.c_int64()
        _check(load_library().adacons_ffn_workspace_bytes(self.shape_ref, int(backward), ctypes.byref(n)), "adacons_ffn_workspace_bytes")
        self.workspace = n.value


_plans, _back_plans = Plans(), Plans()


def check_feedforward(x, w_gate, w_up, w_down, act: str = "silu", like_x=(), like_hidden=(), like_gate=(), like_down=(), want_cuda: bool = True) -> None:
    """Raise ValueError unless x is (token, dim), w_gate and w_up are (hidden, dim), w_down is (dim, hidden), of one 16-bit type on one device, 16-byte aligned with row
    strides that are multiples of 8; the like_*: (name, tensor or None) of x's shape, (token, hidden), w_gate's and w_down's."""
    if x.dim() != 2 or w_gate.dim() != 2 or w_down.dim() != 2:
        raise ValueError("x and the weights must have two dimensions: token, element and out, in")
    if x.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"the feed-forward block takes bfloat16 and float16, got {x.dtype}")
    if act not in ACTS:
        raise ValueError(f"act must be one of {', '.join(ACTS)}, got {act!r}")
    (T, D), F = x.shape, w_gate.shape[0]
    if D < 8 or F < 8 or D % 8 or F % 8 or max(D, F) > 2 ** 18 or T > 2 ** 24:
        raise ValueError(f"dim and hidden are multiples of 8 up to 2^18, tokens at most 2^24, got {D}, {F} and {T}")
    tensors = [("x", x, (T, D)), ("w_gate", w_gate, (F, D)), ("w_up", w_up, (F, D)), ("w_down", w_down, (D, F))]
    for names, shape in ((like_x, (T, D)), (like_hidden, (T, F)), (like_gate, (F, D)), (like_down, (D, F))):
        tensors += [(n, t, shape) for n, t in names if t is not None]
    for name, t, shape in tensors:
        if t.dtype != x.dtype or tuple(t.shape) != shape:
            raise ValueError(f"{name} must be {x.dtype} of shape {shape}, got {t.dtype} {tuple(t.shape)}")
        if t.device != x.device or (want_cuda and not t.is_cuda):
            raise ValueError(f"{name} must be a CUDA tensor on x's device")
        if t.stride(1) != 1 or (t.shape[0] > 1 and (t.stride(0) % 8 != 0 or t.stride(0) < shape[1])):
            raise ValueError(f"{name}: the last stride must be 1 and the other a multiple of 8 and no less than a row, got {t.stride()}")


def feedforward_forward(x, w_gate, w_up, w_down, *, act: str = "silu", keep: bool = True, out=None, gate=None, up=None, workspace=None, stream=None):
    """(out, gate, up): out = (act(gate) up) w_down^T with gate = x w_gate^T and up = x w_up^T, which feedforward_backward wants; with
    keep=False they are not made, and None.  x: (token, dim), bfloat16 or float16; act: one of ACTS ("gelu" by the error function).
    out, gate and up are made here unless given, as is the workspace (a uint8 tensor of workspace_bytes, 16-byte aligned).
    stream: where the kernels go (the current one by default); the caller orders it behind whatever makes the inputs, and its own
    use of the results behind it."""
    keep = bool(keep)
    sig = (layout(x), layout(w_gate), layout(w_up), layout(w_down), act, keep, layout(out), layout(gate), layout(up))
    plan = _plans.known.get(sig)
    if plan is None:
        check_feedforward(x, w_gate, w_up, w_down, act, like_x=[("out", out)], like_hidden=[("gate", gate), ("up", up)])
        if not keep and (gate is not None or up is not None):
            raise ValueError("gate and up are not made with keep=False")
    device = sig[0][3]
    if not here(device, stream):
        results = elsewhere(device, stream, (out, gate, up) if keep else (out, True, True), lambda: feedforward_forward(
            x, w_gate, w_up, w_down, act=act, keep=keep, out=out, gate=gate, up=up, workspace=workspace))
        if results is not None:
            return results
    reads = (x, w_gate, w_up, w_down)
    if starts_with(out, reads) or starts_with(gate, (*reads, out)) or starts_with(up, (*reads, out, gate)):
        raise ValueError("results must not share memory with what is read or with one another")
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    if keep and gate is None:
        gate = x.new_empty((x.shape[0], w_gate.shape[0]))
    if keep and up is None:
        up = x.new_empty((x.shape[0], w_gate.shape[0]))
    if plan is None:
        plan = _plans.remember(sig, _Plan(x, w_gate, act, (x, w_gate, w_up, w_down, out, gate, up), False))
    workspace = _workspace(workspace, plan, x, device)
    for b, t in zip(plan.blocks, (x, w_gate, w_up, w_down, out, gate, up)):
        b.data = address(t)
    _check(load_library().adacons_ffn_forward(plan.shape_ref, *plan.refs, workspace.data_ptr(), workspace.numel() * workspace.element_size(), _raw_stream(None, device)),
           "adacons_ffn_forward")
    return out, gate, up


def _workspace(workspace, plan, x, device):
    if workspace is None:
        return x.new_empty(plan.workspace, dtype=torch.uint8)
    if workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous on x's device")
    return workspace


def workspace_bytes(x, w_gate, backward: bool = False) -> int:
    """Bytes of device memory that the forward or the backward pass works in."""
    return _Plan(x, w_gate, ACTS[0], (), backward).workspace


def feedforward_backward(dout, x, w_gate, w_up, w_down, gate, up, *, act: str = "silu", dx=None, dw_gate=None, dw_up=None, dw_down=None, want=(True, True, True, True),
                         workspace=None, stream=None):
    """(dx, dw_gate, dw_up, dw_down) of feedforward_forward with the same act, from its gate and up and the gradient dout.
    want: which of the four are made; the others are None.  They are made here unless given, as is the workspace (a uint8 tensor of workspace_bytes,
    16-byte aligned).  Between the products gradients are held in the tensors' type (float16: times a power of two where dout is small or they would be
    infinite)."""
    want = tuple(bool(w) for w in want)
    given = (dx, dw_gate, dw_up, dw_down)
    sig = (layout(dout), layout(x), layout(w_gate), layout(w_up), layout(w_down), layout(gate), layout(up), act, want, *(layout(t) for t in given))
    plan = _back_plans.known.get(sig)
    if plan is None:
        check_feedforward(x, w_gate, w_up, w_down, act, like_x=[("dout", dout), ("dx", dx)], like_hidden=[("gate", gate), ("up", up)],
                          like_gate=[("dw_gate", dw_gate), ("dw_up", dw_up)], like_down=[("dw_down", dw_down)])
        if len(want) != 4 or any(t is not None and not w for t, w in zip(given, want)):
            raise ValueError("want says for each of dx, dw_gate, dw_up and dw_down whether it is made; one that is given is")
    device = sig[1][3]
    if not here(device, stream):
        results = elsewhere(device, stream, tuple(t if w else True for t, w in zip(given, want)), lambda: feedforward_backward(
            dout, x, w_gate, w_up, w_down, gate, up, act=act, dx=dx, dw_gate=dw_gate, dw_up=dw_up, dw_down=dw_down, want=want, workspace=workspace))
        if results is not None:
            return results
    reads = (dout, x, w_gate, w_up, w_down, gate, up)
    if any(t is not None for t in given) and any(starts_with(t, (*reads, *given[:k])) for k, t in enumerate(given)):
        raise ValueError("results must not share memory with what is read or with one another")
    made = [t if t is not None or not w else torch.empty_like(like, memory_format=torch.contiguous_format) for t, w, like in zip(given, want, (x, w_gate, w_up, w_down))]
    if plan is None:
        plan = _back_plans.remember(sig, _Plan(x, w_gate, act, (*reads, *made), True))
    workspace = _workspace(workspace, plan, x, device)
    for b, t in zip(plan.blocks, (*reads, *made)):
        b.data = address(t)
    _check(load_library().adacons_ffn_backward(plan.shape_ref, *plan.refs, workspace.data_ptr(), workspace.numel() * workspace.element_size(), _raw_stream(None, device)),
           "adacons_ffn_backward")
    return tuple(made)


def status(stream=None) -> int:
    """The ADACONS_FLAG_TIMEOUT bit of the feed-forward calls on the current device (a given stream's) since the last look (0: all waits ended)."""
    device = getattr(stream, "device", None)
    if device is not None and device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return status(stream)
    v = ctypes.c_uint32()
    _check(load_library().adacons_ffn_get_status(ctypes.byref(v), _stream_handle(stream)), "adacons_ffn_get_status")
    return v.value


def selftest_bounded_wait(x, w_gate, w_up, paired: bool) -> None:
    """The first product on the current device and stream with operands that never come, by a pair of blocks or a lone one: the waits run out (2 s each) and
    status() says so.  bfloat16, a single tile."""
    plan = _Plan(x, w_gate, ACTS[0], (x, w_gate, w_up), False)
    for b, t in zip(plan.blocks, (x, w_gate, w_up)):
        b.data = t.data_ptr()
    workspace = x.new_empty(plan.workspace, dtype=torch.uint8)
    _check(load_library().adacons_selftest_ffn(plan.shape_ref, int(paired), *plan.refs, workspace.data_ptr(), workspace.numel(), _raw_stream(None, x.get_device())),
           "adacons_selftest_ffn")


def gated_feedforward(x, w_gate, w_up, w_down, act: str = "silu"):
    """feedforward_forward's out as a function of x, of any leading dimensions, and the weights that can be differentiated once.  Where no gradient is
    recorded, gate and up are not made."""
    rows = _aligned(x.reshape(-1, x.shape[-1]))
    # asked here: inside a Function's forward gradients are off, and what its inputs need is told whether or not they were on
    keep = torch.is_grad_enabled() and any(t.requires_grad for t in (x, w_gate, w_up, w_down))
    return _FeedForward.apply(rows, *(_aligned(w) for w in (w_gate, w_up, w_down)), act, keep).view(*x.shape[:-1], w_down.shape[0])


def _aligned(t):
    """t, or a copy of it where the kernels could not read it: a broadcast or transposed one, a slice off a 16-byte boundary."""
    if t.dim() == 2 and (t.data_ptr() % 16 != 0 or t.stride(1) != 1 or (t.shape[0] > 1 and (t.stride(0) % 8 != 0 or t.stride(0) < t.shape[1]))):
        return t.clone(memory_format=torch.contiguous_format)
    return t


class _FeedForward(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, w_down, act, keep):
        out, gate, up = feedforward_forward(x, w_gate, w_up, w_down, act=act, keep=keep)
        if keep:
            ctx.save_for_backward(x, w_gate, w_up, w_down, gate, up)
            ctx.act = act
        return out

    @staticmethod
    def backward(ctx, dout):
        x, w_gate, w_up, w_down, gate, up = ctx.saved_tensors
        compute = _Gradient.apply if torch.is_grad_enabled() else _Gradient.compute
        return (*compute(_aligned(dout), x, w_gate, w_up, w_down, gate, up, ctx.act, tuple(ctx.needs_input_grad[:4])), None, None)


class _Gradient(torch.autograd.Function):
    """The gradient where a graph of it is recorded: differentiating it again is an error (taken for a constant, it would silently leave
    terms out of a second derivative)."""

    @staticmethod
    def compute(dout, x, w_gate, w_up, w_down, gate, up, act, want):
        return feedforward_backward(dout, x, w_gate, w_up, w_down, gate, up, act=act, want=want)

    @staticmethod
    def forward(ctx, *args):
        return _Gradient.compute(*args)

    @staticmethod
    def backward(ctx, *grads):
        raise NotImplementedError("the feed-forward block can be differentiated once: its gradient has no gradient of its own")
