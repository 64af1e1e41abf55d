"""Attention and its gradient through the library's kernels.

`attention_forward` and `attention_backward` marshal arguments only; `attention` is the two of them as
one differentiable torch operation.  Tensors are (batch, token, head, element) in bf16 or fp16, with any
strides whose last one is 1 and whose others are multiples of 8: slices of a packed projection, or
head-major memory seen through a transpose, are taken as they are.  There is no fallback.
"""
from __future__ import annotations

import ctypes
import math
import threading

import torch

from .binding import BF16, _check, _raw_stream, _stream_handle, check_stream, load_library, on_stream

F16 = 2
# torch.cuda.current_device() without its look whether the runtime is up: whoever asks here holds a CUDA tensor
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
SHORT_ROWS = 256        # query rows around a key head up to which the backward pass can do without a workspace


class _Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("seq_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class _Shape(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("batch", ctypes.c_int), ("q_heads", ctypes.c_int), ("kv_heads", ctypes.c_int), ("q_len", ctypes.c_int),
                ("kv_len", ctypes.c_int), ("head_dim", ctypes.c_int), ("causal", ctypes.c_int), ("scale", ctypes.c_float), ("kv_lens", ctypes.c_void_p)]


class _Plans(threading.local):
    """Per thread: the argument blocks of layouts that have passed the checks.  Only the data pointers change between
    calls, and nothing of a call is kept but its layout, the scale's value and the kind of mask (a tensor in the key would
    go by its identity: a scale that a program changes in place would stay what it was at the first call)."""

    def __init__(self):
        self.known = {}


_plans = _Plans()


class _Plan:
    """Shape and tensor blocks of one layout, and references to them for the call."""

    def __init__(self, shape, tensors):
        self.shape, self.shape_ref = shape, ctypes.byref(shape)
        self.blocks = [_Tensor(None, *t.stride()[:3]) for t in tensors]
        self.refs = [ctypes.byref(b) for b in self.blocks]
        self.workspace = 0


def _remember(sig, plan):
    if len(_plans.known) >= 1024:        # a program with ever new lengths
        _plans.known.clear()
    _plans.known[sig] = plan
    return plan


def check_attention(q, k, v, kv_lens=None, like_q=(), like_k=(), rows=(), want_cuda: bool = True) -> None:
    """Raise ValueError unless q, k, v (and what is shaped like them) are 4-D tensors of one 16-bit type on one
    device whose sizes fit together; rows: (batch, q_heads, q_len) fp32 tensors; kv_lens: int32 (batch,)."""
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        raise ValueError("q, k and v must have four dimensions: batch, token, head, element")
    if q.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"attention takes bfloat16 and float16, got {q.dtype}")
    B, Sq, Hq, D = q.shape
    if k.shape != v.shape or k.shape[0] != B or k.shape[3] != D:
        raise ValueError(f"k {tuple(k.shape)} and v {tuple(v.shape)} do not fit q {tuple(q.shape)}")
    if k.shape[2] == 0 or Hq == 0 or Hq % k.shape[2] != 0:
        raise ValueError(f"{Hq} query heads cannot share {k.shape[2]} key heads")
    if D % 8 != 0 or not 8 <= D <= 128:
        raise ValueError(f"head sizes are multiples of 8 up to 128, got {D}")
    for name, t, shape in [("k", k, k.shape), ("v", v, k.shape)] + [(n, t, q.shape) for n, t in like_q] + [(n, t, k.shape) for n, t in like_k]:
        if t.dtype != q.dtype or t.shape != shape:
            raise ValueError(f"{name} must be {q.dtype} of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    for name, t in [("q", q), ("k", k), ("v", v)] + list(like_q) + list(like_k):
        if t.device != q.device or (want_cuda and not t.is_cuda):
            raise ValueError(f"{name} must be a CUDA tensor on q's device")
        if t.stride(3) != 1 or any(t.shape[i] > 1 and (t.stride(i) % 8 != 0 or t.stride(i) <= 0) for i in range(3)):
            raise ValueError(f"{name}: the last stride must be 1 and the others positive multiples of 8, got {t.stride()}")
    for name, t in rows:
        if t.dtype != torch.float32 or tuple(t.shape) != (B, Hq, Sq) or not t.is_contiguous() or t.device != q.device:
            raise ValueError(f"{name} must be a contiguous float32 tensor of shape {(B, Hq, Sq)} on q's device")
    if kv_lens is not None and (kv_lens.dtype != torch.int32 or tuple(kv_lens.shape) != (B,) or kv_lens.device != q.device or (B > 1 and kv_lens.stride(0) != 1)):
        raise ValueError(f"kv_lens must be a contiguous int32 tensor of shape {(B,)} on q's device")


def _layout(t):
    return None if t is None else (t.dtype, t.shape, t.stride(), t.get_device())


def _shape(q, k, scale, causal, kv_lens):
    B, Sq, Hq, D = q.shape
    return _Shape(BF16 if q.dtype == torch.bfloat16 else F16, B, Hq, k.shape[2], Sq, k.shape[1], D, int(causal),
                  1.0 / math.sqrt(D) if scale is None else scale, None if kv_lens is None else kv_lens.data_ptr())


def attention_forward(q, k, v, *, scale=None, causal: bool = False, kv_lens=None, out=None, lse=None, stream=None):
    """(out, lse): out = softmax(scale q k^T + mask) v, shaped like q, and the rows' log-sum-exp, (batch,
    q_heads, q_len) fp32.  scale defaults to head_dim^-1/2; kv_lens (int32) hides each batch's keys from there on.
    out and lse are made here unless given; a given out must not share memory with the inputs.
    stream: where the kernels go (the current one by default); the caller orders it behind whatever makes the inputs, and its own
    use of the results behind it."""
    scale, causal = None if scale is None else float(scale), bool(causal)        # as they are now: see _Plans
    sig = (_layout(q), _layout(k), _layout(v), _layout(kv_lens), scale, causal, _layout(out), _layout(lse))
    plan = _plans.known.get(sig)
    if plan is None:
        check_attention(q, k, v, kv_lens, like_q=[] if out is None else [("out", out)], rows=[] if lse is None else [("lse", lse)])
    if sig[0][3] != _current_device():        # the kernels run on the current device
        with torch.cuda.device(sig[0][3]):
            return attention_forward(q, k, v, scale=scale, causal=causal, kv_lens=kv_lens, out=out, lse=lse, stream=stream)
    if stream is not None:
        check_stream(stream, sig[0][3])
        if stream.cuda_stream != _raw_stream(None, sig[0][3]):
            return on_stream(stream, sig[0][3], (out, lse), lambda: attention_forward(q, k, v, scale=scale, causal=causal, kv_lens=kv_lens, out=out, lse=lse))
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if lse is None:
        lse = q.new_empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32)
    if plan is None:
        plan = _remember(sig, _Plan(_shape(q, k, scale, causal, kv_lens), (q, k, v, out)))
    if kv_lens is not None:
        plan.shape.kv_lens = kv_lens.data_ptr()
    for block, t in zip(plan.blocks, (q, k, v, out)):
        block.data = t.data_ptr()
    _check(load_library().adacons_attn_forward(plan.shape_ref, *plan.refs, lse.data_ptr(), _raw_stream(stream, sig[0][3])), "adacons_attn_forward")
    return out, lse


def workspace_bytes(q, k) -> int:
    """Bytes of device memory that attention_backward works in."""
    n = ctypes.c_int64()
    _check(load_library().adacons_attn_workspace_bytes(ctypes.byref(_shape(q, k, None, False, None)), ctypes.byref(n)), "adacons_attn_workspace_bytes")
    return n.value


def _one_launch(q, k) -> bool:
    """Whether the backward pass goes without a workspace: where its blocks all run at once (two an SM up to head size 64)
    the call is bound by the host, and one launch without an allocation is 4 us less (16.0 against 20.2 for 3 x 77
    tokens of 4 heads); where they do not, the repeated statistics show (8 x 256 tokens of 16 heads: 26.0 against 24.7 us).
    In fp16 every block looks through all values of its head as well: 17.8 against 20.3 us at 1024 keys of 64 elements,
    18.9 and 20.5 at 512 of 128, but 23.7 and 20.5 at 1024 of 128."""
    q_tiles, k_tiles = -(-q.shape[1] // 128), -(-k.shape[1] // 128)
    if q.shape[2] // k.shape[2] * q_tiles * 128 > SHORT_ROWS:
        return False
    if q.dtype == torch.float16 and k.shape[1] * (64 if q.shape[3] <= 64 else 128) > 65536:
        return False
    resident = torch.cuda.get_device_properties(q.device).multi_processor_count * (2 if q.shape[3] <= 64 else 1)
    return q.shape[0] * (q_tiles * q.shape[2] + k_tiles * k.shape[2]) <= resident


def attention_backward(dout, q, k, v, out, lse, *, scale=None, causal: bool = False, kv_lens=None, dq=None, dk=None, dv=None, workspace=None,
                       stream=None):
    """(dq, dk, dv) of attention_forward with the same scale, causal and kv_lens, from its out and lse and the
    gradient dout.  workspace: a uint8 tensor of workspace_bytes(q, k), made here if needed and not given.
    dq, dk and dv, where given, must not share memory with the inputs or one another."""
    scale, causal = None if scale is None else float(scale), bool(causal)        # as they are now: see _Plans
    sig = (_layout(q), _layout(k), _layout(v), _layout(kv_lens), scale, causal, _layout(out), _layout(lse), _layout(dout), _layout(dq), _layout(dk), _layout(dv))
    plan = _plans.known.get(sig)
    if plan is None:
        check_attention(q, k, v, kv_lens, like_q=[(n, t) for n, t in (("dout", dout), ("out", out), ("dq", dq)) if t is not None],
                        like_k=[(n, t) for n, t in (("dk", dk), ("dv", dv)) if t is not None], rows=[("lse", lse)])
    if sig[0][3] != _current_device():        # the kernels run on the current device
        with torch.cuda.device(sig[0][3]):
            return attention_backward(dout, q, k, v, out, lse, scale=scale, causal=causal, kv_lens=kv_lens, dq=dq, dk=dk, dv=dv, workspace=workspace, stream=stream)
    if stream is not None:
        check_stream(stream, sig[0][3])
        if stream.cuda_stream != _raw_stream(None, sig[0][3]):
            return on_stream(stream, sig[0][3], (dq, dk, dv), lambda: attention_backward(
                dout, q, k, v, out, lse, scale=scale, causal=causal, kv_lens=kv_lens, dq=dq, dk=dk, dv=dv, workspace=workspace))
    dq = torch.empty_like(q, memory_format=torch.contiguous_format) if dq is None else dq
    dk = torch.empty_like(k, memory_format=torch.contiguous_format) if dk is None else dk
    dv = torch.empty_like(v, memory_format=torch.contiguous_format) if dv is None else dv
    if plan is None:
        plan = _Plan(_shape(q, k, scale, causal, kv_lens), (dout, q, k, v, out, dq, dk, dv))
        if not _one_launch(q, k):
            plan.workspace = workspace_bytes(q, k)
        _remember(sig, plan)
    if workspace is None:
        if plan.workspace:
            workspace = lse.new_empty(plan.workspace // 4)
    elif workspace.get_device() != sig[0][3] or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous on q's device")
    if kv_lens is not None:
        plan.shape.kv_lens = kv_lens.data_ptr()
    for block, t in zip(plan.blocks, (dout, q, k, v, out, dq, dk, dv)):
        block.data = t.data_ptr()
    r = plan.refs
    _check(load_library().adacons_attn_backward(plan.shape_ref, r[0], r[1], r[2], r[3], r[4], lse.data_ptr(), r[5], r[6], r[7],
                                                None if workspace is None else workspace.data_ptr(),
                                                0 if workspace is None else workspace.numel() * workspace.element_size(), _raw_stream(stream, sig[0][3])), "adacons_attn_backward")
    return dq, dk, dv


def status(stream=None) -> int:
    """The ADACONS_FLAG_TIMEOUT bit of the attention calls on the current device (a given stream's) since the last look (0: all waits ended)."""
    device = getattr(stream, "device", None)
    if device is not None and device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return status(stream)
    v = ctypes.c_uint32()
    _check(load_library().adacons_attn_get_status(ctypes.byref(v), _stream_handle(stream)), "adacons_attn_get_status")
    return v.value


def selftest_bounded_wait(q, k, v, out, lse, gradients=None) -> None:
    """The forward pass, or with gradients = (dq, dk, dv) the backward pass, on the current device and stream, with tiles that never come:
    the waits run out (2 s each) and status() says so.  What is written is invalid.  bf16, head sizes up to 64."""
    check_attention(q, k, v, like_q=[("out", out)], rows=[("lse", lse)])
    plan = _Plan(_shape(q, k, None, False, None), (q, k, v, out) + tuple(gradients or ()))
    for block, t in zip(plan.blocks, (q, k, v, out) + tuple(gradients or ())):
        block.data = t.data_ptr()
    workspace = lse.new_empty(workspace_bytes(q, k) // 4)
    _check(load_library().adacons_selftest_attention(plan.shape_ref, *plan.refs[:4], lse.data_ptr(), *(plan.refs[4:] or (None,) * 3), workspace.data_ptr(),
                                                     workspace.numel() * 4, _raw_stream(None, q.get_device())), "adacons_selftest_attention")


def attention(q, k, v, *, scale=None, causal: bool = False, kv_lens=None):
    """attention_forward's out as a function of q, k and v that can be differentiated once.  Not of the scale: a learned temperature
    belongs into q."""
    if getattr(scale, "requires_grad", False):
        raise ValueError("attention has no gradient for its scale: multiply q by a learned temperature instead")
    return _Attention.apply(q, k, v, None if scale is None else float(scale), bool(causal), kv_lens)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, scale, causal, kv_lens):
        out, lse = attention_forward(q, k, v, scale=scale, causal=causal, kv_lens=kv_lens)
        ctx.save_for_backward(q, k, v, out, lse, *([] if kv_lens is None else [kv_lens]))
        ctx.how = (scale, causal)
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, out, lse, *lens = ctx.saved_tensors
        if dout.data_ptr() % 16 != 0 or dout.stride(3) != 1 or any(n > 1 and (s % 8 != 0 or s <= 0) for n, s in zip(dout.shape[:3], dout.stride())):
            dout = dout.clone(memory_format=torch.contiguous_format)        # a broadcast gradient, of a sum for instance, or a slice off a 16-byte boundary
        gradient = _Gradient.apply if torch.is_grad_enabled() else _Gradient.compute
        return (*gradient(dout, q, k, v, out.detach(), lse, lens[0] if lens else None, *ctx.how), None, None, None)


class _Gradient(torch.autograd.Function):
    """The gradient where a graph of it is recorded: it depends on dout, q, k and v, and differentiating it again is an error
    (taken for a constant, it would silently leave terms out of a second derivative)."""

    @staticmethod
    def compute(dout, q, k, v, out, lse, lens, scale, causal):
        return attention_backward(dout, q, k, v, out, lse, scale=scale, causal=causal, kv_lens=lens)

    @staticmethod
    def forward(ctx, *args):
        return _Gradient.compute(*args)

    @staticmethod
    def backward(ctx, *grads):
        raise NotImplementedError("attention can be differentiated once: its gradient has no gradient of its own")
