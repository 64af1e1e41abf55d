"""Distillation from a teacher's top logits through the library's kernels.

A teacher's full logits are rarely kept: for each token there are the K largest and their indices.  `distill_forward` makes
each token's loss, the divergence of the student's distribution from the teacher's over those entries, mixed with the cross entropy of
a label where there are labels; `distill_backward` the gradient of the student's logits; `distill` is the two of them as one
differentiable torch operation.  Argument marshalling only: the arithmetic runs in the library's CUDA kernels, and there is no fallback.
"""
from __future__ import annotations

import ctypes

import torch

from .binding import _check, _raw_stream, load_library
from .calls import Plans, address, elsewhere, here, layout, starts_with
from .norms import _CODES

MAX_TOP = 1024
_BITS = {torch.int32: 32, torch.int64: 64}


class _Matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64)]


class _Shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("dtype", "teacher_dtype", "ids_bits", "labels_bits", "tokens", "vocab", "top")] + \
               [("temperature", ctypes.c_float), ("mix", ctypes.c_float)]


class _Plan:
    def __init__(self, logits, ids, teacher, labels, temperature, mix, matrices):
        self.shape = _Shape(_CODES[logits.dtype], _CODES[teacher.dtype], _BITS[ids.dtype], 0 if labels is None else _BITS[labels.dtype], logits.shape[0], logits.shape[1],
                            ids.shape[1], temperature, mix)
        self.shape_ref = ctypes.byref(self.shape)
        self.blocks = [_Matrix(None, t.stride(0)) for t in matrices]
        self.refs = [ctypes.byref(b) for b in self.blocks]


_plans, _back_plans = Plans(), Plans()


def check_distill(logits, ids, teacher, temperature: float, labels=None, mix: float = 1.0, loss=None, rows=None, dloss=None, out=None, want_cuda: bool = True) -> None:
    """Raise ValueError unless logits is (token, vocabulary), ids and teacher are (token, entry), labels (token,), on one device and of types that the kernels
    have; loss (token,) and rows (2, token) contiguous fp32, dloss fp32 (token,), out like logits."""
    if logits.dim() != 2 or ids.dim() != 2:
        raise ValueError("logits and ids must have two dimensions: token, vocabulary and token, entry")
    T, V = logits.shape
    K = ids.shape[1]
    if V < 1 or V > 2 ** 30 or T > 2 ** 27:
        raise ValueError(f"1 to 2^30 logits of at most 2^27 tokens, got {tuple(logits.shape)}")
    if not 1 <= K <= MAX_TOP:
        raise ValueError(f"1 to {MAX_TOP} entries, got {K}")
    if logits.dtype not in _CODES or teacher.dtype not in _CODES:
        raise ValueError(f"logits are float32, bfloat16 or float16, got {logits.dtype} and {teacher.dtype}")
    if ids.dtype not in _BITS or (labels is not None and labels.dtype not in _BITS):
        raise ValueError("ids and labels are int32 or int64")
    if tuple(ids.shape) != (T, K) or tuple(teacher.shape) != (T, K):
        raise ValueError(f"ids {tuple(ids.shape)} and teacher {tuple(teacher.shape)} do not fit logits {tuple(logits.shape)}")
    if not 2.0 ** -60 <= temperature <= 2.0 ** 60:
        raise ValueError(f"temperature must lie between 2^-60 and 2^60, got {temperature}")
    if not 0 <= mix <= 1:
        raise ValueError("mix lies between 0 and 1")
    if out is not None and (out.dtype != logits.dtype or out.shape != logits.shape):
        raise ValueError(f"out must be {logits.dtype} of shape {tuple(logits.shape)}, got {out.dtype} {tuple(out.shape)}")
    for name, t in (("logits", logits), ("ids", ids), ("teacher", teacher), ("out", out)):
        if t is None:
            continue
        if t.device != logits.device or (want_cuda and not t.is_cuda):
            raise ValueError(f"{name} must be a CUDA tensor on the logits' device")
        if t.shape[1] > 1 and t.stride(1) != 1:
            raise ValueError(f"{name} must have unit stride along a token's row")
    if out is not None and T > 1 and abs(out.stride(0)) < V:
        raise ValueError("out must not be a broadcast view")
    if labels is not None and (tuple(labels.shape) != (T,) or labels.device != logits.device or (T > 1 and labels.stride(0) != 1)):
        raise ValueError(f"labels must be contiguous of shape {(T,)} on the logits' device")
    for name, t, shape in (("loss", loss, (T,)), ("rows", rows, (2, T))):
        if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != shape or not t.is_contiguous() or t.device != logits.device):
            raise ValueError(f"{name} must be a contiguous float32 tensor of shape {shape} on the logits' device")
    if dloss is not None and (dloss.dtype != torch.float32 or tuple(dloss.shape) != (T,) or dloss.device != logits.device):
        raise ValueError(f"dloss must be a float32 tensor of shape {(T,)} on the logits' device")


def _mix(labels, mix) -> float:
    if labels is None:
        return 1.0 if mix is None else float(mix)
    if mix is None:
        raise ValueError("labels need a mix: the divergence's share, the cross entropy has the rest")
    return float(mix)


def distill_forward(logits, ids, teacher, *, temperature: float = 1.0, labels=None, mix=None, loss=None, rows=None, stream=None):
    """(loss, rows): per token  mix temperature^2 KL(p || softmax(logits / temperature)) + (1 - mix) cross_entropy(logits, label),
    p the softmax of teacher / temperature over the token's entries.

    logits: (token, vocabulary); ids, teacher: (token, entry), the entries' indices (int32 or int64) and the teacher's logits there.  An index outside the
    vocabulary (-1, say) or a logit of -inf marks an entry that is not there; a label outside it (-100) one that is unknown.  A token
    without entries has no first term, one without a label no second.  Without labels mix is 1 unless given.
    rows: both log-sum-exps, (2, token) fp32, for the gradient.  loss and rows are made here unless given."""
    temperature, mix = float(temperature), _mix(labels, mix)
    sig = (layout(logits), layout(ids), layout(teacher), layout(labels), temperature, mix, layout(loss), layout(rows))
    plan = _plans.known.get(sig)
    if plan is None:
        check_distill(logits, ids, teacher, temperature, labels, mix, loss, rows)
    device = sig[0][3]
    if not here(device, stream):
        results = elsewhere(device, stream, (loss, rows), lambda: distill_forward(logits, ids, teacher, temperature=temperature, labels=labels, mix=mix, loss=loss, rows=rows))
        if results is not None:
            return results
    if starts_with(loss, (logits, ids, teacher, labels, rows)) or starts_with(rows, (logits, ids, teacher, labels)):
        raise ValueError("loss and rows must not share memory with what is read or with one another")
    if loss is None:
        loss = logits.new_empty(logits.shape[0], dtype=torch.float32)
    if rows is None:
        rows = logits.new_empty((2, logits.shape[0]), dtype=torch.float32)
    if plan is None:
        plan = _plans.remember(sig, _Plan(logits, ids, teacher, labels, temperature, mix, (logits, ids, teacher)))
    for b, t in zip(plan.blocks, (logits, ids, teacher)):
        b.data = t.data_ptr()
    _check(load_library().adacons_distill_forward(plan.shape_ref, *plan.refs, address(labels), loss.data_ptr(), rows.data_ptr(), _raw_stream(None, device)), "adacons_distill_forward")
    return loss, rows


def distill_backward(dloss, logits, ids, teacher, rows, *, temperature: float = 1.0, labels=None, mix=None, out=None, stream=None):
    """The gradient of distill_forward's logits, of their type, from dloss (fp32, one for each token) and the forward pass's rows, with the same arguments.
    out: a new tensor unless given, whose rows lie as the logits' do relative to 16 bytes; logits itself is allowed (they are overwritten), no other overlap."""
    temperature, mix = float(temperature), _mix(labels, mix)
    sig = (layout(dloss), layout(logits), layout(ids), layout(teacher), layout(rows), layout(labels), temperature, mix, layout(out))
    plan = _back_plans.known.get(sig)
    if plan is None:
        check_distill(logits, ids, teacher, temperature, labels, mix, None, rows, dloss, out)
    device = sig[1][3]
    if not here(device, stream):
        results = elsewhere(device, stream, (out,), lambda: (distill_backward(dloss, logits, ids, teacher, rows, temperature=temperature, labels=labels, mix=mix, out=out),))
        if results is not None:
            return results[0]
    if out is not None and (starts_with(out, (dloss, ids, teacher, rows, labels)) or (starts_with(out, (logits,)) and out.stride() != logits.stride())):
        raise ValueError("out may be the logits, otherwise it must not share memory with what is read")
    if out is None:
        # it lies as the logits do relative to 16 bytes, so that both are moved in vectors (one by one they take five times as long): as far behind the first boundary, rows
        # as far apart.  What lies between the rows is not written.
        T, V = logits.shape
        unit = 16 // logits.element_size()
        pad = (logits.stride(0) - V) % unit if T > 1 else 0
        lead = logits.data_ptr() % 16 // logits.element_size()
        if lead:
            out = torch.as_strided(logits.new_empty(lead + T * (V + pad)), (T, V), (V + pad, 1), lead)
        else:
            out = logits.new_empty((T, V + pad))[:, :V]
    if plan is None:
        plan = _back_plans.remember(sig, _Plan(logits, ids, teacher, labels, temperature, mix, (logits, ids, teacher, out)))
    for b, t in zip(plan.blocks, (logits, ids, teacher, out)):
        b.data = t.data_ptr()
    r = plan.refs
    _check(load_library().adacons_distill_backward(plan.shape_ref, dloss.data_ptr(), dloss.stride(0), r[0], r[1], r[2], address(labels), rows.data_ptr(), r[3],
                                                   _raw_stream(None, device)), "adacons_distill_backward")
    return out


def distill(logits, ids, teacher, *, temperature: float = 1.0, labels=None, mix=None):
    """distill_forward's loss, one for each token, as a function of the logits that can be differentiated once.  The teacher is a constant.
    What does not lie as the passes want it, along rows, is copied."""
    for name, t in (("the teacher's logits", teacher), ("the temperature", temperature), ("mix", mix)):
        if getattr(t, "requires_grad", False):
            raise ValueError(f"distillation has no gradient for {name}")
    logits, ids, teacher = (t if t.dim() != 2 or t.shape[1] <= 1 or t.stride(1) == 1 else t.contiguous() for t in (logits, ids, teacher))
    return _Distill.apply(logits, ids, teacher, float(temperature), None if labels is None else labels.contiguous(), _mix(labels, mix))


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids, teacher, temperature, labels, mix):
        loss, rows = distill_forward(logits, ids, teacher, temperature=temperature, labels=labels, mix=mix)
        ctx.save_for_backward(logits, ids, teacher, rows, labels)
        ctx.how = {"temperature": temperature, "mix": mix}
        return loss

    @staticmethod
    def backward(ctx, dloss):
        logits, ids, teacher, rows, labels = ctx.saved_tensors
        compute = _Gradient.apply if torch.is_grad_enabled() else _Gradient.compute
        return compute(dloss, logits, ids, teacher, rows, labels, ctx.how), None, None, None, None, None


class _Gradient(torch.autograd.Function):
    """The gradient where a graph of it is recorded: differentiating it again is an error (taken for a constant, it would silently leave
    terms out of a second derivative)."""

    @staticmethod
    def compute(dloss, logits, ids, teacher, rows, labels, how):
        return distill_backward(dloss, logits, ids, teacher, rows, labels=labels, **how)

    @staticmethod
    def forward(ctx, *args):
        return _Gradient.compute(*args)

    @staticmethod
    def backward(ctx, *grads):
        raise NotImplementedError("distillation can be differentiated once: its gradient has no gradient of its own")
