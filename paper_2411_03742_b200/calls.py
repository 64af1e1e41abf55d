"""What the calls of the operators without a context share: layouts that have passed the checks, devices, streams."""
from __future__ import annotations

import threading

import torch

from .binding import _raw_stream, check_stream, on_stream

# torch.cuda.current_device() without its look whether the runtime is up: whoever asks here holds a CUDA tensor
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


class Plans(threading.local):
    """Per thread: what the checks of a layout have led to, by the layout.  Only data pointers change between calls, and
    nothing of a call is kept but layouts and plain values."""

    def __init__(self):
        self.known = {}

    def remember(self, sig, plan):
        if len(self.known) >= 1024:        # a program with ever new lengths
            self.known.clear()
        self.known[sig] = plan
        return plan


def layout(t):
    return None if t is None else (t.dtype, t.shape, t.stride(), t.get_device())


def here(device: int, stream) -> bool:
    """Whether a call on tensors of `device` can go ahead as it is; elsewhere() makes it otherwise."""
    return stream is None and device == _current_device()


def elsewhere(device: int, stream, given, call):
    """None where a call on tensors of `device` can go ahead as it is; otherwise the results of call() with their device current, or
    with the stream that was asked for current, for whose results that were not `given` the caller's stream is noted as a user."""
    if device != _current_device():
        with torch.cuda.device(device):
            return elsewhere(device, stream, given, call) or call()
    if stream is None:
        return None
    check_stream(stream, device)
    if stream.cuda_stream == _raw_stream(None, device):
        return None
    return on_stream(stream, device, given, call)


def address(t):
    return None if t is None else t.data_ptr()


def starts_with(t, others) -> bool:
    """Whether t, where it has elements, starts where another tensor with elements does."""
    return t is not None and t.numel() > 0 and any(o is not None and o.numel() > 0 and o.data_ptr() == t.data_ptr() for o in others)
