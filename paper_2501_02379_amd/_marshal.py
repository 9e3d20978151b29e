"""What the bindings of the operators around the step share: tensor checks, type codes, streams."""
from __future__ import annotations

import functools

import torch

from . import tgrad as T

REAL_TYPES = {torch.float32: T.TGRAD_F32, torch.bfloat16: T.TGRAD_BF16, torch.float16: T.TGRAD_F16}


def refuse(what: str):
    raise T.TgradError(T.TGRAD_ERR_INVALID_ARG, what)


def used_on(stream, tensors):
    """Tensors of another stream's allocator that kernels on `stream` work on: the caller may let go of them at once, and their memory
    is not handed out again before those kernels have run."""
    for t in tensors:
        if isinstance(t, torch.Tensor) and t.is_cuda:
            t.record_stream(stream)


def on_stream(f):
    """Adds `stream=`: the call runs with that stream current, so that what it allocates belongs to it (memory of another stream's
    could still be in use there, and scratch could be handed out again before the kernels have run)."""
    @functools.wraps(f)
    def run(*args, stream=None, **kw):
        if stream is None:
            return f(*args, **kw)
        for t in (*args, *kw.values()):
            if isinstance(t, torch.Tensor) and t.is_cuda and t.device != stream.device:
                refuse("stream: one of the logits' device")
        with torch.cuda.stream(stream):
            result = f(*args, **kw)
        used_on(stream, (*args, *kw.values()))
        return result
    return run


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def stream_of(device) -> int:
    """The handle of the device's current stream (without a Stream object around it where torch offers that: 0.2 us instead of 2)."""
    if _raw_stream is not None:
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


def vector(t, n, dtype, device, what):
    """Address of a dense vector of n elements (None stays None); anything else is refused."""
    if t is None:
        return None
    if t.dtype is not dtype or t.dim() != 1 or t.numel() != n or t.get_device() != device.index or not t.is_contiguous() or t.is_neg():
        refuse("%s: %s[%d], dense, on the logits' device, no pending negation" % (what, dtype, n))
    return t.data_ptr()


def scalar(t, dtype, device, what):
    """Address of a tensor of one element, of any dimension (None stays None)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != 1 or t.get_device() != device.index or t.is_neg():
        refuse("%s: one %s on the logits' device, no pending negation" % (what, dtype))
    return t.data_ptr()


def check(rc: int, where: str) -> None:
    if rc != T.TGRAD_OK:
        raise T.TgradError(rc, where)


def call(device, fn, where, *args):
    """One library call with `device` current."""
    if torch.cuda.current_device() == device.index:
        rc = fn(*args)
    else:
        with torch.cuda.device(device):
            rc = fn(*args)
    check(rc, where)


