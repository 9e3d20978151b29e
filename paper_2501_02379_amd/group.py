"""A group of tensors - gradients, parameters, moments - for the global gradient norm, clipping and AdamW: ctypes binding of the
tgrad_group_* entry points of include/tgrad.h."""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional, Sequence

import torch

from . import tgrad as T
from ._marshal import REAL_TYPES, call, check, refuse, stream_of, used_on

TYPES = {**REAL_TYPES, torch.complex64: T.TGRAD_C64}


_ENTRY = struct.Struct("=q5Q2i2f")        # tgrad_tensor
assert _ENTRY.size == C.sizeof(T.tgrad_tensor)


def _tensors(tensors, n, what, index):
    """n tensors (or None) on GPU `index`, dense."""
    if tensors is None:
        return [None] * n
    tensors = list(tensors)
    if len(tensors) != n:
        refuse("%s: one for every gradient" % what)
    for t in tensors:
        if t is not None and (t.get_device() != index or not t.is_contiguous()):
            refuse("%s: dense tensors on one GPU" % what)
        if t is not None and (t.is_conj() or t.is_neg()):     # autograd leaves such gradients; memory holds other numbers than the tensor
            refuse("%s: tensors without a pending conjugation or negation (resolve_conj(), resolve_neg())" % what)
    return tensors


def _type(t, what):
    """Elements and type code."""
    kind = TYPES.get(t.dtype)
    if kind is not None:
        return t.numel(), kind
    if t.dtype is torch.int16 and t.shape[-1:] == (2,):
        return t.numel() // 2, T.TGRAD_CBF16
    refuse("%s: float32, bfloat16, float16, complex64, or bf16 pairs as int16[..., 2]" % what)


class Group:
    """Gradients of any shapes and types (float32, bfloat16, float16, complex64) and, for AdamW, their parameters and float32
    moments; bf16 (re, im) pairs are int16 tensors with a trailing axis of 2, as everywhere in this library.  `exp_avg` has the
    gradient's shape (complex64, or float32 with a trailing axis of 2, for a complex tensor), `exp_avg_sq` float32 with one number
    per element.  `outs`: where `tgrad_group_scale` and `tgrad_group_clip` put the scaled gradients (None: in place).

    Every call is enqueued on the stream given here (the device's current one by default) and waits for nothing.  The group
    keeps its tensors alive; where its stream is not the current one they are recorded on it, so that tensors that a bind replaces,
    or those of a group that is dropped, last until the calls before have run.  Results (`tgrad_group_grad_norm`, `tgrad_group_clip`) are a float32 tensor (norm, factor) on the
    device; the buffer behind it also holds the sum of squares in float64, `group.sumsq(result)`.
    """

    def __init__(self, grads: Sequence[torch.Tensor], params=None, exp_avg=None, exp_avg_sq=None, outs=None,
                 lr_scale: Optional[Sequence[float]] = None, weight_decay: Optional[Sequence[float]] = None, stream=None):
        self.lib = T.load()
        self.handle = C.c_void_p(None)
        grads = list(grads)
        if not grads:
            refuse("a group has at least one tensor")
        if not grads[0].is_cuda:
            refuse("grads: tensors on the GPU")
        self.device = grads[0].device
        self.lr_scale, self.weight_decay = lr_scale, weight_decay
        table = self._table(grads, params, exp_avg, exp_avg_sq, outs)
        size = C.c_size_t(0)
        check(self.lib.tgrad_group_query_size(table, len(grads), C.byref(size)), "tgrad_group_query_size")
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        if self.stream.device != self.device:
            refuse("stream: one of the gradients' device")
        with torch.cuda.stream(self.stream):
            self.workspace = torch.empty(size.value, dtype=torch.uint8, device=self.device)
        call(self.device, self.lib.tgrad_group_init, "tgrad_group_init", C.byref(self.handle), table, len(grads),
             self.workspace.data_ptr(), self.stream.cuda_stream)
        self._used(*self.tensors)

    def _table(self, grads, params, exp_avg, exp_avg_sq, outs):
        n, index = len(grads), self.device.index
        grads = _tensors(grads, n, "grads", index)
        params, exp_avg = _tensors(params, n, "params", index), _tensors(exp_avg, n, "exp_avg", index)
        exp_avg_sq, outs = _tensors(exp_avg_sq, n, "exp_avg_sq", index), _tensors(outs, n, "outs", index)
        lr = self.lr_scale if self.lr_scale is not None else [1.0] * n
        wd = self.weight_decay if self.weight_decay is not None else [0.0] * n
        if len(lr) != n or len(wd) != n:
            refuse("lr_scale, weight_decay: one for every gradient")
        entries = []
        for g, p, m, v, o, scale, decay in zip(grads, params, exp_avg, exp_avg_sq, outs, lr, wd):
            if g is None:
                refuse("grads: a tensor each")
            numel, kind = _type(g, "grads")
            if o is not None and (o.dtype is not g.dtype or o.shape != g.shape):
                refuse("outs: the gradient's shape and type")
            pkind = kind
            if p is not None:
                cplx = kind == T.TGRAD_C64 or kind == T.TGRAD_CBF16
                count, pkind = _type(p, "params")
                if cplx and pkind == T.TGRAD_F32 and p.shape[-1:] == (2,):
                    count, pkind = count // 2, T.TGRAD_C64            # complex64 as float32 pairs
                if count != numel or m is None or v is None:
                    refuse("params: the gradient's number of elements, with moments")
                if m.dtype is torch.complex64:
                    size = 2 * m.numel()
                else:
                    size = m.numel() if m.dtype is torch.float32 else -1
                if size != (2 * numel if cplx else numel) or v.dtype is not torch.float32 or v.numel() != numel:
                    refuse("moments: float32, the parameter's size")
            elif m is not None or v is not None:
                refuse("moments belong to parameters")
            try:
                entries.append(_ENTRY.pack(numel, g.data_ptr(), 0 if o is None else o.data_ptr(), 0 if p is None else p.data_ptr(),
                                           0 if m is None else m.data_ptr(), 0 if v is None else v.data_ptr(), kind, pkind, scale, decay))
            except (OverflowError, struct.error):
                refuse("lr_scale, weight_decay: float32 numbers")
        self.tensors = (grads, params, exp_avg, exp_avg_sq, outs)
        return (T.tgrad_tensor * n).from_buffer_copy(b"".join(entries))

    def tgrad_group_bind(self, grads, params=None, exp_avg=None, exp_avg_sq=None, outs=None) -> None:
        """The same tensors at new addresses (gradients allocated anew); what is None stays as it is.  Every tensor is checked and every
        entry written again, 1.6 us a tensor on the host, 2.3 with parameters and moments: gradient buffers that stay where they are
        (`zero_grad(set_to_none=False)`) need none of it."""
        old = self.tensors
        new = [list(x) if x is not None else y for x, y in zip((grads, params, exp_avg, exp_avg_sq, outs), old)]
        if any(len(x) != len(old[0]) for x in new):
            refuse("tgrad_group_bind: as many tensors as at init")
        try:
            table = self._table(*new)
            call(self.device, self.lib.tgrad_group_bind, "tgrad_group_bind", self.handle, table)
        except Exception:
            self.tensors = old
            raise
        self._used(*self.tensors)

    def _used(self, *lists):
        if stream_of(self.device) != self.stream.cuda_stream:
            for tensors in lists:
                used_on(self.stream, tensors)

    def _new(self):
        """A result to be written."""
        if stream_of(self.device) == self.stream.cuda_stream:
            return torch.empty(4, dtype=torch.float32, device=self.device)[2:]
        with torch.cuda.stream(self.stream):
            return torch.empty(4, dtype=torch.float32, device=self.device)[2:]

    def _result(self, r, what):
        """Address of what lies behind an earlier result."""
        if r is None or r.dtype != torch.float32 or r.shape != (2,) or r.stride() != (1,) or r.storage_offset() != 2 or \
                r.device != self.device or r.is_neg():
            refuse("%s: an earlier result" % what)
        return r.data_ptr() - 8

    def tgrad_group_grad_norm(self, max_norm: float, add_sumsq=None, into=None):
        """-> (norm, factor): global norm of all gradients and min(1, max_norm / (norm + 1e-6)).  `add_sumsq`: a float64 tensor
        of one element, the sum of squares of gradients that lie elsewhere.  `into`: an earlier result, overwritten."""
        r = self._new() if into is None else into
        call(self.device, self.lib.tgrad_group_grad_norm, "tgrad_group_grad_norm", self.handle, max_norm, self._add(add_sumsq),
             self._result(r, "into"))
        self._used((add_sumsq, into))
        return r

    def tgrad_group_clip(self, max_norm: float, add_sumsq=None, into=None):
        """`tgrad_group_grad_norm`, and the gradients scaled by the factor; -> (norm, factor)."""
        r = self._new() if into is None else into
        call(self.device, self.lib.tgrad_group_clip, "tgrad_group_clip", self.handle, max_norm, self._add(add_sumsq),
             self._result(r, "into"))
        self._used((add_sumsq, into))
        return r

    def tgrad_group_scale(self, norm) -> None:
        """The gradients times the factor of an earlier result."""
        call(self.device, self.lib.tgrad_group_scale, "tgrad_group_scale", self.handle, self._result(norm, "norm"))
        self._used((norm,))

    def tgrad_group_adamw(self, t: int, *, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, norm=None,
                          skip_nonfinite: bool = False) -> None:
        """One AdamW step after `t` others; `norm`: a result whose factor scales the gradients as they are read."""
        hyper = T.tgrad_adamw(lr, beta1, beta2, eps, int(skip_nonfinite))
        at = self._result(norm, "norm") if norm is not None else None
        call(self.device, self.lib.tgrad_group_adamw, "tgrad_group_adamw", self.handle, C.byref(hyper), int(t), at)
        self._used((norm,))

    @staticmethod
    def sumsq(result):
        """The float64 sum of squares behind a result."""
        return torch.as_strided(result, (2,), (1,), 0).view(torch.float64)

    def _add(self, t):
        if t is None:
            return None
        if t.dtype != torch.float64 or t.numel() != 1 or t.device != self.device or t.is_neg():
            refuse("add_sumsq: one float64 on the device, no pending negation")
        return t.data_ptr()

    def tgrad_group_destroy(self) -> None:
        if self.handle:
            self.lib.tgrad_group_destroy(self.handle)
            self.handle = C.c_void_p(None)

    def __del__(self):
        try:
            self.tgrad_group_destroy()
        except Exception:
            pass
