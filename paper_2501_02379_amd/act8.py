"""Activations and weights in 8 bits: ctypes binding of the quantising, product and activation entry points of include/tgrad.h.

Matrices are 2-D tensors on the GPU, float32, bfloat16 or float16, with dense rows (any stride from row to row).  A call enqueues
its kernels on the device's current stream, or on `stream=`, and waits for nothing; outputs and scratch come from torch's
allocator on that stream, and with `stream=` the arguments are recorded on it, so that they may be let go of at once.

A linear layer trained in 8 bits, with its activation:

    h = tgrad_codes_linear(x, w, keep=True)                    # h.y, and h.x8: what the backward pass needs of x
    a = tgrad_activation(h.y, act="silu", quantize=True)      # a.y: codes for the next product; a.x8: the checkpoint of h.y
    ...
    dh, _ = tgrad_activation_backward(da, a.x8, act="silu")
    dx, dw = tgrad_codes_grad_input(dh, w), tgrad_codes_grad_weight(dh, h.x8)
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import NamedTuple, Optional

import torch

from . import tgrad as T
from ._marshal import REAL_TYPES, call, on_stream_with, refuse, stream_of

ACTS = {"silu": T.TGRAD_ACT_SILU, "gelu": T.TGRAD_ACT_GELU}


class Codes(NamedTuple):
    """rows x cols numbers in 8 bits: codes * scale, a scale for `group` columns (0: for the whole row)."""
    codes: torch.Tensor                   # int8[rows, cols], dense rows
    scale: torch.Tensor                   # float32[rows, ceil(cols / group)], dense
    group: int = 0


class Linear(NamedTuple):
    y: torch.Tensor
    x8: Optional[Codes]


class Activation(NamedTuple):
    y: object                             # a tensor, or Codes where it was asked to quantize
    x8: Optional[Codes]
    gate8: Optional[Codes]


def describe(x, what, like=None, rows=None, cols=None, dtype=None):
    """A matrix as the library takes it; anything it does not take is refused."""
    if not isinstance(x, torch.Tensor):
        refuse(what + ": a 2-D float32, bfloat16 or float16 tensor on the GPU")
    shape, t = x.shape, x.dtype
    code = REAL_TYPES.get(t)
    if len(shape) != 2 or code is None or not x.is_cuda:
        refuse(what + ": a 2-D float32, bfloat16 or float16 tensor on the GPU")
    n, m = shape
    stride, step = x.stride()
    if (step != 1 and m > 1 and n > 0) or x.is_neg():                      # memory holds other numbers than a tensor with that pending
        refuse(what + ": dense rows, no pending negation")
    if like is not None and x.get_device() != like.get_device():
        refuse(what + ": on the other tensors' device")
    if (rows is not None and n != rows) or (cols is not None and m != cols) or (dtype is not None and t is not dtype):
        refuse("%s: %s x %s%s" % (what, "rows" if rows is None else rows, "cols" if cols is None else cols, "" if dtype is None else " of %s" % dtype))
    return T.tgrad_matrix(x.data_ptr(), n, m, stride if n > 1 else m, code)


def describe_codes(c, what, like=None, rows=None, cols=None):
    if not isinstance(c, Codes) or not isinstance(c.codes, torch.Tensor) or not isinstance(c.scale, torch.Tensor):
        refuse(what + ": Codes")
    q, s, g = c
    shape = q.shape
    if len(shape) != 2 or q.dtype is not torch.int8 or not q.is_cuda:
        refuse(what + ": int8 codes on the GPU, 2-D, dense rows")
    n, m = shape
    stride, step = q.stride()
    device = q.get_device()
    if step != 1 and m > 1 and n > 0:
        refuse(what + ": int8 codes on the GPU, 2-D, dense rows")
    if s.dtype is not torch.float32 or s.get_device() != device or not s.is_contiguous() or s.is_neg() or \
            s.numel() != n * (1 if not g else -(-m // g) if g > 0 else -1):
        refuse(what + ": float32 scales, dense, one for each group of columns of each row, on the codes' device, no pending negation")
    if like is not None and device != like.get_device():
        refuse(what + ": on the other tensors' device")
    if (rows is not None and n != rows) or (cols is not None and m != cols):
        refuse("%s: %s x %s" % (what, "rows" if rows is None else rows, "cols" if cols is None else cols))
    return T.tgrad_codes(q.data_ptr(), s.data_ptr(), n, m, stride if n > 1 else m, g)


def new_codes(rows, cols, group, device):
    """Memory for codes, rows at multiples of 16 bytes, and its description."""
    pitch = -(-cols // 16) * 16
    codes = torch.empty((rows, pitch), dtype=torch.int8, device=device)
    scale = torch.empty((rows, -(-cols // group) if group else 1), dtype=torch.float32, device=device)
    return Codes(codes[:, :cols] if pitch != cols else codes, scale, group), \
        T.tgrad_codes(codes.data_ptr(), scale.data_ptr(), rows, cols, pitch, group)


def new_matrix(rows, cols, dtype, device):
    """A new tensor and its description."""
    x = torch.empty((rows, cols), dtype=dtype, device=device)
    return x, T.tgrad_matrix(x.data_ptr(), rows, cols, cols, REAL_TYPES[dtype])


def _result(out, what, like, rows, cols, dtype):
    """`out`, checked, or a new tensor, and its description."""
    if out is None:
        return new_matrix(rows, cols, dtype, like.device)
    return out, describe(out, what, like, rows, cols, dtype)


@functools.lru_cache(maxsize=4096)
def _scratch_bytes(op, tokens, inner, outer):
    n = C.c_size_t(0)
    rc = T.load().tgrad_codes_query_size(op, tokens, inner, outer, C.byref(n))
    if rc != T.TGRAD_OK:
        raise T.TgradError(rc, "tgrad_codes_query_size")
    return n.value


def scratch(n, device):
    """n bytes and their address; no memory where n is 0."""
    if n == 0:
        return None, None
    t = torch.empty(n, dtype=torch.uint8, device=device)
    return t, t.data_ptr()


def _ref(d):
    return None if d is None else C.byref(d)


def _group(group):
    if group not in (0, 32, 64, 128, 256, 512):
        refuse("group: 0 (the whole row), 32, 64, 128, 256 or 512 columns")
    return group


def _act(act):
    if act not in ACTS:
        refuse("act: one of " + ", ".join(ACTS))
    return ACTS[act]


_on_stream = on_stream_with(lambda a: [t for t in a if isinstance(t, torch.Tensor)] if isinstance(a, Codes) else ())


@_on_stream
def tgrad_quantize(x, *, group: int = 0, out: Optional[Codes] = None) -> Codes:
    """x in 8 bits, a scale for `group` columns (0: the whole row).  `out`: where the codes go."""
    d = describe(x, "x")
    dev = x.device
    if out is None:
        out, c = new_codes(d.rows, d.cols, _group(group), dev)
    else:
        c = describe_codes(out, "out", x, d.rows, d.cols)
        if c.group != group:
            refuse("out: codes in groups of `group` columns")
    call(dev, T.load().tgrad_quantize, "tgrad_quantize", C.byref(d), C.byref(c), stream_of(dev))
    return out


@_on_stream
def tgrad_dequantize(codes: Codes, dtype=torch.float32, *, out=None):
    """The values that codes stand for, rounded once to `dtype`."""
    c = describe_codes(codes, "codes")
    if dtype not in REAL_TYPES:
        refuse("dtype: float32, bfloat16 or float16")
    out, d = _result(out, "out", codes.codes, c.rows, c.cols, dtype)
    call(out.device, T.load().tgrad_dequantize, "tgrad_dequantize", C.byref(c), C.byref(d), stream_of(out.device))
    return out


@_on_stream
def tgrad_codes_matmul(x: Codes, weight: Codes, *, dtype=torch.bfloat16, out=None):
    """x (tokens x inner) times weight (outer x inner) transposed, both codes with a scale a row: tokens x outer in `dtype`."""
    c = describe_codes(x, "x")
    w = describe_codes(weight, "weight", x.codes, cols=c.cols)
    if dtype not in REAL_TYPES:
        refuse("dtype: float32, bfloat16 or float16")
    dev = x.codes.device
    y, d = _result(out, "out", x.codes, c.rows, w.rows, dtype)
    ws, at = scratch(_scratch_bytes(T.TGRAD_CODES_MATMUL, c.rows, c.cols, w.rows), dev)
    call(dev, T.load().tgrad_codes_matmul, "tgrad_codes_matmul", C.byref(c), C.byref(w), C.byref(d), at, stream_of(dev))
    return y


@_on_stream
def tgrad_codes_linear(x, weight: Codes, *, keep: bool = False, dtype=None, out=None) -> Linear:
    """x in 8 bits, a scale for each token, times weight transposed.  keep: x's codes come back too, for the backward pass.  `dtype`: of
    the result (x's)."""
    d = describe(x, "x")
    w = describe_codes(weight, "weight", x, cols=d.cols)
    dev = x.device
    dtype = dtype or x.dtype
    if dtype not in REAL_TYPES:
        refuse("dtype: float32, bfloat16 or float16")
    y, e = _result(out, "out", x, d.rows, w.rows, dtype)
    x8, c = new_codes(d.rows, d.cols, 0, dev) if keep else (None, None)
    ws, at = scratch(_scratch_bytes(T.TGRAD_CODES_MATMUL if keep else T.TGRAD_CODES_LINEAR, d.rows, d.cols, w.rows), dev)
    call(dev, T.load().tgrad_codes_linear, "tgrad_codes_linear", C.byref(d), C.byref(w), _ref(c), C.byref(e), at, stream_of(dev))
    return Linear(y, x8)


@_on_stream
def tgrad_codes_grad_input(dy, weight: Codes, *, dtype=None, out=None, unrounded: bool = False):
    """Gradient of a product with respect to its input: dy (tokens x outer) times the values of weight (outer x inner).  `dtype`: of the
    result, dy's or float32.  unrounded: values of codes are not rounded to a two-byte dy's type first, which takes twice as long and leaves the
    result's own rounding as its error."""
    return _gradient(T.TGRAD_CODES_GRAD_INPUT, dy, weight, dtype, out, unrounded)


@_on_stream
def tgrad_codes_grad_weight(dy, x: Codes, *, dtype=None, out=None, unrounded: bool = False):
    """Gradient of a product with respect to its weight: dy (tokens x outer) transposed, times the values of x (tokens x inner).  `dtype`, `unrounded`:
    as above."""
    return _gradient(T.TGRAD_CODES_GRAD_WEIGHT, dy, x, dtype, out, unrounded)


def _gradient(op, dy, codes, dtype, out, unrounded):
    d = describe(dy, "dy")
    dev = dy.device
    dtype = dtype or dy.dtype
    if dtype not in (dy.dtype, torch.float32):
        refuse("dtype: dy's or float32")
    if op == T.TGRAD_CODES_GRAD_INPUT:
        c = describe_codes(codes, "weight", dy, rows=d.cols)
        tokens, outer, rows = d.rows, c.rows, d.rows
    else:
        c = describe_codes(codes, "x", dy, rows=d.rows)
        tokens, outer, rows = d.rows, d.cols, d.cols
    out, e = _result(out, "out", dy, rows, c.cols, dtype)
    if dy.dtype is not torch.float32 and not (unrounded and dtype is torch.float32) and not (d.rows <= 16 and (not c.group or c.cols <= c.group)) and \
            ((d.data or 0) % 16 or d.row_stride % 8 or d.cols % 8 or d.row_stride > 1 << 21):
        op += T.TGRAD_CODES_UNALIGNED                      # where the library copies dy
    if unrounded:
        op += T.TGRAD_CODES_UNROUNDED
    ws, at = scratch(_scratch_bytes(op, tokens, c.cols, outer), dev)
    call(dev, T.load().tgrad_codes_gradient, "tgrad_codes_gradient", op, C.byref(d), C.byref(c), C.byref(e), at, stream_of(dev))
    return out


@_on_stream
def tgrad_activation(x, gate=None, *, act: str = "silu", group: int = 128, keep: bool = True, quantize: bool = False,
                     out=None) -> Activation:
    """act(x), or act(x) * gate, with the checkpoint of x and gate in 8 bits (`keep`), in groups of `group` columns.  quantize: the
    result as codes with a scale a row, for the next product.  act: "silu" or "gelu" (with erf)."""
    d = describe(x, "x")
    dev, code = x.device, _act(act)
    g = describe(gate, "gate", x, d.rows, d.cols, x.dtype) if gate is not None else None
    if keep and not _group(group):
        refuse("group: 32, 64, 128, 256 or 512 columns")
    if quantize and out is None:
        y, e = new_codes(d.rows, d.cols, 0, dev)
    elif quantize:
        y, e = out, describe_codes(out, "out", x, d.rows, d.cols)
    else:
        y, e = _result(out, "out", x, d.rows, d.cols, x.dtype)
    x8, cx = new_codes(d.rows, d.cols, group, dev) if keep else (None, None)
    gate8, cg = new_codes(d.rows, d.cols, group, dev) if keep and g is not None else (None, None)
    call(dev, T.load().tgrad_activation, "tgrad_activation", C.byref(d), _ref(g), code, None if quantize else C.byref(e),
         C.byref(e) if quantize else None, _ref(cx), _ref(cg), stream_of(dev))
    return Activation(y, x8, gate8)


@_on_stream
def tgrad_activation_backward(dy, x8: Codes, gate8: Optional[Codes] = None, *, act: str = "silu", out=None, gate_out=None):
    """-> (dx, dgate) from the checkpoint; dgate is None where there was no gate."""
    d = describe(dy, "dy")
    dev, code = dy.device, _act(act)
    c = describe_codes(x8, "x8", dy, d.rows, d.cols)
    dx, e = _result(out, "out", dy, d.rows, d.cols, dy.dtype)
    if gate8 is None:
        if gate_out is not None:
            refuse("gate_out: only with gate8")
        call(dev, T.load().tgrad_activation_backward, "tgrad_activation_backward", C.byref(d), C.byref(c), None, code, C.byref(e), None,
             stream_of(dev))
        return dx, None
    b = describe_codes(gate8, "gate8", dy, d.rows, d.cols)
    dgate, f = _result(gate_out, "gate_out", dy, d.rows, d.cols, dy.dtype)
    call(dev, T.load().tgrad_activation_backward, "tgrad_activation_backward", C.byref(d), C.byref(c), C.byref(b), code, C.byref(e),
         C.byref(f), stream_of(dev))
    return dx, dgate
