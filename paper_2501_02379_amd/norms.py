"""The norms after and before a block, with the gate and the scale of its residual branch: ctypes binding of the tgrad_block_norm entry
points of include/tgrad.h.  Matrices, streams and memory as in `act8`.

    r = tgrad_block_norm(x, block, post_weight=wa, gate=g, rows_per_gate=n, scale=a, pre_weight=wb)
    # r.x = x + a * g * (norm(block) * wa), r.h = norm(r.x) * wb
    d = tgrad_block_norm_backward(dx, dh, r.x, block, stats=r.stats, post_weight=wa, gate=g, rows_per_gate=n, scale=a, pre_weight=wb)
"""
from __future__ import annotations

import ctypes as C
import functools
import math
from typing import NamedTuple, Optional

import torch

from . import act8
from . import tgrad as T
from .act8 import _ref
from ._marshal import REAL_TYPES, call, refuse, stream_of


class BlockNorm(NamedTuple):
    x: torch.Tensor                       # the stream behind the block (x itself where there is no block)
    h: object                             # the next block's input: a tensor, Codes, or None without a pre_weight
    stats: Optional[torch.Tensor]         # float32[rows, 4], for the backward pass


class BlockNormGrads(NamedTuple):
    dx: torch.Tensor
    dblock: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]         # the gate's size and type
    dpost: Optional[torch.Tensor]         # float32[cols]
    dpre: Optional[torch.Tensor]


def _weight(w, cols, x):
    code = REAL_TYPES.get(w.dtype)
    if code is None or w.dim() != 1 or w.shape[0] != cols or w.get_device() != x.get_device() or not w.is_contiguous() or w.is_neg():
        refuse("post_weight, pre_weight: [cols], dense, float32, bfloat16 or float16, on x's device")
    return w.data_ptr(), code


def _describe(x, rows, cols, block, dtype, post, pre, gate, rows_per_gate, scale, eps, centered):
    if block is None and (post is not None or gate is not None or pre is None):
        refuse("without a block there is a pre_weight, and neither post_weight nor gate")
    post_at, code = _weight(post, cols, x) if post is not None else (None, T.TGRAD_F32)
    pre_at, pre_code = _weight(pre, cols, x) if pre is not None else (None, code)
    if post is None:
        code = pre_code
    if code != pre_code:
        refuse("post_weight, pre_weight: of one type")
    if rows_per_gate < 1:
        refuse("rows_per_gate: at least 1")
    gate_at, gate_stride = None, 0
    if gate is not None:
        g = act8.describe(gate, "gate", x, -(-rows // rows_per_gate), cols, dtype)
        gate_at, gate_stride = g.data, g.row_stride
    if not (math.isfinite(scale) and math.isfinite(eps) and eps > 0):
        refuse("scale: finite; eps: above 0, finite")
    return T.tgrad_block(post_at, pre_at, gate_at, gate_stride, rows_per_gate, code, scale, eps, 1 if centered else 0)


@functools.lru_cache(maxsize=1024)
def _scratch_bytes(rows, cols, rows_per_gate):
    n = C.c_size_t(0)
    rc = T.load().tgrad_block_norm_query_size(rows, cols, rows_per_gate, C.byref(n))
    if rc != T.TGRAD_OK:
        raise T.TgradError(rc, "tgrad_block_norm_query_size")
    return n.value


def _types(x, dtype):
    if x.dtype not in (dtype, torch.float32):
        refuse("x: float32, or the block's type")


@act8._on_stream
def tgrad_block_norm(x, block=None, *, post_weight=None, gate=None, rows_per_gate: int = 1, scale: float = 1.0, pre_weight=None,
                     eps: float = 1e-6, centered: bool = False, quantize: bool = False, dtype=None, keep: bool = True) -> BlockNorm:
    """x + scale * gate * (norm(block) * post_weight), and norm of that * pre_weight.  Without post_weight the block goes in as it is;
    without pre_weight there is no h; without a block h is x's norm.  quantize: h as codes with a scale a row.  `dtype`: of h, where there is no
    block (x's).  keep=False: no stats.  centered: the mean is taken off first."""
    d = act8.describe(x, "x")
    dev = x.device
    b = act8.describe(block, "block", x, d.rows, d.cols) if block is not None else None
    if block is not None and dtype not in (None, block.dtype):
        refuse("dtype: the block's")
    dtype = block.dtype if block is not None else dtype or x.dtype
    if dtype not in REAL_TYPES:
        refuse("dtype: float32, bfloat16 or float16")
    _types(x, dtype)
    desc = _describe(x, d.rows, d.cols, block, dtype, post_weight, pre_weight, gate, rows_per_gate, scale, eps, centered)
    out, o = act8.new_matrix(d.rows, d.cols, x.dtype, dev) if block is not None else (x, None)
    h = e = c = None
    if pre_weight is not None and quantize:
        h, c = act8.new_codes(d.rows, d.cols, 0, dev)
    elif pre_weight is not None:
        h, e = act8.new_matrix(d.rows, d.cols, dtype, dev)
    elif quantize:
        refuse("quantize: with a pre_weight")
    stats = torch.empty((d.rows, 4), dtype=torch.float32, device=dev) if keep else None
    call(dev, T.load().tgrad_block_norm, "tgrad_block_norm", C.byref(desc), C.byref(d), _ref(b), _ref(o), _ref(e), _ref(c),
         stats.data_ptr() if keep else None, stream_of(dev))
    return BlockNorm(out, h, stats)


@act8._on_stream
def tgrad_block_norm_backward(dx, dh, x, block=None, *, stats, post_weight=None, gate=None, rows_per_gate: int = 1, scale: float = 1.0,
                              pre_weight=None, centered: bool = False) -> BlockNormGrads:
    """Gradients for `dx`, the gradient with respect to the stream behind the block from elsewhere (None: none), and `dh` with respect to h
    (None without a pre_weight).  x: the stream behind the block, as the forward call returned it; the other arguments as they were there."""
    o = act8.describe(x, "x")
    dev = x.device
    rows, cols = o.rows, o.cols
    b = act8.describe(block, "block", x, rows, cols) if block is not None else None
    if (dh is None) != (pre_weight is None):
        refuse("dh: with a pre_weight")
    dtype = block.dtype if block is not None else dh.dtype if dh is not None else x.dtype
    if dtype not in REAL_TYPES:
        refuse("dh: float32, bfloat16 or float16")
    _types(x, dtype)
    desc = _describe(x, rows, cols, block, dtype, post_weight, pre_weight, gate, rows_per_gate, scale, 1.0, centered)
    a = act8.describe(dx, "dx", x, rows, cols, x.dtype) if dx is not None else None
    u = act8.describe(dh, "dh", x, rows, cols, dtype) if dh is not None else None
    if stats is None or stats.dtype is not torch.float32 or tuple(stats.shape) != (rows, 4) or stats.device != dev or not stats.is_contiguous() or \
            stats.is_neg() or stats.data_ptr() % 16:
        refuse("stats: float32[rows, 4] of the forward call")
    gx, ex = act8.new_matrix(rows, cols, x.dtype, dev)
    gb, eb = act8.new_matrix(rows, cols, dtype, dev) if block is not None else (None, None)
    gg = torch.empty(gate.shape, dtype=dtype, device=dev) if gate is not None else None
    gpost = torch.empty(cols, dtype=torch.float32, device=dev) if post_weight is not None else None
    gpre = torch.empty(cols, dtype=torch.float32, device=dev) if pre_weight is not None else None
    ws, ws_at = act8.scratch(_scratch_bytes(rows, cols, rows_per_gate if gate is not None else 1), dev)
    at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    call(dev, T.load().tgrad_block_norm_backward, "tgrad_block_norm_backward", C.byref(desc), _ref(a), _ref(u), C.byref(o), _ref(b),
         stats.data_ptr(), C.byref(ex), _ref(eb), at(gg), at(gpost), at(gpre), ws_at, stream_of(dev))
    return BlockNormGrads(gx, gb, gg, gpost, gpre)
