"""Losses on logits and their gradients: ctypes binding of the loss entry points of include/tgrad.h.

Logits are 2-D tensors on the GPU, float32, bfloat16 or float16, with dense rows (any stride from row to row).  A call enqueues
its kernels on the device's current stream, or on `stream=`, and waits for nothing; outputs and scratch come from torch's
allocator on that stream, and with `stream=` the arguments are recorded on it, so that they may be let go of at once.  The
gradient with respect to the logits goes on through autograd as `logits.backward(result.dlogits)`.

The small results of a loss lie in one allocation with its scratch (16 bytes a row, 28 for a preference loss): clone what is to be
kept for long.
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import NamedTuple, Optional

import torch

from . import tgrad as T
from ._marshal import REAL_TYPES, call, on_stream, refuse, scalar, stream_of, vector


class PolicyLoss(NamedTuple):
    stats: torch.Tensor                   # float32[4]: sums of w (pg + kl_beta kl), w pg, w kl, w [clipped]
    logp: torch.Tensor                    # float32[rows]
    dlogits: Optional[torch.Tensor]

    @property
    def loss(self):
        return self.stats[0]


class PreferenceLoss(NamedTuple):
    loss: torch.Tensor                    # float32, 0-d
    rewards: torch.Tensor                 # float32[2 pairs]: the chosen answers', then the rejected ones'
    logp: torch.Tensor                    # float32[rows]
    dlogits: Optional[torch.Tensor]


def _describe(logits, targets, temperature):
    if logits.dim() != 2 or logits.dtype not in REAL_TYPES or not logits.is_cuda:
        refuse("logits: a 2-D float32, bfloat16 or float16 tensor on the GPU")
    rows, vocab = logits.shape
    stride = logits.stride(0) if rows > 1 else vocab
    if (vocab > 1 and logits.stride(1) != 1) or logits.is_neg():       # memory holds other numbers than a tensor with that pending
        refuse("logits: dense rows, no pending negation")
    y = vector(targets, rows, torch.int64, logits.device, "targets")
    return T.tgrad_logits(logits.data_ptr(), rows, vocab, stride, y, REAL_TYPES[logits.dtype], temperature)


def _gradient(logits, out):
    """Where the gradient goes, and its row stride: `out` (logits itself is allowed) or a new tensor."""
    if out is None:
        out = torch.empty_like(logits, memory_format=torch.contiguous_format)
    elif out.shape != logits.shape or out.dtype != logits.dtype or out.device != logits.device or \
            (out.shape[1] > 1 and out.stride(1) != 1) or out.is_neg():
        refuse("out: the logits' shape, type and device, with dense rows, no pending negation")
    return out, (out.stride(0) if out.shape[0] > 1 else out.shape[1])


@functools.lru_cache(maxsize=1024)
def _scratch_floats(rows, pairs):
    n = C.c_size_t(0)
    rc = T.load().tgrad_loss_query_size(rows, pairs, C.byref(n))
    if rc != T.TGRAD_OK:
        raise T.TgradError(rc, "tgrad_loss_query_size")
    return n.value // 4


def _floats(logits, pairs, *sizes):
    """The scratch of a loss and its float32 outputs, one allocation for all of them."""
    scratch = _scratch_floats(logits.shape[0], pairs)
    return torch.empty(scratch + sum(sizes), dtype=torch.float32, device=logits.device).split_with_sizes((scratch,) + sizes)


@on_stream
def tgrad_token_logprobs(logits, targets, *, temperature: float = 1.0):
    """-> (logp, lse), float32[rows]: log-probability of targets[n] in row n and log sum exp of the row, of logits / temperature.
    Rows whose target lies outside the vocabulary (-100, say) have 0 in both and are not read."""
    d = _describe(logits, targets, temperature)
    out = torch.empty(2, d.rows, dtype=torch.float32, device=logits.device)
    logp, lse = out.unbind(0)
    call(logits.device, T.load().tgrad_token_logprobs, "tgrad_token_logprobs", C.byref(d), logp.data_ptr(), lse.data_ptr(),
         stream_of(logits.device))
    return logp, lse


@on_stream
def tgrad_token_logprobs_backward(logits, targets, lse, dlogp, *, temperature: float = 1.0, out=None):
    """-> gradient with respect to the logits, in their type, for the gradient `dlogp` of every log-probability."""
    d = _describe(logits, targets, temperature)
    dx, stride = _gradient(logits, out)
    call(logits.device, T.load().tgrad_token_logprobs_backward, "tgrad_token_logprobs_backward", C.byref(d),
         vector(lse, d.rows, torch.float32, logits.device, "lse"), vector(dlogp, d.rows, torch.float32, logits.device, "dlogp"),
         dx.data_ptr(), stride, stream_of(logits.device))
    return dx


@on_stream
def tgrad_policy_loss(logits, targets, weight, advantage, old_logp, ref_logp=None, *, clip_low: float = 0.2,
                      clip_high: float = 0.2, kl_beta: float = 0.0, temperature: float = 1.0, dloss=None, backward: bool = True,
                      out=None) -> PolicyLoss:
    """Clipped policy loss sum_n w_n (pg_n + kl_beta kl_n) with its gradient; `weight` holds mask and normalisation.  `dloss`: a
    float32 tensor of one element on the device that scales the gradient.  `backward=False`: no gradient.  `out`: where the
    gradient goes (may be `logits`)."""
    d = _describe(logits, targets, temperature)
    dev, rows = logits.device, d.rows
    dx, stride = _gradient(logits, out) if backward else (None, 0)
    ws, stats, logp = _floats(logits, 0, 4, rows)
    hyper = T.tgrad_policy(clip_low, clip_high, kl_beta)
    call(dev, T.load().tgrad_policy_loss, "tgrad_policy_loss", C.byref(d), C.byref(hyper),
         vector(weight, rows, torch.float32, dev, "weight"), vector(advantage, rows, torch.float32, dev, "advantage"),
         vector(old_logp, rows, torch.float32, dev, "old_logp"), vector(ref_logp, rows, torch.float32, dev, "ref_logp"),
         scalar(dloss, torch.float32, dev, "dloss"), ws.data_ptr(), stats.data_ptr(), logp.data_ptr(),
         dx.data_ptr() if backward else None, stride, stream_of(dev))
    return PolicyLoss(stats, logp, dx)


@on_stream
def tgrad_preference_loss(logits, targets, weight, ref_logp, seq_start, *, beta: float = 0.1, label_smoothing: float = 0.0,
                          dloss=None, backward: bool = True, out=None, temperature: float = 1.0) -> PreferenceLoss:
    """Preference loss on paired log ratios with its gradient.  Rows seq_start[i] .. seq_start[i + 1] - 1 are sequence i
    (int64[2 pairs + 1], on the device); the first half of the sequences is chosen, the second half rejected."""
    d = _describe(logits, targets, temperature)
    dev, rows = logits.device, d.rows
    if seq_start.dim() != 1 or seq_start.shape[0] < 3 or seq_start.shape[0] % 2 == 0:
        refuse("seq_start: int64[2 pairs + 1]")
    pairs = seq_start.shape[0] // 2
    dx, stride = _gradient(logits, out) if backward else (None, 0)
    ws, loss, rewards, logp = _floats(logits, pairs, 1, 2 * pairs, rows)
    hyper = T.tgrad_preference(beta, label_smoothing)
    call(dev, T.load().tgrad_preference_loss, "tgrad_preference_loss", C.byref(d), C.byref(hyper), pairs,
         vector(seq_start, 2 * pairs + 1, torch.int64, dev, "seq_start"), vector(weight, rows, torch.float32, dev, "weight"),
         vector(ref_logp, rows, torch.float32, dev, "ref_logp"), scalar(dloss, torch.float32, dev, "dloss"), ws.data_ptr(),
         loss.data_ptr(), rewards.data_ptr(), logp.data_ptr(), dx.data_ptr() if backward else None, stride,
         stream_of(dev))
    return PreferenceLoss(loss[0], rewards, logp, dx)
