"""Gradients of products with codes through the wide tiles and over long sums: the kernel that is meant to run does, and its results are the only right ones.

dy in -2..2 and codes in -3..3 with scale 1: products are whole numbers, partial sums of them far below 2^24 (some 600 is their spread at 40003 terms), so that
float32 sums are exact in any order.  Unrounded values lie in two parts, multiples of 2^-8 in bf16 and 2^-11 in float16 (a code of 1 is 1 - 2^-11 and 2^-11), and sums
below 2^13 of those are exact too.  The result's rounding to its type is the only one, and has one answer.
"""
import re

import pytest
import torch

from paper_2501_02379_amd import act8
from test_gpu_act8 import DEV, TYPES, U, laid, numbers, random_codes, rounded

pytestmark = pytest.mark.gpu

CODE = {"f32": 2, "bf16": 3, "f16": 4}


def launched(call):
    """(result, names of the kernels that the call launched)."""
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA], acc_events=True) as p:
        result = call()
        torch.cuda.synchronize()
    return result, [m.group(0) for e in p.events() for m in [re.search(r"k_\w+(<[^>]*>)?", e.name)] if m]


def whole(rows, cols, low, high, seed):
    return torch.randint(low, high + 1, (rows, cols), generator=torch.Generator().manual_seed(seed), dtype=torch.int8)


# which gradient, tokens, inner, outer; kernel: wide, in splits, inner no multiple of 16
WIDE = [("weight", 300, 3700, 3592, False, True),           # 10 steps of 32, the last one short
        ("weight", 333, 3712, 3600, False, False),          # an odd number
        ("weight", 17, 3712, 3600, False, False), ("weight", 33, 3700, 3600, False, True),
        ("weight", 40003, 512, 768, True, False),           # 38 splits of 33 steps, the last of 30, which ends with three rows
        ("weight", 40003, 500, 760, True, True),
        ("weight", 34848, 512, 768, True, False),           # 33 splits of 33 steps
        ("input", 3700, 3588, 1000, False, True), ("input", 3584, 3584, 1056, False, False), ("input", 3700, 3584, 8, False, False),
        ("input", 2040, 2030, 4104, True, True), ("input", 2048, 2048, 8192, True, False)]


@pytest.mark.parametrize("unrounded", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("which,tokens,inner,outer,split,ragged", WIDE)
def test_wide_tiles_are_exact(which, tokens, inner, outer, split, ragged, dtype, unrounded):
    t = TYPES[dtype][0]
    dy = whole(tokens, outer, -2, 2, 1)
    c = whole(tokens if which == "weight" else outer, inner, -3, 3, 2)
    codes = laid(c, torch.ones(len(c), 1), pad=-inner % 16)
    call = act8.tgrad_codes_grad_weight if which == "weight" else act8.tgrad_codes_grad_input
    given = dy.to(t).to(DEV)
    got, names = launched(lambda: call(given, codes, unrounded=unrounded))
    expected = "k_grad_wide<%d, %d, %s, %s, %d>" % (CODE[dtype], -1 if split else CODE[dtype], str(which == "weight").lower(), str(ragged).lower(), 1 + unrounded)
    assert expected in names and ("k_add_splits<%d>" % CODE[dtype] in names) == split, names
    a = dy.float().t().contiguous() if which == "weight" else dy.float()
    assert torch.equal(got.cpu(), (a @ c.float()).to(t))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("tokens,inner,outer", [(70000, 264, 250), (20001, 33, 48), (300, 264, 2500)])
def test_long_sums_are_exact_in_other_tiles(tokens, inner, outer, dtype):
    t = TYPES[dtype][0]
    dy, cw, cx = whole(tokens, outer, -2, 2, 1), whole(outer, inner, -3, 3, 2), whole(tokens, inner, -3, 3, 3)
    w, x = (laid(c, torch.ones(len(c), 1), pad=-inner % 16) for c in (cw, cx))
    given = dy.to(t).to(DEV)
    for unrounded in (False, True):
        assert torch.equal(act8.tgrad_codes_grad_input(given, w, unrounded=unrounded).cpu(), (dy.float() @ cw.float()).to(t))
        got, names = launched(lambda: act8.tgrad_codes_grad_weight(given, x, unrounded=unrounded))
        assert torch.equal(got.cpu(), (dy.float().t().contiguous() @ cx.float()).to(t))
        kernel = "k_grad_split" if dtype == "f32" else "k_grad_tiles"
        assert any(n.startswith(kernel) for n in names), names


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("tokens,inner,outer", [(70000, 264, 250), (20000, 33, 48), (40003, 500, 768), (300, 3700, 3592)])
def test_long_sums_of_random_numbers(tokens, inner, outer, dtype):
    """In the 2-norm.  Signs are random: what float32 sums of S terms are off by, in any order, is at most 2 sqrt(S) u of the result; the result's rounding is
    known (its own part of the difference), and nothing else is rounded: values are the rounded ones."""
    t = TYPES[dtype][0]
    dy = numbers(tokens, outer, dtype, seed=1)
    x, cx, sx = random_codes(tokens, inner, seed=2, pad=-inner % 16)
    want = dy.cpu().double().t().contiguous() @ rounded(cx, sx, 0, dtype, tokens)
    off = float((act8.tgrad_codes_grad_weight(dy, x).cpu().double() - want).norm())
    assert off <= 1.02 * float((want.to(t).double() - want).norm()) + (2 * tokens ** 0.5 + 4) * U * float(want.norm())
