"""Gradients of products with codes where test_gpu_act8.py has no case: values beyond a type's range, long sums in wide tiles, unrounded values.

u = 2^-24.  Sums of S products of two-byte numbers are off by at most 2 u S sum |a b|, as there.
"""
import ctypes as C

import pytest
import torch

from paper_2501_02379_amd import act8, tgrad as T
from test_gpu_act8 import DEV, TYPES, U, laid, numbers

pytestmark = pytest.mark.gpu


def codes_with(rows, cols, scale, seed=0, group=0, pad=None):
    """Random codes of the given scale (a number, or a tensor of all of them)."""
    g = torch.Generator().manual_seed(seed)
    c = torch.randint(-127, 128, (rows, cols), generator=g, dtype=torch.int8)
    s = torch.as_tensor(scale, dtype=torch.float32).expand(rows, -(-cols // group) if group else 1).contiguous()
    return laid(c, s, group, -cols % 16 if pad is None else pad), c, s


def spread_out(codes, scale, group):
    """Values of codes in float64."""
    g = group or codes.shape[1]
    return codes.double() * scale.double().repeat_interleave(g, 1)[:, :codes.shape[1]]


# tokens, inner, outer: dy times a scale, tiles of 128, wide tiles (the last two, for dx and for dw)
RANGE = [(8, 130, 70), (17, 130, 70), (300, 200, 130), (3700, 3588, 40), (40, 3700, 3592)]


@pytest.mark.parametrize("tokens,inner,outer", RANGE)
@pytest.mark.parametrize("scale", [1000.0, 2.0 ** -26, 2.0 ** -60])
@pytest.mark.parametrize("group", [0, 64])
def test_float16_gradients_of_values_beyond_float16(tokens, inner, outer, scale, group):
    """Codes stand for float32 numbers whatever dy's type is: neither an infinity nor a lost value comes of it, however many tokens there are.  Values are
    rounded to 11 bits, half a step is 2^-11 of each; the result is float32, for results of such values would leave float16 themselves."""
    dy = numbers(tokens, outer, "f16", seed=1, pad=outer % 4)
    w, cw, sw = codes_with(outer, inner, scale, 2, group)
    x, cx, sx = codes_with(tokens, inner, scale, 3, group)
    for got, a, b, terms in ((act8.tgrad_codes_grad_input(dy, w, dtype=torch.float32), dy.cpu().double(), spread_out(cw, sw, group), outer),
                             (act8.tgrad_codes_grad_weight(dy, x, dtype=torch.float32), dy.cpu().double().t().contiguous(), spread_out(cx, sx, group), tokens)):
        bound = (a.abs() @ b.abs()) * (2.0 ** -11 + (6 * terms + 4) * U)
        assert bool(((got.cpu().double() - a @ b).abs() <= bound).all())


@pytest.mark.parametrize("tokens,inner,outer", RANGE)
def test_float16_gradients_of_rows_of_different_sizes(tokens, inner, outer):
    """Rows' scales from 2^-10 to 1000, 20 binary orders; results that fit float16."""
    g = torch.Generator().manual_seed(4)
    rows = lambda n: 2.0 ** (torch.rand(n, 1, generator=g) * 20 - 10)  # noqa: E731
    dy = numbers(tokens, outer, "f16", seed=1, spread=2.0 ** -12)
    w, cw, sw = codes_with(outer, inner, rows(outer), 2)
    x, cx, sx = codes_with(tokens, inner, rows(tokens), 3)
    for got, a, b, terms in ((act8.tgrad_codes_grad_input(dy, w), dy.cpu().double(), spread_out(cw, sw, 0), outer),
                             (act8.tgrad_codes_grad_weight(dy, x), dy.cpu().double().t().contiguous(), spread_out(cx, sx, 0), tokens)):
        want = a @ b
        assert float(want.abs().max()) < 60000
        bound = (a.abs() @ b.abs()) * (2.0 ** -11 + (6 * terms + 4) * U) * (1 + 2.0 ** -11) + want.abs() * 2.0 ** -11 + 2.0 ** -24
        assert bool(((got.cpu().double() - want).abs() <= bound).all())


def test_a_gated_result_beyond_float16():
    """300 * 300 from finite float16 numbers is a good code, and finite in the product's gradient."""
    h = torch.full((40, 64), 300.0, dtype=torch.float16, device=DEV)
    a = act8.tgrad_activation(h, h, quantize=True, keep=False)
    dy = numbers(40, 24, "f16", seed=3, spread=1e-3)
    dy[:, 5] = 0
    dw = act8.tgrad_codes_grad_weight(dy, a.y)
    want = dy.cpu().double().t().contiguous() @ (a.y.codes.cpu().double() * a.y.scale.cpu().double())
    assert bool(dw[5].eq(0).all()) and bool(((dw.cpu().double() - want).abs() <= want.abs() * 2.0 ** -11 + 40 * 90000 * 5e-3 * (2.0 ** -11 + 250 * U)).all())


# ---- unrounded values -----------------------------------------------------------------------------------------------------------

# what the two parts of a value leave of it
PARTS = {"bf16": 2.0 ** -8 * (2.0 ** -7 + 2.0 ** -9), "f16": 2.0 ** -11 * (2.0 ** -10 + 2.0 ** -12)}
# tokens, inner, outer: single tokens, around 16, sums that end within a step, wide tiles (dx, dw), wide tiles with the sum in splits (dw, dx)
UNROUNDED = [(1, 40, 30), (5, 64, 33), (17, 100, 70), (64, 128, 256), (100, 513, 66), (257, 255, 129), (5000, 64, 32), (3700, 3588, 40), (300, 3700, 3592), (40003, 500, 768), (2040, 2030, 4100)]


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("tokens,inner,outer", UNROUNDED)
def test_unrounded_gradients(tokens, inner, outer, dtype, out):
    """A value is off by PARTS of itself, or with a float32 result by u; sums and the result's rounding come on top."""
    t, u, tiny = TYPES[out]
    dy = numbers(tokens, outer, dtype, seed=1, pad=outer % 4, offset=outer % 3)
    for group, pad in ((0, None), (0, 3), (32, None)) if tokens < 20000 else ((0, None),):
        scales = lambda n: torch.rand(n, -(-inner // group) if group else 1, generator=torch.Generator().manual_seed(9)) * 0.02 + 0.001  # noqa: E731
        w, cw, sw = codes_with(outer, inner, scales(outer), 2, group, pad)
        x, cx, sx = codes_with(tokens, inner, scales(tokens), 3, group, pad)
        for call, c, a, b, terms in ((act8.tgrad_codes_grad_input, w, dy.cpu().double(), spread_out(cw, sw, group), outer),
                                     (act8.tgrad_codes_grad_weight, x, dy.cpu().double().t().contiguous(), spread_out(cx, sx, group), tokens)):
            got = call(dy, c, dtype=t, unrounded=True)
            want, size = a @ b, a.abs() @ b.abs()
            value = PARTS[dtype] if out == dtype != "f32" else U
            off = (got.cpu().double() - want).abs()
            assert got.dtype is t and bool((off <= size * (value + (6 * terms + 4) * U) * (1 + u) + want.abs() * u + tiny).all())
            if want.numel() > 2000:
                # That bound is wide where sums are long.  Terms of random signs: what their values are off by is PARTS of the result in the 2-norm, 1/40 of
                # the result's own rounding (some 0.4 u of it), and what float32 sums are off by, in any order, grows as the root of the terms.
                own = float((want.to(t).double() - want).norm())
                assert float(off.norm()) <= 1.02 * own + (2 * terms ** 0.5 + 4) * U * float(want.norm())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tokens,inner,outer", [(17, 130, 70), (300, 200, 130), (3700, 3588, 40)])
def test_an_infinity_in_a_gradient_stays_one(tokens, inner, outer, dtype):
    """Infinite where the other factor is a number but 0, with its sign; NaN where that is 0."""
    dy = numbers(tokens, outer, dtype, seed=2)
    t, n = tokens - 2, outer // 2
    dy[t, n] = float("-inf")
    w, cw, _ = codes_with(outer, inner, 0.01, 4)
    x, cx, _ = codes_with(tokens, inner, 0.01, 5)
    for unrounded in (False, True):
        dx, dw = (f(dy, c, unrounded=unrounded).cpu() for f, c in ((act8.tgrad_codes_grad_input, w), (act8.tgrad_codes_grad_weight, x)))
        for row, codes in ((dx[t], cw[n]), (dw[n], cx[t])):
            assert torch.equal(row.isnan(), codes == 0) and torch.equal(row == float("-inf"), codes > 0) and torch.equal(row == float("inf"), codes < 0)


def test_unrounded_gradients_captured_and_on_another_stream():
    dy, w, x = numbers(700, 300, "bf16", seed=1), codes_with(300, 200, 0.01, 2)[0], codes_with(700, 200, 0.01, 3)[0]
    both = lambda **kw: (act8.tgrad_codes_grad_input(dy, w, unrounded=True, **kw), act8.tgrad_codes_grad_weight(dy, x, unrounded=True, **kw))  # noqa: E731
    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = both(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(3):
        dy.mul_(1.5)
        graph.replay()
        want = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype,out,tokens", [("f32", "f32", 5), ("f32", "f32", 300), ("bf16", "bf16", 5), ("f16", "f16", 16), ("bf16", "f32", 300), ("f16", "f32", 300)])
@pytest.mark.parametrize("value", [float("inf"), float("-inf")])
@pytest.mark.parametrize("inner,outer", [(130, 70), (200, 131)])
def test_an_infinity_stays_one_where_dy_is_split(tokens, inner, outer, dtype, out, value):
    dy = numbers(tokens, outer, dtype, seed=2)
    t, n = tokens - 2, outer // 2
    dy[t, n] = value
    w, cw, _ = codes_with(outer, inner, 0.01, 4)
    x, cx, _ = codes_with(tokens, inner, 0.01, 5)
    dx, dw = (f(dy, c, unrounded=True, dtype=TYPES[out][0]).cpu() for f, c in ((act8.tgrad_codes_grad_input, w), (act8.tgrad_codes_grad_weight, x)))
    for row, codes in ((dx[t], cw[n]), (dw[n], cx[t])):
        assert torch.equal(row.isnan(), codes == 0) and torch.equal(row == value, codes > 0) and torch.equal(row == -value, codes < 0)
    nan = torch.tensor([0x7F800001], dtype=torch.int32, device=DEV).view(torch.float32)              # a NaN whose upper half is infinity's
    if dtype == "f32":
        dy[t, n] = nan
        assert bool(act8.tgrad_codes_grad_input(dy, w)[t].isnan().all()) and bool(act8.tgrad_codes_grad_weight(dy, x)[n].isnan().all())


@pytest.mark.parametrize("tokens,dtype,out,unrounded,group,copied", [
    (300, "f32", "f32", False, 0, False), (300, "f32", "f32", False, 32, False), (16, "bf16", "bf16", False, 0, False), (16, "bf16", "bf16", False, 32, True),
    (17, "bf16", "bf16", False, 0, True), (300, "f16", "f16", True, 0, True), (300, "f16", "f32", False, 0, True), (300, "f16", "f32", True, 0, False),
    (300, "f16", "f32", True, 32, False)])
def test_scratch_for_a_copy_only_where_there_is_one(tokens, dtype, out, unrounded, group, copied, monkeypatch):
    """dy in odd rows is copied into aligned ones where its type has two bytes and tiles read it as it is; other calls ask for no such memory."""
    outer, inner = 131, 64
    dy = numbers(tokens, outer, dtype, seed=2)
    w, x = codes_with(outer, inner, 0.01, 4, group)[0], codes_with(tokens, inner, 0.01, 5, group)[0]
    asked = []
    given = act8.scratch
    monkeypatch.setattr(act8, "scratch", lambda n, device: (asked.append(n), given(n, device))[1])
    for op, call, c in ((T.TGRAD_CODES_GRAD_INPUT, act8.tgrad_codes_grad_input, w), (T.TGRAD_CODES_GRAD_WEIGHT, act8.tgrad_codes_grad_weight, x)):
        n = C.c_size_t(0)
        assert T.load().tgrad_codes_query_size(op + (T.TGRAD_CODES_UNALIGNED if copied else 0), tokens, inner, outer, C.byref(n)) == T.TGRAD_OK
        call(dy, c, dtype=TYPES[out][0], unrounded=unrounded)
        assert asked.pop() == n.value


@pytest.mark.parametrize("tokens,inner,outer", [(3, 200, 90), (8, 4096, 64), (40, 4096, 40), (700, 300, 200)])
def test_no_scratch_for_codes_that_are_kept(tokens, inner, outer, monkeypatch):
    x, w = numbers(tokens, inner, "bf16", seed=1), codes_with(outer, inner, 0.01, 2)[0]
    want = act8.tgrad_codes_linear(x, w).y
    asked = []
    given = act8.scratch
    monkeypatch.setattr(act8, "scratch", lambda n, device: (asked.append(n), given(n, device))[1])
    n = C.c_size_t(0)
    assert T.load().tgrad_codes_query_size(T.TGRAD_CODES_MATMUL, tokens, inner, outer, C.byref(n)) == T.TGRAD_OK
    y, x8 = act8.tgrad_codes_linear(x, w, keep=True)
    assert asked == [n.value] and torch.equal(y, want) and torch.equal(act8.tgrad_codes_matmul(x8, w), want)


@pytest.mark.parametrize("tokens,inner,outer", RANGE)
@pytest.mark.parametrize("scale", [1000.0, 2.0 ** -26, 2.0 ** -130, 2.0 ** 100])
def test_unrounded_float16_values_beyond_float16(tokens, inner, outer, scale):
    """Results that leave float16 are infinite, or at its end; the others are right."""
    dy = (numbers(tokens, outer, "f16", seed=1) * 2.0 ** -6).contiguous()
    w, cw, sw = codes_with(outer, inner, scale, 2)
    x, cx, sx = codes_with(tokens, inner, scale, 3)
    for call, c, a, b, terms in ((act8.tgrad_codes_grad_input, w, dy.cpu().double(), spread_out(cw, sw, 0), outer),
                                 (act8.tgrad_codes_grad_weight, x, dy.cpu().double().t().contiguous(), spread_out(cx, sx, 0), tokens)):
        want, size = a @ b, a.abs() @ b.abs()
        for out in ("f16", "f32"):
            t, u, tiny = TYPES[out]
            got = call(dy, c, dtype=t, unrounded=True).cpu().double()
            fits = want.abs() < 65000 if out == "f16" else torch.ones_like(want, dtype=torch.bool)
            value = PARTS["f16"] if out == "f16" else U
            # float32's own 2^-110 below which dy's last parts are lost, times codes: 2^-103 a term
            lost = terms * 2.0 ** -103 if out == "f32" or tokens <= 16 else 0.0
            off = (got - want).abs()
            assert bool((off <= size * (value + (6 * terms + 4) * U) * (1 + u) + want.abs() * u + tiny + lost)[fits].all())
            assert bool((got[~fits].isinf() | (got[~fits].abs() > 60000)).all())


def test_scales_that_are_no_sizes():
    """A row of codes with a NaN or an infinite scale spoils what it goes into, and float16's power of two is taken from the others."""
    dy = numbers(64, 48, "f16", seed=1)
    w, cw, sw = codes_with(48, 32, 2.0 ** -30, 2)
    for bad in (float("nan"), float("inf")):
        w.scale[7] = bad
        for unrounded in (False, True):
            assert not bool(torch.isfinite(act8.tgrad_codes_grad_input(dy, w, unrounded=unrounded)).any())
            x, cx, sx = codes_with(64, 32, 2.0 ** -30, 3)
            x.scale[5] = bad
            d = act8.tgrad_codes_grad_weight(dy, x, dtype=torch.float32, unrounded=unrounded)
            assert not bool(torch.isfinite(d).any())
