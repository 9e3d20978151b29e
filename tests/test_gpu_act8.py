"""Codes of 8 bits, the products with them and the activations that keep them, against their definitions in float64 on the CPU.

Tolerances.  u = 2^-24 (float32).  Scales and codes have one right value (the largest magnitude over 127 in float32; the exact quotient to nearest
even, which float64 gives: 127 v and a have at most 31 and 24 bits, so a quotient is a border or at least 2^-32 away from one), and so has the
product of two matrices of codes (an exact int32 sum, then one conversion and two products in float32): those are compared bit by bit.
A gradient sums S products, exact in float32 for two-byte types; however they are added, that is off by at most 2 u S sum |a b| (2 u an addition:
matrix instructions need not round to nearest).  In float32 dy * scale is rounded once, split in three parts off by 2^-24 together, and 3 S
products are added: (6 S + 4) u sum |a b|, and so for two-byte types and up to 16 tokens.
silu in float32: exp(-v) is off by (2 |v| + 2) u of itself, the quotient adds 3 u: |y| (2 |v| + 8) u; its slope p (1 + v (1 - p)) three times that of
each term.  gelu: v / sqrt(2) carries 1.5 u, which moves erfc by up to 3 (1 + v^2) u of itself, erfc itself 8 u; exp(-v^2 / 2) (v^2 + 4) u.
Each result is then rounded to its type once.
"""
import numpy as np
import pytest
import torch

from paper_2501_02379_amd import act8, tgrad as T

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": (torch.float32, U, 2.0 ** -149), "bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -133),
         "f16": (torch.float16, 2.0 ** -11, 2.0 ** -24)}


def strided(x, dtype, pad=0, offset=0):
    """x on the GPU as a view with `pad` elements between rows, NaN in them, starting `offset` elements into its memory."""
    rows, cols = x.shape
    flat = torch.full((offset + rows * (cols + pad) + 8,), float("nan"), dtype=dtype)
    view = flat[offset:offset + rows * (cols + pad)].view(rows, cols + pad)
    view[:, :cols] = x.to(dtype)
    dev = flat.to(DEV)
    return dev[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]


def numbers(rows, cols, dtype, seed=0, spread=1.0, pad=0, offset=0):
    g = torch.Generator().manual_seed(seed)
    return strided(torch.randn(rows, cols, generator=g) * spread, TYPES[dtype][0], pad, offset)


def right_codes(x, group=0):
    """(codes, scales) as they have to be, on the CPU."""
    v = x.detach().cpu().double().numpy()
    rows, cols = v.shape
    g = group or cols
    n = -(-cols // g)
    codes, scale = np.zeros((rows, cols), np.int8), np.zeros((rows, n), np.float32)
    for i in range(n):
        part = v[:, i * g:(i + 1) * g]
        top = np.abs(part).max(1)
        bad = ~np.isfinite(top)
        live = ~bad & (top >= 2.0 ** -119)
        scale[:, i] = np.where(bad, np.float32("nan"), np.where(live, top.astype(np.float32) / np.float32(127), 0))
        with np.errstate(all="ignore"):
            q = np.rint(127 * part / np.where(live, top, 1)[:, None])
        codes[:, i * g:(i + 1) * g] = np.where(live[:, None], q, 0).astype(np.int8)
    with np.errstate(all="ignore"):                                  # no value of a finite number is infinite: the scale below, then
        scale = np.where(np.isinf(scale * np.float32(127)), np.nextafter(scale, np.float32(0)), scale)
    return torch.from_numpy(codes), torch.from_numpy(scale)


def values(codes, scale, group):
    g = group or codes.shape[1]
    return codes.float() * scale.repeat_interleave(g, 1)[:, :codes.shape[1]]


def same_codes(c, x):
    codes, scale = right_codes(x, c.group)
    assert torch.equal(c.codes.cpu(), codes)
    assert torch.equal(c.scale.cpu().nan_to_num(nan=-1.0), scale.nan_to_num(nan=-1.0))


def laid(codes, scale, group=0, pad=0, offset=0):
    """Codes on the GPU with the given padding behind every row and start."""
    rows, cols = codes.shape
    flat = torch.full((offset + rows * (cols + pad) + 16,), 77, dtype=torch.int8, device=DEV)
    view = flat[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(codes)
    return act8.Codes(view, scale.to(DEV), group)


def random_codes(rows, cols, group=0, seed=0, pad=0, offset=0):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(-127, 128, (rows, cols), generator=g, dtype=torch.int8)
    scale = torch.rand(rows, -(-cols // group) if group else 1, generator=g) * 0.02 + 0.001
    return laid(codes, scale, group, pad, offset), codes, scale


SHAPES = [(1, 1), (3, 7), (2, 64), (5, 513), (4, 2048), (3, 2055), (300, 40), (2, 8192), (3, 16389), (1, 32768), (2, 40003), (1, 131072)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("group", [0, 32, 128, 512])
def test_codes_and_back(rows, cols, dtype, group):
    x = numbers(rows, cols, dtype, seed=rows * cols, pad=cols % 5, offset=cols % 3)
    c = act8.tgrad_quantize(x, group=group)
    same_codes(c, x)
    want = values(c.codes.cpu(), c.scale.cpu(), group)
    for t in TYPES.values():
        assert torch.equal(act8.tgrad_dequantize(c, t[0]).cpu(), want.to(t[0]))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_quotients_on_and_next_to_borders(dtype):
    t = TYPES[dtype][0]
    x = torch.zeros(4, 600)
    for r, a in enumerate((4.0, 1.984375, 254.0, 3.0)):
        x[r, 0] = a
        k = torch.arange(-127, 127)
        x[r, 1:255] = (2 * k + 1) * a / 254                       # halves, exact ones where the type has them
        at = x[r, 1:255].to(t)
        x[r, 255:509] = torch.nextafter(at, torch.full_like(at, float("inf"))).float()
        x[r, 300:509] = torch.nextafter(at, torch.full_like(at, float("-inf"))).float()[:209]
    x = x.clamp(-254, 254).to(t).to(DEV)
    same_codes(act8.tgrad_quantize(x), x)
    same_codes(act8.tgrad_quantize(x, group=64), x)


@pytest.mark.parametrize("group", [0, 32])
def test_groups_of_zeros_infinities_and_tiny_numbers(group):
    x = torch.randn(8, 100, generator=torch.Generator().manual_seed(1))
    x[0] = 0
    x[1, 40] = float("inf")
    x[2, 99] = float("nan")
    x[3] *= 2.0 ** -130
    x[4] *= 2.0 ** -117
    x[5] *= 2.0 ** 125
    x[6, 3] = float("-inf")
    x[7, 64] = 3.4028234e38
    x = x.to(DEV)
    c = act8.tgrad_quantize(x, group=group)
    same_codes(c, x)
    back = act8.tgrad_dequantize(c).cpu()
    assert bool(back[0].eq(0).all()) and bool(back[3].eq(0).all()) and bool(back[1, 32:64].isnan().all()) and bool(back[2, 96:].isnan().all())
    assert bool(torch.isfinite(back[[4, 5, 7]]).all())
    if group == 0:
        assert bool(back[1].isnan().all())


@pytest.mark.parametrize("rows,cols", [(0, 5), (0, 4096)])
def test_no_rows(rows, cols):
    x = torch.empty(rows, cols, device=DEV)
    c = act8.tgrad_quantize(x, group=32)
    assert act8.tgrad_dequantize(c).shape == (0, cols)
    w, _, _ = random_codes(6, cols)
    assert act8.tgrad_codes_linear(x, w).y.shape == (0, 6)
    assert act8.tgrad_codes_matmul(act8.tgrad_quantize(x), w).shape == (0, 6)
    assert act8.tgrad_activation(x, x, quantize=True).y.codes.shape == (0, cols)
    dy = torch.empty(0, 6, device=DEV)
    assert act8.tgrad_codes_grad_input(dy, w).shape == (0, cols)
    assert bool(act8.tgrad_codes_grad_weight(dy, c).eq(0).all())


def test_what_lies_between_rows_stays():
    x = numbers(5, 100, "bf16")
    out = act8.Codes(torch.full((5, 120), 55, dtype=torch.int8, device=DEV)[:, :100], torch.zeros(5, 4, device=DEV), 32)
    act8.tgrad_quantize(x, group=32, out=out)
    assert bool(out.codes.as_strided((5, 20), (120, 1), 100).eq(55).all())
    y = torch.full((5, 131), 9.0, dtype=torch.bfloat16, device=DEV)
    w, _, _ = random_codes(101, 100)
    act8.tgrad_codes_linear(x, w, out=y[:, 7:108])
    assert bool(y[:, :7].eq(9).all()) and bool(y[:, 108:].eq(9).all()) and not bool(y[:, 7:108].eq(9).all())
    act8.tgrad_codes_grad_input(y[:, 7:108], w, out=(z := torch.full((5, 109), 9.0, dtype=torch.bfloat16, device=DEV))[:, 1:101])
    assert bool(z[:, :1].eq(9).all()) and bool(z[:, 101:].eq(9).all())
    act8.tgrad_codes_grad_weight(y[:, 7:108], out, out=(z := torch.full((103, 109), 9.0, dtype=torch.bfloat16, device=DEV))[1:102, 3:103])
    assert bool(z[[0, 102]].eq(9).all()) and bool(z[:, :3].eq(9).all()) and bool(z[:, 103:].eq(9).all())


# ---- products -------------------------------------------------------------------------------------------------------------

# tokens, inner, outer: single tokens, a few, ordinary; sums of odd length, shorter than a step, long ones
PRODUCTS = [(1, 1, 1), (1, 16, 5), (1, 4096, 300), (2, 100, 64), (3, 129, 1000), (7, 8190, 33), (16, 256, 257), (17, 1000, 130), (33, 64, 64),
            (64, 640, 513), (100, 77, 300), (130, 1300, 260), (256, 512, 256), (257, 257, 257), (300, 128, 1024), (511, 2304, 700), (3600, 333, 3700), (20, 5000, 40), (32, 2049, 515),
            (29, 9000, 3800),
            (1, 131072, 3), (40, 131072, 17)]


def right_product(codes, scale, wcodes, wscale, dtype):
    exact = codes.double() @ wcodes.double().t()                   # sums below 2^31 are exact in float64
    return (exact.float() * scale * wscale.view(1, -1)).to(dtype)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("tokens,inner,outer", PRODUCTS)
def test_products_of_codes(tokens, inner, outer, dtype):
    t = TYPES[dtype][0]
    for pads in ((0, 0, 0, 0), (-inner % 16, 0, -inner % 16, 0), (3, 1, 5, 2)):
        x, cx, sx = random_codes(tokens, inner, seed=1, pad=pads[0], offset=pads[1])
        w, cw, sw = random_codes(outer, inner, seed=2, pad=pads[2], offset=pads[3])
        assert torch.equal(act8.tgrad_codes_matmul(x, w, dtype=t).cpu(), right_product(cx, sx, cw, sw, t))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("tokens,inner,outer", PRODUCTS)
def test_linear_is_quantize_and_product(tokens, inner, outer, dtype):
    t = TYPES[dtype][0]
    x = numbers(tokens, inner, dtype, seed=tokens, pad=inner % 3)
    w, cw, sw = random_codes(outer, inner, seed=2, pad=-inner % 16)
    codes, scale = right_codes(x)
    want = right_product(codes, scale, cw, sw, t)
    y, x8 = act8.tgrad_codes_linear(x, w, keep=True)
    same_codes(x8, x)
    assert torch.equal(y.cpu(), want)
    y, x8 = act8.tgrad_codes_linear(x, w)
    assert x8 is None and torch.equal(y.cpu(), want)


def test_largest_sums_of_codes_fit():
    for sign in (1, -1):
        x = laid(torch.full((2, 131072), 127, dtype=torch.int8), torch.ones(2, 1))
        w = laid(torch.full((3, 131072), 127 * sign, dtype=torch.int8), torch.ones(3, 1))
        assert bool(act8.tgrad_codes_matmul(x, w, dtype=torch.float32).eq(float(np.float32(127 * 127 * 131072 * sign))).all())


def test_a_token_with_a_nan_spoils_its_own_row_alone():
    for tokens in (1, 5, 200):
        x = numbers(tokens, 300, "bf16")
        x[tokens // 2, 17] = float("nan")
        w, _, _ = random_codes(70, 300)
        y = act8.tgrad_codes_linear(x, w).y
        assert bool(y[tokens // 2].isnan().all()) and int(y.isnan().any(1).sum()) == 1


GRADS = [(1, 1, 1), (1, 300, 77), (5, 64, 33), (31, 65, 130), (64, 128, 256), (100, 513, 66), (257, 255, 129), (640, 96, 300), (2051, 70, 40),
         (300, 1030, 520), (5000, 64, 32), (20000, 33, 48), (3584, 96, 100),
         (3700, 3588, 40), (40, 3700, 3592),
         (70000, 264, 250), (257, 2090, 2050)]


def close_gradient(got, a, b, dtype, out, terms):
    """got against a @ b, a gradient of products of a and b (float64)."""
    want, size = a @ b, a.abs() @ b.abs()
    u, tiny = TYPES[out][1:]
    per = 6 * terms + 4                                             # the larger of the two
    bound = size * per * U * (1 + u) + want.abs() * u + tiny
    assert got.dtype == TYPES[out][0]
    off = (got.cpu().double() - want).abs()
    assert bool((off <= bound).all()), float((off / bound.clamp(min=1e-300)).max())


def rounded(codes, scale, group, dtype, tokens):
    """What the gradients multiply with: values of codes, rounded to a two-byte type but for a few tokens and one scale a row."""
    return values(codes, scale, group).to(TYPES[dtype][0]).double() if dtype != "f32" and (tokens > 16 or 0 < group < codes.shape[1]) else codes.double() * scale.double().repeat_interleave(group or codes.shape[1], 1)[:, :codes.shape[1]]


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f16", "f32")])
@pytest.mark.parametrize("tokens,inner,outer", GRADS)
def test_gradients(tokens, inner, outer, dtype, out):
    dy = numbers(tokens, outer, dtype, seed=3, pad=outer % 4, offset=outer % 3)
    for pad, offset, group in ((-inner % 16, 0, 0), (0, 1, 0), (-inner % 16, 0, 32), (5, 2, 128)):
        w, cw, sw = random_codes(outer, inner, group, seed=4, pad=pad, offset=offset)
        got = act8.tgrad_codes_grad_input(dy, w, dtype=TYPES[out][0])
        close_gradient(got, dy.cpu().double(), rounded(cw, sw, group, dtype, tokens), dtype, out, outer)
        x, cx, sx = random_codes(tokens, inner, group, seed=5, pad=pad, offset=offset)
        got = act8.tgrad_codes_grad_weight(dy, x, dtype=TYPES[out][0])
        close_gradient(got, dy.cpu().double().t().contiguous(), rounded(cx, sx, group, dtype, tokens), dtype, out, tokens)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_gradients_of_whole_numbers_are_exact(dtype):
    """Sums of whole numbers below 2^24 have one value, whatever the order."""
    g = torch.Generator().manual_seed(0)
    for tokens, inner, outer in ((777, 260, 515), (4096, 192, 256)):
        dy = torch.randint(-2, 3, (tokens, outer), generator=g).to(TYPES[dtype][0])
        cw, cx = (torch.randint(-9, 10, (n, inner), generator=g, dtype=torch.int8) for n in (outer, tokens))
        w, x = (laid(c, torch.ones(len(c), 1), pad=-inner % 16) for c in (cw, cx))
        got = act8.tgrad_codes_grad_input(dy.to(DEV), w, dtype=torch.float32)
        assert torch.equal(got.cpu().double(), dy.double() @ cw.double())
        got = act8.tgrad_codes_grad_weight(dy.to(DEV), x, dtype=torch.float32)
        assert torch.equal(got.cpu().double(), dy.double().t().contiguous() @ cx.double())


def test_gradients_are_those_of_the_product():
    """<dy, product> as a function of its factors is linear in each: its differences are the gradients."""
    dy = numbers(20, 30, "f32", seed=7).cpu().double()
    x, cx, sx = random_codes(20, 50, seed=8)
    w, cw, sw = random_codes(30, 50, seed=9)
    vx, vw = cx.double() * sx.double(), cw.double() * sw.double()
    loss = lambda a, b: float((dy * (a @ b.t())).sum())  # noqa: E731
    dx = act8.tgrad_codes_grad_input(dy.float().to(DEV), w).cpu().double()
    dw = act8.tgrad_codes_grad_weight(dy.float().to(DEV), x).cpu().double()
    g = torch.Generator().manual_seed(2)
    for _ in range(8):
        e, f = torch.randn(20, 50, generator=g, dtype=torch.float64), torch.randn(30, 50, generator=g, dtype=torch.float64)
        # 4 u (6 * 30 + 4) of the terms' sizes, as above, and 1e-12 of the losses for the differences in float64
        for grad, d, diff, size in ((dx, e, loss(vx + e, vw) - loss(vx, vw), dy.abs() @ vw.abs()), (dw, f, loss(vx, vw + f) - loss(vx, vw), dy.abs().t() @ vx.abs())):
            assert abs(float((grad * d).sum()) - diff) <= float((size * d.abs()).sum()) * (6 * 30 + 4) * U + 1e-12 * abs(loss(vx, vw)) + 1e-9


# ---- activation -------------------------------------------------------------------------------------------------------------

def act_of(name, v):
    """The activation, its slope, and what float32 may be off by in each."""
    if name == "silu":
        p = torch.sigmoid(v)
        k = (2 * v.abs() + 8) * U
        return v * p, p * (1 + v * (1 - p)), (v * p).abs() * k + 1e-36, (p + (p * v * (1 - p)).abs()) * 3 * k + 1e-36
    p, d = torch.special.erfc(v * -0.5 ** 0.5) / 2, torch.exp(-v * v / 2) / np.sqrt(2 * np.pi)
    k = (3 * (1 + v * v) + 12) * U
    return v * p, p + v * d, (v * p).abs() * k + 1e-36, (p + (v * d).abs()) * k + 1e-36


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (5, 200), (2, 4096), (3, 9001), (1, 33000), (70, 129)])
def test_activation_and_its_backward_pass(rows, cols, dtype, act, gated):
    t, u, tiny = TYPES[dtype]
    group = {1: 32, 31: 32, 200: 64, 4096: 128, 9001: 512, 33000: 256, 129: 128}[cols]
    x = numbers(rows, cols, dtype, seed=cols, spread=2.5, pad=cols % 3, offset=1)
    gate = numbers(rows, cols, dtype, seed=cols + 1, pad=cols % 2) if gated else None
    if cols > 40:
        x[0, :5] = torch.tensor([-100.0, 100.0, 0.0, -20.0, 30.0]).to(t)
    v = x.cpu().double()
    y, _, off, _ = act_of(act, v)
    if gated:
        y, off = y * gate.cpu().double(), off * gate.cpu().double().abs() + (y * gate.cpu().double()).abs() * U
    a = act8.tgrad_activation(x, gate, act=act, group=group)
    assert a.y.dtype is t and bool(((a.y.cpu().double() - y).abs() <= off * (1 + u) + y.abs() * u + tiny).all())
    same_codes(a.x8, x)
    if gated:
        same_codes(a.gate8, gate)
    assert act8.tgrad_activation(x, gate, act=act, keep=False).x8 is None

    # in 8 bits: the scale is that of the right largest number, codes are off by what the numbers are, and half a step
    q = act8.tgrad_activation(x, gate, act=act, group=group, quantize=True)
    assert torch.equal(q.x8.codes, a.x8.codes) and (not gated or torch.equal(q.gate8.scale, a.gate8.scale))
    top = y.abs().amax(1, keepdim=True)
    assert bool(((q.y.scale.cpu().double() * 127 - top).abs() <= off.amax(1, keepdim=True) + 2 * U * top).all())
    s = q.y.scale.cpu().double()
    assert bool(((q.y.codes.cpu().double() * s - y).abs() <= s * (0.5 + 127 * 2 * U) + off + off.amax(1, keepdim=True)).all())

    dy = numbers(rows, cols, dtype, seed=5, pad=2)
    dx, dgate = act8.tgrad_activation_backward(dy, a.x8, a.gate8, act=act)
    v = values(a.x8.codes.cpu(), a.x8.scale.cpu(), group).double()
    y, slope, off, off_slope = act_of(act, v)
    d = dy.cpu().double()
    g = values(a.gate8.codes.cpu(), a.gate8.scale.cpu(), group).double() if gated else torch.ones_like(d)
    want = d * g * slope
    assert dx.dtype is t and bool(((dx.cpu().double() - want).abs() <= (d * g).abs() * off_slope + want.abs() * (u + 3 * U) + tiny).all())
    h = 1e-5                                                        # central differences: h^2 / 6 times a third derivative below 2, and float64's rounding
    diff = (act_of(act, v + h)[0] - act_of(act, v - h)[0]) / (2 * h)
    assert bool(((dx.cpu().double() - d * g * diff).abs() <= (d * g).abs() * (off_slope + 1e-9) + want.abs() * (u + 3 * U) + tiny).all())
    if gated:
        want = d * y
        assert bool(((dgate.cpu().double() - want).abs() <= d.abs() * off + want.abs() * (u + 2 * U) + tiny).all())
    else:
        assert dgate is None


def test_gradients_go_into_halves_of_one_matrix():
    both = numbers(9, 400, "bf16", seed=2)
    a = act8.tgrad_activation(both[:, :200], both[:, 200:], group=32)
    dy = numbers(9, 200, "bf16", seed=3)
    out = torch.full((9, 400), 5.0, dtype=torch.bfloat16, device=DEV)
    act8.tgrad_activation_backward(dy, a.x8, a.gate8, out=out[:, :200], gate_out=out[:, 200:])
    dx, dgate = act8.tgrad_activation_backward(dy, a.x8, a.gate8)
    assert torch.equal(out, torch.cat([dx, dgate], 1))


# ---- far rows, streams, graphs --------------------------------------------------------------------------------------------------

def test_rows_behind_4_gib():
    stride = (1 << 30) + 8
    x = torch.empty(2 * stride + 600, dtype=torch.bfloat16, device=DEV).as_strided((3, 600), (stride, 1))
    x.copy_(numbers(3, 600, "bf16"))
    q = torch.empty(2 * stride + 600, dtype=torch.int8, device=DEV).as_strided((3, 600), (stride, 1))
    c = act8.Codes(q, torch.empty(3, 1, device=DEV), 0)
    act8.tgrad_quantize(x, out=c)
    same_codes(c, x)
    near = act8.tgrad_quantize(x.clone())
    w, _, _ = random_codes(40, 600, seed=1)
    y = torch.empty(2 * stride + 40, dtype=torch.bfloat16, device=DEV).as_strided((3, 40), (stride, 1))
    act8.tgrad_codes_matmul(c, w, out=y)
    assert torch.equal(y, act8.tgrad_codes_matmul(near, w))
    dx = x                                                          # its memory is free now
    act8.tgrad_codes_grad_input(y, w, out=dx)
    assert torch.equal(dx, act8.tgrad_codes_grad_input(y.clone(), w))
    assert torch.equal(act8.tgrad_codes_grad_weight(y, c), act8.tgrad_codes_grad_weight(y.clone(), near))
    a, b = act8.tgrad_activation(dx), act8.tgrad_activation(dx.clone())
    assert torch.equal(a.y, b.y) and torch.equal(a.x8.codes, b.x8.codes)


def _layer(x, w, w2, dy):
    h = act8.tgrad_codes_linear(x, w, keep=True)
    a = act8.tgrad_activation(h.y, quantize=True)
    y = act8.tgrad_codes_matmul(a.y, w2)
    da = act8.tgrad_codes_grad_input(dy, w2)
    dw2 = act8.tgrad_codes_grad_weight(dy, a.y)
    dh, _ = act8.tgrad_activation_backward(da, a.x8)
    return y, dw2, act8.tgrad_codes_grad_input(dh, w), act8.tgrad_codes_grad_weight(dh, h.x8)


@pytest.mark.parametrize("tokens", [1, 200, 3000])
def test_captured_and_replayed(tokens):
    w, w2 = random_codes(300, 128, seed=1)[0], random_codes(96, 300, seed=2)[0]
    x, dy = numbers(tokens, 128, "bf16"), numbers(tokens, 96, "bf16", seed=4)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _layer(x, w, w2, dy)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _layer(x, w, w2, dy)
    for seed in range(4):
        x.copy_(numbers(tokens, 128, "bf16", seed=10 + seed))
        graph.replay()
        want = _layer(x, w, w2, dy)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_on_another_stream():
    w, w2 = random_codes(300, 128, seed=1)[0], random_codes(96, 300, seed=2)[0]
    x, dy = numbers(500, 128, "bf16"), numbers(500, 96, "bf16", seed=4)
    want = _layer(x, w, w2, dy)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    h = act8.tgrad_codes_linear(x, w, keep=True, stream=s)
    a = act8.tgrad_activation(h.y, quantize=True, stream=s)
    da = act8.tgrad_codes_grad_input(dy, w2, stream=s)
    dh, _ = act8.tgrad_activation_backward(da, a.x8, stream=s)
    got = (act8.tgrad_codes_matmul(a.y, w2, stream=s), act8.tgrad_codes_grad_weight(dy, a.y, stream=s), act8.tgrad_codes_grad_input(dh, w, stream=s),
           act8.tgrad_codes_grad_weight(dh, h.x8, stream=s))
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))


# ---- refusals -------------------------------------------------------------------------------------------------------------------

def test_refusals():
    x, w = numbers(4, 64, "bf16"), random_codes(8, 64)[0]
    c = act8.tgrad_quantize(x)
    grouped = act8.tgrad_quantize(x, group=32)
    dy = numbers(4, 8, "bf16")
    long = act8.Codes(torch.zeros(1, 131073, dtype=torch.int8, device=DEV), torch.ones(1, 1, device=DEV), 0)
    for call in (lambda: act8.tgrad_quantize(x.cpu()), lambda: act8.tgrad_quantize(x[0]), lambda: act8.tgrad_quantize(x.t()), lambda: act8.tgrad_quantize(x.double()),
                 lambda: act8.tgrad_quantize(x, group=16), lambda: act8.tgrad_quantize(x, group=-32), lambda: act8.tgrad_quantize(x, out=grouped),
                 lambda: act8.tgrad_quantize(torch._neg_view(x)), lambda: act8.tgrad_dequantize(c, torch.float64),
                 lambda: act8.tgrad_dequantize(act8.Codes(c.codes, c.scale[:3], 0)), lambda: act8.tgrad_dequantize(act8.Codes(c.codes, c.scale, 32)),
                 lambda: act8.tgrad_dequantize(act8.Codes(c.codes.float(), c.scale, 0)), lambda: act8.tgrad_dequantize((c.codes, c.scale, 0)),
                 lambda: act8.tgrad_codes_matmul(grouped, w), lambda: act8.tgrad_codes_matmul(c, random_codes(8, 63)[0]),
                 lambda: act8.tgrad_codes_matmul(c, w, out=torch.empty(4, 9, device=DEV, dtype=torch.bfloat16)), lambda: act8.tgrad_codes_matmul(long, long),
                 lambda: act8.tgrad_codes_matmul(c, w, dtype=torch.int8), lambda: act8.tgrad_codes_linear(x, grouped), lambda: act8.tgrad_codes_linear(x.t(), w),
                 lambda: act8.tgrad_codes_grad_input(dy, c), lambda: act8.tgrad_codes_grad_input(dy, w, dtype=torch.float16),
                 lambda: act8.tgrad_codes_grad_weight(dy, random_codes(5, 64)[0]), lambda: act8.tgrad_activation(x, x[:, :32]),
                 lambda: act8.tgrad_activation(x, x.float()), lambda: act8.tgrad_activation(x, act="tanh"), lambda: act8.tgrad_activation(x, group=0),
                 lambda: act8.tgrad_activation_backward(dy, grouped), lambda: act8.tgrad_activation_backward(x, grouped, gate_out=x),
                 lambda: act8.tgrad_activation_backward(x, grouped, act="relu")):
        with pytest.raises(T.TgradError):
            call()
    torch.cuda.synchronize()


def test_results_go_where_they_are_told():
    x = numbers(40, 300, "bf16", seed=3)
    want = act8.tgrad_activation(x, x, quantize=True)
    out = laid(torch.zeros(40, 300, dtype=torch.int8), torch.zeros(40, 1), pad=5, offset=3)
    got = act8.tgrad_activation(x, x, quantize=True, out=out)
    assert got.y is out and torch.equal(out.codes, want.y.codes) and torch.equal(out.scale, want.y.scale)
    w, _, _ = random_codes(70, 300, seed=1)
    h = act8.tgrad_codes_linear(x, w, keep=True, dtype=torch.float32, out=(y := torch.empty(40, 90, device=DEV))[:, 9:79])
    assert h.y.data_ptr() == y[:, 9:].data_ptr() and torch.equal(h.y, act8.tgrad_codes_matmul(h.x8, w, dtype=torch.float32))
    for bad in (lambda: act8.tgrad_activation(x, quantize=True, out=act8.tgrad_quantize(x, group=32)), lambda: act8.tgrad_activation(x, out=want.y),
                lambda: act8.tgrad_activation(x, quantize=True, out=torch.empty_like(x))):
        with pytest.raises(T.TgradError):
            bad()


@pytest.mark.parametrize("tokens,inner,outer", [(5, 200, 90), (300, 300, 100), (3600, 3600, 136), (3601, 3590, 135)])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_nan_in_a_gradient_stays_in_its_row_and_column(tokens, inner, outer, dtype, value):
    dy = numbers(tokens, outer, dtype, seed=2)
    t, n = tokens - 2, outer // 2
    dy[t, n] = value
    w, x = random_codes(outer, inner, seed=4, pad=-inner % 16)[0], random_codes(tokens, inner, seed=5, pad=-inner % 16)[0]
    dx, dw = act8.tgrad_codes_grad_input(dy, w), act8.tgrad_codes_grad_weight(dy, x)
    for got, r in ((dx, t), (dw, n)):                               # an infinity times a code of 0 is NaN too
        assert not bool(torch.isfinite(got[r]).any()) and int((~torch.isfinite(got)).any(1).sum()) == 1


def test_the_same_bits_every_time():
    dy, w, x = numbers(5000, 300, "f16", seed=1), random_codes(300, 200, seed=2)[0], random_codes(5000, 200, seed=3)[0]
    first = act8.tgrad_codes_grad_input(dy, w), act8.tgrad_codes_grad_weight(dy, x)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, (act8.tgrad_codes_grad_input(dy, w), act8.tgrad_codes_grad_weight(dy, x))))
