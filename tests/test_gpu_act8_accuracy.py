"""Activations in float32 over the whole range of their argument, against float64: an error of a few u, u = 2^-24, of the result's terms wherever they lie.

exp(-|v|) with its argument's rounding made good: 4 u (the instruction is right to one unit, 2 u); 1 + that and its reciprocal 3 u, products 2 u: silu 10 u of itself,
slope p (1 + v (1 - p)) 9 u for p, 10 for v (1 - p), 3 for what joins them: 24 u of the terms' sizes.  gelu's tail exp(-v^2 / 2) t P(t): the exponential 4 u; t = 1 / (1 + 0.4 z)
3.5 u, and P moves by at most 1.6 times that of itself (|t P'| <= 1.6 P on 0..1); the fit 2 u; Horner's ten steps of terms up to 2.4 P in
size 2.4 * 2 u each for the last three, which alone keep their size: 15 u; products 3 u: 34 u of the tail, 40 u with what is made of it.  Below float32's normal range exp(-|v|)
and p are rounded by 2^-150 each, which |v| < 103 makes 2^-142 of silu; slopes below 2^-120 are left out of the relative bound.
"""
import pytest
import torch

from paper_2501_02379_amd import act8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


def arguments(low, high):
    g = torch.Generator().manual_seed(1)
    at = torch.cat([torch.linspace(low, high, 40001, dtype=torch.float64), (torch.rand(30000, generator=g, dtype=torch.float64) - 0.5) * 8,
                    10.0 ** (torch.rand(3000, generator=g, dtype=torch.float64) * 8 - 8), -(10.0 ** (torch.rand(3000, generator=g, dtype=torch.float64) * 8 - 8))])
    return at.clamp(low, high).float().view(1, -1)


def of(act, v):
    """(value, slope, sizes of the slope's terms) in float64; tails through functions that keep them."""
    if act == "silu":
        p, q = torch.sigmoid(v), torch.sigmoid(-v)
        return v * p, p * (1 + v * q), p * (1 + (v * q).abs())
    p, d = torch.special.erfc(v * -0.5 ** 0.5) / 2, torch.exp(-v * v / 2) / (2 * torch.pi) ** 0.5
    return v * p, p + v * d, p + (v * d).abs()


@pytest.mark.parametrize("act,low,high,of_value,of_slope", [("silu", -103.0, 90.0, 10, 24), ("gelu", -12.5, 12.5, 40, 44)])
def test_float32_activations_keep_their_tails(act, low, high, of_value, of_slope):
    x = arguments(low, high).to(DEV)
    y = act8.tgrad_activation(x, act=act, keep=False).y.cpu().double()
    want = of(act, x.cpu().double())[0]
    assert bool(((y - want).abs() <= want.abs() * (of_value + 1) * U + 2.0 ** -142).all())
    if act == "silu":
        assert bool(y.cpu()[x.cpu() < -88].ne(0).any())                       # what float32 still holds there
    # the slope at what a checkpoint stands for; groups of 32 neighbours, so that it spans the range
    c = act8.tgrad_quantize(x, group=32)
    v = act8.tgrad_dequantize(c).cpu().double()
    dx, _ = act8.tgrad_activation_backward(torch.ones_like(x), c, act=act)
    _, slope, size = of(act, v)
    assert bool(((dx.cpu().double() - slope).abs() <= size * of_slope * U + 2.0 ** -120).all())


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_ends_of_the_range(act, dtype):
    inf, nan = float("inf"), float("nan")
    x = torch.tensor([[inf, nan, 0.0, -0.0, 60000.0, -60000.0, torch.finfo(dtype).max, torch.finfo(dtype).min]], dtype=dtype, device=DEV)
    y = act8.tgrad_activation(x, act=act, keep=False).y[0].cpu()
    assert y[0] == inf and y[1].isnan() and bool(y[2:4].eq(0).all()) and bool(y[[5, 7]].eq(0).all()) and torch.equal(y[[4, 6]], x[0, [4, 6]].cpu())
    x = torch.tensor([[100.0, -100.0, 0.0, 1e30, -1e30]], device=DEV).to(torch.float32)
    c = act8.tgrad_quantize(x.t().contiguous())                                # a scale each
    dx, _ = act8.tgrad_activation_backward(torch.ones(5, 1, device=DEV).to(dtype), c, act=act)
    assert dx.flatten().tolist() == [1.0, 0.0, 0.5, 1.0, 0.0] or dtype is torch.float32 and bool((dx.flatten().cpu() - torch.tensor([1.0, 0, 0.5, 1, 0])).abs().lt(1e-35).all())
