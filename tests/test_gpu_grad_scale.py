"""tgrad_set_grad_scale: a step with a factor is the step on the gradient times that factor.

Tolerance.  By a power of two nothing is rounded differently: the bits are the same.  By another factor every number of the scaled
gradient, and every scaled compressed value, carries one rounding (2^-24) more, and the core's sums their own errors (some 2^-22 of their
largest terms); the update divides by sqrt(V), so that a relative error of the moments is one of the update: 1e-5 of its norm is 40 times
that.  This needs a core that is no rounding noise: the factors come from a gradient that no step sees (with two modes, the core of the
gradient that its own singular vectors compress is diagonal, and AdamUpdate makes whole steps of the noise beside the diagonal).
"""
import numpy as np
import pytest
import torch

from paper_2501_02379_amd import group, tgrad as T

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
#        shape, ranks, k, what it runs
CASES = {
    "ends_core": ((16, 16, 8, 5), (8, 8, 4, 3), 103),
    "core2": ((12, 10, 16, 9), (4, 4, 5, 4), 90),
    "wide_core": ((70, 9, 12, 17), (40, 4, 6, 8), 200),
    "no_core": ((130, 3, 40, 33), (64, 2, 33, 20), 300),
    "two_modes": ((40, 33), (10, 9), 25),
    "generic_last": ((6, 7, 80), (3, 4, 50), 60),
    "no_sparse": ((16, 16, 8, 5), (8, 8, 4, 3), 0),
}


def make(shape, ranks, k, order=T.TGRAD_ORDER_US_LR, grad="c64", seed=1):
    gen = torch.Generator().manual_seed(seed)
    cfg = T.make_config(shape, ranks, k, lr=1e-2, beta1=0.9, beta2=0.99, refresh_every=0, order=order, weight_decay=0.01,
                        grad_dtype=T.TGRAD_CBF16 if grad == "bf16" else T.TGRAD_C64)
    grads = []
    for _ in range(4):
        g = torch.randn(*shape, 2, generator=gen)
        g.view(-1, 2)[::53] *= 10
        grads.append(g.to(torch.bfloat16) if grad == "bf16" else g)
    w = torch.randn(*shape, 2, generator=gen)
    return cfg, grads, w


def send(g):
    return (g.view(torch.int16) if g.dtype == torch.bfloat16 else g).contiguous().to(DEV)


def run(cfg, grads, w, factors, scale=None):
    """Steps of a context that starts from the given support and factors; -> W, moments, reported values."""
    ctx = T.Context(cfg, device=DEV)
    if factors is None:
        ctx.tgrad_refresh_factors(send(grads[3]))
    else:
        for what, value in factors.items():
            ctx.tgrad_set_state(what, value)
    kept = {T.STATE_FACTOR0 + n: ctx.tgrad_get_state(T.STATE_FACTOR0 + n) for n in range(cfg.ndim)}
    kept[T.STATE_INDICES] = ctx.tgrad_get_state(T.STATE_INDICES)
    wd = w.to(DEV)
    if scale is not None:
        ctx.tgrad_set_grad_scale(torch.full((1,), scale, device=DEV))
    for g in grads[:3]:
        ctx.tgrad_step(wd, send(g))
    out = [wd.cpu().numpy()] + [ctx.tgrad_get_state(s) for s in (T.STATE_CORE_M, T.STATE_CORE_V, T.STATE_SPARSE_M, T.STATE_SPARSE_V,
                                                                T.STATE_SPARSE_G, T.STATE_CORE_G)]
    ctx.tgrad_destroy()
    return out, kept


@pytest.mark.parametrize("order", [T.TGRAD_ORDER_US_LR, T.TGRAD_ORDER_LR_US, T.TGRAD_ORDER_SUM])
@pytest.mark.parametrize("name", list(CASES))
def test_a_power_of_two_changes_no_bit(name, order):
    cfg, grads, w = make(*CASES[name], order=order)
    _, kept = run(cfg, grads, w, None)
    want, _ = run(cfg, [g * 0.25 for g in grads], w, kept)
    got, _ = run(cfg, grads, w, kept, scale=0.25)
    plain, _ = run(cfg, grads, w, kept)
    one, _ = run(cfg, grads, w, kept, scale=1.0)
    generic = name in ("generic_last",)                        # its sparse values are replaced by the update they make
    for i, (a, b) in enumerate(zip(want, got)):
        if not (generic and i == 5):
            assert np.array_equal(a, b), i
    for i, (a, b) in enumerate(zip(plain, one)):
        if not (generic and i == 5):
            assert np.array_equal(a, b), i


@pytest.mark.parametrize("grad", ["c64", "bf16"])
@pytest.mark.parametrize("name", list(CASES))
def test_any_factor(name, grad):
    cfg, grads, w = make(*CASES[name], grad=grad)
    _, kept = run(cfg, grads, w, None)
    cfg32, _, _ = make(*CASES[name])
    scale = float(np.float32(0.137))
    want, _ = run(cfg32, [g.float() * scale for g in grads], w, kept)
    got, _ = run(cfg, grads, w, kept, scale=scale)
    dw, dw2 = want[0] - w.numpy(), got[0] - w.numpy()
    assert np.linalg.norm(dw - dw2) <= 1e-5 * np.linalg.norm(dw)


def test_the_factor_is_read_when_the_step_runs_and_none_ends_it():
    cfg, grads, w = make(*CASES["ends_core"])
    ctx = T.Context(cfg, device=DEV)
    g = send(grads[0])
    ctx.tgrad_refresh_factors(g)
    factor = torch.ones(1, device=DEV)
    ctx.tgrad_set_grad_scale(factor)
    wd = w.to(DEV)
    ctx.tgrad_step(wd, g)
    one = ctx.tgrad_get_state(T.STATE_CORE_G)
    factor.fill_(0.5)
    ctx.tgrad_step(wd, g)
    assert np.array_equal(ctx.tgrad_get_state(T.STATE_CORE_G), 0.5 * one)
    ctx.tgrad_set_grad_scale(None)
    ctx.tgrad_step(wd, g)
    assert np.array_equal(ctx.tgrad_get_state(T.STATE_CORE_G), one)
    for bad in (torch.ones(1), torch.ones(2, device=DEV), torch.ones(1, device=DEV, dtype=torch.float64)):
        with pytest.raises(T.TgradError):
            ctx.tgrad_set_grad_scale(bad)
    assert T.load().tgrad_set_grad_scale(None, None) == T.TGRAD_ERR_INVALID_ARG
    ctx.tgrad_destroy()


def test_clipping_a_spectral_gradient_and_the_rest_together():
    """One norm over a spectral gradient and dense ones; both kinds of step take its factor from the device."""
    cfg, grads, w = make(*CASES["ends_core"])
    gen = torch.Generator().manual_seed(3)
    dense = torch.randn(300, generator=gen).to(DEV)
    p, m, v = torch.zeros(300, device=DEV), torch.zeros(300, device=DEV), torch.zeros(300, device=DEV)
    spectral = send(grads[0])
    everything = group.Group([torch.view_as_complex(spectral), dense])
    rest = group.Group([dense], [p], [m], [v])
    ctx = T.Context(cfg, device=DEV)
    ctx.tgrad_refresh_factors(spectral)
    norm = everything.tgrad_group_grad_norm(1.0)
    ctx.tgrad_set_grad_scale(norm[1:])
    wd = w.to(DEV)
    ctx.tgrad_step(wd, spectral)
    rest.tgrad_group_adamw(0, lr=1e-2, norm=norm)
    total = float((spectral.double().square().sum() + dense.double().square().sum()).sqrt())
    coef = 1.0 / (total + 1e-6)
    assert abs(float(norm[0]) - total) <= 1e-6 * total
    assert torch.allclose(m, dense * (0.1 * coef), rtol=1e-5, atol=0)
    core = ctx.tgrad_get_state(T.STATE_CORE_G)
    ctx.tgrad_set_grad_scale(None)
    ctx.tgrad_step(wd, spectral)
    raw = ctx.tgrad_get_state(T.STATE_CORE_G)
    assert np.linalg.norm(core - coef * raw) <= 1e-5 * np.linalg.norm(core)
    ctx.tgrad_destroy()
