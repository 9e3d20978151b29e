"""Groups of tensors: arguments that are not what they should be, infinite norms, tensors that are let go while the device still
works on them."""
import math

import numpy as np
import pytest
import torch

from paper_2501_02379_amd import group, losses, tgrad as T

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_scaling_needs_an_earlier_result():
    """None is no factor, and a result whose two numbers do not lie side by side is none; nothing is written."""
    g = [torch.randn(5000, device=DEV), torch.randn(70, device=DEV)]
    was = [t.clone() for t in g]
    grp = group.Group(g)
    apart = torch.ones(6, device=DEV)[2::2]
    assert apart.shape == (2,) and apart.storage_offset() == 2
    for bad in (lambda: grp.tgrad_group_scale(None), lambda: grp.tgrad_group_scale(apart), lambda: grp.tgrad_group_grad_norm(1.0, into=apart),
                lambda: grp.tgrad_group_clip(1.0, into=apart), lambda: grp.tgrad_group_clip(1.0, into=torch.ones(2, device=DEV))):
        with pytest.raises(T.TgradError):
            bad()
    assert all(torch.equal(a, b) for a, b in zip(g, was))
    grp.tgrad_group_scale(grp.tgrad_group_grad_norm(1.0))
    assert not torch.equal(g[0], was[0])


def busy():
    """A side stream with some tens of milliseconds of waiting in front of what comes next."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    return side


def test_replaced_tensors_last_until_the_groups_stream_has_passed():
    n = 9_700_001
    x = torch.full((n,), 2.0, device=DEV)
    want = 2.0 * n ** 0.5
    torch.cuda.synchronize()
    side = busy()
    grp = group.Group([x], stream=side)
    r = grp.tgrad_group_grad_norm(1.0)
    at = x.data_ptr()
    grp.tgrad_group_bind([torch.ones(n, device=DEV)])
    del x
    fresh = torch.full((n,), 7.0, device=DEV)
    assert fresh.data_ptr() != at
    torch.cuda.synchronize()
    assert abs(float(r[0]) - want) <= 1e-6 * want


def test_tensors_of_a_dropped_group_last_too():
    n = 9_800_003
    x, m, v, g = (torch.full((n,), k, device=DEV) for k in (1.0, 0.0, 0.0, 3.0))
    torch.cuda.synchronize()
    side = busy()
    grp = group.Group([g], [x], [m], [v], stream=side)
    grp.tgrad_group_adamw(0, lr=1e-2)
    at = {t.data_ptr() for t in (m, v, g)}
    del grp, m, v, g
    fresh = [torch.full((n,), 7.0, device=DEV) for _ in range(3)]
    assert not at & {t.data_ptr() for t in fresh}
    torch.cuda.synchronize()
    assert bool(((x - 0.99).abs() < 1e-6).all()) and all(bool((t == 7).all()) for t in fresh)


def test_arguments_of_a_loss_on_another_stream_last():
    rows, vocab = 503, 20_011
    x = torch.zeros(rows, vocab, device=DEV)
    y = torch.zeros(rows, dtype=torch.int64, device=DEV)
    torch.cuda.synchronize()
    side = busy()
    logp, _ = losses.tgrad_token_logprobs(x, targets=y, stream=side)
    at = x.data_ptr()
    del x
    fresh = torch.randn(rows, vocab, device=DEV)
    assert fresh.data_ptr() != at
    torch.cuda.synchronize()
    assert bool(((logp + math.log(vocab)).abs() < 1e-5).all())


def test_a_replaced_factor_lasts():
    shape = (16, 16, 8, 5)
    side = torch.cuda.Stream()
    w, g = torch.zeros(*shape, 2, device=DEV), torch.randn(*shape, 2, device=DEV)
    ctx = T.Context(T.make_config(shape, (8, 8, 4, 3), 103), stream=side)
    torch.cuda.synchronize()
    ctx.tgrad_step(w, g)                                               # loads the kernels: what follows takes the host less than the wait
    scale = torch.full((1,), 0.5, device=DEV)
    at = scale.data_ptr()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    ctx.tgrad_set_grad_scale(scale)
    ctx.tgrad_step(w, g)
    done = torch.cuda.Event()
    done.record(side)
    ctx.tgrad_set_grad_scale(None)
    del scale
    fresh = [torch.zeros(1, device=DEV) for _ in range(64)]
    assert not done.query()                                            # or this test shows nothing
    assert at not in {t.data_ptr() for t in fresh}
    torch.cuda.synchronize()
    ctx.tgrad_destroy()


def test_an_unbounded_norm():
    """max_norm = inf only measures: factor 1, and still 0 for an infinite norm, NaN for a NaN."""
    x = torch.full((300,), 1e4, device=DEV)
    grp = group.Group([x])
    assert float(grp.tgrad_group_grad_norm(math.inf)[1]) == 1
    for bad in (math.inf, -math.inf):
        x[7] = bad
        norm, coef = grp.tgrad_group_grad_norm(math.inf).tolist()
        assert norm == math.inf and coef == 0
    x[9] = math.nan
    assert all(math.isnan(k) for k in grp.tgrad_group_grad_norm(math.inf).tolist())


def test_rates_and_decays_of_any_sequence():
    """Arrays and tuples as well as lists; an empty one is not one for every gradient."""
    def step(lr_scale, weight_decay):
        p, g = [torch.ones(50, device=DEV), torch.ones(60, device=DEV)], [torch.ones(50, device=DEV), torch.ones(60, device=DEV)]
        m, v = [torch.zeros_like(t) for t in p], [torch.zeros_like(t) for t in p]
        group.Group(g, p, m, v, lr_scale=lr_scale, weight_decay=weight_decay).tgrad_group_adamw(0, lr=0.1)
        return torch.cat(p)

    want = step([1.0, 0.5], [0.0, 0.25])
    assert torch.equal(step(np.array([1.0, 0.5]), np.array([0.0, 0.25], dtype=np.float32)), want)
    assert torch.equal(step((1.0, 0.5), torch.tensor([0.0, 0.25])), want)
    for bad in (([], None), (None, ()), ([1.0], None)):
        with pytest.raises(T.TgradError):
            step(*bad)


def test_an_overflowed_step_left_out_for_both_kinds_of_parameter():
    """The norm read on the host in front of tgrad_step, skip_nonfinite for the rest: weights and moments as if the gradient had not been."""
    shape, steps = (16, 16, 8, 5), 6
    gen = torch.Generator().manual_seed(3)
    spectral = [torch.randn(*shape, 2, generator=gen) for _ in range(steps)]
    dense = [torch.randn(3000, generator=gen) for _ in range(steps)]

    def train(overflow):
        ctx = T.Context(T.make_config(shape, (8, 8, 4, 3), 103, lr=1e-2, refresh_every=2))
        w, p = torch.ones(*shape, 2, device=DEV), torch.ones(3000, device=DEV)
        gs, gd = torch.zeros_like(w), torch.zeros_like(p)
        m, v = torch.zeros_like(p), torch.zeros_like(p)
        every, rest = group.Group([gs, gd]), group.Group([gd], [p], [m], [v])
        norm = every.tgrad_group_grad_norm(1.0)
        ctx.tgrad_set_grad_scale(norm[1:])
        t = 0
        for k in range(steps):
            for bad in ((True, False) if overflow and k in (0, 3) else (False,)):
                gs.copy_(spectral[k])
                gd.copy_(dense[k])
                if bad:
                    gs[1, 2, 3, 4, 0] = gd[5] = math.inf
                every.tgrad_group_grad_norm(1.0, into=norm)
                rest.tgrad_group_adamw(t, lr=1e-2, norm=norm, skip_nonfinite=True)
                if math.isfinite(float(norm[0])):
                    ctx.tgrad_step(w, gs)
                    t += 1
        got = [w, p, m, v] + [torch.from_numpy(ctx.tgrad_get_state(s)) for s in (T.STATE_CORE_M, T.STATE_CORE_V, T.STATE_SPARSE_M)]
        ctx.tgrad_destroy()
        return got

    for a, b in zip(train(True), train(False)):
        assert torch.equal(a, b) and bool(torch.isfinite(torch.view_as_real(a) if a.is_complex() else a).all())


def test_streams_of_another_gpu_are_refused():
    from types import SimpleNamespace
    other = SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0)
    x, y = torch.zeros(3, 5, device=DEV), torch.zeros(3, dtype=torch.int64, device=DEV)
    for bad in (lambda: losses.tgrad_token_logprobs(x, y, stream=other), lambda: losses.tgrad_token_logprobs(logits=x, targets=y, stream=other),
                lambda: group.Group([x], stream=other)):
        with pytest.raises(T.TgradError):
            bad()
