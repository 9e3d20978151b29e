"""Global gradient norm, clipping and AdamW over a group of tensors, against their definitions in float64 on the CPU.

Tolerances.  u = 2^-24.  The norm is summed in float64 and rounded once: 2 u.  The factor has three float32 operations behind it:
4 u.  A scaled gradient carries the factor's error, a product's and the rounding to its type.  AdamW: a moment is two products and a
sum, of a gradient that carries the factor's error: 8 u of the absolute terms (16 u of the squared one); the root and the quotient
halve and add relative errors, 16 u of the step in all, and the parameter two roundings more and that to its type.
"""
import numpy as np
import pytest
import torch

from paper_2501_02379_amd import group, tgrad as T

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
ROUND = {torch.float32: (U, 2.0 ** -149), torch.bfloat16: (2.0 ** -8, 2.0 ** -133), torch.float16: (2.0 ** -11, 2.0 ** -25),
         torch.complex64: (U, 2.0 ** -149), torch.int16: (2.0 ** -8, 2.0 ** -133)}
KINDS = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "c64": torch.complex64, "cbf16": torch.int16}
SIZES = [1, 2, 7, 8, 63, 255, 257, 4095, 4096, 4097, 8191, 12289, 100003]


def tensor(n, kind, gen, scale=1.0, offset=0):
    """n elements in device memory that start `offset` elements behind an allocation's start; bf16 pairs as int16[n, 2]."""
    dt = KINDS[kind]
    if dt == torch.int16:
        v = (torch.randn(n + offset, 2, generator=gen) * scale).to(torch.bfloat16).view(torch.int16)
    elif dt == torch.complex64:
        v = torch.randn(n + offset, dtype=dt, generator=gen) * scale
    else:
        v = (torch.randn(n + offset, generator=gen) * scale).to(dt)
    return v.to(DEV)[offset:]


def wide(t):
    """float64 / complex128 on the CPU."""
    t = t.detach().cpu()
    if t.dtype == torch.int16:
        return torch.view_as_complex(t.view(torch.bfloat16).double().contiguous())
    return t.to(torch.complex128) if t.is_complex() else t.double()


def parts(z):
    return torch.view_as_real(z) if z.is_complex() else z


def norm_of(grads):
    return float(sum(parts(wide(g)).square().sum() for g in grads).sqrt())


def close_scaled(got, g, coef):
    want = parts(wide(g)) * coef
    u, tiny = ROUND[g.dtype]
    assert bool(((parts(wide(got)) - want).abs() <= want.abs() * (u + 8 * U) + tiny).all())


@pytest.mark.parametrize("offset", [0, 1, 3, 8])
@pytest.mark.parametrize("kind", list(KINDS))
def test_norm_and_clipping(kind, offset):
    gen = torch.Generator().manual_seed(offset)
    grads = [tensor(n, kind, gen, 0.01, offset) for n in SIZES]
    before = [g.clone() for g in grads]
    outs = [torch.zeros_like(g) for g in grads]
    want = norm_of(grads)
    g = group.Group(grads, outs=outs)
    r = g.tgrad_group_grad_norm(1.0)
    assert abs(float(r[0]) - want) <= 2 * U * want
    assert abs(float(g.sumsq(r)) - want * want) <= 1e-12 * want * want
    coef = min(1.0, 1.0 / (want + 1e-6))
    assert coef < 1 and abs(float(r[1]) - coef) <= 4 * U * coef
    r2 = g.tgrad_group_clip(0.5)
    for o, b, x in zip(outs, before, grads):
        assert torch.equal(x, b)                                  # untouched: they have somewhere else to go
        close_scaled(o, b, 0.5 / (want + 1e-6))
    same = group.Group(grads)
    r3 = same.tgrad_group_clip(0.5)
    assert torch.equal(r2, r3)
    for o, x in zip(outs, grads):
        assert torch.equal(o, x)
    once = [x.clone() for x in grads]
    r4 = same.tgrad_group_clip(1e9)                               # within the bound: nothing changes
    assert float(r4[1]) == 1.0 and all(torch.equal(a, b) for a, b in zip(once, grads))
    g.tgrad_group_grad_norm(1e9, into=r2)
    g.tgrad_group_scale(r2)                                       # copied where it has to be
    assert all(torch.equal(a, b) for a, b in zip(outs, grads))


def test_mixed_types_many_tensors_and_empty_ones():
    gen = torch.Generator().manual_seed(1)
    r = np.random.RandomState(1)
    grads = [tensor(int(r.choice([0, 1, 5, 130, 4096, 5000])), list(KINDS)[i % 5], gen, 0.1, int(r.randint(0, 4))) for i in range(1500)]
    want = norm_of(grads)
    before = [x.clone() for x in grads]
    g = group.Group(grads)
    a, b = g.tgrad_group_grad_norm(2.0), g.tgrad_group_grad_norm(2.0)
    assert torch.equal(a, b) and abs(float(a[0]) - want) <= 2 * U * want
    g.tgrad_group_scale(a)
    for x, y in zip(grads, before):
        if x.numel():
            close_scaled(x, y, 2.0 / (want + 1e-6))
    none = group.Group([torch.empty(0, device=DEV), torch.empty(0, 2, dtype=torch.int16, device=DEV)])
    n = none.tgrad_group_clip(1.0)
    assert float(n[0]) == 0 and float(n[1]) == 1


def test_sums_from_elsewhere_and_extremes():
    x = torch.full((1000,), 3e30, device=DEV)
    y = torch.full((1000,), 1e-30, device=DEV)
    gx, gy = group.Group([x]), group.Group([y])
    rx, ry = gx.tgrad_group_grad_norm(1.0), gy.tgrad_group_grad_norm(1.0)
    wx, wy = float(np.float32(3e30)) * 1000 ** 0.5, float(np.float32(1e-30)) * 1000 ** 0.5
    assert abs(float(rx[0]) - wx) <= 2 * U * wx and abs(float(ry[0]) - wy) <= 2 * U * wy and float(ry[1]) == 1
    z = torch.full((4,), 2.0, device=DEV)
    gz = group.Group([z, x[:0]])
    rz = gz.tgrad_group_grad_norm(1.0)
    three = gz.tgrad_group_grad_norm(1.0, add_sumsq=torch.full((1,), 9.0, dtype=torch.float64, device=DEV))
    assert float(rz[0]) == 4 and float(three[0]) == 5
    both = gz.tgrad_group_grad_norm(1.0, add_sumsq=gz.sumsq(rz), into=rz)       # the result over what it adds
    assert abs(float(both[0]) - 32 ** 0.5) <= 1e-6
    for bad, coef in ((float("inf"), 0.0), (float("-inf"), 0.0), (float("nan"), None)):
        z[3] = bad
        r = gz.tgrad_group_grad_norm(1.0)
        assert not np.isfinite(float(r[0]))
        assert float(r[1]) == coef if coef is not None else np.isnan(float(r[1]))
    z.zero_()
    r = gz.tgrad_group_grad_norm(1.0)
    assert float(r[0]) == 0 and float(r[1]) == 1
    z.fill_(1.0)
    r = gz.tgrad_group_clip(0.0)
    assert float(r[1]) == 0 and not bool(z.any())


def adamw_reference(g, p, m, v, coef, lr, b1, b2, eps, wd, t):
    g, p, m, v = wide(g) * coef, wide(p), wide(m), wide(v)
    if g.is_complex() and not m.is_complex():
        m = torch.view_as_complex(m.contiguous())
    if g.is_complex() and not p.is_complex():
        p = torch.view_as_complex(p.contiguous())
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g.abs().square()
    c1, c2 = 1 - b1 ** (t + 1), 1 - b2 ** (t + 1)
    size = (v1 / c2).sqrt() + eps
    step = lr * (m1 / c1) / size
    m_off = 8 * U * (b1 * parts(m).abs() + (1 - b1) * parts(g).abs())
    v_off = 16 * U * v1
    # d size / size <= v_off / (2 v1), in the other terms 16 u
    p_off = 4 * U * parts(p).abs() + 32 * U * parts(step).abs() + (m_off * lr / c1) / (size[..., None] if g.is_complex() else size)
    return p * (1 - lr * wd) - step, m1, v1, p_off, m_off, v_off


def within(got, want, off, dtype):
    u, tiny = ROUND[dtype]
    got, want = parts(wide(got)).reshape(-1), parts(want).reshape(-1)
    assert bool(((got - want).abs() <= off.reshape(-1) + want.abs() * (u + U) + tiny).all()), float(((got - want).abs() / (off.reshape(-1) + want.abs() * (u + U) + tiny)).max())


PAIRS = [("f32", "f32"), ("bf16", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("f16", "f16"), ("f32", "f16"), ("bf16", "f16"),
         ("f16", "bf16"), ("c64", "c64"), ("cbf16", "c64"), ("cbf16", "cbf16"), ("c64", "cbf16")]


@pytest.mark.parametrize("offsets", [(0, 0, 0, 0), (1, 1, 1, 1), (8, 4, 12, 4), (3, 0, 5, 2)])
@pytest.mark.parametrize("kinds", PAIRS, ids=["-".join(p) for p in PAIRS])
def test_adamw(kinds, offsets):
    gen = torch.Generator().manual_seed(11)
    gk, pk = kinds
    cplx = gk in ("c64", "cbf16")
    mk = "c64" if cplx else "f32"
    grads = [tensor(n, gk, gen, 0.02, offsets[0]) for n in SIZES]
    params = [tensor(n, pk, gen, 0.5, offsets[1]) for n in SIZES]
    m = [tensor(n, mk, gen, 0.01, offsets[2]) for n in SIZES]
    v = [tensor(n, "f32", gen, 0.01, offsets[3]).square_() for n in SIZES]
    for k in (3, 5):                                                            # first steps: no state yet
        m[k].zero_()
        v[k].zero_()
    wd = [0.1 * (i % 3) for i in range(len(SIZES))]
    scale = [1.0 if i % 2 else 0.5 for i in range(len(SIZES))]
    old = [[t.clone() for t in s] for s in (grads, params, m, v)]
    g = group.Group(grads, params, m, v, lr_scale=scale, weight_decay=wd)
    for t, clip in ((7, True), (0, False)):
        norm = g.tgrad_group_grad_norm(0.3) if clip else None
        before = [[t_.clone() for t_ in s] for s in (params, m, v)]
        g.tgrad_group_adamw(t, lr=3e-3, beta1=0.9, beta2=0.98, eps=1e-8, norm=norm)
        coef = min(1.0, 0.3 / (norm_of(grads) + 1e-6)) if clip else 1.0
        for i in range(len(SIZES)):
            assert torch.equal(grads[i], old[0][i])
            wp, wm, wv, po, mo, vo = adamw_reference(grads[i], before[0][i], before[1][i], before[2][i], coef,
                                                     3e-3 * float(np.float32(scale[i])), 0.9, 0.98, 1e-8, float(np.float32(wd[i])), t)
            within(m[i], wm, mo, torch.float32)
            within(v[i], wv, vo, torch.float32)
            within(params[i], wp, po, params[i].dtype)


def test_adamw_complex_as_pairs_and_as_complex_are_one():
    """complex64 tensors, and this library's float32[..., 2] weights with bf16 or complex64 gradients."""
    gen = torch.Generator().manual_seed(12)
    g = tensor(5000, "c64", gen)
    p, m, v = tensor(5000, "c64", gen), tensor(5000, "c64", gen, 0.1), tensor(5000, "f32", gen).square_()
    p2, m2, v2 = torch.view_as_real(p).clone(), torch.view_as_real(m).clone(), v.clone()
    group.Group([g], [p], [m], [v]).tgrad_group_adamw(3, lr=0.1)
    group.Group([g], [p2], [m2], [v2]).tgrad_group_adamw(3, lr=0.1)
    assert torch.equal(torch.view_as_real(p), p2) and torch.equal(torch.view_as_real(m), m2) and torch.equal(v, v2)


def test_adamw_skips_what_is_not_finite():
    gen = torch.Generator().manual_seed(13)
    g, p, m, v = (tensor(9000, "f32", gen) for _ in range(4))
    v.square_()
    grp = group.Group([g], [p], [m], [v])
    for bad in (float("nan"), float("inf")):
        g[77] = bad
        old = [t.clone() for t in (p, m, v)]
        norm = grp.tgrad_group_grad_norm(1.0)
        grp.tgrad_group_adamw(0, lr=0.1, norm=norm, skip_nonfinite=True)
        assert all(torch.equal(a, b) for a, b in zip(old, (p, m, v)))
    g[77] = 0.5
    norm = grp.tgrad_group_grad_norm(1.0)
    grp.tgrad_group_adamw(0, lr=0.1, norm=norm, skip_nonfinite=True)
    assert not torch.equal(old[0], p) and bool(torch.isfinite(p).all())


def test_bind_moves_a_group_to_other_tensors():
    gen = torch.Generator().manual_seed(14)
    sizes = [5, 4097, 300]
    a, b = [tensor(n, "bf16", gen) for n in sizes], [tensor(n, "bf16", gen, 3.0) for n in sizes]
    g = group.Group(a)
    ra = g.tgrad_group_grad_norm(1.0)
    g.tgrad_group_bind(b)
    rb = g.tgrad_group_grad_norm(1.0)
    assert abs(float(ra[0]) - norm_of(a)) <= 2 * U * norm_of(a) and abs(float(rb[0]) - norm_of(b)) <= 2 * U * norm_of(b)
    for bad in ([b[0], b[1]], [b[1], b[0], b[2]], [x.float() for x in b]):
        with pytest.raises(T.TgradError):
            g.tgrad_group_bind(bad)
    with pytest.raises(T.TgradError):
        g.tgrad_group_bind(b, outs=a)
    assert torch.equal(g.tgrad_group_grad_norm(1.0), rb)


def test_large_tensor_beyond_32_bit_offsets():
    """2.2e9 bf16 numbers: pieces past 2^31 elements and 2^32 bytes."""
    n = (1 << 31) + (1 << 26) + 5
    x = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    at = [0, (1 << 31) - 1, 1 << 31, (1 << 31) + 4097, n - 1]
    for k in at:
        x[k] = 2.0
    g = group.Group([x])
    r = g.tgrad_group_clip(1.0)
    assert abs(float(r[0]) - 20 ** 0.5) <= 1e-6
    want = torch.tensor(2.0 / (20 ** 0.5 + 1e-6)).to(torch.bfloat16)
    assert all(x[k].cpu() == want for k in at) and int(torch.count_nonzero(x)) == len(at)


def test_another_stream_and_graph_replays():
    gen = torch.Generator().manual_seed(15)
    grads = [tensor(n, "bf16", gen) for n in SIZES]
    params, m = [tensor(n, "f32", gen) for n in SIZES], [torch.zeros(n, device=DEV) for n in SIZES]
    v = [torch.zeros(n, device=DEV) for n in SIZES]
    eager = [[t.clone() for t in s] for s in (params, m, v)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = group.Group(grads, params, m, v, stream=side)
    e = group.Group(grads, *eager)
    result = g.tgrad_group_grad_norm(1.0)
    graph = torch.cuda.CUDAGraph()
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        g.tgrad_group_grad_norm(1.0, into=result)
        g.tgrad_group_adamw(4, lr=1e-2, norm=result)
    for k in range(4):
        for x in grads:
            x.mul_(1.0 + 0.25 * k)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        r = e.tgrad_group_grad_norm(1.0)
        e.tgrad_group_adamw(4, lr=1e-2, norm=r)
        assert torch.equal(r, result)
        for a, b in zip((params, m, v), eager):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_the_binding_refuses():
    x = torch.zeros(8, device=DEV)
    z = torch.zeros(8, dtype=torch.complex64, device=DEV)
    for bad in (lambda: group.Group([x.double()]), lambda: group.Group([x.view(2, 4).t()]), lambda: group.Group([x], [x.clone()]),
                lambda: group.Group([x], exp_avg=[x.clone()]), lambda: group.Group([x], [x.clone()], [x.clone()], [x[:4]]),
                lambda: group.Group([x], [x], [x.clone()], [x.clone()]), lambda: group.Group([x], [z], [z.clone()], [x.clone()]),
                lambda: group.Group([x], outs=[x[:4]]), lambda: group.Group([x], outs=[x.clone(), x.clone()]),
                lambda: group.Group([x], weight_decay=[-1.0]), lambda: group.Group([x], lr_scale=[1.0, 2.0])):
        with pytest.raises(T.TgradError):
            bad()
    g = group.Group([x])
    h = group.Group([x], [x.clone()], [x.clone()], [x.clone()])
    r = g.tgrad_group_grad_norm(1.0)
    for bad in (lambda: g.tgrad_group_adamw(0, lr=0.1), lambda: g.tgrad_group_grad_norm(-1.0), lambda: g.tgrad_group_grad_norm(float("nan")),
                lambda: h.tgrad_group_adamw(-1, lr=0.1), lambda: h.tgrad_group_adamw(0, lr=-0.1), lambda: h.tgrad_group_adamw(0, lr=0.1, beta1=1.0),
                lambda: h.tgrad_group_adamw(0, lr=0.1, skip_nonfinite=True), lambda: h.tgrad_group_adamw(0, lr=0.1, eps=float("nan")),
                lambda: g.tgrad_group_scale(x), lambda: g.tgrad_group_grad_norm(1.0, add_sumsq=x)):
        with pytest.raises(T.TgradError):
            bad()
    assert float(r[1]) == 1


def test_tensors_that_memory_does_not_hold():
    """Autograd leaves gradients whose conjugation is still pending: their memory holds other numbers, so they are refused."""
    p = torch.randn(6, dtype=torch.complex64, device=DEV, requires_grad=True)
    p.conj().backward(torch.randn(6, dtype=torch.complex64, device=DEV))
    assert p.grad.is_conj()
    moments = [torch.zeros(6, dtype=torch.complex64, device=DEV)], [torch.zeros(6, device=DEV)]
    with pytest.raises(T.TgradError):
        group.Group([p.grad])
    g = group.Group([p.grad.resolve_conj()], [p.detach()], *moments)
    with pytest.raises(T.TgradError):
        g.tgrad_group_bind([p.grad])
    with pytest.raises(T.TgradError):
        group.Group([torch._neg_view(torch.randn(6, device=DEV))])
    assert bool(torch.isfinite(g.tgrad_group_grad_norm(1.0)).all())
