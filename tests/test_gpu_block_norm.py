"""The norms around a block, forward and backward, against their formulas in float64 on the CPU.

Tolerances.  u = 2^-24.  A thread adds up at most 32 numbers one by one, lanes and wavefronts at most 10 + 16 more, so a sum of one sign is off by at most
60 u of itself, and a factor 1 / sqrt(mean + eps) by 33 u.  A mean is off by d = 60 u mean |v|, and a normed number n by 36 u |n| + r d.  A sum
over a row's products g n is off by (60 + 40) u sum |g n| and by r d sum |g|.  With K = 200 u for all of that, and sizes added where terms are:
  dx   K (|dx_out| + r (|g| + |n| mean |g n| + mean |g|)) + r^2 d (|g| / |..| ...): the mean's error moves n by r d, hence dx by r (r d) (mean |g n| + |n| mean |g|)
Sums over T rows add T u of the sum of sizes.  Each result is rounded to its type once.
"""
import pytest
import torch

from paper_2501_02379_amd import act8, norms, tgrad as T

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
K = 200 * U
EPS = 1e-6
TYPES = {"f32": (torch.float32, U, 2.0 ** -149), "bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -133),
         "f16": (torch.float16, 2.0 ** -11, 2.0 ** -24)}


def randn(gen, rows, cols, dtype, spread=1.0, mean=0.0, pad=0):
    flat = torch.full((rows, cols + pad), float("nan"))
    flat[:, :cols] = torch.randn(rows, cols, generator=gen) * spread + mean
    return flat.to(TYPES[dtype][0]).to(DEV)[:, :cols]


def make(rows, cols, stream="f32", dtype="f32", shared=1, weights="f32", seed=0, pad=0, mean=0.3):
    g = torch.Generator().manual_seed(seed)
    wt = TYPES[weights][0]
    return {"x": randn(g, rows, cols, stream, 2.0, mean, pad), "block": randn(g, rows, cols, dtype, 0.7, mean, pad),
            "gate": randn(g, -(-rows // shared), cols, dtype, 0.3, 0.5, pad), "post": (1 + 0.2 * torch.randn(cols, generator=g)).to(wt).to(DEV),
            "pre": (1 + 0.2 * torch.randn(cols, generator=g)).to(wt).to(DEV), "dx": randn(g, rows, cols, stream, 0.5, 0.0, pad),
            "dh": randn(g, rows, cols, dtype, 0.5, 0.0, pad)}


def d64(t):
    return t.detach().cpu().double()


def normed(v, centered):
    """n, r and the mean's possible error, in float64."""
    m = v.mean(1, keepdim=True) if centered else 0.0
    d = 60 * U * v.abs().mean(1, keepdim=True) if centered else torch.zeros(len(v), 1, dtype=torch.float64)
    r = ((v - m).square().mean(1, keepdim=True) + EPS).rsqrt()
    return (v - m) * r, r, d


def close(got, want, size, dtype):
    u, tiny = TYPES[dtype][1:]
    assert got.dtype is TYPES[dtype][0]
    off, bound = (d64(got) - want).abs(), size * (1 + u) + want.abs() * u + tiny
    assert bool((off <= bound).all()), float((off / bound.clamp(min=1e-300)).max())


def spread_gate(s, shared, rows):
    return d64(s["gate"])[torch.arange(rows) // shared]


def check(rows, cols, stream, dtype, shared, centered, weights="f32", pad=0, scale=0.7, with_post=True, with_gate=True, with_pre=True, with_dx=True, seed=0):
    s = make(rows, cols, stream, dtype, shared, weights, seed, pad)
    args = {"post_weight": s["post"] if with_post else None, "gate": s["gate"] if with_gate else None, "rows_per_gate": shared, "scale": scale,
            "pre_weight": s["pre"] if with_pre else None, "centered": centered}
    f = norms.tgrad_block_norm(s["x"], s["block"], eps=EPS, **args)
    b, x = d64(s["block"]), d64(s["x"])
    gate = spread_gate(s, shared, rows) if with_gate else torch.ones(rows, cols, dtype=torch.float64)
    post = d64(s["post"]) if with_post else torch.ones(cols, dtype=torch.float64)
    pre = d64(s["pre"])
    nb, rb, db = normed(b, centered) if with_post else (b, torch.ones(rows, 1, dtype=torch.float64), torch.zeros(rows, 1, dtype=torch.float64))
    branch = scale * gate * nb * post
    close(f.x, x + branch, K * (branch.abs() + x.abs()) + (scale * gate * post).abs() * rb * db, stream)
    nx, rx, dx_mean = normed(d64(f.x), centered)
    if with_pre:
        close(f.h, nx * pre, (K * nx.abs() + rx * dx_mean) * pre.abs(), dtype)
        q = norms.tgrad_block_norm(s["x"], s["block"], eps=EPS, quantize=True, **args)
        assert torch.equal(q.x, f.x)
        step = d64(q.h.scale)
        off = (K * nx.abs() + rx * dx_mean) * pre.abs()
        assert bool(((d64(act8.tgrad_dequantize(q.h)) - nx * pre).abs() <= step * (0.5 + 130 * U) + off + off.amax(1, keepdim=True)).all())
    else:
        assert f.h is None

    # backward
    up, dh = d64(s["dx"]) if with_dx else torch.zeros(rows, cols, dtype=torch.float64), d64(s["dh"])
    r = norms.tgrad_block_norm_backward(s["dx"] if with_dx else None, s["dh"] if with_pre else None, f.x, s["block"], stats=f.stats, **args)

    def back(u, u_size, n, rr, d):
        m = u.mean(1, keepdim=True) if centered else 0.0
        want = rr * (u - n * (u * n).mean(1, keepdim=True) - m)
        size = rr * (u_size + n.abs() * (u_size * n.abs()).mean(1, keepdim=True) + u_size.mean(1, keepdim=True))
        slip = rr * rr * d * ((u_size * n.abs()).mean(1, keepdim=True) + n.abs() * u_size.mean(1, keepdim=True))
        return want, size, slip

    if with_pre:
        want, size, slip = back(dh * pre, (dh * pre).abs(), nx, rx, dx_mean)
        want, size = want + up, size + up.abs()
        off = K * size + slip
    else:
        want, size, off = up, up.abs(), 0 * up
    close(r.dx, want, off, stream)
    dx, dx_off = want, off + 2 * U * size
    u, u_off = scale * dx * gate * post, (scale * gate * post).abs() * dx_off
    if with_post:
        want, size, slip = back(u, u.abs(), nb, rb, db)
        carried = rb * (u_off + nb.abs() * (u_off * nb.abs()).mean(1, keepdim=True) + u_off.mean(1, keepdim=True))
        close(r.dblock, want, K * size + slip + carried, dtype)
        n_off = K * nb.abs() + rb * db
        want = (scale * dx * gate * nb).sum(0)
        size = (scale * dx * gate * nb).abs().sum(0)
        close(r.dpost, want, (rows + 8) * U * size + ((scale * gate).abs() * (dx_off * nb.abs() + dx.abs() * n_off)).sum(0), "f32")
    else:
        close(r.dblock, u, u_off + 4 * U * u.abs(), dtype)
        n_off = 0 * nb
        assert r.dpost is None
    if with_gate:
        each, each_off = scale * dx * nb * post, (scale * post).abs() * (dx_off * nb.abs() + dx.abs() * n_off)
        group = torch.arange(rows) // shared
        add = lambda t: torch.zeros(len(s["gate"]), cols, dtype=torch.float64).index_add_(0, group, t)  # noqa: E731
        close(r.dgate, add(each), add(each_off) + (min(shared, rows) + 8) * U * add(each.abs()), dtype)
    else:
        assert r.dgate is None
    if with_pre:
        close(r.dpre, (dh * nx).sum(0), (rows + 8) * U * (dh * nx).abs().sum(0) + (dh.abs() * (K * nx.abs() + rx * dx_mean)).sum(0), "f32")
    else:
        assert r.dpre is None


SIZES = [(1, 1, 1), (1, 4096, 1), (3, 7, 1), (5, 64, 2), (70, 500, 70), (9, 513, 4), (33, 1537, 11), (40, 2048, 1), (20, 4096, 20), (17, 4100, 5),
         (6, 8192, 6), (5, 8200, 2), (4, 16384, 4), (3, 16400, 3), (5, 32768, 5), (4, 32761, 1)]


@pytest.mark.parametrize("centered", [False, True])
@pytest.mark.parametrize("stream,dtype", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("f32", "f16")])
@pytest.mark.parametrize("rows,cols,shared", SIZES)
def test_forward_and_backward(rows, cols, shared, stream, dtype, centered):
    check(rows, cols, stream, dtype, shared, centered, weights="f32" if cols % 2 else dtype, pad=cols % 3)


@pytest.mark.parametrize("rows,shared", [(2000, 2000), (2500, 1), (2500, 3), (3000, 1000), (2049, 700), (5000, 2), (3000, 10 ** 9)])
@pytest.mark.parametrize("cols", [40, 600])
def test_rows_in_chunks(rows, cols, shared):
    check(rows, cols, "f32", "f32", shared, False)


@pytest.mark.parametrize("parts", [{"with_post": False}, {"with_gate": False}, {"with_pre": False}, {"with_dx": False}, {"with_post": False, "with_gate": False},
                                   {"with_pre": False, "with_post": False}, {"scale": 0.0}, {"scale": -2.5}])
def test_parts(parts):
    check(37, 777, "bf16", "bf16", 9, False, **parts)
    check(37, 776, "f32", "f16", 9, True, **parts)


@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 300), (600, 129), (3, 20000)])
@pytest.mark.parametrize("stream,dtype", [("f32", "f32"), ("bf16", "bf16"), ("f32", "f16")])
def test_a_norm_alone(rows, cols, stream, dtype):
    s = make(rows, cols, stream, dtype)
    f = norms.tgrad_block_norm(s["x"], pre_weight=s["pre"], eps=EPS, dtype=TYPES[dtype][0])
    assert f.x is s["x"]
    n, r, _ = normed(d64(s["x"]), False)
    pre, dh = d64(s["pre"]), d64(s["dh"])
    close(f.h, n * pre, K * (n * pre).abs(), dtype)
    b = norms.tgrad_block_norm_backward(None, s["dh"], s["x"], stats=f.stats, pre_weight=s["pre"])
    g = dh * pre
    close(b.dx, r * (g - n * (g * n).mean(1, keepdim=True)), K * r * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True)), stream)
    close(b.dpre, (dh * n).sum(0), ((rows + 8) * U + K) * (dh * n).abs().sum(0), "f32")
    assert b.dblock is None and b.dgate is None and b.dpost is None


@pytest.mark.parametrize("centered", [False, True])
def test_gradients_are_differences(centered):
    """The change of <dx, x_out> + <dh, h> along random directions, by central differences in float64."""
    rows, cols, shared, scale = 6, 50, 4, 0.6
    s = {k: d64(v) for k, v in make(rows, cols, shared=shared).items()}

    def loss(x, block, gate, post, pre):
        g = gate.repeat_interleave(shared, 0)[:rows]
        y = x + scale * g * normed(block, centered)[0] * post
        return float((s["dx"] * y).sum() + (s["dh"] * (normed(y, centered)[0] * pre)).sum())

    dev = {k: v.float().to(DEV) for k, v in s.items()}
    args = {"post_weight": dev["post"], "gate": dev["gate"], "rows_per_gate": shared, "scale": scale, "pre_weight": dev["pre"], "centered": centered}
    f = norms.tgrad_block_norm(dev["x"], dev["block"], eps=EPS, **args)
    b = norms.tgrad_block_norm_backward(dev["dx"], dev["dh"], f.x, dev["block"], stats=f.stats, **args)
    grads = [d64(t) for t in (b.dx, b.dblock, b.dgate, b.dpost, b.dpre)]
    at = [s[k] for k in ("x", "block", "gate", "post", "pre")]
    g = torch.Generator().manual_seed(3)
    h = 1e-5
    for _ in range(6):
        way = [torch.randn(t.shape, generator=g, dtype=torch.float64) for t in at]
        for i in range(5):
            shifted = lambda e: [t + (e * w if j == i else 0) for j, (t, w) in enumerate(zip(at, way))]  # noqa: E731
            diff = (loss(*shifted(h)) - loss(*shifted(-h))) / (2 * h)
            # h^2 times third derivatives of order 10, and 2 K of the gradient's terms
            assert abs(float((grads[i] * way[i]).sum()) - diff) <= 2 * K * float((grads[i].abs().amax() * way[i].abs()).sum()) * 4 + 1e-8


def test_far_means_and_rows_of_zeros():
    x = torch.randn(5, 1000, generator=torch.Generator().manual_seed(0))
    x[1] += 1000
    x[2] = 0
    x[3] = 4.0
    x = x.to(DEV)
    w = torch.ones(1000, device=DEV)
    f = norms.tgrad_block_norm(x, pre_weight=w, eps=EPS, centered=True)
    n, r, d = normed(d64(x), True)
    close(f.h, n, K * n.abs() + r * d, "f32")
    assert bool(f.h[2:4].eq(0).all())
    assert bool(norms.tgrad_block_norm(x, pre_weight=w).h[2].eq(0).all())


def test_a_nan_stays_in_its_row():
    s = make(9, 300, "bf16", "bf16", 9)
    s["block"][4, 100] = float("nan")
    s["x"][6, 7] = float("inf")
    f = norms.tgrad_block_norm(s["x"], s["block"], post_weight=s["post"], gate=s["gate"], rows_per_gate=9, pre_weight=s["pre"], quantize=True)
    h = act8.tgrad_dequantize(f.h)
    assert h.isnan().any(1).tolist() == [i in (4, 6) for i in range(9)] and bool(f.x[4].isnan().all())


def test_no_rows():
    s = make(0, 64)
    f = norms.tgrad_block_norm(s["x"], s["block"], post_weight=s["post"], gate=s["gate"], pre_weight=s["pre"])
    assert f.x.shape == f.h.shape == (0, 64)
    b = norms.tgrad_block_norm_backward(s["dx"], s["dh"], f.x, s["block"], stats=f.stats, post_weight=s["post"], gate=s["gate"], pre_weight=s["pre"])
    assert b.dx.shape == (0, 64) and bool(b.dpost.eq(0).all()) and bool(b.dpre.eq(0).all())


def test_rows_behind_4_gib():
    stride = (1 << 30) + 8
    s = make(3, 700, "bf16", "bf16", 3)
    far = torch.empty(2 * stride + 700, dtype=torch.bfloat16, device=DEV).as_strided((3, 700), (stride, 1))
    far.copy_(s["x"])
    args = {"post_weight": s["post"], "gate": s["gate"], "rows_per_gate": 3, "pre_weight": s["pre"]}
    f, want = norms.tgrad_block_norm(far, s["block"], **args), norms.tgrad_block_norm(s["x"], s["block"], **args)
    assert torch.equal(f.x, want.x) and torch.equal(f.h, want.h)
    far.copy_(f.x)
    b, c = (norms.tgrad_block_norm_backward(s["dx"], s["dh"], x, s["block"], stats=f.stats, **args) for x in (far, f.x))
    assert all(torch.equal(p, q) for p, q in zip(b, c))


def test_captured_replayed_and_on_another_stream():
    s = make(900, 640, "f32", "bf16", 300)
    args = {"post_weight": s["post"], "gate": s["gate"], "rows_per_gate": 300, "scale": 0.5, "pre_weight": s["pre"]}

    def both(**kw):
        f = norms.tgrad_block_norm(s["x"], s["block"], **args, **kw)
        return (f.x, f.h) + tuple(norms.tgrad_block_norm_backward(s["dx"], s["dh"], f.x, s["block"], stats=f.stats, **args, **kw))

    side = torch.cuda.Stream()
    want = both()
    torch.cuda.synchronize()
    got = both(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for i in range(4):
        s["block"].mul_(1.25)
        graph.replay()
        want = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    s = make(4, 64, "bf16", "bf16", 2)
    f = norms.tgrad_block_norm(s["x"], s["block"], post_weight=s["post"], pre_weight=s["pre"])
    ok = {"post_weight": s["post"], "gate": s["gate"], "rows_per_gate": 2, "pre_weight": s["pre"]}
    wide = torch.zeros(1, 32769, device=DEV)
    norm, back = norms.tgrad_block_norm, norms.tgrad_block_norm_backward
    for call in (lambda: norm(s["x"], s["block"][:3], **ok), lambda: norm(s["x"].half(), s["block"], **ok), lambda: norm(s["x"], s["block"].float(), **ok),
                 lambda: norm(s["x"], s["block"], **{**ok, "rows_per_gate": 0}), lambda: norm(s["x"], s["block"], **{**ok, "rows_per_gate": 1}),
                 lambda: norm(s["x"], s["block"], **{**ok, "post_weight": s["post"][:63]}), lambda: norm(s["x"], s["block"], **{**ok, "pre_weight": s["pre"].half()}),
                 lambda: norm(s["x"], s["block"], **ok, eps=0.0), lambda: norm(s["x"], s["block"], **ok, scale=float("nan")), lambda: norm(s["x"]),
                 lambda: norm(s["x"], post_weight=s["post"], pre_weight=s["pre"]), lambda: norm(s["x"], gate=s["gate"], rows_per_gate=2, pre_weight=s["pre"]),
                 lambda: norm(s["x"], s["block"], quantize=True), lambda: norm(s["x"], s["block"], **ok, dtype=torch.float16),
                 lambda: norm(wide, pre_weight=wide[0]), lambda: norm(s["x"].t(), pre_weight=s["pre"]),
                 lambda: back(s["dx"], None, f.x, s["block"], stats=f.stats, **ok), lambda: back(s["dx"], s["dh"], f.x, s["block"], stats=f.stats[:3], **ok),
                 lambda: back(s["dx"].float(), s["dh"], f.x, s["block"], stats=f.stats, **ok), lambda: back(s["dx"], s["dh"].float(), f.x, s["block"], stats=f.stats, **ok),
                 lambda: back(s["dx"], s["dh"], f.x, stats=f.stats, **ok)):
        with pytest.raises(T.TgradError):
            call()
    torch.cuda.synchronize()
