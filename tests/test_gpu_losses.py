"""Token log-probabilities, the clipped policy loss and the preference loss with their gradients, against their definitions in
float64 on the CPU.

Tolerances.  u = 2^-24 (float32).  An exponent (x - max) log2(e) / T carries 3 roundings, so a term of the sum is off by at most
4 u |log p| of itself, which weighted with the terms is at most 4 u ln(vocab); adding the terms up adds u per addition on the
longest chain, at most vocab / 64 of them (64 lanes at least); the logarithm of the sum, the products and differences of numbers up to the largest
|z| add 4 u |z|.  So |logp error| <= E = 4 u (max |z| + |logp| + ln(vocab) + 4) + u vocab / 64.  A softmax entry is off by p (E + 4 u |log p|), and its
gradient d ([v = y] - p) is then rounded to the type once.
"""
import math

import numpy as np
import pytest
import torch

from paper_2501_02379_amd import losses, tgrad as T

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": (torch.float32, U, 2.0 ** -149), "bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -133),
         "f16": (torch.float16, 2.0 ** -11, 2.0 ** -25)}


def make(rows, vocab, dtype="f32", stride=None, offset=0, spread=3.0, seed=0):
    """Logits as a view with the given row stride and first element, and targets."""
    g = torch.Generator().manual_seed(seed)
    stride = stride or vocab
    flat = torch.empty(offset + rows * stride + 8, dtype=TYPES[dtype][0]).fill_(float("nan"))
    x = flat[offset:offset + rows * stride].view(rows, stride)[:, :vocab] if rows else torch.empty(0, vocab, dtype=TYPES[dtype][0])
    x.copy_((torch.randn(rows, vocab, generator=g) * spread).to(x.dtype))
    y = torch.randint(0, vocab, (rows,), generator=g)
    if rows:
        x[torch.arange(rows), y] += 2.0
    dev = flat.to(DEV)
    return (dev[offset:offset + rows * stride].view(rows, stride)[:, :vocab] if rows else x.to(DEV)), y.to(DEV)


def scores(x, y, temperature=1.0):
    """float64 on the CPU: z, lse, logp; ignored rows have 0."""
    z = x.detach().cpu().double() / float(np.float32(temperature))
    y = y.cpu()
    live = (y >= 0) & (y < x.shape[1])
    lse = torch.logsumexp(z, 1) if len(z) else z.new_zeros(0)
    logp = z.gather(1, torch.where(live, y, 0)[:, None])[:, 0] - lse
    return z, torch.where(live, lse, 0.0), torch.where(live, logp, 0.0), live


def logp_bound(z, logp):
    top = torch.where(torch.isfinite(z) & (z.abs() < 1e6), z.abs(), 0.0).amax(1)
    v = z.shape[1]
    return 4 * U * (top + logp.abs() + math.log(v) + 4) + U * v / 64


def gradient(z, lse, y, d):
    """dlogits in float64 for d = d loss / d z_y - rows with d = 0 are zero - and the softmax."""
    p = (z - lse[:, None]).exp()
    g = -p * d[:, None]
    rows = torch.arange(len(z))
    on = d != 0
    g[rows[on], y.cpu()[on]] += d[on]
    return torch.where(on[:, None], g, 0.0), p


def close_gradient(got, g, p, d, z, logp, y, dtype, d_error=0.0):
    _, u, tiny = TYPES[dtype]
    e = logp_bound(z, logp)[:, None] + 4 * U * torch.where(p > 0, -p.clamp(min=1e-300).log(), 0.0)
    bound = g.abs() * (u + 4 * U) + d.abs()[:, None] * p * e * (1 + u) + tiny + torch.as_tensor(d_error).reshape(-1, 1) * (p + 1e-30)
    at = torch.where((y.cpu() >= 0) & (y.cpu() < z.shape[1]), y.cpu(), 0)[:, None]
    bound.scatter_add_(1, at, (d.abs() * 4 * U + torch.as_tensor(d_error)).reshape(-1, 1).expand(len(z), 1))
    off = (got.cpu().double() - g).abs()
    assert got.dtype == TYPES[dtype][0]
    assert bool((off <= bound).all()), float((off / bound).max())


SHAPES = [(1, 1), (3, 2), (2, 63), (5, 64), (4, 65), (7, 255), (3, 1021), (2, 4096), (3, 4099), (2, 9001), (2, 32768), (2, 50001),
          (1, 131072), (1, 150001), (2, 270001)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_logprobs_and_their_gradient(rows, vocab, dtype):
    x, y = make(rows, vocab, dtype, seed=vocab)
    z, lse, logp, _ = scores(x, y)
    got, got_lse = losses.tgrad_token_logprobs(x, y)
    e = logp_bound(z, logp)
    assert bool(((got.cpu().double() - logp).abs() <= e).all()) and bool(((got_lse.cpu().double() - lse).abs() <= e + U * lse.abs()).all())
    d = torch.linspace(-2, 3, rows)
    dx = losses.tgrad_token_logprobs_backward(x, y, got_lse, d.to(DEV))
    g, p = gradient(z, lse, y, d.double())
    # lse is a rounded float32 here: half an ulp of it is a relative error of every p
    close_gradient(dx, g, p, d.double(), z, logp, y, dtype, d_error=(d.double().abs() * (2 * U * lse.abs() + e)))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("stride,offset", [(1000, 0), (1001, 0), (1001, 1), (1008, 3), (1016, 8), (1000, 5), (4000, 2)])
def test_strides_and_alignments(stride, offset, dtype):
    """Every row starts somewhere else; what lies between the rows is neither read nor written."""
    rows, vocab = 9, 1000
    x, y = make(rows, vocab, dtype, stride, offset, seed=offset)
    z, lse, logp, _ = scores(x, y, 0.7)
    out = torch.full((rows, stride + 2), 7.0, device=DEV, dtype=x.dtype)[:, 1:1 + vocab]
    w = torch.ones(rows, device=DEV)
    r = losses.tgrad_policy_loss(x, y, w, w, logp.float().to(DEV), temperature=0.7, out=out)
    assert r.dlogits is out
    assert bool(((r.logp.cpu().double() - logp).abs() <= logp_bound(z, logp)).all())
    d = -torch.exp(r.logp.cpu().double() - logp.float().double()) / float(np.float32(0.7))
    g, p = gradient(z, lse, y, d)
    close_gradient(out, g, p, d, z, logp, y, dtype, d_error=d.abs() * 16 * U)
    whole = out._base if out._base is not None else out
    whole = torch.as_strided(out, (rows, stride + 2), (stride + 2, 1), 0)
    assert bool((whole[:, 0] == 7).all()) and bool((whole[:, 1 + vocab:] == 7).all())


def policy_reference(x, y, w, adv, old, ref, low, high, beta, temperature):
    z, lse, logp, live = scores(x, y, temperature)
    w, adv, old = w.cpu().double(), adv.cpu().double(), old.cpu().double()
    on = live & (w != 0)
    r = (logp - old).exp()
    low, high = float(np.float32(1) - np.float32(low)), float(np.float32(1) + np.float32(high))
    whole, cut = r * adv, r.clamp(low, high) * adv
    clipped = cut < whole
    pg, slope = -torch.minimum(whole, cut), torch.where(clipped, 0.0, -whole)
    kl = torch.zeros_like(pg)
    if ref is not None:
        q = ref.cpu().double() - logp
        kl = q.expm1() - q
        slope = slope - beta * q.expm1()
    parts = torch.stack([pg + beta * kl, pg, kl, clipped.double()]) * w
    parts = torch.where(on, parts, 0.0)
    return z, lse, torch.where(on, logp, 0.0), torch.where(on, w * slope, 0.0), parts


def policy_inputs(x, y, seed, temperature=1.0, masked=0.3):
    g = torch.Generator().manual_seed(seed + 1000)
    rows = x.shape[0]
    _, _, logp, _ = scores(x, y, temperature)
    ratio = torch.randn(rows, generator=g, dtype=torch.float64) * 0.3
    for edge in (math.log(0.8), math.log(1.25)):                       # off the edges, which rounding would decide
        ratio = torch.where((ratio - edge).abs() < 1e-3, ratio + 0.01, ratio)
    old = (logp - ratio).float().to(DEV)
    ref = (logp + torch.randn(rows, generator=g, dtype=torch.float64) * 0.5).float().to(DEV)
    adv = torch.randn(rows, generator=g).to(DEV)
    w = (torch.rand(rows, generator=g) >= masked).float().to(DEV) / max(1, rows)
    return w, adv, old, ref


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,vocab,temperature,beta", [(1, 1, 1.0, 0.1), (17, 5, 0.5, 0.0), (33, 1021, 1.0, 0.05), (8, 4097, 1.3, 0.2),
                                                         (6, 32768, 0.7, 0.05), (3, 50001, 1.0, 0.05), (3, 131072, 1.0, 0.1), (2, 200003, 1.0, 0.05)])
def test_policy_loss_and_gradient(rows, vocab, temperature, beta, dtype):
    x, y = make(rows, vocab, dtype, stride=vocab + 3, seed=rows)
    w, adv, old, ref = policy_inputs(x, y, rows, temperature)
    scale = 1024.0
    dloss = torch.full((1,), scale, device=DEV)
    z, lse, logp, slope, parts = policy_reference(x, y, w, adv, old, ref, 0.2, 0.25, float(np.float32(beta)), temperature)
    r = losses.tgrad_policy_loss(x, y, w, adv, old, ref, clip_low=0.2, clip_high=0.25, kl_beta=beta, temperature=temperature, dloss=dloss)
    e = logp_bound(z, logp)
    assert bool(((r.logp.cpu().double() - logp).abs() <= e).all())
    wd = w.cpu().double()
    ratio_error = wd * (adv.cpu().double().abs() * 2 + beta * 3) * (e + 8 * U) * 4      # ratios and exp(d) below 4 here
    stats = r.stats.cpu().double()
    assert abs(stats[3] - parts[3].sum()) <= rows * U
    for q in (0, 1, 2):
        scale_q = 3.0 if q == 2 else 1.0
        assert abs(stats[q] - parts[q].sum()) <= scale_q * (ratio_error + wd * 3 * (e + 8 * U) * (q == 2)).sum() + 2 * U * parts[q].abs().sum(), q
    d = slope * scale / float(np.float32(temperature))
    g, p = gradient(z, lse, y, d)
    close_gradient(r.dlogits, g, p, d, z, logp, y, dtype, d_error=ratio_error * scale / temperature + 8 * U * d.abs())
    again = losses.tgrad_policy_loss(x, y, w, adv, old, ref, clip_low=0.2, clip_high=0.25, kl_beta=beta, temperature=temperature, dloss=dloss)
    assert torch.equal(again.stats, r.stats) and torch.equal(again.dlogits, r.dlogits)
    alone = losses.tgrad_policy_loss(x, y, w, adv, old, ref, clip_low=0.2, clip_high=0.25, kl_beta=beta, temperature=temperature, backward=False)
    assert alone.dlogits is None and torch.equal(alone.stats, r.stats) and torch.equal(alone.logp, r.logp)
    inplace = x.clone()
    assert losses.tgrad_policy_loss(inplace, y, w, adv, old, ref, clip_low=0.2, clip_high=0.25, kl_beta=beta, temperature=temperature,
                                    dloss=dloss, out=inplace).dlogits is inplace
    assert torch.equal(inplace, r.dlogits)


@pytest.mark.parametrize("vocab", [37, 5003])
def test_policy_gradient_against_differences(vocab):
    """d loss along random directions, from the float64 loss at both sides (step 1e-4: the third derivative's part is below 1e-7)."""
    rows = 12
    x, y = make(rows, vocab, "f32", seed=3)
    w, adv, old, ref = policy_inputs(x, y, 3)
    r = losses.tgrad_policy_loss(x, y, w, adv, old, ref, clip_low=0.2, clip_high=0.25, kl_beta=0.3)
    g = torch.Generator().manual_seed(9)
    for _ in range(6):
        v = torch.randn(rows, vocab, generator=g, dtype=torch.float64)
        h = 1e-4
        side = [policy_reference(x.cpu().double() + s * h * v, y, w, adv, old, ref, 0.2, 0.25, float(np.float32(0.3)), 1.0)[4][0].sum() for s in (1, -1)]
        slope = float(side[0] - side[1]) / (2 * h)
        got = float((r.dlogits.cpu().double() * v).sum())
        assert abs(got - slope) <= 1e-5 * float((r.dlogits.cpu().double().abs() * v.abs()).sum()) + 1e-6


def test_policy_without_reference_or_kl():
    x, y = make(40, 777, "f32", seed=5)
    w, adv, old, ref = policy_inputs(x, y, 5)
    a = losses.tgrad_policy_loss(x, y, w, adv, old)
    b = losses.tgrad_policy_loss(x, y, w, adv, old, ref, kl_beta=0.0)
    assert float(a.stats[2]) == 0 and float(b.stats[2]) > 0
    assert torch.equal(a.dlogits, b.dlogits) and torch.equal(a.stats[:2], b.stats[:2]) and torch.equal(a.stats[0], a.stats[1])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_ignored_rows_are_not_read(dtype):
    """NaN everywhere in a row of weight 0, or without a target, changes nothing; its gradient is 0."""
    rows, vocab = 16, 2050
    x, y = make(rows, vocab, dtype, seed=6)
    w, adv, old, ref = policy_inputs(x, y, 6, masked=0.0)
    w[3], w[15] = 0, 0
    y[5], y[6], y[7] = -100, vocab, -1
    off = [3, 5, 6, 7, 15]
    want = losses.tgrad_policy_loss(x, y, w, adv, old, ref, kl_beta=0.1)
    start = torch.tensor([0, 4, 8, 12, 16], device=DEV)
    want2 = losses.tgrad_preference_loss(x, y, w, ref, start)
    for t in (x, adv, old, ref):
        t[off] = float("nan")
    y[3] = 1 << 40
    got = losses.tgrad_policy_loss(x, y, w, adv, old, ref, kl_beta=0.1)
    got2 = losses.tgrad_preference_loss(x, y, w, ref, start)
    for a, b in ((want.stats, got.stats), (want.logp, got.logp), (want.dlogits, got.dlogits), (want2.loss, got2.loss),
                 (want2.rewards, got2.rewards), (want2.logp, got2.logp), (want2.dlogits, got2.dlogits)):
        assert torch.equal(a, b) and bool(torch.isfinite(b).all())
    assert not bool(got.dlogits[off].any()) and not bool(got.logp[off].any()) and not bool(got2.dlogits[off].any())
    logp, lse = losses.tgrad_token_logprobs(x, y)
    assert not bool(logp[[3, 5, 6, 7]].any()) and not bool(lse[[3, 5, 6, 7]].any()) and bool(torch.isnan(logp[15]))


def test_all_rows_ignored():
    x, y = make(5, 100, "bf16")
    z = torch.zeros(5, device=DEV)
    r = losses.tgrad_policy_loss(x, y, z, z, z, z, kl_beta=0.1)
    assert not bool(r.stats.any()) and not bool(r.dlogits.any())
    r = losses.tgrad_preference_loss(x, y, z, z, torch.tensor([0, 2, 5], device=DEV))
    assert abs(float(r.loss) - math.log(2)) < 1e-7 and not bool(r.rewards.any()) and not bool(r.dlogits.any())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", [9, 3000, 40000])
def test_barred_entries(vocab, dtype):
    """Entries of -inf, or of the type's lowest value, at the front, at the end and in runs longer than a thread's share."""
    lowest = torch.finfo(TYPES[dtype][0]).min
    for value in (-math.inf, lowest):
        x, y = make(6, vocab, dtype, seed=7)
        x[0, 1:] = value                                       # one entry left
        y[0] = 0
        x[1, : vocab // 2] = value
        y[1] = vocab - 1
        x[2, vocab // 2:] = value
        y[2] = 1
        x[3, ::2] = value
        y[3] = 1
        x[4, 1:vocab - 1] = value
        y[4] = vocab - 1
        z, lse, logp, _ = scores(x, y)
        got, got_lse = losses.tgrad_token_logprobs(x, y)
        assert bool(((got.cpu().double() - logp).abs() <= logp_bound(z, logp)).all())
        w = torch.ones(6, device=DEV)
        r = losses.tgrad_policy_loss(x, y, w, w, got)
        d = -torch.exp(r.logp.cpu().double() - got.cpu().double())
        g, p = gradient(z, lse, y, d)
        close_gradient(r.dlogits, g, p, d, z, logp, y, dtype, d_error=8 * U * d.abs())
    x, y = make(2, vocab, dtype, seed=8)
    x[0] = lowest                                              # all the same: a uniform row
    got, _ = losses.tgrad_token_logprobs(x, y)
    assert abs(float(got[0]) + math.log(vocab)) <= 4 * U * (math.log(vocab) + 4) + U * vocab / 64
    x[0] = -math.inf                                           # nothing may be chosen
    got, _ = losses.tgrad_token_logprobs(x, y)
    assert bool(torch.isnan(got[0])) and bool(torch.isfinite(got[1]))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_a_bad_entry_spoils_its_row_alone(dtype):
    for vocab in (70, 5000, 60001):
        for bad in (math.nan, math.inf):
            for at in (0, 1, vocab // 2, vocab - 1):
                x, y = make(3, vocab, dtype, seed=9)
                w, adv, old, ref = policy_inputs(x, y, 9, masked=0.0)
                fine = losses.tgrad_policy_loss(x, y, w, adv, old, ref)
                x[1, at] = bad
                r = losses.tgrad_policy_loss(x, y, w, adv, old, ref)
                logp, _ = losses.tgrad_token_logprobs(x, y)
                assert bool(torch.isnan(r.logp[1])) and bool(torch.isnan(logp[1])) and bool(torch.isnan(r.stats[0]))
                assert torch.equal(r.dlogits[[0, 2]], fine.dlogits[[0, 2]]) and torch.equal(r.logp[[0, 2]], fine.logp[[0, 2]])
                assert bool(torch.isnan(r.dlogits[1]).all())


def preference_reference(x, y, w, ref, start, beta, smoothing, temperature=1.0):
    z, lse, logp, live = scores(x, y, temperature)
    w, ref, start = w.cpu().double(), ref.cpu().double(), start.cpu().tolist()
    on = live & (w != 0)
    beta, smoothing = float(np.float32(beta)), float(np.float32(smoothing))
    gap = torch.where(on, w * (logp - ref), 0.0)
    pairs = len(start) // 2
    seq = [(max(0, min(a, len(w))), max(0, min(b, len(w)))) for a, b in zip(start, start[1:])]
    rewards = torch.stack([beta * gap[a:b].sum() if b > a else torch.zeros((), dtype=torch.float64) for a, b in seq])
    h = rewards[:pairs] - rewards[pairs:]
    loss = -((1 - smoothing) * torch.nn.functional.logsigmoid(h) + smoothing * torch.nn.functional.logsigmoid(-h)).mean()
    dh = beta * (smoothing * torch.sigmoid(h) - (1 - smoothing) * torch.sigmoid(-h)) / pairs
    slope = torch.zeros_like(w)
    for i, (a, b) in enumerate(seq):
        if b > a:
            slope[a:b] = (dh[i] if i < pairs else -dh[i - pairs]) * w[a:b]
    return z, lse, torch.where(on, logp, 0.0), torch.where(on, slope, 0.0), loss, rewards


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("lengths,vocab,beta,smoothing", [
    ([1, 1], 11, 0.1, 0.0), ([5, 0, 7, 3], 1021, 0.5, 0.1), ([0, 0], 64, 0.1, 0.0), ([3, 300, 1, 2, 40, 0], 515, 0.1, 0.05),
    ([4, 6], 70001, 2.0, 0.0), ([2, 2, 2, 2], 32768, 40.0, 0.25)])
def test_preference_loss_and_gradient(lengths, vocab, beta, smoothing, dtype):
    rows = sum(lengths)
    x, y = make(rows, vocab, dtype, stride=vocab + 5, seed=rows)
    g = torch.Generator().manual_seed(rows)
    w = (torch.rand(rows, generator=g) < 0.7).float() * torch.rand(rows, generator=g)
    ref = (scores(x, y)[2] + 0.3 * torch.randn(rows, generator=g, dtype=torch.float64)).float()
    start = torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], device=DEV)
    dloss = torch.full((1,), 256.0, device=DEV)
    r = losses.tgrad_preference_loss(x, y, w.to(DEV), ref.to(DEV), start, beta=beta, label_smoothing=smoothing, dloss=dloss)
    z, lse, logp, slope, loss, rewards = preference_reference(x, y, w, ref, start, beta, smoothing)
    e = logp_bound(z, logp) if rows else logp
    assert bool(((r.logp.cpu().double() - logp).abs() <= e).all())
    off = beta * torch.stack([(w.double() * e)[a:b].sum() for a, b in zip(start.tolist(), start.tolist()[1:])])
    assert bool(((r.rewards.cpu().double() - rewards).abs() <= off + 2 * U * rewards.abs()).all())
    pairs = len(lengths) // 2
    h_off = (off[:pairs] + off[pairs:])
    assert abs(float(r.loss) - float(loss)) <= float(h_off.mean()) + 4 * U * abs(float(loss))
    if rows:
        d = slope * 256.0
        gr, p = gradient(z, lse, y, d)
        d_off = 256.0 * beta * w.double() * float(h_off.max()) + 8 * U * d.abs()
        close_gradient(r.dlogits, gr, p, d, z, logp, y, dtype, d_error=d_off)
    alone = losses.tgrad_preference_loss(x, y, w.to(DEV), ref.to(DEV), start, beta=beta, label_smoothing=smoothing, backward=False)
    assert alone.dlogits is None and torch.equal(alone.loss, r.loss) and torch.equal(alone.rewards, r.rewards)
    if rows:
        inplace = x.clone()
        losses.tgrad_preference_loss(inplace, y, w.to(DEV), ref.to(DEV), start, beta=beta, label_smoothing=smoothing, dloss=dloss, out=inplace)
        assert torch.equal(inplace, r.dlogits)


def test_preference_gradient_against_differences():
    lengths, vocab = [4, 9, 6, 2], 300
    rows = sum(lengths)
    x, y = make(rows, vocab, "f32", seed=21)
    g = torch.Generator().manual_seed(21)
    w, ref = torch.rand(rows, generator=g), scores(x, y)[2].float()
    start = torch.tensor([0, 4, 13, 19, 21], device=DEV)
    r = losses.tgrad_preference_loss(x, y, w.to(DEV), ref.to(DEV), start, beta=0.7, label_smoothing=0.1)
    for _ in range(6):
        v = torch.randn(rows, vocab, generator=g, dtype=torch.float64)
        h = 1e-4
        side = [preference_reference(x.cpu().double() + s * h * v, y, w, ref, start, 0.7, 0.1)[4] for s in (1, -1)]
        got = r.dlogits.cpu().double()
        assert abs(float((got * v).sum()) - float(side[0] - side[1]) / (2 * h)) <= 1e-5 * float((got.abs() * v.abs()).sum()) + 1e-6


def test_sequence_bounds_outside_the_rows():
    """Bounds are taken as the nearest inside; rows before, between and behind the sequences have no gradient."""
    x, y = make(20, 130, "f32", seed=30)
    w, ref = torch.ones(20, device=DEV), scores(x, y)[2].float().to(DEV) + 0.2
    start = torch.tensor([-7, 5, 5, 11, 1 << 40], device=DEV)
    r = losses.tgrad_preference_loss(x, y, w, ref, start)
    same = losses.tgrad_preference_loss(x, y, w, ref, torch.tensor([0, 5, 5, 11, 20], device=DEV))
    assert torch.equal(r.loss, same.loss) and torch.equal(r.dlogits, same.dlogits) and torch.equal(r.rewards, same.rewards)
    part = losses.tgrad_preference_loss(x, y, w, ref, torch.tensor([4, 8, 15], device=DEV))
    assert not bool(part.dlogits[:4].any()) and not bool(part.dlogits[15:].any()) and bool(part.dlogits[4:15].any(1).all())


def test_no_rows():
    x = torch.empty(0, 50, device=DEV)
    y, z = torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV)
    assert losses.tgrad_token_logprobs(x, y)[0].shape == (0,)
    r = losses.tgrad_policy_loss(x, y, z, z, z)
    assert not bool(r.stats.any()) and r.dlogits.shape == (0, 50)
    r = losses.tgrad_preference_loss(x, y, z, z, torch.zeros(3, dtype=torch.int64, device=DEV))
    assert abs(float(r.loss) - math.log(2)) < 1e-7


def test_rows_beyond_32_bit_offsets():
    """Row starts past 2^31 elements, and past 2^32 bytes."""
    rows, vocab, stride = 70, 3001, (1 << 25) + 3
    flat = torch.zeros(rows * stride, dtype=torch.bfloat16, device=DEV)
    x = flat.view(rows, stride)[:, :vocab]
    small, y = make(rows, vocab, "bf16", seed=40)
    x.copy_(small)
    w, adv, old, ref = policy_inputs(small, y, 40)
    a = losses.tgrad_policy_loss(x, y, w, adv, old, ref, kl_beta=0.1, out=x)
    b = losses.tgrad_policy_loss(small, y, w, adv, old, ref, kl_beta=0.1)
    assert torch.equal(a.stats, b.stats) and torch.equal(a.dlogits, b.dlogits)


def test_another_stream():
    x, y = make(300, 20001, "bf16", seed=50)
    w, adv, old, ref = policy_inputs(x, y, 50)
    want = losses.tgrad_policy_loss(x, y, w, adv, old, ref, kl_beta=0.1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [losses.tgrad_policy_loss(x, y, w, adv, old, ref, kl_beta=0.1, stream=side) for _ in range(4)]
    torch.cuda.current_stream().wait_stream(side)
    for r in got:
        assert torch.equal(r.stats, want.stats) and torch.equal(r.dlogits, want.dlogits)


def test_graph_replays():
    """Both losses inside a captured graph: every replay, with eager work in between and new inputs, as the eager call."""
    x, y = make(64, 5003, "bf16", seed=60)
    w, adv, old, ref = policy_inputs(x, y, 60)
    start = torch.tensor([0, 20, 30, 40, 64], device=DEV)

    def both():
        return losses.tgrad_policy_loss(x, y, w, adv, old, ref, kl_beta=0.1), losses.tgrad_preference_loss(x, y, w, ref, start)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p, q = both()
    for k in range(4):
        x.copy_(make(64, 5003, "bf16", seed=61 + k)[0])
        graph.replay()
        torch.cuda.synchronize()
        pe, qe = both()
        assert torch.equal(p.stats, pe.stats) and torch.equal(p.dlogits, pe.dlogits)
        assert torch.equal(q.loss, qe.loss) and torch.equal(q.dlogits, qe.dlogits) and torch.equal(q.rewards, qe.rewards)


def test_the_bindings_refuse():
    x, y = make(4, 10, "f32")
    w = torch.zeros(4, device=DEV)
    for bad in (lambda: losses.tgrad_token_logprobs(x.double(), y), lambda: losses.tgrad_token_logprobs(x.t(), y),
                lambda: losses.tgrad_token_logprobs(x, y.int()), lambda: losses.tgrad_token_logprobs(x, y[:3]),
                lambda: losses.tgrad_token_logprobs(x, y, temperature=0.0), lambda: losses.tgrad_token_logprobs(x[0], y),
                lambda: losses.tgrad_policy_loss(x, y, w.double(), w, w), lambda: losses.tgrad_policy_loss(x, y, w.cpu(), w, w),
                lambda: losses.tgrad_policy_loss(x, y, w, w, w, clip_low=1.5),
                lambda: losses.tgrad_policy_loss(x, y, w, w, w, out=torch.empty(4, 11, device=DEV)),
                lambda: losses.tgrad_preference_loss(x, y, w, w, torch.zeros(4, dtype=torch.int64, device=DEV)),
                lambda: losses.tgrad_preference_loss(x, y, w, w, torch.zeros(3, dtype=torch.int64, device=DEV), beta=0.0)):
        with pytest.raises(T.TgradError):
            bad()


def test_more_rows_than_one_launch_takes():
    """2^26 + 300 rows of three numbers: a wavefront each is more than 2^32 threads."""
    rows, vocab = (1 << 26) + 300, 3
    x = torch.zeros(rows, vocab, dtype=torch.float16, device=DEV)
    y = torch.full((rows,), -100, device=DEV)
    live = torch.tensor([0, 1, (1 << 26) - 2, (1 << 26) - 1, 1 << 26, rows - 1])
    y[live.to(DEV)] = 1
    x[live.to(DEV)] = torch.tensor([0.0, 1.0, -1.0], dtype=torch.float16, device=DEV)
    logp, _ = losses.tgrad_token_logprobs(x, y)
    want = 1.0 - math.log(math.exp(0.0) + math.exp(1.0) + math.exp(-1.0))
    assert int(torch.count_nonzero(logp)) == len(live) and bool(((logp[live.to(DEV)] - want).abs() < 1e-6).all())
    ones = torch.ones(rows, device=DEV)
    r = losses.tgrad_policy_loss(x, y, ones, ones, logp)
    assert abs(float(r.stats[0]) + len(live)) < 1e-5
    p = torch.softmax(x[live.to(DEV)].double(), 1).cpu()
    p[:, 1] -= 1
    assert bool(((r.dlogits[live.to(DEV)].double().cpu() - p).abs() < 1e-3).all())
    assert int(torch.count_nonzero(r.dlogits)) == 3 * len(live)
    start = torch.tensor([0, 2, rows], device=DEV)
    q = losses.tgrad_preference_loss(x, y, ones, torch.zeros_like(logp), start)
    assert int(torch.count_nonzero(q.dlogits)) == 3 * len(live)
    assert bool((torch.sign(q.dlogits[live.to(DEV), 1]).cpu() == torch.tensor([-1, -1, 1, 1, 1, 1])).all())


@pytest.mark.parametrize("temperature", [1.0, 0.01])
@pytest.mark.parametrize("offset", [300.0, -5000.0, 30000.0, -60000.0, 3e6, -3e6, 1e30, -1e30, 3e38])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_far_from_zero(dtype, offset, temperature):
    """Only differences within a row count, wherever the row lies: entries equal to the offset, one step of the type below it, and
    far below.  In the bounds |z| is then the distance to the row's maximum, of entries that are not negligible."""
    if dtype == "f16" and abs(offset) > 65000:
        pytest.skip("beyond float16")
    for vocab in (50, 3001, 20002):
        g = torch.Generator().manual_seed(vocab)
        top = torch.tensor(offset).to(TYPES[dtype][0])
        low = torch.tensor(-math.inf).to(top.dtype)
        below = torch.nextafter(top, low) if dtype != "bf16" else (top.double() * (1 - math.copysign(2.0 ** -7, offset))).to(top.dtype)
        pick = torch.randint(0, 3, (4, vocab), generator=g)
        x = torch.where(pick == 0, top, torch.where(pick == 1, below, (below.double() - abs(float(below)) * 0.1).to(top.dtype)))
        x = torch.where(torch.isfinite(x), x, below)
        y = torch.randint(0, vocab, (4,), generator=g)
        x[torch.arange(4), y] = top
        shift = x.double().amax(1, keepdim=True)                        # the reference too, relative to the maximum
        xs = x.double() - shift
        z, lse, logp, _ = scores(xs, y, temperature)
        lse = lse + shift[:, 0] / float(np.float32(temperature))
        near = torch.clamp(z, min=-200)
        e = logp_bound(near, logp)
        xd, yd = x.to(DEV), y.to(DEV)
        got, got_lse = losses.tgrad_token_logprobs(xd, yd, temperature=temperature)
        assert bool(((got.cpu().double() - logp).abs() <= e).all())
        if float(lse.abs().max()) < 3.4e38:                            # a float32 holds it
            assert bool(((got_lse.cpu().double() - lse).abs() <= e + 4 * U * lse.abs()).all())
        w = torch.ones(4, device=DEV)
        r = losses.tgrad_policy_loss(xd, yd, w, w, got, temperature=temperature)
        d = -torch.exp(r.logp.cpu().double() - got.cpu().double()) / float(np.float32(temperature))
        gr, p = gradient(near, torch.logsumexp(near, 1), y, d)
        close_gradient(r.dlogits, gr, p, d, near, logp, y, dtype, d_error=8 * U * d.abs())
        start = torch.tensor([0, 2, 4], device=DEV)
        q = losses.tgrad_preference_loss(xd, yd, w, (logp - 0.3).float().to(DEV), start, temperature=temperature)
        assert bool(((q.logp.cpu().double() - logp).abs() <= e).all()) and bool(((r.logp.cpu().double() - logp).abs() <= e).all())
        s = preference_reference(xs, y, w, (logp - 0.3).float(), start, 0.1, 0.0, temperature)[3] / float(np.float32(temperature))
        gr, p = gradient(near, torch.logsumexp(near, 1), y, s)
        close_gradient(q.dlogits, gr, p, s, near, logp, y, dtype, d_error=s.abs() * (8 * U + 0.4 * float(e.max())))
        inplace = xd.clone()
        losses.tgrad_policy_loss(inplace, yd, w, w, got, temperature=temperature, out=inplace)
        assert torch.equal(inplace, r.dlogits)


def test_loss_scale_of_any_dimension():
    x, y = make(12, 300, "bf16", seed=9)
    w, adv, old, ref = policy_inputs(x, y, 9)
    start = torch.tensor([0, 5, 12], device=DEV)
    scale = torch.full((1,), 8.0, device=DEV)
    for s in (scale[0], scale.reshape(1, 1)):
        assert torch.equal(losses.tgrad_policy_loss(x, y, w, adv, old, ref, dloss=scale).dlogits,
                           losses.tgrad_policy_loss(x, y, w, adv, old, ref, dloss=s).dlogits)
        assert torch.equal(losses.tgrad_preference_loss(x, y, w, ref, start, dloss=scale).dlogits,
                           losses.tgrad_preference_loss(x, y, w, ref, start, dloss=s).dlogits)
    for s in (torch.ones(2, device=DEV), torch.ones((), dtype=torch.float64, device=DEV), torch.ones(())):
        with pytest.raises(T.TgradError):
            losses.tgrad_policy_loss(x, y, w, adv, old, ref, dloss=s)
