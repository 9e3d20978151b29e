"""The operators of a training step around `tgrad_step`, as measurable cases.

`logprobs` scores given tokens (the old and the reference policy of a fine-tuning step, single tokens too), `policy` is the
clipped policy loss with a KL term and its gradient with respect to the logits, `preference` the loss on paired log ratios and
its gradient, `clip` the global norm over all gradients of a model and the clipped gradients, `step` the global norm and an
AdamW step of all parameters under the clip factor.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "c64": 8}
CLIP_LOW, CLIP_HIGH, KL_BETA, PAIR_BETA, SMOOTHING = 0.2, 0.28, 0.05, 0.1, 0.05
LR, BETA1, BETA2, EPS, DECAY, DONE = 3e-4, 0.9, 0.95, 1e-8, 0.1, 1203     # DONE: optimizer steps behind the state
MOST = 8192 * 131072                                                      # logits of the largest case


def _rows(name, op, rows, vocab, dtype, stride=None, masked=0.0, barred=0, temperature=1.0, kl=True):
    """rows x vocab logits, `stride` elements from row to row; a share of the rows is a prompt's or padding (`masked`), the last
    `barred` entries of the vocabulary may not be chosen (their logits are -inf)."""
    c = {"op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "stride": stride or vocab, "masked": masked, "barred": barred,
         "temperature": temperature, "kl": kl}
    return {**c, "name": name} if name else c


def _pairs(name, pairs, tokens, vocab, dtype, masked=0.3, barred=0, loss_scale=1.0, empty=False):
    """`pairs` answers chosen and rejected, of up to `tokens` tokens each; `empty`: one rejected answer has none."""
    c = {"op": "preference", "pairs": pairs, "tokens": tokens, "vocab": vocab, "dtype": dtype, "masked": masked, "barred": barred,
         "loss_scale": loss_scale, "empty": empty}
    return {**c, "name": name} if name else c


def _model(name, op, model, width, layers, other, grad, param="f32", packed=False, bound=1.0):
    """Parameters of `model`: "fno" (width channels, other x (other / 2 + 1) modes) or "tokens" (width, vocabulary of `other`).
    packed: the tensors lie end to end in one buffer, with no alignment (gradient buckets)."""
    c = {"op": op, "model": model, "width": width, "layers": layers, "other": other, "grad": grad, "param": param, "packed": packed,
         "bound": bound}
    return {**c, "name": name} if name else c


def listed():
    return [
        # one position of 8 sequences scored while they are written: latency
        _rows("logprobs_decode", "logprobs", 8, 65536, "bf16"),
        # the reference policy's scores of a rollout
        _rows("logprobs_rollout", "logprobs", 4096, 131072, "bf16", masked=0.25),
        # byte-like vocabulary, a few short answers: latency of loss and gradient, odd rows
        _rows("policy_small", "policy", 61, 1021, "f32", masked=0.2),
        # ordinary: odd vocabulary in rows padded to a multiple of 64, entries barred, sampled at a temperature
        _rows("policy_ordinary", "policy", 2048, 50001, "bf16", stride=50048, masked=0.25, barred=33, temperature=0.7),
        # single precision, rows longer than a compute unit can hold
        _rows("policy_wide_f32", "policy", 1024, 200003, "f32", masked=0.1, kl=False),
        # the largest
        _rows("policy_large", "policy", 8192, 131072, "bf16", masked=0.25),
        # ordinary preference batch
        _pairs("preference_ordinary", 16, 160, 32768, "bf16"),
        # half precision under a loss scale, ragged answers, odd vocabulary, an empty answer
        _pairs("preference_f16", 8, 700, 100003, "f16", barred=5, loss_scale=65536.0, empty=True),
        # the small FNO's gradients: latency
        _model("clip_small", "clip", "fno", 16, 4, 8, "f32"),
        # a layer of 128 channels and 128 x 65 modes with the rest of the model, complex gradients
        _model("clip_fno", "clip", "fno", 128, 1, 128, "f32"),
        # AdamW of a small FNO, every tensor dense
        _model("step_small", "step", "fno", 32, 4, 12, "f32"),
        # AdamW of a language model: bf16 gradient buckets packed end to end, float32 parameters
        _model("step_tokens", "step", "tokens", 2048, 8, 32768, "bf16", packed=True),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["logprobs", "policy", "policy", "preference", "clip", "step"])
    if op in ("logprobs", "policy"):
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        vocab = _log(rng, 300, 200000)
        rows = _log(rng, 1, min(16384, MOST // (vocab * (2 if dtype == "f32" else 1))))
        stride = vocab if rng.random() < 0.6 else vocab + rng.choice([1, 7, 64])
        return _rows(None, op, rows, vocab, dtype, stride, rng.choice([0.0, 0.2, 0.5]), rng.choice([0, 0, vocab // 50]),
                     rng.choice([1.0, 1.0, 0.7, 1.3]), rng.random() < 0.7)
    if op == "preference":
        vocab = _log(rng, 300, 200000)
        tokens = _log(rng, 8, 1500)
        pairs = _log(rng, 1, max(1, min(64, MOST // (4 * vocab * tokens))))
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        return _pairs(None, pairs, tokens, vocab, dtype, rng.choice([0.1, 0.3, 0.5]), rng.choice([0, vocab // 50]),
                      65536.0 if dtype == "f16" else 1.0, rng.random() < 0.3)
    if rng.random() < 0.5:
        return _model(None, op, "fno", rng.choice([16, 24, 32, 48, 64, 90]), rng.randint(1, 5), _log(rng, 4, 48), "f32",
                      packed=rng.random() < 0.4, bound=rng.choice([1.0, 1e6]))
    return _model(None, op, "tokens", 8 * _log(rng, 8, 160), rng.randint(1, 8), _log(rng, 500, 40000),
                  rng.choice(["bf16", "f16", "f32"]), rng.choice(["f32", "f32", "bf16"]), rng.random() < 0.5, rng.choice([1.0, 1e6]))


# ---- inputs ---------------------------------------------------------------------------------------------------------------

def _lengths(case):
    """Tokens of every answer, the chosen ones first: a property of the case, not of the seed."""
    r = random.Random("%(pairs)d %(tokens)d %(vocab)d" % case)
    n = [r.randint(max(1, case["tokens"] // 3), case["tokens"]) for _ in range(2 * case["pairs"])]
    if case["empty"]:
        n[-1] = 0
    return n


def _row_count(case):
    return case["rows"] if "rows" in case else sum(_lengths(case))


def _masked_count(case):
    if "rows" in case:
        return int(case["rows"] * case["masked"])
    return sum(int(n * case["masked"]) for n in _lengths(case))


def _logits(case, rows, gen):
    """Logits with the given token likely, as a model in training has them, and the tokens."""
    vocab, stride = case["vocab"], case.get("stride", case["vocab"])
    x = torch.randn(rows, stride, device=DEV, dtype=TYPES[case["dtype"]], generator=gen).mul_(2.0)
    live = vocab - case["barred"]
    y = torch.randint(0, live, (rows,), device=DEV, generator=gen)
    at = torch.arange(rows, device=DEV)
    x[at, y] += 8.0 + 2.0 * torch.randn(rows, device=DEV, generator=gen).to(x.dtype)
    x = x[:, :vocab]
    if case["barred"]:
        x[:, live:] = -math.inf
    return x, y


def _scores(x, y, temperature):
    """Log-probabilities of y in float32, a block of rows at a time."""
    got = torch.empty(x.shape[0], device=DEV)
    for a in range(0, x.shape[0], 512):
        z = x[a:a + 512].float() / temperature
        got[a:a + 512] = z.gather(1, y[a:a + 512, None])[:, 0] - torch.logsumexp(z, 1)
    return got


def _beside(log_ratio):
    """Log ratios moved off the two places where clipping sets in, which rounding would decide."""
    for edge in (math.log1p(-CLIP_LOW), math.log1p(CLIP_HIGH)):
        log_ratio = torch.where((log_ratio - edge).abs() < 1e-3, log_ratio + 4e-3, log_ratio)
    return log_ratio


def _shapes(case):
    """(shape, complex, decays) of every parameter."""
    w, other = case["width"], case["other"]
    if case["model"] == "fno":
        s = [((3, 2 * w), False, True), ((2 * w,), False, False), ((2 * w, w), False, True), ((w,), False, False)]
        for _ in range(case["layers"]):
            s += [((w, w, other, other // 2 + 1), True, False), ((w, w), False, True), ((w,), False, False)]
        return s + [((w, 2 * w), False, True), ((2 * w,), False, False), ((2 * w, 1), False, True), ((1,), False, False)]
    s = [((other, w), False, True)]
    for _ in range(case["layers"]):
        s += [((w,), False, False), ((3 * w, w), False, True), ((w, w), False, True), ((w,), False, False),
              ((2 * (11 * w // 4), w), False, True), ((w, 11 * w // 4), False, True)]
    return s + [((w,), False, False)]


def _places(case):
    """The tensors by buffer: {(complex, decays): ([(offset, shape)], elements)}."""
    by = {}
    for shape, cplx, decays in _shapes(case):
        places, end = by.setdefault((cplx, decays), ([], 0))
        places.append((end, shape))
        n = math.prod(shape)
        by[(cplx, decays)] = (places, end + (n if case["packed"] else -(-n // 64) * 64))
    return by


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": case}
    if case["op"] in ("clip", "step"):
        s["flats"] = []
        for (cplx, decays), (places, n) in _places(case).items():
            kind = torch.complex64 if cplx else TYPES[case["grad"]]
            f = {"decay": DECAY if decays else 0.0, "complex": cplx, "places": places}
            f["grad"] = torch.randn(n, device=DEV, dtype=kind, generator=gen).mul_(2e-3)
            f["grad"][::97] *= 20.0
            if case["op"] == "clip":
                f["out"] = torch.zeros_like(f["grad"])
            else:
                real = torch.complex64 if cplx else torch.float32
                f["param"] = torch.randn(n, device=DEV, dtype=real, generator=gen).mul_(0.02)
                f["param"] = f["param"] if cplx else f["param"].to(TYPES[case["param"]])
                f["exp_avg"] = torch.randn(n, device=DEV, dtype=real, generator=gen).mul_(5e-4)
                f["exp_avg_sq"] = torch.randn(n, device=DEV, generator=gen).mul_(1e-3).square_().add_(1e-8)
            ends = [at + math.prod(shape) for at, shape in places]
            for end, after in zip(ends, [at for at, _ in places[1:]] + [n]):        # nothing lies between the tensors
                for k in ("grad", "param", "exp_avg", "exp_avg_sq"):
                    if k in f and after > end:
                        f[k][end:after] = 0
            s["flats"].append(f)
        return s
    rows = _row_count(case)
    s["logits"], s["targets"] = _logits(case, rows, gen)
    if case["op"] == "preference":
        n = _lengths(case)
        s["start"] = torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], device=DEV)
        s["weight"] = torch.cat([(torch.arange(k) >= int(k * case["masked"])).float() for k in n]).to(DEV)
        s["dloss"] = torch.full((1,), case["loss_scale"], device=DEV)
        s["ref_logp"] = _scores(s["logits"], s["targets"], 1.0) + 0.2 * torch.randn(rows, device=DEV, generator=gen)
        return s
    off = torch.randperm(rows, device=DEV, generator=gen)[:_masked_count(case)]
    if case["op"] == "logprobs":
        s["targets"][off] = -100
        return s
    logp = _scores(s["logits"], s["targets"], case["temperature"])
    s["old_logp"] = logp - _beside(0.2 * torch.randn(rows, device=DEV, generator=gen))
    s["ref_logp"] = logp + 0.3 * torch.randn(rows, device=DEV, generator=gen) if case["kl"] else None
    s["advantage"] = torch.randn(rows, device=DEV, generator=gen)
    s["weight"] = torch.full((rows,), 1.0 / max(1, rows - len(off)), device=DEV)
    s["weight"][off] = 0.0
    return s


def work(case):
    if case["op"] in ("clip", "step"):
        b = f = 0
        for (cplx, _), (places, _) in _places(case).items():
            n = sum(math.prod(shape) for _, shape in places)
            g = 8 if cplx else BYTES[case["grad"]]
            if case["op"] == "clip":
                b, f = b + 2 * g * n, f + (6 if cplx else 3) * n
            else:
                p = 8 if cplx else BYTES[case["param"]]
                b, f = b + (g + 2 * p + (24 if cplx else 16)) * n, f + (30 if cplx else 17) * n
        return {"bytes": b, "flops": f}
    rows = _row_count(case)
    read = (rows - _masked_count(case)) * case["vocab"]
    size = BYTES[case["dtype"]]
    if case["op"] == "logprobs":
        return {"bytes": read * size + rows * 16, "flops": 5 * read}
    return {"bytes": (read + rows * case["vocab"]) * size + rows * 28, "flops": 9 * read}


# ---- the operators in elementary torch operations -------------------------------------------------------------------------

def _plain_logprobs(x, y, temperature):
    live = (y >= 0) & (y < x.shape[1])
    z = x.float() / temperature
    top = z.amax(1, keepdim=True)
    lse = (z - top).exp().sum(1).log() + top[:, 0]
    logp = z.gather(1, torch.where(live, y, 0)[:, None])[:, 0] - lse
    return z, torch.where(live, logp, 0.0), torch.where(live, lse, 0.0)


def _plain_gradient(z, lse, y, dlogp, temperature, dtype):
    d = dlogp / temperature
    g = (z - lse[:, None]).exp_().mul_(-d[:, None])
    g[torch.arange(len(y), device=z.device), y] += d
    return torch.where((dlogp != 0)[:, None], g, 0.0).to(dtype)


def _plain_policy(s):
    c = s["case"]
    z, logp, lse = _plain_logprobs(s["logits"], s["targets"], c["temperature"])
    w, a = s["weight"], s["advantage"]
    used = w != 0
    r = (logp - s["old_logp"]).exp()
    whole, cut = r * a, r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a
    pg, clipped = -torch.minimum(whole, cut), cut < whole
    dlogp = torch.where(clipped, 0.0, -whole)
    kl = torch.zeros_like(pg)
    if s["ref_logp"] is not None:
        d = s["ref_logp"] - logp
        kl = d.expm1() - d
        dlogp = dlogp - KL_BETA * d.expm1()
    each = torch.stack([pg + KL_BETA * kl, pg, kl, clipped.float()]) * w
    stats = torch.where(used, each, 0.0).sum(1)
    dlogits = _plain_gradient(z, lse, s["targets"], torch.where(used, w * dlogp, 0.0), c["temperature"], s["logits"].dtype)
    return {"stats": stats, "logp": torch.where(used, logp, 0.0), "dlogits": dlogits}


def _softplus(x):
    return x.clamp(min=0) + (-x.abs()).exp().log1p()


def _sums(v, start):
    c = torch.cat([v.new_zeros(1, dtype=torch.float64), v.double().cumsum(0)])
    return (c[start[1:]] - c[start[:-1]]).to(v.dtype)


def _preference_tail(s, logp):
    """Loss, rewards and the gradient of every log-probability, in logp's precision."""
    w, start, pairs = s["weight"].to(logp.dtype), s["start"], s["case"]["pairs"]
    reward = PAIR_BETA * _sums(torch.where(w != 0, w * (logp - s["ref_logp"].to(logp.dtype)), 0.0), start)
    h = reward[:pairs] - reward[pairs:]
    loss = ((1 - SMOOTHING) * _softplus(-h) + SMOOTHING * _softplus(h)).mean()
    dh = PAIR_BETA * (SMOOTHING / (1 + (-h).exp()) - (1 - SMOOTHING) / (1 + h.exp())) / pairs * s["dloss"].to(logp.dtype)
    of = torch.searchsorted(start, torch.arange(len(w), device=w.device), right=True) - 1
    return loss, reward, w * torch.cat([dh, -dh])[of]


def _plain_preference(s):
    z, logp, lse = _plain_logprobs(s["logits"], s["targets"], 1.0)
    loss, reward, dlogp = _preference_tail(s, logp)
    dlogits = _plain_gradient(z, lse, s["targets"], dlogp, 1.0, s["logits"].dtype)
    return {"loss": loss, "rewards": reward, "logp": torch.where(s["weight"] != 0, logp, 0.0), "dlogits": dlogits}


def _real(x):
    return torch.view_as_real(x) if x.is_complex() else x


def _plain_norm(flats, bound):
    norm = torch.stack([_real(f["grad"]).float().square().sum() for f in flats]).sum().sqrt()
    return norm, (bound / (norm + 1e-6)).clamp(max=1.0)


def _plain_clip(s):
    norm, coef = _plain_norm(s["flats"], s["case"]["bound"])
    return {"norm": norm, "grads": [f["out"].copy_((f["grad"] if f["complex"] else f["grad"].float()) * coef) for f in s["flats"]]}


def _plain_adamw(f, coef):
    g = _real(f["grad"]).float() * coef
    m, v, p = _real(f["exp_avg"]), f["exp_avg_sq"], _real(f["param"])
    m.mul_(BETA1).add_(g * (1 - BETA1))
    v.mul_(BETA2).add_((g.square().sum(-1) if f["complex"] else g.square()) * (1 - BETA2))
    size = (v / (1 - BETA2 ** (DONE + 1))).sqrt() + EPS
    move = m / (1 - BETA1 ** (DONE + 1)) / (size[:, None] if f["complex"] else size)
    p.copy_(p.float() * (1 - LR * f["decay"]) - LR * move)
    return f["param"], f["exp_avg"], f["exp_avg_sq"]


def _plain_step(s):
    norm, coef = _plain_norm(s["flats"], s["case"]["bound"])
    return {"norm": norm, "state": [_plain_adamw(f, coef) for f in s["flats"]]}


# ---- this library's operators -----------------------------------------------------------------------------------------------

def _own_group(s):
    """The group of a model's tensors, which a training program keeps from step to step."""
    if "group" not in s:
        from paper_2501_02379_amd import group
        names = ("grad", "out") if s["case"]["op"] == "clip" else ("grad", "param", "exp_avg", "exp_avg_sq")
        every = [(f, at, shape) for f in s["flats"] for at, shape in f["places"]]
        views = {k: [f[k][at:at + math.prod(shape)].view(shape) for f, at, shape in every] for k in names}
        s["group"] = group.Group(views["grad"], params=views.get("param"), exp_avg=views.get("exp_avg"),
                                 exp_avg_sq=views.get("exp_avg_sq"), outs=views.get("out"),
                                 weight_decay=[f["decay"] for f, _, _ in every])
    return s["group"]


def _own(s):
    c = s["case"]
    if c["op"] == "clip":
        norm = _own_group(s).tgrad_group_clip(c["bound"])
        return {"norm": norm[0], "grads": [f["out"] for f in s["flats"]]}
    if c["op"] == "step":
        g = _own_group(s)
        norm = g.tgrad_group_grad_norm(c["bound"])
        g.tgrad_group_adamw(DONE, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, norm=norm)
        return {"norm": norm[0], "state": [(f["param"], f["exp_avg"], f["exp_avg_sq"]) for f in s["flats"]]}
    from paper_2501_02379_amd import losses
    if c["op"] == "logprobs":
        logp, lse = losses.tgrad_token_logprobs(s["logits"], s["targets"], temperature=c["temperature"])
        return {"logp": logp, "lse": lse}
    if c["op"] == "policy":
        r = losses.tgrad_policy_loss(s["logits"], s["targets"], s["weight"], s["advantage"], s["old_logp"], s["ref_logp"],
                                     clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_beta=KL_BETA, temperature=c["temperature"])
        return {"stats": r.stats, "logp": r.logp, "dlogits": r.dlogits}
    r = losses.tgrad_preference_loss(s["logits"], s["targets"], s["weight"], s["ref_logp"], s["start"], beta=PAIR_BETA,
                                     label_smoothing=SMOOTHING, dloss=s["dloss"])
    return {"loss": r.loss, "rewards": r.rewards, "logp": r.logp, "dlogits": r.dlogits}


def run(state):
    if own:
        return _own(state)
    c = state["case"]
    if c["op"] == "logprobs":
        _, logp, lse = _plain_logprobs(state["logits"], state["targets"], c["temperature"])
        return {"logp": logp, "lse": lse}
    return {"policy": _plain_policy, "preference": _plain_preference, "clip": _plain_clip, "step": _plain_step}[c["op"]](state)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------

def _exact_scores(x, y, temperature):
    """Log-probabilities and log sums, a block of rows at a time; rows without a token have neither."""
    n = x.shape[0]
    logp, lse = torch.zeros(n, device=DEV, dtype=torch.float64), torch.zeros(n, device=DEV, dtype=torch.float64)
    for a in range(0, n, 256):
        z = x[a:a + 256].double() / temperature
        k = torch.logsumexp(z, 1)
        t = y[a:a + 256]
        ok = (t >= 0) & (t < x.shape[1])
        lse[a:a + 256] = torch.where(ok, k, 0.0)
        logp[a:a + 256] = torch.where(ok, z.gather(1, t.clamp(0, x.shape[1] - 1)[:, None])[:, 0] - k, 0.0)
    return logp, lse


def _exact_dlogits(x, y, lse, dlogp, temperature):
    """d loss / d logits = dlogp / T (1[v = y] - softmax_v), in float32 where float64 would not fit beside the rest."""
    out = torch.zeros(x.shape, device=DEV, dtype=torch.float64 if x.numel() < 1 << 29 else torch.float32)
    for a in range(0, x.shape[0], 256):
        p = -(x[a:a + 256].double() / temperature - lse[a:a + 256, None]).exp()
        p.scatter_add_(1, y[a:a + 256, None], torch.ones_like(p[:, :1]))
        d = dlogp[a:a + 256, None]
        out[a:a + 256] = torch.where(d != 0, p * d / temperature, 0.0)
    return out


def _exact_policy(s):
    c, x, y = s["case"], s["logits"], s["targets"]
    logp, lse = _exact_scores(x, y, c["temperature"])
    w, a = s["weight"].double(), s["advantage"].double()
    ratio = torch.exp(logp - s["old_logp"].double())
    bounded = torch.clamp(ratio, 1 - CLIP_LOW, 1 + CLIP_HIGH)
    gain, capped = ratio * a, bounded * a
    term = -torch.where(capped < gain, capped, gain)
    slope = -torch.where(capped < gain, torch.zeros_like(gain), gain)
    kl = torch.zeros_like(term)
    if s["ref_logp"] is not None:
        q = torch.exp(s["ref_logp"].double() - logp)
        kl = q - 1 - (s["ref_logp"].double() - logp)
        slope = slope + KL_BETA * (1 - q)
    on = w != 0
    total = lambda v: (v * w)[on].sum()  # noqa: E731
    stats = torch.stack([total(term + KL_BETA * kl), total(term), total(kl), total((capped < gain).double())])
    return {"stats": stats, "logp": torch.where(on, logp, 0.0),
            "dlogits": _exact_dlogits(x, y, lse, torch.where(on, w * slope, 0.0), c["temperature"])}


def _exact_preference(s):
    x, y, pairs = s["logits"], s["targets"], s["case"]["pairs"]
    logp, lse = _exact_scores(x, y, 1.0)
    w = s["weight"].double()
    gap = w * (logp - s["ref_logp"].double())
    n = _lengths(s["case"])
    reward = torch.stack([PAIR_BETA * part.sum() for part in torch.split(gap, n)])
    h = reward[:pairs] - reward[pairs:]
    loss = -((1 - SMOOTHING) * torch.log(torch.sigmoid(h)) + SMOOTHING * torch.log(torch.sigmoid(-h))).sum() / pairs
    dh = PAIR_BETA * (SMOOTHING * torch.sigmoid(h) - (1 - SMOOTHING) * torch.sigmoid(-h)) / pairs * s["dloss"].double()
    dlogp = w * torch.repeat_interleave(torch.cat([dh, -dh]), torch.tensor(n, device=DEV))
    return {"loss": loss, "rewards": reward, "logp": torch.where(w != 0, logp, 0.0), "dlogits": _exact_dlogits(x, y, lse, dlogp, 1.0)}


def _exact_model(s):
    c = s["case"]
    wide = lambda x: x.to(torch.complex128) if x.is_complex() else x.double()  # noqa: E731
    norm = sum(wide(f["grad"]).abs().square().sum() for f in s["flats"]).sqrt()
    coef = min(1.0, c["bound"] / (float(norm) + 1e-6))
    got = []
    for f in s["flats"]:
        g = wide(f["grad"]) * coef
        if c["op"] == "clip":
            got.append(g)
            continue
        m = BETA1 * wide(f["exp_avg"]) + (1 - BETA1) * g
        v = BETA2 * f["exp_avg_sq"].double() + (1 - BETA2) * g.abs().square()
        del g
        move = m / (1 - BETA1 ** (DONE + 1)) / (torch.sqrt(v / (1 - BETA2 ** (DONE + 1))) + EPS)
        got.append((wide(f["param"]) * (1 - LR * f["decay"]) - LR * move, m, v))
    return {"norm": norm, "grads": got} if c["op"] == "clip" else {"norm": norm, "state": got}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "logprobs":
        logp, lse = _exact_scores(s["logits"], s["targets"], case["temperature"])
        return {"logp": logp, "lse": lse}
    return {"policy": _exact_policy, "preference": _exact_preference}.get(case["op"], _exact_model)(s)
