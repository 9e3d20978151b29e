"""A training step from the loss to the weights: a small Fourier neural operator that chooses one of V levels at every grid point.

The model sees a random field u on a periodic grid and emits a distribution over V levels for each point; the levels are meant
to follow the field's smoothed square.  Two phases of fine-tuning:

  preference  pairs of level sequences for the same field, a chosen one near the target and a rejected one further off
              (`losses.tgrad_preference_loss` against a frozen reference, scored with `losses.tgrad_token_logprobs`);
  policy      sequences sampled from the model itself, rewarded by their distance to the target (`losses.tgrad_policy_loss`, clipped,
              with a KL term towards the same reference).

In both, the loss's gradient goes back through torch's autograd, one norm is taken over all gradients
(`group.Group.tgrad_group_grad_norm`), and its clip factor is handed on where it lies, on the device: the spectral weights take
`tgrad_step` under it (sparse plus low-rank, `Context.tgrad_set_grad_scale`), everything else `tgrad_group_adamw`.

    python examples/field_policy.py [--steps 150]
"""
from __future__ import annotations

import argparse
import copy
import os
import sys
from fractions import Fraction

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2501_02379_amd import group, losses, sizing, tgrad as T  # noqa: E402

POINTS, WIDTH, MODES, LAYERS, LEVELS = 64, 32, 17, 2, 33


class FieldPolicy(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.lift = torch.nn.Linear(2, WIDTH)
        self.spectral = torch.nn.ParameterList(
            torch.nn.Parameter(torch.randn(WIDTH, WIDTH, MODES, 2) / WIDTH) for _ in range(LAYERS))      # (re, im) pairs, as tgrad has them
        self.local = torch.nn.ModuleList(torch.nn.Linear(WIDTH, WIDTH) for _ in range(LAYERS))
        self.head = torch.nn.Linear(WIDTH, LEVELS)

    def forward(self, u):
        x = torch.linspace(0, 1, POINTS + 1, device=u.device)[:-1].expand_as(u)
        h = self.lift(torch.stack([u, x], -1))
        for w, local in zip(self.spectral, self.local):
            f = torch.fft.rfft(h, dim=1)[:, :MODES]                                                      # (batch, mode, in)
            f = (f.unsqueeze(-1) * torch.view_as_complex(w).permute(2, 0, 1)).sum(2)
            h = torch.nn.functional.gelu(torch.fft.irfft(f, n=POINTS, dim=1) + local(h))
        return self.head(h)                                                                              # (batch, point, level)


class Trainer:
    """The optimizer of the model: a context per spectral weight, one group for the rest, one group for the norm over everything."""

    def __init__(self, model, device, lr):
        self.lr, self.t = lr, 0
        self.spectral = list(model.spectral)
        ids = {id(p) for p in self.spectral}
        self.rest = [p for p in model.parameters() if id(p) not in ids]
        for p in self.spectral + self.rest:
            p.grad = torch.zeros_like(p)                                                                 # addresses that stay
        shape = (WIDTH, WIDTH, MODES)
        cfg = T.make_config(shape, [sizing.rank_from_ratio(Fraction(1, 2), i) for i in shape],
                            sizing.sparse_count(Fraction(1, 100), WIDTH * WIDTH * MODES), lr=lr, refresh_every=50)
        self.contexts = [T.Context(cfg, device=device) for _ in self.spectral]
        self.every = group.Group([p.grad for p in self.spectral + self.rest])
        self.dense = group.Group([p.grad for p in self.rest], [p.data for p in self.rest],
                                 [torch.zeros_like(p) for p in self.rest], [torch.zeros_like(p) for p in self.rest],
                                 weight_decay=[0.01 if p.dim() > 1 else 0.0 for p in self.rest])
        self.norm = self.every.tgrad_group_grad_norm(1.0)
        for c in self.contexts:
            c.tgrad_set_grad_scale(self.norm[1:])

    def step(self, logits, dlogits):
        for p in self.spectral + self.rest:
            p.grad.zero_()
        logits.backward(dlogits.view_as(logits))
        self.every.tgrad_group_grad_norm(1.0, into=self.norm)
        for c, w in zip(self.contexts, self.spectral):
            c.tgrad_step(w.data, w.grad)
        self.dense.tgrad_group_adamw(self.t, lr=self.lr, norm=self.norm)
        self.t += 1

    def close(self):
        for c in self.contexts:
            c.tgrad_destroy()


def fields(batch, gen, device):
    """Random smooth fields and the level each point should have."""
    k = torch.arange(1, 6, device=device)
    a = torch.randn(batch, 5, 2, device=device, generator=gen) / k[:, None]
    x = torch.linspace(0, 2 * torch.pi, POINTS + 1, device=device)[:-1]
    u = (a[:, :, :1] * torch.cos(k[:, None] * x) + a[:, :, 1:] * torch.sin(k[:, None] * x)).sum(1)
    q = torch.fft.rfft(u * u)
    q[:, 4:] = 0
    target = torch.tanh(torch.fft.irfft(q, n=POINTS))
    return u, ((target + 1) / 2 * (LEVELS - 1)).round().long().clamp(0, LEVELS - 1)


def distance(levels, target):
    return (levels - target).abs().float() / LEVELS


def preference_step(model, reference, trainer, gen, device, pairs=32):
    u, target = fields(pairs, gen, device)
    near = (target + torch.randint(-1, 2, target.shape, device=device, generator=gen)).clamp(0, LEVELS - 1)
    far = torch.randint(0, LEVELS, target.shape, device=device, generator=gen)
    tokens = torch.cat([near, far]).view(-1)
    both = torch.cat([u, u])
    logits = model(both)
    with torch.no_grad():
        ref, _ = losses.tgrad_token_logprobs(reference(both).view(-1, LEVELS), tokens)
    start = torch.arange(2 * pairs + 1, device=device) * POINTS
    weight = torch.ones(2 * pairs * POINTS, device=device)
    r = losses.tgrad_preference_loss(logits.detach().view(-1, LEVELS), tokens, weight, ref, start, beta=0.1)
    trainer.step(logits, r.dlogits)
    return r.loss


def policy_step(model, reference, trainer, gen, device, batch=64, epochs=2):
    """Sample, reward, and `epochs` steps on the same samples."""
    u, target = fields(batch, gen, device)
    with torch.no_grad():
        old_logits = model(u).view(-1, LEVELS)
        tokens = torch.multinomial(torch.softmax(old_logits, 1), 1, generator=gen)[:, 0]
        old, _ = losses.tgrad_token_logprobs(old_logits, tokens)
        ref, _ = losses.tgrad_token_logprobs(reference(u).view(-1, LEVELS), tokens)
    miss = distance(tokens.view_as(target), target)
    advantage = ((miss.mean() - miss) / (miss.std() + 1e-6)).view(-1)
    weight = torch.full_like(advantage, 1.0 / advantage.numel())
    for _ in range(epochs):
        logits = model(u)
        r = losses.tgrad_policy_loss(logits.detach().view(-1, LEVELS), tokens, weight, advantage, old, ref, clip_low=0.2, clip_high=0.28,
                                     kl_beta=0.02)
        trainer.step(logits, r.dlogits)
    return miss.mean(), r.stats


def main(steps=150, seed=0, device="cuda:0", say=print):
    """-> (preference losses, mean distances to the target) of every step."""
    torch.manual_seed(seed)
    gen = torch.Generator(device=device).manual_seed(seed)
    model = FieldPolicy().to(device)
    reference = copy.deepcopy(model).requires_grad_(False)
    trainer = Trainer(model, device, lr=3e-3)
    preference = [preference_step(model, reference, trainer, gen, device) for _ in range(steps)]
    reference = copy.deepcopy(model).requires_grad_(False)
    policy = [policy_step(model, reference, trainer, gen, device) for _ in range(steps)]
    preference, missed = torch.stack(preference).tolist(), torch.stack([m for m, _ in policy]).tolist()
    kl, clipped = policy[-1][1][2:].tolist()
    say("preference loss %.3f -> %.3f" % (preference[0], preference[-1]))
    say("distance to the target, in levels %.2f -> %.2f; last step: KL %.4f, clipped %.3f, gradient norm %.3f" %
        (missed[0] * LEVELS, missed[-1] * LEVELS, kl, clipped, float(trainer.norm[0])))
    trainer.close()
    return preference, missed


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=150)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    main(a.steps, a.seed)
