"""A Bayesian next-token model on the token-model operators, sampled with
Hamiltonian Monte Carlo: what ``Sampler``'s embedding, gated block, linear layer
and categorical likelihood are for, put together.

The model: tokens t_i with targets y_i in [0, V),
  x_i = sqrt(D) E[t_i],   h_i = silu(x_i Wg^T) * (x_i Wu^T),
  o_i = h_i Wd^T + x_i,   y_i ~ Categorical(softmax(o_i Wo^T + b)),
every parameter with prior N(0, s^2).  Its potential is
  U = sum_i -log p(y_i | t_i) + sum |w|^2 / (2 s^2)
(up to a constant); positions with a negative target are not observed.

Run ``python -m paper_1912_11554_amd.token_model`` for a short example.
"""
from __future__ import annotations

import math

import torch

NAMES = ("embedding", "gate", "up", "down", "head", "bias")


class TokenModel:
    """Tokens and targets (int64 device vectors) with the model's sizes:
    V classes, width D, F columns in the gated block."""

    def __init__(self, sampler, tokens, targets, V, D, F, prior_scale=1.0):
        self.s, self.tokens, self.targets = sampler, tokens, targets
        self.V, self.D, self.F, self.prior_scale = V, D, F, prior_scale

    def shapes(self):
        V, D, F = self.V, self.D, self.F
        return dict(embedding=(V, D), gate=(F, D), up=(F, D), down=(D, F), head=(V, D), bias=(V,))

    def init(self, seed=0, scale=0.1, dtype=torch.float32):
        g = torch.Generator(device=self.tokens.device).manual_seed(seed)
        return {k: (torch.randn(*q, generator=g, device=self.tokens.device) * scale).to(dtype)
                for k, q in self.shapes().items()}

    def logits(self, w, tokens):
        """Logits [N, V] at tokens [N]: one token in generation, or many."""
        s = self.s
        x = s.embedding(tokens, w["embedding"], scale=math.sqrt(self.D))
        o = s.linear(s.gated(x, w["gate"], w["up"]), w["down"], residual=x)
        return s.linear(o, w["head"], bias=w["bias"])

    def potential(self, w):
        """U (float64 scalar tensor)."""
        total = self.s.categorical(self.logits(w, self.tokens), self.targets).double().sum()
        return total + self._prior(w)

    def _prior(self, w):
        return sum(v.double().square().sum() for v in w.values()) / (2 * self.prior_scale ** 2)

    def potential_grad(self, w):
        """U and its gradient (a dict like w)."""
        s, scale = self.s, math.sqrt(self.D)
        x = s.embedding(self.tokens, w["embedding"], scale=scale)
        h, pre = s.gated(x, w["gate"], w["up"], save=True)
        o = s.linear(h, w["down"], residual=x)
        z = s.linear(o, w["head"], bias=w["bias"])
        _, total, dz = s.categorical(z, self.targets, grad=True, out=z)
        do, dhead, dbias = s.linear_grad(dz, o, w["head"])
        dh, ddown, _ = s.linear_grad(do, h, w["down"], bias=False)
        dx, dgate, dup = s.gated_grad(dh, x, w["gate"], w["up"], pre)
        dx += do  # the block's residual
        g = dict(embedding=s.embedding_grad(self.tokens, dx, self.V, scale=scale), gate=dgate, up=dup, down=ddown,
                 head=dhead, bias=dbias)
        for k in NAMES:
            g[k].add_(w[k], alpha=1 / self.prior_scale ** 2)
        return total + self._prior(w), g

    def leapfrog(self, w, p, grad, step_size, steps):
        """``steps`` leapfrog steps from positions w, momenta p and the
        gradient at w (none is changed).  Returns positions, momenta, U and the
        gradient at the end.  Positions are float32 (see ``sample``)."""
        _need_f32(w)
        if steps < 1:
            raise ValueError(f"a trajectory has at least one step, got {steps}")
        w = {k: v.clone() for k, v in w.items()}
        p = {k: v.clone() for k, v in p.items()}
        U = None
        for _ in range(steps):
            for k in NAMES:
                p[k].sub_(grad[k], alpha=step_size / 2)
                w[k].add_(p[k], alpha=step_size)
            U, grad = self.potential_grad(w)
            for k in NAMES:
                p[k].sub_(grad[k], alpha=step_size / 2)
        return w, p, U, grad

    def sample(self, w, *, step_size, steps, num_samples, seed=0):
        """Hamiltonian Monte Carlo from w with unit masses.  Returns the last
        position and, per sample, U and whether the proposal was taken.

        Positions are float32: rounded to bfloat16 at every step they would
        neither run backwards nor preserve volume, which the acceptance
        probability relies on (``potential`` and ``potential_grad`` take both)."""
        _need_f32(w)
        g = torch.Generator(device=self.tokens.device).manual_seed(seed)
        U, grad = self.potential_grad(w)
        trace = []
        for _ in range(num_samples):
            p = {k: torch.randn(v.shape, generator=g, device=v.device) for k, v in w.items()}
            w2, p2, U2, grad2 = self.leapfrog(w, p, grad, step_size, steps)
            dH = (U2 + kinetic(p2)) - (U + kinetic(p))
            take = bool(torch.rand((), generator=g, device=dH.device, dtype=torch.float64) < torch.exp(-dH))
            if take:
                w, U, grad = w2, U2, grad2
            trace.append((float(U), take))
        return w, trace


def _need_f32(w):
    for k, v in w.items():
        if v.dtype != torch.float32:
            raise TypeError(f"{k}: positions of a trajectory must be float32, got {v.dtype}")


def kinetic(p):
    return sum(v.double().square().sum() for v in p.values()) / 2


def main():
    from . import Sampler
    sampler = Sampler(0)
    V, D, F, N = 100, 16, 32, 1000
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens = (V * torch.rand(N, device="cuda", generator=g) ** 3).long()
    targets = (tokens * 7 + 3) % V  # a rule to learn
    m = TokenModel(sampler, tokens, targets, V, D, F)
    w, trace = m.sample(m.init(seed=2), step_size=0.001, steps=100, num_samples=25, seed=3)
    for i, (U, take) in enumerate(trace):
        print(f"sample {i}: U = {U:.1f}{'' if take else ' (proposal refused)'}")
    nll = sampler.categorical(m.logits(w, tokens), targets)
    print(f"mean negative log-likelihood of the last draw: {float(nll.mean()):.3f} (uniform: {math.log(V):.3f})")
    sampler.close()


if __name__ == "__main__":
    main()
