"""Supervised training of a small mixture-of-experts language model in a random subspace, then the attribution of its texts.

theta = theta0 + S^T omega (the intrinsic-dimension parameterisation) for a tied embedding, a router and its experts'
matrices; omega is trained on texts that count upwards.  Each step: lift omega, look the tokens up, dropout, the experts,
the router's balance loss, the log-probabilities straight from the hidden states and the embedding (no logits in memory),
every gradient, the sketch of the gradients, AdamW on omega.  At the end each text's own gradient of the output matrix is
sketched and compared with the others', as data attribution does.

    python examples/subspace_lm.py [steps]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2402_03994_amd import (AdamW, Sketch, balance_loss, dropout, dropout_grad, embed, embed_grad,  # noqa: E402
                                  linear_logp, linear_logp_grad)

VOCAB, WIDTH, EXPERTS, TOP, D = 1000, 64, 8, 2, 4096
TEXTS, LENGTH, PROMPT = 8, 48, 8
RATE, BALANCE, SEED = 0.1, 0.01, 5


def texts(device, seed: int):
    g = torch.Generator(device=device).manual_seed(seed)
    start = torch.randint(0, VOCAB, (TEXTS, 1), generator=g, device=device)
    both = (start + torch.arange(LENGTH + 1, device=device)) % VOCAB
    targets = both[:, 1:].clone()
    targets[:, :PROMPT] = -100  # prompts teach nothing
    return both[:, :-1].contiguous(), targets.contiguous()


def forward(E, R, X, tokens, step, rate=RATE):
    """Hidden states [texts, length, width] and what their gradient needs."""
    x = embed(E, tokens, scale=WIDTH ** 0.5)
    a = dropout(x, rate, SEED, step, site=0)
    flat = a.view(-1, WIDTH)
    route = flat @ R.T
    p = torch.softmax(route, 1)
    top = torch.sort(p, dim=1, descending=True).indices[:, :TOP].contiguous()
    gate = torch.zeros_like(p).scatter_(1, top, 1.0)  # of the chosen experts
    each = torch.matmul(flat, X.transpose(1, 2).contiguous())  # [experts, tokens, width]
    h = dropout((each * (p * gate).T[:, :, None]).sum(0), rate, SEED, step, site=1, residual=flat)
    return h.view(*tokens.shape, WIDTH), (flat, route, p, top, gate, each)


def gradients(E, R, X, tokens, targets, weights, step, rate=RATE):
    """(loss, balance, dE, dR, dX): cross entropy summed with `weights`, and the balance loss."""
    h, (flat, route, p, top, gate, each) = forward(E, R, X, tokens, step, rate)
    logp, stats = linear_logp(h, E, targets)
    loss = -(weights * logp).sum()
    dh, dE = linear_logp_grad(h, E, targets, stats, -weights)
    dh = dh.view(-1, WIDTH)
    dy = dropout_grad(dh, rate, SEED, step, site=1)
    dp = (each * dy).sum(2).T * gate
    b = balance_loss(route, top, coef=BALANCE)
    droute = p * (dp - (p * dp).sum(1, keepdim=True)) + b.dlogits
    deach = dy * (p * gate).T[:, :, None]
    dX = torch.matmul(deach.transpose(1, 2).contiguous(), flat)
    da = dh + droute @ R + torch.matmul(deach, X).sum(0)
    dx = dropout_grad(da, rate, SEED, step, site=0).view(*tokens.shape, WIDTH)
    embed_grad(dx, tokens, VOCAB, scale=WIDTH ** 0.5, out=dE, accumulate=True)  # tied: onto the output matrix's gradient
    return loss, b, dE, droute.T @ flat, dX


class Model:
    def __init__(self, device, seed: int = 0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.shapes = [(VOCAB, WIDTH), (EXPERTS, WIDTH), (EXPERTS * WIDTH, WIDTH)]
        self.theta0 = [torch.randn(r * c, generator=g, device=device) * s for (r, c), s in zip(self.shapes, (0.1, 0.02, 0.05))]
        self.sketch = Sketch("afjl", self.shapes, D, seed=seed, device=device)
        self.omega = torch.zeros(1, D, device=device)
        self.opt = AdamW([D], decay=[0.0], device=device)

    def lift(self):
        E, R, X = self.sketch.apply_T(self.omega, theta0=self.theta0)
        return E.view(VOCAB, WIDTH), R.view(EXPERTS, WIDTH), X.view(EXPERTS, WIDTH, WIDTH)

    def step(self, tokens, targets, step, lr):
        weights = (targets >= 0).float()
        weights /= weights.sum()
        loss, b, *grads = gradients(*self.lift(), tokens, targets, weights, step)
        self.opt.step([self.omega], [self.sketch.apply([d.view(1, -1) for d in grads])], step, lr=lr, max_norm=1.0)
        return loss, b.loss, b.counts


def main(steps: int = 60):
    device = torch.device("cuda", torch.cuda.current_device())
    model = Model(device)
    tokens, targets = texts(device, 1)
    losses = [model.step(tokens, targets, k + 1, lr=0.02) for k in range(steps)]

    # attribution: each text's own gradient of the output matrix, sketched to D numbers
    E, R, X = model.lift()
    h, _ = forward(E, R, X, tokens, 0, rate=0.0)
    _, stats = linear_logp(h, E, targets)
    _, per_text = linear_logp_grad(h, E, targets, stats, -(targets >= 0).float(), per_example=True, hidden_grad=False)
    exact = per_text.view(TEXTS, -1)
    sketch = Sketch("afjl", [(VOCAB, WIDTH)], D, seed=1, device=device)
    s = sketch.apply([exact])
    cos = torch.nn.functional.cosine_similarity(s[0:1], s[1:])
    want = torch.nn.functional.cosine_similarity(exact[0:1], exact[1:])
    return [float(x[0]) for x in losses], [float(x[1]) for x in losses], losses[-1][2].tolist(), float((cos - want).abs().max())


if __name__ == "__main__":
    loss, balance, counts, err = main(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
    print(f"cross entropy {loss[0]:.4f} -> {loss[-1]:.4f}")
    print(f"balance loss  {balance[0]:.5f} -> {balance[-1]:.5f}, tokens per expert {counts}")
    print(f"largest error of a sketched cosine: {err:.3f}")
