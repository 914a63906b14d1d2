"""Preference training of a small bigram model in a random subspace, then the attribution of its last batch.

theta = theta0 + S^T omega (the intrinsic-dimension parameterisation) for an embedding and an output matrix; omega is
trained on pairs of texts with the preference loss, then on sampled texts with the clipped policy loss.  Each step:
lift omega, look the tokens up, logits, the loss and its gradient at the logits, the embedding's gradient, the sketch
of the gradients, AdamW with 8-bit moments on omega.  At the end the texts' own embedding gradients are sketched and
compared with each other, as data attribution does.

    python examples/subspace_preference.py [steps]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2402_03994_amd import (AdamW, Sketch, embed, embed_grad, policy_loss, preference_loss,  # noqa: E402
                                  token_logp, token_logp_grad)

VOCAB, WIDTH, D = 1000, 64, 4096
PAIRS, LENGTH, PROMPT = 8, 48, 8


class Model:
    """theta0 + S^T omega and the gradient with respect to omega."""

    def __init__(self, device, seed: int = 0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.shapes = [(VOCAB, WIDTH), (VOCAB, WIDTH)]
        self.theta0 = [torch.randn(r * c, generator=g, device=device) * 0.1 for r, c in self.shapes]
        self.sketch = Sketch("afjl", self.shapes, D, seed=seed, device=device)
        self.omega = torch.zeros(1, D, device=device)
        self.opt = AdamW([D], state="8bit", decay=[0.0], seed=seed, device=device)
        self.steps = 0

    def lift(self):
        return [t.view(VOCAB, WIDTH) for t in self.sketch.apply_T(self.omega, theta0=self.theta0)]

    def logits(self, tokens):
        self.E, self.H = self.lift()
        self.x = embed(self.E, tokens, scale=WIDTH ** 0.5)
        return self.x @ self.H.T

    def step(self, tokens, dlogits, lr):
        dH = dlogits.T @ self.x
        dE = embed_grad(dlogits @ self.H, tokens, VOCAB, scale=WIDTH ** 0.5)
        domega = self.sketch.apply([dE.view(1, -1), dH.view(1, -1)])
        self.steps += 1
        return self.opt.step([self.omega], [domega], self.steps, lr=lr, max_norm=1.0)


def texts(device, seed: int):
    """Pairs over the same prompt: the chosen text counts upwards, the rejected one is random."""
    g = torch.Generator(device=device).manual_seed(seed)
    start = torch.randint(0, VOCAB, (PAIRS, 1), generator=g, device=device)
    chosen = (start + torch.arange(LENGTH + 1, device=device)) % VOCAB
    rejected = torch.randint(0, VOCAB, (PAIRS, LENGTH + 1), generator=g, device=device)
    rejected[:, :PROMPT] = chosen[:, :PROMPT]
    both = torch.stack([chosen, rejected], 1).view(2 * PAIRS, LENGTH + 1)
    targets = both[:, 1:].clone()
    targets[:, :PROMPT] = -100  # prompts teach nothing
    offsets = torch.arange(2 * PAIRS + 1, device=device) * LENGTH
    return both[:, :-1].reshape(-1).contiguous(), targets.reshape(-1), offsets


def main(steps: int = 60):
    device = torch.device("cuda", torch.cuda.current_device())
    model = Model(device)
    tokens, targets, offsets = texts(device, 1)
    ref, _ = token_logp(model.logits(tokens), targets)  # omega = 0: the reference model
    preference = []
    for _ in range(steps):
        r = preference_loss(model.logits(tokens), targets, offsets, ref, beta=0.1)
        model.step(tokens, r.dlogits, lr=0.01)
        preference.append(r.loss)

    # rewards for the same texts: the chosen ones good, the others bad; several clipped updates per batch
    old, _ = token_logp(model.logits(tokens), targets)
    adv = torch.tensor([1.0, -1.0], device=device).repeat(PAIRS).repeat_interleave(LENGTH)
    mask = (targets >= 0).float()
    policy = []
    for _ in range(10):
        r = policy_loss(model.logits(tokens), targets, old, adv, mask / mask.sum(), ref_logp=ref, kl_coef=0.01)
        model.step(tokens, r.dlogits, lr=0.005)
        policy.append(r.loss)

    # attribution: each text's own gradient of the embedding, sketched to D numbers
    logits = model.logits(tokens)
    _, stats = token_logp(logits, targets)
    dx = token_logp_grad(logits, targets, stats, -mask) @ model.H
    per_text = embed_grad(dx.view(2 * PAIRS, LENGTH, WIDTH), tokens.view(2 * PAIRS, LENGTH), VOCAB, scale=WIDTH ** 0.5,
                          per_example=True)
    s = model.sketch.apply([per_text.view(2 * PAIRS, -1)])
    exact = per_text.view(2 * PAIRS, -1)
    cos = torch.nn.functional.cosine_similarity(s[0:1], s[1:])
    want = torch.nn.functional.cosine_similarity(exact[0:1], exact[1:])
    return torch.stack(preference).tolist(), torch.stack(policy).tolist(), (cos - want).abs().max().item()


if __name__ == "__main__":
    pref, pol, err = main(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
    print(f"preference loss {pref[0]:.4f} -> {pref[-1]:.4f}")
    print(f"policy loss     {pol[0]:.4f} -> {pol[-1]:.4f}")
    print(f"largest error of a sketched cosine: {err:.3f}")
