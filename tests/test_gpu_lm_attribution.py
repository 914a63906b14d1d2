"""The attribution of examples/subspace_lm.py: gradients of each text, as Sketch.apply takes them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    spec = importlib.util.spec_from_file_location("subspace_lm", os.path.join(ROOT, "examples", "subspace_lm.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_gradients_of_the_texts_add_up_to_the_batch(ex):
    """Each text's gradient, in a call of its own, among the others and their sum: roundings of sums of 48 and 384 terms and of
    eight more, each below 2^-24 of the sizes of what is added, 2^-20 of the terms' products besides."""
    import paper_2402_03994_amd as fw
    dev = torch.device("cuda", 0)
    E, R, X = ex.Model(dev).lift()
    tokens, targets = ex.texts(dev, 1)
    h, _ = ex.forward(E, R, X, tokens, 0, rate=0.0)
    c = -(targets >= 0).float()
    _, stats = fw.linear_logp(h, E, targets)
    _, each = fw.linear_logp_grad(h, E, targets, stats, c, per_example=True, hidden_grad=False)
    _, whole = fw.linear_logp_grad(h, E, targets, stats, c, hidden_grad=False)
    # sizes of the terms: |g|^T |h|, g of both signs
    live = (targets >= 0)[..., None]
    p = torch.softmax(h.double() @ E.double().T, 2)
    g = (torch.zeros_like(p).scatter_(2, targets.clamp_min(0)[..., None], 1.0) - p).abs() * live
    size = torch.stack([a.T.contiguous() @ b for a, b in zip(g, h.double().abs())])
    tol = (384 + 48 + 8) * 2.0 ** -24 + 2.0 ** -20
    assert ((each.double().sum(0) - whole.double()).abs() <= tol * size.sum(0) + 1e-12).all()
    for b in range(ex.TEXTS):
        lone = fw.linear_logp_grad(h[b], E, targets[b], stats[b], c[b], hidden_grad=False)[1]
        assert torch.equal(lone, each[b])


def test_cosines_of_sketched_gradients(ex):
    """A sketch to D numbers moves the cosine of two vectors by about (1 - cos^2) / sqrt(D): six of these."""
    assert ex.main(3)[3] < 6 / ex.D ** 0.5
