"""What a gradient from hidden states keeps of numbers that are small beside others: entries of vocabulary rows that no
position finds likely, examples beside ones with far larger factors, rows of the weight beside a far larger one.

Tolerances are those of test_gpu_linear.py, with the bounds taken row by row: an entry of a row of dweight is a sum over the
example's own positions, whose terms are held to 2^-21 of themselves or 2^-37 of the row's largest term; an entry of dhidden
is a sum over the vocabulary, held alike.  log p of a position and its entries of g come from the same logits: p to r = 2 (scale X
+ E) of itself, the target's 1 - p to r of itself and to roundings of p: 2^-22 of it, and 2^-24 for each addition to a sum z
that is near 1 already, at most 16 + 2 + 1 in a tile and 3 + 2 + 15 where the tiles of a small vocabulary are joined.
"""
import numpy as np
import pytest
import torch

from oracle import train as O
from test_gpu_linear import BF16, F32, HALF, errors, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    from paper_2402_03994_amd import _lib
    _lib.load()
    return torch.device("cuda", 0)


def make(T, V, d, seed, pull=0.0):
    """pull: the logit of each target above the others', about."""
    g = torch.Generator().manual_seed(seed)
    W = torch.randn(V, d, generator=g) * (1.5 / d ** 0.5)
    t = torch.randint(0, V // 3, (T,), generator=g)  # two thirds of the vocabulary are nobody's target
    h = torch.randn(T, d, generator=g)
    h += pull / 1.5 * torch.nn.functional.normalize(W[t], dim=1)
    return h, W, t, torch.randn(T, generator=g)


def check(dev, h, W, t, c, batch, dt=F32, g_bits=22, odt=None, alone=None):
    """Both gradients, each row against its own size.  g_bits: to which g is held; alone: examples that are compared with the
    same ones in a call of their own."""
    import paper_2402_03994_amd as fw
    T, (V, d) = len(t), W.shape
    n = T // batch
    shape = (batch, n) if batch > 1 else (T,)
    hd, Wd, td, cd = h.to(dev).view(*shape, d), W.to(dev), t.to(dev).view(shape), c.to(dev).view(shape)
    _, stats = fw.linear_logp(hd, Wd, td)
    dh, dw = fw.linear_logp_grad(hd, Wd, td, stats, cd, per_example=batch > 1, out_dtype=odt)
    again = fw.linear_logp_grad(hd, Wd, td, stats, cd, per_example=batch > 1, out_dtype=odt)
    assert torch.equal(again[0], dh) and torch.equal(again[1], dw)
    for b in alone or ():
        lone = fw.linear_logp_grad(hd[b], Wd, td[b], stats[b], cd[b], out_dtype=odt)[1]
        assert torch.equal(lone, dw[b]), b
    hn, Wn, tn, cn = f64(h), f64(W), t.numpy(), f64(c)
    rh, rw, g, p = O.linear_logp_grad(hn, Wn, tn, cn, 1.0, batch)
    live = (tn >= 0) & (tn < V)
    cs = np.where(live, np.abs(cn), 0.0)[:, None]
    _, rp = errors(hn, Wn, dt, 1.0)
    at = np.flatnonzero(live)
    eg = cs * p * rp + np.abs(g) * 2.0 ** -g_bits
    eg[at, tn[at]] = cs[at, 0] * ((1 - p[at, tn[at]]) * (rp[at].max(1) + 2.0 ** -g_bits) + (4 + 39) * 2.0 ** -24)
    ag, aW, ah = np.abs(g) + eg, np.abs(Wn), np.abs(hn)
    more, floor = (2.0 ** -20, 2.0 ** -37) if dt == F32 else (0.0, 0.0)
    odt = odt or dt
    tol = eg @ aW + ((3 * V + 64) * 2.0 ** -24 + more) * (ag @ aW) + HALF[dt] * np.abs(rh) + 1e-37
    tol += floor * V * (ag * aW.max(1)).max(1, keepdims=True)
    err = np.abs(f64(dh).reshape(T, d) - rh)
    assert (err <= tol).all(), (err / tol).max()
    for b in range(batch):
        r = slice(b * n, b * n + n)
        tol = eg[r].T @ ah[r] + ((3 * n + 8) * 2.0 ** -24 + more) * (ag[r].T @ ah[r]) + HALF[odt] * np.abs(rw[b]) + 1e-37
        tol += floor * n * (ag[r] * ah[r].max(1, keepdims=True)).max(0)[:, None]
        err = np.abs(f64(dw).reshape(batch, V, d)[b] - rw[b])
        assert (err <= tol).all(), (b, (err / tol).max())
    return g, p


SIZES = [(9, 1), (15, 3), (70, 1), (120, 3), (1300, 1), (1200, 4)]


@pytest.mark.parametrize("T,batch", SIZES)
def test_vocabulary_that_no_position_finds_likely(dev, T, batch):
    """Targets 12 to 40 above the rest: most rows of dweight have entries of 1e-6 to 1e-18 alone."""
    for pull in (12.0, 25.0, 40.0):
        h, W, t, c = make(T, 400, 64, T, pull)
        g, p = check(dev, h, W, t, c, batch)
        if pull == 25.0:
            assert np.median(p[:, 200:]) < 1e-10


@pytest.mark.parametrize("T,batch", [s for s in SIZES if s[1] > 1] + [(4400, 4)])
def test_examples_far_apart(dev, T, batch):
    """Factors of 2^-40, 2^-14, 1 and 2^30: each example's gradient is what it is alone, to the bit where the same kernels
    form it (16 positions and fewer have their own)."""
    h, W, t, c = make(T, 300, 96, T, 4.0)
    n = T // batch
    for b, k in enumerate((-40, 0, 30, -14)[:batch]):
        c[b * n:b * n + n] *= 2.0 ** k
    check(dev, h, W, t, c, batch, alone=range(batch))


@pytest.mark.parametrize("T", [9, 70, 1300])
def test_hidden_states_far_apart(dev, T):
    """Positions whose hidden states are 2^-20 and 2^15 of others', with logits of the same size: what they add to a row of
    dweight differs as much."""
    h, W, t, c = make(T, 300, 96, T + 1, 4.0)
    W[:, 90:] = 0.0  # features that no logit sees
    h[:, 90:] *= torch.exp2(torch.randint(-20, 16, (T, 1), generator=torch.Generator().manual_seed(T)).float())
    check(dev, h, W, t, c, 1)
