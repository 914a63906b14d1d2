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


def check(dev, h, W, t, c, batch, dt=F32, g_bits=22, odt=None, alone=None, t_bits=None):
    """Both gradients, each row against its own size.  g_bits: to which g is held, t_bits: its targets' entries; alone: examples that are compared with the
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
    eg[at, tn[at]] = cs[at, 0] * ((1 - p[at, tn[at]]) * (rp[at].max(1) + 2.0 ** -(t_bits or g_bits)) + (4 + 39) * 2.0 ** -24)
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


@pytest.mark.parametrize("far", [10, 20, 30])
def test_positions_far_apart_in_features_of_their_own(dev, far):
    """The last 16 of 32 positions have 2^-far of the others' factors and all that there is of half the features."""
    h, W, t, c = make(32, 300, 64, far, 2.0)
    h[:16, 32:] = 0.0
    h[16:, :32] = 0.0
    c[16:] *= 2.0 ** -far
    g, _ = check(dev, h, W, t, c, 1)
    # a quarter of these features' largest entries is above what the check lets pass
    assert 32 * 2.0 ** -37 * (np.abs(g) * f64(h).max(1, keepdims=True)).max() < np.abs(g.T @ f64(h))[:, 32:].max() / 4


@pytest.mark.parametrize("T", [9, 70, 1300])
def test_hidden_states_far_apart(dev, T):
    """Positions whose hidden states are 2^-20 and 2^15 of others', with logits of the same size: what they add to a row of
    dweight differs as much."""
    h, W, t, c = make(T, 300, 96, T + 1, 4.0)
    W[:, 90:] = 0.0  # features that no logit sees
    h[:, 90:] *= torch.exp2(torch.randint(-20, 16, (T, 1), generator=torch.Generator().manual_seed(T)).float())
    check(dev, h, W, t, c, 1)


@pytest.mark.parametrize("T,batch", [(9, 1), (70, 1), (120, 3), (1300, 1)])
def test_weight_with_a_row_far_above_the_others(dev, T, batch):
    """A row 2^15 above the others, in a feature that the hidden states do not have: the others keep their bits."""
    for pull in (4.0, 9.0):
        h, W, t, c = make(T, 500, 128, T + 2, pull)
        h[:, 0] = 0.0
        W[:, 0] = 0.0
        W[450] = 0.0
        W[450, 0] = 2.0 ** 15
        check(dev, h, W, t, c, batch)


@pytest.mark.parametrize("T,batch", [(9, 1), (70, 1), (120, 3), (1300, 1)])
@pytest.mark.parametrize("powers", [(0, 16, 0, -70, 20, 0, -100), (20, 0, -70, -100, 0, 16, 0), (-100, -70, 0, 0, 16, 20, 20)])
def test_weight_of_blocks_far_apart(dev, T, batch, powers):
    """Every 64 rows another power of two: large ones in a feature that the hidden states do not have, small ones altogether."""
    h, W, t, c = make(T, 64 * len(powers) - 5, 128, T + 3, 4.0)
    h[:, 0], W[:, 0] = 0.0, 0.0
    for b, k in enumerate(powers):
        if k > 0:
            W[64 * b:64 * b + 64, 0] = 2.0 ** k
        else:
            W[64 * b:64 * b + 64] *= 2.0 ** k
    check(dev, h, W, t, c, batch)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("T", [9, 40, 1200])
def test_statistics_and_gradient_from_the_same_logits(dev, T, dt):
    """Positions with one hidden state and targets 0, 1, ..: example b's gradient has -p_v h in row v, and log p_v is
    position v's.  Both come from the same logit and statistics, whatever errors these have: log p rounds to 2^-24 of itself and
    twice of the logit's distance to the largest, which is no more; p, 1 / z, log z, g and dweight to 16 2^-24 together (bf16: g
    to 2^-16).  A row of the weight 2^22 above the others, in a feature that the hidden state does not have."""
    import paper_2402_03994_amd as fw
    V, d, n = 300, 64, min(T, 40)
    h, W, _, _ = make(1, V, d, T)
    h[:, 0], W[:, 0], W[290] = 0.0, 0.0, 0.0
    W[290, 0] = 2.0 ** 22
    h, W, t = h.expand(T, d).to(dt).contiguous().to(dev), W.to(dt).to(dev), torch.arange(T, device=dev) % V
    logp, stats = fw.linear_logp(h[:, None], W, t[:, None])
    _, dw = fw.linear_logp_grad(h[:, None], W, t[:, None], stats, torch.ones(T, 1, device=dev), per_example=True, out_dtype=F32)
    k = int(h[0].abs().argmax())
    p = f64(-dw[:, :n, k] / h[0, k].float())[n - 1:]  # of the last position among the n, and those behind
    want = f64(logp)[:n, 0]
    tol = (3 * np.abs(want) + 16) * 2.0 ** -24 + (2.0 ** -16 if dt == BF16 else 0.0)
    other = np.arange(n)[None] != (np.arange(n - 1, T) % V)[:, None]
    assert (np.abs(p * np.exp(-want) - 1) <= tol)[other].all(), (np.abs(p * np.exp(-want) - 1) / tol)[other].max()


@pytest.mark.parametrize("T,batch", [(33, 1), (231, 7), (264, 8), (1320, 40), (16 * 256, 16), (40, 40)])
def test_bf16_examples_in_any_company(dev, T, batch):
    """dweight in fp32: up to 256 positions an example g is held in two bf16, however many examples there are."""
    h, W, t, c = make(T, 300, 64, 5, 4.0)
    check(dev, h.to(BF16), W.to(BF16), t, c, batch, BF16, g_bits=16, odt=F32,
          alone=range(0, batch, 5) if batch > 1 and T // batch > 16 else None)


@pytest.mark.parametrize("T,batch,odt", [(300, 1, F32), (700, 1, F32), (1400, 1, F32), (1400, 1, BF16), (1200, 4, F32),
                                         (264, 8, BF16), (2600, 2, F32), (66000, 1, F32)])
def test_bf16_targets_of_many_positions(dev, T, batch, odt):
    """Above that g's entries round to bf16, but the targets', most of their rows, are held to 2^-16 in both gradients."""
    V = 300 if T < 60000 else 40
    h, W, t, c = make(T, V, 72, 6, 6.0)
    t[::7] = -1
    t[1::7] = V
    check(dev, h.to(BF16), W.to(BF16), t, c, batch, BF16, g_bits=8, t_bits=16, odt=odt)


def test_bf16_targets_of_many_rows_and_features(dev):
    """The largest tiles: rows of dweight that one position has for its target, against fp64 on the device.  The target's entry
    is held to 2^-16; the others round by 2^-8 of themselves at most, independently: 2^-8 of the root of the sum of their
    terms' squares (a p can be e^8.7 / (30000 e^1.1) = 0.07, so that no bound fits all rows); the logits of deviation 1.5 move
    an entry by 2^-17 of itself."""
    import paper_2402_03994_amd as fw
    T, V, d = 4200, 30000, 4096
    g = torch.Generator(device=dev).manual_seed(16)
    h = torch.randn(T, d, generator=g, device=dev).to(BF16)
    W = (torch.randn(V, d, generator=g, device=dev) * (1.5 / d ** 0.5)).to(BF16)
    t, c = torch.randint(-300, V, (T,), generator=g, device=dev), torch.rand(T, generator=g, device=dev) + 0.5
    _, stats = fw.linear_logp(h, W, t)
    _, dw = fw.linear_logp_grad(h, W, t, stats, c, hidden_grad=False, out_dtype=F32)
    live = (t >= 0).nonzero()[:, 0]
    G = torch.softmax(h[live].double() @ W.double().T, 1).neg_()
    G.scatter_add_(1, t[live][:, None], torch.ones(len(live), 1, dtype=torch.float64, device=dev)).mul_(c[live].double()[:, None])
    want = G.T.contiguous() @ h[live].double()
    once = torch.bincount(t[live], minlength=V) == 1
    one = torch.zeros_like(G).scatter_(1, t[live][:, None], 1.0) * G
    size = h[live].double().square().sum(1)  # of the hidden states, squared
    others = (G - one).square().T.contiguous() @ size
    tol = (2.0 ** -16 + 2.0 ** -17) * (one.square().T.contiguous() @ size).sqrt() + 2.0 ** -8 * others.sqrt()
    err = (dw.double() - want).norm(dim=1)
    assert int(once.sum()) > 3000 and (err / tol)[once].max() <= 1, (err / tol)[once].max()
    assert (tol / want.norm(dim=1))[once].median() < 2.0 ** -13


def test_few_rows_add_up_in_several_sums(dev):
    """fp32, up to 16 rows: logits of 4096 products and a deviation of 5.  A sum of n products in a row, of which it is the root of
    k / n behind k of them, rounds to 2^-24 / sqrt(3) of that each time: sqrt(n / 6) 2^-24 of the whole.  Eight sums of 512 add up to
    sqrt(4096 / 48) 2^-24 = 9.2 2^-24 of the deviation, one sum to 26 2^-24; log p and log z themselves, of size 20, to 12 2^-24.
    Half as much again for the mean of 640 of them."""
    import paper_2402_03994_amd as fw
    g = torch.Generator().manual_seed(8)
    h, W = torch.randn(16, 4096, generator=g).to(dev), (torch.randn(64, 4096, generator=g) * (5 / 64)).to(dev)
    x = h.double() @ W.double().T
    err = []
    for v in range(0, 40):
        t = torch.full((16,), v, device=dev)
        err.append(fw.linear_logp(h, W, t)[0].double() - torch.log_softmax(x, 1)[:, v])
    assert torch.stack(err).square().mean().sqrt() <= 1.5 * (46.0 ** 2 + 12.0 ** 2) ** 0.5 * 2.0 ** -24
