"""GPU parity of dropout and of a router's balance loss with their fp64 definitions (oracle/train.py).

Tolerances: masks and counts are equal.  Dropout in fp32: the scale (2^-24), the product with the sum (one rounding of the
result, 2^-24; a product alone one of its own) and the output's.  Balance: p to (4 A + 24) 2^-24 of itself for logits A below
the largest (exponent, exponential, sum of up to 64 columns in a row and 6 steps, reciprocal, product); sums over tokens up
to tokens / 8 additions in a thread; products with f add 4 roundings of their sizes.
"""
import numpy as np
import pytest
import torch

from oracle import train as O

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    from paper_2402_03994_amd import _lib
    _lib.load()
    return torch.device("cuda", 0)


def f64(t):
    return t.detach().cpu().double().numpy()


def rows(t, dev, lead=0, pad=0):
    r, c = t.shape
    buf = torch.full((lead + r * (c + pad),), float("nan"), dtype=t.dtype, device=dev)
    v = buf[lead:].view(r, c + pad)[:, :c]
    v.copy_(t)
    return v


def drop_tol(x, ref, kept, t, dt):
    size = np.abs(np.where(kept, np.nan_to_num(x), 0.0)) * (65536.0 / (65536 - t) if t < 65536 else 0.0)
    return 2.0 ** -23 * size + (2.0 ** -24 + HALF[dt]) * np.abs(ref) + 1e-45


@pytest.mark.parametrize("T,width", [(1, 1), (1, 7), (1, 8), (3, 5), (1, 768), (7, 64), (33, 250), (129, 1001), (500, 2048)])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_dropout(dev, T, width, dt):
    import paper_2402_03994_amd as fw
    g = torch.Generator().manual_seed(T * width)
    x, r = torch.randn(T, width, generator=g).to(dt), torch.randn(T, width, generator=g).to(dt)
    for p, seed, step, site, lead, pad in ((0.1, 7, 0, 0, 0, 0), (0.5, (5 << 32) + 3, 2 ** 32 - 1, 2 ** 32 - 1, 1, 0),
                                           (0.25, 2 ** 64 - 1, 12345, 9, 0, 3), (0.37, 1, 1, 1, 8, 8)):
        t = int(np.floor(65536 * p + 0.5))
        xd, rd = rows(x, dev, lead, pad), rows(r, dev, lead, pad)
        for res in (None, rd):
            got = fw.dropout(xd, p, seed, step, site, residual=res)
            ref, kept = O.dropout(f64(x), p, seed, step, site, None if res is None else f64(r))
            assert got.dtype == dt and got.shape == x.shape and got.is_contiguous()
            assert (np.abs(f64(got) - ref) <= drop_tol(f64(x), ref, kept, t, dt)).all()
            if res is None:
                assert np.array_equal(f64(got) != 0, kept & (f64(x) != 0))
            # in place, and into rows of another stride
            for src in ([xd] if res is None else [xd, rd]):
                a, b = rows(x, dev, lead, pad), rows(r, dev, lead, pad)
                into = a if src is xd else b
                same = fw.dropout(a, p, seed, step, site, residual=None if res is None else b, out=into)
                assert same.data_ptr() == into.data_ptr() and torch.equal(same, got)
            wide = rows(torch.zeros(T, width, dtype=dt), dev, 2, 5)
            assert torch.equal(fw.dropout(xd, p, seed, step, site, residual=res, out=wide), got)
        assert torch.equal(fw.dropout_grad(xd, p, seed, step, site), fw.dropout(xd, p, seed, step, site))


@pytest.mark.parametrize("dt", [F32, BF16])
def test_dropout_ends(dev, dt):
    """p = 0 and 1, what is dropped may be anything, shapes of any rank, nothing to do, steps held on the device."""
    import paper_2402_03994_amd as fw
    x = torch.randn(4, 5, 6, device=dev).to(dt)
    assert torch.equal(fw.dropout(x, 0.0, 1, 2), x)
    r = torch.randn_like(x)
    assert torch.equal(fw.dropout(x, 1.0, 1, 2, residual=r), r) and not fw.dropout(torch.full_like(x, float("nan")), 1.0, 1, 2).any()
    y = fw.dropout(x, 0.5, 1, 2)
    bad = torch.where(y == 0, float("inf"), x)
    assert torch.equal(fw.dropout(bad, 0.5, 1, 2), y)
    assert torch.equal(fw.dropout(x.view(-1), 0.5, 1, 2).view_as(y), y) and torch.equal(fw.dropout(x.view(20, 6), 0.5, 1, 2).view_as(y), y)
    assert fw.dropout(x[:0], 0.5, 1, 2).shape == (0, 5, 6)
    for n in (0, 3, 2 ** 32 - 1):
        at = torch.tensor([n], device=dev)
        assert torch.equal(fw.dropout(x, 0.5, 1, at), fw.dropout(x, 0.5, 1, n))
    for call in (lambda: fw.dropout(x[:, :, ::2], 0.1, 0, 0), lambda: fw.dropout(x.transpose(0, 1), 0.1, 0, 0),
                 lambda: fw.dropout(x.half(), 0.1, 0, 0), lambda: fw.dropout(x, 0.1, 0, 0, residual=r[:1]),
                 lambda: fw.dropout(x, 0.1, 0, 0, out=r.half()), lambda: fw.dropout(x, 0.1, 0, torch.tensor(1))):
        with pytest.raises(ValueError):
            call()


def test_dropout_gradient_against_differences(dev):
    import paper_2402_03994_amd as fw
    x, dy = torch.randn(50, 30, device=dev), torch.randn(50, 30, device=dev)
    g = fw.dropout_grad(dy, 0.3, 4, 5, 6)
    u = torch.randn_like(x)
    f = lambda v: (fw.dropout(v, 0.3, 4, 5, 6).double() * dy.double()).sum()  # noqa: E731
    want = (f(x + u) - f(x - u)) / 2  # linear
    assert abs(want - (g.double() * u.double()).sum()) < 2.0 ** -21 * (g.abs() * (u.abs() + x.abs())).double().sum()


def test_dropout_past_32_bits(dev):
    """More than 2^32 elements, whose blocks' numbers pass 2^29 and byte offsets 2^33."""
    import paper_2402_03994_amd as fw
    n = (1 << 32) + 4099
    x = torch.ones(n, dtype=BF16, device=dev)
    fw.dropout(x, 0.5, 3, 4, 5, out=x)
    at = (1 << 32) - 64
    i = np.arange(at, n)
    w = O.philox(i // 8, 4, 5, 13, 3)[np.arange(len(i)), (i // 2) % 4]
    assert np.array_equal(f64(x[at:]) != 0, np.where(i % 2, w >> 16, w & 0xFFFF) >= 32768)
    assert abs(float((x[:1 << 24] != 0).float().mean()) - 0.5) < 5 * 0.5 / 4096


def test_dropout_of_the_most_elements(dev):
    """2^35 of them (64 GiB), more groups of eight than a grid has threads."""
    import paper_2402_03994_amd as fw
    n = 1 << 35
    x = torch.ones(n, dtype=BF16, device=dev)
    fw.dropout(x, 0.5, 3, 4, 5, out=x)
    for at in (0, (1 << 34) - 2048, n - 4096):
        i = np.arange(at, at + 4096)
        w = O.philox(i // 8, 4, 5, 13, 3)[np.arange(4096), (i // 2) % 4]
        assert np.array_equal(f64(x[at:at + 4096]) != 0, np.where(i % 2, w >> 16, w & 0xFFFF) >= 32768)


# --- balance ----------------------------------------------------------------------------------------------
def check_balance(dev, T, E, k, dt, lead=0, pad=0, index=torch.int64, coef=0.3, seed=0):
    import paper_2402_03994_amd as fw
    g = torch.Generator().manual_seed(T + E + k + seed)
    x = (torch.randn(T, E, generator=g) * 2 + torch.randn(E, generator=g)).to(dt)
    ids = torch.randint(0, E, (T, k), generator=g)
    ids[torch.rand(T, k, generator=g) < 0.1] = -1
    ids[torch.rand(T, k, generator=g) < 0.1] = E
    ids[torch.rand(T, generator=g) < 0.1] = -5
    dead = ~((ids >= 0) & (ids < E)).any(1)
    x[dead] = float("nan")
    xd, idd = rows(x, dev, lead, pad), ids.to(dev).to(index)
    r = fw.balance_loss(xd, idd, coef=coef)
    c32 = float(np.float32(coef))
    size_c = abs(c32)  # an error's bound has no sign: |coef x - coef y| = |coef| |x - y|
    loss, counts, probs, d = O.balance_loss(f64(x), ids.numpy(), c32)
    assert np.array_equal(r.counts.cpu().numpy(), counts) and r.counts.dtype == torch.int64
    live = ~dead.numpy()
    A = np.nan_to_num(np.abs(f64(x) - f64(x).max(1, keepdims=True)))
    p = np.where(live[:, None], O.softmax_rows(np.nan_to_num(f64(x)), 1.0)[0], 0.0)
    n = max(1, live.sum())
    ep = p * (4 * A + 100) * 2.0 ** -24
    eprob = ep.sum(0) / n + probs * (T / 8 + 16) * 2.0 ** -24
    assert (np.abs(f64(r.probs) - probs) <= eprob).all()
    f = counts / (n * k)
    assert abs(float(r.loss) - loss) <= size_c * E * (f * eprob).sum() + 2.0 ** -22 * abs(loss) + 1e-45
    s = (p @ f)[:, None]
    size = f + s
    # s: errors of p and of a sum of E products; f - s: 2^-23 of both
    es = (ep @ f)[:, None] + (E + 8) * 2.0 ** -24 * s
    tol = size_c * E / n * (ep * size + p * (es + 2.0 ** -22 * size)) + (HALF[dt] + 2.0 ** -22) * np.abs(d) + 1e-45
    assert (np.abs(f64(r.dlogits) - d) <= tol).all()
    assert not f64(r.dlogits)[dead.numpy()].any() and r.dlogits.dtype == dt
    again = fw.balance_loss(xd, idd, coef=coef, grad=False)
    assert again.dlogits is None and torch.equal(again.loss, r.loss) and torch.equal(again.probs, r.probs)
    same = fw.balance_loss(xd, idd, coef=coef, out=xd)
    assert torch.equal(same.dlogits, r.dlogits) and torch.equal(same.loss, r.loss)


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (61, 8, 2), (5, 3, 4), (300, 9, 1), (1000, 33, 3), (513, 60, 4), (700, 64, 8),
                                   (129, 65, 5), (333, 128, 2), (2000, 200, 6), (40, 257, 8), (600, 512, 3), (100, 513, 70),
                                   (50, 1025, 2), (20, 2048, 9), (20000, 16, 2), (70000, 7, 1), (3000, 2048, 9), (6144, 60, 4),
                                   (6145, 60, 4), (9000, 512, 3), (9000, 513, 3), (66000, 130, 1)])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_balance(dev, T, E, k, dt):
    check_balance(dev, T, E, k, dt)


@pytest.mark.parametrize("kw", [dict(lead=1, pad=3), dict(lead=3, pad=8), dict(index=torch.int32), dict(coef=-2.0)])
def test_balance_layouts(dev, kw):
    for dt in (F32, BF16):
        check_balance(dev, 200, 60, 4, dt, **kw)


def test_balance_ends(dev):
    """No tokens, none unmasked, rows of -inf, an id that stands twice."""
    import paper_2402_03994_amd as fw
    x, ids = torch.randn(30, 12, device=dev), torch.randint(0, 12, (30, 2), device=dev)
    for r in (fw.balance_loss(x[:0], ids[:0]), fw.balance_loss(x, torch.full_like(ids, -1))):
        assert not r.loss and not r.counts.any() and not r.probs.any() and not r.dlogits.any()
    ids[:, 1] = ids[:, 0]
    r = fw.balance_loss(x, ids)
    assert torch.equal(r.counts, 2 * torch.bincount(ids[:, 0], minlength=12))
    x[3] = float("-inf")
    x[4, 5:] = float("-inf")
    r = fw.balance_loss(x, ids)
    loss, _, probs, d = O.balance_loss(f64(x), ids.cpu().numpy(), 1.0)
    assert abs(float(r.loss) - loss) < 1e-5 and np.abs(f64(r.probs) - probs).max() < 1e-6 and np.abs(f64(r.dlogits) - d).max() < 1e-6
    for call in (lambda: fw.balance_loss(x, ids[:5]), lambda: fw.balance_loss(x, ids[:, :0]), lambda: fw.balance_loss(x, ids.float()),
                 lambda: fw.balance_loss(x.half(), ids), lambda: fw.balance_loss(x, ids, out=x[:5]),
                 lambda: fw.balance_loss(x[:, ::2], ids)):
        with pytest.raises(ValueError):
            call()
