"""GPU parity of the training-step operators with their fp64 definitions (oracle/train.py).

Tolerances, all worked out from the arithmetic:
* a value that is rounded once is within half a unit of its last place (2^-24 in fp32, 2^-8 in bf16, relative);
* a sum of k fp32 terms is within k 2^-24 of the sum of their sizes;
* log-probabilities: the exponent scale (x - m) carries 2 roundings of its size A, the exponential unit one more
  (2^-23 of its value), the sum of V of them by 256 threads or more at most V / 256 + 16 additions in a row; so
  log z and log p are within E(A, V) = (4 A + V / 256 + 32) 2^-24, and a probability is within twice that, relative.
"""
import numpy as np
import pytest
import torch

from oracle import train as O

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}  # 24 and 8 significant bits


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    from paper_2402_03994_amd import _lib
    _lib.load()
    return torch.device("cuda", 0)


def host(t):
    return t.detach().cpu().double().numpy()


def odd(t, dev, lead=1, pad=0):
    """t on the device, starting `lead` elements into its storage, rows padded by `pad` entries of NaN."""
    r, c = t.shape
    buf = torch.full((lead + r * (c + pad),), float("nan"), dtype=t.dtype, device=dev)
    v = buf[lead:].view(r, c + pad)[:, :c]
    v.copy_(t)
    return v


# --- embedding --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("width", [1, 3, 64, 257, 768, 4100])
@pytest.mark.parametrize("wdt,odt", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
def test_embed(dev, width, wdt, odt):
    import paper_2402_03994_amd as fw
    g = torch.Generator().manual_seed(width)
    w = torch.randn(37, width, generator=g).to(wdt)
    for shape, idt, lead, pad in (((1,), torch.int64, 0, 0), ((3, 5), torch.int32, 1, 0), ((301,), torch.int64, 3, 5)):
        ids = torch.randint(-3, 40, shape, generator=g).to(idt)
        out = fw.embed(odd(w, dev, lead, pad), ids.to(dev), scale=1.7, out_dtype=odt)
        ref = O.embed(w.double().numpy(), ids.numpy(), np.float32(1.7))
        assert out.dtype == odt and out.shape == (*shape, width)
        err = np.abs(host(out) - ref)
        assert (err <= (HALF[odt] + 2.0 ** -24) * np.abs(ref)).all()
    assert fw.embed(w.to(dev), torch.empty(0, dtype=torch.int64, device=dev)).shape == (0, width)


def test_embed_offsets_past_32_bits(dev):
    import paper_2402_03994_amd as fw
    w = torch.empty(1 << 20, 2100, dtype=BF16, device=dev)  # 2.2e9 elements
    ids = torch.tensor([0, (1 << 20) - 1, 1 << 20, 1022900], device=dev)
    w[ids[[0, 1, 3]]] = torch.randn(3, 2100, device=dev).to(BF16)
    out = fw.embed(w, ids)
    assert torch.equal(out[[0, 1, 3]], w[ids[[0, 1, 3]]]) and not out[2].any()


GRAD = [(1, 1, 1, 1), (1, 2, 5, 3), (1, 63, 9, 64), (3, 100, 50, 33), (2, 1000, 1, 130), (1, 5000, 3000, 96),
        (4, 4097, 700, 65), (1, 40000, 128256, 8), (1, 20000, 40, 24), (5, 7, 4000, 768)]


@pytest.mark.parametrize("batch,n,vocab,width", GRAD)
@pytest.mark.parametrize("dt,odt,accumulate", [(F32, F32, False), (BF16, F32, True), (F32, BF16, True),
                                               (BF16, BF16, False)])
def test_embed_grad(dev, batch, n, vocab, width, dt, odt, accumulate):
    import paper_2402_03994_amd as fw
    r = np.random.default_rng(n + width)
    ids = np.minimum((vocab + 1.0) ** r.random((batch, n)) - 1, vocab - 1).astype(np.int64)  # a few ids often, most rarely
    ids[r.random((batch, n)) < 0.1] = -1
    ids[r.random((batch, n)) < 0.05] = vocab
    dy = torch.from_numpy(r.standard_normal((batch * n, width)).astype(np.float32)).to(dt)
    dyd = odd(dy, dev, 1, 2 if width > 1 else 0)
    if dyd.is_contiguous() or batch == 1:
        dyd = dyd.reshape(batch, n, width) if dyd.is_contiguous() else dyd.unflatten(0, (batch, n))
    else:
        dyd = dyd.unflatten(0, (batch, n))
    idd = torch.from_numpy(ids).to(dev)
    if n % 2:
        idd = idd.int()
    shape = (batch, vocab, width)
    before = torch.from_numpy(r.standard_normal(shape).astype(np.float32)).to(odt) if accumulate else None
    for per in (True, False):
        out = None
        if accumulate:
            out = (before if per else before[0]).to(dev).clone()
        got = fw.embed_grad(dyd, idd, vocab, scale=0.3, per_example=per, out=out, out_dtype=odt, accumulate=accumulate)
        again = None if not accumulate else (before if per else before[0]).to(dev).clone()
        assert torch.equal(got, fw.embed_grad(dyd, idd, vocab, scale=0.3, per_example=per, out=again, out_dtype=odt,
                                              accumulate=accumulate))
        groups = [slice(b * n, b * n + n) for b in range(batch)] if per else [slice(0, batch * n)]
        got = host(got).reshape(len(groups), vocab, width)
        for b, s in enumerate(groups):
            i = ids.reshape(-1)[s]
            ref, size = O.embed_grad(dy.double().numpy()[s], i, vocab, np.float64(np.float32(0.3)))
            if accumulate:
                ref = ref + before[b].double().numpy()
                size = size + np.abs(before[b].double().numpy())
            runs = np.bincount(i[(i >= 0) & (i < vocab)], minlength=vocab)[:, None]
            tol = (runs + 3) * 2.0 ** -24 * size + HALF[odt] * np.abs(ref)
            assert (np.abs(got[b] - ref) <= tol).all()


def test_embed_grad_without_tokens(dev):
    import paper_2402_03994_amd as fw
    none = torch.empty(0, 6, device=dev), torch.empty(0, dtype=torch.int64, device=dev)
    assert not fw.embed_grad(*none, 11).any()
    kept = torch.ones(11, 6, device=dev)
    fw.embed_grad(*none, 11, out=kept, accumulate=True)
    assert (kept == 1).all()
    out = fw.embed_grad(torch.ones(2, 0, 6, device=dev), torch.empty(2, 0, dtype=torch.int32, device=dev), 11,
                        per_example=True)
    assert out.shape == (2, 11, 6) and not out.any()
    masked = fw.embed_grad(torch.full((4, 6), float("nan"), device=dev), torch.full((4,), -1, device=dev), 11)
    assert not masked.any()  # what a masked token brings is not looked at


# --- logits -----------------------------------------------------------------------------------------------
VOCABS = [1, 2, 63, 64, 65, 1000, 2049, 4099, 8200, 33000, 50257, 70001, 128256, 140003, 300001]


def make_logits(rows, vocab, dt, seed):
    """Rows of every kind, their targets and which are masked."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab, generator=g) * 3
    t = torch.randint(0, vocab, (rows,), generator=g)
    x[torch.arange(rows), t] += torch.rand(rows, generator=g) * 10
    low = torch.finfo(dt).min
    for k in range(rows):
        kind = k % 9
        if kind == 1:
            x[k] = low                                    # the lowest value everywhere: uniform
        elif kind == 2:
            x[k, torch.rand(vocab, generator=g) < 0.5] = -float("inf")
            x[k, t[k]] = 1.0
        elif kind == 3:
            x[k] = float("nan")                           # masked below
            t[k] = -100 if k % 2 else vocab
        elif kind == 4:
            x[k] = -float("inf")                          # nothing left
        elif kind == 5:
            x[k] += 500.0                                 # a large common part
        elif kind == 6 and vocab > 1:
            x[k, t[k]] = -float("inf")                    # the target is ruled out
        elif kind == 7:
            x[k, torch.arange(vocab) != t[k]] = low       # one entry left
    return x.to(dt), t


def exponent_sizes(x, scale):
    """Per entry |scale (x - m)| where it can matter (beyond 100 both sides are 0 to 1e-43)."""
    x = x.double().numpy()
    with np.errstate(all="ignore"):
        m = np.nan_to_num(x.max(1, keepdims=True), neginf=0.0)
        return np.minimum(np.nan_to_num(np.abs(x - m) * scale, posinf=0.0, nan=0.0), 110.0)


def err_logp(A, vocab):
    return (4 * A + vocab / 256 + 32) * 2.0 ** -24


def check_logp(got, ref, A, vocab, x, scale):
    fin = np.isfinite(ref)
    assert np.array_equal(got[~fin], ref[~fin], equal_nan=True)
    # the target's own exponent, of any size, is rounded too
    assert (np.abs(got - ref)[fin] <= (err_logp(A.max(1), vocab) + np.abs(ref) * 2.0 ** -22)[fin]).all()


def check_grad(got, ref, c, p, A, vocab, scale, dt):
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    tol = np.abs(c)[:, None] * scale * (2 * err_logp(A, vocab) + 2 * err_logp(0.0, vocab)) * np.nan_to_num(p)
    tol = tol + (HALF[dt] + 2.0 ** -22) * np.abs(ref) + 1e-37
    ok = ~np.isnan(ref)
    assert (np.abs(got - ref)[ok] <= tol[ok]).all()


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("dt", [F32, BF16])
def test_token_logp_and_gradient(dev, vocab, dt):
    import paper_2402_03994_amd as fw
    rows = 27 if vocab < 60000 else 11
    x, t = make_logits(rows, vocab, dt, vocab)
    r = np.random.default_rng(vocab)
    c = torch.from_numpy(r.standard_normal(rows).astype(np.float32))
    c[min(5, rows - 1)] = 0.0
    for lead, pad, scale, idt in ((0, 0, 1.0, torch.int64), (1, 3, 0.7, torch.int32)):
        xd, td = odd(x, dev, lead, pad), t.to(idt).to(dev)
        s = float(np.float32(scale))
        logp, stats = fw.token_logp(xd, td, scale=scale)
        A = exponent_sizes(x, s)
        check_logp(host(logp), O.token_logp(x.double().numpy(), t.numpy(), s), A, vocab, x, s)
        ref = O.token_logp_grad(x.double().numpy(), t.numpy(), c.double().numpy(), s)
        p = O.softmax_rows(x.double().numpy(), s)[0]
        d = fw.token_logp_grad(xd, td, stats, c.to(dev), scale=scale)
        check_grad(host(d), ref, c.double().numpy(), p, A, vocab, s, dt)
        into = odd(torch.zeros(rows, vocab, dtype=dt), dev, 2, 1)  # another alignment than the logits'
        fw.token_logp_grad(xd, td, stats, c.to(dev), scale=scale, out=into)
        assert np.array_equal(host(into), host(d), equal_nan=True)
        fw.token_logp_grad(xd, td, stats, c.to(dev), scale=scale, out=xd)  # in place
        assert np.array_equal(host(xd), host(d), equal_nan=True)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_what_is_not_finite_follows_the_formula(dev, bad):
    import paper_2402_03994_amd as fw
    x = torch.randn(3, 500)
    x[1, 17] = bad
    t = torch.tensor([3, 4, 5], device=dev)
    logp, stats = fw.token_logp(x.to(dev), t)
    d = fw.token_logp_grad(x.to(dev), t, stats, torch.ones(3, device=dev))
    assert torch.isfinite(logp[[0, 2]]).all() and torch.isfinite(d[[0, 2]]).all()
    assert torch.isnan(logp[1]) and torch.isnan(d[1]).any()


@pytest.mark.parametrize("rows", [1, 2, 9, 300])
def test_token_logp_rows(dev, rows):
    import paper_2402_03994_amd as fw
    x, t = make_logits(rows, 1003, F32, rows)
    got = host(fw.token_logp(x.to(dev), t.to(dev))[0])
    check_logp(got, O.token_logp(x.double().numpy(), t.numpy(), 1.0), exponent_sizes(x, 1.0), 1003, x, 1.0)
    for n in (0,):
        e = torch.empty(n, 1003, device=dev), torch.empty(n, dtype=torch.int64, device=dev)
        logp, stats = fw.token_logp(*e)
        assert logp.shape == (0,) and fw.token_logp_grad(*e, stats, logp).shape == (0, 1003)


def test_logits_past_32_bits(dev):
    import paper_2402_03994_amd as fw
    rows, vocab = 34000, 65000  # 2.2e9 entries
    x = torch.zeros(rows, vocab, dtype=BF16, device=dev)
    t = torch.full((rows,), -1, device=dev)
    at = [0, 33038, 33999]  # on both sides of entry 2^31
    x[at] = torch.randn(3, vocab, device=dev).to(BF16)
    t[at] = torch.tensor([5, 64999, 7], device=dev)
    logp, stats = fw.token_logp(x, t)
    ref = O.token_logp(x[at].double().cpu().numpy(), t[at].cpu().numpy(), 1.0)
    assert np.abs(host(logp[at]) - ref).max() <= err_logp(20.0, vocab)
    c = torch.ones(rows, device=dev)
    d = fw.token_logp_grad(x, t, stats, c)
    ref = O.token_logp_grad(x[at].double().cpu().numpy(), t[at].cpu().numpy(), np.ones(3), 1.0)
    assert np.abs(host(d[at]) - ref).max() <= 2.0 ** -9
    assert not d[1:33038].any() and not d[33039:33999].any()


def policy_inputs(x, t, seed):
    r = np.random.default_rng(seed)
    n = len(t)
    lp = O.token_logp(x.double().numpy(), t.numpy(), 1.0)
    lp = np.where(np.isfinite(lp), lp, -1.0)
    # ratios inside and outside of [0.8, 1.2], not at the bounds themselves
    old = lp - r.choice([-0.5, -0.1, 0.0, 0.1, 0.5], n)
    adv, w, ref = r.standard_normal(n), r.random(n) / n, lp + 0.3 * r.standard_normal(n)
    w[::7] = 0.0
    masked = (t.numpy() < 0) | (t.numpy() >= x.shape[1])
    for v in (old, adv, w, ref):
        v[masked] = np.nan  # not looked at there
    return [torch.from_numpy(v.astype(np.float32)) for v in (old, adv, w, ref)]


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("dt,kl", [(F32, 0.0), (F32, 0.2), (BF16, 0.2)])
def test_policy_loss(dev, vocab, dt, kl):
    import paper_2402_03994_amd as fw
    rows = 27 if vocab < 60000 else 11
    x, t = make_logits(rows, vocab, dt, vocab + 1)
    # rows whose target is ruled out make the divergence infinite: they are looked at by the other operators
    t[[k for k in range(rows) if k % 9 in (4, 6)]] = -1
    old, adv, w, ref = policy_inputs(x, t, vocab)
    xd = odd(x, dev, 1, 3)
    got = fw.policy_loss(xd, t.to(dev), old.to(dev), adv.to(dev), w.to(dev), ref_logp=ref.to(dev) if kl else None,
                         kl_coef=kl)
    f = lambda v: v.double().numpy()  # noqa: E731
    lo, k32 = float(np.float32(0.2)), float(np.float32(kl))
    loss, logp, tok, d = O.policy(f(x), t.numpy(), f(old), f(adv), f(w), f(ref), lo, lo, k32, 1.0)
    live = (t.numpy() >= 0) & (t.numpy() < vocab) & (f(w) != 0)
    A, p = exponent_sizes(x, 1.0), O.softmax_rows(f(x), 1.0)[0]
    check_logp(host(got.logp), logp, A, vocab, x, 1.0)
    # a log-probability that is off by e moves the ratios by e of their sizes
    e = err_logp(A.max(1), vocab) + (np.abs(logp) + 4) * 2.0 ** -22
    z = lambda v: np.where(live, v, 0.0)  # noqa: E731
    size = z(np.abs(f(adv)) * np.exp(logp - f(old)) + k32 * (2 + np.exp(f(ref) - logp)))
    assert (np.abs(host(got.token_loss) - tok) <= size * e + 2.0 ** -22 * size).all()
    assert abs(float(got.loss) - loss) <= (z(f(w)) * (size * e + 2.0 ** -22 * size)).sum() + 2.0 ** -24 * abs(loss)
    dd, tol_c = host(got.dlogits), z(f(w)) * size * (e + 2.0 ** -22)
    c = z(f(w)) * O.policy_tokens(z(logp), z(f(old)), z(f(adv)), z(f(ref)), lo, lo, k32)[1]
    tol = np.abs(c)[:, None] * (2 * err_logp(A, vocab) + 2 * err_logp(0.0, vocab)) * np.nan_to_num(p) \
        + tol_c[:, None] + (HALF[dt] + 2.0 ** -22) * np.abs(d) + 1e-37
    assert (np.abs(dd - d) <= tol).all()
    assert not dd[~live].any()
    same = fw.policy_loss(xd, t.to(dev), old.to(dev), adv.to(dev), w.to(dev), ref_logp=ref.to(dev) if kl else None,
                          kl_coef=kl, grad=False)
    assert same.dlogits is None and torch.equal(same.loss, got.loss) and torch.equal(same.logp, got.logp)
    inplace = fw.policy_loss(xd, t.to(dev), old.to(dev), adv.to(dev), w.to(dev), ref_logp=ref.to(dev) if kl else None,
                             kl_coef=kl, out=xd)
    assert torch.equal(inplace.dlogits, got.dlogits) and torch.equal(inplace.loss, got.loss)


@pytest.mark.parametrize("vocab", [5, 1000, 4099, 50257, 140003])
@pytest.mark.parametrize("dt,average,eps", [(F32, False, 0.0), (F32, True, 0.1), (BF16, False, 0.1)])
def test_preference_loss(dev, vocab, dt, average, eps):
    import paper_2402_03994_amd as fw
    rows = 31
    x, t = make_logits(rows, vocab, dt, vocab + 2)
    t[[k for k in range(rows) if k % 9 in (1, 4, 6)]] = -1  # (4, 6: logs of 0)
    offs = np.array([0, 4, 4, 5, 16, 28, 29])  # an empty text, a text of one, and two rows after the last
    r = np.random.default_rng(vocab)
    ref = O.token_logp(x.double().numpy(), t.numpy(), 1.0) + 0.5 * r.standard_normal(rows)
    ref[(t.numpy() < 0) | (t.numpy() >= vocab)] = np.nan
    ref = torch.from_numpy(ref.astype(np.float32))
    xd = odd(x, dev, 1, 1)
    offd = torch.from_numpy(offs).to(dev)
    call = lambda **k: fw.preference_loss(xd, t.to(dev), offd, ref.to(dev), beta=0.3, label_smoothing=eps,  # noqa: E731
                                          average=average, **k)
    got = call()
    b, e32 = float(np.float32(0.3)), float(np.float32(eps))
    loss, seq, pair, d = O.preference(x.double().numpy(), t.numpy(), offs, ref.double().numpy(), b, e32, average, 1.0)
    A, p = exponent_sizes(x, 1.0), O.softmax_rows(x.double().numpy(), 1.0)[0]
    lp = O.token_logp(x.double().numpy(), t.numpy(), 1.0)
    e = np.where(lp != 0, err_logp(A.max(1), vocab) + np.abs(lp) * 2.0 ** -22, 0.0)
    es = np.array([e[a:z].sum() for a, z in zip(offs, offs[1:])])
    assert (np.abs(host(got.seq_logp) - seq) <= es + 2.0 ** -23 * np.abs(seq)).all()
    ep = b * (es[0::2] + es[1::2]) + 2.0 ** -23 * np.abs(pair)
    assert (np.abs(host(got.pair_loss) - pair) <= ep).all()
    assert abs(float(got.loss) - loss) <= ep.mean() + 2.0 ** -23 * abs(loss)
    # a row's factor is b / pairs at most, and moves with b d like its size
    c = np.zeros(rows)
    for i, (a, z) in enumerate(zip(offs, offs[1:])):
        c[a:z] = b / 3 * (1 + ep[i // 2])
    ce = np.zeros(rows)
    for i, (a, z) in enumerate(zip(offs, offs[1:])):
        ce[a:z] = b / 3 * (ep[i // 2] + 2.0 ** -22)
    tol = c[:, None] * (2 * err_logp(A, vocab) + 2 * err_logp(0.0, vocab)) * np.nan_to_num(p) + ce[:, None] \
        + (HALF[dt] + 2.0 ** -22) * np.abs(d) + 1e-37
    assert (np.abs(host(got.dlogits) - d) <= tol).all()
    assert not got.dlogits[29:].any()
    assert torch.equal(call(grad=False).loss, got.loss) and call(grad=False).dlogits is None
    offd = offd.int()
    again = call(out=xd)  # in place, with 32-bit offsets
    assert torch.equal(again.dlogits, got.dlogits) and torch.equal(again.loss, got.loss)


def test_losses_agree_with_differences(dev):
    """The gradient against differences of the kernels' own loss, along one direction."""
    import paper_2402_03994_amd as fw
    rows, vocab = 24, 700
    x, t = torch.randn(rows, vocab, device=dev) * 2, torch.randint(0, vocab, (rows,), device=dev)
    lp = fw.token_logp(x, t)[0]
    old, adv, w = lp - 0.05, torch.randn(rows, device=dev), torch.full((rows,), 1.0 / rows, device=dev)
    ref, offs = lp + 0.1 * torch.randn(rows, device=dev), torch.tensor([0, 7, 12, 18, 24], device=dev)
    for f in (lambda y: fw.policy_loss(y, t, old, adv, w, ref_logp=ref, kl_coef=0.1),
              lambda y: fw.preference_loss(y, t, offs, ref, beta=0.5)):
        d = f(x).dlogits
        u = d / d.norm()
        h = 2.0 ** -4
        slope = (float(f(x + h * u).loss) - float(f(x - h * u).loss)) / (2 * h)
        want = float((d * u).sum())
        # h^2 / 6 of third derivatives (below the first one's size here), and the losses' own 1e-6 / h
        assert abs(slope - want) <= h * h * abs(want) + 1e-4


def test_losses_on_another_stream(dev):
    import paper_2402_03994_amd as fw
    x, t = torch.randn(64, 5000, device=dev), torch.randint(0, 5000, (64,), device=dev)
    a = fw.token_logp(x, t)[0]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        y = x * 2
        b = fw.token_logp(y, t, scale=0.5)[0]
        e = fw.embed_grad(y, t, 5000)
    s.synchronize()
    assert (a - b).abs().max() < 1e-5
    assert torch.equal(e, fw.embed_grad(x * 2, t, 5000))


def test_graph_replays(dev):
    import paper_2402_03994_amd as fw
    n, vocab = 48, 3001
    x, t = torch.randn(n, vocab, device=dev), torch.randint(0, vocab, (n,), device=dev)
    w = torch.randn(vocab, 32, device=dev)
    v = [torch.randn(n, device=dev) for _ in range(3)]
    offs = torch.tensor([0, 10, 48], device=dev)
    opt, p = fw.AdamW([(vocab, 32)], state="8bit"), torch.randn(vocab, 32, device=dev)

    def step():
        e = fw.embed(w, t)
        a = fw.policy_loss(x, t, v[0], v[1], v[2], ref_logp=v[0], kl_coef=0.1)
        b = fw.preference_loss(x, t, offs, v[0])
        g = fw.embed_grad(e, t, vocab)
        norm = opt.step([p], [g], 1, lr=0.01, max_norm=1.0)
        return [e, a.loss, a.dlogits, b.loss, b.dlogits, g, norm, p, opt.m, opt.v]

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for k in range(4):
        x.normal_()
        v[0].normal_()
        start = p.clone(), opt.m.clone(), opt.v.clone(), opt.m_exp.clone(), opt.v_exp.clone()
        want = [o.clone() for o in step()]
        for dst, src in zip((p, opt.m, opt.v, opt.m_exp, opt.v_exp), start):
            dst.copy_(src)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), k


# --- AdamW ------------------------------------------------------------------------------------------------
SIZES = [1, 63, 64, 65, 1023, 4095, 4096, 4097, 10000, 3]


def padded(flat, sizes):
    out, at = [], 0
    for n in sizes:
        out += [flat[at:at + n], np.zeros(-n % 64, flat.dtype)]
        at += n
    return np.concatenate(out)


def unpadded(flat, sizes):
    out, at = [], 0
    for n in sizes:
        out.append(flat[at:at + n])
        at += n + -n % 64
    return np.concatenate(out)


@pytest.mark.parametrize("state", ["f32", "8bit"])
@pytest.mark.parametrize("pdt,gdt,master", [(F32, F32, False), (F32, BF16, False), (BF16, BF16, False), (BF16, F32, True),
                                            (BF16, BF16, True), (BF16, F32, False)])
@pytest.mark.parametrize("clip", [None, 0.5])
def test_adamw(dev, state, pdt, gdt, master, clip):
    import paper_2402_03994_amd as fw
    sizes = SIZES * 14 if clip else SIZES  # 140 tensors: two launches
    total = sum(sizes)
    r = np.random.default_rng(11)
    decay = [float(k % 3 > 0) for k in range(len(sizes))]
    opt = fw.AdamW(sizes, state=state, decay=decay, seed=2 ** 40 + 5)
    p0 = torch.from_numpy(r.standard_normal(total).astype(np.float32))
    buf = torch.zeros(total + 1, dtype=pdt, device=dev)[1:]  # parameters one after the other from an odd start
    buf.copy_(p0)
    mast = torch.zeros(total + 3, device=dev)[3:].copy_(p0) if master else None
    split = lambda t: list(torch.split(t, sizes))  # noqa: E731
    hp = p0.numpy().astype(np.float64) if master else host(buf)
    m, v = np.zeros(total, np.float32), np.zeros(total, np.float32)
    wd = np.concatenate([np.full(n, 0.1 * d) for n, d in zip(sizes, decay)])
    gs = torch.tensor(0.75, device=dev)
    for step in (1, 2, 3, 70000):
        g = torch.from_numpy((r.standard_normal(total) * np.exp(2 * r.standard_normal(total)) * 0.01).astype(np.float32))
        gd = torch.zeros(total + 1, dtype=gdt, device=dev)[1:].copy_(g)
        norm = opt.step(split(buf), split(gd), step, lr=0.01, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1,
                        masters=split(mast) if master else None, grad_scale=gs, max_norm=clip)
        gh = host(gd).astype(np.float32)
        s = np.float32(0.75)
        if clip:
            want = 0.75 * np.sqrt((gh.astype(np.float64) ** 2).sum())
            assert abs(float(norm) - want) <= 2.0 ** -23 * want
            s = s * min(np.float32(1.0), np.float32(clip) / (np.float32(float(norm)) + np.float32(1e-6)))
        m, v = O.adamw_moments(m, v, gh, 0.9, 0.99, s)
        ref = O.adamw_param(hp, m, v, step, 0.01, 0.9, 0.99, 1e-6, wd)
        upd = np.abs(ref - hp)
        # the update is off by a few roundings of its size, the parameter by one more of its own
        tol = 2.0 ** -20 * upd + 2.0 ** -23 * np.abs(hp)
        if state == "8bit":
            u = [O.adamw_words(n, step, l, 2 ** 40 + 5) for l, n in enumerate(sizes)]
            um, uv = (padded(np.concatenate([w[k] for w in u]).astype(np.int64), sizes).reshape(-1, 64) for k in (0, 1))
            cm, em = O.encode8(padded(m, sizes).reshape(-1, 64), 15, um)
            cv, ev = O.encode8(padded(v, sizes).reshape(-1, 64), 31, uv)
            assert np.array_equal(opt.m_exp.cpu().numpy(), em) and np.array_equal(opt.v_exp.cpu().numpy(), ev)
            assert np.array_equal(opt.m.cpu().numpy().reshape(-1, 64), cm)
            assert np.array_equal(opt.v.cpu().numpy().reshape(-1, 64), cv)
            mp, vp = O.decode8(cm, em, 15).reshape(-1), O.decode8(cv, ev, 31).reshape(-1)
            got = opt.moments()
            assert np.array_equal(got[0].cpu().numpy(), mp) and np.array_equal(got[1].cpu().numpy(), vp)
            m, v = unpadded(mp, sizes), unpadded(vp, sizes)
        else:
            assert np.array_equal(unpadded(opt.m.cpu().numpy(), sizes), m)
            assert np.array_equal(unpadded(opt.v.cpu().numpy(), sizes), v)
        if master:
            assert (np.abs(host(mast) - ref) <= tol).all()
            assert torch.equal(buf, mast.to(BF16))
            hp = host(mast)
        elif pdt == BF16:
            # what the random number makes of ref - tol and of ref + tol, or anything in between
            u = np.concatenate([O.adamw_words(n, step, l, 2 ** 40 + 5)[2] for l, n in enumerate(sizes)])
            lo, hi = (((ref + k * np.sign(ref) * tol).astype(np.float32).view(np.uint32).astype(np.int64) + u) >> 16 << 16
                      for k in (-1, 1))
            got = host(buf)
            a, b = (w.astype(np.uint32).view(np.float32).astype(np.float64) for w in (lo, hi))
            assert (((np.abs(a) <= np.abs(got)) & (np.abs(got) <= np.abs(b))) | (np.abs(ref) < 1e-6)).all()
            hp = got
        else:
            assert (np.abs(host(buf) - ref) <= tol).all()
            hp = host(buf)


@pytest.mark.parametrize("state", ["f32", "8bit"])
def test_adamw_skips_a_step_that_is_not_finite(dev, state):
    import paper_2402_03994_amd as fw
    opt, p = fw.AdamW([300, (5, 7)], state=state), [torch.randn(300, device=dev), torch.randn(5, 7, device=dev)]
    g = [torch.randn_like(t) for t in p]
    opt.step(p, g, 1, lr=0.1)
    kept = [t.clone() for t in (*p, *opt.state_dict().values())]
    for s in (float("inf"), float("nan")):
        opt.step(p, g, 2, lr=0.1, grad_scale=torch.tensor(s, device=dev))
    g[1][2, 3] = float("nan")
    assert torch.isnan(opt.step(p, g, 2, lr=0.1, max_norm=1.0))
    assert all(torch.equal(a, b) for a, b in zip(kept, (*p, *opt.state_dict().values())))
    # without a norm to tell, a NaN stays where it is: its block of 64 in 8 bits
    opt.step(p, g, 2, lr=0.1)
    m, v = opt.moments()
    n = torch.isnan(m).nonzero()[:, 0].tolist()
    assert n == ([320 + 17] if state == "f32" else list(range(320, 384)))
    assert torch.isfinite(p[0]).all()


def test_adamw_in_8_bits_keeps_slow_averages(dev):
    """v follows E g^2 under b2 = 0.999 although one step changes it by less than half a code, up and down."""
    import paper_2402_03994_amd as fw
    n = 1 << 14
    opt, p = fw.AdamW([n], state="8bit", seed=3), [torch.zeros(n, device=dev)]
    g = torch.Generator(device=dev).manual_seed(1)
    for level, steps in ((1.0, 1500), (0.25, 3000)):
        for k in range(steps):
            opt.step(p, [torch.randn(n, generator=g, device=dev) * level], k + 1, lr=0.0, weight_decay=0.0)
        v = opt.moments()[1]
        want = level ** 2 * (1 - 0.999 ** steps) + (0.999 ** steps * (1 - 0.999 ** 1500) if level < 1 else 0.0)
        # n averages of 1000 terms with a spread below their own size each
        assert abs(float(v.mean()) - want) < 0.02 * want


def test_adamw_state_comes_back(dev):
    import paper_2402_03994_amd as fw
    a, b = (fw.AdamW([1000, 17], state="8bit", seed=9) for _ in range(2))
    p = [torch.randn(1000, device=dev), torch.randn(17, device=dev)]
    q = [t.clone() for t in p]
    g = [torch.randn_like(t) for t in p]
    a.step(p, g, 1, lr=0.1)
    b.load_state_dict(a.state_dict())
    q = [t.clone() for t in p]
    a.step(p, g, 2, lr=0.1)
    b.step(q, g, 2, lr=0.1)
    assert all(torch.equal(x, y) for x, y in zip(p, q)) and torch.equal(a.m, b.m)
    with pytest.raises(ValueError):
        b.load_state_dict({"m": a.m})
    with pytest.raises(ValueError):
        b.step(p[:1], g[:1], 3, lr=0.1)
    with pytest.raises(ValueError):
        b.step(p, [g[0].double(), g[1]], 3, lr=0.1)
    with pytest.raises(ValueError):
        b.step(p, g, 3, lr=0.1, max_norm=0.0)
    with pytest.raises(fw.SketchError):
        b.step(p, g, 0, lr=0.1)
    with pytest.raises(fw.SketchError):
        b.step(p, g, 3, lr=0.1, betas=(0.9, 1.0))
    with pytest.raises(ValueError):
        fw.AdamW([10], state="16bit")


def test_binding_refuses(dev):
    import paper_2402_03994_amd as fw
    x, t, v = torch.zeros(4, 8, device=dev), torch.zeros(4, dtype=torch.int64, device=dev), torch.zeros(4, device=dev)
    bad = [lambda: fw.embed(x.half(), t), lambda: fw.embed(x.t(), t), lambda: fw.embed(x, t.float()),
           lambda: fw.embed(x, t, out=torch.empty(4, 7, device=dev)), lambda: fw.embed(x, t.cpu()),
           lambda: fw.embed_grad(x, t[:3], 8), lambda: fw.embed_grad(x, t, 8, per_example=True),
           lambda: fw.embed_grad(x, t, 8, accumulate=True), lambda: fw.embed_grad(x, t, 8, out=x),
           lambda: fw.token_logp(x.t(), t), lambda: fw.token_logp(x, t[:3]), lambda: fw.token_logp(x[0], t),
           lambda: fw.token_logp(x[:1].expand(4, 8), t), lambda: fw.token_logp_grad(x, t, v, v),
           lambda: fw.token_logp_grad(x, t, torch.zeros(4, 2, device=dev), v[:3]),
           lambda: fw.policy_loss(x, t, v, v, v[:3]), lambda: fw.policy_loss(x, t, v.double(), v, v),
           lambda: fw.policy_loss(x, t, v, v, v, out=x.bfloat16()),
           lambda: fw.preference_loss(x, t, t[:2], v), lambda: fw.preference_loss(x, t, t[:3], v[::2])]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(k)
    with pytest.raises(fw.SketchError):
        fw.policy_loss(x, t, v, v, v, kl_coef=0.1)
    with pytest.raises(fw.SketchError):
        fw.token_logp(x, t, scale=0.0)


def test_adamw_norm_of_many_chunks(dev):
    """Lists of more than 256 chunks have their norm added up by a kernel of its own."""
    import paper_2402_03994_amd as fw
    sizes = [3_000_001, 70, 1_500_000]
    opt = fw.AdamW(sizes)
    g = [torch.randn(n, device=dev) * 0.01 for n in sizes]
    p = [torch.zeros(n, device=dev) for n in sizes]
    want = np.sqrt(sum((host(t) ** 2).sum() for t in g))
    norm = opt.step(p, g, 1, lr=0.1, betas=(0.5, 0.5), eps=1e-3, weight_decay=0.0, max_norm=2.0)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    s = np.float32(2.0) / (np.float32(float(norm)) + np.float32(1e-6))
    for n, at, t in zip(sizes, (0, 3_000_064, 3_000_192), g):
        m, v = O.adamw_moments(np.zeros(n, np.float32), np.zeros(n, np.float32), t.cpu().numpy(), 0.5, 0.5, s)
        assert np.array_equal(opt.m[at:at + n].cpu().numpy(), m) and np.array_equal(opt.v[at:at + n].cpu().numpy(), v)


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-8])
def test_adamw_small_second_moments(dev, eps):
    """Second moments down to the smallest fp32 numbers, with and without an eps that hides them."""
    import paper_2402_03994_amd as fw
    n = 4000
    opt = fw.AdamW([n])
    g = torch.logspace(-24, 3, n, device=dev)  # squares from 0 to 1e6
    g[n // 2:] *= -1
    p = torch.zeros(n, device=dev)
    opt.step([p], [g], 1, lr=1.0, betas=(0.9, 0.999), eps=eps, weight_decay=0.0)
    m, v = opt.m[:n].cpu().numpy(), opt.v[:n].cpu().numpy()
    ref = O.adamw_param(np.zeros(n), m, v, 1, 1.0, 0.9, 0.999, eps, 0.0)
    got = host(p)
    big = ~np.isfinite(ref) | (np.abs(ref) > 1e30)  # v = 0: m / eps
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    # beta powers in fp32 and a few roundings of the ratio
    assert (np.abs(got - ref)[~big] <= 2.0 ** -20 * np.abs(ref)[~big]).all()
    assert np.array_equal(np.sign(got[big]), np.sign(ref[big]))


def test_embed_grad_of_many_runs(dev):
    """More than 16 sorted runs: two rounds of merges."""
    import paper_2402_03994_amd as fw
    r = np.random.default_rng(8)
    n, vocab = 70001, 90000
    ids = np.minimum((vocab + 1.0) ** r.random(n) - 1, vocab - 1).astype(np.int64)
    ids[:300] = -1
    dy = r.standard_normal((n, 3)).astype(np.float32)
    got = host(fw.embed_grad(torch.from_numpy(dy).to(dev), torch.from_numpy(ids).to(dev), vocab))
    ref, size = O.embed_grad(dy, ids, vocab, 1.0)
    runs = np.bincount(ids[ids >= 0], minlength=vocab)[:, None]
    assert (np.abs(got - ref) <= (runs + 3) * 2.0 ** -24 * size).all()


def test_example_trains(dev):
    """The operators and the sketch together: both losses fall, sketched gradients keep their angles."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "subspace_preference.py")
    spec = importlib.util.spec_from_file_location("subspace_preference", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    pref, pol, err = ex.main(40)
    assert abs(pref[0] - np.log(2)) < 1e-6  # no difference from the reference yet
    assert pref[-1] < 0.5 * pref[0]
    assert pol[-1] < pol[0]
    assert err < 6 / np.sqrt(ex.D)  # a cosine of two sketched vectors is off by about 1 / sqrt(D)


def test_adamw_many_tensors(dev):
    """More tensors than one launch takes, the norm over all of them."""
    import paper_2402_03994_amd as fw
    sizes = [1 + 37 * k % 611 for k in range(400)]
    opt = fw.AdamW(sizes, decay=[k % 2 for k in range(400)])
    g = [torch.randn(n, device=dev) for n in sizes]
    p = [torch.randn(n, device=dev) for n in sizes]
    before = np.concatenate([host(t) for t in p])
    gh = np.concatenate([t.cpu().numpy() for t in g])
    norm = opt.step(p, g, 1, lr=0.1, eps=1e-6, weight_decay=0.1, max_norm=1.0)
    want = np.sqrt((gh.astype(np.float64) ** 2).sum())
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    s = np.float32(1.0) / (np.float32(float(norm)) + np.float32(1e-6))
    m, v = O.adamw_moments(np.zeros_like(gh), np.zeros_like(gh), gh, 0.9, 0.999, s)
    assert np.array_equal(unpadded(opt.m.cpu().numpy(), sizes), m) and np.array_equal(unpadded(opt.v.cpu().numpy(), sizes), v)
    wd = np.concatenate([np.full(n, 0.1 * (k % 2)) for k, n in enumerate(sizes)])
    ref = O.adamw_param(before, m, v, 1, 0.1, 0.9, 0.999, 1e-6, wd)
    assert (np.abs(np.concatenate([host(t) for t in p]) - ref) <= 2.0 ** -20 * np.abs(ref - before) + 2.0 ** -23 * np.abs(before)).all()


def test_policy_divergence_near_the_reference(dev):
    """u = ref - logp down to 1e-6: the divergence e^u - 1 - u and its derivative e^u - 1 do not lose what u is."""
    import paper_2402_03994_amd as fw
    n, vocab = 64, 300
    x, t = torch.randn(n, vocab, device=dev), torch.randint(0, vocab, (n,), device=dev)
    lp = fw.token_logp(x, t)[0]
    ref = lp + torch.logspace(-6, 0, n, device=dev) * torch.where(torch.arange(n, device=dev) % 2 == 0, 1.0, -1.0)
    zero, one = torch.zeros(n, device=dev), torch.ones(n, device=dev)
    r = fw.policy_loss(x, t, lp, zero, one, ref_logp=ref, kl_coef=1.0)
    assert torch.equal(r.logp, lp)
    u = host(ref) - host(lp)  # exact in fp32
    # expm1 is off by a unit of its last place or two, and the difference is rounded once
    assert (np.abs(host(r.token_loss) - (np.expm1(u) - u)) <= 2.0 ** -21 * np.abs(np.expm1(u))).all()
    d = O.token_logp_grad(host(x), t.cpu().numpy(), -np.expm1(u), 1.0)
    assert (np.abs(host(r.dlogits) - d) <= (2.0 ** -20 + 2 * err_logp(10.0, vocab)) * np.abs(np.expm1(u))[:, None]).all()


@pytest.mark.parametrize("vocab", [2, 65, 3000, 50257, 140003])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_logits_of_any_size(dev, vocab, dt):
    """Rows around values so large that the product with the scale loses the difference, with ties and with entries
    far below, and scales at both ends of the type."""
    import paper_2402_03994_amd as fw
    g = torch.Generator().manual_seed(vocab)
    bases = [1e9, -1e9, 3e8, 4.5e8, -4.5e8, 1e20, -1e20, 3e38, -3e38, 0.0, 7.0]
    rows = len(bases)
    t = torch.randint(0, vocab, (rows,), generator=g)
    c = torch.randn(rows, generator=g)
    for scale in (1.0, 1e-35, 1e35):
        x = torch.tensor(bases)[:, None].repeat(1, vocab).to(dt)
        far = torch.rand(rows, vocab, generator=g) < 0.25
        x = torch.where(far, (torch.tensor(bases)[:, None] - 2 * torch.tensor(bases)[:, None].abs().clamp(max=1e38) * 0.1
                              - 1.0).to(dt), x)
        x[:, : vocab // 2] = torch.where(torch.tensor(bases)[:, None] < 1e37, torch.tensor(-3e38).to(dt), x[:, : vocab // 2])
        if scale < 1.0:
            x = x.clamp(min=0.0)  # differences of finite logits stay finite
        s = float(np.float32(scale))
        xd, td = odd(x, dev, 1, 1), t.to(dev)
        logp, stats = fw.token_logp(xd, td, scale=scale)
        A = exponent_sizes(x, s)
        with np.errstate(all="ignore"):
            want = O.token_logp(x.double().numpy(), t.numpy(), s)
        big = np.abs(want) > 3e38  # beyond fp32
        assert (host(logp)[big] < -3e38).all()
        check_logp(np.where(big, 0.0, host(logp)), np.where(big, 0.0, want), A, vocab, x, s)
        ref = O.token_logp_grad(x.double().numpy(), t.numpy(), c.double().numpy(), s)
        p = O.softmax_rows(x.double().numpy(), s)[0]
        d = fw.token_logp_grad(xd, td, stats, c.to(dev), scale=scale)
        check_grad(host(d), ref, c.double().numpy(), p, A, vocab, s, dt)
        if scale == 1.0:
            ok = np.abs(want) < 80.0  # where the ratio to the old policy is of any use
            w = torch.from_numpy(np.where(ok, c.numpy(), 0.0).astype(np.float32)).to(dev)
            r = fw.policy_loss(xd, td, logp, torch.ones(rows, device=dev), w)
            assert np.array_equal(host(r.logp)[ok], host(logp)[ok])
            cw = -np.where(ok, c.double().numpy(), 0.0)
            ref = O.token_logp_grad(x.double().numpy(), t.numpy(), cw, s)
            check_grad(host(r.dlogits), ref, cw, p, A, vocab, s, dt)


@pytest.mark.parametrize("batch,n,vocab", [(65_000, 4_100, 2_200), (1, (1 << 28) - 8, 1 << 20)])
def test_embed_grad_of_more_than_one_grid(dev, batch, n, vocab):
    """What the ranking (8.4 million workgroups of 512 threads here) and the merging (2^28 entries, 16 threads each) need
    is more than a launch of 2^32 threads takes.  Whole numbers: every sum is exact."""
    import paper_2402_03994_amd as fw
    if batch > 1:
        blocks = batch * 2 * 64 + batch * vocab * 4 // 8192
        assert blocks * 512 >= 1 << 32
    else:
        assert -(-batch * n * 16 // 256) * 256 >= 1 << 32
    g = torch.Generator(device=dev).manual_seed(n)
    ids = torch.randint(0, vocab, (batch, n), generator=g, device=dev, dtype=torch.int32)
    dy = torch.randint(-2, 3, (batch, n, 1), generator=g, device=dev, dtype=torch.int8).to(BF16)
    got = fw.embed_grad(dy, ids, vocab, per_example=True)
    key = (ids + torch.arange(batch, device=dev)[:, None] * vocab).view(-1)
    ref = torch.zeros(batch * vocab, device=dev).index_add_(0, key, dy.view(-1).float())
    assert torch.equal(got.view(-1), ref)


@pytest.mark.parametrize("state", ["f32", "8bit"])
@pytest.mark.parametrize("bits", [0x7FFFFFFF, -1, 0x7FC00000, 0x7F80FFFF])
def test_adamw_random_rounding_keeps_nan(dev, state, bits):
    """A NaN whose bits are all ones has no room for a random addend: bf16 parameters must not come out as zeros."""
    import paper_2402_03994_amd as fw
    n = 4096 + 77
    opt = fw.AdamW([n], state=state, seed=5)
    p = torch.full((n,), 0.5, dtype=BF16, device=dev)
    g = torch.ones(n, device=dev)
    bad = torch.arange(n, device=dev) % 97 == 3
    g.view(torch.int32)[bad] = bits
    opt.step([p], [g], 1, lr=0.125)
    assert torch.isnan(p[bad]).all()
    assert torch.isfinite(p[~bad]).all()
    if state == "f32":  # the same NaN from a moment
        q = torch.full((n,), 0.5, dtype=BF16, device=dev)
        opt.m.zero_()
        opt.v.zero_()
        opt.m[:n].view(torch.int32)[bad] = bits
        opt.step([q], [torch.ones(n, device=dev)], 1, lr=0.125)
        assert torch.isnan(q[bad]).all() and torch.isfinite(q[~bad]).all()


@pytest.mark.parametrize("state,master", [("f32", False), ("8bit", False), ("f32", True), ("8bit", True)])
def test_adamw_quotient_is_rounded_correctly(dev, state, master):
    """A first step from zero parameters with b1 = b2 = 0 and lr = 1 leaves p = -g / (sqrt(g^2) + eps): the square root,
    the sum and the quotient round once each, 3 times 2^-24."""
    import paper_2402_03994_amd as fw
    n = 1 << 20
    gen = torch.Generator().manual_seed(3)
    g = torch.exp(8 * torch.randn(n, generator=gen)).clamp(2.0 ** -20, 2.0 ** 20)
    opt = fw.AdamW([n], state=state)
    p = torch.zeros(n, dtype=BF16 if master else F32, device=dev)
    mast = torch.zeros(n, device=dev) if master else None
    eps = 2.0 ** -6
    opt.step([p], [g.to(dev)], 1, lr=1.0, betas=(0.0, 0.0), eps=eps, weight_decay=0.0, masters=[mast] if master else None)
    v = (g * g).double().numpy()
    ref = -g.double().numpy() / (np.sqrt(v) + eps)
    got = host(mast if master else p)
    assert (np.abs(got - ref) <= 3 * 2.0 ** -24 * 1.000001 * np.abs(ref)).all()


@pytest.mark.parametrize("state", ["f32", "8bit"])
def test_adamw_small_second_moments_under_a_large_correction(dev, state):
    """b2 next to 1 makes the bias correction 1 / sqrt(1 - b2^t) large, and v far below 2^-126 counts beside eps."""
    import paper_2402_03994_amd as fw
    n = 512
    opt = fw.AdamW([n], state=state)
    p, g = torch.zeros(n, dtype=BF16, device=dev), torch.full((n,), 1e-13, device=dev)
    b2 = 1 - 1e-14
    opt.step([p], [g], 1, lr=1.0, betas=(0.0, b2), eps=1e-12, weight_decay=0.0)
    m, v = O.adamw_moments(np.zeros(1, np.float32), np.zeros(1, np.float32), np.full(1, 1e-13, np.float32), 0.0, b2, 1.0)
    assert 0 < v[0] < 2.0 ** -126
    want = float(O.adamw_param(np.zeros(1), m, v, 1, 1.0, 0.0, b2, 1e-12, 0.0)[0])
    assert abs(want + 1 / 11) < 1e-3
    assert (np.abs(host(p) - want) <= 2.0 ** -7 * abs(want)).all()  # up or down to a neighbour in bf16


@pytest.mark.parametrize("scale", [1.0, 0.7])
@pytest.mark.parametrize("vocab,rows", [(300, 5), (2500, 600), (15013, 5), (140003, 3)])
def test_small_entries_of_an_fp32_gradient(dev, vocab, rows, scale):
    """Entries far below the largest keep fp32's precision.  x - m is exact here; an entry p_j rounds in the hardware's
    exponential (2 halves of a unit), its correction, the factor c / z and the product with it, and z = 1.01 at most in
    its last few additions (8): 13 times 2^-24."""
    import paper_2402_03994_amd as fw
    r = np.random.default_rng(vocab)
    x = -r.integers(64 * 16, 64 * 80, (rows, vocab)) / 64.0
    t = r.integers(0, vocab, rows)
    x[np.arange(rows), t] = 0.0
    s = float(np.float32(scale))
    if s < 1:
        x[x < 0] -= 8.0
    xd, td = torch.from_numpy(x.astype(np.float32)).to(dev), torch.from_numpy(t).to(dev)
    p = O.softmax_rows(x, s)[0]
    other = np.arange(vocab)[None, :] != t[:, None]
    one = torch.ones(rows, device=dev)
    logp, stats = fw.token_logp(xd, td, scale=scale)
    d = host(fw.token_logp_grad(xd, td, stats, one, scale=scale))
    tol = 13 * 2.0 ** -24 * s * p
    assert (np.abs(d + s * p) <= tol)[other].all()
    d = host(fw.policy_loss(xd, td, logp, -one, one, scale=scale).dlogits)  # ratio 1: the factor is 1
    assert (np.abs(d + s * p) <= tol)[other].all()


def test_writes_in_place_are_seen_by_autograd(dev):
    """A graph that has saved what a call overwrites refuses its backward pass, as after any in-place operation."""
    import paper_2402_03994_amd as fw
    w = torch.randn(40, 8, device=dev, requires_grad=True)
    t = torch.randint(0, 8, (40,), device=dev)
    v = torch.zeros(40, device=dev)
    stats = fw.token_logp(w.detach(), t)[1]
    offs = torch.tensor([0, 20, 40], device=dev)
    opt = fw.AdamW([(40, 8)])

    def masters():
        p = torch.zeros(40, 8, dtype=BF16, device=dev, requires_grad=True)
        y = p * p
        opt.step([p], [torch.ones(40, 8, device=dev)], 1, lr=0.1, masters=[w.detach()])
        with pytest.raises(RuntimeError, match="inplace"):
            y.sum().backward()

    d = lambda: w.detach()  # noqa: E731  (shares the version of w)
    for write in (lambda: opt.step([w], [torch.ones(40, 8, device=dev)], 1, lr=0.1), masters,
                  lambda: fw.embed(torch.randn(9, 8, device=dev), t, out=d()),
                  lambda: fw.embed_grad(torch.randn(5, 8, device=dev), t[:5], 40, out=d()),
                  lambda: fw.token_logp_grad(d(), t, stats, v, out=d()),
                  lambda: fw.policy_loss(d(), t, v, v, v, out=d()),
                  lambda: fw.preference_loss(d(), t, offs, v, out=d())):
        y = w * w
        write()
        with pytest.raises(RuntimeError, match="inplace"):
            y.sum().backward()
    y = w * w  # what only reads changes nothing
    fw.policy_loss(d(), t, v, v, v)
    fw.embed(d(), t)
    y.sum().backward()


def test_adamw_refuses_what_fp32_does_not_hold(dev):
    """The step's numbers are fp32: an eps that becomes 0 would make 0 / 0 of a zero gradient, a rate that overflows NaN."""
    import paper_2402_03994_amd as fw
    opt, p, g = fw.AdamW([70]), [torch.ones(70, device=dev)], [torch.zeros(70, device=dev)]
    for kw in (dict(eps=1e-50), dict(eps=1e39), dict(lr=1e39), dict(lr=1e20, weight_decay=1e20),
               dict(lr=1e38, betas=(0.999, 0.999))):
        with pytest.raises(fw.SketchError):
            opt.step(p, g, 1, **{**dict(lr=0.1), **kw})
    assert (p[0] == 1).all() and not opt.m.any()
    for eps in (1e-39, 1e38):
        opt.step(p, g, 1, lr=0.1, eps=eps, weight_decay=0.0, max_norm=float("inf"))
        assert (p[0] == 1).all()


def test_adamw_refuses_lists_of_other_things(dev):
    import paper_2402_03994_amd as fw
    opt, p, g = fw.AdamW([5, 7]), [torch.ones(5, device=dev), torch.ones(7, device=dev)], None
    g = [torch.ones_like(t) for t in p]
    for bad in ([g[0], None], [None, None], [], None, g[0], [g[0], 3.0], [g[0], g[1].cpu()], [g[0], g[1].bfloat16()]):
        with pytest.raises(ValueError):
            opt.step(p, bad, 1, lr=0.1)
        with pytest.raises(ValueError):
            opt.step(bad, g, 1, lr=0.1)
    assert all((t == 1).all() for t in p)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_targets_too_far_for_a_difference(dev, dt):
    """x_t - m overflows while scale (x_t - m) does not."""
    import paper_2402_03994_amd as fw
    x = torch.full((3, 100), -3e38).to(dt)
    x[:, 7] = 3e38
    x[1] = -float("inf")
    x[1, 7] = 3e38
    t = torch.tensor([5, 5, 7])
    for scale in (0.25, 2.0 ** -100, 2.0 ** -120):
        logp, stats = fw.token_logp(x.to(dev), t.to(dev), scale=scale)
        want = O.token_logp(x.double().numpy(), t.numpy(), scale)
        assert np.isfinite(want[[0, 2]]).all() and want[1] == -np.inf
        got = host(logp)
        assert got[1] == -np.inf and (np.abs(got - want)[[0, 2]] <= 2.0 ** -22 * np.abs(want[[0, 2]])).all()
        one = torch.ones(3, device=dev)
        d = fw.policy_loss(x.to(dev), t.to(dev), logp.clamp(min=-3e38), one, one, scale=scale)
        assert np.array_equal(host(d.logp), got)


def test_stream_without_the_short_way(dev, monkeypatch):
    """torch's own function for the raw stream is a shortcut: without it the public way gives the same stream."""
    import paper_2402_03994_amd as fw
    from paper_2402_03994_amd import sketch
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        want = sketch._stream_ptr(dev)
        assert want == side.cuda_stream
        monkeypatch.setattr(sketch, "_raw_stream", None)
        assert sketch._stream_ptr(dev) == want
        x = fw.embed(torch.ones(3, 4, device=dev), torch.tensor([0, 2], device=dev))
    side.synchronize()
    assert (x == 1).all()
    assert sketch._stream_ptr(dev) == torch.cuda.current_stream(dev).cuda_stream


# a vocabulary and a number of rows for each shape that a row's threads take (vectors of 4 or 8 columns by the type), with
# gradients on both sides of the size from which they are stored past the caches
SHAPES = [(F32, 1500, 515), (F32, 2500, 1030), (F32, 6007, 27), (F32, 15013, 27), (F32, 30522, 27), (F32, 32000, 530),
          (BF16, 3001, 515), (BF16, 5003, 1030), (BF16, 20011, 27), (BF16, 30522, 27), (BF16, 32000, 1061)]


@pytest.mark.parametrize("dt,vocab,rows", SHAPES)
def test_losses_of_every_row_shape(dev, dt, vocab, rows):
    import paper_2402_03994_amd as fw
    x, t = make_logits(rows, vocab, dt, vocab + rows)
    t[[k for k in range(rows) if k % 9 in (4, 6)]] = -1  # logs of 0: looked at elsewhere
    old, adv, w, ref = policy_inputs(x, t, vocab)
    f = lambda v: v.double().numpy()  # noqa: E731
    xh, th = f(x), t.numpy()
    lo, kl = float(np.float32(0.2)), float(np.float32(0.2))
    loss, logp, tok, dref = O.policy(xh, th, f(old), f(adv), f(w), f(ref), lo, lo, kl, 1.0)
    live = (th >= 0) & (th < vocab) & (f(w) != 0)
    A, p = exponent_sizes(x, 1.0), np.nan_to_num(O.softmax_rows(xh, 1.0)[0])
    z = lambda v: np.where(live, v, 0.0)  # noqa: E731
    e = err_logp(A.max(1), vocab) + (np.abs(logp) + 4) * 2.0 ** -22
    size = z(np.abs(f(adv)) * np.exp(logp - f(old)) + kl * (2 + np.exp(f(ref) - logp)))
    c = z(f(w)) * O.policy_tokens(z(logp), z(f(old)), z(f(adv)), z(f(ref)), lo, lo, kl)[1]
    rel = (2 * err_logp(A, vocab) + 2 * err_logp(0.0, vocab)) * p
    tol = np.abs(c)[:, None] * rel + (z(f(w)) * size * (e + 2.0 ** -22))[:, None] + (HALF[dt] + 2.0 ** -22) * np.abs(dref) + 1e-37
    for lead, pad in ((0, 0), (1, 3)):
        xd, args = odd(x, dev, lead, pad), [v.to(dev) for v in (t, old, adv, w)]
        got = fw.policy_loss(xd, *args, ref_logp=ref.to(dev), kl_coef=0.2)
        check_logp(host(got.logp), logp, A, vocab, x, 1.0)
        assert (np.abs(host(got.token_loss) - tok) <= size * e + 2.0 ** -22 * size).all()
        assert abs(float(got.loss) - loss) <= (z(f(w)) * (size * e + 2.0 ** -22 * size)).sum() + 2.0 ** -24 * abs(loss)
        assert (np.abs(host(got.dlogits) - dref) <= tol).all()
        lp, stats = fw.token_logp(xd, args[0])
        check_logp(host(lp), O.token_logp(xh, th, 1.0), A, vocab, x, 1.0)
        cd = torch.from_numpy(np.where(live, c, 0.0).astype(np.float32))
        d = fw.token_logp_grad(xd, args[0], stats, cd.to(dev))
        dlog = O.token_logp_grad(xh, th, f(cd), 1.0)
        assert (np.abs(host(d) - dlog) <= np.abs(f(cd))[:, None] * rel + (HALF[dt] + 2.0 ** -22) * np.abs(dlog) + 1e-37).all()
        keep = xd.clone()
        assert torch.equal(fw.token_logp_grad(xd, args[0], stats, cd.to(dev), out=xd), d)  # in place
        xd.copy_(keep)
        again = fw.policy_loss(xd, *args, ref_logp=ref.to(dev), kl_coef=0.2, out=xd)
        assert torch.equal(again.dlogits, got.dlogits) and torch.equal(again.loss, got.loss)


@pytest.mark.parametrize("n,vocab,width,dt", [(300_001, 5000, 3, F32), (600_001, 5000, 3, BF16), (140_001, 300, 515, BF16),
                                              (280_001, 300, 515, F32), (600_001, 7, 8, BF16)])
def test_embed_grad_in_larger_tiles(dev, n, vocab, width, dt):
    """Long batches are added up 32 and 64 tokens at a time.  The entries are small whole numbers, so that every sum is
    exact in fp32, whatever its order."""
    import paper_2402_03994_amd as fw
    g = torch.Generator(device=dev).manual_seed(n)
    ids = ((vocab + 1.0) ** torch.rand(n, generator=g, device=dev, dtype=torch.float64) - 1).long().clamp_(0, vocab - 1)
    ids[torch.rand(n, generator=g, device=dev) < 0.3] = vocab // 2  # an id that crosses thousands of tiles
    ids[torch.rand(n, generator=g, device=dev) < 0.05] = -1
    ids[-70:] = vocab
    dy = torch.randint(-3, 4, (n, width), generator=g, device=dev).to(dt)
    live = (ids >= 0) & (ids < vocab)
    ref = torch.zeros(vocab, width, dtype=torch.float64, device=dev).index_add_(0, ids[live], dy[live].double())
    assert torch.equal(fw.embed_grad(dy, ids, vocab, scale=0.5).double(), 0.5 * ref)
    out = torch.randint(-3, 4, (vocab, width), generator=g, device=dev).float()
    want = 0.5 * ref + out
    assert torch.equal(fw.embed_grad(dy, ids.int(), vocab, scale=0.5, out=out, accumulate=True).double(), want)


@pytest.mark.parametrize("odt", [F32, BF16])
@pytest.mark.parametrize("lead", range(1, 9))
def test_embed_grad_zeroes_its_own_memory_alone(dev, odt, lead):
    """An output at any address, between entries that are somebody else's."""
    import paper_2402_03994_amd as fw
    n, vocab, width = 1100, 301, 7
    buf = torch.full((lead + vocab * width + 9,), 5.0, dtype=odt, device=dev)
    out = buf[lead:lead + vocab * width].view(vocab, width)
    ids = torch.arange(n, device=dev) % 50 * 3
    got = fw.embed_grad(torch.ones(n, width, device=dev), ids, vocab, out=out)
    assert got.data_ptr() == out.data_ptr()
    ref = torch.zeros(vocab, device=dev).index_add_(0, ids, torch.ones(n, device=dev))
    assert torch.equal(out.float(), ref[:, None].expand(vocab, width))
    assert (buf[:lead] == 5).all() and (buf[lead + vocab * width:] == 5).all()


@pytest.mark.parametrize("state", ["f32", "8bit"])
@pytest.mark.parametrize("pdt,gdt,master", [(F32, F32, False), (F32, BF16, False), (BF16, BF16, False), (BF16, F32, True),
                                            (BF16, BF16, True), (BF16, F32, False)])
def test_adamw_of_two_launches(dev, state, pdt, gdt, master):
    """180 tensors of 234 chunks: two launches that each form the norm, with every kind of state and parameter."""
    assert len(SIZES) * 18 > 160 and sum((n + 4095) // 4096 for n in SIZES) * 18 <= 256
    two_launches(dev, state, pdt, gdt, master, SIZES * 18)


def two_launches(dev, state, pdt, gdt, master, sizes):
    import paper_2402_03994_amd as fw
    total, seed = sum(sizes), 2 ** 40 + 5
    r = np.random.default_rng(12)
    decay = [float(k % 3 > 0) for k in range(len(sizes))]
    split = lambda t: list(torch.split(t, sizes))  # noqa: E731
    p0 = torch.from_numpy(r.standard_normal(total).astype(np.float32))
    buf = p0.to(pdt).to(dev)
    mast = p0.to(dev) if master else None
    hp = p0.double().numpy() if master else host(buf)
    opt = fw.AdamW(sizes, state=state, decay=decay, seed=seed)
    m, v = np.zeros(total, np.float32), np.zeros(total, np.float32)
    wd = np.concatenate([np.full(n, 0.1 * d) for n, d in zip(sizes, decay)])
    words = lambda k, step: np.concatenate([O.adamw_words(n, step, l, seed)[k] for l, n in enumerate(sizes)])  # noqa: E731
    for step in (1, 2):
        g = torch.from_numpy((r.standard_normal(total) * 0.01).astype(np.float32)).to(gdt)
        norm = float(opt.step(split(buf), split(g.to(dev)), step, lr=0.01, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1,
                              masters=split(mast) if master else None, max_norm=0.5))
        gh = g.float().numpy()
        want = np.sqrt((gh.astype(np.float64) ** 2).sum())
        assert want > 0.5 and abs(norm - want) <= 2.0 ** -23 * want
        s = min(np.float32(1.0), np.float32(0.5) / (np.float32(norm) + np.float32(1e-6)))
        m, v = O.adamw_moments(m, v, gh, 0.9, 0.99, s)
        ref = O.adamw_param(hp, m, v, step, 0.01, 0.9, 0.99, 1e-6, wd)
        tol = 2.0 ** -20 * np.abs(ref - hp) + 2.0 ** -23 * np.abs(hp)
        if state == "8bit":
            for x, k, top, code, exp in ((m, 0, 15, opt.m, opt.m_exp), (v, 1, 31, opt.v, opt.v_exp)):
                u = padded(words(k, step).astype(np.int64), sizes).reshape(-1, 64)
                c, e = O.encode8(padded(x, sizes).reshape(-1, 64), top, u)
                assert np.array_equal(exp.cpu().numpy(), e) and np.array_equal(code.cpu().numpy().reshape(-1, 64), c)
                x[:] = unpadded(O.decode8(c, e, top).reshape(-1), sizes)
        else:
            assert np.array_equal(unpadded(opt.m.cpu().numpy(), sizes), m)
            assert np.array_equal(unpadded(opt.v.cpu().numpy(), sizes), v)
        if pdt == BF16 and not master:
            u = words(2, step)
            a, b = (np.abs(((((ref + k * np.sign(ref) * tol).astype(np.float32).view(np.uint32).astype(np.int64) + u) >> 16 << 16)
                            .astype(np.uint32)).view(np.float32).astype(np.float64)) for k in (-1, 1))
            hp = host(buf)
            assert (((a <= np.abs(hp)) & (np.abs(hp) <= b)) | (np.abs(ref) < 1e-6)).all()
        else:
            hp = host(mast if master else buf)
            assert (np.abs(hp - ref) <= tol).all()
            assert not master or torch.equal(buf, mast.to(BF16))


@pytest.mark.parametrize("dt,vocab,rows", [(F32, 1501, 25000), (BF16, 5003, 15000), (F32, 50257, 700), (BF16, 50257, 1400),
                                           (BF16, 32000, 2300)])
def test_large_outputs_are_those_of_their_thirds(dev, dt, vocab, rows):
    """Gradients and lookups that are stored past the caches, in place too, against calls whose outputs are not."""
    import paper_2402_03994_amd as fw
    g = torch.Generator(device=dev).manual_seed(rows)
    x = torch.randn(rows, vocab, generator=g, device=dev).mul_(2).to(dt)
    t = torch.randint(-1, vocab, (rows,), generator=g, device=dev)
    old, adv, w = (torch.randn(rows, generator=g, device=dev) for _ in range(3))
    third = -(-rows // 3)
    assert third * vocab * x.element_size() < 64 << 20 < x.numel() * x.element_size()
    lp, stats = fw.token_logp(x, t)
    old = lp - 0.1 * old
    parts = [slice(k, min(k + third, rows)) for k in range(0, rows, third)]
    for scale in (1.0, 0.5):
        whole = fw.policy_loss(x, t, old, adv, w, scale=scale).dlogits
        for s in parts:
            assert torch.equal(whole[s], fw.policy_loss(x[s], t[s], old[s], adv[s], w[s], scale=scale).dlogits)
    d = fw.token_logp_grad(x, t, stats, w)
    for s in parts:
        assert torch.equal(d[s], fw.token_logp_grad(x[s], t[s], stats[s], w[s]))
    ids = torch.randint(-1, rows, (rows,), generator=g, device=dev)
    e = fw.embed(x, ids, scale=0.7)
    for s in parts:
        assert torch.equal(e[s], fw.embed(x, ids[s], scale=0.7))
    y = x.clone()
    fw.token_logp_grad(y, t, stats, w, out=y)
    assert torch.equal(y, d)
    y.copy_(x)
    fw.policy_loss(y, t, old, adv, w, scale=0.5, out=y)
    assert torch.equal(y, whole)


def test_errors_of_earlier_calls_are_not_reported(dev):
    """What an unrelated call to the runtime has left as its last error is none of the next operator's."""
    import ctypes

    import paper_2402_03994_amd as fw
    with open("/proc/self/maps") as maps:
        path = next(line.split()[-1] for line in maps if "libamdhip64.so" in line)
    hip = ctypes.CDLL(path)
    w, t = torch.randn(8, 4, device=dev), torch.tensor([1, 7, 3], device=dev)
    opt, g = fw.AdamW([(8, 4)]), torch.ones(8, 4, device=dev)
    want, low = w[t].clone(), t % 4
    for call in (lambda: torch.equal(fw.embed(w, t), want), lambda: fw.embed_grad(want, t, 8).abs().sum() > 0,
                 lambda: torch.isfinite(fw.token_logp(w[:3], low)[0]).all(), lambda: opt.step([w], [g], 1, lr=0.1) is None):
        assert hip.hipSetDevice(99) != 0  # refused by the runtime, nothing is queued
        assert call()
