"""The fp64 definitions of the training-step operators, pinned by differences, closed forms and statistics."""
import numpy as np
import pytest

from oracle import train as O


def numeric(f, x, h=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = h
        g[i] = (f(x + e) - f(x - e)) / (2 * h)
    return g


def data(rows, vocab, seed):
    r = np.random.default_rng(seed)
    return r, r.standard_normal((rows, vocab)) * 2, r.integers(0, vocab, rows)


# central differences: h^2 f''' / 6 (under 1e-9 here) and 1e-16 / h of rounding
TOL = 1e-8


@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_logp_gradient_against_differences(scale):
    r, x, t = data(4, 7, 0)
    t[1] = -100
    c = r.standard_normal(4)
    g = O.token_logp_grad(x, t, c, scale)
    n = numeric(lambda y: (c * O.token_logp(y, t, scale)).sum(), x)
    assert np.abs(g - n).max() < TOL


@pytest.mark.parametrize("kl", [0.0, 0.3])
def test_policy_gradient_against_differences(kl):
    r, x, t = data(9, 5, 1)
    t[4] = 7
    lp = O.token_logp(x, np.where(t < 5, t, -1), 1.3)
    old = lp - np.array([0.5, -0.5, 0.05, 0.0, 0.1, 0.5, -0.5, -0.05, 0.1])  # outside and inside the bounds
    adv = np.array([1.0, 1.0, 1.0, 1.0, 1.0, -1.0, -1.0, -1.0, 0.0])
    w, ref = r.random(9), lp + 0.3 * r.standard_normal(9)
    w[3] = 0.0
    g = O.policy(x, t, old, adv, w, ref, 0.2, 0.2, kl, 1.3)[3]
    n = numeric(lambda y: O.policy(y, t, old, adv, w, ref, 0.2, 0.2, kl, 1.3)[0], x)
    assert np.abs(g - n).max() < TOL
    assert (g[3] == 0).all() and (g[4] == 0).all()


@pytest.mark.parametrize("average", [False, True])
@pytest.mark.parametrize("eps", [0.0, 0.1])
def test_preference_gradient_against_differences(average, eps):
    r, x, t = data(11, 6, 2)
    t[[0, 5]] = -1
    o = np.array([0, 3, 5, 5, 10])  # an empty text, and a last row outside all of them
    ref = r.standard_normal(11) - 2
    g = O.preference(x, t, o, ref, 0.4, eps, average, 1.0)[3]
    n = numeric(lambda y: O.preference(y, t, o, ref, 0.4, eps, average, 1.0)[0], x)
    assert np.abs(g - n).max() < TOL
    assert (g[10] == 0).all()


def test_embed_gradient_is_the_transpose():
    r = np.random.default_rng(3)
    w, dy, ids = r.standard_normal((9, 4)), r.standard_normal((20, 4)), r.integers(-2, 11, 20)
    a = (O.embed(w, ids, 1.5) * dy).sum()
    b = (O.embed_grad(dy, ids, 9, 1.5)[0] * w).sum()
    assert abs(a - b) < 1e-12


@pytest.mark.parametrize("top", [15, 31])
def test_codes_are_kept_and_bracket_what_they_stand_for(top):
    r = np.random.default_rng(4)
    x = (r.standard_normal((50, 64)) * np.exp(3 * r.standard_normal((50, 64)))).astype(np.float32)
    x = x if top == 15 else np.abs(x)
    lo = O.decode8(*O.encode8(x, top, np.zeros(x.shape, np.int64)), top)
    hi = O.decode8(*O.encode8(x, top, np.full(x.shape, 0xFFFF)), top)
    assert (np.abs(lo) <= np.abs(x)).all() and (np.abs(hi) >= np.abs(x) * (1 - 2.0 ** -16)).all()
    # neighbours: an eighth of the value apart, or of the smallest normal one
    big = np.abs(x).max(1, keepdims=True)
    assert (np.abs(hi - lo) <= np.maximum(np.abs(x), big * 2.0 ** (2 - top)) / 8).all()
    c, e = O.encode8(lo, top, np.full(x.shape, 0xFFFF))  # what a code stands for stays
    assert np.array_equal(O.decode8(c, e, top), lo)


def test_rounding_has_the_right_mean():
    r = np.random.default_rng(5)
    x = r.standard_normal((1, 64)).astype(np.float32)
    n, total = 4000, np.zeros((1, 64))
    for k in range(n):
        total += O.decode8(*O.encode8(x, 15, r.integers(0, 1 << 16, (1, 64))), 15)
    step = np.maximum(np.abs(x), np.abs(x).max() * 2.0 ** -13) / 8
    assert (np.abs(total / n - x) < 5 * step / 2 / np.sqrt(n)).all()  # the variance is at most (step / 2)^2


def test_philox_words_match_the_c_oracle():
    kat = [[int(w, 16) for w in line.split()] for line in open(__file__.replace("test_oracle_train.py",
           "golden/philox4x32_10_kat.txt")) if line.strip() and not line.startswith("#")]
    for row in kat:
        c, k, want = row[:4], row[4:6], row[6:10]
        got = O.philox(np.array([c[0]]), c[1], c[2], c[3], k[0] | k[1] << 32)[0]
        assert [int(v) for v in got] == want
