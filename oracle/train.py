"""fp64 definitions of the training-step operators (include/sketch_train.h), in numpy.

The 8-bit AdamW state is defined by fp32 arithmetic and a rounding with given random words; that part is evaluated
in fp32 and integers as the header states it, everything else in fp64.
"""
from __future__ import annotations

import numpy as np


def embed(weight, ids, scale):
    w = np.asarray(weight, dtype=np.float64)
    ids = np.asarray(ids)
    live = (ids >= 0) & (ids < len(w))
    return np.where(live[..., None], scale * w[np.where(live, ids, 0)], 0.0)


def embed_grad(dy, ids, vocab, scale):
    """dy [n, width], ids [n] -> (gradient [vocab, width], sum of |terms|)."""
    dy = np.asarray(dy, dtype=np.float64)
    out, size = np.zeros((vocab, dy.shape[1])), np.zeros((vocab, dy.shape[1]))
    live = (np.asarray(ids) >= 0) & (np.asarray(ids) < vocab)
    np.add.at(out, np.asarray(ids)[live], scale * dy[live])
    np.add.at(size, np.asarray(ids)[live], np.abs(scale * dy[live]))
    return out, size


def softmax_rows(x, scale):
    """(p, log p) of each row in fp64; a row without an entry above -inf has p = 0 and log p = -inf."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(all="ignore"):
        m = x.max(1, keepdims=True)
        m = np.where(m == -np.inf, 0.0, m)
        a = (x - m) * scale
        z = np.exp(a).sum(1, keepdims=True)
        p = np.where(z == 0, 0.0, np.exp(a) / z)
        lp = np.where(z == 0, -np.inf, a - np.log(z))
    return p, lp


def token_logp(x, targets, scale):
    t = np.asarray(targets)
    live = (t >= 0) & (t < x.shape[1])
    out = np.zeros(len(t))
    if live.any():
        lp = softmax_rows(np.asarray(x)[live], scale)[1]
        out[live] = lp[np.arange(live.sum()), t[live]]
    return out


def token_logp_grad(x, targets, dlogp, scale):
    t, c = np.asarray(targets), np.asarray(dlogp, dtype=np.float64)
    out = np.zeros(x.shape)
    live = (t >= 0) & (t < x.shape[1])
    live &= np.where(live, c, 0.0) != 0
    if live.any():
        p, lp = softmax_rows(np.asarray(x)[live], scale)
        one = np.zeros_like(p)
        one[np.arange(len(p)), t[live]] = 1.0
        empty = (lp == -np.inf).all(1)
        out[live] = np.where(empty[:, None], 0.0, c[live][:, None] * scale * (one - p))
    return out


def policy_tokens(logp, old, adv, ref, lo, hi, kl):
    """(l_t, d l_t / d logp_t)."""
    logp, old, adv = (np.asarray(v, dtype=np.float64) for v in (logp, old, adv))
    r = np.exp(logp - old)
    free, held = adv * r, adv * np.clip(r, 1 - lo, 1 + hi)
    l, d = -np.minimum(free, held), np.where(free <= held, -free, 0.0)
    if kl:
        u = np.asarray(ref, dtype=np.float64) - logp
        l, d = l + kl * (np.expm1(u) - u), d - kl * np.expm1(u)
    return l, d


def policy(x, targets, old, adv, weights, ref, lo, hi, kl, scale):
    """(loss, logp, l_t, dlogits)."""
    t, w = np.asarray(targets), np.asarray(weights, dtype=np.float64)
    live = (t >= 0) & (t < x.shape[1]) & (w != 0)
    logp = token_logp(x, np.where(live, t, -1), scale)
    l, d = np.zeros(len(t)), np.zeros(len(t))
    pick = lambda v: None if v is None else np.asarray(v)[live]  # noqa: E731
    l[live], d[live] = policy_tokens(logp[live], pick(old), pick(adv), pick(ref), lo, hi, kl)
    c = np.where(live, w, 0.0) * d
    return (np.where(live, w, 0.0) * l).sum(), logp, l, token_logp_grad(x, np.where(live, t, -1), c, scale)


def preference(x, targets, offsets, ref, beta, eps, average, scale):
    """(loss, seq_logp, pair_loss, dlogits)."""
    t, o = np.asarray(targets), np.asarray(offsets)
    live = (t >= 0) & (t < x.shape[1])
    logp = token_logp(x, t, scale)
    seq, gap, share = [], [], []
    for a, b in zip(o, o[1:]):
        k = live[a:b]
        n = max(1, int(k.sum())) if average else 1
        seq.append(logp[a:b][k].sum() / n)
        gap.append((logp[a:b][k] - np.asarray(ref, dtype=np.float64)[a:b][k]).sum() / n)
        share.append(1.0 / n)
    d = beta * (np.array(gap[0::2]) - np.array(gap[1::2]))
    pair = (1 - eps) * np.logaddexp(0, -d) + eps * np.logaddexp(0, d)
    sig = lambda u: np.exp(-np.logaddexp(0, -u))  # noqa: E731
    c = -beta / len(d) * ((1 - eps) * sig(-d) - eps * sig(d))
    rowc = np.zeros(len(t))
    for i, (a, b) in enumerate(zip(o, o[1:])):
        rowc[a:b] = (c[i // 2] if i % 2 == 0 else -c[i // 2]) * share[i]
    return pair.mean(), np.array(seq), pair, token_logp_grad(x, t, np.where(live, rowc, 0.0), scale)


# --- AdamW ------------------------------------------------------------------------------------------------
def philox(q, step, layer, stream, seed):
    """Philox4x32-10 at the counters (q, step, layer, stream): uint32 words [..., 4]."""
    m = np.uint64(0xFFFFFFFF)
    q = np.asarray(q, dtype=np.uint64)
    c = [q & m, np.full_like(q, step), np.full_like(q, layer), np.full_like(q, stream)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & m, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, -1).astype(np.uint32)


def encode8(x, top, u):
    """Codes and exponent bytes of fp32 x [blocks, 64], rounded with the 16-bit random numbers u."""
    bits = np.abs(x).view(np.uint32)
    big = bits.max(1).astype(np.int64)
    eb = np.where(big >= 0x7F800000, 255, np.minimum((big + 0x0FFFFF) >> 23, 255))
    with np.errstate(all="ignore"):
        y = np.ldexp(np.abs(x), (top - eb)[:, None].astype(np.int32)).astype(np.float32)
    code = (y.view(np.uint32).astype(np.int64) + (u.astype(np.int64) << 4 | 8)) >> 20
    if top == 15:
        code |= (x.view(np.uint32) >> 31).astype(np.int64) << 7
    return np.where((eb == 255)[:, None], 0, code).astype(np.uint8), eb.astype(np.uint8)


def decode8(code, eb, top):
    c = code.astype(np.uint32)
    y = ((c & np.uint32(0x7F if top == 15 else 0xFF)) << np.uint32(20)).view(np.float32)
    y = np.ldexp(y, (eb.astype(np.int32) - top)[:, None]).astype(np.float32)
    if top == 15:
        y = np.where(c & 0x80, -y, y)
    return np.where((eb == 255)[:, None], np.float32(np.nan), y).astype(np.float32)


def adamw_moments(m, v, g, b1, b2, s):
    """The two moments in fp32, every product and sum rounded by itself (g, m, v fp32, s fp32)."""
    f = np.float32
    with np.errstate(all="ignore"):
        g = g * f(s)
        m = m * f(b1) + g * f(1.0 - b1)
        v = v * f(b2) + (g * g) * f(1.0 - b2)
    return m, v


def adamw_param(p, m, v, step, lr, b1, b2, eps, wd):
    """The parameter in fp64 from the (new) moments."""
    p, m, v = (np.asarray(t, dtype=np.float64) for t in (p, m, v))
    with np.errstate(all="ignore"):
        return p - lr * wd * p - lr * (m / (1 - b1 ** step)) / (np.sqrt(v / (1 - b2 ** step)) + eps)


def adamw_words(n, step, layer, seed):
    """The 16-bit random numbers (m, v, p) of elements 0 .. n-1 of tensor `layer` at a step."""
    i = np.arange(n)
    w = philox(i // 4, step, layer, 11, seed)[i, i % 4]
    p = philox(i // 8, step, layer, 12, seed)[i, (i // 2) % 4]
    return w >> 16, w & 0xFFFF, np.where(i % 2, p >> 16, p & 0xFFFF)


def linear_logp(hidden, weight, targets, scale):
    """log softmax(scale hidden weight^T)[targets] by rows."""
    t = np.asarray(targets)
    live = (t >= 0) & (t < len(weight))
    out = np.zeros(len(t))
    if live.any():
        x = np.asarray(hidden, dtype=np.float64)[live] @ np.asarray(weight, dtype=np.float64).T
        out[live] = softmax_rows(x, scale)[1][np.arange(live.sum()), t[live]]
    return out


def linear_logp_grad(hidden, weight, targets, dlogp, scale, batch=1):
    """(dhidden [T, width], dweight [batch, vocab, width], g [T, vocab] at the logits, p [T, vocab])."""
    t, c = np.asarray(targets), np.asarray(dlogp, dtype=np.float64)
    W = np.asarray(weight, dtype=np.float64)
    live = (t >= 0) & (t < len(W))
    live &= np.where(live, c, 0.0) != 0
    h = np.where(live[:, None], np.asarray(hidden, dtype=np.float64), 0.0)
    x = h @ W.T
    g = token_logp_grad(x, np.where(live, t, -1), c, scale)
    p = np.where(live[:, None], softmax_rows(x, scale)[0], 0.0)
    n = len(t) // batch
    dw = np.stack([g[b * n:b * n + n].T @ h[b * n:b * n + n] for b in range(batch)])
    return g @ W, dw, g, p


# --- dropout and a router's balance loss ------------------------------------------------------------------
def dropout_words(n, step, site, seed):
    """The 16-bit random numbers of elements 0 .. n-1."""
    i = np.arange(n)
    w = philox(np.arange((n + 7) // 8), step, site, 13, seed)[i // 8, (i // 2) % 4]
    return np.where(i % 2, w >> 16, w & 0xFFFF)


def dropout(x, p, seed, step, site, residual=None):
    """(out, kept), x and residual of any shape."""
    x = np.asarray(x, dtype=np.float64)
    t = int(np.floor(65536 * p + 0.5))
    kept = (dropout_words(x.size, step, site, seed) >= t).reshape(x.shape)
    out = np.where(kept, np.where(kept, x, 0.0) * (65536.0 / (65536 - t) if t < 65536 else 0.0), 0.0)
    return (out if residual is None else out + np.asarray(residual, dtype=np.float64)), kept


def balance_loss(x, ids, coef):
    """(loss, counts, probs, dlogits)."""
    ids = np.asarray(ids)
    E = np.shape(x)[1]
    valid = (ids >= 0) & (ids < E)
    live = valid.any(1)
    n = live.sum()
    counts = np.bincount(ids[valid].astype(np.int64), minlength=E)
    if n == 0:
        return 0.0, counts, np.zeros(E), np.zeros(np.shape(x))
    p = softmax_rows(np.where(live[:, None], np.asarray(x, dtype=np.float64), 0.0), 1.0)[0] * live[:, None]
    f, probs = counts / (n * ids.shape[1]), p.sum(0) / n
    return coef * E * (f * probs).sum(), counts, probs, coef * E / n * p * (f - (p @ f)[:, None])
