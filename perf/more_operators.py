"""Performance cases of further training-step operators: log-probabilities of tokens straight from hidden states and the
output matrix with their gradients, dropout whose mask is drawn again where it is needed, and the balance loss of a
router with its counts and gradient.

Sizes follow the library's own workloads (GPT-2-small, a 1.3B decoder and Llama-3-8B tensors); draw() spreads them over
vocabularies, widths, lengths, batches, experts and data types, odd sizes among them.

The plain forms are elementary torch operations in 32 bits, rounded once at the end. exact() evaluates the
definitions in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False
F32, BF16 = "f32", "bf16"
TORCH = {F32: torch.float32, BF16: torch.bfloat16}
DEV = "cuda"
SEED, STREAM = 11, 13  # of the dropout masks


# --- the cases --------------------------------------------------------------------------------------------
def listed():
    return [
        # how likely one sampled token was: one row against GPT-2's output matrix
        dict(name="linear_one", op="linear", B=1, T=1, vocab=50257, width=768, grad=False, per_example=False, scale=1.0, dtype=BF16),
        # the scores of a few long texts
        dict(name="linear_scores_f32", op="linear", B=1, T=2000, vocab=50257, width=768, grad=False, per_example=False, scale=1.0,
             dtype=F32),
        # a short text through a small model of an odd width
        dict(name="linear_short", op="linear", B=1, T=61, vocab=8000, width=250, grad=True, per_example=False, scale=0.7, dtype=F32),
        # supervised fine-tuning of GPT-2, prompts masked
        dict(name="linear_sft_bf16", op="linear", B=1, T=4096, vocab=50257, width=768, grad=True, per_example=False, scale=1.0,
             dtype=BF16),
        # per-example gradients of GPT-2's output matrix, as the sketches of data attribution take them
        dict(name="linear_examples", op="linear", B=8, T=257, vocab=50257, width=768, grad=True, per_example=True, scale=1.0,
             dtype=F32),
        # a packed batch of a large-vocabulary model
        dict(name="linear_packed_bf16", op="linear", B=1, T=8192, vocab=128256, width=4096, grad=True, per_example=False, scale=1.0,
             dtype=BF16),
        # the embedding of one token
        dict(name="dropout_one", op="dropout", T=1, width=768, p=0.1, grad=False, residual=False, dtype=F32),
        # the end of a block over a long packed batch, with the residual stream
        dict(name="dropout_block_bf16", op="dropout", T=32768, width=4096, p=0.1, grad=False, residual=True, dtype=BF16),
        # the gradient through it in a small model of an odd width
        dict(name="dropout_grad", op="dropout", T=1023, width=1001, p=0.25, grad=True, residual=False, dtype=F32),
        # a short text through a router of eight experts
        dict(name="balance_short", op="balance", T=61, experts=8, k=2, dtype=F32),
        # an odd number of experts
        dict(name="balance_odd", op="balance", T=5000, experts=60, k=4, dtype=F32),
        # a large batch over many experts
        dict(name="balance_batch_bf16", op="balance", T=65536, experts=256, k=8, dtype=BF16),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def _width(rng, a, b):
    """A model width: mostly multiples of 64, now and then any number."""
    w = _log(rng, a, b)
    return w if rng.random() < 0.3 else max(64, w // 64 * 64)


def _one(rng):
    op, dt = rng.choice(["linear", "linear", "dropout", "balance"]), rng.choice([F32, BF16])
    if op == "linear":
        grad = rng.random() < 0.7
        per = grad and rng.random() < 0.3
        return dict(op=op, B=_log(rng, 2, 16) if per else 1, T=_log(rng, 1, 1024 if per else 8192), vocab=_log(rng, 1000, 130000),
                    width=_width(rng, 64, 4096), grad=grad, per_example=per, scale=rng.choice([1.0, 1.0, 0.7]), dtype=dt)
    if op == "dropout":
        grad = rng.random() < 0.5
        return dict(op=op, T=_log(rng, 1, 32768), width=_width(rng, 64, 4096), p=rng.choice([0.05, 0.1, 0.25, 0.5]), grad=grad,
                    residual=not grad and rng.random() < 0.5, dtype=dt)
    e = _log(rng, 4, 512)
    return dict(op=op, T=_log(rng, 1, 65536), experts=e, k=rng.randint(1, min(8, e)), dtype=dt)


def _cost(c):
    w = work(c)  # of the plain form: products in 32 bits
    return w["bytes"] / 4e12 + w["flops"] / 1e14


def draw(rng):
    top, most = max(map(_cost, listed())), max(work(c)["bytes"] for c in listed())
    while True:
        c = _one(rng)
        if _cost(c) <= top and work(c)["bytes"] <= most:
            return c


PROMPT = 0.4  # the share of each text that its targets leave out (prompts)


def work(c):
    """Inputs read once, outputs written once, the products of unmasked rows: the logits, and with the gradient two more."""
    e = 2 if c["dtype"] == BF16 else 4
    if c["op"] == "dropout":
        n = c["T"] * c["width"]
        return {"bytes": float(n * e * (3 if c["residual"] else 2)), "flops": 2.0 * n}
    if c["op"] == "balance":
        n = c["T"] * c["experts"]
        return {"bytes": float(2 * n * e + 8 * c["T"] * c["k"]), "flops": 8.0 * n}
    T, V, w = c["B"] * c["T"], c["vocab"], c["width"]
    act = T if c["T"] < 8 else T * (1 - PROMPT)
    read = (act + V) * w * e + 12.0 * T
    if not c["grad"]:
        return {"bytes": read, "flops": 2.0 * act * V * w}
    return {"bytes": read + (T + V * (c["B"] if c["per_example"] else 1)) * w * e, "flops": 6.0 * act * V * w}


# --- inputs -----------------------------------------------------------------------------------------------
def _tokens(shape, vocab, g):
    """Token ids by frequency: id k comes about as 1 / k, as in text."""
    u = torch.rand(shape, generator=g, device=DEV, dtype=torch.float64)
    return (float(vocab + 1) ** u - 1).long().clamp_(0, vocab - 1)


def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt, s = TORCH[c["dtype"]], dict(c)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    if c["op"] == "dropout":
        s["x"] = (normal(c["T"], c["width"]) * (0.01 if c["grad"] else 1.0)).to(dt)
        s["res"] = normal(c["T"], c["width"]).to(dt) if c["residual"] else None
        s["step"] = seed % 100000
        return s
    if c["op"] == "balance":
        # some experts are preferred, a tenth of the tokens is padding
        x = normal(c["T"], c["experts"]) + 0.7 * normal(c["experts"])
        s["logits"] = x.to(dt)
        pad = torch.rand(c["T"], generator=g, device=DEV) < 0.1
        pad[0] = False
        s["experts"] = torch.where(pad[:, None], -1, torch.sort(s["logits"], dim=1, descending=True, stable=True).indices[:, :c["k"]])
        return s
    B, T, V, w = c["B"], c["T"], c["vocab"], c["width"]
    s["weight"] = (normal(V, w) * 0.02).to(dt)
    target = _tokens((B, T), V, g)
    # states of a trained model: normed, a few large features, turned to the target's row (logits 1 to 13 above the others')
    spread = torch.where(torch.rand(w, generator=g, device=DEV) < 0.01, 6.0, 1.0)
    pull = (1 + 12 * torch.rand((B, T, 1), generator=g, device=DEV)) / (0.0004 * w)
    s["hidden"] = (normal(B, T, w) * spread + pull * s["weight"][target].float()).to(dt)
    at = torch.arange(T, device=DEV)
    answer = (at >= (PROMPT if T >= 8 else 0.0) * T).expand(B, T)
    s["targets"] = torch.where(answer, target, -100)
    s["dlogp"] = -answer.float() / (answer.sum(1, keepdim=True) if c["per_example"] else answer.sum())
    if not c["per_example"]:
        s.update({k: s[k][0] for k in ("hidden", "targets", "dlogp")})
    return s


# --- the plain forms --------------------------------------------------------------------------------------
def _plain_linear(s):
    W, scale, target = s["weight"].float(), s["scale"], s["targets"].reshape(-1)
    h = s["hidden"].float().reshape(-1, s["width"])
    a = (h @ W.T).mul_(scale)
    a -= a.max(1, keepdim=True).values
    row, live = torch.arange(len(target), device=DEV), target >= 0
    at = a[row, target.clamp_min(0)]
    e = a.exp_()
    z = e.sum(1)
    logp = torch.where(live, at - torch.log(z), 0.0).view(s["targets"].shape)
    if not s["grad"]:
        return {"logp": logp}
    c = torch.where(live, s["dlogp"].reshape(-1) * scale, 0.0)
    g = e.mul_((-c / z)[:, None])
    g[row, target.clamp_min(0)] += c
    dh = (g @ W).to(s["hidden"].dtype).view(s["hidden"].shape)
    if s["per_example"]:
        dw = g.view(s["B"], s["T"], -1).transpose(1, 2) @ h.view(s["B"], s["T"], -1)
    else:
        dw = g.T @ h
    return {"logp": logp, "dhidden": dh, "dweight": dw.to(s["weight"].dtype)}


_M32 = 0xFFFFFFFF


def _philox(q, step, layer, stream):
    """Philox4x32-10 blocks (Salmon et al., SC'11) at the counters (q, step, layer, stream): [..., 4] words."""
    c0, c1, c2, c3 = q & _M32, torch.full_like(q, step), torch.full_like(q, layer), torch.full_like(q, stream)
    k0, k1 = SEED & _M32, SEED >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # modulo 2^64: both halves are taken below
        c0, c1, c2, c3 = (((p1 >> 32) & _M32) ^ c1) ^ k0, p1 & _M32, (((p0 >> 32) & _M32) ^ c3) ^ k1, p0 & _M32
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    return torch.stack([c0, c1, c2, c3], -1)


def _plain_dropout(s):
    x = s["x"]
    n = x.numel()
    w = _philox(torch.arange((n + 7) // 8, device=DEV), s["step"], 3, STREAM)
    u = torch.stack([w & 0xFFFF, w >> 16], -1).reshape(-1)[:n].view(x.shape)
    t = math.floor(s["p"] * 65536 + 0.5)
    y = torch.where(u >= t, x.float() * (65536 / (65536 - t)), 0.0)
    if s["res"] is not None:
        y += s["res"].float()
    return y.to(x.dtype)


def _plain_balance(s):
    x, ids = s["logits"].float(), s["experts"]
    E, k = x.shape[1], ids.shape[1]
    live = (ids >= 0).any(1)
    n = live.sum()
    e = torch.exp(x - x.max(1, keepdim=True).values)
    p = torch.where(live[:, None], e / e.sum(1, keepdim=True), 0.0)
    # an entry for the ids of padding, left out again
    counts = torch.zeros(E + 1, dtype=torch.int64, device=DEV)
    counts = counts.index_add_(0, torch.where(ids >= 0, ids, E).view(-1), torch.ones_like(ids).view(-1))[:E]
    f = counts / (n * k).float()
    probs = p.sum(0) / n
    d = p * (f - (p * f).sum(1, keepdim=True)) * (0.01 * E / n)
    return {"loss": 0.01 * E * (f * probs).sum(), "counts": counts, "probs": probs, "dlogits": d.to(s["logits"].dtype)}


PLAIN = {"linear": _plain_linear, "dropout": _plain_dropout, "balance": _plain_balance}


# --- the framework's operators ----------------------------------------------------------------------------
def _own(s):
    import paper_2402_03994_amd as fw

    if s["op"] == "dropout":
        if s["grad"]:
            return fw.dropout_grad(s["x"], s["p"], seed=SEED, step=s["step"], site=3)
        return fw.dropout(s["x"], s["p"], seed=SEED, step=s["step"], site=3, residual=s["res"])
    if s["op"] == "balance":
        r = fw.balance_loss(s["logits"], s["experts"], coef=0.01)
        return {"loss": r.loss, "counts": r.counts, "probs": r.probs, "dlogits": r.dlogits}
    logp, stats = fw.linear_logp(s["hidden"], s["weight"], s["targets"], scale=s["scale"])
    if not s["grad"]:
        return {"logp": logp}
    dh, dw = fw.linear_logp_grad(s["hidden"], s["weight"], s["targets"], stats, s["dlogp"], scale=s["scale"],
                                 per_example=s["per_example"])
    return {"logp": logp, "dhidden": dh, "dweight": dw}


def run(s):
    return _own(s) if own else PLAIN[s["op"]](s)


# --- the definitions in 64 bits ---------------------------------------------------------------------------
def _words(block, key, counter):
    """The four words of Philox4x32-10 at (block, *counter): products from 16-bit halves of the multiplier."""
    v = [block.clone()] + [torch.zeros_like(block) + x for x in counter]
    key = list(key)

    def halves(x, mult):
        low = x * (mult & 0xFFFF)
        mid = (low >> 16) + x * (mult >> 16)  # below 2^49
        return mid >> 16, ((mid & 0xFFFF) << 16) | (low & 0xFFFF)

    for r in range(10):
        (h0, l0), (h2, l2) = halves(v[0], 0xD2511F53), halves(v[2], 0xCD9E8D57)
        v = [h2 ^ v[1] ^ key[0], l2, h0 ^ v[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    return v


def exact(c, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = kept
    if c["op"] == "dropout":
        x = s["x"].double().reshape(-1)
        i = torch.arange(x.numel(), device=DEV)
        w = torch.cat([t[:, None] for t in _words(torch.arange((len(i) + 7) // 8, device=DEV), (SEED, 0), (s["step"], 3, STREAM))], 1)
        u = (w.view(-1)[i // 2] >> (16 * (i % 2))) & 0xFFFF
        t = round(65536 * c["p"])
        y = torch.zeros_like(x)
        kept = u >= t
        y[kept] = x[kept] * 65536 / (65536 - t)
        y = y.view(s["x"].shape)
        return y if s["res"] is None else y + s["res"].double()
    if c["op"] == "balance":
        rows = (s["experts"] >= 0).any(1).nonzero()[:, 0]
        E, ids = c["experts"], s["experts"][rows]
        p = torch.softmax(s["logits"][rows].double(), 1)
        counts = torch.bincount(ids.reshape(-1), minlength=E)
        f, probs = counts.double() / ids.numel(), p.mean(0)
        d = torch.zeros(s["logits"].shape, dtype=torch.float64, device=DEV)
        d[rows] = 0.01 * E / len(rows) * p * (f - (p @ f)[:, None])
        return {"loss": 0.01 * E * torch.dot(f, probs), "counts": None, "probs": probs, "dlogits": d}
    scale, W = c["scale"], s["weight"].double()
    flat = {k: s[k].reshape(-1) for k in ("targets", "dlogp")}
    rows = (flat["targets"] >= 0).nonzero()[:, 0]
    h = s["hidden"].reshape(-1, c["width"])[rows].double()
    t = flat["targets"][rows][:, None]
    ls = torch.log_softmax(scale * torch.mm(h, W.t().contiguous()), 1)
    logp = torch.zeros(len(flat["targets"]), dtype=torch.float64, device=DEV)
    logp[rows] = ls.gather(1, t)[:, 0]
    out = {"logp": logp.view(s["targets"].shape)}
    if not c["grad"]:
        return out
    g = ls.exp_().neg_().scatter_add_(1, t, torch.ones_like(t, dtype=torch.float64))
    g.mul_(scale * flat["dlogp"][rows].double()[:, None])
    dh = torch.zeros((len(logp), c["width"]), dtype=torch.float64, device=DEV)
    dh[rows] = torch.mm(g, W)
    text = rows // c["T"]
    parts = [(text == b).nonzero()[:, 0] for b in range(c["B"])] if c["per_example"] else [torch.arange(len(rows), device=DEV)]
    dw = torch.stack([torch.mm(g[r].t().contiguous(), h[r]) for r in parts])
    return {**out, "dhidden": dh.view(s["hidden"].shape), "dweight": dw if c["per_example"] else dw[0]}
