"""Performance cases of the training-step operators: embedding lookup and its gradient, token log-probabilities,
the clipped policy loss and the preference loss with their gradients, and the AdamW step over a parameter list.

Sizes follow the library's own workloads (GPT-2-small, a 1.3B decoder and Llama-3-8B tensors); draw() spreads them
over vocabularies, widths, lengths, batches and data types, odd sizes among them.

The plain forms are elementary torch operations in 32 bits, rounded once at the end. exact() evaluates the
definitions in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False
F32, BF16 = "f32", "bf16"
TORCH = {F32: torch.float32, BF16: torch.bfloat16}
DEV = "cuda"
BLOCK = 64  # elements of one AdamW block (tensors start at multiples of it in the flat buffers)
BETAS, EPS, DECAY, LR, SEED = (0.9, 0.999), 1e-8, 0.1, 1e-3, 7


# --- the cases --------------------------------------------------------------------------------------------
def listed():
    return [
        # the next token of one sequence: launch and latency only
        dict(name="embed_one", op="embed", T=1, vocab=50257, width=768, dtype=F32),
        # a long packed batch of a large bf16 model
        dict(name="embed_packed_bf16", op="embed", T=32768, vocab=128256, width=4096, dtype=BF16),
        # the gradient of a small embedding over one short text
        dict(name="embed_grad_short", op="embed_grad", B=1, T=333, vocab=8000, width=256, per_example=False, dtype=F32),
        # per-example gradients of GPT-2's embedding, as the sketches of data attribution take them
        dict(name="embed_grad_examples", op="embed_grad", B=8, T=1024, vocab=50257, width=768, per_example=True, dtype=F32),
        # the probability of one sampled token
        dict(name="logp_one", op="logp", T=1, vocab=50257, pad=0, grad=False, dtype=F32),
        # supervised fine-tuning: log-probabilities and their gradient, prompts masked
        dict(name="logp_sft_bf16", op="logp", T=4096, vocab=50257, pad=47, grad=True, dtype=BF16),
        # a clipped policy update on one short answer
        dict(name="policy_short", op="policy", T=61, vocab=50257, pad=0, kl=0.0, dtype=F32),
        # and on a batch of rollouts of a large-vocabulary model, with the divergence from a reference model
        dict(name="policy_rollouts_bf16", op="policy", T=8192, vocab=128256, pad=0, kl=0.05, dtype=BF16),
        # a preference update on a single pair
        dict(name="preference_pair", op="preference", T=411, pairs=1, vocab=50257, pad=47, average=False, smooth=0.0, dtype=F32),
        # and on a packed batch of pairs
        dict(name="preference_batch_bf16", op="preference", T=16384, pairs=16, vocab=50257, pad=0, average=False, smooth=0.1,
             dtype=BF16),
        # the optimiser of an intrinsic-dimension run: one vector of 2^16 entries, clipped
        dict(name="adamw_omega", op="adamw", model="flat", n=1 << 16, state="f32", pdtype=F32, gdtype=F32, master=False,
             clip=True),
        # all of GPT-2 small in bf16 with moments in 8 bits
        dict(name="adamw_gpt2_8bit", op="adamw", model="gpt2", width=768, vocab=50257, blocks=12, state="8bit", pdtype=BF16,
             gdtype=BF16, master=False, clip=False),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def _width(rng, a, b):
    """A model width: mostly multiples of 64, now and then any number."""
    w = _log(rng, a, b)
    return w if rng.random() < 0.3 else max(64, w // 64 * 64)


def _one(rng):
    op = rng.choice(["embed", "embed_grad", "logp", "policy", "preference", "adamw"])
    dt, vocab = rng.choice([F32, BF16]), _log(rng, 1000, 130000)
    if op == "embed":
        return dict(op=op, T=_log(rng, 1, 32768), vocab=vocab, width=_width(rng, 64, 4096), dtype=dt)
    if op == "embed_grad":
        per = rng.random() < 0.5
        return dict(op=op, B=_log(rng, 1, 16), T=_log(rng, 1, 4096), vocab=vocab, width=_width(rng, 64, 4096),
                    per_example=per, dtype=dt)
    if op == "adamw":
        state, pdt = rng.choice(["f32", "8bit"]), dt
        master = pdt == BF16 and rng.random() < 0.5
        # clipping goes with 32-bit moments: a norm that is summed in another order moves codes by a whole step
        c = dict(op=op, state=state, pdtype=pdt, gdtype=rng.choice([pdt, F32]), master=master,
                 clip=state == "f32" and rng.random() < 0.5)
        if rng.random() < 0.4:
            return dict(c, model="flat", n=_log(rng, 1000, 1 << 26))
        return dict(c, model="gpt2", width=_width(rng, 128, 768), vocab=_log(rng, 1000, 51000), blocks=rng.randint(1, 12))
    c = dict(op=op, T=_log(rng, 1, 16384), vocab=vocab, pad=rng.choice([0, 0, -vocab % 64, 7]), dtype=dt)
    if op == "logp":
        return dict(c, grad=rng.random() < 0.7)
    if op == "policy":
        return dict(c, kl=rng.choice([0.0, 0.05]))
    pairs = _log(rng, 1, 32)
    return dict(c, T=max(c["T"], 16 * pairs), pairs=pairs, average=rng.random() < 0.5, smooth=rng.choice([0.0, 0.1]))


def draw(rng):
    top = max(work(c)["bytes"] for c in listed())
    while True:
        c = _one(rng)
        if work(c)["bytes"] <= top:
            return c


def _distinct(T, vocab):
    """How many different ids T tokens of _tokens() hold, on average."""
    k = torch.arange(vocab, dtype=torch.float64)
    p = torch.log((k + 2) / (k + 1)) / math.log(vocab + 1)
    return float((1 - (1 - p) ** T).sum())


PROMPT = 0.4  # the share of each text that its targets leave out (prompts)


def work(c):
    """Inputs read once, outputs written once; masked rows of logits need not be read."""
    op = c["op"]
    if op == "adamw":
        n = sum(-(-r * k // BLOCK) * BLOCK for r, k in _shapes(c))
        p, g = (2 if c[k] == BF16 else 4 for k in ("pdtype", "gdtype"))
        mom = 16 if c["state"] == "f32" else 4 + 8  # 8 bits: read, written, and written out as the values they stand for
        return {"bytes": float(n * (2 * p + g + mom + (8 if c["master"] else 0))), "flops": 16.0 * n}
    e = 2 if c["dtype"] == BF16 else 4
    if op == "embed":
        rows = _distinct(c["T"], c["vocab"])
        return {"bytes": float(c["width"] * e * (rows + c["T"]) + 8 * c["T"]), "flops": float(c["T"] * c["width"])}
    if op == "embed_grad":
        t = c["B"] * c["T"]
        out = c["vocab"] * c["width"] * 4 * (c["B"] if c["per_example"] else 1)
        return {"bytes": float(t * c["width"] * e + 8 * t + out), "flops": 2.0 * t * c["width"]}
    T, V = c["T"], c["vocab"]
    act = T if T < 8 else T * (1 - PROMPT)
    if op == "logp" and not c["grad"]:
        return {"bytes": act * V * e + 20.0 * T, "flops": 4.0 * act * V}
    return {"bytes": act * V * e + T * V * e + 32.0 * T, "flops": 8.0 * act * V}


# --- inputs -----------------------------------------------------------------------------------------------
def _tokens(shape, vocab, g):
    """Token ids by frequency: id k comes about as 1 / k, as in text."""
    u = torch.rand(shape, generator=g, device=DEV, dtype=torch.float64)
    return (float(vocab + 1) ** u - 1).long().clamp_(0, vocab - 1)


def _cuts(T, n, seed):
    """Offsets of n texts of ragged lengths (one at least each) in T packed tokens."""
    r = random.Random(seed)
    return torch.tensor([0] + sorted(r.sample(range(1, T), n - 1)) + [T], dtype=torch.int64, device=DEV)


def _logits(c, g):
    """Logits with the peaks of a trained model at their targets: a view of rows of vocab + pad entries."""
    T, V = c["T"], c["vocab"]
    x = torch.randn((T, V + c["pad"]), generator=g, device=DEV, dtype=TORCH[c["dtype"]]).mul_(2)
    t = _tokens((T,), V, g)
    x[torch.arange(T, device=DEV), t] += (4 + 10 * torch.rand(T, generator=g, device=DEV)).to(x.dtype)
    return x[:, :V], t


def _shapes(c):
    if c["model"] == "flat":
        return [(1, c["n"])]
    w = c["width"]
    s = [(c["vocab"], w), (1024, w)]
    for _ in range(c["blocks"]):
        s += [(1, w), (1, w), (w, 3 * w), (1, 3 * w), (w, w), (1, w), (1, w), (1, w), (w, 4 * w), (1, 4 * w), (4 * w, w), (1, w)]
    return s + [(1, w), (1, w)]


def _adamw_state(c, seed, g):
    shapes = _shapes(c)
    numel = [r * k for r, k in shapes]
    blocks = [-(-n // BLOCK) for n in numel]
    nb = sum(blocks)
    bl = torch.tensor(blocks, device=DEV)
    s = {"first": torch.repeat_interleave(torch.cumsum(bl, 0) - bl, bl), "layer": torch.repeat_interleave(torch.arange(len(bl), device=DEV), bl),
         "decay": torch.repeat_interleave(torch.tensor([float(r > 1 or c["model"] == "flat") for r, _ in shapes], device=DEV), bl)[:, None]}
    # 0 where a tensor's last block is padded
    live = torch.ones(nb * BLOCK, device=DEV)
    at = 0
    for n, b in zip(numel, blocks):
        live[at + n:at + b * BLOCK] = 0
        at += b * BLOCK
    live = live.view(nb, BLOCK)
    spread = torch.exp(torch.randn((nb, 1), generator=g, device=DEV))  # of the gradients' sizes from block to block

    def normal(std):
        return torch.randn((nb, BLOCK), generator=g, device=DEV) * std * live

    grad = normal(1e-3 * spread)
    m, v = 0.3 * normal(1e-3 * spread), (grad * grad + (1e-3 * spread) ** 2 * live) * 0.5
    p = normal(0.02)
    s["p"] = p.to(TORCH[c["pdtype"]])
    s["master"] = p if c["master"] else None
    s["g"] = grad.to(TORCH[c["gdtype"]])
    if c["state"] == "8bit":
        s["m"], s["m_exp"] = _encode(m, 15, 1 << 19)
        s["v"], s["v_exp"] = _encode(v, 31, 1 << 19)
    else:
        s["m"], s["v"], s["m_exp"], s["v_exp"] = m, v, None, None
    s["scale"] = torch.tensor(0.5 + random.Random(seed).random(), device=DEV)  # of the gradients, as a loss scale leaves it
    s["step"] = 1000
    if own:
        from paper_2402_03994_amd import AdamW

        s["opt"] = AdamW(shapes, state=c["state"], decay=[float(r > 1 or c["model"] == "flat") for r, _ in shapes], seed=SEED)
        s["opt"].load_state_dict({k: s[k].reshape(-1) for k in ("m", "v", "m_exp", "v_exp") if s[k] is not None})

        def views(flat):
            out, a = [], 0
            for n, b in zip(numel, blocks):
                out.append(flat.view(-1)[a:a + n])
                a += b * BLOCK
            return out

        s["params"], s["grads"] = views(s["p"]), views(s["g"])
        s["masters"] = views(s["master"]) if c["master"] else None
    return s


def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(c)
    op = c["op"]
    if op == "adamw":
        s.update(_adamw_state(c, seed, g))
        return s
    if op == "embed":
        s["weight"] = (torch.randn((c["vocab"], c["width"]), generator=g, device=DEV) * 0.02).to(TORCH[c["dtype"]])
        s["tokens"] = _tokens((c["T"],), c["vocab"], g)
        s["scale"] = math.sqrt(c["width"])
        return s
    if op == "embed_grad":
        s["dy"] = (torch.randn((c["B"], c["T"], c["width"]), generator=g, device=DEV) * 0.01).to(TORCH[c["dtype"]])
        s["tokens"] = _tokens((c["B"], c["T"]), c["vocab"], g)
        s["scale"] = math.sqrt(c["width"])
        return s
    T = c["T"]
    s["logits"], target = _logits(c, g)
    n = 2 * c["pairs"] if op == "preference" else max(1, T // 512)
    cuts = _cuts(T, n, seed)
    at = torch.arange(T, device=DEV)
    text = torch.searchsorted(cuts, at, right=True) - 1
    answer = (at - cuts[text]) >= (PROMPT if T >= 8 else 0.0) * (cuts[text + 1] - cuts[text])
    answer = answer | (at == cuts[text + 1] - 1)  # one token at least
    s["targets"] = torch.where(answer, target, -100)
    if op == "logp":
        s["dlogp"] = -answer.float() / answer.sum()
        return s
    logp = torch.where(answer, _logp(s["logits"], target, 1.0)[0], 0.0)
    s["ref"] = logp + 0.3 * torch.randn(T, generator=g, device=DEV) * answer
    if op == "preference":
        s["offsets"] = cuts
        return s
    # what the sampling policy gave: near the present one, kept in steps of 1/64
    s["old"] = logp - torch.round(torch.randn(T, generator=g, device=DEV) * 0.15 * 64) / 64 * answer
    s["adv"] = torch.randn(n, generator=g, device=DEV)[text]
    s["weights"] = answer.float() / answer.sum()
    return s


# --- the plain forms --------------------------------------------------------------------------------------
def _logp(logits, target, scale):
    """log softmax(scale x)[target] by rows, with exp(scale (x - max)) and its sum."""
    x = logits.float()
    a = (x - x.max(1, keepdim=True).values) * scale
    e = torch.exp(a)
    z = e.sum(1)
    t = target.clamp(0, x.shape[1] - 1)
    return a[torch.arange(len(t), device=DEV), t] - torch.log(z), e, z


def _dlogits(e, z, target, dlogp, dtype):
    d = e * (-dlogp / z)[:, None]
    live = torch.arange(len(z), device=DEV)
    d[live, target.clamp_min(0)] += dlogp
    return torch.where((target >= 0)[:, None], d, 0.0).to(dtype)


def _plain_preference(s):
    target, cuts = s["targets"], s["offsets"]
    logp, e, z = _logp(s["logits"], target, 1.0)
    answer = target >= 0
    text = torch.searchsorted(cuts, torch.arange(len(target), device=DEV), right=True) - 1
    zero = torch.zeros(len(cuts) - 1, device=DEV)
    count = zero.index_add(0, text, answer.float())
    share = 1.0 / count.clamp_min(1) if s["average"] else torch.ones_like(count)
    seq = zero.index_add(0, text, torch.where(answer, logp, 0.0)) * share
    gap = zero.index_add(0, text, torch.where(answer, logp - s["ref"], 0.0)) * share
    d = gap[0::2] - gap[1::2]
    b, eps, P = 0.1, s["smooth"], s["pairs"]
    soft = lambda u: torch.clamp_min(u, 0) + torch.log1p(torch.exp(-u.abs()))  # noqa: E731
    each = (1 - eps) * soft(-b * d) + eps * soft(b * d)
    c = -b / P * ((1 - eps) / (1 + torch.exp(b * d)) - eps / (1 + torch.exp(-b * d)))
    dseq = torch.stack([c, -c], 1).reshape(-1) * share
    dlogits = _dlogits(e, z, target, torch.where(answer, dseq[text], 0.0), s["logits"].dtype)
    return {"loss": each.mean(), "seq_logp": seq, "pair_loss": each, "dlogits": dlogits}


def _plain_policy(s):
    target = s["targets"]
    answer = target >= 0
    logp, e, z = _logp(s["logits"], target, 1.0)
    logp = torch.where(answer, logp, 0.0)
    A, r = s["adv"], torch.exp(logp - s["old"])
    free, held = A * r, A * r.clamp(0.8, 1.2)
    each, d = -torch.minimum(free, held), torch.where(free <= held, -free, 0.0)
    if s["kl"]:
        u = s["ref"] - logp
        each, d = each + s["kl"] * (torch.exp(u) - u - 1), d + s["kl"] * (1 - torch.exp(u))
    each, d = torch.where(answer, each, 0.0), torch.where(answer, d, 0.0) * s["weights"]
    return {"loss": (each * s["weights"]).sum(), "logp": logp, "token_loss": each,
            "dlogits": _dlogits(e, z, target, d, s["logits"].dtype)}


_M32 = 0xFFFFFFFF


def _philox(q, step, layer, stream):
    """Philox4x32-10 blocks (Salmon et al., SC'11) at the counters (q, step, layer, stream): [..., 4] words."""
    c0, c1, c2, c3 = q & _M32, torch.full_like(q, step), layer.expand_as(q), torch.full_like(q, stream)
    k0, k1 = SEED & _M32, SEED >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # modulo 2^64: both halves are taken below
        c0, c1, c2, c3 = (((p1 >> 32) & _M32) ^ c1) ^ k0, p1 & _M32, (((p0 >> 32) & _M32) ^ c3) ^ k1, p0 & _M32
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    return torch.stack([c0, c1, c2, c3], -1)


def _pow2(e):
    """2^e for whole e in [-126, 127]."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _encode(x, top, dither):
    """Codes (the sign bit first where `top` is 15) and biased block exponents of x [blocks, 64]: |x| 2^-E as a small
    float whose largest exponent field is `top`, the 20 bits below its mantissa rounded by `dither` < 2^20."""
    big = x.abs().amax(1, keepdim=True).contiguous()
    E = ((big.view(torch.int32) + 0x0FFFFF) >> 23) - 127
    y = (x.abs() * _pow2(-E)) * _pow2(torch.full_like(E, top - 127))
    code = (y.view(torch.int32) + dither) >> 20
    if top == 15:
        code = code | ((x < 0).int() << 7)
    return code.to(torch.uint8), (E + 127).to(torch.uint8)[:, 0]


def _decode(code, exp, top):
    c = code.int()
    y = ((c & (0x7F if top == 15 else 0xFF)) << 20).view(torch.float32) * _pow2(torch.full_like(c, 127 - top)) \
        * _pow2(exp.int() - 127)[:, None]
    return torch.where(c >= 128, -y, y) if top == 15 else y


def _plain_adamw(s):
    s["step"] += 1
    (b1, b2), t = BETAS, s["step"]
    g = s["g"].float()
    scale, out = s["scale"], {}
    if s["clip"]:
        out["norm"] = scale * torch.sqrt((g * g).sum())
        scale = scale * torch.clamp_max(1.0 / (out["norm"] + 1e-6), 1.0)
    g = g * scale
    low = s["state"] == "8bit"
    m, v = (_decode(s["m"], s["m_exp"], 15), _decode(s["v"], s["v_exp"], 31)) if low else (s["m"], s["v"])
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    p = s["p"].float() if s["master"] is None else s["master"]
    p = p * (1 - LR * DECAY * s["decay"]) - (LR / (1 - b1 ** t)) * (m / (torch.sqrt(v) * (1 / math.sqrt(1 - b2 ** t)) + EPS))
    e4 = (torch.arange(len(m), device=DEV) - s["first"])[:, None] * (BLOCK // 4)  # a block's first group of four
    if low:
        w = _philox(e4 + torch.arange(BLOCK // 4, device=DEV), t, s["layer"][:, None], 11).reshape(m.shape)
        s["m"], s["m_exp"] = _encode(m, 15, (w >> 16).int() << 4 | 8)
        s["v"], s["v_exp"] = _encode(v, 31, (w & 0xFFFF).int() << 4 | 8)
        m, v = _decode(s["m"], s["m_exp"], 15), _decode(s["v"], s["v_exp"], 31)
    else:
        s["m"], s["v"] = m, v
    if s["master"] is not None:
        s["master"] = out["master"] = p
    elif s["p"].dtype == torch.bfloat16:  # rounded up with the probability of what is cut off
        w = _philox(e4 // 2 + torch.arange(BLOCK // 8, device=DEV), t, s["layer"][:, None], 12)
        r = torch.stack([w & 0xFFFF, w >> 16], -1).reshape(p.shape)
        p = ((p.view(torch.int32) + r.int()) & -65536).view(torch.float32)
    s["p"] = p.to(s["p"].dtype)
    return {**out, "p": s["p"].view(-1), "m": m.view(-1), "v": v.view(-1)}


def _plain_embed(s):
    return (s["weight"][s["tokens"]].float() * s["scale"]).to(s["weight"].dtype)


def _plain_embed_grad(s):
    B, V = s["B"] if s["per_example"] else 1, s["vocab"]
    key = s["tokens"] + (torch.arange(s["B"], device=DEV)[:, None] * V if s["per_example"] else 0)
    out = torch.zeros((B * V, s["width"]), device=DEV)
    out = out.index_add_(0, key.view(-1), s["dy"].view(-1, s["width"]).float()).mul_(s["scale"])
    return out.view(B, V, -1) if s["per_example"] else out


def _plain_logp(s):
    target = s["targets"]
    logp, e, z = _logp(s["logits"], target, 1.0)
    logp = torch.where(target >= 0, logp, 0.0)
    return [logp, _dlogits(e, z, target, s["dlogp"], s["logits"].dtype)] if s["grad"] else [logp]


PLAIN = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "logp": _plain_logp, "policy": _plain_policy,
         "preference": _plain_preference, "adamw": _plain_adamw}


# --- the framework's operators ----------------------------------------------------------------------------
def _own(s):
    import paper_2402_03994_amd as fw

    op = s["op"]
    if op == "embed":
        return fw.embed(s["weight"], s["tokens"], scale=s["scale"])
    if op == "embed_grad":
        return fw.embed_grad(s["dy"], s["tokens"], s["vocab"], scale=s["scale"], per_example=s["per_example"])
    if op == "logp":
        logp, stats = fw.token_logp(s["logits"], s["targets"])
        if not s["grad"]:
            return [logp]
        return [logp, fw.token_logp_grad(s["logits"], s["targets"], stats, s["dlogp"])]
    if op == "policy":
        r = fw.policy_loss(s["logits"], s["targets"], s["old"], s["adv"], s["weights"], ref_logp=s["ref"] if s["kl"] else None,
                           clip=(0.2, 0.2), kl_coef=s["kl"])
        return {"loss": r.loss, "logp": r.logp, "token_loss": r.token_loss, "dlogits": r.dlogits}
    if op == "preference":
        r = fw.preference_loss(s["logits"], s["targets"], s["offsets"], s["ref"], beta=0.1, label_smoothing=s["smooth"],
                               average=s["average"])
        return {"loss": r.loss, "seq_logp": r.seq_logp, "pair_loss": r.pair_loss, "dlogits": r.dlogits}
    s["step"] += 1
    norm = s["opt"].step(s["params"], s["grads"], s["step"], lr=LR, betas=BETAS, eps=EPS, weight_decay=DECAY,
                         masters=s["masters"], grad_scale=s["scale"], max_norm=1.0 if s["clip"] else None)
    m, v = s["opt"].moments()
    out = {"p": s["p"].view(-1), "m": m, "v": v}
    if s["clip"]:
        out["norm"] = norm
    if s["master"] is not None:
        out["master"] = s["master"]
    return out


def run(s):
    return _own(s) if own else PLAIN[s["op"]](s)


# --- the definitions in 64 bits ---------------------------------------------------------------------------
def exact(c, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = kept
    op = c["op"]
    if op == "embed":
        return torch.index_select(s["weight"].double(), 0, s["tokens"]) * s["scale"]
    if op == "embed_grad":
        out = torch.zeros((c["B"], c["vocab"], c["width"]) if c["per_example"] else (1, c["vocab"], c["width"]),
                          dtype=torch.float64, device=DEV)
        for b in range(c["B"]):
            out[b if c["per_example"] else 0].index_add_(0, s["tokens"][b], s["dy"][b].double() * s["scale"])
        return out if c["per_example"] else out[0]
    if op == "adamw":
        return _exact_adamw(c, s)
    rows = (s["targets"] >= 0).nonzero()[:, 0]
    x = s["logits"].index_select(0, rows).double()
    t = s["targets"][rows][:, None]
    x = x.sub_(torch.logsumexp(x, 1, keepdim=True))
    lp = torch.zeros(c["T"], dtype=torch.float64, device=DEV)
    lp[rows] = x.gather(1, t)[:, 0]

    def gradient(dlp):
        d = dlp[rows][:, None]
        q = torch.exp(x).mul_(-d).scatter_add_(1, t, d)
        out = torch.zeros((c["T"], c["vocab"]), dtype=torch.float64, device=DEV)
        out[rows] = q
        return out

    if op == "logp":
        return [lp, gradient(s["dlogp"].double())] if c["grad"] else [lp]
    if op == "policy":
        A, w, r = s["adv"].double()[rows], s["weights"].double()[rows], torch.exp(lp - s["old"].double())[rows]
        inside = torch.where(A > 0, r <= 1 + 0.2, r >= 1 - 0.2)
        surrogate = A * torch.where(inside, r, torch.where(A > 0, 1 + 0.2, 1 - 0.2).double())
        u = (s["ref"].double() - lp)[rows]
        each, dlp = torch.zeros_like(lp), torch.zeros_like(lp)
        each[rows] = c["kl"] * (torch.expm1(u) - u) - surrogate
        dlp[rows] = w * (-c["kl"] * torch.expm1(u) - torch.where(inside, A * r, 0.0))
        return {"loss": (w * each[rows]).sum(), "logp": lp, "token_loss": each, "dlogits": gradient(dlp)}
    ends = s["offsets"].tolist()
    at = [slice(a, b) for a, b in zip(ends, ends[1:])]
    n = [max(1, int((s["targets"][a] >= 0).sum())) if c["average"] else 1 for a in at]
    seq = torch.stack([lp[a].sum() / k for a, k in zip(at, n)])
    ref = torch.stack([(s["ref"][a].double() * (s["targets"][a] >= 0)).sum() / k for a, k in zip(at, n)])
    h = (seq - ref).view(-1, 2)
    z = 0.1 * (h[:, 0] - h[:, 1])
    ls = torch.nn.functional.logsigmoid
    each = -(1 - c["smooth"]) * ls(z) - c["smooth"] * ls(-z)
    dz = (c["smooth"] * torch.sigmoid(z) - (1 - c["smooth"]) * torch.sigmoid(-z)) * 0.1 / c["pairs"]
    dlp = torch.zeros_like(lp)
    for i, a in enumerate(at):
        dlp[a] = (dz[i // 2] if i % 2 == 0 else -dz[i // 2]) / n[i]
    return {"loss": each.mean(), "seq_logp": seq, "pair_loss": each, "dlogits": gradient(dlp)}


def _exact_adamw(c, s):
    """Moments in 8 bits are defined by 32-bit arithmetic and its rounding: they have no value in 64 bits."""
    low, t = c["state"] == "8bit", s["step"] + 1
    g = s["g"].double() * s["scale"].double()
    out = {"norm": g.norm()} if c["clip"] else {}
    if c["clip"]:
        g = g * min(1.0, 1.0 / (float(out["norm"]) + 1e-6))
    if low:
        sign = 1 - 2 * (s["m"].long() >> 7)
        m, v = (torch.where(k >> b > 0, (1 + (k & 7) / 8.0) * 2.0 ** ((k >> b) - top), (k & 7) / 8.0 * 2.0 ** (1 - top)).double()
                * 2.0 ** (e[:, None].double() - 127)
                for k, e, b, top in ((s["m"].long() & 127, s["m_exp"], 3, 15), (s["v"].long(), s["v_exp"], 3, 31)))
        m = m * sign
    else:
        m, v = s["m"].double(), s["v"].double()
    m = BETAS[0] * m + (1 - BETAS[0]) * g
    v = BETAS[1] * v + (1 - BETAS[1]) * g ** 2
    p = (s["p"] if s["master"] is None else s["master"]).double()
    p = p - LR * DECAY * s["decay"].double() * p - LR * (m / (1 - BETAS[0] ** t)) / (torch.sqrt(v / (1 - BETAS[1] ** t)) + EPS)
    if s["master"] is not None:
        out["master"] = p
    return {**out, "p": p.view(-1), "m": None if low else m.view(-1), "v": None if low else v.view(-1)}
