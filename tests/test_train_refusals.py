"""What the training-step operators refuse, before any device is touched (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2402_03994_amd as fw
from paper_2402_03994_amd import _lib

P = 4096  # a non-NULL address that is never used: every call here is refused, or has nothing to do


def logits(**kw):
    d = dict(data=P, targets=P, rows=2, vocab=8, ld=8, scale=1.0, dtype=0, index=1, device=0)
    d.update(kw)
    return ctypes.byref(_lib.Logits(*[d[k] for k, _ in _lib.Logits._fields_]))


BAD_LOGITS = [(dict(dtype=2), -2), (dict(index=7), -2), (dict(rows=-1), -1), (dict(vocab=0), -1), (dict(ld=7), -1),
              (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1),
              (dict(scale=float("inf")), -1), (dict(vocab=1 << 31, ld=1 << 31), -5), (dict(rows=1 << 31), -5),
              (dict(data=None), -1), (dict(targets=None), -1)]


@pytest.mark.parametrize("kw,code", BAD_LOGITS)
def test_losses_refuse_bad_logits(kw, code):
    L = _lib.load()
    x = logits(**kw)
    assert L.sketch_token_logp(x, P, P, None) == code
    assert L.sketch_token_logp_grad(x, P, P, P, 8, None) == code
    assert L.sketch_policy_loss(x, P, P, P, None, 0.2, 0.2, 0.0, P, P, P, P, 8, None) == code
    assert L.sketch_preference_loss(x, P, 1, 1, P, 0.1, 0.0, 0, P, P, P, P, 8, P, 1 << 40, None) == code
    assert len(L.sketch_last_error()) > 0


def test_losses_refuse_bad_arguments():
    L = _lib.load()
    x = logits()
    assert L.sketch_token_logp(None, P, P, None) == -1
    assert L.sketch_token_logp(x, None, P, None) == -1
    assert L.sketch_token_logp_grad(x, None, P, P, 8, None) == -1
    assert L.sketch_token_logp_grad(x, P, P, P, 7, None) == -1       # rows of the gradient overlap
    assert L.sketch_token_logp_grad(logits(ld=9), P, P, P, 8, None) == -1  # in place with another stride
    for lo, hi, kl in ((-0.1, 0.2, 0.0), (0.2, -0.1, 0.0), (float("nan"), 0.2, 0.0), (0.2, 0.2, float("inf")),
                       (0.2, 0.2, 0.1)):  # the last: a divergence without its reference
        assert L.sketch_policy_loss(x, P, P, P, None, lo, hi, kl, P, P, P, P + 64, 8, None) == -1
    assert L.sketch_policy_loss(x, P, P, None, None, 0.2, 0.2, 0.0, P, P, P, P + 64, 8, None) == -1
    assert L.sketch_policy_loss(x, P, P, P, None, 0.2, 0.2, 0.0, None, P, P, P + 64, 8, None) == -1
    args = dict(o=P, oi=1, pairs=1, ref=P, beta=0.1, eps=0.0, loss=P, work=P, nw=1 << 20)

    def preference(**kw):
        a = {**args, **kw}
        return L.sketch_preference_loss(x, a["o"], a["oi"], a["pairs"], a["ref"], a["beta"], a["eps"], 0, a["loss"], P, P,
                                        P + 64, 8, a["work"], a["nw"], None)

    assert preference(oi=2) == -2
    for kw in (dict(o=None), dict(pairs=0), dict(ref=None), dict(beta=float("nan")), dict(eps=-0.1), dict(eps=1.1),
               dict(loss=None), dict(work=None), dict(nw=L.sketch_preference_work_bytes(2) - 1)):
        assert preference(**kw) == -1, kw
    assert preference(pairs=1 << 31) == -5
    assert L.sketch_preference_work_bytes(0) == 0


def test_embedding_refuses_bad_arguments():
    L = _lib.load()

    def embed(w=P, dt=0, vocab=4, width=8, ld=8, ids=P, index=1, n=3, out=P, od=0):
        return L.sketch_embed(w, dt, vocab, width, ld, ids, index, n, 1.0, out, od, 0, None)

    for kw, code in ((dict(w=None), -1), (dict(dt=2), -2), (dict(od=-1), -2), (dict(index=3), -2), (dict(vocab=0), -1),
                     (dict(width=0), -1), (dict(ld=7), -1), (dict(n=-1), -1), (dict(ids=None), -1), (dict(out=None), -1),
                     (dict(n=1 << 31), -5)):
        assert embed(**kw) == code, kw
    assert embed(n=0, ids=None, out=None) == 0  # nothing to look up

    def grad(dy=P, dt=0, ld=8, ids=P, index=1, batch=2, n=3, vocab=4, width=8, out=P, od=0, work=P, nw=None):
        nw = L.sketch_embed_grad_work_bytes(batch, n, width) if nw is None else nw
        return L.sketch_embed_grad(dy, dt, ld, ids, index, batch, n, vocab, width, 1.0, out, od, 0, work, nw, 0, None)

    for kw, code in ((dict(dy=None), -1), (dict(dt=2), -2), (dict(od=5), -2), (dict(index=2), -2), (dict(ld=7), -1),
                     (dict(ids=None), -1), (dict(batch=0), -1), (dict(n=-1), -1), (dict(vocab=0), -1),
                     (dict(width=0), -1), (dict(out=None), -1), (dict(work=None), -1), (dict(nw=0), -1),
                     (dict(vocab=(1 << 20) + 1), -5), (dict(batch=1 << 16, n=1 << 15), -5)):
        assert grad(**kw) == code, kw
    assert L.sketch_embed_grad_work_bytes(0, 1, 1) == 0


def test_adamw_refuses_bad_arguments():
    L = _lib.load()
    h = ctypes.c_void_p(99)
    n2 = (ctypes.c_int64 * 2)(5, 7)

    def create(numel=n2, decay=None, k=2, state=0):
        h.value = 99
        return L.sketch_adamw_create(numel, decay, k, state, 0, 0, ctypes.byref(h))

    assert L.sketch_adamw_create(n2, None, 2, 0, 0, 0, None) == -1
    for kw in (dict(numel=None), dict(k=0), dict(state=2), dict(numel=(ctypes.c_int64 * 2)(5, 0)),
               dict(numel=(ctypes.c_int64 * 2)(5, 1 << 34)), dict(decay=(ctypes.c_float * 2)(1.0, float("nan")))):
        assert create(**kw) == -1, kw
        assert h.value is None  # *out cleared on failure
    ptrs = (ctypes.c_void_p * 2)(P, P)
    assert L.sketch_adamw_apply(None, ctypes.byref(_lib.AdamWStep()), ptrs, 0, ptrs, 0, None, None) == -1
    assert L.sketch_adamw_moments(None, P, P, P, P, P, P, None) == -1
    assert L.sketch_adamw_state_elems(None) == 0
    L.sketch_adamw_destroy(None)  # no-op


def test_binding_refuses_host_tensors_and_wrong_shapes():
    x, t = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64)
    v = torch.zeros(2)
    for call in (lambda: fw.embed(x, t), lambda: fw.embed_grad(x, t, 8), lambda: fw.token_logp(x, t),
                 lambda: fw.policy_loss(x, t, v, v, v),
                 lambda: fw.preference_loss(x, t, torch.tensor([0, 1, 2]), v)):
        with pytest.raises(ValueError):
            call()


def test_losses_refuse_scales_that_fp32_products_do_not_hold():
    """scale log2 e has to be finite, and a difference of finite logits that overflows has to be an exponential of 0."""
    L = _lib.load()
    for scale in (3e38, 1.8e38, 7e-37, 1e-39, 1e-45):
        x = logits(scale=scale, rows=0)  # refused whatever the rows
        assert L.sketch_token_logp(x, P, P, None) == -1, scale
        assert L.sketch_token_logp_grad(x, P, P, P, 8, None) == -1
        assert L.sketch_policy_loss(x, P, P, P, None, 0.2, 0.2, 0.0, P, P, P, P, 8, None) == -1
        assert L.sketch_preference_loss(x, P, 1, 1, P, 0.1, 0.0, 0, P, P, P, P, 8, P, 1 << 40, None) == -1
    for scale in (1.7e38, 1.0, 7.6e-37):
        assert L.sketch_token_logp(logits(scale=scale, rows=0), P, P, None) == 0


@pytest.mark.parametrize("device", [-1, 99])
def test_a_device_that_does_not_exist_is_refused(device):
    """Nothing is queued on another device instead."""
    L = _lib.load()
    x = logits(device=device)
    assert L.sketch_token_logp(x, P, P, None) == -1
    assert L.sketch_token_logp_grad(x, P, P, P + 64, 8, None) == -1
    assert L.sketch_policy_loss(x, P, P, P, None, 0.2, 0.2, 0.0, P, P, P, P + 64, 8, None) == -1
    assert L.sketch_preference_loss(x, P, 1, 1, P, 0.1, 0.0, 0, P, P, P, P + 64, 8, P, 1 << 40, None) == -1
    assert L.sketch_embed(P, 0, 4, 8, 8, P, 1, 3, 1.0, P, 0, device, None) == -1
    nw = L.sketch_embed_grad_work_bytes(2, 3, 8)
    assert L.sketch_embed_grad(P, 0, 8, P, 1, 2, 3, 4, 8, 1.0, P, 0, 0, P, nw, device, None) == -1
    assert b"device" in L.sketch_last_error()
