"""Binding of the training-step operators (include/sketch_train.h) for torch tensors.

Argument marshalling only: the embedding lookup and its gradient, the token
log-probabilities, the policy and preference losses with their gradients and
the AdamW step run in the HIP kernels of libsketch.so on torch's current
stream.  The losses return the gradient with respect to the logits next to the
loss: a model continues with logits.backward(dlogits).  No call records itself for
autograd (embed() of a weight that requires a gradient gives a tensor without one);
what a call overwrites counts as modified in place, so that a graph that has saved
it refuses its backward pass.
"""
from __future__ import annotations

import array
import ctypes
import operator
from typing import NamedTuple, Optional, Sequence

import torch
from torch.autograd.graph import increment_version

from . import _lib
from .sketch import _DT, _stream_ptr

_INDEX = {torch.int32: _lib.SK_I32, torch.int64: _lib.SK_I64}
_get_dtype = operator.attrgetter("dtype")
_STATE = {"f32": _lib.SK_ADAMW_F32, "8bit": _lib.SK_ADAMW_8BIT}


class PolicyLoss(NamedTuple):
    """loss (scalar), logp and token_loss [T] float32, dlogits (None without grad)."""
    loss: torch.Tensor
    logp: torch.Tensor
    token_loss: torch.Tensor
    dlogits: Optional[torch.Tensor]


class PreferenceLoss(NamedTuple):
    """loss (scalar), seq_logp [2 pairs] and pair_loss [pairs] float32, dlogits (None without grad)."""
    loss: torch.Tensor
    seq_logp: torch.Tensor
    pair_loss: torch.Tensor
    dlogits: Optional[torch.Tensor]


def _dtype(t: torch.Tensor, name: str) -> int:
    if t.dtype not in _DT:
        raise ValueError(f"{name} must be float32 or bfloat16")
    return _DT[t.dtype]


def _ids(t: torch.Tensor, name: str, device) -> int:
    if t.dtype not in _INDEX or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous int32 or int64 on {device}")
    return _INDEX[t.dtype]


def _on_gpu(t: torch.Tensor, name: str) -> torch.device:
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a ROCm device")
    return t.device


def _vec(t: torch.Tensor, n: int, device, name: str) -> int:
    if t.dtype != torch.float32 or t.device != device or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous float32 [{n}] on {device}")
    return t.data_ptr()


def _rows(t: torch.Tensor, name: str) -> int:
    """The row stride of a matrix whose rows are contiguous."""
    if t.dim() != 2 or t.shape[1] < 1:
        raise ValueError(f"{name} must be a matrix with at least one column")
    n, width = t.shape
    if t.is_contiguous():
        return width
    ld = t.stride(0) if n > 1 else width
    if (t.stride(1) != 1 and width > 1) or ld < width:
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return ld


def embed(weight: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, out: Optional[torch.Tensor] = None,
          out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """scale * weight[tokens]: [*tokens.shape, width] in the weight's type (or out_dtype).

    weight [vocab, width] may have a row stride; a token outside [0, vocab) gives a row of zeros."""
    device = _on_gpu(weight, "weight")
    ld = _rows(weight, "weight")
    index = _ids(tokens, "tokens", device)
    shape = (*tokens.shape, weight.shape[1])
    given = out is not None
    if not given:
        out = torch.empty(shape, dtype=out_dtype or weight.dtype, device=device)
    elif out.shape != shape or out.device != device or not out.is_contiguous() or \
            (out_dtype is not None and out.dtype != out_dtype):
        raise ValueError(f"out must be contiguous {list(shape)} on {device}")
    _lib.check(_lib.load().sketch_embed(weight.data_ptr(), _dtype(weight, "weight"), weight.shape[0], weight.shape[1], ld,
                                        tokens.data_ptr(), index, tokens.numel(), scale, out.data_ptr(),
                                        _dtype(out, "out"), device.index, _stream_ptr(device)))
    if given:
        increment_version(out)
    return out


def embed_grad(dy: torch.Tensor, tokens: torch.Tensor, vocab: int, scale: float = 1.0, per_example: bool = False,
               out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.float32,
               accumulate: bool = False) -> torch.Tensor:
    """The gradient of embed() with respect to the weight: out[v] (+)= scale * sum of dy over the tokens equal to v.

    dy [*tokens.shape, width].  per_example: one gradient [vocab, width] for each entry of tokens' first axis, so that
    out [batch, vocab, width], viewed as [batch, vocab * width], is what Sketch.apply takes; else out [vocab, width].
    accumulate adds to `out`.  Sums are kept in fp32, in an order that the ids, the sizes and the types set."""
    device = _on_gpu(dy, "dy")
    if dy.shape[:-1] != tokens.shape or dy.dim() < 2 or dy.shape[-1] < 1:
        raise ValueError("dy must be [*tokens.shape, width]")
    index = _ids(tokens, "tokens", device)
    width = ld = dy.shape[-1]
    if not dy.is_contiguous():
        try:
            ld = _rows(dy.view(-1, width), "dy")
        except RuntimeError:
            raise ValueError("dy must have rows of one stride") from None
    if per_example and tokens.dim() < 2:
        raise ValueError("per_example needs tokens [batch, ...]")
    batch = tokens.shape[0] if per_example else 1
    shape = (batch, vocab, width) if per_example else (vocab, width)
    given = out is not None
    if not given:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty(shape, dtype=out_dtype, device=device)
    elif out.shape != shape or out.device != device or not out.is_contiguous():
        raise ValueError(f"out must be contiguous {list(shape)} on {device}")
    if batch == 0:
        return out
    lib = _lib.load()
    n = tokens.numel() // batch
    nw = lib.sketch_embed_grad_work_bytes(batch, n, width)
    work = torch.empty(nw, dtype=torch.uint8, device=device)
    _lib.check(lib.sketch_embed_grad(dy.data_ptr(), _dtype(dy, "dy"), ld, tokens.data_ptr(), index, batch, n, vocab,
                                     width, scale, out.data_ptr(), _dtype(out, "out"), int(accumulate),
                                     work.data_ptr(), nw, device.index, _stream_ptr(device)))
    if given:
        increment_version(out)
    return out


def _logits(logits: torch.Tensor, targets: torch.Tensor, scale: float) -> _lib.Logits:
    device = _on_gpu(logits, "logits")
    ld = _rows(logits, "logits")
    index = _ids(targets, "targets", device)
    if targets.dim() != 1 or targets.shape[0] != logits.shape[0]:
        raise ValueError("targets must be [T] for logits [T, vocab]")
    return _lib.Logits(logits.data_ptr(), targets.data_ptr(), logits.shape[0], logits.shape[1], ld, scale,
                       _dtype(logits, "logits"), index, device.index)


def _dlogits(logits: torch.Tensor, out: Optional[torch.Tensor]):
    """The gradient's tensor and its row stride.  A new one keeps the row stride of logits that are padded by up to 64
    columns, so that rows of both start at the same place of 16 bytes."""
    if out is None:
        n, vocab = logits.shape
        ld = logits.stride(0) if n > 1 else vocab
        if vocab < ld <= vocab + 64:
            return torch.empty((n, ld), dtype=logits.dtype, device=logits.device)[:, :vocab], ld
        return torch.empty((n, vocab), dtype=logits.dtype, device=logits.device), vocab
    if out.shape != logits.shape or out.dtype != logits.dtype or out.device != logits.device:
        raise ValueError("out must have the shape, type and device of the logits")
    return out, _rows(out, "out")


def token_logp(logits: torch.Tensor, targets: torch.Tensor, scale: float = 1.0):
    """(logp [T], stats [T, 2]) float32: log softmax(scale * logits)[targets] by rows, and what token_logp_grad needs.

    logits [T, vocab] (float32 or bfloat16, rows may have a stride); targets [T], a target outside [0, vocab) masks
    its row (logp 0, the row is not read)."""
    x = _logits(logits, targets, scale)
    n = logits.shape[0]
    logp = torch.empty(n, dtype=torch.float32, device=logits.device)
    stats = torch.empty((n, 2), dtype=torch.float32, device=logits.device)
    _lib.check(_lib.load().sketch_token_logp(ctypes.byref(x), logp.data_ptr(), stats.data_ptr(),
                                             _stream_ptr(logits.device)))
    return logp, stats


def token_logp_grad(logits: torch.Tensor, targets: torch.Tensor, stats: torch.Tensor, dlogp: torch.Tensor,
                    scale: float = 1.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of sum(dlogp * logp) with respect to the logits, in their type.  out may be the logits; a new tensor
    has the row stride of logits that are padded by up to 64 columns (and is not contiguous then)."""
    x = _logits(logits, targets, scale)
    n = logits.shape[0]
    if stats.dtype != torch.float32 or stats.device != logits.device or stats.shape != (n, 2) or not stats.is_contiguous():
        raise ValueError(f"stats must be contiguous float32 [{n}, 2] on {logits.device}")
    dp = _vec(dlogp, n, logits.device, "dlogp")
    d, ld = _dlogits(logits, out)
    _lib.check(_lib.load().sketch_token_logp_grad(ctypes.byref(x), stats.data_ptr(), dp, d.data_ptr(), ld,
                                                  _stream_ptr(logits.device)))
    if out is not None:
        increment_version(out)
    return d


def policy_loss(logits: torch.Tensor, targets: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor,
                weights: torch.Tensor, ref_logp: Optional[torch.Tensor] = None, clip=(0.2, 0.2), kl_coef: float = 0.0,
                scale: float = 1.0, grad: bool = True, out: Optional[torch.Tensor] = None) -> PolicyLoss:
    """sum_t weights_t (-min(r A, clip(r, 1 - clip[0], 1 + clip[1]) A) + kl_coef (e^u - u - 1)) with
    r = exp(logp - old_logp), u = ref_logp - logp, and its gradient with respect to the logits.

    Rows with a masked target or weight 0 are not read.  The weights set the mean that is meant (over tokens:
    mask / mask.sum(); over texts: mask / (texts * length)).  out (where grad) may be the logits; a new dlogits has their
    row stride, as token_logp_grad's."""
    x = _logits(logits, targets, scale)
    device, n = logits.device, logits.shape[0]
    args = [_vec(t, n, device, name) for t, name in ((old_logp, "old_logp"), (advantages, "advantages"),
                                                     (weights, "weights"))]
    args.append(None if ref_logp is None else _vec(ref_logp, n, device, "ref_logp"))
    loss = torch.empty((), dtype=torch.float32, device=device)
    logp = torch.empty(n, dtype=torch.float32, device=device)
    token_loss = torch.empty(n, dtype=torch.float32, device=device)
    d, ld = _dlogits(logits, out) if grad else (None, 0)
    _lib.check(_lib.load().sketch_policy_loss(ctypes.byref(x), *args, clip[0], clip[1], kl_coef, loss.data_ptr(),
                                              logp.data_ptr(), token_loss.data_ptr(),
                                              d.data_ptr() if grad else None, ld, _stream_ptr(device)))
    if grad and out is not None:
        increment_version(out)
    return PolicyLoss(loss, logp, token_loss, d)


def preference_loss(logits: torch.Tensor, targets: torch.Tensor, offsets: torch.Tensor, ref_logp: torch.Tensor,
                    beta: float = 0.1, label_smoothing: float = 0.0, average: bool = False, scale: float = 1.0,
                    grad: bool = True, out: Optional[torch.Tensor] = None) -> PreferenceLoss:
    """The mean over pairs of -log sigmoid(beta d) (smoothed), d = how much more the chosen text (rows offsets[2p] ..
    offsets[2p + 1]) has gained on the reference model than the rejected one that follows it, and its gradient with
    respect to the logits.

    ref_logp [T]: the reference model's token_logp.  average: texts by their mean instead of their sum.  Masked
    targets (prompts, padding) count nothing.  out (where grad) may be the logits; a new dlogits has their row stride, as
    token_logp_grad's."""
    x = _logits(logits, targets, scale)
    device, n = logits.device, logits.shape[0]
    index = _ids(offsets, "offsets", device)
    if offsets.dim() != 1 or offsets.shape[0] < 3 or offsets.shape[0] % 2 == 0:
        raise ValueError("offsets must be [2 pairs + 1]")
    pairs = offsets.shape[0] // 2
    ref = _vec(ref_logp, n, device, "ref_logp")
    small = torch.empty(1 + 3 * pairs, dtype=torch.float32, device=device)
    d, ld = _dlogits(logits, out) if grad else (None, 0)
    lib = _lib.load()
    nw = lib.sketch_preference_work_bytes(n)
    work = torch.empty(nw, dtype=torch.uint8, device=device)
    at = small.data_ptr()
    _lib.check(lib.sketch_preference_loss(ctypes.byref(x), offsets.data_ptr(), index, pairs, ref, beta, label_smoothing,
                                          int(average), at, at + 4, at + 4 + 8 * pairs, d.data_ptr() if grad else None,
                                          ld, work.data_ptr(), nw, _stream_ptr(device)))
    if grad and out is not None:
        increment_version(out)
    return PreferenceLoss(small[0], small[1:1 + 2 * pairs], small[1 + 2 * pairs:], d)


class AdamW:
    """AdamW over a list of parameter tensors, stepped in one launch for up to 160 of them.

    shapes: per tensor its shape or element count.  state: "f32" or "8bit" moments (a byte an element and an exponent
    byte for each 64; rounded up or down at random from `seed`, step and place, so that two runs agree).  decay: a
    factor of weight_decay per tensor (0 for biases and norms).
    m, v (and m_exp, v_exp with "8bit") are the state: each tensor's elements, padded to a multiple of 64, in list
    order.
    A list has one type: a model of two takes a handle for each, and clips by a norm of each, or by a common one that its
    program forms and passes in grad_scale.
    The numbers of a step are taken when it is called: a captured graph repeats that very step, random words included, at
    every replay, and is no way to go on training."""

    def __init__(self, shapes: Sequence, state: str = "f32", decay: Optional[Sequence[float]] = None, seed: int = 0,
                 device=None):
        self.lib = _lib.load()
        self.device = torch.device("cuda", torch.cuda.current_device() if device is None else
                                   torch.device(device).index or 0)
        if state not in _STATE:
            raise ValueError("state must be 'f32' or '8bit'")
        self.state = state
        self.seed = int(seed)
        self.numels = []
        for s in shapes:
            n = 1
            for v in (s if isinstance(s, (tuple, list, torch.Size)) else (s,)):
                n *= int(v)
            self.numels.append(n)
        if decay is not None and len(decay) != len(self.numels):
            raise ValueError("decay must hold one factor per tensor")
        k = len(self.numels)
        h = ctypes.c_void_p()
        _lib.check(self.lib.sketch_adamw_create((ctypes.c_int64 * k)(*self.numels),
                                                None if decay is None else (ctypes.c_float * k)(*decay), k,
                                                _STATE[state], self.seed, self.device.index, ctypes.byref(h)))
        self._h = h
        n = self.elems = int(self.lib.sketch_adamw_state_elems(h))
        dt = torch.float32 if state == "f32" else torch.uint8
        self.m = torch.zeros(n, dtype=dt, device=self.device)
        self.v = torch.zeros(n, dtype=dt, device=self.device)
        self.m_exp = self.v_exp = None
        if state == "8bit":
            self.m_exp = torch.zeros(n // 64, dtype=torch.uint8, device=self.device)
            self.v_exp = torch.zeros(n // 64, dtype=torch.uint8, device=self.device)

    def close(self):
        if getattr(self, "_h", None):
            self.lib.sketch_adamw_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def state_dict(self) -> dict:
        return {k: getattr(self, k) for k in ("m", "v", "m_exp", "v_exp") if getattr(self, k) is not None}

    def load_state_dict(self, d: dict) -> None:
        own = self.state_dict()
        if set(d) != set(own):
            raise ValueError(f"the state holds {sorted(own)}")
        for k, t in own.items():
            if d[k].shape != t.shape or d[k].dtype != t.dtype:
                raise ValueError(f"{k} must be {t.dtype} {list(t.shape)}")
        for k, t in own.items():
            t.copy_(d[k])

    def _pointers(self, tensors, name, dtype=None):
        # one C-level pass per property: a list of 150 parameters is checked in a third of a loop's time
        T = torch.Tensor
        try:
            dt = tensors[0].dtype if dtype is None else dtype
            same = list(map(T.numel, tensors)) == self.numels and set(map(_get_dtype, tensors)) == {dt} and \
                set(map(T.get_device, tensors)) == {self.device.index} and all(map(T.is_contiguous, tensors))
        except (TypeError, AttributeError, LookupError):  # not a list, or not of tensors
            dt, same = dtype, False
        if not same:
            raise ValueError(f"{name}: contiguous {dt or 'float32 or bfloat16'} tensors on {self.device} with these counts are "
                             f"needed: {self.numels[:8]}{'..' if len(self.numels) > 8 else ''}")
        at = array.array("Q", list(map(T.data_ptr, tensors)))  # two thirds of the time of filling the ctypes array itself
        return (ctypes.c_void_p * len(tensors)).from_buffer(at), dt

    def step(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], step: int, lr: float,
             betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
             masters: Optional[Sequence[torch.Tensor]] = None, grad_scale: Optional[torch.Tensor] = None,
             max_norm: Optional[float] = None) -> Optional[torch.Tensor]:
        """One step (1, 2, ..) on params (float32 or bfloat16, in place), one type for all of them and one for all grads;
        every tensor of the list takes part, so that each needs a gradient.

        masters: float32 copies of bfloat16 params that the step is taken on; without them bfloat16 params are rounded
        at random.  grad_scale: one float32 on the device that multiplies the gradients; a step where it is not finite
        changes nothing.  max_norm: clip the 2-norm of all scaled gradients, which is returned (device scalar)."""
        pp, pdt = self._pointers(params, "params")
        gp, gdt = self._pointers(grads, "grads")
        if pdt not in _DT or gdt not in _DT:
            raise ValueError("params and grads must be float32 or bfloat16")
        mp = None if masters is None else self._pointers(masters, "masters", torch.float32)[0]
        if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1 or
                                       grad_scale.device != self.device):
            raise ValueError(f"grad_scale must be one float32 on {self.device}")
        norm = None
        if max_norm is not None:
            if not max_norm > 0:
                raise ValueError("max_norm must be positive")
            norm = torch.empty((), dtype=torch.float32, device=self.device)
        a = _lib.AdamWStep(int(step), lr, betas[0], betas[1], eps, weight_decay, max_norm or 0.0,
                           None if grad_scale is None else grad_scale.data_ptr(),
                           None if norm is None else norm.data_ptr(), self.m.data_ptr(), self.v.data_ptr(),
                           None if self.m_exp is None else self.m_exp.data_ptr(),
                           None if self.v_exp is None else self.v_exp.data_ptr())
        _lib.check(self.lib.sketch_adamw_apply(self._h, ctypes.byref(a), pp, _DT[pdt], gp, _DT[gdt], mp,
                                               _stream_ptr(self.device)))
        increment_version(params if masters is None else [*params, *masters])
        return norm

    def moments(self):
        """(m, v) as the float32 values they stand for, laid out as the state (which it is, with state "f32")."""
        if self.state == "f32":
            return self.m, self.v
        m = torch.empty(self.elems, dtype=torch.float32, device=self.device)
        v = torch.empty(self.elems, dtype=torch.float32, device=self.device)
        _lib.check(self.lib.sketch_adamw_moments(self._h, self.m.data_ptr(), self.m_exp.data_ptr(), self.v.data_ptr(),
                                                 self.v_exp.data_ptr(), m.data_ptr(), v.data_ptr(),
                                                 _stream_ptr(self.device)))
        return m, v
