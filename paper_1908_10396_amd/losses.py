"""Binding of the losses of log probabilities (include/avq.h): argument marshalling only.

Log probabilities are contiguous fp32 tensors on the GPU, as `log_probs` and `list_log_probs` return them; the gradient that
a *_grad form returns is what those operators' *_grad forms take as grad_logp. Each *_grad form returns the loss too. None
of this takes part in torch's autograd. Sequences of tokens lie side by side, sequence s from offsets[s] to offsets[s + 1] (int32);
a mask (torch.bool, one a token) says which tokens count.
"""
import collections

import torch

from . import _check, lib
from .rows import _matrix, _on, _same_device, _type, _vector

PreferenceLoss = collections.namedtuple("PreferenceLoss", "loss logit reward")
PreferenceLoss.__doc__ = """What preference_loss returns, fp32: loss and logit [pairs], reward [2 pairs] (the preferred answer's, then the other's)."""
PolicyLoss = collections.namedtuple("PolicyLoss", "loss kl clipped")
PolicyLoss.__doc__ = """What policy_loss returns, fp32 [sequences]: loss, kl (zeros without ref) and the share of clipped tokens."""

_F32 = torch.float32


def _needed(t, what, n, dtype=_F32):
    if t is None:
        raise ValueError("%s is needed" % what)
    return _vector(t, what, n, dtype)


def _distill(logp, teacher, teacher_lse, temperature, grad_loss, stream):
    kind = _type(teacher, "teacher")
    tp, lt = _matrix(teacher, "teacher")
    rows, m = teacher.shape
    if isinstance(logp, torch.Tensor) and tuple(logp.shape) != (rows, m):
        raise ValueError("logp: shape %s, expected %s" % (tuple(logp.shape), (rows, m)))
    lp, sp = _needed(logp, "logp", rows * m), _vector(teacher_lse, "teacher_lse", rows, _F32)
    up = None if grad_loss is None else _vector(grad_loss, "grad_loss", rows, _F32)
    _same_device(logp, teacher, teacher_lse, grad_loss)
    with _on(logp, stream) as st:
        loss = logp.new_empty(rows)
        if up is None:
            _check(lib().avq_distill_loss(lp, tp, kind, rows, m, lt, sp, temperature, loss.data_ptr(), st))
            return None, loss
        grad = torch.empty_like(logp)
        _check(lib().avq_distill_loss_grad(lp, tp, kind, rows, m, lt, sp, temperature, up, loss.data_ptr(), grad.data_ptr(), st))
    return grad, loss


def distill_loss(logp, teacher, teacher_lse=None, temperature=1.0, stream=None):
    """avq_distill_loss: [rows], from the student's log probabilities [rows][m] of the teacher's best rows, the teacher's
    logits of them (fp32, bf16 or f16; -inf: padding) and, where what lies beside them counts, the lse [rows] of all of its
    logits / temperature."""
    return _distill(logp, teacher, teacher_lse, temperature, None, stream)[1]


def distill_loss_grad(logp, teacher, grad_loss, teacher_lse=None, temperature=1.0, stream=None):
    """avq_distill_loss_grad: (grad_logp [rows][m], loss [rows]) for the gradient of the whole with respect to each row's loss."""
    if grad_loss is None:
        raise ValueError("grad_loss is needed")
    return _distill(logp, teacher, teacher_lse, temperature, grad_loss, stream)


def _sequences(logp, offsets):
    """(tokens, sequences): logp [tokens], offsets [sequences + 1]."""
    if not isinstance(logp, torch.Tensor) or logp.dim() != 1:
        raise ValueError("logp must have one dimension")
    if not isinstance(offsets, torch.Tensor) or offsets.dtype != torch.int32 or not offsets.is_contiguous():
        raise TypeError("offsets must be a contiguous CUDA tensor of dtype torch.int32")
    if offsets.dim() != 1 or offsets.numel() < 1:
        raise ValueError("offsets: shape %s, expected (sequences + 1,)" % (tuple(offsets.shape),))
    return logp.numel(), offsets.numel() - 1


def _part_sums(nbytes, like):
    """(tensor, pointer, bytes) of the scratch that few long sequences need; most calls need none, and most of theirs is host time."""
    if nbytes <= 0:
        _check(nbytes)
        return None, None, 0
    t = torch.empty(nbytes, dtype=torch.uint8, device=like.device)
    return t, t.data_ptr(), nbytes


def _preference(logp, offsets, grad_loss, ref, mask, beta, margin, smoothing, average, stream):
    tokens, sequences = _sequences(logp, offsets)
    if sequences % 2:
        raise ValueError("offsets: %d sequences, expected pairs" % sequences)
    pairs = sequences // 2
    lp, rp, mp = _vector(logp, "logp", tokens, _F32), _vector(ref, "ref", tokens, _F32), _vector(mask, "mask", tokens, torch.bool)
    up = None if grad_loss is None else _vector(grad_loss, "grad_loss", pairs, _F32)
    _same_device(logp, offsets, ref, mask, grad_loss)
    with _on(logp, stream) as st:
        ws, wp, wn = _part_sums(lib().avq_preference_loss_scratch(tokens, pairs), logp)
        # (a few microseconds are most of a small call: tensors made one by one take less than views of one)
        loss, logit, reward = logp.new_empty(pairs), logp.new_empty(pairs), logp.new_empty(sequences)
        args = (lp, rp, mp, tokens, offsets.data_ptr(), pairs, beta, margin, smoothing, 1 if average else 0)
        if up is None:
            grad = None
            _check(lib().avq_preference_loss(*args, loss.data_ptr(), logit.data_ptr(), reward.data_ptr(), wp, wn, st))
        else:
            grad = logp.new_empty(tokens)
            _check(lib().avq_preference_loss_grad(*args, up, loss.data_ptr(), logit.data_ptr(), reward.data_ptr(), grad.data_ptr(), wp, wn, st))
    return grad, PreferenceLoss(loss, logit, reward)


def preference_loss(logp, offsets, ref=None, mask=None, beta=0.1, margin=0.0, smoothing=0.0, average=False, stream=None):
    """avq_preference_loss: sequence 2 p of the tokens' log probabilities is preferred to sequence 2 p + 1. ref: the same of a
    reference model, or None. Returns PreferenceLoss."""
    return _preference(logp, offsets, None, ref, mask, beta, margin, smoothing, average, stream)[1]


def preference_loss_grad(logp, offsets, grad_loss, ref=None, mask=None, beta=0.1, margin=0.0, smoothing=0.0, average=False, stream=None):
    """avq_preference_loss_grad: (grad_logp [tokens], PreferenceLoss) for the gradient of the whole with respect to each pair's loss."""
    if grad_loss is None:
        raise ValueError("grad_loss is needed")
    return _preference(logp, offsets, grad_loss, ref, mask, beta, margin, smoothing, average, stream)


def _policy(logp, old, advantage, offsets, grad_loss, ref, mask, clip, kl, average, each, stream):
    tokens, sequences = _sequences(logp, offsets)
    low, high = clip if isinstance(clip, (tuple, list)) else (clip, clip)
    lp, op, rp = _vector(logp, "logp", tokens, _F32), _needed(old, "old", tokens), _vector(ref, "ref", tokens, _F32)
    mp = _vector(mask, "mask", tokens, torch.bool)
    if not isinstance(advantage, torch.Tensor) or advantage.dim() != 1 or advantage.shape[0] not in (tokens, sequences):
        raise ValueError("advantage must have one value a token or a sequence")
    if each is None:
        each = advantage.shape[0] == tokens
    ap = _vector(advantage, "advantage", tokens if each else sequences, _F32)
    up = None if grad_loss is None else _vector(grad_loss, "grad_loss", sequences, _F32)
    _same_device(logp, old, advantage, offsets, ref, mask, grad_loss)
    with _on(logp, stream) as st:
        ws, wp, wn = _part_sums(lib().avq_policy_loss_scratch(tokens, sequences), logp)
        loss, kls, clipped = logp.new_empty(sequences), logp.new_empty(sequences), logp.new_empty(sequences)
        args = (lp, op, rp, ap, 1 if each else 0, mp, tokens, offsets.data_ptr(), sequences, low, high, kl, 1 if average else 0)
        if up is None:
            grad = None
            _check(lib().avq_policy_loss(*args, loss.data_ptr(), kls.data_ptr(), clipped.data_ptr(), wp, wn, st))
        else:
            grad = logp.new_empty(tokens)
            _check(lib().avq_policy_loss_grad(*args, up, loss.data_ptr(), kls.data_ptr(), clipped.data_ptr(), grad.data_ptr(), wp, wn, st))
    return grad, PolicyLoss(loss, kls, clipped)


def policy_loss(logp, old, advantage, offsets, ref=None, mask=None, clip=0.2, kl=0.0, average=True, each=None, stream=None):
    """avq_policy_loss: logp, old (those of the policy that gave the answers) and ref (of a reference, or None) are log
    probabilities of tokens; advantage has one value a token or a sequence (as each says, or its length: one a token where there
    are as many of both); clip: (low, high) or one for both; kl: the weight of the divergence from ref. Returns PolicyLoss."""
    return _policy(logp, old, advantage, offsets, None, ref, mask, clip, kl, average, each, stream)[1]


def policy_loss_grad(logp, old, advantage, offsets, grad_loss, ref=None, mask=None, clip=0.2, kl=0.0, average=True, each=None, stream=None):
    """avq_policy_loss_grad: (grad_logp [tokens], PolicyLoss) for the gradient of the whole with respect to each sequence's loss."""
    if grad_loss is None:
        raise ValueError("grad_loss is needed")
    return _policy(logp, old, advantage, offsets, grad_loss, ref, mask, clip, kl, average, each, stream)
