"""More operators of a training step between a bucket's copy-out and copy-in.

``gated_linear`` is both projections of a gated feed-forward with their
activation and product; ``Checkpoint`` is a matrix kept in 8 bits for the
backward pass, which the gradients here and ``block.linear_backward`` read as
they would the matrix itself; ``policy_loss`` is the clipped policy loss of
sampled tokens.  Each has its gradient.

Buffers, streams, errors, types and strides are as in ``block``.  The work runs
in the HIP kernels behind ``include/fsdp_step.h``, which states each operator's
formulas.
"""

from __future__ import annotations

from typing import NamedTuple

import torch

from . import _native
from .block import _activation

__all__ = ["Checkpoint", "checkpoint_save", "checkpoint_restore", "gated_linear", "gated_linear_backward", "policy_loss",
           "policy_loss_backward"]

GROUP = 32                   # FSDP_STEP_GROUP

_native_step = None


def _lib():
    global _native_step
    if _native_step is None:
        _native_step = _native.load_step()
    return _native_step


def _check(status: int, where: str) -> None:
    if status != 0:
        from .bucket import FsdpError
        raise FsdpError(status, where, _lib().last_error())


class Checkpoint(NamedTuple):
    """A matrix [rows, cols] in 8 bits: ``codes`` (int8, its shape) times the
    powers of two of ``scales`` (uint8, [rows, ceil(cols / 32)], the exponent +
    127), one for each 32 neighbouring columns of a row.  A scale is the least
    with which its largest value rounds to 127 or less; codes are rounded to
    nearest even.  A group that holds a value that is not finite stands for NaN
    (scale 255).  What it stands for is exact in every type between the ends
    of its range: from 65280 on in fp16, and from 255 * 2^120 on in all, the
    largest of a group may become infinite; groups below 2^-18 that were not
    saved from fp16 are rounded to multiples of 2^-24 where they are read as
    fp16.  Both tensors may have any row stride."""
    codes: torch.Tensor
    scales: torch.Tensor

    @classmethod
    def empty(cls, rows: int, cols: int, device="cuda") -> "Checkpoint":
        """Buffers for a matrix [rows, cols]: 33 bytes for 32 values."""
        return cls(torch.empty(rows, cols, dtype=torch.int8, device=device),
                   torch.empty(rows, -(-cols // GROUP), dtype=torch.uint8, device=device))


def checkpoint_save(x: torch.Tensor, checkpoint: Checkpoint, *, stream=None) -> None:
    """``x`` [rows, cols] to 8 bits."""
    _check(_lib().save(x, checkpoint, stream), "fsdp_step_save")


def checkpoint_restore(checkpoint: Checkpoint, out: torch.Tensor, *, stream=None) -> None:
    """What the 8 bits stand for, to ``out`` [rows, cols]."""
    _check(_lib().restore(checkpoint, out, stream), "fsdp_step_restore")


def gated_linear(x: torch.Tensor, gate_weight: torch.Tensor, up_weight: torch.Tensor, out: torch.Tensor, *, activation="silu",
                 gate=None, up=None, stream=None) -> None:
    """Both projections of a gated feed-forward, in one product:

        g = x @ gate_weight.T        u = x @ up_weight.T        out = activation(g) * u

    ``x`` [m, k], the weights [n, k], ``out`` [m, n], all of one type;
    activations as ``linear``'s.  ``gate`` and ``up`` keep g and u for the
    gradient: both or neither, two tensors [m, n] of that type, or two
    ``Checkpoint``.
    """
    _check(_lib().gated(x, gate_weight, up_weight, out, _activation(activation), gate, up, stream), "fsdp_step_gated")


def gated_linear_backward(dout: torch.Tensor, x, gate_weight: torch.Tensor, up_weight: torch.Tensor, gate, up, *,
                          activation="silu", out=None, dx=None, dgate_weight=None, dup_weight=None, stream=None) -> None:
    """The gradient of ``gated_linear`` from that of its output and from what
    it kept:

        dg = dout * u * activation'(g)          du = dout * activation(g)
        dx = dg @ gate_weight + du @ up_weight
        dgate_weight = dg.T @ x                 dup_weight = du.T @ x

    Writes the outputs that are given (the weights' gradients both or neither).
    ``out`` receives activation(g) * u again, so that the product after it need
    not keep its input; it may be ``dout``.  ``x``, and ``gate`` and ``up``
    alike, are tensors or ``Checkpoint``."""
    _check(_lib().gated_grad(dout, x, gate_weight, up_weight, gate, up, _activation(activation), out, dx, dgate_weight, dup_weight,
                             stream), "fsdp_step_gated_grad")


def policy_loss(logits: torch.Tensor, actions: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor, loss=None, logp=None,
                lse=None, *, ref_logp=None, clip_low: float = 0.2, clip_high: float = 0.2, kl_weight: float = 0.0,
                temperature: float = 1.0, dloss=None, dlogits=None, stream=None) -> None:
    """The clipped policy loss of sampled tokens with its KL term, for every
    token:

        logp = log softmax(logits / temperature)[action]        r = exp(logp - old_logp)
        loss = -min(r * advantage, clip(r, 1 - clip_low, 1 + clip_high) * advantage)
               + kl_weight * (exp(d) - d - 1),      d = ref_logp - logp

    ``logits`` [tokens, vocab]; ``actions`` [tokens] (int32 or int64; negative:
    the token counts for nothing); ``old_logp``, ``advantages``, ``ref_logp``
    (needed with a ``kl_weight``), ``loss``, ``logp`` and ``lse`` (the logsumexp
    of logits / temperature, for ``policy_loss_backward``) are [tokens] in
    float32.  With ``dloss`` [tokens], the weight of each token's loss,
    ``dlogits`` receives the gradient in the same pass; it may be ``logits``.  A
    masked token has loss, logp and gradient 0, one with an action beyond the
    vocabulary NaN.
    """
    _check(_lib().policy(False, logits, actions, old_logp, advantages, ref_logp, dloss, loss, logp, lse, dlogits, clip_low, clip_high,
                         kl_weight, temperature, stream), "fsdp_step_policy")


def policy_loss_backward(dloss: torch.Tensor, logits: torch.Tensor, actions: torch.Tensor, old_logp: torch.Tensor,
                         advantages: torch.Tensor, lse: torch.Tensor, dlogits: torch.Tensor, *, ref_logp=None, clip_low: float = 0.2,
                         clip_high: float = 0.2, kl_weight: float = 0.0, temperature: float = 1.0, stream=None) -> None:
    """The gradient of ``policy_loss`` with respect to the logits, from the
    ``lse`` it wrote for them and the gradient ``dloss`` [tokens] of the losses.
    ``dlogits`` may be ``logits``.  An ``lse`` is rounded to 32 bits: up to a
    size of 2^14 the probabilities and the ratio share what that leaves of them
    (2^-24 of its size); of larger ones, as a small temperature or a row at a
    mask's value has them, the row's own is formed again."""
    _check(_lib().policy(True, logits, actions, old_logp, advantages, ref_logp, dloss, None, None, lse, dlogits, clip_low, clip_high,
                         kl_weight, temperature, stream), "fsdp_step_policy_grad")
