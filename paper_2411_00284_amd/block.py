"""The operators of a training step between a bucket's copy-out and copy-in.

``BucketPlan.ag_unpack`` leaves a block's full parameters on the device, and
``BucketPlan.rs_pack`` takes their full gradients.  The functions here run
what lies between the two: the norms before and after a block
(``block_norm``), its matrix products (``linear``) and a distillation loss
(``distill_loss``), each with its gradient.  They read the parameters where
the copy-out wrote them and write the gradients where the copy-in reads them.

As everywhere in this package, the caller owns every buffer, outputs are
passed in, a call enqueues its kernels on the current stream (or ``stream``,
a torch stream or a HIP handle) and returns at once.  A wrong argument raises
``TypeError`` or ``ValueError``, a status of the library ``FsdpError``; then
nothing has been enqueued.  Matrices are two-dimensional with contiguous
columns and any row stride; tensors need no alignment beyond an element's.
Types are bfloat16, float16 and float32.  What a call needs as scratch memory
comes from torch's caching allocator, on the call's stream.

The work runs in the HIP kernels behind ``include/fsdp_block.h``, which
states each operator's formulas; sums are held in 32 bits.
"""

from __future__ import annotations

import torch

from . import _native

__all__ = ["block_norm", "block_norm_backward", "linear", "linear_backward", "distill_loss", "distill_loss_backward"]

# As FSDP_ACT_* numbers them.
ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}

_native_block = None


def _lib():
    global _native_block
    if _native_block is None:
        _native_block = _native.load_block()
    return _native_block


def _check(status: int, where: str) -> None:
    if status != 0:
        from .bucket import FsdpError
        raise FsdpError(status, where, _lib().last_error())


def _activation(name) -> int:
    if name not in ACTIVATIONS:
        raise ValueError("activation must be None, 'none', 'relu', 'silu', 'gelu' or 'gelu_tanh'")
    return ACTIVATIONS[name]


def block_norm(x: torch.Tensor, *, branch=None, pre_weight=None, post_weight=None, gate=None, y=None, h=None,
               residual_scale: float = 1.0, branch_scale: float = 1.0, eps: float = 1e-5, stream=None) -> None:
    """The norm after a block with its gate and residual add, and the norm
    before the next one: with ``rms(v) = v / sqrt(mean(v^2) + eps)``,

        n = rms(branch) * post_weight              (branch itself without post_weight)
        y = residual_scale * x + branch_scale * gate * n
        h = rms(y) * pre_weight

    ``x``, ``y`` [tokens, hidden] are the residual stream, of the block's type
    or float32; ``branch`` (the block's output) and ``h`` are of the block's
    type, the weights [hidden] of that or float32.  ``gate`` is [hidden], or
    [rows, hidden] with ``tokens / rows`` consecutive tokens to a row.  Without
    a branch only ``h = rms(residual_scale * x) * pre_weight`` is left.  ``y``
    and ``h`` are written where given; ``y`` may be ``x``, ``h`` may be
    ``branch``.  ``hidden`` is at most 16384.
    """
    _check(_lib().norm(x, branch, post_weight, gate, pre_weight, y, h, eps, residual_scale, branch_scale, stream),
           "fsdp_block_norm")


def block_norm_backward(y: torch.Tensor, *, dy=None, dh=None, branch=None, pre_weight=None, post_weight=None, gate=None,
                        dx=None, dbranch=None, dpre_weight=None, dpost_weight=None, dgate=None,
                        residual_scale: float = 1.0, branch_scale: float = 1.0, eps: float = 1e-5, stream=None) -> None:
    """The gradient of ``block_norm`` from the ``y`` it wrote, the gradient
    ``dy`` that reaches y from what follows it and that of h, ``dh`` (each may
    be left out).  Writes the outputs that are given: ``dx`` (may be ``dy``),
    ``dbranch`` (may be ``branch`` or ``dh``), the weights' gradients summed
    over the tokens, and ``dgate`` summed over the tokens of each row."""
    _check(_lib().norm_grad(y, dy, dh, branch, post_weight, gate, pre_weight, dx, dbranch, dpre_weight, dpost_weight, dgate,
                            eps, residual_scale, branch_scale, stream), "fsdp_block_norm_grad")


def linear(x: torch.Tensor, weight: torch.Tensor, out: torch.Tensor, *, bias=None, activation=None, times=None,
           residual=None, pre=None, stream=None) -> None:
    """A matrix product with its epilogue:

        z   = x @ weight.T + bias
        out = activation(z) * times + residual

    ``x`` [m, k], ``weight`` [n, k] (a parameter as ``ag_unpack`` leaves it,
    viewed in its shape), ``bias`` [n]; ``times``, ``residual`` and ``out``
    [m, n], all of one type.  ``activation`` is None, "relu", "silu", "gelu" or
    "gelu_tanh".  ``pre`` [m, n] receives z, which the gradient of an activation
    needs.  ``out`` may be ``times`` or ``residual``.
    """
    _check(_lib().linear(x, weight, out, bias, _activation(activation), times, residual, pre, stream), "fsdp_block_linear")


def linear_backward(dout: torch.Tensor, x, weight: torch.Tensor, *, activation=None, pre=None, times=None,
                    dx=None, dweight=None, dbias=None, dtimes=None, stream=None) -> None:
    """The gradient of ``linear`` from that of its output:

        dz = dout * times * activation'(z)         dtimes  = dout * activation(z)
        dx = dz @ weight                           dweight = dz.T @ x
        dbias = dz summed over the rows            (the residual's gradient is dout itself)

    Writes the outputs that are given.  ``pre`` is what ``linear`` wrote there;
    it is needed with an activation and for ``dtimes`` (which may be
    ``times``).  ``x`` and ``pre`` may each be a ``step.Checkpoint``."""
    if isinstance(x, tuple) or isinstance(pre, tuple):
        from . import step
        return step._check(step._lib().linear_grad(dout, x, weight, _activation(activation), pre, times, dx, dweight, dbias, dtimes,
                                                   stream), "fsdp_step_linear_grad")
    _check(_lib().linear_grad(dout, x, weight, _activation(activation), pre, times, dx, dweight, dbias, dtimes, stream),
           "fsdp_block_linear_grad")


def distill_loss(logits: torch.Tensor, teacher: torch.Tensor, ids: torch.Tensor, loss=None, lse=None, *,
                 temperature: float = 1.0, teacher_lse=None, dloss=None, dlogits=None, stream=None) -> None:
    """Distillation from a teacher's top logits, for every token:

        p = softmax(teacher / temperature)         over the token's entries
        loss = temperature^2 * sum_k p_k * (log p_k - log softmax(logits / temperature)[ids_k])

    ``logits`` [tokens, vocab]; ``teacher`` [tokens, top] holds the teacher's
    logits at the places ``ids`` (int32 or int64; negative: no entry).  With
    ``teacher_lse`` [tokens] (float32), the logsumexp of the teacher's whole row
    divided by the temperature, p is its probabilities over the whole vocabulary
    instead.  ``loss`` and ``lse`` (the logsumexp of logits / temperature, for
    ``distill_loss_backward``) are [tokens] in float32.  With ``dloss`` [tokens],
    the weight of each token's loss, ``dlogits`` receives the gradient in the
    same pass; it may be ``logits``.  A token without entries has loss and
    gradient 0, one with an id beyond the vocabulary NaN.  ``top`` is at most
    1024.
    """
    _check(_lib().distill(False, logits, teacher, ids, teacher_lse, dloss, loss, lse, dlogits, temperature, stream),
           "fsdp_block_distill")


def distill_loss_backward(dloss: torch.Tensor, logits: torch.Tensor, teacher: torch.Tensor, ids: torch.Tensor,
                          lse: torch.Tensor, dlogits: torch.Tensor, *, temperature: float = 1.0, teacher_lse=None,
                          stream=None) -> None:
    """The gradient of ``distill_loss`` with respect to the logits, from the
    ``lse`` it wrote and the gradient ``dloss`` [tokens] of the losses.
    ``dlogits`` may be ``logits``."""
    _check(_lib().distill(True, logits, teacher, ids, teacher_lse, dloss, None, lse, dlogits, temperature, stream),
           "fsdp_block_distill_grad")
