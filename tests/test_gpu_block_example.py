"""The example's step against autograd in 64 bits, and its training."""

from __future__ import annotations

import importlib.util
import os

import pytest
import torch

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("distill_step", os.path.join(ROOT, "examples", "distill_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def reference(student, params, x, teacher, ids, tau):
    """Losses and gradients by autograd, in 64 bits."""
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in params.items()}

    def rms(v):
        return v * (v.pow(2).mean(1, keepdim=True) + 1e-5).rsqrt()

    stream = x.cpu().double()
    h = rms(stream) * p["0.ffn_norm"]
    for b in range(student.blocks):
        z = h @ p[f"{b}.w1"].t()
        out = (z * torch.sigmoid(z) * (h @ p[f"{b}.w3"].t())) @ p[f"{b}.w2"].t()
        stream = stream + p[f"{b}.gate"] * rms(out) * p[f"{b}.post_norm"]
        h = rms(stream) * p[f"{b + 1}.ffn_norm" if b + 1 < student.blocks else "norm"]
    logq = torch.log_softmax(h @ p["output"].t() / tau, 1).gather(1, ids.cpu().long())
    logp = torch.log_softmax(teacher.cpu().double() / tau, 1)
    loss = tau * tau * (logp.exp() * (logp - logq)).sum(1)
    loss.mean().backward()
    return loss.detach(), {k: v.grad for k, v in p.items()}


def test_step_against_autograd(example):
    """Every activation and gradient on the way is rounded to bf16 (unit 2^-8):
    some twenty roundings of relative size 2^-9 on average, independent of each
    other, leave a few per cent of a gradient at most in the 2-norm."""
    g = torch.Generator().manual_seed(3)
    student = example.Student(96, 200, 1000, 2)
    ranks = example.Ranks(student, 3, g)
    S = ranks.plan.chunk_elems
    for r in range(3):
        ranks.plan.ag_pack(r, ranks.shards[r], ranks.gathered[r * S:(r + 1) * S])
    ranks.plan.ag_unpack(ranks.gathered, ranks.flat)
    x, teacher, ids = example.batch(student, 130, 20, g)
    weight = torch.full((130,), 1 / 130, device="cuda")
    loss = ranks.student.loss_and_gradients(ranks.params, ranks.grads, x, teacher, ids, weight, 2.0)
    want, grads = reference(student, ranks.params, x, teacher, ids, 2.0)
    assert (loss.cpu().double() - want).norm() <= 0.02 * want.norm()
    for k, v in grads.items():
        off = (ranks.grads[k].cpu().double() - v).norm() / v.norm()
        assert off <= 0.05, (k, off)


def test_training_lowers_the_loss(example):
    losses = example.main(steps=6, tokens=256, vocab=1024, top=32)
    assert losses[-1] < 0.9 * losses[0] and all(b < a for a, b in zip(losses, losses[1:]))
