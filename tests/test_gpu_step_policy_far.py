"""The policy loss's gradient from a saved logsumexp that 32 bits hold too
coarsely: small temperatures, and rows at a mask's finite value or far from 0.

From 2^14 on the call takes the row's own maximum and sum again, so that its
results are those of softmax(logits / temperature); below, those of the value that
was saved, whose rounding (2^-11 at most) they share."""

from __future__ import annotations

import pytest
import torch

from block_util import DTYPES, close
from paper_2411_00284_amd import policy_loss, policy_loss_backward
from test_gpu_step_policy import make, options, reference

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

KEPT = 2.0 ** 14


def check(made, opt, where):
    """The gradient from the saved lse against 64 bits, and in the logits' place."""
    logits, actions, old, adv, ref, dloss = made
    g = [v.cuda() for v in (logits, actions, old, adv)]
    more = dict(opt, ref_logp=ref.cuda()) if opt["kl_weight"] else opt
    lse = torch.empty(logits.shape[0], device="cuda")
    policy_loss(*g, lse=lse, **more)
    saved = lse.cpu()
    back = torch.full_like(g[0], float("nan"))
    policy_loss_backward(dloss.cuda(), *g, lse, back, **more)
    far, counts = saved.abs() >= KEPT, (actions >= 0) & (dloss != 0)
    want, off = torch.zeros(logits.shape, dtype=torch.float64), torch.zeros(logits.shape, dtype=torch.float64)
    for rows, given in ((counts & far, None), (counts & ~far, saved)):
        if bool(rows.any()):
            part = reference(*(v[rows] for v in made[:5]), opt, dloss[rows], None if given is None else given[rows])
            want[rows], off[rows] = part[0][3], part[1][3]
    off += (dloss.double() / opt["temperature"] * adv.double()).abs()[:, None] * 2.0 ** -120 * counts[:, None]     # exponentials below 2^-126 are 0
    assert bool(torch.isfinite(off).all())
    close(back, want, off, where)
    policy_loss_backward(dloss.cuda(), *g, lse, g[0], **more)
    assert torch.equal(g[0], back), where
    return far


@pytest.mark.parametrize("power", [-10, -11, -13, -17, -20, -66, -126])
@pytest.mark.parametrize("vocab", [300, 20011])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_temperatures(dtype, vocab, power):
    """Some actions that stand out, some that have no probability, a prompt's and one without weight."""
    print("far lse", dtype, vocab, power, flush=True)
    tau = torch.tensor(1.3 * 2.0 ** power).item()               # a 32-bit value, of which no logit is a multiple
    made = list(make(111, 12, vocab, DTYPES[dtype], tau))
    logits, actions = made[0], made[1]
    actions[:6], actions[10] = logits[:6].float().argmax(1), 0
    logits[6:8, :2], actions[6:8] = 12.0, 1                     # of two that share all of it
    d = logits.double() - logits.double().max(1, keepdim=True).values
    now = torch.log_softmax(d / tau, 1).gather(1, actions[:, None])[:, 0]
    made[2] = now.clamp(min=-2.0 ** 25).float() + torch.tensor([0.1, -0.1, 0.3] * 4)
    made[4] = made[2] + 0.2
    actions[10], made[5][11] = -1, 0.0
    far = check(made, options(0.1 if power >= -20 else 0.0, tau=tau), (dtype, vocab, power))
    assert not far[10]
    if power != -11:                                            # rows on both sides
        assert far[:10].tolist() == [power < -11] * 10


@pytest.mark.parametrize("vocab", [300, 6001, 20011])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_rows_far_from_zero(dtype, vocab):
    """Rows at the type's lowest value, all or all but a run at -inf, beside a higher mask; rows of large
    logits of either sign."""
    print("far rows", dtype, vocab, flush=True)
    dtype = DTYPES[dtype]
    made = list(make(121, 7, vocab, dtype))
    logits, actions = made[0], made[1]
    lowest = torch.finfo(dtype).min
    logits[:3] = lowest
    logits[1, vocab // 2:] = float("-inf")
    logits[2, ::3] = -1e4
    logits[3] += 3e4
    logits[4] -= 5e4
    actions[:3] = torch.tensor([5, 7, 9])
    d = logits.double() - logits.double().max(1, keepdim=True).values
    now = torch.log_softmax(d, 1).gather(1, actions[:, None])[:, 0].float()
    made[2], made[4] = now + torch.tensor([0.1, -0.1, 0.05, 0.3, -0.3, 0.1, 0.0]), now + 0.2
    assert check(made, options(), (dtype, vocab)).tolist() == [True, True, False, True, True, False, False]


@pytest.mark.parametrize("tokens,vocab", [(300, 2003), (300, 6001), (9, 20011), (300, 20011)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_bits_of_the_one_pass(dtype, tokens, vocab):
    """In every form of the kernel that both calls take: the row's own sums are the first call's, and so are all bits."""
    print("far forms", dtype, tokens, vocab, flush=True)
    logits, actions, old, adv, ref, dloss = make(131, tokens, vocab, DTYPES[dtype])
    logits[::3] += 3e4
    actions[::5], dloss[1::7] = -1, 0.0
    g, more = [v.cuda() for v in (logits, actions, old, adv)], dict(options(), ref_logp=ref.cuda(), dloss=dloss.cuda())
    lse, first, back = torch.empty(tokens, device="cuda"), torch.empty_like(g[0]), torch.full_like(g[0], float("nan"))
    policy_loss(*g, lse=lse, dlogits=first, **more)
    policy_loss_backward(more.pop("dloss"), *g, lse, back, **more)
    far = lse.abs() >= KEPT
    assert bool(far.any()) and not bool(far.all()) and torch.equal(first[far], back[far])
    masked = g[1] < 0
    assert not bool(back[masked].any()) and not bool(back[1::7].any()) and bool(back[far].any())
