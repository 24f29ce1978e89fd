"""Distillation over masked logits: a mask of a finite value (the type's lowest,
or -1e10) over runs of the vocabulary, over all of it but one place, and over
whole rows, in every launch form; the teacher's entries masked likewise.
Against the formulas in 64 bits, shifted by the row's largest value, so that
they hold for rows that are one value throughout."""

from __future__ import annotations

import math

import pytest
import torch

from block_util import DTYPES, E32, close, normal
from paper_2411_00284_amd import distill_loss, distill_loss_backward

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

TOP = 12


def shifted(v, tau):
    """(log softmax, its largest value over tau, log of its sum), row by row."""
    top = v.max(1, keepdim=True).values
    s = (v - top) / tau
    log_sum = torch.exp(s).sum(1, keepdim=True).log()
    return s - log_sum, top / tau, log_sum


def reference(logits, teacher, ids, tau, dloss, lse=None):
    """(loss, lse, dlogits) in 64 bits and the bounds of their errors: an
    exponential of x is off by a few units of 2^-24 of itself, times 1 + |x|."""
    logq, far, log_sum = shifted(logits.double(), tau)
    own = (far + log_sum)[:, 0]
    if lse is not None:
        logq = logits.double() / tau - lse.double()[:, None]
    logp = shifted(teacher.double(), tau)[0]
    p, at = torch.exp(logp), ids.long()
    picked = logq.gather(1, at)
    few = 24 * E32
    held = p > 0
    loss = tau * tau * torch.where(held, p * (logp - picked), 0.0).sum(1)
    eloss = tau * tau * few * torch.where(held, p * (1 + logp.abs()) * ((logp - picked).abs() + 1), 0.0).sum(1)
    q, c = torch.exp(logq), (dloss * tau).double()[:, None]
    dense = torch.zeros_like(logq).scatter_add_(1, at, p)
    few_p = torch.zeros_like(logq).scatter_add_(1, at, p * (1 + logp.abs().clamp(max=200)))
    top = logp.abs().clamp(max=200).max(1, keepdim=True).values
    eg = few * c.abs() * ((2 + top + logq.abs().clamp(max=200)) * q + few_p)
    return loss, own, c * (q - dense), eloss, 4 * E32 * (1 + own.abs()), eg


def rows(vocab, dtype, low):
    """(logits, teacher, ids, whether the row's lse can give its gradient): the
    entries lie where the student is not masked, or anywhere if all is."""
    base = normal(11, 1, vocab, dtype=dtype, scale=2.5)[0]
    half, unit = vocab // 2, 16 // base.element_size()
    last = vocab - vocab % unit                                # the elements after the whole units
    g = torch.Generator().manual_seed(5)
    out = []

    def add(keep, fill=low, saved=True, teacher=None, value=None):
        """`keep`: the places that are not masked."""
        logits = torch.full((vocab,), fill, dtype=dtype) if value is None else value
        live = torch.arange(vocab)[keep]
        logits[keep] = base[keep]
        where = live if live.numel() else torch.arange(vocab)
        ids = where[torch.randint(0, where.numel(), (TOP,), generator=g)]
        out.append((logits, normal(20 + len(out), TOP) if teacher is None else teacher, ids, saved))

    add(slice(half, vocab))                                    # the first half is masked: whole units of every thread
    add(slice(0, half))
    add(slice(min(8192, half), vocab))
    add(slice(half, half + 1))                                 # all but one place
    add(slice(0, 1))
    add(slice(vocab - 1, vocab))
    add(slice(0, last if last < vocab else vocab - 1))         # the last elements only are masked
    add(slice(0, 0), saved=False)                              # all of it
    mixed = torch.full((vocab,), low, dtype=dtype)
    mixed[:half] = -math.inf
    add(slice(vocab - 3, vocab), value=mixed.clone())
    mixed = torch.full((vocab,), -math.inf, dtype=dtype)
    mixed[half:] = low
    add(slice(3, 5), value=mixed)
    add(slice(0, vocab), teacher=torch.full((TOP,), torch.finfo(torch.float32).min))        # the teacher's entries: all masked,
    teacher = normal(77, TOP)
    teacher[2:9] = torch.finfo(torch.float32).min
    add(slice(0, vocab), teacher=teacher)                      # and some
    logits, teacher, ids, saved = zip(*out)
    return torch.stack(logits), torch.stack(teacher), torch.stack(ids), torch.tensor(saved)


# tokens, vocabulary in 16 bits and in 32: one for each launch form (threads of a row, units that each holds)
FORMS = [(12, 2003, 2003), (24, 20011, 20011), (300, 20011, 12001), (300, 40009, 20011)]


@pytest.mark.parametrize("tau", [1.0, 2.0, 0.5])
@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("dtype,low", [("bf16", None), ("bf16", -1e10), ("f16", None), ("f32", None), ("f32", -1e10)])
def test_masked(dtype, low, form, tau):
    dtype = DTYPES[dtype]
    tokens, vocab = form[0], form[2 if dtype is torch.float32 else 1]
    low = torch.finfo(dtype).min if low is None else low
    print("distill masks", dtype, low, form, tau, flush=True)
    logits, teacher, ids, saved = rows(vocab, dtype, low)
    n = logits.shape[0]
    of = torch.arange(tokens) % n if tokens >= n else torch.arange(n)          # the rows again and again
    dloss = normal(3, n).abs() + 0.5
    gl, gt, gi, gd = logits[of].cuda(), teacher[of].cuda(), ids[of].cuda(), dloss[of].cuda()
    t = gl.shape[0]
    loss, lse, dl = torch.empty(t, device="cuda"), torch.empty(t, device="cuda"), torch.empty_like(gl)
    distill_loss(gl, gt, gi, loss, lse, temperature=tau, dloss=gd, dlogits=dl)
    wl, we, wg, el, ee, eg = reference(logits, teacher, ids, tau, dloss)
    close(loss[:n], wl, el, "loss")
    close(lse[:n], we, ee, "lse")
    close(dl[:n], wg, eg, "dlogits")
    for first in range(n, t - n + 1, n):
        assert torch.equal(dl[first:first + n], dl[:n]) and torch.equal(loss[first:first + n], loss[:n])
    alone = torch.empty(t, device="cuda")
    distill_loss(gl, gt, gi, alone, temperature=tau)
    close(alone[:n], wl, el, "loss alone")
    back = torch.empty_like(gl)
    distill_loss_backward(gd, gl, gt, gi, lse, back, temperature=tau)
    _, _, wg, _, _, eg = reference(logits[saved], teacher[saved], ids[saved], tau, dloss[saved], lse[:n].cpu()[saved])
    close(back[:n][saved.cuda()], wg, eg, "dlogits from lse")


@pytest.mark.parametrize("tau", [1e-3, 1e-20, 1e-30, 2.0 ** -126, 2.0 ** -140])
@pytest.mark.parametrize("vocab", [2003, 20011])
def test_small_temperatures(tau, vocab):
    """q and p go over to one hot; tau is subnormal at last."""
    tau = torch.tensor(tau).item()
    n = 5
    logits = normal(3, n, vocab).round(decimals=1)
    logits[:, 17] = 9.0                                        # the largest by a margin
    logits[1, 18] = 9.0                                        # a tie
    teacher = normal(4, n, TOP).round(decimals=1)
    teacher[:, 5] = 8.0
    ids = torch.randint(20, vocab, (n, TOP), generator=torch.Generator().manual_seed(1))
    ids[:, 5] = 17
    ids[2, 5] = 30                                             # the teacher's choice is not the student's
    dloss = torch.ones(n) / tau if tau > 1e-25 else torch.ones(n)
    loss, dl = torch.empty(n, device="cuda"), torch.empty(n, vocab, device="cuda")
    distill_loss(logits.cuda(), teacher.cuda(), ids.cuda(), loss, temperature=tau, dloss=dloss.cuda(), dlogits=dl)
    wl, _, wg, el, _, eg = reference(logits, teacher, ids, tau, dloss)
    close(loss, wl, el, "loss")
    close(dl, wg, eg, "dlogits")
