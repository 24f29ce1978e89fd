"""Distillation from a teacher's top logits, against the formulas in 64 bits, at
the sizes, types and values where it can go wrong."""

from __future__ import annotations

import math

import pytest
import torch

from block_util import DTYPES, E32, Mat, blank, close, normal
from paper_2411_00284_amd import FsdpError, distill_loss, distill_loss_backward

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def reference(logits, teacher, ids, tau, teacher_lse, dloss, lse=None):
    """(loss, lse, dlogits) in 64 bits and the bounds of their errors.  An
    exponential of x is off by a few units of 2^-24 of itself, times 1 + |x|."""
    s, held = logits.double() / tau, ids >= 0
    v = torch.where(held, teacher.double() / tau, -math.inf)
    at = torch.where(held, ids, 0).long()
    live = (v > -math.inf).any(1)
    norm = teacher_lse.double() if teacher_lse is not None else torch.where(live, torch.logsumexp(v, 1), 0.0)
    logp = v - norm[:, None]
    p = torch.exp(logp)
    own = torch.logsumexp(s, 1)
    logq = s - (own if lse is None else lse.double())[:, None]
    picked = logq.gather(1, at)
    terms = torch.where(held & (p > 0), p * (logp - picked), 0.0)
    loss = torch.where(live, tau * tau * terms.sum(1), 0.0)
    # every term carries its p's error and that of the two logsumexps (whose sums lose some units of 2^-24)
    few = 24 * E32
    spread = torch.where(held & (p > 0), p * (1 + logp.abs()) * ((logp - picked).abs() + 1), 0.0)
    eloss = tau * tau * few * spread.sum(1)
    q, mass = torch.exp(logq), p.sum(1, keepdim=True)
    dense = torch.zeros_like(s).scatter_add_(1, at, torch.where(held, p, 0.0))
    c = (dloss * tau).double()[:, None]
    grad = torch.where((live & (dloss != 0))[:, None], c * (mass * q - dense), 0.0)
    # a saved lse is rounded to 32 bits: that is in `lse` already
    far = (1 + logq.abs().clamp(max=200)) * mass * q
    few_p = torch.zeros_like(s).scatter_add_(1, at, torch.where(held, p * (1 + logp.abs().clamp(max=200)), 0.0))
    top = torch.where(held, logp, 0.0).abs().clamp(max=200).max(1, keepdim=True).values
    eg = few * c.abs() * (far + few_p + (1 + top) * mass * q)
    return loss, torch.where(live, own, 0.0), grad, eloss, 4 * E32 * (1 + own.abs()), eg


def make(seed, tokens, vocab, top, dtype, teacher_dtype, scale=2.5):
    logits = normal(seed, tokens, vocab, dtype=dtype, scale=scale)
    whole = logits.float() * 0.8 + normal(seed + 1, tokens, vocab)
    values, ids = whole.topk(top, 1)
    return logits, values.to(teacher_dtype), ids, whole


# tokens, vocab, top, logits' type, teacher's type, ids' type, temperature, tail, gap, shift
SHAPES = [
    (1, 1, 1, "f32", "f32", torch.int32, 1.0, False, 0, 0),
    (3, 2, 2, "bf16", "bf16", torch.int64, 2.0, False, 0, 0),
    (4, 1000, 1, "f16", "f32", torch.int32, 0.5, False, 3, 1),
    (2, 4096, 1024, "bf16", "f16", torch.int32, 1.0, False, 0, 0),
    (7, 8191, 64, "bf16", "bf16", torch.int64, 2.0, True, 1, 1),
    (5, 8193, 100, "f32", "bf16", torch.int32, 1.5, True, 1, 0),
    (3, 16384, 65, "f16", "f16", torch.int32, 1.0, False, 0, 0),
    (2, 32001, 256, "f32", "f32", torch.int64, 0.7, True, 0, 1),
    (9, 50257, 128, "bf16", "f32", torch.int32, 3.0, False, 7, 3),
    (2, 65537, 20, "f16", "bf16", torch.int32, 1.0, True, 0, 1),
    (2, 128256, 64, "bf16", "bf16", torch.int32, 2.0, False, 0, 0),
    (1, 131080, 512, "bf16", "f32", torch.int64, 1.0, False, 0, 0),
    (1, 151936, 50, "f32", "f32", torch.int32, 1.0, False, 0, 0),
    (1, 300001, 50, "bf16", "f32", torch.int32, 1.0, False, 0, 1),
]


@pytest.mark.parametrize("case", SHAPES, ids=str)
def test_loss_and_gradient(case):
    tokens, vocab, top, dtype, teacher_dtype, id_type, tau, tail, gap, shift = case
    dtype, teacher_dtype = DTYPES[dtype], DTYPES[teacher_dtype]
    print("distill", case, flush=True)
    logits, values, ids, whole = make(11, tokens, vocab, top, dtype, teacher_dtype)
    tlse = torch.logsumexp(whole / tau, 1) if tail else None
    dloss = normal(13, tokens)
    gl, gt, gi = Mat(logits, gap, shift), values.cuda(), ids.to(id_type).cuda()
    gtl = None if tlse is None else tlse.cuda()
    loss, lse = blank(None, tokens, torch.float32, 0, shift), blank(None, tokens, torch.float32)
    dl = blank(tokens, vocab, dtype, gap, shift)
    distill_loss(gl.t, gt, gi, loss.t, lse.t, temperature=tau, teacher_lse=gtl, dloss=dloss.cuda(), dlogits=dl.t)
    wl, we, wg, el, ee, eg = reference(logits, values, ids, tau, tlse, dloss)
    close(loss.t, wl, el, "loss")
    close(lse.t, we, ee, "lse")
    close(dl.t, wg, eg, "dlogits")
    assert dl.intact() and loss.intact() and lse.intact() and gl.intact()
    alone = torch.empty(tokens, device="cuda")
    distill_loss(gl.t, gt, gi, alone, temperature=tau, teacher_lse=gtl)
    assert torch.equal(alone, loss.t)
    back = blank(tokens, vocab, dtype, gap, shift)
    distill_loss_backward(dloss.cuda(), gl.t, gt, gi, lse.t, back.t, temperature=tau, teacher_lse=gtl)
    _, _, wg, _, _, eg = reference(logits, values, ids, tau, tlse, dloss, lse.t.cpu())
    close(back.t, wg, eg, "dlogits from lse")
    assert back.intact()
    distill_loss_backward(dloss.cuda(), gl.t, gt, gi, lse.t, gl.t, temperature=tau, teacher_lse=gtl)
    assert torch.equal(gl.t, back.t) and gl.intact()           # in place


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [700, 20011])
def test_rows(dtype, vocab):
    """Rows with fewer entries, none, entries of no mass, repeated ids, a zero
    weight over NaN, masked logits; ids beyond the vocabulary are NaN."""
    dtype = DTYPES[dtype]
    tokens, top, tau = 12, 40, 1.25
    logits, values, ids, _ = make(21, tokens, vocab, top, dtype, torch.float32)
    low = torch.finfo(dtype).min
    dloss = normal(23, tokens)
    ids[0] = -1
    values[0] = math.nan                                       # not used
    logits[0] = math.nan
    ids[1, 5:], values[1, 5:] = -1, math.inf
    ids[2, 0], ids[2, 3] = -7, -2147483648
    values[3] = -math.inf
    ids[4, 7] = ids[4, 2]
    ids[5] = ids[5, 0]
    logits[6], dloss[6] = math.nan, 0.0
    masked = torch.ones(vocab, dtype=torch.bool)
    masked[ids[7].long()] = False
    masked[::3] = False
    logits[7, masked] = -math.inf
    logits[8, masked] = low
    values[9, 10:] = torch.finfo(torch.float32).min
    logits[10, ids[10, 1].long()] = -math.inf                  # an entry that the student rules out: the loss is infinite
    ids[11, 3] = vocab
    gl, gt, gi, gd = logits.cuda(), values.cuda(), ids.to(torch.int32).cuda(), dloss.cuda()
    loss, lse, dl = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda"), torch.empty_like(gl)
    distill_loss(gl, gt, gi, loss, lse, temperature=tau, dloss=gd, dlogits=dl)
    fine = [1, 2, 3, 4, 5, 7, 8, 9, 10]
    wl, we, wg, el, ee, eg = reference(logits[fine], values[fine], ids[fine], tau, None, dloss[fine])
    assert wl[-1] == math.inf
    close(loss[fine], wl, el, "loss")
    close(lse[fine], we, ee, "lse")
    close(dl[fine], wg, eg, "dlogits")
    assert loss[0] == 0 and lse[0] == 0 and not dl[0].any() and not dl[3].any()
    assert bool(loss[6].isnan()) and not dl[6].any()
    assert bool(loss[11].isnan()) and bool(dl[11].isnan().all())
    back = torch.empty_like(gl)
    distill_loss_backward(gd, gl, gt, gi, lse, back, temperature=tau)
    _, _, wg, _, _, eg = reference(logits[fine], values[fine], ids[fine], tau, None, dloss[fine], lse[fine].cpu())
    close(back[fine], wg, eg, "dlogits from lse")
    assert not back[0].any() and not back[6].any() and bool(back[11].isnan().all())
    wide = gi.long()
    wide[11, 3] = 1 << 40                                      # and in 64 bits
    again = torch.empty_like(gl)
    distill_loss(gl, gt, wide, loss, lse, temperature=tau, dloss=gd, dlogits=again)
    assert torch.equal(again.view(torch.uint8), dl.view(torch.uint8))


def test_far_logits():
    """Logits far from 0: the same loss and gradient as near it."""
    logits, values, ids, _ = make(31, 3, 3001, 30, torch.float32, torch.float32)
    logits, values = logits.round(decimals=1) * 64, values
    logits = (logits / 8).round() * 0.125
    dloss = torch.ones(3)
    for shift in (0.0, 4096.0, -16384.0):
        moved = logits + shift                                 # exact: eighths
        loss, dl = torch.empty(3, device="cuda"), torch.empty(3, 3001, device="cuda")
        distill_loss(moved.cuda(), values.cuda(), ids.cuda(), loss, temperature=1.0, dloss=dloss.cuda(), dlogits=dl)
        wl, _, wg, el, _, eg = reference(logits, values, ids, 1.0, None, dloss)
        close(loss, wl, el, "loss")
        close(dl, wg, eg, "dlogits")


def test_no_tokens():
    e = torch.empty(0, 100, dtype=torch.bfloat16, device="cuda")
    t, i = torch.empty(0, 4, device="cuda"), torch.empty(0, 4, dtype=torch.int32, device="cuda")
    n = torch.empty(0, device="cuda")
    distill_loss(e, t, i, n, n, dloss=n, dlogits=torch.empty_like(e))
    distill_loss_backward(n, e, t, i, n, torch.empty_like(e))


def test_differences():
    """The gradient against central differences of the forward kernel, in
    float32: off by step^2 / 6 third derivatives (below tau^2 / tau^3 for a unit
    direction) and by the loss's rounding over the step."""
    tau, step = 1.5, 3e-2
    logits, values, ids, _ = make(41, 4, 60, 9, torch.float32, torch.float32)
    dl, lse, loss = torch.empty(4, 60, device="cuda"), torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    one = torch.ones(4, device="cuda")
    distill_loss(logits.cuda(), values.cuda(), ids.cuda(), loss, lse, temperature=tau, dloss=one, dlogits=dl)
    d = normal(43, 4, 60)
    d = d / d.norm(dim=1, keepdim=True)
    side = []
    for sign in (1, -1):
        out = torch.empty(4, device="cuda")
        distill_loss((logits + sign * step * d).cuda(), values.cuda(), ids.cuda(), out, temperature=tau)
        side.append(out.cpu().double())
    slope = (dl.cpu().double() * d).sum(1)
    assert bool(((side[0] - side[1]) / (2 * step) - slope).abs().max() <= step ** 2 / 6 / tau + 50 * E32 * (1 + loss.abs().max()) / step)
    assert bool(dl.double().sum(1).abs().max() < 60 * 24 * E32)          # a softmax's gradient sums to 0


def test_repeats_and_streams():
    logits, values, ids, _ = make(51, 40, 9001, 33, torch.bfloat16, torch.bfloat16)
    gl, gt, gi, gd = logits.cuda(), values.cuda(), ids.cuda(), normal(53, 40).cuda()
    side = torch.cuda.Stream()
    got = []
    for stream in (None, side, side.cuda_stream, None):
        loss, dl = torch.empty(40, device="cuda"), torch.empty_like(gl)
        torch.cuda.synchronize()
        distill_loss(gl, gt, gi, loss, dloss=gd, dlogits=dl, stream=stream)
        torch.cuda.synchronize()
        got.append((loss, dl))
    assert all(torch.equal(a, b) for g in got[1:] for a, b in zip(g, got[0]))


def test_refusals():
    s = torch.zeros(4, 100, dtype=torch.bfloat16, device="cuda")
    t, i = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 8, dtype=torch.int32, device="cuda")
    loss, dl = torch.full((4,), 3.0, device="cuda"), torch.full_like(s, 3)
    for error, args, kwargs in [
        (ValueError, (s, t[:3], i, loss), {}),
        (ValueError, (s, t, i[:, :7], loss), {}),
        (ValueError, (s[0], t, i, loss), {}),
        (ValueError, (s, t, i, loss[:3]), {}),
        (TypeError, (s, t, i.float(), loss), {}),
        (TypeError, (s, t, i.short(), loss), {}),
        (TypeError, (s, t, i, loss.half()), {}),
        (TypeError, (s, t.double(), i, loss), {}),
        (ValueError, (s, t, i, loss), {"dlogits": dl}),
        (ValueError, (s, t, i, loss), {"dloss": loss}),
        (TypeError, (s, t, i, loss), {"dloss": loss, "dlogits": dl.float()}),
        (ValueError, (s, t, i.t().contiguous().t(), loss), {}),
        (FsdpError, (s, t, i), {}),
        (FsdpError, (s, t, i, loss), {"temperature": 0.0}),
        (FsdpError, (s, t, i, loss), {"temperature": -1.0}),
        (FsdpError, (s, t, i, loss), {"temperature": math.inf}),
        (FsdpError, (s, t, i, loss), {"temperature": math.nan}),
        (FsdpError, (s, t, i, loss, loss), {}),
        (FsdpError, (s, t[:, :0], i[:, :0], loss), {}),
        (FsdpError, (s[:, :0], t, i, loss), {}),
        (ValueError, (s.cpu(), t, i, loss), {}),
    ]:
        with pytest.raises(error):
            distill_loss(*args, **kwargs)
    many, where = torch.zeros(4, 1025, device="cuda"), torch.zeros(4, 1025, dtype=torch.int32, device="cuda")
    with pytest.raises(FsdpError):
        distill_loss(s, many, where, loss)
    two = torch.zeros(5, 100, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(FsdpError):
        distill_loss_backward(loss, two[:4], t, i, loss, two[1:])
    torch.cuda.synchronize()
    assert bool((loss == 3).all()) and bool((dl == 3).all()) and not s.any()


def test_long_offsets():
    """Rows whose offsets pass 2^32 elements."""
    vocab, stride = 300, (1 << 31) + 4096
    raw = torch.empty(2 * stride + 4096, dtype=torch.bfloat16, device="cuda")
    s, d = raw.as_strided((3, vocab), (stride, 1), 0), raw.as_strided((3, vocab), (stride, 1), 512)
    logits, values, ids, _ = make(61, 3, vocab, 5, torch.bfloat16, torch.float32)
    s.copy_(logits)
    loss, want = torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    one, dw = torch.ones(3, device="cuda"), torch.empty(3, vocab, dtype=torch.bfloat16, device="cuda")
    distill_loss(s, values.cuda(), ids.cuda(), loss, dloss=one, dlogits=d)
    distill_loss(s.contiguous(), values.cuda(), ids.cuda(), want, dloss=one, dlogits=dw)
    assert torch.equal(loss, want) and torch.equal(d, dw)
