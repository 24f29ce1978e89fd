"""The clipped policy loss with its KL term, against the formulas in 64 bits, at
the sizes, types, masks and values where it can go wrong."""

from __future__ import annotations

import math

import pytest
import torch

from block_util import DTYPES, E32, Mat, blank, close, normal
from paper_2411_00284_amd import FsdpError, policy_loss, policy_loss_backward
from step_shapes import POLICIES

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

# What an exponential of x, and a sum of them, are off by in units of themselves, times 1 + |x|.
FEW = 24 * E32


def reference(logits, actions, old, adv, ref, opt, dloss, lse=None):
    """loss, logp, lse, dlogits in 64 bits, and the bounds of their errors."""
    tau, low, high, kl = opt["temperature"], opt["clip_low"], opt["clip_high"], opt["kl_weight"]
    s = logits.double()
    top = s.max(1, keepdim=True).values
    log_sum = torch.exp((s - top) / tau).sum(1, keepdim=True).log()
    own = (top / tau + log_sum)[:, 0]
    logq = (s - top) / tau - log_sum if lse is None else s / tau - lse.double()[:, None]
    live, at = actions >= 0, actions.clamp(min=0).long()[:, None]
    logp = logq.gather(1, at)[:, 0]
    elogp = FEW + 2 * E32 * log_sum[:, 0].abs() if lse is None else 4 * E32 * torch.ones_like(own)
    r, a = torch.exp(logp - old.double()), adv.double()
    # the kernel has the options in 32 bits
    lo, hi = 1 - torch.tensor(low).double(), 1 + torch.tensor(high).double()
    gain, clipped = r * a, r.clamp(lo, hi) * a
    border = torch.minimum((r - lo).abs(), (r - hi).abs())
    assert bool((border > 2 * r * elogp).all()), "a ratio at a border: another seed"
    loss, slope = -torch.minimum(gain, clipped), torch.where(gain <= clipped, -gain, 0.0)
    moves = gain.abs()                                          # how far logp moves the slope
    if kl:
        d = ref.double() - logp
        weight = torch.tensor(kl).double()
        loss, slope, moves = loss + weight * (torch.expm1(d) - d), slope - weight * torch.expm1(d), moves + weight * d.exp()
    # r, the KL term and their products in 32 bits: an exponential of x is off by (2 + |x|) units (x rounded), a
    # product by one; 1 +- clip rounds too
    exact = 8 * E32 * (1 + (logp - old.double()).abs()) * gain.abs() + 4 * E32 * a.abs()
    if kl:
        exact = exact + 8 * E32 * (1 + d.abs()) * weight.abs() * (d.exp() + 1) * d.abs().clamp(max=1)
    eloss = 1.01 * (gain.abs() + (moves + slope.abs())) * elogp + exact
    zero = lambda v: torch.where(live, v, 0.0)  # noqa: E731
    c = (dloss.double() / tau)[:, None]
    q = torch.exp(logq)
    delta = torch.zeros_like(q).scatter_(1, at, 1.0)
    grad = torch.where((live & (dloss != 0))[:, None], c * slope[:, None] * (delta - q), 0.0)
    eg = c.abs() * (1.01 * moves * elogp + exact + 4 * E32 * slope.abs())[:, None] * (delta - q).abs()
    eg = eg + (c * slope[:, None]).abs() * (FEW * (1 + logq.abs().clamp(max=200)) + elogp[:, None]) * (q + delta * (1 - q).abs())
    return (zero(loss), zero(logp), zero(own), grad), (zero(eloss), zero(elogp), zero(4 * E32 * (1 + own.abs())), eg)


def make(seed, tokens, vocab, dtype, tau=1.0, scale=2.5):
    logits = normal(seed, tokens, vocab, dtype=dtype, scale=scale)
    g = torch.Generator().manual_seed(seed)
    few = torch.randint(0, vocab, (tokens, 32), generator=g)
    actions = few.gather(1, logits.gather(1, few).float().argmax(1, keepdim=True))
    now = (torch.log_softmax(logits.double() / tau, 1).gather(1, actions)[:, 0]).float()
    return (logits, actions[:, 0], now + normal(seed + 1, tokens, scale=0.2), normal(seed + 2, tokens),
            now + normal(seed + 3, tokens, scale=0.4), normal(seed + 4, tokens))


def options(kl=0.1, low=0.2, high=0.2, tau=1.0):
    return dict(kl_weight=kl, clip_low=low, clip_high=high, temperature=tau)


def run(case, dtype, opt, id_type=torch.int32, gap=0, shift=0):
    """All three calls, in one tensor's place too."""
    logits, actions, old, adv, ref, dloss = case
    tokens, vocab = logits.shape
    gl = Mat(logits, gap, shift)
    put = lambda v: Mat(v, 0, shift).t  # noqa: E731
    args = (actions.to(id_type).cuda(), put(old), put(adv))
    more = dict(opt, ref_logp=put(ref)) if opt["kl_weight"] else opt
    gd = put(dloss)
    outs = [blank(None, tokens, torch.float32, 0, shift) for _ in range(3)]
    dl, back = blank(tokens, vocab, dtype, gap, shift), blank(tokens, vocab, dtype, gap, shift)
    policy_loss(gl.t, *args, outs[0].t, outs[1].t, outs[2].t, dloss=gd, dlogits=dl.t, **more)
    want, bound = reference(logits, actions, old, adv, ref, opt, dloss)
    for v, w, e, name in zip((*outs, dl), want, bound, ("loss", "logp", "lse", "dlogits")):
        close(v.t, w, e, name)
        assert v.intact(), name
    alone = torch.empty(tokens, device="cuda")
    policy_loss(gl.t, *args, alone, **more)
    # A loss alone may go in another form, whose threads add other parts of the row.
    close(alone, want[0], bound[0], "loss alone")
    policy_loss_backward(gd, gl.t, *args, outs[2].t, back.t, **more)
    want, bound = reference(logits, actions, old, adv, ref, opt, dloss, outs[2].t.cpu())
    close(back.t, want[3], bound[3], "dlogits from lse")
    assert back.intact() and gl.intact()
    policy_loss_backward(gd, gl.t, *args, outs[2].t, gl.t, **more)
    assert torch.equal(gl.t, back.t) and gl.intact()
    gl = Mat(logits, gap, shift)
    policy_loss(gl.t, *args, dloss=gd, dlogits=gl.t, **more)
    assert torch.equal(gl.t, dl.t) and gl.intact()


@pytest.mark.parametrize("case", POLICIES, ids=str)
def test_forms(case):
    print("policy form", case, flush=True)
    dtype, tokens, vocab = case
    made = make(11, tokens, vocab, DTYPES[dtype])
    made[1][::5] = -1
    run(made, DTYPES[dtype], options())


# tokens, vocab, logits' type, actions' type, kl, clip, temperature, gap, shift
SHAPES = [
    (1, 1, "f32", torch.int32, 0.1, (0.2, 0.2), 1.0, 0, 0),
    (3, 2, "bf16", torch.int64, 0.0, (0.1, 0.3), 2.0, 0, 0),
    (4, 1000, "f16", torch.int32, 0.05, (0.2, 0.28), 0.5, 3, 1),
    (7, 8191, "bf16", torch.int64, 0.5, (0.0, 0.0), 1.0, 1, 1),
    (5, 8193, "f32", torch.int32, 0.0, (1.0, math.inf), 1.5, 1, 0),
    (3, 16384, "f16", torch.int32, -0.1, (0.2, 0.2), 1.0, 0, 0),
    (2, 32001, "f32", torch.int64, 0.1, (0.2, 0.2), 0.7, 0, 1),
    (9, 50257, "bf16", torch.int32, 0.1, (0.3, 0.2), 3.0, 7, 3),
    (2, 128256, "bf16", torch.int32, 0.1, (0.2, 0.2), 1.0, 0, 0),
    (1, 151936, "f32", torch.int32, 0.1, (0.2, 0.2), 1.0, 0, 0),
    (1, 300001, "bf16", torch.int64, 0.1, (0.2, 0.2), 1.0, 0, 1),
]


@pytest.mark.parametrize("case", SHAPES, ids=str)
def test_loss_and_gradient(case):
    tokens, vocab, dtype, id_type, kl, (low, high), tau, gap, shift = case
    print("policy", case, flush=True)
    dtype = DTYPES[dtype]
    run(make(21, tokens, vocab, dtype, tau), dtype, options(kl, low, high, tau), id_type, gap, shift)


@pytest.mark.parametrize("place", ["first", "last"])
@pytest.mark.parametrize("vocab", [37, 700, 2050, 20011])
def test_places_of_the_action(place, vocab):
    """At the row's ends, and in the elements after its whole units."""
    for dtype in (torch.bfloat16, torch.float32):
        made = list(make(31, 6, vocab, dtype))
        unit = 16 // made[0].element_size()
        made[1] = torch.tensor([0, 1, unit - 1, unit, 7, 3]) if place == "first" else vocab - 1 - torch.tensor([0, 1, unit - 1, unit, 7, 3])
        now = torch.log_softmax(made[0].double(), 1).gather(1, made[1][:, None])[:, 0].float()
        made[2], made[4] = now + normal(5, 6, scale=0.05), now + normal(6, 6, scale=0.3)
        run(made, dtype, options())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("vocab", [300, 20011])
@pytest.mark.parametrize("low", ["infinite", "lowest", "-1e4"])
def test_masked_logits(dtype, vocab, low):
    """Masks over runs of the vocabulary, over all but the action, and (of a
    finite value) over whole rows, whose distribution is uniform."""
    dtype = DTYPES[dtype]
    value = {"infinite": -math.inf, "lowest": torch.finfo(dtype).min, "-1e4": -1e4}[low]
    made = list(make(41, 5, vocab, dtype))
    logits, actions = made[0], made[1]
    keep = logits.gather(1, actions[:, None]).clone()
    logits[0, :vocab // 2] = value
    logits[1, vocab // 3:] = value
    logits[2] = value
    logits.scatter_(1, actions[:, None], keep)
    logits[3, ::2] = value
    logits[3, actions[3]] = keep[3, 0]
    if low != "infinite":
        logits[4] = value
    now = torch.log_softmax((logits.double() - logits.double().max(1, keepdim=True).values), 1).gather(1, actions[:, None])[:, 0].float()
    made[2], made[4] = now + normal(7, 5, scale=0.05), now + normal(8, 5, scale=0.3)
    rows = slice(0, 5) if low == "-1e4" else slice(0, 4)
    part = [v[rows] for v in made]
    run(part, dtype, options())
    # A row at a mask of the lowest value: its saved lse cannot give its gradient, the one pass does.
    outs = [torch.empty(5, device="cuda") for _ in range(3)]
    dl = torch.empty(5, vocab, dtype=dtype, device="cuda")
    args = [v.cuda() for v in made]
    policy_loss(args[0], args[1], args[2], args[3], *outs, ref_logp=args[4], dloss=args[5], dlogits=dl, **options())
    want, bound = reference(*made[:5], options(), made[5])
    for v, w, e, name in zip((*outs, dl), want, bound, ("loss", "logp", "lse", "dlogits")):
        close(v, w, e, name)


@pytest.mark.parametrize("vocab", [700, 20011])
def test_rows(vocab):
    """Masked tokens whatever their values, an action beyond the vocabulary, a
    zero weight over NaN, NaN and infinite logits, no advantage, an action that
    is ruled out, a row without a distribution."""
    tokens = 12
    for dtype in (torch.bfloat16, torch.float32):
        logits, actions, old, adv, ref, dloss = make(51, tokens, vocab, dtype)
        logits[0], old[0], adv[0], ref[0], actions[0] = math.nan, math.nan, math.inf, math.nan, -1
        actions[1] = -2147483648
        actions[2] = vocab
        logits[3], dloss[3] = math.nan, 0.0
        logits[4, 5] = math.nan
        logits[5, 6] = math.inf
        logits[6] = -math.inf
        adv[7], old[7] = 0.0, -math.inf
        adv[8] = 0.0
        logits[9, actions[9]], adv[9] = -math.inf, 2.0
        dloss[10] = 0.0
        old[11] = old[11] - 300.0                               # a ratio past any float: clipped where it gains
        adv[11] = 1.0
        put = [v.cuda() for v in (logits, actions, old, adv)]
        loss, logp, lse = (torch.full((tokens,), 7.0, device="cuda") for _ in range(3))
        dl = torch.full((tokens, vocab), 7.0, dtype=dtype, device="cuda")
        policy_loss(*put, loss, logp, lse, dloss=dloss.cuda(), dlogits=dl, **options(0.0))
        loss, logp, lse, dl = (v.cpu() for v in (loss, logp, lse, dl))
        for row in (0, 1):
            assert loss[row] == 0 and logp[row] == 0 and lse[row] == 0 and not dl[row].any()
        assert loss[2].isnan() and logp[2].isnan() and dl[2].isnan().all()
        assert not dl[3].any() and loss[3].isnan()
        for row in (4, 5, 6):
            assert loss[row].isnan() and dl[row].isnan().all()
        for row in (7, 8):
            assert loss[row] == 0 and not dl[row].any() and logp[row].isfinite()
        assert logp[9] == -math.inf and loss[9] == 0 and not dl[9].any()
        assert not dl[10].any() and loss[10].isfinite()
        assert abs(loss[11] + 1.2) < 1e-6 and not dl[11].any()
        back = torch.full((tokens, vocab), 7.0, dtype=dtype, device="cuda")
        policy_loss_backward(dloss.cuda(), *put, lse.cuda(), back, **options(0.0))
        assert torch.equal(back.cpu().isnan(), dl.isnan()) and not back[[0, 1, 3, 7, 8, 9, 10, 11]].any()


def test_small_temperatures():
    """Near one-hot distributions: 0 and 1 for probabilities, gradients of the
    size of 1 / temperature, nothing NaN."""
    tokens, vocab = 6, 300
    for dtype in (torch.bfloat16, torch.float32):
        logits, actions, _, adv, _, dloss = make(101, tokens, vocab, dtype)
        actions[:3] = logits[:3].float().argmax(1)
        logits[0, actions[0]] += 1
        for tau in (1e-3, 1e-20, 2.0 ** -126):
            logp = ((logits.double() - logits.double().max(1, keepdim=True).values) / tau)
            logp = (logp - torch.logsumexp(logp, 1, keepdim=True)).gather(1, actions[:, None])[:, 0]
            old = logp.clamp(min=-80).float()
            outs = [torch.empty(tokens, device="cuda") for _ in range(2)]
            dl = torch.empty(tokens, vocab, dtype=dtype, device="cuda")
            policy_loss(logits.cuda(), actions.cuda(), old.cuda(), adv.cuda(), *outs, temperature=tau, dloss=dloss.cuda(), dlogits=dl)
            assert not any(bool(v.isnan().any()) for v in (*outs, dl)), (dtype, tau)
            assert abs(float(outs[1][0])) < 1e-6                       # the action that stands out: probability 1


def test_past_the_clip():
    """Four rows on each side of both borders: the gradient is zero where a
    larger gain is clipped, and only there."""
    logits = normal(61, 8, 100)
    actions = torch.arange(8)
    now = torch.log_softmax(logits.double(), 1).gather(1, actions[:, None])[:, 0]
    ratio = torch.tensor([1.3, 1.3, 0.7, 0.7, 1.1, 1.1, 0.9, 0.9]).double()
    adv = torch.tensor([2.0, -2.0] * 4)
    old = (now - ratio.log()).float()
    loss, dl = torch.empty(8, device="cuda"), torch.empty(8, 100, device="cuda")
    policy_loss(logits.cuda(), actions.cuda(), old.cuda(), adv.cuda(), loss, dloss=torch.ones(8, device="cuda"), dlogits=dl)
    assert (dl != 0).any(1).tolist() == [False, True, True, False, True, True, True, True]
    want = torch.tensor([-2.4, 2.6, -1.4, 1.6, -2.2, 2.2, -1.8, 1.8])
    assert (loss.cpu() - want).abs().max() < 1e-5              # ratios are 32-bit values of a logarithm below 8: 2^-21


def test_differences():
    """The gradient against central differences of the loss in 64 bits of the
    kernel's own formulas, off by step^2 / 6 third derivatives (at most 20 times
    the slopes here) and by the loss's rounding over the step."""
    tokens, vocab, step = 6, 40, 1e-2
    logits, actions, old, adv, ref, _ = make(71, tokens, vocab, torch.float32, scale=1.0)
    args, opt = [v.cuda() for v in (actions, old, adv)], dict(options(0.3, 0.9, 3.0), ref_logp=ref.cuda())

    def total(x):
        loss = torch.empty(tokens, device="cuda")
        policy_loss(x.cuda(), *args, loss, **opt)
        return loss.double().sum().item()

    dl = torch.empty(tokens, vocab, device="cuda")
    policy_loss(logits.cuda(), *args, dloss=torch.ones(tokens, device="cuda"), dlogits=dl, **opt)
    for seed in range(4):
        d = normal(80 + seed, tokens, vocab)
        d = d / d.norm()
        slope = (dl.cpu().double() * d).sum().item()
        diff = (total(logits + step * d) - total(logits - step * d)) / (2 * step)
        size = float(adv.abs().sum()) + 1
        assert abs(diff - slope) <= 20 * size * step * step / 6 + 40 * E32 * size / step


def test_repeats_streams_and_far_rows():
    tokens, vocab = 300, 4099
    made = [v.cuda() for v in make(81, tokens, vocab, torch.bfloat16)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def run(logits, stream):
        loss, lse, dl = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda"), torch.empty_like(made[0])
        torch.cuda.synchronize()
        policy_loss(logits, *made[1:4], loss, None, lse, ref_logp=made[4], dloss=made[5], dlogits=dl, stream=stream, **options())
        torch.cuda.synchronize()
        return loss, lse, dl

    first = run(made[0], None)
    for stream in (None, side, side.cuda_stream):
        assert all(torch.equal(a, b) for a, b in zip(first, run(made[0], stream)))
    stride = (1 << 24) + 8                                     # 300 rows: offsets past 2^32 elements
    raw = torch.empty((tokens - 1) * stride + vocab, dtype=torch.bfloat16, device="cuda")
    far = raw.as_strided((tokens, vocab), (stride, 1))
    far.copy_(made[0])
    loss, dl = torch.empty(tokens, device="cuda"), far
    policy_loss(far, *made[1:4], loss, ref_logp=made[4], dloss=made[5], dlogits=dl, **options())
    assert torch.equal(loss, first[0]) and torch.equal(far, first[2])


def test_empty_and_refusals():
    logits, actions, old, adv, ref, dloss = (v.cuda() for v in make(91, 4, 50, torch.bfloat16))
    e = torch.empty(0, device="cuda")
    policy_loss(logits[:0], actions[:0], e, e, e.clone())
    loss, dl = torch.full((4,), 3.0, device="cuda"), torch.full_like(logits, 3)
    for error, args, more in [
        (TypeError, (logits, actions.float(), old, adv, loss), {}),
        (TypeError, (logits.double(), actions, old, adv, loss), {}),
        (TypeError, (logits, actions, old.half(), adv, loss), {}),
        (TypeError, (logits, actions, None, adv, loss), {}),
        (TypeError, (logits, actions, old, adv, loss.double()), {}),
        (TypeError, (logits, actions, old, adv, loss), {"kl_weight": "much"}),
        (TypeError, (logits, actions, old, adv), {"dloss": dloss, "dlogits": dl.float()}),
        (ValueError, (logits[0], actions, old, adv, loss), {}),
        (ValueError, (logits, actions[:3], old, adv, loss), {}),
        (ValueError, (logits, actions, old[:3], adv, loss), {}),
        (ValueError, (logits, actions, old, adv, loss), {"dlogits": dl}),
        (ValueError, (logits, actions, old, adv, loss), {"dloss": dloss, "dlogits": dl[:, :49]}),
        (ValueError, (logits, actions.cpu(), old, adv, loss), {}),
        (FsdpError, (logits, actions, old, adv, loss), {"kl_weight": 0.1}),
        (FsdpError, (logits, actions, old, adv, loss), {"kl_weight": math.inf, "ref_logp": ref}),
        (FsdpError, (logits, actions, old, adv, loss), {"clip_low": 1.5}),
        (FsdpError, (logits, actions, old, adv, loss), {"clip_low": -0.1}),
        (FsdpError, (logits, actions, old, adv, loss), {"clip_high": math.nan}),
        (FsdpError, (logits, actions, old, adv, loss), {"temperature": 0.0}),
        (FsdpError, (logits, actions, old, adv), {}),
        (FsdpError, (logits, actions, old, adv, old), {}),
        (FsdpError, (logits, actions, old, adv, loss, loss), {}),
        (FsdpError, (logits[:, :0], actions, old, adv, loss), {}),
    ]:
        with pytest.raises(error):
            policy_loss(*args, **more)
    for error, args in [
        (TypeError, (dloss, logits, actions, old, adv, loss, None)),
        (ValueError, (dloss[:3], logits, actions, old, adv, loss, dl)),
        (FsdpError, (dloss, logits, actions, old, adv, None, dl)),
    ]:
        with pytest.raises((error, ValueError) if error is TypeError else error):
            policy_loss_backward(*args)
    torch.cuda.synchronize()
    assert bool((loss == 3).all()) and bool((dl == 3).all())
