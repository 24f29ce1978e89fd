"""The norms around a block and their gradient, against the formulas in 64
bits, at the sizes, types, strides and values where they can go wrong."""

from __future__ import annotations

import math

import pytest
import torch

from block_util import DTYPES, E32, Mat, UNIT, blank, close, normal
from paper_2411_00284_amd import FsdpError, block_norm, block_norm_backward

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

EPS = 1e-5


def rms(v, eps=EPS):
    r = (v.pow(2).mean(1, keepdim=True) + eps).rsqrt()
    return v * r, r


def rows_of(gate, tokens):
    g = gate.double().reshape(-1, gate.shape[-1])
    return g.repeat_interleave(tokens // g.shape[0], 0) if tokens else g[:0]


def forward(x, branch, post, gate, pre, rs, bs, eps=EPS):
    """(y, h, bound of y's 32-bit error, bound of h's)."""
    n = x.shape[1]
    y = rs * x.double()
    e = 4 * E32 * y.abs()
    if branch is not None:
        b = branch.double()
        if post is not None:
            b = rms(b, eps)[0] * post.double()
        if gate is not None:
            b = b * rows_of(gate, x.shape[0])
        y = y + bs * b
        # a row's mean square is a sum of n terms of one sign, its root halves the relative error
        e = e + (n / 2 + 12) * E32 * (bs * b).abs()
    e = e + E32 * y.abs()
    h = eh = None
    if pre is not None:
        u, r = rms(y, eps)
        h = u * pre.double()
        # an error of y scales through the norm: directly, and through the row's root mean square
        rel = (e * y.abs()).mean(1, keepdim=True) * r * r
        eh = (r * e + u.abs() * (rel + (n / 2 + 12) * E32)) * pre.double().abs()
    return y, h, e, eh


def gate_of(seed, rows, hidden, dtype):
    if rows is None:
        return None
    return normal(seed, hidden, dtype=dtype) if rows == 0 else normal(seed, rows, hidden, dtype=dtype)


# tokens, hidden, block type, stream type, weights' type, gate rows (None: no gate, 0: a vector), post norm, strides' gap, shift
SHAPES = [
    (1, 1, "bf16", "bf16", "bf16", 0, True, 0, 0),
    (1, 4096, "bf16", "bf16", "bf16", 1, True, 0, 0),
    (3, 7, "f16", "f32", "f32", 3, True, 3, 1),
    (5, 64, "f32", "f32", "f32", 5, True, 0, 0),
    (17, 511, "bf16", "f32", "bf16", None, True, 5, 3),
    (4, 512, "f16", "f16", "f16", 2, False, 0, 0),
    (9, 513, "bf16", "bf16", "f32", 3, True, 0, 1),
    (33, 771, "f16", "f16", "f16", 0, True, 1, 1),
    (300, 1024, "bf16", "bf16", "bf16", 2, True, 8, 8),
    (6, 1025, "f32", "f32", "f32", 0, False, 7, 1),
    (7, 2048, "bf16", "f32", "f32", 7, True, 0, 0),
    (11, 2049, "f16", "f32", "f16", None, False, 1, 1),
    (700, 3001, "bf16", "bf16", "bf16", 7, True, 0, 0),
    (12, 4097, "bf16", "f32", "bf16", 4, True, 2, 5),
    (1100, 8192, "bf16", "f32", "f32", 2, True, 0, 0),
    (5, 8193, "f32", "f32", "f32", 5, True, 0, 1),
    (600, 16384, "bf16", "bf16", "bf16", 1, True, 0, 0),
    (3, 16383, "f16", "f32", "f16", 3, True, 1, 1),
]


@pytest.mark.parametrize("case", SHAPES, ids=str)
def test_forward(case):
    tokens, hidden, block, stream, weights, rows, post, gap, shift = case
    block, stream, weights = DTYPES[block], DTYPES[stream], DTYPES[weights]
    print("norm", case, flush=True)
    x, b = normal(1, tokens, hidden, dtype=stream, scale=3), normal(2, tokens, hidden, dtype=block)
    pre, pw = normal(3, hidden, dtype=weights, shift=1), normal(4, hidden, dtype=weights, shift=1) if post else None
    gate = gate_of(5, rows, hidden, block)
    dev = lambda v: None if v is None else Mat(v, shift=shift).t  # noqa: E731
    gx, gb = Mat(x, gap, shift), Mat(b, gap, shift)
    y, h = blank(tokens, hidden, stream, gap, shift), blank(tokens, hidden, block, gap, shift)
    block_norm(gx.t, branch=gb.t, pre_weight=dev(pre), post_weight=dev(pw), gate=None if gate is None else gate.cuda(),
               y=y.t, h=h.t, residual_scale=0.75, branch_scale=1.25, eps=EPS)
    wy, wh, ey, eh = forward(x, b, pw, gate, pre, 0.75, 1.25)
    close(y.t, wy, ey, "y")
    close(h.t, wh, eh, "h")
    assert y.intact() and h.intact() and gx.intact() and gb.intact()


def test_forms():
    """Only h, only y, no branch, and in place: the same values."""
    x, b, w = normal(1, 37, 900, dtype=torch.bfloat16), normal(2, 37, 900, dtype=torch.bfloat16), normal(3, 900, dtype=torch.bfloat16)
    x, b, w = x.cuda(), b.cuda(), w.cuda()
    y, h = torch.empty_like(x), torch.empty_like(x)
    block_norm(x, branch=b, pre_weight=w, post_weight=w, y=y, h=h)
    y2, h2 = torch.empty_like(x), torch.empty_like(x)
    block_norm(x, branch=b, post_weight=w, y=y2)
    block_norm(x, branch=b, pre_weight=w, post_weight=w, h=h2)
    assert torch.equal(y, y2) and torch.equal(h, h2)
    x2, b2 = x.clone(), b.clone()
    block_norm(x2, branch=b2, pre_weight=w, post_weight=w, y=x2, h=b2)
    assert torch.equal(y, x2) and torch.equal(h, b2)
    block_norm(x, pre_weight=w, h=h2, residual_scale=2.0)
    _, want, _, eh = forward(x.cpu(), None, None, None, w.cpu(), 2.0, 1.0)
    close(h2, want, eh, "h without a branch")
    one = torch.empty(1, 900, dtype=torch.bfloat16, device="cuda")
    block_norm(x[5:6], branch=b[5:6], pre_weight=w, post_weight=w, h=one)
    assert torch.equal(one, h[5:6])                            # a row does not depend on the others


def test_values():
    """Rows of zeros, of the type's lowest value, infinities and NaN; the other
    rows keep theirs."""
    x, b = normal(1, 6, 1000), normal(2, 6, 1000)
    low = torch.finfo(torch.float32).min
    x[0], b[0] = 0.0, 0.0
    b[1] = 0.0
    b[2, 5] = math.nan
    b[3, 7] = math.inf
    x[4] = low
    w = normal(3, 1000)
    y, h = torch.empty(6, 1000, device="cuda"), torch.empty(6, 1000, device="cuda")
    block_norm(x.cuda(), branch=b.cuda(), pre_weight=w.cuda(), post_weight=w.cuda(), y=y, h=h, eps=EPS)
    wy, wh, ey, eh = forward(x, b, w, None, w, 1.0, 1.0)
    fine = [0, 1, 5]
    close(y[fine], wy[fine], ey[fine], "y")
    close(h[fine], wh[fine], eh[fine], "h")
    assert bool((h[0] == 0).all())                             # 0 / sqrt(eps), not 0 / 0
    assert bool(y[2].isnan().all()) and bool(h[2].isnan().all())
    assert bool(y[3, 7].isnan())                               # inf / inf
    assert torch.equal(y[4].cpu(), wy[4].float())
    assert bool((h[4] == 0).all())                             # the mean square passes fp32: v / inf


def test_no_tokens():
    for dtype in (torch.bfloat16, torch.float32):
        e, w = torch.empty(0, 64, dtype=dtype, device="cuda"), torch.ones(64, dtype=dtype, device="cuda")
        block_norm(e, branch=e, pre_weight=w, post_weight=w, y=torch.empty_like(e), h=torch.empty_like(e))
        g = torch.ones(5, 64, dtype=dtype, device="cuda")
        dw, dp, dg = torch.full_like(w, 7), torch.full_like(w, 7), torch.full_like(g, 7)
        block_norm_backward(e, dy=e, dh=e, branch=e, pre_weight=w, post_weight=w, gate=g, dx=torch.empty_like(e),
                            dbranch=torch.empty_like(e), dpre_weight=dw, dpost_weight=dp, dgate=dg)
        assert not dw.any() and not dp.any() and not dg.any()


# ------------------------------------------------------------------ gradient


def gradient(y, dy, dh, branch, post, gate, pre, rs, bs, eps=EPS):
    """The gradients in 64 bits and the bounds of their 32-bit errors."""
    t, n = y.shape
    c = (n + 30) * E32
    out, bound = {}, {}
    g = dy.double() if dy is not None else torch.zeros(t, n, dtype=torch.float64)
    e = E32 * g.abs()
    if dh is not None:
        u, r = rms(y.double(), eps)
        du = dh.double() * pre.double()
        m, mabs = (du * u).mean(1, keepdim=True), (du * u).abs().mean(1, keepdim=True)
        g = g + r * (du - u * m)
        e = e + c * r * (du.abs() + u.abs() * (mabs + m.abs())) + 2 * E32 * g.abs()
        out["dpre_weight"] = (dh.double() * u).sum(0)
        bound["dpre_weight"] = (t + n / 2 + 30) * E32 * (dh.double() * u).abs().sum(0)
    out["dx"], bound["dx"] = rs * g, abs(rs) * e + 2 * E32 * (rs * g).abs()
    if branch is not None:
        b, rb = branch.double(), torch.ones(t, 1, dtype=torch.float64)
        ub = b
        if post is not None:
            ub, rb = rms(b, eps)
        normed = ub * post.double() if post is not None else ub
        dn, en = bs * g, abs(bs) * e + 4 * E32 * (bs * g).abs()
        rel = (n / 2 + 12) * E32
        if gate is not None:
            q = gate.reshape(-1, n).shape[0]
            out["dgate"] = (dn * normed).reshape(q, t // q, n).sum(1)
            bound["dgate"] = (en * normed.abs() + (rel + t * E32) * (dn * normed).abs()).reshape(q, t // q, n).sum(1)
            k = rows_of(gate, t)
            dn, en = dn * k, en * k.abs() + 2 * E32 * (dn * k).abs()
        if post is not None:
            out["dpost_weight"] = (dn * ub).sum(0)
            bound["dpost_weight"] = (en * ub.abs() + (rel + t * E32) * (dn * ub).abs()).sum(0)
            dn, en = dn * post.double(), en * post.double().abs() + 2 * E32 * (dn * post.double()).abs()
            m, mabs = (dn * ub).mean(1, keepdim=True), (dn * ub).abs().mean(1, keepdim=True)
            want = rb * (dn - ub * m)
            en = rb * (en + ub.abs() * (en * ub.abs()).mean(1, keepdim=True)) + c * rb * (dn.abs() + 2 * ub.abs() * mabs)
            dn = want
        out["dbranch"], bound["dbranch"] = dn, en
    return out, bound


def run_gradient(y, dy, dh, branch, post, gate, pre, rs=1.0, bs=1.0, gap=0, shift=0, stream=None):
    t, n = y.shape
    put = lambda v: None if v is None else Mat(v, gap if v.dim() == 2 else 0, shift).t  # noqa: E731
    got = {"dx": blank(t, n, y.dtype, gap, shift)}
    if branch is not None:
        got["dbranch"] = blank(t, n, branch.dtype, gap, shift)
    if dh is not None:
        got["dpre_weight"] = blank(None, n, pre.dtype, 0, shift)
    if post is not None:
        got["dpost_weight"] = blank(None, n, post.dtype, 0, shift)
    if gate is not None:
        got["dgate"] = Mat(torch.full_like(gate, math.nan), 0, shift)
    block_norm_backward(put(y), dy=put(dy), dh=put(dh), branch=put(branch), pre_weight=put(pre), post_weight=put(post),
                        gate=None if gate is None else gate.cuda(), residual_scale=rs, branch_scale=bs, eps=EPS, stream=stream,
                        **{k: v.t for k, v in got.items()})
    assert all(v.intact() for v in got.values())
    return {k: v.t for k, v in got.items()}


@pytest.mark.parametrize("case", SHAPES, ids=str)
def test_gradient(case):
    tokens, hidden, block, stream, weights, rows, post, gap, shift = case
    block, stream, weights = DTYPES[block], DTYPES[stream], DTYPES[weights]
    print("norm gradient", case, flush=True)
    y, b = normal(1, tokens, hidden, dtype=stream, scale=3), normal(2, tokens, hidden, dtype=block)
    dy, dh = normal(6, tokens, hidden, dtype=stream), normal(7, tokens, hidden, dtype=block)
    pre, pw = normal(3, hidden, dtype=weights, shift=1), normal(4, hidden, dtype=weights, shift=1) if post else None
    gate = gate_of(5, rows, hidden, block)
    got = run_gradient(y, dy, dh, b, pw, gate, pre, 0.75, 1.25, gap, shift)
    want, bound = gradient(y, dy, dh, b, pw, gate, pre, 0.75, 1.25)
    for k in want:
        close(got[k].reshape(want[k].shape), want[k], bound[k], k)


@pytest.mark.parametrize("tokens,rows", [(4096, 4096), (4096, 2048), (4100, 4), (4096, 3), (6000, 1000), (1, 1), (2000, None)])
def test_gate_groups(tokens, rows):
    """Every way of dealing a gate's rows to units of tokens."""
    if rows is not None and tokens % rows:
        tokens -= tokens % rows
    n = 40
    y, b = normal(1, tokens, n, dtype=torch.bfloat16), normal(2, tokens, n, dtype=torch.bfloat16)
    dy, dh = normal(6, tokens, n, dtype=torch.bfloat16), normal(7, tokens, n, dtype=torch.bfloat16)
    w, gate = normal(3, n, dtype=torch.bfloat16), gate_of(5, rows, n, torch.bfloat16)
    got = run_gradient(y, dy, dh, b, w, gate, w)
    want, bound = gradient(y, dy, dh, b, w, gate, w, 1.0, 1.0)
    for k in want:
        close(got[k].reshape(want[k].shape), want[k], bound[k], k)


def test_gradient_forms():
    """Without dy, without dh, without the branch; in place; some outputs only."""
    t, n = 50, 1300
    y, b = normal(1, t, n, dtype=torch.bfloat16), normal(2, t, n, dtype=torch.bfloat16)
    dy, dh = normal(6, t, n, dtype=torch.bfloat16), normal(7, t, n, dtype=torch.bfloat16)
    w = normal(3, n, dtype=torch.bfloat16)
    for args in ((y, None, dh, b, w, None, w), (y, dy, None, b, w, None, None), (y, dy, dh, None, None, None, w),
                 (y, dy, None, b, None, w, None)):
        got = run_gradient(*args)
        want, bound = gradient(*args, 1.0, 1.0)
        for k in want:
            close(got[k].reshape(want[k].shape), want[k], bound[k], k)
    whole = run_gradient(y, dy, dh, b, w, w, w)
    gy, gdy, gdh, gb, gw = y.cuda(), dy.cuda(), dh.cuda(), b.cuda(), w.cuda()
    dw = torch.empty_like(gw)
    block_norm_backward(gy, dy=gdy, dh=gdh, branch=gb, pre_weight=gw, post_weight=gw, gate=gw, dx=gdy, dbranch=gb, dpost_weight=dw)
    assert torch.equal(gdy, whole["dx"]) and torch.equal(gb, whole["dbranch"]) and torch.equal(dw, whole["dpost_weight"])
    gdy, gb, only = dy.cuda(), b.cuda(), torch.empty_like(gw)
    block_norm_backward(gy, dy=gdy, dh=gdh, branch=gb, pre_weight=gw, post_weight=gw, gate=gw, dbranch=gdh, dgate=only)
    assert torch.equal(gdh, whole["dbranch"]) and torch.equal(only, whole["dgate"])


def test_differences():
    """The gradient against central differences of the forward kernel, in
    float32.  With step s, a difference is off by s^2/6 times a third derivative
    (of the order of the loss) and by the forward's rounding over s."""
    t, n, step = 4, 96, 1e-2
    x, b, w, p, g = normal(1, t, n), normal(2, t, n), normal(3, n, shift=1), normal(4, n, shift=1), normal(5, 2, n)
    cy, ch = normal(6, t, n), normal(7, t, n)
    names = ["x", "branch", "post", "gate", "pre"]

    def loss(v):
        y, h = torch.empty(t, n, device="cuda"), torch.empty(t, n, device="cuda")
        block_norm(v["x"].cuda(), branch=v["branch"].cuda(), pre_weight=v["pre"].cuda(), post_weight=v["post"].cuda(),
                   gate=v["gate"].cuda(), y=y, h=h, residual_scale=0.5, branch_scale=2.0, eps=EPS)
        return ((y.cpu().double() * cy).sum() + (h.cpu().double() * ch).sum()).item(), y.cpu()

    v = dict(zip(names, (x, b, p, g, w)))
    y = loss(v)[1]
    got = run_gradient(y, cy, ch, b, p, g, w, 0.5, 2.0)
    pairs = {"x": "dx", "branch": "dbranch", "post": "dpost_weight", "gate": "dgate", "pre": "dpre_weight"}
    size = math.sqrt(t * n)
    for i, k in enumerate(names):
        d = normal(20 + i, *v[k].shape)
        d = d / d.norm()
        up, down = loss({**v, k: v[k] + step * d})[0], loss({**v, k: v[k] - step * d})[0]
        slope = (got[pairs[k]].cpu().double().reshape(d.shape) * d).sum().item()
        # cotangents and values are of order 1: a directional third derivative is at most some tens
        # times the norm of the cotangents; the rounding of 2 t n terms adds up to E32 * their norm
        assert abs((up - down) / (2 * step) - slope) <= 30 * size * step * step / 6 + 50 * E32 * size / step, k


def test_repeats_and_streams():
    """The same call gives the same bits, on another stream too."""
    t, n = 2000, 1024
    y, b = normal(1, t, n, dtype=torch.bfloat16), normal(2, t, n, dtype=torch.bfloat16)
    dy, dh = normal(6, t, n, dtype=torch.bfloat16), normal(7, t, n, dtype=torch.bfloat16)
    w = normal(3, n, dtype=torch.bfloat16)
    first = run_gradient(y, dy, dh, b, w, w, w)
    side = torch.cuda.Stream()
    for stream in (None, side, side.cuda_stream):
        with torch.cuda.stream(side):
            again = run_gradient(y, dy, dh, b, w, w, w, stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(first[k], again[k]) for k in first)


def test_refusals():
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    y, h = torch.full_like(x, 3), torch.full_like(x, 3)
    bad = [
        (ValueError, dict(pre_weight=w)),
        (ValueError, dict(h=h)),
        (TypeError, dict(y=y.float())),
        (TypeError, dict(pre_weight=w.half(), h=h)),
        (ValueError, dict(pre_weight=w[:32], h=h)),
        (ValueError, dict(branch=x[:2], y=y)),
        (ValueError, dict(branch=x, gate=w[:32], y=y)),
        (FsdpError, dict(branch=x, gate=torch.zeros(3, 64, dtype=torch.bfloat16, device="cuda"), y=y)),
        (FsdpError, dict(gate=w, y=y)),
        (FsdpError, dict(pre_weight=w, h=h, eps=-1.0)),
        (FsdpError, dict(pre_weight=w, h=h, residual_scale=math.nan)),
        (TypeError, dict(pre_weight=w, h=h, eps="small")),
        (ValueError, dict(y=y.t().contiguous().t())),
        (ValueError, dict(y=y.cpu())),
        (TypeError, dict(y=[1])),
        (FsdpError, dict(pre_weight=w, y=y, h=y)),
        (FsdpError, dict(pre_weight=w, h=x)),
        (TypeError, dict(y=y, stream="s")),
    ]
    for error, kwargs in bad:
        with pytest.raises(error):
            block_norm(x, **kwargs)
    wide = torch.zeros(1, 16385, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(FsdpError):
        block_norm(wide, y=torch.empty_like(wide))
    with pytest.raises(ValueError):
        block_norm(torch.zeros(64, dtype=torch.bfloat16, device="cuda"), y=y)
    for error, kwargs in [(ValueError, dict(dh=x)), (ValueError, dict(dbranch=y)), (FsdpError, dict(dpost_weight=w)),
                          (ValueError, dict(dgate=w)), (FsdpError, dict(dy=y, dx=x)), (TypeError, dict(dy=y.float()))]:
        with pytest.raises(error):
            block_norm_backward(x, **kwargs)
    torch.cuda.synchronize()
    assert bool((y == 3).all()) and bool((h == 3).all()) and not x.any()


def test_long_offsets():
    """Rows whose offsets pass 2^32 elements."""
    n, stride = 96, (1 << 31) + 4096
    raw = torch.empty(2 * stride + n, dtype=torch.bfloat16, device="cuda")
    x = raw.as_strided((3, n), (stride, 1))
    x.copy_(normal(1, 3, n, dtype=torch.bfloat16))
    w = normal(3, n, dtype=torch.bfloat16).cuda()
    h, want = torch.empty(3, n, dtype=torch.bfloat16, device="cuda"), torch.empty(3, n, dtype=torch.bfloat16, device="cuda")
    block_norm(x, pre_weight=w, h=h)
    block_norm(x.contiguous(), pre_weight=w, h=want)
    assert torch.equal(h, want)
