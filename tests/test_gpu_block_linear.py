"""The matrix product with its epilogue and its gradient, against the formulas
in 64 bits, at the sizes, types, strides and values where they can go wrong."""

from __future__ import annotations

import math

import pytest
import torch

from block_util import DTYPES, E32, Mat, UNIT, blank, close, normal
from paper_2411_00284_amd import FsdpError, linear, linear_backward

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def curve(z, act):
    """Value and slope of the activation, in 64 bits."""
    if act in (None, "none"):
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "silu":
        q = torch.sigmoid(z)
        return z * q, q + z * q * (1 - q)
    if act == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z ** 3))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)


# The activations' slopes are at most 1.13; their 32-bit values (an exponential or an erfc, a few products) are off by
# at most some 16 units of 2^-24 of (1 + z^2) |z| near the tails, where the exponent's own error grows with z^2.
def act_bound(z):
    return 16 * E32 * (1 + z * z) * (z.abs() + 1)


def forward(x, w, bias, act, times, residual):
    k = x.shape[1]
    xd, wd = x.double(), w.double()
    z, e = xd @ wd.t(), (k + 8) * E32 * (xd.abs() @ wd.abs().t())
    if bias is not None:
        z = z + bias.double()
    e = e + 2 * E32 * z.abs()
    out, eo = curve(z, act)[0], 1.13 * e
    if act not in (None, "none"):
        eo = eo + act_bound(z)
    if times is not None:
        out, eo = out * times.double(), eo * times.double().abs() + E32 * (out * times.double()).abs()
    if residual is not None:
        out = out + residual.double()
    return z, e, out, eo + 2 * E32 * out.abs()


# m, n, k, type, activation, bias, times, residual, pre, gap, shift
FORWARD = [
    (1, 1, 1, "bf16", None, False, False, False, False, 0, 0),
    (1, 4096, 256, "bf16", "silu", False, True, False, False, 0, 0),
    (1, 688, 4096, "f16", None, True, False, True, True, 0, 0),
    (2, 333, 1001, "bf16", "gelu", True, True, True, True, 3, 1),
    (5, 1000, 72, "f32", "gelu_tanh", True, False, False, True, 0, 0),
    (8, 24, 8192, "bf16", None, False, False, False, False, 8, 0),
    (15, 257, 688, "f16", "relu", False, False, True, False, 8, 8),
    (16, 512, 256, "bf16", "silu", False, False, False, True, 0, 0),
    (17, 129, 2050, "bf16", None, True, False, False, False, 2, 0),
    (33, 1024, 4100, "f16", "silu", True, True, True, True, 4, 4),
    (64, 256, 688, "bf16", "gelu", True, False, True, False, 0, 0),
    (77, 511, 123, "f32", "silu", True, True, True, True, 1, 1),
    (128, 128, 64, "bf16", None, False, False, False, False, 0, 0),
    (200, 300, 1027, "f16", "gelu", True, False, False, True, 0, 0),
    (255, 1040, 520, "bf16", "silu", False, True, False, True, 8, 0),
    (257, 769, 1000, "bf16", None, True, False, True, False, 0, 0),
    (513, 1025, 584, "f16", "gelu_tanh", True, True, True, True, 8, 8),
    (1025, 2047, 2056, "bf16", "relu", True, False, True, True, 0, 0),
    (300, 260, 700, "f32", None, False, False, True, False, 4, 4),
    (1000, 688, 256, "f32", "gelu", True, True, True, True, 0, 0),
    (2049, 4104, 72, "bf16", "silu", False, True, False, False, 0, 0),
    # The other tiles, and tiles whose sum over k is cut.
    (776, 1287, 72, "bf16", "silu", True, True, True, True, 1, 0),
    (136, 2056, 4104, "f16", "gelu", True, False, True, False, 8, 0),
    (8200, 136, 72, "bf16", "gelu_tanh", True, True, False, True, 0, 0),
    (2056, 136, 8200, "f16", None, True, False, True, False, 0, 8),
    (391, 8200, 72, "f16", "relu", False, True, True, True, 8, 0),
    (520, 14344, 72, "bf16", None, True, False, False, False, 0, 0),
    (8200, 136, 8200, "bf16", "silu", False, False, True, True, 0, 0),
    # A last round of tiles of its own: rows, columns.
    (4101, 4104, 520, "bf16", "silu", True, True, False, True, 8, 0),
    (1020, 18437, 520, "f16", None, True, False, True, False, 3, 0),
]


@pytest.mark.parametrize("case", FORWARD, ids=str)
def test_forward(case):
    m, n, k, dtype, act, has_bias, has_times, has_residual, has_pre, gap, shift = case
    dtype = DTYPES[dtype]
    print("linear", case, flush=True)
    x, w = normal(1, m, k, dtype=dtype), normal(2, n, k, dtype=dtype, scale=k ** -0.5)
    bias = normal(3, n, dtype=dtype) if has_bias else None
    times = normal(4, m, n, dtype=dtype) if has_times else None
    residual = normal(5, m, n, dtype=dtype) if has_residual else None
    put = lambda v: None if v is None else Mat(v, gap, shift).t  # noqa: E731
    out = blank(m, n, dtype, gap, shift)
    pre = blank(m, n, dtype, gap, shift) if has_pre else None
    linear(put(x), put(w), out.t, bias=None if bias is None else Mat(bias, 0, shift).t, activation=act, times=put(times),
           residual=put(residual), pre=pre.t if pre else None)
    z, ez, want, eo = forward(x, w, bias, act, times, residual)
    close(out.t, want, eo, "out")
    assert out.intact()
    if pre:
        close(pre.t, z, ez, "pre")
        assert pre.intact()


def test_in_place_and_slices():
    """out on times, on residual, and beside its inputs in one buffer."""
    m, n, k = 70, 328, 256
    x, w = normal(1, m, k, dtype=torch.bfloat16).cuda(), normal(2, n, k, dtype=torch.bfloat16, scale=0.05).cuda()
    f, r = normal(4, m, n, dtype=torch.bfloat16).cuda(), normal(5, m, n, dtype=torch.bfloat16).cuda()
    want = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    linear(x, w, want, activation="silu", times=f, residual=r)
    f2, r2 = f.clone(), r.clone()
    linear(x, w, f2, activation="silu", times=f2, residual=r)
    linear(x, w, r2, activation="silu", times=f, residual=r2)
    assert torch.equal(f2, want) and torch.equal(r2, want)
    both = torch.empty(m, k + 2 * n, dtype=torch.bfloat16, device="cuda")
    both[:, :k], both[:, k:k + n] = x, f
    linear(both[:, :k], w, both[:, k + n:], activation="silu", times=both[:, k:k + n], residual=r)
    assert torch.equal(both[:, k + n:], want) and torch.equal(both[:, :k], x) and torch.equal(both[:, k:k + n], f)


@pytest.mark.parametrize("m", [3, 300])
@pytest.mark.parametrize("k", [264, 1000])
def test_values(m, k):
    """A NaN or an infinity stays in its row or column; the type's lowest value
    as a masked bias; memory after a row of k is not read into the sum."""
    n = 260
    x, w, bias = normal(1, m, k, dtype=torch.bfloat16), normal(2, n, k, dtype=torch.bfloat16), normal(3, n, dtype=torch.bfloat16)
    x[1, 7], w[5, 3] = math.nan, math.inf
    bias[9] = torch.finfo(torch.bfloat16).min
    out = blank(m, n, torch.bfloat16, 16)
    linear(Mat(x, 8).t, Mat(w, 24).t, out.t, bias=bias.cuda(), activation="gelu")
    z, _, want, eo = forward(x, w, bias, "gelu", None, None)
    got = out.t.cpu()
    assert bool(got[1].isnan().all())
    rows = [i for i in range(m) if i != 1]
    cols = [j for j in range(n) if j not in (5, 9)]
    close(got[rows][:, cols], want[rows][:, cols], eo[rows][:, cols], "the others")
    up, down = z[rows, 5] == math.inf, z[rows, 5] == -math.inf
    assert bool((got[rows, 5][up] == math.inf).all()) and bool(got[rows, 5][down].isnan().all())
    assert bool((got[rows, 9] == 0).all())
    assert out.intact()


def test_relu_and_nan():
    x = torch.tensor([[math.nan], [1.0], [-1.0], [-0.0]], dtype=torch.float32, device="cuda")
    out = torch.empty(4, 1, device="cuda")
    linear(x, torch.ones(1, 1, device="cuda"), out, activation="relu")
    assert bool(out[0].isnan()) and out[1:].flatten().tolist() == [1.0, 0.0, 0.0]


def test_empty():
    for dtype in (torch.bfloat16, torch.float32):
        x, w = torch.empty(0, 64, dtype=dtype, device="cuda"), torch.ones(32, 64, dtype=dtype, device="cuda")
        linear(x, w, torch.empty(0, 32, dtype=dtype, device="cuda"), activation="silu")
        dw, db = torch.full_like(w, 7), torch.full((32,), 7, dtype=dtype, device="cuda")
        linear_backward(torch.empty(0, 32, dtype=dtype, device="cuda"), x, w, dx=torch.empty_like(x), dweight=dw, dbias=db)
        assert not dw.any() and not db.any()
        x, w = torch.ones(9, 64, dtype=dtype, device="cuda"), torch.empty(0, 64, dtype=dtype, device="cuda")
        linear(x, w, torch.empty(9, 0, dtype=dtype, device="cuda"))
        dx = torch.full_like(x, 7)
        linear_backward(torch.empty(9, 0, dtype=dtype, device="cuda"), x, w, dx=dx, dweight=torch.empty_like(w))
        assert not dx.any()


# ------------------------------------------------------------------ gradient


def gradient(dout, x, w, act, pre, times):
    """The gradients in 64 bits, and the bounds of the errors before the last
    rounding: 32-bit sums of factors of which dz is rounded to the type where
    it is not dout itself."""
    m, n = dout.shape
    k = x.shape[1]
    u = UNIT[x.dtype]
    d = dout.double()
    value, slope = curve(pre.double(), act) if pre is not None else (None, 1.0)
    dz = d * slope
    e = torch.zeros_like(d)
    if act not in (None, "none"):
        # the slopes' curvature is below 1.2
        e = d.abs() * act_bound(pre.double())
    out, bound = {}, {}
    if times is not None:
        t = times.double()
        out["dtimes"] = d * value
        bound["dtimes"] = d.abs() * act_bound(pre.double()) + 2 * E32 * (d * value).abs()
        dz, e = dz * t, e * t.abs()
    e = e + 4 * E32 * dz.abs()
    out["dbias"], bound["dbias"] = dz.sum(0), (e + (m + 4) * E32 * dz.abs()).sum(0)
    own = times is not None or act not in (None, "none")
    es = e + (u * (dz.abs() + e) if own else 0.0)      # of dz as it enters the products
    if own and x.dtype is torch.float16:
        es = es + 2.0 ** -25
    out["dx"], bound["dx"] = dz @ w.double(), es @ w.double().abs() + (n + 8) * E32 * (dz.abs() @ w.double().abs())
    out["dweight"] = dz.t() @ x.double()
    bound["dweight"] = es.t() @ x.double().abs() + (m + 8) * E32 * (dz.abs().t() @ x.double().abs())
    return out, bound


# m, n, k, type, activation, times, bias, gap, shift
GRADIENT = [
    (1, 1, 1, "bf16", None, False, True, 0, 0),
    (1, 688, 256, "bf16", "silu", True, True, 0, 0),
    (3, 129, 131, "f16", "gelu", True, True, 1, 1),
    (16, 64, 520, "f32", "gelu_tanh", False, True, 0, 0),
    (31, 1000, 72, "bf16", None, True, False, 8, 0),
    (64, 256, 688, "bf16", "relu", False, True, 0, 0),
    (130, 255, 257, "bf16", None, False, True, 0, 0),
    (256, 512, 256, "f16", "silu", True, True, 0, 0),
    (300, 1032, 328, "bf16", "gelu", False, True, 8, 8),
    (513, 264, 1024, "bf16", "silu", True, False, 0, 0),
    (777, 301, 503, "f32", "silu", True, True, 3, 1),
    (1025, 2056, 264, "bf16", "gelu_tanh", True, True, 0, 0),
    (2048, 136, 2048, "f16", None, False, False, 0, 0),
    (4100, 72, 96, "bf16", "silu", False, True, 0, 0),
    (1000, 688, 256, "f32", "gelu", False, True, 4, 4),
    # The other tiles, for dx and for dweight.
    (776, 72, 1287, "bf16", "silu", True, True, 1, 0),
    (8200, 72, 136, "f16", None, False, True, 0, 0),
    (391, 72, 8200, "bf16", "gelu", False, False, 8, 0),
    (520, 72, 14344, "f16", "relu", True, True, 0, 0),
    (72, 776, 1288, "f16", "gelu", False, True, 0, 8),
    (72, 8200, 136, "bf16", None, True, False, 0, 0),
    (72, 391, 8200, "f16", "silu", False, True, 0, 0),
    (72, 520, 14344, "bf16", None, False, True, 0, 0),
    # A last round of tiles of its own, for dx and for dweight.
    (4101, 520, 4104, "bf16", None, False, False, 8, 0),
    (520, 1020, 18437, "f16", "relu", False, True, 0, 0),
]


@pytest.mark.parametrize("case", GRADIENT, ids=str)
def test_gradient(case):
    m, n, k, dtype, act, has_times, has_bias, gap, shift = case
    dtype = DTYPES[dtype]
    print("linear gradient", case, flush=True)
    x, w = normal(1, m, k, dtype=dtype), normal(2, n, k, dtype=dtype, scale=n ** -0.5)
    dout, times = normal(3, m, n, dtype=dtype), normal(4, m, n, dtype=dtype) if has_times else None
    pre = normal(5, m, n, dtype=dtype, scale=1.5) if act or has_times else None
    put = lambda v: None if v is None else Mat(v, gap, shift).t  # noqa: E731
    got = {"dx": blank(m, k, dtype, gap, shift), "dweight": blank(n, k, dtype, gap, shift)}
    if has_bias:
        got["dbias"] = blank(None, n, dtype, 0, shift)
    if has_times:
        got["dtimes"] = blank(m, n, dtype, gap, shift)
    linear_backward(put(dout), put(x), put(w), activation=act, pre=put(pre), times=put(times), **{q: v.t for q, v in got.items()})
    want, bound = gradient(dout, x, w, act, pre, times)
    for q, v in got.items():
        close(v.t, want[q], bound[q], q)
        assert v.intact()


def test_gradient_forms():
    """Each output alone, dtimes on times: the same bits as all together."""
    m, n, k = 90, 264, 136
    x, w = normal(1, m, k, dtype=torch.bfloat16).cuda(), normal(2, n, k, dtype=torch.bfloat16).cuda()
    dout, times, pre = (normal(s, m, n, dtype=torch.bfloat16).cuda() for s in (3, 4, 5))
    shapes = {"dx": (m, k), "dweight": (n, k), "dbias": (n,), "dtimes": (m, n)}
    whole = {q: torch.empty(s, dtype=torch.bfloat16, device="cuda") for q, s in shapes.items()}
    linear_backward(dout, x, w, activation="silu", pre=pre, times=times, **whole)
    for q, s in shapes.items():
        alone = torch.empty(s, dtype=torch.bfloat16, device="cuda")
        linear_backward(dout, x, w, activation="silu", pre=pre, times=times, **{q: alone})
        assert torch.equal(alone, whole[q]), q
    again = times.clone()
    linear_backward(dout, x, w, activation="silu", pre=pre, times=again, dtimes=again)
    assert torch.equal(again, whole["dtimes"])
    linear_backward(dout, x, w)                                # nothing is wanted: nothing is done


def test_differences():
    """The gradient against central differences of the forward kernel, in
    float32: off by step^2 / 6 third derivatives and by rounding over the step."""
    m, n, k, step = 5, 12, 40, 1e-2
    v = {"x": normal(1, m, k), "weight": normal(2, n, k, scale=0.3), "bias": normal(3, n), "times": normal(4, m, n)}
    cot = normal(5, m, n)
    for act in (None, "silu", "gelu", "gelu_tanh"):
        def run(a):
            out, pre = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
            linear(a["x"].cuda(), a["weight"].cuda(), out, bias=a["bias"].cuda(), activation=act, times=a["times"].cuda(), pre=pre)
            return (out.cpu().double() * cot).sum().item(), pre
        pre = run(v)[1]
        got = {"x": torch.empty(m, k, device="cuda"), "weight": torch.empty(n, k, device="cuda"),
               "bias": torch.empty(n, device="cuda"), "times": torch.empty(m, n, device="cuda")}
        linear_backward(cot.cuda(), v["x"].cuda(), v["weight"].cuda(), activation=act, pre=pre, times=v["times"].cuda(),
                        dx=got["x"], dweight=got["weight"], dbias=got["bias"], dtimes=got["times"])
        size = math.sqrt(m * n)
        for i, q in enumerate(v):
            d = normal(30 + i, *v[q].shape)
            d = d / d.norm()
            slope = (got[q].cpu().double() * d).sum().item()
            diff = (run({**v, q: v[q] + step * d})[0] - run({**v, q: v[q] - step * d})[0]) / (2 * step)
            # third derivatives of the activations are below 2; a step moves z by at most |x| or |w| (about 7) times it
            assert abs(diff - slope) <= 2 * 7 ** 3 * size * step * step / 6 + 50 * E32 * size / step, (act, q)


def test_repeats_and_streams():
    """The same call gives the same bits, on another stream too."""
    m, n, k = 130, 4104, 1032
    x, w = normal(1, m, k, dtype=torch.bfloat16).cuda(), normal(2, n, k, dtype=torch.bfloat16).cuda()
    dout = normal(3, m, n, dtype=torch.bfloat16).cuda()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def run(stream):
        out, dx, dw, db = (torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in ((m, n), (m, k), (n, k), (n,)))
        torch.cuda.synchronize()
        linear(x, w, out, stream=stream)
        linear(x[:1], w, out[:1], stream=stream)
        linear_backward(dout, x, w, activation="relu", pre=out, dx=dx, dweight=dw, dbias=db, stream=stream)
        torch.cuda.synchronize()
        return out, dx, dw, db

    first = run(None)
    for stream in (None, side, side.cuda_stream):
        assert all(torch.equal(a, b) for a, b in zip(first, run(stream)))


def test_refusals():
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(32, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full((4, 32), 3, dtype=torch.bfloat16, device="cuda")
    cases = [
        (ValueError, (x, w[:, :63], out), {}),
        (ValueError, (x, w, out[:, :31]), {}),
        (ValueError, (x, w, out[:3]), {}),
        (ValueError, (x[0], w, out), {}),
        (ValueError, (x, w.cpu(), out), {}),
        (ValueError, (x, w, out.t().contiguous().t()), {}),
        (TypeError, (x, w.half(), out), {}),
        (TypeError, (x.double(), w.double(), out.double()), {}),
        (TypeError, (x, w, None), {}),
        (TypeError, (x, w, out), {"bias": out[0].float()}),
        (ValueError, (x, w, out), {"bias": out[:, 0]}),
        (ValueError, (x, w, out), {"activation": "swish"}),
        (ValueError, (x, w, out), {"times": out[:2]}),
        (FsdpError, (x, w, out), {"pre": out}),
        (FsdpError, (x, w, x[:, :32]), {}),
        (FsdpError, (x, w, out), {"residual": out, "times": out, "pre": out}),
        (FsdpError, (x[:, :0], w[:, :0], out), {}),
    ]
    for error, args, kwargs in cases:
        with pytest.raises(error):
            linear(*args, **kwargs)
    dx = torch.full_like(x, 3)
    for error, args, kwargs in [
        (FsdpError, (out, x, w), {"activation": "silu", "dx": dx}),
        (ValueError, (out, x, w), {"dtimes": torch.zeros_like(out)}),
        (FsdpError, (out, x, w), {"times": out, "dtimes": torch.zeros_like(out)}),
        (FsdpError, (out, x, w), {"dx": x}),
        (ValueError, (out, x, w), {"dweight": x}),
        (TypeError, (out, x, w), {"dx": dx.float()}),
    ]:
        with pytest.raises(error):
            linear_backward(*args, **kwargs)
    torch.cuda.synchronize()
    assert bool((out == 3).all()) and bool((dx == 3).all())


def test_long_offsets():
    """Rows whose offsets pass 2^32 elements, in every operand that is read or
    written."""
    m, n, k, stride = 3, 24, 40, (1 << 31) + 4096
    raw = torch.empty(2 * stride + 4096, dtype=torch.bfloat16, device="cuda")
    x = raw.as_strided((m, k), (stride, 1), 0)
    w, dw = raw.as_strided((3, k), (stride, 1), 64), raw.as_strided((3, k), (stride, 1), 128)
    out = raw.as_strided((m, 3), (stride, 1), 192)
    x.copy_(normal(1, m, k, dtype=torch.bfloat16))
    w.copy_(normal(2, 3, k, dtype=torch.bfloat16))
    want, dwant = torch.empty(m, 3, dtype=torch.bfloat16, device="cuda"), torch.empty(3, k, dtype=torch.bfloat16, device="cuda")
    linear(x, w, out)
    linear(x.contiguous(), w.contiguous(), want)
    assert torch.equal(out, want)
    linear_backward(out, x, w, dweight=dw)
    linear_backward(out.contiguous(), x.contiguous(), w.contiguous(), dweight=dwant)
    assert torch.equal(dw, dwant)
