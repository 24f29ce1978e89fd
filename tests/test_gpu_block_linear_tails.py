"""The activations and their slopes far from 0, value by value: with k = 1 and a
factor of one, z is an input.

Bounds, relative to the value.  A 32-bit exponential of an argument that is held
in two parts is off by 4 units of 2^-24, a reciprocal by 2, each product or sum
by one: 12 for a sigmoid times z.  GELU's normal distribution adds the 9 of its
polynomial (5e-7) and the roundings of its argument: 32.  The argument of
GELU's tanh form, a rounded polynomial u of z, carries 4 units of itself into the
exponent: 12 + 8 |u|.  Slopes are sums of two terms, each so bounded.  Results
of an exponential below 2^-126 are 0."""

from __future__ import annotations

import math

import pytest
import torch

from block_util import DTYPES, E32, UNIT, close
from paper_2411_00284_amd import linear, linear_backward

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

FLUSH = 2.0 ** -126
SWEEP = {"silu": 100.0, "gelu": 14.0, "gelu_tanh": 100.0, "relu": 100.0}


def curve(z, act):
    """(value, slope, bound of the value, of the slope) in 64 bits, without
    cancellation in the tails."""
    if act == "relu":
        zero = torch.zeros_like(z)
        return z.clamp(min=0), (z > 0).double(), zero, zero
    if act == "gelu":
        cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        peak = z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        flush = (1 + z.abs()) * FLUSH
        return z * cdf, cdf + peak, 32 * E32 * (z * cdf).abs() + flush, 32 * E32 * (cdf + peak.abs()) + flush
    c = math.sqrt(2 / math.pi)
    u, du, grow = (z, torch.ones_like(z), 0.0) if act == "silu" else (2 * c * (z + 0.044715 * z ** 3),
                                                                     2 * c * (1 + 3 * 0.044715 * z * z), 8.0)
    q, r = torch.sigmoid(u), torch.sigmoid(-u)
    k = (12 + grow * u.abs().clamp(max=200) / 2) * E32
    side = z * q * r * du
    flush = (1 + z.abs() * (1 + du)) * FLUSH
    return z * q, q + side, k * (z * q).abs() + flush, k * (q + 2 * side.abs()) + flush


def sweep(act, dtype):
    top = SWEEP[act]
    z = torch.cat([torch.linspace(-top, top, 6001, dtype=torch.float64), torch.linspace(-6, 6, 2001, dtype=torch.float64),
                   torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e-4, -1e-4], dtype=torch.float64)])
    return z.to(dtype)


def rounded(bound, want, dtype):
    """32-bit bounds hold for fp32; in 16 bits the hardware's exponential of a
    rounded argument, 1 + |its argument| units more, disappears in the rounding."""
    return bound if dtype is torch.float32 else bound + 0.02 * UNIT[dtype] * want.abs()


@pytest.mark.parametrize("rows", [1, 3, 40])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("act", list(SWEEP))
def test_values(act, dtype, rows):
    dtype = DTYPES[dtype]
    z = sweep(act, dtype)
    out = torch.empty(rows, z.numel(), dtype=dtype, device="cuda")
    pre = torch.empty_like(out)
    linear(torch.ones(rows, 1, dtype=dtype, device="cuda"), z.cuda()[:, None], out, activation=act, pre=pre)
    assert all(torch.equal(p.cpu(), z) for p in pre)
    want, _, bound, _ = curve(z.double(), act)
    for row in out:
        close(row, want, rounded(bound, want, dtype), act)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("act", list(SWEEP))
def test_slopes(act, dtype):
    """dtimes is the value, dbias the slope, of a gradient and a factor of one;
    dx is the slope, as it enters the products, through a weight of one."""
    dtype = DTYPES[dtype]
    z = sweep(act, dtype)
    m = z.numel()
    one = torch.ones(1, m, dtype=dtype, device="cuda")
    got = {"dbias": torch.empty(m, dtype=dtype, device="cuda"), "dtimes": torch.empty_like(one)}
    linear_backward(one, one[:, :1], one.t(), activation=act, pre=z.cuda()[None], times=one, **got)
    value, slope, ev, es = curve(z.double(), act)
    close(got["dtimes"][0], value, rounded(ev, value, dtype), "value")
    close(got["dbias"], slope, rounded(es, slope, dtype), "slope")
    tall = torch.empty(m, 1, dtype=dtype, device="cuda")
    linear_backward(one.t().contiguous(), one.t().contiguous(), one[:, :1], activation=act, pre=z.cuda()[:, None], dx=tall)
    close(tall[:, 0], slope, rounded(es, slope, dtype), "dx")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", list(SWEEP))
def test_huge(act, dtype):
    """Finite z whose square or cube is not: the curves' limits."""
    dtype = DTYPES[dtype]
    z = torch.tensor([1e13, 1e19, 3e19, 1e25, 3e38], dtype=torch.float64).to(dtype)
    z = torch.cat([z, -z])
    up = (z > 0).to(dtype)
    one = torch.ones(1, z.numel(), dtype=dtype, device="cuda")
    out, slope, value = torch.empty_like(one), torch.empty(z.numel(), dtype=dtype, device="cuda"), torch.empty_like(one)
    linear(one[:, :1], z.cuda()[:, None], out, activation=act)
    linear_backward(one, one[:, :1], one.t(), activation=act, pre=z.cuda()[None], times=one, dbias=slope, dtimes=value)
    assert torch.equal(out[0].cpu(), z * up) and torch.equal(value[0].cpu(), z * up)
    assert torch.equal(slope.cpu(), up)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("act", list(SWEEP))
def test_not_numbers(act, dtype):
    """NaN stays NaN, infinity where the curve has it."""
    dtype = DTYPES[dtype]
    z = torch.tensor([math.nan, math.inf], dtype=dtype)
    one = torch.ones(1, 2, dtype=dtype, device="cuda")
    out, value, slope = torch.empty_like(one), torch.empty_like(one), torch.empty(2, dtype=dtype, device="cuda")
    linear(one[:, :1], z.cuda()[:, None], out, activation=act)
    linear_backward(one, one[:, :1], one.t(), activation=act, pre=z.cuda()[None], times=one, dbias=slope, dtimes=value)
    assert bool(out[0, 0].isnan()) and bool(value[0, 0].isnan()) and bool(slope[0].isnan())
    assert out[0, 1] == math.inf and value[0, 1] == math.inf
