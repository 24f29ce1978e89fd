"""Formulas in 64 bits and error bounds for the tests of the step's operators
(beside block_util)."""

from __future__ import annotations

import torch

from block_util import E32, UNIT, Mat
from paper_2411_00284_amd import Checkpoint
from test_gpu_block_linear import act_bound, curve

GROUP = 32


def groups(cols):
    return -(-cols // GROUP)


def steps_of(most):
    """The scale, as a power of two, of groups whose largest magnitude is ``most`` (64 bits)."""
    _, e = torch.frexp(most)                                     # most = f 2^e, f in [1/2, 1)
    e = (e - 7).clamp(min=-126)                                  # most / 2^(e - 7) lies in [64, 128)
    e = torch.where(torch.round(torch.ldexp(most, -e)) > 127, e + 1, e)
    return torch.where(most == 0, -126, e)


def to_8bit(x):
    """Codes and scale bytes by the definition, on the CPU."""
    rows, cols = x.shape
    v = torch.zeros(rows, groups(cols) * GROUP, dtype=torch.float64)
    v[:, :cols] = x.double()
    v = v.view(rows, -1, GROUP)
    fine = torch.isfinite(v).all(2)
    v = torch.where(fine[:, :, None], v, 0.0)
    e = steps_of(v.abs().amax(2)) if cols else torch.zeros(rows, 0, dtype=torch.int64)
    codes = torch.round(torch.ldexp(v, -e[:, :, None])).reshape(rows, -1)[:, :cols]
    assert not codes.numel() or codes.abs().max() <= 127
    return codes.to(torch.int8).contiguous(), torch.where(fine, e + 127, 255).to(torch.uint8)


def stands_for(codes, scales):
    """In 64 bits."""
    scale = torch.where(scales == 255, float("nan"), torch.exp2(scales.double() - 127))
    return codes.double() * scale.repeat_interleave(GROUP, 1)[:, :codes.shape[1]]


class Bytes(Mat):
    """A Mat of int8 or uint8 (block_util counts elements of two or four bytes)."""

    def intact(self) -> bool:
        b = self.raw.clone()
        b.as_strided((self.rows, self.cols), (self.stride, 1), 64 + self.shift).view(torch.uint8).fill_(0xFF)
        return bool((b.view(torch.uint8) == 0xFF).all())


class Saved:
    """A Checkpoint in poisoned memory: ``of`` a matrix, or empty."""

    def __init__(self, x=None, rows=0, cols=0, gap=0, shift=0):
        if x is None:
            codes, scales = torch.zeros(rows, cols, dtype=torch.int8), torch.zeros(rows, groups(cols), dtype=torch.uint8)
        else:
            codes, scales = to_8bit(x)
        self.codes, self.scales = Bytes(codes, gap, shift), Bytes(scales, gap, shift)
        self.c = Checkpoint(self.codes.t, self.scales.t)

    def values(self):
        return stands_for(self.codes.t.cpu(), self.scales.t.cpu())

    def intact(self):
        return self.codes.intact() and self.scales.intact()


def gated(x, gw, uw, act):
    """g, u, out and the bounds of their errors before the last rounding."""
    k = x.shape[1]
    xd = x.double()

    def product(w):
        z = xd @ w.double().t()
        return z, (k + 8) * E32 * (xd.abs() @ w.double().abs().t()) + 2 * E32 * z.abs()

    (g, eg), (u, eu) = product(gw), product(uw)
    value = curve(g, act)[0]
    ev = 1.13 * eg + (act_bound(g) if act not in (None, "none") else 0.0)
    out = value * u
    return g, eg, u, eu, out, ev * u.abs() + value.abs() * eu + ev * eu + 2 * E32 * out.abs()


def near_saved(saved, z, e, what):
    """Whether 8 bits hold z, which the kernel knew to within e: the scale is that of a largest
    magnitude within e, and every value is off by half a step and e."""
    rows, cols = z.shape
    codes, scales = saved.codes.t.cpu(), saved.scales.t.cpu()
    pad = torch.zeros(rows, groups(cols) * GROUP, dtype=torch.float64)
    low, high = pad.clone(), pad.clone()
    low[:, :cols], high[:, :cols] = (z.abs() - e).clamp(min=0), z.abs() + e
    exponent = scales.int() - 127
    least, most = (steps_of(v.view(rows, -1, GROUP).amax(2)) for v in (low, high))
    assert bool(((exponent >= least) & (exponent <= most)).all()), f"{what}: scales"
    step = torch.exp2(exponent.double()).repeat_interleave(GROUP, 1)[:, :cols]
    off = (codes.double() * step - z).abs()
    assert bool((off <= step / 2 + e).all()), f"{what}: {(off - step / 2 - e).max().item()}"


def gated_gradient(dout, x, gw, uw, gate, up, act):
    """The gradients in 64 bits of what x, gate and up stand for, and bounds as
    test_gpu_block_linear.gradient has them."""
    m, n = dout.shape
    k = x.shape[1]
    unit = UNIT[dout.dtype]
    d, g, u = dout.double(), gate.double(), up.double()
    value, slope = curve(g, act)
    ea = act_bound(g) if act not in (None, "none") else torch.zeros_like(g)
    dg, du = d * u * slope, d * value
    eg, eu = (d * u).abs() * ea + 4 * E32 * dg.abs(), d.abs() * ea + 4 * E32 * du.abs()
    tiny = 2.0 ** -25 if dout.dtype is torch.float16 else 0.0
    eg, eu = eg + unit * (dg.abs() + eg) + tiny, eu + unit * (du.abs() + eu) + tiny
    want = {"out": value * u, "dx": dg @ gw.double() + du @ uw.double(), "dgate_weight": dg.t() @ x.double(),
            "dup_weight": du.t() @ x.double()}
    xa, ga, ua = x.double().abs(), gw.double().abs(), uw.double().abs()
    bound = {"out": ea * u.abs() + 2 * E32 * (value * u).abs(),
             "dx": eg @ ga + eu @ ua + (2 * n + 8) * E32 * (dg.abs() @ ga + du.abs() @ ua),
             "dgate_weight": eg.t() @ xa + (m + 8) * E32 * (dg.abs().t() @ xa),
             "dup_weight": eu.t() @ xa + (m + 8) * E32 * (du.abs().t() @ xa)}
    return want, bound
