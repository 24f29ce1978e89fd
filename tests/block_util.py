"""Helpers for the tests of the block operators: device matrices with row
strides inside poisoned memory, and error bounds.

Bounds.  An output that is rounded once to a type with unit roundoff u from a
value computed in 32 bits is off by at most u |v| + e, where e bounds the
32-bit error; a 32-bit sum of n terms, in any order, is off by at most
(n + c) 2^-24 times the sum of their magnitudes, with c for the roundings of
the terms themselves.
"""

from __future__ import annotations

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
# Half the distance of the smallest subnormals: what rounding may lose near 0.
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}
E32 = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
DEVICE = "cuda"
PAD = 64                     # poisoned elements before the first row and after the last


class Mat:
    """A [rows, cols] view with a row stride, in memory whose other bytes are
    0xFF (NaN patterns)."""

    def __init__(self, values: torch.Tensor, gap: int = 0, shift: int = 0):
        rows, cols = values.shape if values.dim() == 2 else (1, values.numel())
        self.stride = cols + gap
        self.raw = torch.empty(2 * PAD + shift + max(rows, 1) * self.stride, dtype=values.dtype, device=DEVICE)
        self.raw.view(torch.uint8).fill_(0xFF)
        self.t = self.raw.as_strided((rows, cols), (self.stride, 1), PAD + shift)
        self.t.copy_(values.reshape(rows, cols))
        if values.dim() == 1:
            self.t = self.t[0]
        self.rows, self.cols, self.shift = rows, cols, shift

    def intact(self) -> bool:
        """Whether nothing but the view has been written."""
        b = self.raw.clone()
        b.as_strided((self.rows, self.cols), (self.stride, 1), PAD + self.shift).view(torch.int16 if b.element_size() == 2
                                                                                     else torch.int32).fill_(-1)
        return bool((b.view(torch.uint8) == 0xFF).all())


def blank(rows, cols, dtype, gap=0, shift=0):
    """An output: NaN everywhere."""
    return Mat(torch.full((rows, cols) if rows is not None else (cols,), float("nan"), dtype=dtype), gap, shift)


def normal(seed, *shape, dtype=torch.float32, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * scale + shift).to(dtype)


def close(got, want, bound, what):
    """|got - want| <= u |want| + bound + the type's tiny, element by element;
    NaN and infinities in the same places."""
    got = got.detach().cpu()
    u, tiny = UNIT[got.dtype], TINY[got.dtype]
    g = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(g), torch.isnan(want)), f"{what}: NaN in other places"
    top = torch.finfo(got.dtype).max
    off = (g - want).abs()
    allowed = u * want.abs() + bound * (1 + 2 * u) + tiny
    inf_ok = (~fine) & (g == want)
    big_ok = fine & torch.isinf(g) & (want.abs() + allowed >= top) & (g.sign() == want.sign())
    bad = ~(torch.isnan(want) | inf_ok | big_ok | (off <= allowed))
    if bool(bad.any()):
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values off, first at {at}: got {g[at].item()!r}, "
                             f"want {want[at].item()!r}, allowed {(torch.as_tensor(allowed).expand_as(want))[at].item()!r}")
