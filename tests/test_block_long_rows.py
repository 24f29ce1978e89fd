"""Matrix products of long rows, on the host.  A tile's rows lie within 2^31
bytes of its first, or the 32-bit offsets of its loads miss them: no call may
take a form that cannot reach its operands, and what no form reaches is refused."""

from __future__ import annotations

import re

import pytest

from test_block_host import OVERFLOW, Linear, LinearGrad, refused
from test_block_launch_forms import BF16, F16, F32, SIZE, at, linear, linear_grad
from test_block_launch_forms import launches  # noqa: F401

REACH = (1 << 31) - 16


def reached(kernel, dtype, rows_a, rows_b, row, columns_a=None, columns_b=None):
    """Whether a launch reaches operands laid in rows of `row` elements (a
    "columns" operand: rows of `columns` elements, of which a step takes 64 or 32)."""
    t = re.search(r"product_kernelI\w+?Lb([01])ELb([01])ELi(\d+)ELi(\d+)E", kernel)
    assert t, kernel
    size, deep = SIZE[dtype], 128 // SIZE[dtype]
    tile_a, tile_b = int(t.group(3)), int(t.group(4))
    for by_columns, tile, rows, columns in ((t.group(1), tile_a, rows_a, columns_a), (t.group(2), tile_b, rows_b, columns_b)):
        if by_columns == "1":
            end = (deep - 1) * columns * size + tile * size
        else:
            end = (min(tile, rows) - 1) * row * size + 128
        if end > REACH:
            return False
    return True


@pytest.mark.parametrize("m,n,k,dtype", [
    (2048, 2048, 5242880, BF16), (1024, 1024, 9437184, F16), (64, 64, 1 << 24, BF16), (40, 50, 20_000_000, BF16),
    (8, 8, 1 << 26, F16), (8, 16, 1 << 25, F32), (64, 128, 4_000_000, F32), (300, 300, 2_500_000, BF16), (6000, 300, 1 << 20, BF16),
])
def test_forward(launches, m, n, k, dtype):  # noqa: F811
    _, (names,), _ = launches([linear(m, n, k, dtype)])
    products = [p for p in names if "product_kernel" in p]
    assert products and all(reached(p, dtype, m, n, k) for p in products), names


@pytest.mark.parametrize("m,n,k,dtype", [
    (64, 64, 16_000_000, BF16),      # dx: the weight's rows by columns; dweight: x's
    (64, 8_000_000, 64, BF16),       # dx: long rows of dz
    (128, 4_200_000, 8, F16),
    (64, 4_000_000, 128, F32),
])
def test_gradient(launches, m, n, k, dtype):  # noqa: F811
    calls = [linear_grad(m, n, k, dtype, dx=at(5)), linear_grad(m, n, k, dtype, dweight=at(6)),
             linear_grad(m, n, k, dtype, 2, dx=at(5))]
    _, names, _ = launches(calls)
    for i, launched in enumerate(names):
        products = [p for p in launched if "product_kernel" in p]
        assert products
        for p in products:
            assert reached(p, dtype, n, k, m, n, k) if i == 1 else reached(p, dtype, m, k, n, None, k), p


@pytest.mark.parametrize("m,n,k,dtype", [(64, 64, 1 << 25, 0), (128, 128, 4_300_000, F32), (64, 128, 1 << 23, F32), (5, 64, 1 << 28, F16)])
def test_refusals(m, n, k, dtype):
    args = Linear(m=m, n=n, k=k, dtype=dtype, x=at(0), weight=at(1), out=at(2), x_stride=k, weight_stride=k, out_stride=n)
    for name in ("fsdp_block_linear", "fsdp_block_linear_workspace"):
        refused(name, args, OVERFLOW, "rows")


@pytest.mark.parametrize("m,n,k,out", [(64, 64, 1 << 25, "dx"), (64, 64, 1 << 25, "dweight"), (64, 1 << 25, 64, "dx"),
                                       (64, 1 << 25, 64, "dweight")])
def test_gradient_refusals(m, n, k, out):
    strides = dict(dout_stride=n, x_stride=k, weight_stride=k, dx_stride=k, dweight_stride=k)
    args = LinearGrad(m=m, n=n, k=k, dout=at(0), x=at(1), weight=at(2), **strides, **{out: at(5)})
    for name in ("fsdp_block_linear_grad", "fsdp_block_linear_grad_workspace"):
        refused(name, args, OVERFLOW, "rows")


def test_few_rows_of_any_length(launches):  # noqa: F811
    """Up to four rows of x: no tiles, 64-bit offsets."""
    _, names, _ = launches([linear(m, 64, 1 << 28, d) for m in (1, 4) for d in (BF16, F32)])
    assert all(len(n) == 1 and "row_kernel" in n[0] for n in names)


def test_nothing_to_sum(launches):  # noqa: F811
    """dweight without rows of x, dx without outputs: zeros, of any size."""
    _, names, _ = launches([linear_grad(0, 64, 1 << 25, BF16, dweight=at(6)), linear_grad(64, 0, 1 << 25, BF16, dx=at(5))])
    assert all(len(n) in (1, 2) and all("product_kernel" in p for p in n) for n in names)
