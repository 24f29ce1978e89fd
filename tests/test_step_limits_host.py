"""The sizes that the step's products take, and the rows of x that go without
tiles, as the header states them, on the host."""

from __future__ import annotations

import pytest

from step_calls import BF16, F32, gated, gated_grad, linear_grad
from test_step_host import GATED, OVERFLOW, SAVED, refused
from test_step_launch_forms import launches  # noqa: F401  (a fixture)


@pytest.mark.parametrize("name,limit", [("gated", 1 << 29), ("gated_grad", 1 << 29), ("linear_grad", 1 << 30)])
def test_sizes_stop_below_their_limit(name, limit):
    for size in ("m", "n"):
        refused(f"fsdp_step_{name}_workspace", name, dict(k=16) | {size: limit}, OVERFLOW, "a size is 2^")
        refused(f"fsdp_step_{name}_workspace", name, dict(k=16) | {size: limit - 1}, OVERFLOW, "too many tiles")
    refused(f"fsdp_step_{name}_workspace", name, dict(k=limit), OVERFLOW, "a size is 2^")


LONG = 1 << 25                                                   # 64 rows of it pass 2^31 bytes


@pytest.mark.parametrize("m", [1, 4, 5])
def test_rows_kept_in_8_bits_go_in_tiles(launches, m):  # noqa: F811
    """Up to four rows go without tiles, at any address and length, unless they are kept in 8 bits."""
    long = dict(k=LONG, x_stride=LONG, gate_weight_stride=LONG, up_weight_stride=LONG, gate_weight=1 << 40, up_weight=1 << 41, out=1 << 42,
                gate=1 << 43, up=1 << 44, gate_scales=1 << 45, up_scales=1 << 46, x=1 << 39)
    refused("fsdp_step_gated_workspace", "gated", {**GATED, **SAVED, **long, "m": m}, OVERFLOW, "rows")
    calls = [gated(m, 300, 701, d, kept) for d in (BF16, F32) for kept in (None, "type", "8bit")]
    for call, names in zip(calls, launches(calls)[0]):
        kept = dict((f, v) for f, _, v in call[1])["gate_scales"]
        laid = sum("pad_kernel" in n for n, _, _ in names)
        assert laid == (m > 4 or kept is not None), (m, names)
        assert any("gated_row_kernel" in n for n, _, _ in names) == (not laid)
