"""What matrices in 8 bits stand for at the ends of the types they are read into."""

from __future__ import annotations

import pytest
import torch

from block_util import DTYPES, normal
from paper_2411_00284_amd import checkpoint_restore, checkpoint_save
from step_util import Saved, stands_for, to_8bit

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def restored(x, dtype):
    """x saved in its own type and read into another; and what it stands for, in 64 bits."""
    saved, out = Saved(rows=x.shape[0], cols=x.shape[1]), torch.empty(x.shape, dtype=dtype, device="cuda")
    checkpoint_save(x.cuda(), saved.c)
    checkpoint_restore(saved.c, out)
    want = stands_for(*to_8bit(x))
    assert torch.equal(saved.values(), want)
    return out.cpu(), want


def test_small_values_into_fp16():
    """A row's largest magnitude is 1.5 2^e.  From a step of 2^-24 on (e >= -18), and of groups
    saved from fp16 whatever their size, fp16 holds every code; of smaller ones the nearest fp16 value
    is read, off by half of 2^-24."""
    rows = list(range(-30, -9))
    x = (torch.rand(len(rows), 64, generator=torch.Generator().manual_seed(3), dtype=torch.float64) * 2 - 1) * 1.5
    x[:, ::32] = 1.5
    x = torch.ldexp(x, torch.tensor(rows)[:, None]).float()
    got, want = restored(x, torch.float16)
    assert torch.equal(got, want.half())
    exact = (got.double() == want).all(1)
    assert exact.tolist() == [e >= -18 for e in rows]
    assert bool(((got.double() - want).abs() <= 2.0 ** -25).all())
    got, want = restored(x.half(), torch.float16)
    assert torch.equal(got.double(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_largest_values(dtype):
    """A group whose largest magnitude rounds up to a power of two past the type's range is infinite there, of
    one below that finite."""
    dtype = DTYPES[dtype]
    top = 16.0 if dtype is torch.float16 else 128.0            # the range ends before 2^top
    x = normal(5, 2, 64, dtype=torch.float64)
    border = 2.0 ** top * (255 / 256)                           # 127.5 steps
    x[0, ::32], x[1, ::32] = border, border * (127 / 127.5)
    x = x.to(dtype)
    assert bool(torch.isfinite(x).all())
    got, want = restored(x, dtype)
    assert torch.equal(got, want.to(dtype)) and bool((want[0, ::32] == 2.0 ** top).all())
    assert bool(torch.isinf(got[0, ::32]).all()) and bool(torch.isfinite(got[1]).all())
