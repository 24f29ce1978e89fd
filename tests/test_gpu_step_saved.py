"""Matrices in 8 bits and back, against the definition, bit for bit."""

from __future__ import annotations

import math

import pytest
import torch

from block_util import DTYPES, Mat, blank, normal
from paper_2411_00284_amd import Checkpoint, FsdpError, checkpoint_restore, checkpoint_save
from step_util import Bytes, Saved, groups, stands_for, to_8bit

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}


def check(x, gap=0, shift=0):
    rows, cols = x.shape
    codes, scales = to_8bit(x)
    got, out = Saved(rows=rows, cols=cols, gap=gap, shift=shift), blank(rows, cols, x.dtype, gap, shift)
    checkpoint_save(Mat(x, gap, shift).t, got.c)
    checkpoint_restore(got.c, out.t)
    assert torch.equal(got.scales.t.cpu(), scales)
    assert torch.equal(got.codes.t.cpu(), codes)
    want = stands_for(codes, scales).to(x.dtype)
    back = out.t.cpu()
    assert torch.equal(back.isnan(), want.isnan()) and torch.equal(back.nan_to_num(), want.nan_to_num())
    assert got.intact() and out.intact()
    return codes, scales


SHAPES = [(1, 1, 0, 0), (1, 31, 0, 0), (1, 32, 0, 0), (2, 33, 1, 1), (3, 7, 3, 0), (5, 64, 0, 0), (7, 500, 8, 8), (4, 512, 0, 0),
          (9, 513, 0, 3), (130, 1000, 0, 0), (1, 28672, 0, 0), (1021, 771, 5, 1), (300, 4096, 0, 0), (17000, 40, 0, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_there_and_back(shape, dtype):
    rows, cols, gap, shift = shape
    print("checkpoint", shape, dtype, flush=True)
    x = normal(3, rows, cols, dtype=torch.float64)
    # Groups of all sizes.
    x *= torch.exp2(torch.randint(-12, 8, (rows, 1), generator=torch.Generator().manual_seed(4)).double())
    check(x.to(DTYPES[dtype]), gap, shift)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_borders(dtype):
    """Largest magnitudes on both sides of where a scale doubles, ties between
    codes, the type's ends, zeros, and values that are not finite."""
    dtype = DTYPES[dtype]
    info = torch.finfo(dtype)
    tops = []
    for e in (0.0, -3.0, 7.0):
        for top in (127.0, 127.25, 127.5, 127.75, 128.0, 64.0, 63.75):
            tops.append(math.ldexp(top, int(e)))
    tops += [info.max, info.max / 2, info.tiny, 100 * info.tiny, TINY[dtype], 3 * TINY[dtype], 0.0, math.inf, -math.inf, math.nan]
    x = torch.zeros(len(tops), 70, dtype=torch.float64)
    for i, top in enumerate(tops):
        x[i, 0::2] = torch.linspace(-1, 1, 35, dtype=torch.float64) * (top if math.isfinite(top) else 5.0)
        x[i, 40] = -top if math.isfinite(top) else top          # the second group; the first and the last hold less
        x[i, 41:48] = (x[i, 40].abs() / 128 * torch.tensor([0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 0.25])) if math.isfinite(top) else 1.0
    codes, scales = check(x.to(dtype))
    # Only the group that holds it stands for NaN.
    assert (scales == 255).sum() == 3 and (scales[-3:, 1] == 255).all()
    assert (scales[len(tops) - 4] == 1).all() and not codes[len(tops) - 4].any()


def test_exact_in_every_type():
    """What 8 bits stand for is a value of 16-bit types too."""
    for dtype in (torch.bfloat16, torch.float16):
        x = normal(5, 40, 200, dtype=dtype, scale=30.0)
        s = Saved(x)
        wide, narrow = torch.empty(40, 200, device="cuda"), torch.empty(40, 200, dtype=dtype, device="cuda")
        checkpoint_restore(s.c, wide)
        checkpoint_restore(s.c, narrow)
        assert torch.equal(narrow.float(), wide)
        assert (wide.cpu().double() - x.double()).abs().max() <= x.abs().max().double() / 64 / 2
        again = Saved(rows=40, cols=200)                         # and keeps its values
        checkpoint_save(narrow, again.c)
        assert torch.equal(again.values(), s.values())


def test_restore_of_any_bytes():
    """Every scale and code that a byte can be: powers of two to the type's ends."""
    codes = torch.arange(256, dtype=torch.uint8).view(torch.int8).repeat(256, 1)
    scales = torch.arange(256, dtype=torch.uint8)[:, None].repeat(1, 8)
    c = Checkpoint(Bytes(codes).t, Bytes(scales).t)
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        out = blank(256, 256, dtype)
        checkpoint_restore(c, out.t)
        want = stands_for(codes, scales).to(torch.float32).to(dtype)
        got = out.t.cpu()
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got[:255], want[:255]) and out.intact()


def test_slices_streams_and_repeats():
    """Column slices of one buffer, another stream, the same bits."""
    x = normal(6, 100, 400, dtype=torch.bfloat16).cuda()
    whole = torch.empty(100, 400, dtype=torch.int8, device="cuda")
    scales = torch.empty(100, 2, 7, dtype=torch.uint8, device="cuda")
    halves = [Checkpoint(whole[:, i * 200:(i + 1) * 200], scales[:, i]) for i in range(2)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i, h in enumerate(halves):
        checkpoint_save(x[:, i * 200:(i + 1) * 200], h, stream=side if i else None)
    torch.cuda.synchronize()
    for i, h in enumerate(halves):
        codes, want = to_8bit(x[:, i * 200:(i + 1) * 200].cpu())
        assert torch.equal(h.codes.cpu(), codes) and torch.equal(h.scales.cpu(), want)
        for _ in range(2):
            again = Checkpoint.empty(100, 200)
            checkpoint_save(x[:, i * 200:(i + 1) * 200], again, stream=side.cuda_stream)
            side.synchronize()
            assert torch.equal(again.codes, h.codes) and torch.equal(again.scales, h.scales)


def test_long_offsets():
    """Rows whose offsets pass 2^32 bytes, in every operand."""
    rows, cols, stride = 3, 40, (1 << 32) + 4096
    raw = torch.empty(2 * stride + 4096, dtype=torch.int8, device="cuda")
    codes, scales = raw.as_strided((rows, cols), (stride, 1), 0), raw.view(torch.uint8).as_strided((rows, 2), (stride, 1), 64)
    x = raw.view(torch.bfloat16).as_strided((rows, cols), (stride // 2, 1), 64)
    back = raw.view(torch.bfloat16).as_strided((rows, cols), (stride // 2, 1), 128)
    x.copy_(normal(1, rows, cols, dtype=torch.bfloat16))
    checkpoint_save(x, Checkpoint(codes, scales))
    checkpoint_restore(Checkpoint(codes, scales), back)
    want_codes, want_scales = to_8bit(x.cpu())
    assert torch.equal(codes.cpu(), want_codes) and torch.equal(scales.cpu(), want_scales)
    assert torch.equal(back.cpu().double(), stands_for(want_codes, want_scales))


def test_empty():
    for rows, cols in ((0, 40), (5, 0), (0, 0)):
        c = Checkpoint.empty(rows, cols)
        assert c.scales.shape == (rows, groups(cols))
        checkpoint_save(torch.empty(rows, cols, device="cuda"), c)
        checkpoint_restore(c, torch.empty(rows, cols, device="cuda"))


def test_refusals():
    x = torch.ones(4, 64, dtype=torch.bfloat16, device="cuda")
    c = Checkpoint.empty(4, 64)
    c.codes.fill_(7)
    for error, args in [
        (TypeError, (x, x)),
        (TypeError, (x, (c.codes,))),
        (TypeError, (x, None)),
        (TypeError, (x.double(), c)),
        (TypeError, (x, Checkpoint(c.codes.view(torch.uint8), c.scales))),
        (TypeError, (x, Checkpoint(c.codes, c.scales.view(torch.int8)))),
        (ValueError, (x[:3], c)),
        (ValueError, (x, Checkpoint(c.codes, c.scales[:, :1]))),
        (ValueError, (x, Checkpoint(c.codes[:, :63], c.scales))),
        (ValueError, (x[0], c)),
        (ValueError, (x, Checkpoint(c.codes.cpu(), c.scales))),
        (ValueError, (x, Checkpoint(c.codes.t().contiguous().t(), c.scales))),
        (FsdpError, (x, Checkpoint(x.view(torch.int8)[:, :64], c.scales))),
        (FsdpError, (x, Checkpoint(c.codes, c.codes.view(torch.uint8)[:, :2]))),
    ]:
        with pytest.raises(error):
            checkpoint_save(*args)
    out = torch.ones(4, 64, dtype=torch.bfloat16, device="cuda")
    for error, args in [
        (TypeError, (x, out)),
        (TypeError, (c, out.double())),
        (ValueError, (c, out[:3])),
        (ValueError, (c, out.t().contiguous().t())),
        (FsdpError, (Checkpoint(out.view(torch.int8)[:, :64], c.scales), out)),
    ]:
        with pytest.raises(error):
            checkpoint_restore(*args)
    torch.cuda.synchronize()
    assert bool((c.codes == 7).all()) and bool((out == 1).all())
