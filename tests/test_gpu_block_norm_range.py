"""The norms' gradient over the range of fp32: rows so large or so small that
the cube of their inverse root mean square is none of its values, in every width's
form.  The squares of a row still add up within the range."""

from __future__ import annotations

import math

import pytest
import torch

from block_util import blank, close, normal
from paper_2411_00284_amd import block_norm_backward
from test_gpu_block_norm import gradient

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

LARGE = [1.0, 1e12, 1e14, 1e15, 1e16, 5e16]
SMALL = [1.0, 1e-10, 1e-13, 1e-14, 1e-15, 1e-16]


@pytest.mark.parametrize("hidden", [256, 1000, 2048, 4096, 8192, 16384])
@pytest.mark.parametrize("block", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scales,eps", [(LARGE, 1e-5), (LARGE, 0.0), (SMALL, 0.0)], ids=["large", "large without eps", "small"])
@pytest.mark.parametrize("with_dy", [True, False])
def test_rows(hidden, block, scales, eps, with_dy):
    print("norm gradient range", hidden, block, scales[-1], eps, with_dy, flush=True)
    t = len(scales)
    s = torch.tensor(scales, dtype=torch.float64)[:, None]
    y = (normal(1, t, hidden, dtype=torch.float64) * s).float()
    b = (normal(2, t, hidden, dtype=torch.float64) * s.flip(0)).to(block)
    # a gradient of y of the size of the norm's own
    dy = (normal(6, t, hidden, dtype=torch.float64) / s).float() if with_dy else None
    dh = normal(7, t, hidden, dtype=block)
    pre, post = normal(3, hidden, shift=1), normal(4, hidden, shift=1)
    got = {"dx": blank(t, hidden, torch.float32), "dbranch": blank(t, hidden, block),
           "dpre_weight": blank(None, hidden, torch.float32), "dpost_weight": blank(None, hidden, torch.float32)}
    block_norm_backward(y.cuda(), dy=None if dy is None else dy.cuda(), dh=dh.cuda(), branch=b.cuda(), pre_weight=pre.cuda(),
                        post_weight=post.cuda(), eps=eps, **{k: v.t for k, v in got.items()})
    want, bound = gradient(y, dy, dh, b, post, None, pre, 1.0, 1.0, eps)
    for k in want:
        close(got[k].t, want[k], bound[k], k)
        assert got[k].intact()


def test_a_branch_without_its_norm():
    """Without post_weight the branch is a summand: its gradient does not depend
    on its values."""
    t, n = 3, 500
    dy, b, gate = normal(6, t, n), normal(2, t, n), normal(5, n)
    b[0, 3], b[1, 4], b[2, 5] = math.inf, -math.inf, math.nan
    out = torch.empty(t, n, device="cuda")
    block_norm_backward(b.cuda(), dy=dy.cuda(), branch=b.cuda(), gate=gate.cuda(), dbranch=out, branch_scale=0.5)
    assert torch.equal(out.cpu(), (0.5 * dy) * gate)
