"""fp32 sums of the step's gradients over more terms than a run of 512."""

from __future__ import annotations

import torch
import pytest

from paper_2411_00284_amd import linear_backward
from step_util import Saved

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def test_linear_from_8_bits():
    """A sum of 2^25 and then ones: beside 2^25 a one (two of them too) is rounded away, so that a run
    after the other loses those of the first run only, where one long sum would lose all of them."""
    m, n, k, big = 2048, 1024, 4096, 2.0 ** 25
    x, weight = torch.ones(m, k), torch.ones(n, k)
    x[0], weight[0] = big, big
    dx, dweight = torch.empty(m, k, device="cuda"), torch.empty(n, k, device="cuda")
    linear_backward(torch.ones(m, n, device="cuda"), Saved(x).c, weight.cuda(), dx=dx, dweight=dweight)
    for got, terms in ((dx, n), (dweight, m)):
        # 511 ones of the first run, and the rounding of the joined sums to multiples of 4
        assert float((got.double() - (big + terms - 1)).abs().max()) <= 511 + 4
