"""Launches of the largest sizes that the block operators accept, on the host: a
launch holds below 2^32 threads along x and 2^16 workgroups along y."""

from __future__ import annotations

import json
import os
import subprocess
import sys

import pytest

from paper_2411_00284_amd import _native
from test_block_launch_forms import BF16, F32, at, distill, linear, linear_grad, norm, norm_grad

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def grids(tmp_path_factory):
    stub = str(tmp_path_factory.mktemp("stub") / "hip_grid_stub.so")
    subprocess.run(["gcc", "-std=gnu99", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", os.path.join(HERE, "hip_grid_stub.c"), "-o",
                    stub], check=True)

    def run(calls):
        res = subprocess.run([sys.executable, os.path.join(HERE, "block_grid_worker.py"), stub, _native.BLOCK_LIB_PATH], text=True,
                             input=json.dumps(calls), capture_output=True, timeout=300)
        assert res.returncode == 0, res.stderr
        return json.loads(res.stdout)

    return run


WIDE = 1 << 28


@pytest.mark.parametrize("calls", [
    [linear(m, n, k, d) for m in (1, 2, 4, 5, 64) for n, k in ((WIDE, 16), (WIDE // 2, 64)) for d in (BF16, F32)],
    [linear_grad(m, WIDE, 16, BF16, 2, dbias=at(40)) for m in (0, 1, 40)],
    [linear_grad(m, WIDE, 8, BF16, dweight=at(40)) for m in (0, 1, 4)],
    [linear_grad(WIDE, 16, 16, BF16, 2, dbias=at(40), dx=at(44))],
    [linear(WIDE, 16, 16, BF16)],
    [norm(1 << 40, 64, BF16, F32, F32), norm_grad(1 << 36, 64, BF16, F32, F32), norm_grad(60000, 16384, BF16, F32, F32, 60000),
     norm_grad(0, 16384, BF16, F32, F32, 60000)],
    [distill(1 << 32, 8, BF16), distill(1 << 32, 8, F32, grad=True), distill(1 << 24, 20000, BF16, grad=True)],
], ids=["linear", "dbias", "dweight", "tall dx", "tall", "norms", "distill"])
def test_launches_fit(grids, calls):
    spread = 1 << 52                                   # made-up matrices far from each other
    calls = [[name, [(f, k, None if k == "p" and v is None else ((v >> 36) - 15) * spread if k == "p" else v) for f, k, v in fields]]
             for name, fields in calls]
    for launched in grids(calls):
        assert launched
        for name, threads, rows in launched:
            assert 0 < threads < 1 << 32 and 0 < rows < 1 << 16, (name, threads, rows)
