"""Which kernels the step's operators launch, on the host: the library is loaded
against a stub of the HIP runtime that records launches and runs nothing, in a
child process."""

from __future__ import annotations

import json
import os
import re
import subprocess
import sys

import pytest

from paper_2411_00284_amd import _native
from step_calls import BF16, CODE, F16, F32, gated, gated_grad, linear_grad, policy, restore, save
from step_shapes import FORWARD, GRADIENT, POLICIES, ROWS

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    stub = str(tmp_path_factory.mktemp("stub") / "hip_grid_stub.so")
    subprocess.run(["gcc", "-std=gnu99", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", os.path.join(HERE, "hip_grid_stub.c"), "-o",
                    stub], check=True)

    def run(calls):
        res = subprocess.run([sys.executable, os.path.join(HERE, "step_launch_worker.py"), stub, _native.STEP_LIB_PATH], text=True,
                             input=json.dumps(calls), capture_output=True, timeout=300)
        assert res.returncode == 0, res.stderr
        got = json.loads(res.stdout)
        return got["launched"], set(got["kernels"])

    return run


def test_launches_per_call(launches):
    """The number of kernels that the header states."""
    calls = [
        (save(100, 4096), 1), (save(0, 64), 0), (restore(100, 4095), 1), (restore(5, 0), 0),
        (gated(1, 4096, 4096), 1), (gated(4, 4096, 4096, kept="type"), 1), (gated(0, 64, 64), 0), (gated(64, 0, 64), 0),
        (gated(4096, 4096, 4096), 1), (gated(64, 256, 8192), 2), (gated(700, 700, 701), 2), (gated(4101, 2052, 520), 2),
        (gated_grad(4096, 4096, 4096), 3), (gated_grad(4096, 4096, 4096, saved=True, saved_x=True), 4),
        (gated_grad(90, 200, 300, outs=("out",)), 1), (gated_grad(0, 64, 64), 1), (gated_grad(64, 0, 64), 1),
        (gated_grad(90, 200, 300, outs=()), 0),
        (linear_grad(4096, 4096, 4096), 3), (linear_grad(4096, 4096, 4096, act=2, outs=("dx", "dweight", "dbias")), 5),
        (linear_grad(0, 64, 64, outs=("dx", "dweight", "dbias")), 2),
        (policy(100, 32000), 1), (policy(100, 32000, grad=True), 1), (policy(100, 32000, grad=True, backward=True), 1),
        (policy(0, 32000), 0),
    ]
    launched, _ = launches([c for c, _ in calls])
    assert [len(n) for n in launched] == [n for _, n in calls], [[name for name, _, _ in n] for n in launched]


def test_every_kernel_has_a_shape(launches):
    """No kernel is built that no call launches, and each is compared with 64
    bits by the test_gpu_step_*.py."""
    calls = []
    for d, shape in FORWARD:
        calls += [gated(*shape, CODE[d], kept) for kept in ("8bit", "type")]
    calls += [gated(m, n, k, CODE[d]) for d, m, n, k in ROWS]
    for d, shape in GRADIENT:
        calls.append(gated_grad(*shape, CODE[d], saved=True, saved_x=True))
    for d in (BF16, F16, F32):
        # test_gpu_step_gated.test_forward, test_gradient and test_linear_from_8_bits, test_gpu_step_saved.test_there_and_back
        calls += [gated(17, 129, 2050, d, "8bit"), gated_grad(256, 512, 256, d), linear_grad(776, 72, 1287, d, 2, outs=("dx", "dweight", "dbias")),
                  linear_grad(300, 1032, 328, d, 3, saved=False, outs=("dx", "dweight", "dbias")), save(9, 513, d), restore(9, 513, d)]
    for d, tokens, vocab in POLICIES:
        calls += [policy(tokens, vocab, CODE[d]), policy(tokens, vocab, CODE[d], grad=True),
                  policy(tokens, vocab, CODE[d], grad=True, backward=True)]
    launched, built = launches(calls)
    reached = {name for names in launched for name, _, _ in names}
    assert reached <= built
    assert not built - reached, sorted(built - reached)


WIDE = 1 << 27


@pytest.mark.parametrize("calls", [
    [gated(m, n, k, d) for m in (1, 2, 4, 5, 64) for n, k in ((WIDE // 2, 16), (WIDE // 4, 64)) for d in (BF16, F32)],
    [gated_grad(m, WIDE // 2, 16, BF16, outs=("out",)) for m in (0, 1, 40)],
    [gated_grad(m, WIDE // 2, 8, BF16, outs=("dgate_weight", "dup_weight")) for m in (0, 1, 4)],
    [gated_grad(WIDE, 16, 16, BF16, outs=("out", "dx")), gated(WIDE, 16, 16, BF16, "8bit")],
    [save((1 << 31) - 1, 64), restore((1 << 31) - 1, 64), save(3, 1 << 30, F32), restore(3, 1 << 30, F32)],
    [policy(1 << 32, 8), policy(1 << 32, 8, F32, grad=True), policy(1 << 24, 20000, grad=True)],
], ids=["gated", "out", "weights", "tall", "saved", "policy"])
def test_launches_fit(launches, calls):
    """A launch holds below 2^32 threads along x and 2^16 workgroups along y."""
    spread = 1 << 54                                   # made-up matrices far from each other
    calls = [[name, [(f, k, None if k == "p" and v is None else ((v >> 46) - 15) * spread if k == "p" else v) for f, k, v in fields]]
             for name, fields in calls]
    for launched in launches(calls)[0]:
        for name, threads, rows in launched:
            assert 0 < threads < 1 << 32 and 0 < rows < 1 << 16, (name, threads, rows)


REACH = (1 << 31) - 16


@pytest.mark.parametrize("m,n,k,dtype", [(2048, 1024, 5242880, BF16), (64, 64, 1 << 23, F16), (40, 25, 7_000_000, BF16), (64, 64, 4_000_000, F32),
                                         (5, 64, 4_000_000, F32)])
def test_long_rows(launches, m, n, k, dtype):
    """A tile's rows lie within 2^31 bytes of its first: no call takes a form that cannot reach its operands."""
    size = 4 if dtype == F32 else 2
    for name, _, _ in launches([gated(m, n, k, dtype)])[0][0]:
        t = re.search(r"pair_kernelI\w+?GatedForwardELi(\d+)ELi(\d+)E", name)
        if t:
            assert (min(int(t.group(1)), m) - 1) * k * size + 128 <= REACH and (int(t.group(2)) // 2 - 1) * k * size + 128 <= REACH, name
