"""Which kernels the block operators launch, on the host: the library is loaded
against a stub of the HIP runtime that records launches by name and runs
nothing, in a child process."""

from __future__ import annotations

import itertools
import json
import os
import re
import subprocess
import sys

import pytest

from paper_2411_00284_amd import _native

HERE = os.path.dirname(os.path.abspath(__file__))
HEADER = os.path.join(os.path.dirname(HERE), "include", "fsdp_block.h")
BF16, F32, F16 = 0, 1, 2
SIZE = {BF16: 2, F32: 4, F16: 2}
KIND = {"int64_t": "q", "int32_t": "i", "float": "f", "fsdp_dtype": "i", "fsdp_activation": "i"}


def fields_of(name):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct fsdp_%s_args \{(.*?)\}" % name, text, re.S).group(1)
    out = []
    for line in body.split(";"):
        line = " ".join(line.split())
        if line:
            kind, names = re.match(r"((?:const )?\w+ ?\*?) ?(.*)", line).groups()
            for n in names.split(","):
                pointer = "*" in kind or "*" in n
                out.append((n.strip(" *"), "p" if pointer else KIND[kind.replace("const", "").strip()]))
    return out


FIELDS = {n: fields_of(n) for n in ("norm", "norm_grad", "linear", "linear_grad", "distill")}


def call(function, **values):
    struct = {"fsdp_block_norm": "norm", "fsdp_block_norm_grad": "norm_grad", "fsdp_block_linear": "linear",
              "fsdp_block_linear_grad": "linear_grad"}.get(function, "distill")
    assert set(values) <= {f for f, _ in FIELDS[struct]}, values
    return [function, [(f, k, values.get(f, None if k == "p" else 0)) for f, k in FIELDS[struct]]]


def at(k, shift=0):
    return (1 << 40) + (k << 36) + shift


def norm(tokens, hidden, block, stream, weight):
    return call("fsdp_block_norm", tokens=tokens, hidden=hidden, block_dtype=block, stream_dtype=stream, weight_dtype=weight,
                residual_scale=1.0, branch_scale=1.0, x=at(0), branch=at(1), post_weight=at(2), pre_weight=at(3), y=at(4),
                h=at(5), x_stride=hidden, branch_stride=hidden, y_stride=hidden, h_stride=hidden)


def norm_grad(tokens, hidden, block, stream, weight, gate_rows=0, sums=True):
    more = dict(gate=at(9), dgate=at(10), gate_rows=gate_rows) if gate_rows else {}
    if sums:
        more |= dict(dpre_weight=at(7), dpost_weight=at(8))
    return call("fsdp_block_norm_grad", tokens=tokens, hidden=hidden, block_dtype=block, stream_dtype=stream, weight_dtype=weight,
                residual_scale=1.0, branch_scale=1.0, y=at(0), dh=at(1), branch=at(2), post_weight=at(3), pre_weight=at(4),
                dx=at(5), dbranch=at(6), y_stride=hidden, dh_stride=hidden, branch_stride=hidden, dx_stride=hidden,
                dbranch_stride=hidden, **more)


def linear(m, n, k, dtype=BF16, shift=0):
    return call("fsdp_block_linear", m=m, n=n, k=k, dtype=dtype, x=at(0, shift), weight=at(1), out=at(2), x_stride=k,
                weight_stride=k, out_stride=n)


def linear_grad(m, n, k, dtype=BF16, act=0, **outs):
    strides = dict(dout_stride=n, x_stride=k, weight_stride=k, pre_stride=n, dx_stride=k, dweight_stride=k)
    return call("fsdp_block_linear_grad", m=m, n=n, k=k, dtype=dtype, activation=act, dout=at(0), x=at(1), weight=at(2),
                pre=at(3) if act else None, **strides, **outs)


def distill(tokens, vocab, dtype, grad=False, backward=False):
    outs = dict(dloss=at(4), dlogits=at(5), dlogits_stride=vocab) if grad else {}
    outs |= dict(lse=at(6)) if backward else dict(loss=at(3))
    return call("fsdp_block_distill_grad" if backward else "fsdp_block_distill", tokens=tokens, vocab=vocab, top=8, dtype=dtype,
                teacher_dtype=F32, temperature=1.0, logits=at(0), teacher=at(1), ids=at(2), logits_stride=vocab, **outs)


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    stub = str(tmp_path_factory.mktemp("stub") / "hip_stub.so")
    subprocess.run(["gcc", "-std=gnu99", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", os.path.join(HERE, "hip_stub.c"), "-o", stub],
                   check=True)

    def demangled(names):
        out = subprocess.run(["c++filt"], input="\n".join(names), capture_output=True, text=True, check=True).stdout
        return [n.replace("fsdp_block::(anonymous namespace)::", "").split("(", 1)[0].removeprefix("void ") for n in out.splitlines()]

    def run(calls):
        res = subprocess.run([sys.executable, os.path.join(HERE, "block_launch_worker.py"), stub, _native.BLOCK_LIB_PATH],
                             text=True, input=json.dumps(calls), capture_output=True, timeout=300)
        assert res.returncode == 0, res.stderr
        got = json.loads(res.stdout)
        return [demangled(names) if names else [] for names in got["launched"]], got["launched"], set(got["kernels"])

    return run


def heads(names):
    return [re.sub(r"<.*|I\w+$", "", n).split("ILi")[0] for n in names]


def test_launches_per_call(launches):
    """The number of kernels that the header states."""
    names, _, _ = launches([
        norm(100, 4096, BF16, F32, BF16),
        norm_grad(100, 4096, BF16, F32, BF16),
        norm_grad(100, 4096, BF16, F32, BF16, sums=False),
        norm_grad(100, 4096, BF16, BF16, BF16, gate_rows=100, sums=False),
        norm_grad(0, 4096, BF16, BF16, BF16),
        linear(1, 4096, 4096),
        linear(4096, 4096, 4096),
        linear(64, 256, 8192),
        linear(700, 700, 701),
        linear(0, 4096, 4096),
        linear(4096, 14336, 4096),
        linear(4101, 4104, 520),
        linear(1020, 18440, 520),
        linear_grad(4096, 4096, 4096, dx=at(5), dweight=at(6)),
        linear_grad(4096, 4096, 4096, act=2, dx=at(5), dweight=at(6), dbias=at(7)),
        linear_grad(0, 64, 64, dx=at(5), dweight=at(6), dbias=at(7)),
        distill(100, 32000, BF16),
        distill(100, 32000, BF16, grad=True),
        distill(100, 32000, BF16, grad=True, backward=True),
        distill(0, 32000, BF16),
    ])
    assert [len(n) for n in names] == [1, 2, 1, 1, 1, 1, 1, 2, 2, 0, 2, 2, 2, 2, 4, 2, 1, 1, 1, 0]
    assert "row_kernel" in names[5][0] and "join_parts" in names[7][1] and "pad_kernel" in names[8][0]


def test_every_kernel_is_reached(launches):
    """No kernel is built that no call launches."""
    types = [(BF16, BF16, BF16), (BF16, BF16, F32), (BF16, F32, BF16), (BF16, F32, F32), (F16, F16, F16), (F16, F16, F32),
             (F16, F32, F16), (F16, F32, F32), (F32, F32, F32)]
    calls = []
    for (b, s, w), hidden in itertools.product(types, (256, 1000, 2048, 4096, 8192, 16384)):
        calls += [norm(1000, hidden, b, s, w), norm_grad(1000, hidden, b, s, w)]
    for d in (BF16, F16, F32):
        calls += [linear(m, 4096, 4096, d) for m in (1, 2, 4)]
        calls += [linear(m, n, k, d) for m, n, k in ((16, 4096, 4096), (1024, 4096, 4096), (2048, 4096, 4096), (8192, 8192, 8192),
                                                     (300, 257, 8191), (64, 256, 8192), (128, 14336, 1024))]
        calls += [linear_grad(m, n, k, d, 2, dx=at(5), dweight=at(6), dbias=at(7))
                  for m, n, k in ((64, 4096, 64), (64, 256, 8192), (1024, 4096, 4096), (2048, 4096, 4096), (4096, 1024, 4096),
                                  (512, 2048, 512), (8192, 8192, 8192), (4096, 2048, 2048), (1024, 2048, 4096), (256, 512, 1024), (4096, 4096, 1024),
                                  (8192, 4096, 14336), (128, 1024, 14336), (1024, 128, 14336))]
        for tokens, vocab in ((5, 32000), (5000, 1000), (5000, 6000), (5000, 128256)):
            calls += [distill(tokens, vocab, d), distill(tokens, vocab, d, grad=True)]
    _, mangled, built = launches(calls)
    reached = {n for names in mangled for n in names}
    assert reached <= built
    assert not built - reached, sorted(built - reached)
