"""Which inputs an output of the block operators may be: those that the kernels
read where they write and nowhere else.  On the host: a refusal comes before any
HIP call."""

from __future__ import annotations

import pytest

from test_block_host import BF16, F16, F32, OVERLAP, Distill, Linear, LinearGrad, Norm, NormGrad, at, refused
from test_block_launch_forms import call as stub_call
from test_block_launch_forms import launches  # noqa: F401


def linear(**more):
    base = dict(m=16, n=16, k=16, x=at(0), weight=at(1), out=at(2), x_stride=16, weight_stride=16, out_stride=16)
    return Linear(**{**base, **more})


def linear_grad(**more):
    base = dict(m=16, n=16, k=16, dout=at(0), x=at(1), weight=at(2), pre=at(3), times=at(4), dtimes=at(5), dweight=at(6),
                activation=2)
    strides = {s + "_stride": 16 for s in ("dout", "x", "weight", "pre", "times", "dtimes", "dweight")}
    return LinearGrad(**{**base, **strides, **more})


def norm(**more):
    base = dict(tokens=4, hidden=64, x=at(0), branch=at(1), pre_weight=at(2), y=at(3), h=at(4), x_stride=64, branch_stride=64,
                y_stride=64, h_stride=64, eps=1e-5, residual_scale=1, branch_scale=1)
    return Norm(**{**base, **more})


def norm_grad(**more):
    base = dict(tokens=4, hidden=64, y=at(0), dy=at(1), dh=at(2), branch=at(3), pre_weight=at(4), dx=at(5), dbranch=at(6),
                eps=1e-5, residual_scale=1, branch_scale=1)
    strides = {s + "_stride": 64 for s in ("y", "dy", "dh", "branch", "dx", "dbranch")}
    return NormGrad(**{**base, **strides, **more})


def distill(**more):
    base = dict(tokens=4, vocab=8, top=8, temperature=1, logits=at(0), teacher=at(1), ids=at(2), loss=at(3), dloss=at(4),
                dlogits=at(5), logits_stride=8, dlogits_stride=8)
    return Distill(**{**base, **more})


@pytest.mark.parametrize("args,text", [
    # x is read by every column of out: it is no place for out even where it is the residual or the factor too
    (linear(out=at(0), residual=at(0), residual_stride=16), "out overlaps x"),
    (linear(out=at(0), times=at(0), times_stride=16), "out overlaps x"),
    (linear(out=at(1), residual=at(1), residual_stride=16), "out overlaps weight"),
    # the first row of out's place, read by all rows
    (linear(out=at(3), residual=at(3), residual_stride=16, bias=at(3)), "out overlaps bias"),
])
def test_linear(args, text):
    refused("fsdp_block_linear_workspace", args, OVERLAP, text)
    refused("fsdp_block_linear", args, OVERLAP, text)


@pytest.mark.parametrize("more,text", [
    (dict(times=at(1), dtimes=at(1)), "dtimes overlaps x"),
    (dict(times=at(2), dtimes=at(2)), "dtimes overlaps weight"),
    (dict(dtimes=at(1)), "dtimes overlaps x"),
    (dict(dtimes=at(0)), "dtimes overlaps dout"),
])
def test_linear_grad(more, text):
    refused("fsdp_block_linear_grad_workspace", linear_grad(**more), OVERLAP, text)


@pytest.mark.parametrize("more,text", [
    (dict(y=at(0), gate=at(0), gate_rows=1), "y overlaps gate"),
    (dict(h=at(1), gate=at(1), gate_rows=1), "h overlaps gate"),
    (dict(y=at(0), gate=at(0), gate_rows=4), "y overlaps gate"),
    (dict(h=at(1), pre_weight=at(1)), "h overlaps pre_weight"),
    (dict(h=at(1), post_weight=at(1)), "h overlaps post_weight"),
    (dict(y=at(0), stream_dtype=F32, branch=at(0)), "y overlaps branch"),          # another type
])
def test_norm(more, text):
    refused("fsdp_block_norm", norm(**more), OVERLAP, text)


@pytest.mark.parametrize("more,text", [
    (dict(dx=at(1), gate=at(1), gate_rows=1), "dx overlaps gate"),
    (dict(dbranch=at(3), pre_weight=at(3)), "dbranch overlaps pre_weight"),
    (dict(dbranch=at(2), post_weight=at(2)), "dbranch overlaps post_weight"),
    (dict(dx=at(3), dbranch=at(3)), "overlaps"),
])
def test_norm_grad(more, text):
    refused("fsdp_block_norm_grad_workspace", norm_grad(**more), OVERLAP, text)


def test_distill():
    refused("fsdp_block_distill", distill(dlogits=at(2), ids_64=0), OVERLAP, "dlogits overlaps ids")
    refused("fsdp_block_distill", distill(dlogits=at(0), teacher=at(0), teacher_dtype=F16, dtype=BF16), OVERLAP,
            "dlogits overlaps teacher")


def test_what_an_output_may_be(launches):
    """None of these is an overlap: every call is made (against a stub of the
    HIP runtime that runs nothing)."""
    calls = [
        ("fsdp_block_linear", linear(out=at(3), times=at(3), times_stride=16, residual=at(3), residual_stride=16)),
        ("fsdp_block_linear_grad", linear_grad()),
        ("fsdp_block_linear_grad", linear_grad(dtimes=at(4))),
        ("fsdp_block_linear_grad", linear_grad(times=at(0), dtimes=at(0))),
        ("fsdp_block_linear_grad", linear_grad(times=at(3), dtimes=at(3))),
        ("fsdp_block_norm", norm(y=at(0))),
        ("fsdp_block_norm", norm(y=at(0), branch=at(0))),
        ("fsdp_block_norm", norm(y=at(0), h=at(1))),
        ("fsdp_block_norm_grad", norm_grad(dx=at(1), dbranch=at(3))),
        ("fsdp_block_norm_grad", norm_grad(dx=at(1), dy=at(1), y=at(1), dbranch=at(2))),
        ("fsdp_block_distill", distill(dlogits=at(0))),
        ("fsdp_block_distill", distill(dlogits=at(0), teacher=at(0))),
    ]
    names, _, _ = launches([stub_call(name, **{f: getattr(args, f) for f, _ in args._fields_}) for name, args in calls])
    assert all(names)
