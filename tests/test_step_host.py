"""The C ABI of the step's operators on the host: the header is C, the library
exports what it declares, and bad arguments are refused before any HIP call
(this machine may have no GPU)."""

from __future__ import annotations

import ctypes
import math
import os
import re
import subprocess

import pytest
import torch  # noqa: F401  (before the library: one HIP runtime)

import paper_2411_00284_amd as fw
from paper_2411_00284_amd import _native
from step_calls import FIELDS, header

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BLOCK = ctypes.CDLL(_native.BLOCK_LIB_PATH)
LIB = ctypes.CDLL(_native.STEP_LIB_PATH)
BLOCK.fsdp_block_last_error.restype = ctypes.c_char_p
INVALID, ALIGN, OVERFLOW, TOO_MANY, OVERLAP = 1, 2, 3, 4, 7
KINDS = {"p": ctypes.c_void_p, "q": ctypes.c_int64, "i": ctypes.c_int32, "f": ctypes.c_float}


def status_of(function, struct, values):
    args = None
    if values is not None:
        assert set(values) <= {f for f, _ in FIELDS[struct]}, values
        args = type("Args", (ctypes.Structure,), {"_fields_": [(f, KINDS[k]) for f, k in FIELDS[struct]]})()
        for f, v in values.items():
            setattr(args, f, v)
    f = getattr(LIB, function)
    f.restype = ctypes.c_int32
    p = ctypes.byref(args) if args is not None else None
    if function.endswith("_workspace"):
        return f(p, ctypes.byref(ctypes.c_int64(-1)))
    return f(p, ctypes.c_void_p(0), ctypes.c_int64(0), None) if hasattr(LIB, function + "_workspace") else f(p, None)


def refused(function, struct, values, status, text):
    assert status_of(function, struct, values) == status, BLOCK.fsdp_block_last_error()
    assert text in BLOCK.fsdp_block_last_error().decode(), BLOCK.fsdp_block_last_error()


def at(k):
    """A made-up device address: the calls here fail before using it."""
    return (k + 1) << 24


def test_header_compiles_as_c():
    src = '#include "fsdp_step.h"\nint main(void){fsdp_step_gated_args a = {0}; (void)a; return FSDP_STEP_GROUP;}\n'
    res = subprocess.run(["gcc", "-std=c99", "-x", "c", "-fsyntax-only", "-D__HIP_PLATFORM_AMD__",
                          f"-I{os.path.join(ROOT, 'include')}", "-I/opt/rocm/include", "-"], input=src, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr


def test_library_exports_what_the_header_declares():
    names = set(re.findall(r"\b(fsdp_[a-z0-9_]+)\s*\(", header()))
    out = subprocess.run(["nm", "-D", "--defined-only", _native.STEP_LIB_PATH], capture_output=True, text=True, check=True).stdout
    exported = {line.split()[-1] for line in out.splitlines() if " T " in line}
    assert len(names) == 10 and names <= exported


SAVE = dict(rows=4, cols=64, x=at(0), codes=at(1), scales=at(2), x_stride=64, codes_stride=64, scales_stride=2)


@pytest.mark.parametrize("more,status,text", [
    (dict(rows=-1), INVALID, "negative"),
    (dict(cols=-1), INVALID, "negative"),
    (dict(rows=1 << 31), OVERFLOW, "rows"),
    (dict(cols=(1 << 30) + 1), OVERFLOW, "cols"),
    (dict(dtype=3), INVALID, "dtype"),
    (dict(dtype=1 << 8), INVALID, "dtype"),
    (dict(x=None), INVALID, "x is NULL"),
    (dict(codes=None), INVALID, "codes is NULL"),
    (dict(scales=None), INVALID, "scales is NULL"),
    (dict(x=at(0) + 1), ALIGN, "x is not"),
    (dict(x_stride=63), INVALID, "stride"),
    (dict(codes_stride=63), INVALID, "stride"),
    (dict(scales_stride=1), INVALID, "stride"),
    (dict(cols=65), INVALID, "stride"),
])
def test_saved_refusals(more, status, text):
    for name in ("save", "restore"):
        refused("fsdp_step_" + name, name, {**SAVE, **more}, status, text)


@pytest.mark.parametrize("name,more,text", [
    ("save", dict(codes=at(0)), "codes overlaps x"),
    ("save", dict(scales=at(0) + 127), "scales overlaps x"),
    ("save", dict(scales=at(1) + 10), "overlaps"),
    ("restore", dict(x=at(1)), "x overlaps codes"),
    ("restore", dict(x=at(2)), "x overlaps scales"),
])
def test_saved_places(name, more, text):
    refused("fsdp_step_" + name, name, {**SAVE, **more}, OVERLAP, text)


GATED = dict(m=4, n=64, k=8, x=at(0), gate_weight=at(1), up_weight=at(2), out=at(3), x_stride=8, gate_weight_stride=8,
             up_weight_stride=8, out_stride=64)
KEPT = dict(gate=at(4), up=at(5), gate_stride=64, up_stride=64)
SAVED = dict(KEPT, gate_scales=at(6), up_scales=at(7), gate_scales_stride=2, up_scales_stride=2)


@pytest.mark.parametrize("more,status,text", [
    (dict(m=-1), INVALID, "negative"),
    (dict(k=0), INVALID, "k must"),
    (dict(dtype=7), INVALID, "dtype"),
    (dict(activation=5), INVALID, "activation"),
    (dict(n=1 << 30), OVERFLOW, "size"),
    (dict(m=1 << 28, n=1 << 20, out_stride=1 << 20), OVERFLOW, "tiles"),
    (dict(x=None), INVALID, "x is NULL"),
    (dict(up_weight=None), INVALID, "up_weight is NULL"),
    (dict(out=None), INVALID, "out is NULL"),
    (dict(gate_weight=at(1) + 1), ALIGN, "gate_weight"),
    (dict(out=at(0)), OVERLAP, "out overlaps x"),
    (dict(out=at(2)), OVERLAP, "out overlaps up_weight"),
    (dict(gate=at(4), gate_stride=64), INVALID, "go together"),
    (dict(KEPT, gate_scales=at(6), gate_scales_stride=2), INVALID, "go together"),
    (dict(gate_scales=at(6), up_scales=at(7), gate_scales_stride=2, up_scales_stride=2), INVALID, "needs gate"),
    (dict(SAVED, gate_scales_stride=1), INVALID, "stride"),
    (dict(SAVED, up=at(4)), OVERLAP, "overlaps"),
    (dict(SAVED, up_scales=at(6)), OVERLAP, "overlaps"),
    (dict(KEPT, gate=at(3)), OVERLAP, "overlaps"),
    (dict(m=64, n=64, k=1 << 25, x_stride=1 << 25, gate_weight_stride=1 << 25, up_weight_stride=1 << 25, gate_weight=at(1 << 12),
          up_weight=at(1 << 13), out=at(1 << 14)), OVERFLOW, "rows"),
])
def test_gated_refusals(more, status, text):
    for name in ("fsdp_step_gated", "fsdp_step_gated_workspace"):
        refused(name, "gated", {**GATED, **more}, status, text)


GRAD = dict(m=4, n=64, k=8, dout=at(0), x=at(1), gate_weight=at(2), up_weight=at(3), gate=at(4), up=at(5), dout_stride=64, x_stride=8,
            gate_weight_stride=8, up_weight_stride=8, gate_stride=64, up_stride=64)
DX = dict(dx=at(8), dx_stride=8)
DW = dict(dgate_weight=at(9), dup_weight=at(10), dgate_weight_stride=8, dup_weight_stride=8)


@pytest.mark.parametrize("more,status,text", [
    (dict(m=-1), INVALID, "negative"),
    (dict(dtype=-1), INVALID, "dtype"),
    (dict(activation=-1), INVALID, "activation"),
    (dict(DX, gate=None), INVALID, "gate is NULL"),
    (dict(DX, dout=None), INVALID, "dout is NULL"),
    (dict(out=at(8), out_stride=64, dout=None), INVALID, "dout is NULL"),
    (dict(DX, gate_weight=None), INVALID, "gate_weight is NULL"),
    (dict(DW, x=None), INVALID, "x is NULL"),
    (dict(dgate_weight=at(9), dgate_weight_stride=8), INVALID, "go together"),
    (dict(DX, gate_scales=at(6), gate_scales_stride=2), INVALID, "go together"),
    (dict(DX, out=at(4), out_stride=64), OVERLAP, "out overlaps gate"),
    (dict(DX, out=at(0), out_stride=64, gate=at(0)), OVERLAP, "out overlaps gate"),
    (dict(out=at(0), out_stride=65), OVERLAP, "out overlaps dout"),
    (dict(DX, dx=at(0)), OVERLAP, "dx overlaps dout"),
    (dict(DW, dgate_weight=at(2)), OVERLAP, "dgate_weight overlaps gate_weight"),
    (dict(DW, dup_weight=at(9)), OVERLAP, "overlaps"),
    (dict(DW, x_scales=at(9) + 5, x_scales_stride=1), OVERLAP, "overlaps x_scales"),
])
def test_gated_grad_refusals(more, status, text):
    for name in ("fsdp_step_gated_grad", "fsdp_step_gated_grad_workspace"):
        refused(name, "gated_grad", {**GRAD, **more}, status, text)


@pytest.mark.parametrize("more,status,text", [
    (dict(activation=2, dx=at(8), dx_stride=8), INVALID, "pre is NULL"),
    (dict(dtimes=at(8), dtimes_stride=64), INVALID, "dtimes needs times"),
    (dict(dx=at(1), dx_stride=8), OVERLAP, "dx overlaps x"),
    (dict(dweight=at(6), dweight_stride=8), OVERLAP, "dweight overlaps x_scales"),
    (dict(dweight=at(8), dweight_stride=8, x=None), INVALID, "x is NULL"),
    (dict(dx=at(8), dx_stride=8, weight=None), INVALID, "weight is NULL"),
])
def test_linear_grad_refusals(more, status, text):
    base = dict(m=4, n=64, k=8, dout=at(0), x=at(1), x_scales=at(6), weight=at(2), dout_stride=64, x_stride=8, x_scales_stride=1,
                weight_stride=8)
    for name in ("fsdp_step_linear_grad", "fsdp_step_linear_grad_workspace"):
        refused(name, "linear_grad", {**base, **more}, status, text)


POLICY = dict(tokens=4, vocab=100, temperature=1, clip_low=0.2, clip_high=0.2, logits=at(0), actions=at(1), old_logp=at(2),
              advantages=at(3), loss=at(4), logits_stride=100)


@pytest.mark.parametrize("more,status,text", [
    (dict(tokens=-2), INVALID, "tokens"),
    (dict(vocab=0), INVALID, "vocab"),
    (dict(vocab=1 << 31), OVERFLOW, "vocab"),
    (dict(dtype=9), INVALID, "dtype"),
    (dict(actions_64=2), INVALID, "actions_64"),
    (dict(temperature=0), INVALID, "temperature"),
    (dict(temperature=math.inf), INVALID, "temperature"),
    (dict(temperature=1e-40), INVALID, "temperature"),
    (dict(clip_low=1.5), INVALID, "clip_low"),
    (dict(clip_low=math.nan), INVALID, "clip_low"),
    (dict(clip_high=-1), INVALID, "clip_high"),
    (dict(kl_weight=math.nan, ref_logp=at(6)), INVALID, "kl_weight"),
    (dict(kl_weight=0.1), INVALID, "ref_logp"),
    (dict(loss=None), INVALID, "wanted"),
    (dict(actions=None), INVALID, "actions is NULL"),
    (dict(old_logp=None), INVALID, "old_logp is NULL"),
    (dict(advantages=at(3) + 2), ALIGN, "advantages"),
    (dict(actions=at(1) + 4, actions_64=1), ALIGN, "actions"),
    (dict(dlogits=at(5), dlogits_stride=100), INVALID, "dloss is NULL"),
    (dict(loss=at(0)), OVERLAP, "loss overlaps logits"),
    (dict(loss=at(2) + 12), OVERLAP, "loss overlaps old_logp"),
    (dict(logp=at(4)), OVERLAP, "overlaps"),
    (dict(dlogits=at(0), dlogits_stride=101, dloss=at(6)), OVERLAP, "dlogits overlaps logits"),
])
def test_policy_refusals(more, status, text):
    refused("fsdp_step_policy", "policy", {**POLICY, **more}, status, text)


def test_policy_grad_refusals():
    refused("fsdp_step_policy_grad", "policy", POLICY, INVALID, "lse and dlogits")


def test_null_args():
    for name, struct in [(n, s) for s in FIELDS for n in ("fsdp_step_" + s, f"fsdp_step_{s}_workspace") if hasattr(LIB, n)]:
        refused(name, struct, None, INVALID, "NULL")


def test_nothing_to_do_makes_no_hip_call():
    assert status_of("fsdp_step_save", "save", dict(cols=5)) == 0
    assert status_of("fsdp_step_restore", "restore", dict(rows=5)) == 0
    assert status_of("fsdp_step_policy", "policy", dict(vocab=5, temperature=1)) == 0


def test_binding_refuses_host_tensors():
    x, c = torch.zeros(4, 64), fw.Checkpoint.empty(4, 64, device="cpu")
    assert c.codes.shape == (4, 64) and c.scales.shape == (4, 2)
    for call in (lambda: fw.checkpoint_save(x, c), lambda: fw.checkpoint_restore(c, x), lambda: fw.gated_linear(x, x, x, x[:, :4]),
                 lambda: fw.gated_linear_backward(x[:, :4], x, x, x, x[:, :4], x[:, :4], dx=x),
                 lambda: fw.linear_backward(x[:, :4], c, x, dx=x), lambda: fw.policy_loss(x, x[:, 0].int(), x[:, 0], x[:, 0], x[:, 0])):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(ValueError, match="activation"):
        fw.gated_linear(x, x, x, x[:, :4], activation="tanh")
