"""The C ABI of the block operators on the host: the header is C, the library
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

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "fsdp_block.h")
LIB = ctypes.CDLL(_native.BLOCK_LIB_PATH)
LIB.fsdp_block_last_error.restype = ctypes.c_char_p
INVALID, ALIGN, OVERFLOW, TOO_MANY, OVERLAP = 1, 2, 3, 4, 7
BF16, F32, F16 = 0, 1, 2


def header():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def struct(name):
    """The ctypes structure of a struct of the header."""
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), header(), re.S).group(1)
    fields = []
    for line in body.split(";"):
        line = " ".join(line.split())
        if not line:
            continue
        words = re.match(r"((?:const )?\w+ ?\*?) ?(.*)", line)
        kind, names = words.group(1).strip(), words.group(2)
        for n in names.split(","):
            n = n.strip()
            pointer = "*" in kind or n.startswith("*")
            base = kind.replace("const", "").replace("*", "").strip()
            c = ctypes.c_void_p if pointer else {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "float": ctypes.c_float,
                                                 "fsdp_dtype": ctypes.c_int32, "fsdp_activation": ctypes.c_int32}[base]
            fields.append((n.lstrip("* "), c))
    return type(name, (ctypes.Structure,), {"_fields_": fields})


Norm, NormGrad, Linear, LinearGrad, Distill = (struct("fsdp_%s_args" % n) for n in ("norm", "norm_grad", "linear", "linear_grad",
                                                                                     "distill"))


def call(name, args, workspace=None):
    f = getattr(LIB, name)
    f.restype = ctypes.c_int32
    if name.endswith("_workspace"):
        n = ctypes.c_int64(-1)
        return f(ctypes.byref(args) if args is not None else None, ctypes.byref(n))
    if name in ("fsdp_block_norm_grad", "fsdp_block_linear", "fsdp_block_linear_grad"):
        return f(ctypes.byref(args) if args is not None else None, ctypes.c_void_p(workspace), ctypes.c_int64(0), None)
    return f(ctypes.byref(args) if args is not None else None, None)


def refused(name, args, status, text):
    assert call(name, args) == status, LIB.fsdp_block_last_error()
    assert text in LIB.fsdp_block_last_error().decode()


def at(k):
    """A made-up device address: the calls here fail before using it."""
    return (k + 1) << 24


def test_header_compiles_as_c():
    src = '#include "fsdp_block.h"\nint main(void){fsdp_norm_args a = {0}; (void)a; return FSDP_ACT_NONE;}\n'
    res = subprocess.run(["gcc", "-std=c99", "-x", "c", "-fsyntax-only", "-D__HIP_PLATFORM_AMD__",
                          f"-I{os.path.join(ROOT, 'include')}", "-I/opt/rocm/include", "-"], input=src, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr


def test_library_exports_what_the_header_declares():
    names = set(re.findall(r"\b(fsdp_[a-z0-9_]+)\s*\(", header()))
    out = subprocess.run(["nm", "-D", "--defined-only", _native.BLOCK_LIB_PATH], capture_output=True, text=True, check=True).stdout
    exported = {line.split()[-1] for line in out.splitlines() if " T " in line}
    assert names and names <= exported


def norm(**more):
    base = dict(tokens=4, hidden=64, x=at(0), pre_weight=at(1), h=at(2), x_stride=64, h_stride=64, eps=1e-5, residual_scale=1,
                branch_scale=1)
    return Norm(**{**base, **more})


@pytest.mark.parametrize("more,status,text", [
    (dict(tokens=-1), INVALID, "tokens"),
    (dict(hidden=0), INVALID, "hidden"),
    (dict(hidden=16385), OVERFLOW, "hidden"),
    (dict(block_dtype=3), INVALID, "dtype"),
    (dict(stream_dtype=F16), INVALID, "stream"),
    (dict(weight_dtype=F16), INVALID, "weights"),
    (dict(eps=math.nan), INVALID, "eps"),
    (dict(branch_scale=math.inf), INVALID, "finite"),
    (dict(post_weight=at(3)), INVALID, "branch"),
    (dict(branch=at(3), branch_stride=64, gate=at(4)), INVALID, "gate_rows"),
    (dict(branch=at(3), branch_stride=64, gate=at(4), gate_rows=3), INVALID, "evenly"),
    (dict(h=None), INVALID, "wanted"),
    (dict(pre_weight=None), INVALID, "pre_weight"),
    (dict(x=None), INVALID, "x is NULL"),
    (dict(x=at(0) + 1), ALIGN, "x is not"),
    (dict(x_stride=63), INVALID, "stride"),
    (dict(x_stride=1 << 62), OVERFLOW, "x"),
    (dict(h=at(0)), OVERLAP, "h overlaps x"),
    (dict(h=at(0) + 2 * 63), OVERLAP, "h overlaps x"),
    (dict(h=at(1) - 2), OVERLAP, "h overlaps pre_weight"),
    (dict(y=at(0), y_stride=65), OVERLAP, "y overlaps x"),
    (dict(x_stride=128, h=at(0) + 2 * 63, h_stride=128), OVERLAP, "h overlaps x"),
])
def test_norm_refusals(more, status, text):
    refused("fsdp_block_norm", norm(**more), status, text)


@pytest.mark.parametrize("more,status,text", [
    (dict(dh=at(1)), INVALID, "go together"),
    (dict(dpre_weight=at(1)), INVALID, "pre_weight"),
    (dict(dpost_weight=at(1)), INVALID, "post_weight"),
    (dict(dbranch=at(1)), INVALID, "branch"),
    (dict(dgate=at(1)), INVALID, "gate"),
    (dict(dh=at(1), dh_stride=64, pre_weight=at(2), y=None), INVALID, "y is NULL"),
    (dict(dx=at(0), dx_stride=64), OVERLAP, "dx overlaps y"),
])
def test_norm_grad_refusals(more, status, text):
    base = dict(tokens=4, hidden=64, y=at(0), y_stride=64, eps=1e-5, residual_scale=1, branch_scale=1)
    for name in ("fsdp_block_norm_grad", "fsdp_block_norm_grad_workspace"):
        refused(name, NormGrad(**{**base, **more}), status, text)


@pytest.mark.parametrize("more,status,text", [
    (dict(m=-1), INVALID, "negative"),
    (dict(k=0), INVALID, "k must"),
    (dict(dtype=7), INVALID, "dtype"),
    (dict(activation=5), INVALID, "activation"),
    (dict(activation=-1), INVALID, "activation"),
    (dict(m=1 << 31), OVERFLOW, "size"),
    (dict(m=1 << 29, n=1 << 20, x_stride=8, weight_stride=8, out_stride=1 << 20), OVERFLOW, "tiles"),
    (dict(x=None), INVALID, "x is NULL"),
    (dict(weight=at(1) + 1), ALIGN, "weight"),
    (dict(out=None), INVALID, "out is NULL"),
    (dict(out=at(0)), OVERLAP, "out overlaps x"),
    (dict(pre=at(2), pre_stride=16), OVERLAP, "overlaps"),
    (dict(times=at(2), times_stride=17), OVERLAP, "out overlaps times"),
])
def test_linear_refusals(more, status, text):
    base = dict(m=4, n=16, k=8, x=at(0), weight=at(1), out=at(2), x_stride=8, weight_stride=8, out_stride=16)
    for name in ("fsdp_block_linear", "fsdp_block_linear_workspace"):
        refused(name, Linear(**{**base, **more}), status, text)


@pytest.mark.parametrize("more,status,text", [
    (dict(activation=2, dx=at(4), dx_stride=8), INVALID, "pre is NULL"),
    (dict(dtimes=at(4), dtimes_stride=16), INVALID, "dtimes needs times"),
    (dict(dtimes=at(4), dtimes_stride=16, times=at(5), times_stride=16), INVALID, "pre is NULL"),
    (dict(dx=at(1), dx_stride=8), OVERLAP, "dx overlaps x"),
    (dict(dweight=at(2), dweight_stride=8), OVERLAP, "dweight overlaps weight"),
    (dict(dx=at(4), dx_stride=8, weight=None), INVALID, "weight is NULL"),
])
def test_linear_grad_refusals(more, status, text):
    base = dict(m=4, n=16, k=8, dout=at(0), x=at(1), weight=at(2), dout_stride=16, x_stride=8, weight_stride=8)
    for name in ("fsdp_block_linear_grad", "fsdp_block_linear_grad_workspace"):
        refused(name, LinearGrad(**{**base, **more}), status, text)


@pytest.mark.parametrize("more,status,text", [
    (dict(tokens=-2), INVALID, "tokens"),
    (dict(vocab=0), INVALID, "vocab"),
    (dict(vocab=1 << 31), OVERFLOW, "vocab"),
    (dict(top=1025), TOO_MANY, "top"),
    (dict(teacher_dtype=9), INVALID, "dtype"),
    (dict(ids_64=2), INVALID, "ids_64"),
    (dict(temperature=0), INVALID, "temperature"),
    (dict(temperature=math.nan), INVALID, "temperature"),
    (dict(loss=None), INVALID, "wanted"),
    (dict(ids=None), INVALID, "ids is NULL"),
    (dict(ids=at(2) + 4, ids_64=1), ALIGN, "ids"),
    (dict(dlogits=at(5), dlogits_stride=100), INVALID, "dloss is NULL"),
    (dict(loss=at(0)), OVERLAP, "loss overlaps logits"),
])
def test_distill_refusals(more, status, text):
    base = dict(tokens=4, vocab=100, top=8, temperature=1, logits=at(0), teacher=at(1), ids=at(2), loss=at(3), logits_stride=100)
    refused("fsdp_block_distill", Distill(**{**base, **more}), status, text)


def test_null_args_and_workspace():
    for name in ("fsdp_block_norm", "fsdp_block_norm_grad", "fsdp_block_norm_grad_workspace", "fsdp_block_linear",
                 "fsdp_block_linear_workspace", "fsdp_block_linear_grad", "fsdp_block_linear_grad_workspace",
                 "fsdp_block_distill", "fsdp_block_distill_grad"):
        refused(name, None, INVALID, "NULL")
    LIB.fsdp_block_linear_workspace.restype = ctypes.c_int32
    assert LIB.fsdp_block_linear_workspace(ctypes.byref(Linear()), None) == INVALID


def test_nothing_to_do_makes_no_hip_call():
    assert call("fsdp_block_norm", norm(tokens=0)) == 0
    assert call("fsdp_block_distill", Distill(tokens=0, vocab=5, top=1, temperature=1)) == 0
    # column slices of one buffer may interleave: refused later for its workspace or by HIP, not as an overlap
    assert call("fsdp_block_norm", norm(tokens=0, x_stride=128, h=at(0) + 2 * 64, h_stride=128)) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError, match="device tensor"):
        fw.block_norm(x, y=torch.empty_like(x))
    with pytest.raises(ValueError, match="device tensor"):
        fw.linear(x, x, torch.empty(4, 4))
    with pytest.raises(ValueError, match="device tensor"):
        fw.distill_loss(x, x, x.int(), torch.empty(4))
    with pytest.raises(ValueError, match="activation"):
        fw.linear(x, x, torch.empty(4, 4), activation="tanh")
