"""Calls of fsdp_step.h with made-up addresses, for the host tests."""

from __future__ import annotations

import os
import re

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "fsdp_step.h")
BF16, F32, F16 = 0, 1, 2
CODE = {"bf16": BF16, "f16": F16, "f32": F32}
KIND = {"int64_t": "q", "int32_t": "i", "float": "f", "fsdp_dtype": "i", "fsdp_activation": "i"}
NAMES = ("save", "restore", "gated", "gated_grad", "linear_grad", "policy")


def header():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def fields_of(name):
    """(field, kind) of a struct of the header, in order."""
    body = re.search(r"typedef struct fsdp_step_%s_args \{(.*?)\}" % name, header(), re.S).group(1)
    out = []
    for line in body.split(";"):
        line = " ".join(line.split())
        if line:
            kind, names = re.match(r"((?:const )?\w+ ?\*?) ?(.*)", line).groups()
            for n in names.split(","):
                pointer = "*" in kind or "*" in n
                out.append((n.strip(" *"), "p" if pointer else KIND[kind.replace("const", "").strip()]))
    return out


FIELDS = {n: fields_of(n) for n in NAMES}


def call(name, function=None, **values):
    assert set(values) <= {f for f, _ in FIELDS[name]}, values
    return ["fsdp_step_" + (function or name), [(f, k, values.get(f, None if k == "p" else 0)) for f, k in FIELDS[name]]]


def at(k, shift=0):
    return (1 << 50) + (k << 46) + shift


def groups(cols):
    return -(-cols // 32)


def save(rows, cols, dtype=BF16):
    return call("save", rows=rows, cols=cols, dtype=dtype, x=at(0), codes=at(1), scales=at(2), x_stride=cols, codes_stride=cols,
                scales_stride=groups(cols))


def restore(rows, cols, dtype=BF16):
    return call("restore", rows=rows, cols=cols, dtype=dtype, x=at(0), codes=at(1), scales=at(2), x_stride=cols, codes_stride=cols,
                scales_stride=groups(cols))


def kept_args(m, n, saved):
    got = dict(gate=at(4), up=at(5), gate_stride=n, up_stride=n)
    return got | dict(gate_scales=at(6), up_scales=at(7), gate_scales_stride=groups(n), up_scales_stride=groups(n)) if saved else got


def gated(m, n, k, dtype=BF16, kept=None, shift=0):
    """``kept``: None, "type" or "8bit"."""
    more = kept_args(m, n, kept == "8bit") if kept else {}
    return call("gated", m=m, n=n, k=k, dtype=dtype, activation=2, x=at(0, shift), gate_weight=at(1), up_weight=at(2), out=at(3),
                x_stride=k, gate_weight_stride=k, up_weight_stride=k, out_stride=n, **more)


def gated_grad(m, n, k, dtype=BF16, saved=False, saved_x=False, outs=("out", "dx", "dgate_weight", "dup_weight")):
    strides = dict(dout_stride=n, x_stride=k, gate_weight_stride=k, up_weight_stride=k, out_stride=n, dx_stride=k,
                   dgate_weight_stride=k, dup_weight_stride=k)
    more = dict(x_scales=at(12), x_scales_stride=groups(k)) if saved_x else {}
    return call("gated_grad", m=m, n=n, k=k, dtype=dtype, activation=2, dout=at(0), x=at(1), gate_weight=at(2), up_weight=at(3),
                **kept_args(m, n, saved), **strides, **more, **{o: at(8 + i) for i, o in enumerate(outs)})


def linear_grad(m, n, k, dtype=BF16, act=0, saved=True, saved_x=True, outs=("dx", "dweight")):
    strides = dict(dout_stride=n, x_stride=k, weight_stride=k, pre_stride=n, dx_stride=k, dweight_stride=k)
    more = dict(x_scales=at(12), x_scales_stride=groups(k)) if saved_x else {}
    if act:
        more |= dict(pre=at(3)) | (dict(pre_scales=at(13), pre_scales_stride=groups(n)) if saved else {})
    return call("linear_grad", m=m, n=n, k=k, dtype=dtype, activation=act, dout=at(0), x=at(1), weight=at(2), **strides, **more,
                **{o: at(8 + i) for i, o in enumerate(outs)})


def policy(tokens, vocab, dtype=BF16, grad=False, backward=False):
    outs = dict(dloss=at(4), dlogits=at(5), dlogits_stride=vocab) if grad else {}
    outs |= dict(lse=at(6)) if backward else dict(loss=at(7))
    return call("policy", "policy_grad" if backward else "policy", tokens=tokens, vocab=vocab, dtype=dtype, clip_low=0.2,
                clip_high=0.2, temperature=1.0, logits=at(0), actions=at(1), old_logp=at(2), advantages=at(3), logits_stride=vocab,
                **outs)
