"""The gated feed-forward and its gradient, and a linear layer's gradient from 8
bits, against the formulas in 64 bits, at the sizes, types, strides and values
where they can go wrong."""

from __future__ import annotations

import math

import pytest
import torch

import test_gpu_block_linear as L
from block_util import DTYPES, E32, Mat, blank, close, normal
from paper_2411_00284_amd import (Checkpoint, FsdpError, checkpoint_restore, checkpoint_save, gated_linear, gated_linear_backward,
                                  linear_backward)
from step_shapes import FORWARD, GRADIENT, ROWS
from step_util import Saved, gated, gated_gradient, near_saved

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def run_forward(m, n, k, dtype, act, kept, gap=0, shift=0):
    x, gw, uw = (normal(s, *shape, dtype=dtype, scale=c) for s, shape, c in ((1, (m, k), 1.0), (2, (n, k), k ** -0.5), (3, (n, k), k ** -0.5)))
    out, keep = blank(m, n, dtype, gap, shift), {}
    if kept == "type":
        keep = {q: blank(m, n, dtype, gap, shift) for q in ("gate", "up")}
        args = {q: v.t for q, v in keep.items()}
    elif kept == "8bit":
        keep = {q: Saved(rows=m, cols=n, gap=gap, shift=shift) for q in ("gate", "up")}
        args = {q: v.c for q, v in keep.items()}
    else:
        args = {}
    gated_linear(Mat(x, gap, shift).t, Mat(gw, gap, shift).t, Mat(uw, 2 * gap, shift).t, out.t, activation=act, **args)
    g, eg, u, eu, want, eo = gated(x, gw, uw, act)
    close(out.t, want, eo, "out")
    assert out.intact()
    for q, z, e in (("gate", g, eg), ("up", u, eu)):
        if kept == "type":
            close(keep[q].t, z, e, q)
        elif kept == "8bit":
            near_saved(keep[q], z, e, q)
        assert not kept or keep[q].intact()


@pytest.mark.parametrize("dtype,shape", FORWARD, ids=str)
def test_forward_forms(dtype, shape):
    for kept in ("8bit", "type"):
        print("gated form", dtype, shape, kept, flush=True)
        run_forward(*shape, DTYPES[dtype], "silu", kept)


@pytest.mark.parametrize("dtype,m,n,k", ROWS, ids=str)
def test_rows(dtype, m, n, k):
    for kept in (None, "type", "8bit"):
        print("gated rows", dtype, m, n, k, kept, flush=True)
        run_forward(m, n, k, DTYPES[dtype], "gelu", kept)


# m, n, k, type, activation, kept, gap, shift
FORWARD_EDGES = [
    (1, 1, 1, "bf16", None, "type", 0, 0),
    (1, 4096, 256, "bf16", "silu", None, 0, 0),
    (2, 333, 1001, "f16", "gelu", "type", 3, 1),
    (3, 31, 72, "f32", "relu", "8bit", 1, 1),
    (5, 33, 72, "f32", "gelu_tanh", "8bit", 0, 0),
    (5, 1, 8, "bf16", "silu", "8bit", 0, 0),
    (15, 257, 688, "f16", "relu", "8bit", 8, 8),
    (17, 129, 2050, "bf16", None, "8bit", 2, 0),
    (64, 64, 64, "bf16", "silu", "type", 0, 0),
    (77, 511, 123, "f32", "silu", "type", 1, 1),
    (128, 65, 1, "bf16", "silu", "8bit", 0, 0),
    (257, 769, 1000, "bf16", "gelu", "8bit", 8, 0),
    (513, 1025, 584, "f16", "gelu_tanh", "type", 8, 8),
    (1025, 2047, 72, "bf16", "relu", "8bit", 1, 0),
    (2056, 136, 8200, "f16", None, "type", 0, 8),
    (1020, 9220, 520, "bf16", "silu", "8bit", 0, 0),
]


@pytest.mark.parametrize("case", FORWARD_EDGES, ids=str)
def test_forward(case):
    m, n, k, dtype, act, kept, gap, shift = case
    print("gated", case, flush=True)
    run_forward(m, n, k, DTYPES[dtype], act, kept, gap, shift)


def run_gradient(m, n, k, dtype, act, saved, saved_x, gap=0, shift=0, only=None):
    x, gw, uw = (normal(s, *shape, dtype=dtype, scale=c) for s, shape, c in ((1, (m, k), 1.0), (2, (n, k), n ** -0.5), (3, (n, k), n ** -0.5)))
    dout, gate, up = normal(4, m, n, dtype=dtype), normal(5, m, n, dtype=dtype, scale=1.5), normal(6, m, n, dtype=dtype)
    put = lambda v: Mat(v, gap, shift).t  # noqa: E731
    args, values = {}, {}
    for q, v, s in (("x", x, saved_x), ("gate", gate, saved), ("up", up, saved)):
        if s:
            held = Saved(v, gap=gap, shift=shift)
            args[q], values[q] = held.c, held.values()
        else:
            args[q], values[q] = put(v), v
    shapes = {"out": (m, n), "dx": (m, k), "dgate_weight": (n, k), "dup_weight": (n, k)}
    got = {q: blank(*s, dtype, gap, shift) for q, s in shapes.items() if only is None or q in only}
    gated_linear_backward(put(dout), args["x"], put(gw), put(uw), args["gate"], args["up"], activation=act,
                          **{q: v.t for q, v in got.items()})
    want, bound = gated_gradient(dout, values["x"], gw, uw, values["gate"], values["up"], act)
    for q, v in got.items():
        close(v.t, want[q], bound[q], q)
        assert v.intact()


@pytest.mark.parametrize("dtype,shape", GRADIENT, ids=str)
def test_gradient_forms(dtype, shape):
    print("gated gradient form", dtype, shape, flush=True)
    run_gradient(*shape, DTYPES[dtype], "silu", True, True)


# m, n, k, type, activation, gate and up in 8 bits, x too, gap, shift
GRADIENT_EDGES = [
    (1, 1, 1, "bf16", None, False, False, 0, 0),
    (1, 688, 256, "bf16", "silu", True, True, 0, 0),
    (3, 129, 131, "f16", "gelu", False, True, 1, 1),
    (16, 64, 520, "f32", "gelu_tanh", False, False, 0, 0),
    (31, 1000, 72, "bf16", None, True, False, 8, 0),
    (64, 256, 688, "bf16", "relu", False, False, 0, 0),
    (130, 255, 257, "bf16", "silu", True, True, 0, 0),
    (256, 512, 256, "f16", "silu", False, False, 0, 0),
    (300, 1032, 328, "bf16", "gelu", True, True, 8, 8),
    (777, 301, 503, "f32", "silu", True, True, 3, 1),
    (1000, 688, 256, "f32", "gelu", False, False, 4, 4),
    (513, 33, 1024, "f16", "relu", True, False, 0, 0),
    (4100, 72, 96, "bf16", "gelu_tanh", False, True, 0, 0),
]


@pytest.mark.parametrize("case", GRADIENT_EDGES, ids=str)
def test_gradient(case):
    m, n, k, dtype, act, saved, saved_x, gap, shift = case
    print("gated gradient", case, flush=True)
    run_gradient(m, n, k, DTYPES[dtype], act, saved, saved_x, gap, shift)


@pytest.mark.parametrize("only", [("out",), ("dx",), ("dgate_weight", "dup_weight"), ("out", "dgate_weight", "dup_weight")], ids=str)
def test_outputs_alone(only):
    run_gradient(90, 264, 136, torch.bfloat16, "silu", True, True, only=only)


# m, n, k, type, activation, x in 8 bits, pre in 8 bits, times, bias, gap, shift
LINEAR = [
    (1, 1, 1, "bf16", None, True, False, False, True, 0, 0),
    (1, 688, 256, "bf16", "silu", True, True, True, True, 0, 0),
    (3, 129, 131, "f16", "gelu", True, False, True, True, 1, 1),
    (16, 64, 520, "f32", "gelu_tanh", False, True, False, True, 0, 0),
    (31, 1000, 72, "bf16", None, True, False, True, False, 8, 0),
    (130, 255, 257, "bf16", None, True, False, False, True, 0, 0),
    (130, 256, 257, "f16", None, True, False, False, False, 0, 0),
    (300, 1032, 328, "bf16", "gelu", False, True, False, True, 8, 8),
    (777, 301, 503, "f32", "silu", True, True, True, True, 3, 1),
    (1025, 2056, 264, "bf16", "gelu_tanh", True, True, True, True, 0, 0),
    (776, 72, 1287, "f16", "silu", True, True, True, True, 1, 0),
    (3000, 33, 40, "bf16", "relu", True, True, False, True, 0, 0),
    (1000, 688, 256, "f32", "gelu", True, True, False, True, 4, 4),
]


@pytest.mark.parametrize("case", LINEAR, ids=str)
def test_linear_from_8_bits(case):
    m, n, k, dtype, act, saved_x, saved_pre, has_times, has_bias, gap, shift = case
    dtype = DTYPES[dtype]
    print("linear gradient from 8 bits", case, flush=True)
    x, w = normal(1, m, k, dtype=dtype), normal(2, n, k, dtype=dtype, scale=n ** -0.5)
    dout, times = normal(3, m, n, dtype=dtype), normal(4, m, n, dtype=dtype) if has_times else None
    pre = normal(5, m, n, dtype=dtype, scale=1.5) if act or has_times else None
    put = lambda v: None if v is None else Mat(v, gap, shift).t  # noqa: E731
    held_x, held_pre = Saved(x, gap=gap, shift=shift), None if pre is None else Saved(pre, gap=gap, shift=shift)
    got = {"dx": blank(m, k, dtype, gap, shift), "dweight": blank(n, k, dtype, gap, shift)}
    if has_bias:
        got["dbias"] = blank(None, n, dtype, 0, shift)
    if has_times:
        got["dtimes"] = blank(m, n, dtype, gap, shift)
    linear_backward(put(dout), held_x.c if saved_x else put(x), put(w), activation=act, pre=held_pre.c if saved_pre else put(pre),
                    times=put(times), **{q: v.t for q, v in got.items()})
    # What 8 bits stand for is a value of the type.
    want, bound = L.gradient(dout, held_x.values().to(dtype) if saved_x else x, w, act, held_pre.values().to(dtype) if saved_pre else pre, times)
    for q, v in got.items():
        close(v.t, want[q], bound[q], q)
        assert v.intact()


def test_places():
    """out in dout's place; column slices of one buffer; each output alone: the same bits."""
    m, n, k = 70, 328, 256
    x, gw, uw = (normal(s, *shape, dtype=torch.bfloat16, scale=0.3).cuda() for s, shape in ((1, (m, k)), (2, (n, k)), (3, (n, k))))
    dout = normal(4, m, n, dtype=torch.bfloat16).cuda()
    out, gate, up = (torch.empty(m, n, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    gated_linear(x, gw, uw, out, gate=gate, up=up)
    wide = torch.empty(m, 3 * n, dtype=torch.bfloat16, device="cuda")
    both = torch.cat([gw, uw], 1)                                   # the weights as slices of one matrix
    gated_linear(x, both[:, :k], both[:, k:], wide[:, :n], gate=wide[:, n:2 * n], up=wide[:, 2 * n:])
    assert torch.equal(wide, torch.cat([out, gate, up], 1))
    stacked = torch.cat([gw, uw])                                   # and one after the other
    gated_linear(x, stacked[:n], stacked[n:], wide[:, :n])
    assert torch.equal(wide[:, :n], out)
    shapes = {"out": (m, n), "dx": (m, k), "dgate_weight": (n, k), "dup_weight": (n, k)}
    whole = {q: torch.empty(s, dtype=torch.bfloat16, device="cuda") for q, s in shapes.items()}
    gated_linear_backward(dout, x, gw, uw, gate, up, **whole)
    for q in ("out", "dx"):
        alone = torch.empty(shapes[q], dtype=torch.bfloat16, device="cuda")
        gated_linear_backward(dout, x, gw, uw, gate, up, **{q: alone})
        assert torch.equal(alone, whole[q]), q
    place, dx = dout.clone(), torch.empty_like(x)
    gated_linear_backward(place, x, gw, uw, gate, up, out=place, dx=dx)
    assert torch.equal(place, whole["out"]) and torch.equal(dx, whole["dx"])
    gated_linear_backward(dout, x, both[:, :k], both[:, k:], gate, up, dx=dx)
    assert torch.equal(dx, whole["dx"])
    d = torch.empty(2 * n, k, dtype=torch.bfloat16, device="cuda")
    gated_linear_backward(dout, x, gw, uw, gate, up, dgate_weight=d[:n], dup_weight=d[n:])
    assert torch.equal(d, torch.cat([whole["dgate_weight"], whole["dup_weight"]]))
    gated_linear_backward(dout, x, gw, uw, gate, up)                # nothing is wanted: nothing is done


def test_weights_apart():
    """Weights of two row strides, one of them off the 16-byte grid."""
    m, n, k = 130, 72, 264
    x, gw, uw = (normal(s, *shape, dtype=torch.float16) for s, shape in ((1, (m, k)), (2, (n, k)), (3, (n, k))))
    dout, gate, up = (normal(s, m, n, dtype=torch.float16).cuda() for s in (4, 5, 6))
    wants = None
    for a, b in (((0, 0), (0, 0)), ((8, 0), (16, 0)), ((0, 0), (3, 1)), ((5, 1), (8, 0))):
        out, dx = blank(m, n, torch.float16), blank(m, k, torch.float16)
        g, u = Mat(gw, *a).t, Mat(uw, *b).t
        gated_linear(x.cuda(), g, u, out.t)
        gated_linear_backward(dout, x.cuda(), g, u, gate, up, dx=dx.t)
        got = (out.t.clone(), dx.t.clone())
        wants = wants or got
        assert all(torch.equal(p, q) for p, q in zip(got, wants)), (a, b)


def test_values():
    """A NaN or an infinity stays in its row or column, and in its group of 8
    bits; memory beside a matrix is not read into the sums."""
    m, n, k = 300, 260, 264
    x, gw, uw = normal(1, m, k, dtype=torch.bfloat16), normal(2, n, k, dtype=torch.bfloat16), normal(3, n, k, dtype=torch.bfloat16)
    x[1, 7], gw[5, 3], uw[40, 2] = math.nan, math.inf, -math.inf
    for rows in (3, m):
        out, keep = blank(rows, n, torch.bfloat16, 16), [Saved(rows=rows, cols=n, gap=4) for _ in range(2)]
        gated_linear(Mat(x[:rows], 8).t, Mat(gw, 24).t, Mat(uw, 40).t, out.t, gate=keep[0].c, up=keep[1].c)
        g, eg, u, eu, want, eo = gated(x[:rows], gw, uw, "silu")
        others = [i for i in range(rows) if i != 1]
        columns = [j for j in range(n) if j not in (5, 40)]
        got = out.t.cpu()
        assert bool(got[1].isnan().all())
        close(got[others][:, columns], want[others][:, columns], eo[others][:, columns], "the others")
        assert not got[others][:, 40].isfinite().any()
        for held, bad in zip(keep, (0, 1)):
            scales = held.scales.t.cpu()
            assert bool((scales[1] == 255).all()) and bool((scales[others][:, bad] == 255).all())
            assert not (scales[others][:, [j for j in range(9) if j != bad]] == 255).any()
        assert out.intact() and keep[0].intact() and keep[1].intact()


def test_a_nan_of_8_bits_reaches_its_gradients():
    m, n, k = 20, 96, 64
    gate, up, x = normal(1, m, n), normal(2, m, n), normal(3, m, k)
    gate[4, 50] = math.nan
    gw, uw, dout = (normal(s, *shape).cuda() for s, shape in ((4, (n, k)), (5, (n, k)), (6, (m, n))))
    out, dx, dg, du = torch.empty(m, n, device="cuda"), torch.empty(m, k, device="cuda"), torch.empty(n, k, device="cuda"), torch.empty(n, k, device="cuda")
    gated_linear_backward(dout, x.cuda(), gw, uw, Saved(gate).c, Saved(up).c, out=out, dx=dx, dgate_weight=dg, dup_weight=du)
    assert torch.equal(out.isnan().any(1).cpu(), torch.arange(m) == 4) and torch.equal(dx.isnan().all(1).cpu(), torch.arange(m) == 4)
    group = (torch.arange(n) // 32 == 1)
    assert torch.equal(dg.isnan().any(1).cpu(), group) and torch.equal(du.isnan().any(1).cpu(), group)


def test_empty():
    for dtype in (torch.bfloat16, torch.float32):
        def new(*shape):
            return torch.full(shape, 7, dtype=dtype, device="cuda")
        w = new(32, 64)
        gated_linear(new(0, 64), w, w.clone(), new(0, 32), gate=Checkpoint.empty(0, 32), up=Checkpoint.empty(0, 32))
        dg, du = new(32, 64), new(32, 64)
        gated_linear_backward(new(0, 32), new(0, 64), w, w.clone(), new(0, 32), new(0, 32), out=new(0, 32), dx=new(0, 64),
                              dgate_weight=dg, dup_weight=du)
        assert not dg.any() and not du.any()
        dw = new(32, 64)
        linear_backward(new(0, 32), Checkpoint.empty(0, 64), w, dx=new(0, 64), dweight=dw, dbias=(db := new(32)))
        assert not dw.any() and not db.any()
        dx = new(9, 64)
        gated_linear(new(9, 64), new(0, 64), new(0, 64), new(9, 0))
        gated_linear_backward(new(9, 0), new(9, 64), new(0, 64), new(0, 64), new(9, 0), new(9, 0), dx=dx, dgate_weight=new(0, 64),
                              dup_weight=new(0, 64))
        assert not dx.any()
        dx.fill_(7)
        linear_backward(new(9, 0), Checkpoint.empty(9, 64), new(0, 64), dx=dx, dweight=new(0, 64))
        assert not dx.any()


def test_differences():
    """The gradient against central differences of the forward kernel, in
    float32: off by step^2 / 6 third derivatives and by rounding over the step."""
    m, n, k, step = 5, 12, 40, 1e-2
    v = {"x": normal(1, m, k), "gate_weight": normal(2, n, k, scale=0.3), "up_weight": normal(3, n, k, scale=0.3)}
    cot = normal(5, m, n)
    for act in (None, "silu", "gelu", "gelu_tanh"):
        def run(a):
            out, g, u = (torch.empty(m, n, device="cuda") for _ in range(3))
            gated_linear(a["x"].cuda(), a["gate_weight"].cuda(), a["up_weight"].cuda(), out, activation=act, gate=g, up=u)
            return (out.cpu().double() * cot).sum().item(), g, u
        _, g, u = run(v)
        got = {"x": torch.empty(m, k, device="cuda"), "gate_weight": torch.empty(n, k, device="cuda"),
               "up_weight": torch.empty(n, k, device="cuda")}
        gated_linear_backward(cot.cuda(), v["x"].cuda(), v["gate_weight"].cuda(), v["up_weight"].cuda(), g, u, activation=act,
                              dx=got["x"], dgate_weight=got["gate_weight"], dup_weight=got["up_weight"])
        size = math.sqrt(m * n)
        for i, q in enumerate(v):
            d = normal(30 + i, *v[q].shape)
            d = d / d.norm()
            slope = (got[q].cpu().double() * d).sum().item()
            diff = (run({**v, q: v[q] + step * d})[0] - run({**v, q: v[q] - step * d})[0]) / (2 * step)
            # a step moves g and u by at most 7 times it; the third derivative of act(g) u is at most 2 |u| + 3 * 1.2, |u| below 8
            assert abs(diff - slope) <= 20 * 7 ** 3 * size * step * step / 6 + 400 * E32 * size / step, (act, q)


def test_repeats_and_streams():
    """The same call gives the same bits, on another stream too."""
    m, n, k = 130, 4104, 1032
    x, gw, uw = (normal(s, *shape, dtype=torch.bfloat16).cuda() for s, shape in ((1, (m, k)), (2, (n, k)), (3, (n, k))))
    dout = normal(4, m, n, dtype=torch.bfloat16).cuda()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def run(stream):
        new = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        out, one, dx, dg, du = new(m, n), new(1, n), new(m, k), new(n, k), new(n, k)
        kept, saved_x = [Checkpoint.empty(m, n) for _ in range(2)], Checkpoint.empty(m, k)
        torch.cuda.synchronize()
        gated_linear(x, gw, uw, out, gate=kept[0], up=kept[1], stream=stream)
        gated_linear(x[:1], gw, uw, one, stream=stream)
        checkpoint_save(x, saved_x, stream=stream)
        gated_linear_backward(dout, saved_x, gw, uw, *kept, dx=dx, dgate_weight=dg, dup_weight=du, stream=stream)
        torch.cuda.synchronize()
        return out, one, dx, dg, du, *kept[0], *kept[1]

    first = run(None)
    for stream in (None, side, side.cuda_stream):
        assert all(torch.equal(a, b) for a, b in zip(first, run(stream)))


def test_8_bits_as_their_values():
    """The gradient from 8 bits is that from the values they stand for, bit for
    bit: they are exact in the type."""
    m, n, k = 200, 264, 136
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        x, gate, up = (normal(s, m, c, dtype=dtype) for s, c in ((1, k), (2, n), (3, n)))
        gw, uw, dout = (normal(s, *shape, dtype=dtype).cuda() for s, shape in ((4, (n, k)), (5, (n, k)), (6, (m, n))))
        held = [Saved(v).c for v in (x, gate, up)]
        values = [torch.empty(v.shape, dtype=dtype, device="cuda") for v in (x, gate, up)]
        for h, v in zip(held, values):
            checkpoint_restore(h, v)
        got = []
        for xs, gs, us in (held, values):
            outs = {q: torch.empty(s, dtype=dtype, device="cuda")
                    for q, s in (("out", (m, n)), ("dx", (m, k)), ("dgate_weight", (n, k)), ("dup_weight", (n, k)))}
            gated_linear_backward(dout, xs, gw, uw, gs, us, activation="gelu", **outs)
            lin = {q: torch.empty(s, dtype=dtype, device="cuda") for q, s in (("dx", (m, k)), ("dweight", (n, k)), ("dbias", (n,)))}
            linear_backward(dout, xs, gw, activation="gelu", pre=gs, **lin)
            got.append([*outs.values(), *lin.values()])
        assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("m,n,k", [(4101, 2052, 520), (1976, 2186, 328)])
def test_rows_that_are_not_finite_stay_alone(m, n, k):
    """In tiles that lie in out whole and in those at its edges."""
    x, gw, uw = (normal(s, *shape).cuda() for s, shape in ((1, (m, k)), (2, (n, k)), (3, (n, k))))
    bad = [0, 17, 1000, m - 1]
    poisoned = x.clone()
    poisoned[bad, 5] = torch.tensor([float("inf"), float("nan"), -float("inf"), float("nan")], dtype=x.dtype, device="cuda")
    results = []
    for v in (x, poisoned):
        out, gate, up = torch.empty(m, n, dtype=x.dtype, device="cuda"), Checkpoint.empty(m, n), Checkpoint.empty(m, n)
        gated_linear(v, gw, uw, out, gate=gate, up=up)
        results.append((out, *gate, *up))
    good = torch.ones(m, dtype=torch.bool)
    good[bad] = False
    for clean, other in zip(*results):
        assert torch.equal(clean[good.cuda()], other[good.cuda()])
    for codes, scales in (results[1][1:3], results[1][3:5]):
        assert bool((scales[bad] == 255).all()) and bool((codes[bad] == 0).all())


def test_long_sums_in_fp32():
    """Sums over many terms go in runs of 512.  Of random terms the sum of i is sqrt(i / n) of that
    of n, and each addition off by at most 2^-24 of it: all additions of a run by 2^-24 sqrt(512 / 2),
    of R runs by as much of the whole, and their sum by 2^-24 sqrt(R / 2) more."""
    off = lambda got, want: float((got.double() - want).norm() / want.norm())  # noqa: E731
    bound = lambda terms: 2.0**-24 * (256 + (terms + 511) // 512 / 2 + 1) ** 0.5  # noqa: E731
    new = lambda s, *shape: normal(s, *shape, dtype=torch.float32).cuda()  # noqa: E731
    m, n, k = 1910, 1024, 7864
    x, gw, uw = new(1, m, k), new(2, n, k), new(3, n, k)
    out, gate, up = (torch.empty(m, n, device="cuda") for _ in range(3))
    gated_linear(x, gw, uw, out, activation="none", gate=gate, up=up)
    assert off(gate, x.double() @ gw.double().t()) <= bound(k)
    assert off(up, x.double() @ uw.double().t()) <= bound(k)
    m, n, k = 4096, 1024, 1024
    x, gw, uw, gate, up, dout = new(1, m, k), new(2, n, k), new(3, n, k), new(4, m, n), new(5, m, n), new(6, m, n)
    dx, dg, du = torch.empty_like(x), torch.empty_like(gw), torch.empty_like(uw)
    gated_linear_backward(dout, x, gw, uw, gate, up, activation="none", dx=dx, dgate_weight=dg, dup_weight=du)
    first, second = (dout * up).double(), (dout * gate).double()
    assert off(dg, first.t() @ x.double()) <= bound(m)
    assert off(du, second.t() @ x.double()) <= bound(m)
    assert off(dx, first @ gw.double() + second @ uw.double()) <= bound(2 * n)


@pytest.mark.parametrize("m,n,k", [(300, 1032, 328), (61, 250, 2100), (776, 72, 1287), (2100, 61, 125)])
def test_linear_in_fp32_has_its_bits(m, n, k):
    """A linear layer's gradient in fp32 goes in the same parts from 8 bits as from
    the values they stand for."""
    weight, dout = normal(1, n, k, dtype=torch.float32).cuda(), normal(2, m, n, dtype=torch.float32).cuda()
    held = [Saved(normal(s, m, c, dtype=torch.float32)).c for s, c in ((3, k), (4, n))]
    values = [torch.empty(h.codes.shape, device="cuda") for h in held]
    for h, v in zip(held, values):
        checkpoint_restore(h, v)
    got = []
    for x, pre in (held, values):
        outs = {q: torch.empty(s, device="cuda") for q, s in (("dx", (m, k)), ("dweight", (n, k)))}
        linear_backward(dout, x, weight, activation="silu", pre=pre, **outs)
        got.append(list(outs.values()))
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_refusals():
    new = lambda *s: torch.full(s, 3, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    x, gw, uw, out, gate, up = new(4, 64), new(32, 64), new(32, 64), new(4, 32), new(4, 32), new(4, 32)
    c, d = Checkpoint.empty(4, 32), Checkpoint.empty(4, 32)
    for error, args, more in [
        (ValueError, (x, gw[:, :63], uw, out), {}),
        (ValueError, (x, gw, uw[:31], out), {}),
        (ValueError, (x, gw, uw, out[:, :31]), {}),
        (TypeError, (x, gw, uw.half(), out), {}),
        (TypeError, (x.double(), gw, uw, out), {}),
        (TypeError, (x, gw, uw, None), {}),
        (ValueError, (x, gw, uw, out), {"activation": "swish"}),
        (ValueError, (x, gw, uw, out), {"gate": gate}),
        (TypeError, (x, gw, uw, out), {"gate": gate, "up": c}),
        (TypeError, (x, gw, uw, out), {"gate": gate.float(), "up": up.float()}),
        (ValueError, (x, gw, uw, out), {"gate": Checkpoint(c.codes, c.scales[:3]), "up": d}),
        (FsdpError, (x, gw, uw, out), {"gate": gate, "up": gate}),
        (FsdpError, (x, gw, uw, out), {"gate": out, "up": up}),
        (FsdpError, (x, gw, uw, out), {"gate": c, "up": c}),
        (FsdpError, (x, gw, uw, x[:, :32]), {}),
        (FsdpError, (x[:, :0], gw[:, :0], uw[:, :0], out), {}),
    ]:
        with pytest.raises(error):
            gated_linear(*args, **more)
    dx, dw, dv = new(4, 64), new(32, 64), new(32, 64)
    for error, args, more in [
        (ValueError, (out, x, gw, uw, gate, up), {"dgate_weight": dw}),
        (TypeError, (out, x, gw, uw, gate, None), {"dx": dx}),
        (TypeError, (out, x, gw, uw, gate, c), {"dx": dx}),
        (TypeError, (out, (x,), gw, uw, gate, up), {"dx": dx}),
        (ValueError, (out, c, gw, uw, gate, up), {"dx": dx}),
        (TypeError, (out, x, gw, uw, gate, up), {"dx": dx.float()}),
        (FsdpError, (out, x, gw, uw, gate, up), {"dgate_weight": dw, "dup_weight": dw}),
        (FsdpError, (out, x, gw, uw, gate, up), {"dx": x}),
        (FsdpError, (out, x, gw, uw, gate, up), {"out": gate}),
        (FsdpError, (out, x, gw, uw, out, up), {"out": out}),
    ]:
        with pytest.raises(error):
            gated_linear_backward(*args, **more)
    held = Checkpoint.empty(4, 64)
    for error, args, more in [
        (FsdpError, (out, held, gw), {"activation": "silu", "dx": dx}),
        (ValueError, (out, held, gw), {"dtimes": gate}),
        (ValueError, (out, held, gw), {"activation": "silu", "pre": held, "dx": dx}),
        (ValueError, (out, Checkpoint(held.codes, held.scales[:, :1]), gw), {"dweight": dw}),
        (TypeError, (out, held, gw.half()), {"dweight": dw}),
        (FsdpError, (out, held, gw), {"dx": gw[:4]}),
    ]:
        with pytest.raises(error):
            linear_backward(*args, **more)
    torch.cuda.synchronize()
    for t in (x, gw, uw, out, gate, up, dx, dw, dv):
        assert bool((t == 3).all())


def test_long_offsets():
    """Rows whose offsets pass 2^32 elements, in every operand that is read or
    written."""
    m, n, k, stride = 5, 3, 40, (1 << 31) + 4096
    raw = torch.empty((m - 1) * stride + 4096, dtype=torch.bfloat16, device="cuda")
    at = iter(range(0, 4096, 64))
    far = lambda rows, cols: raw.as_strided((rows, cols), (stride, 1), next(at))  # noqa: E731
    near = lambda rows, cols: torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    got = []
    for new in (far, near):
        x, gw, uw, dout = new(m, k), new(n, k), new(n, k), new(m, n)
        for i, t in enumerate((x, gw, uw, dout)):
            t.copy_(normal(i, *t.shape, dtype=torch.bfloat16))
        out, gate, up, one, again, dx, dg, du = new(m, n), new(m, n), new(m, n), new(1, n), new(m, n), new(m, k), new(n, k), new(n, k)
        gated_linear(x, gw, uw, out, gate=gate, up=up)
        gated_linear(x[4:], gw, uw, one)
        gated_linear_backward(dout, x, gw, uw, gate, up, out=again, dx=dx, dgate_weight=dg, dup_weight=du)
        got.append([t.contiguous() for t in (out, gate, up, one, again, dx, dg, du)])
    assert all(torch.equal(a, b) for a, b in zip(*got))
