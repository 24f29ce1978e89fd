"""Every kernel of the block operators against the formulas in 64 bits: each
combination of types in each form, at the shapes of block_shapes.py."""

from __future__ import annotations

import pytest
import torch

import test_gpu_block_distill as D
import test_gpu_block_linear as L
import test_gpu_block_norm as N
from block_shapes import DISTILLS, NORM_TOKENS, NORMS, PRODUCTS, ROWS, linear_sizes
from block_util import DTYPES, Mat, blank, close, normal
from paper_2411_00284_amd import block_norm, distill_loss, distill_loss_backward, linear, linear_backward

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


@pytest.mark.parametrize("types,hidden", NORMS, ids=str)
def test_norm(types, hidden):
    print("norm form", types, hidden, flush=True)
    block, stream, weights = (DTYPES[t] for t in types)
    t = NORM_TOKENS
    x, b = normal(1, t, hidden, dtype=stream, scale=3), normal(2, t, hidden, dtype=block)
    pre, post, gate = normal(3, hidden, dtype=weights, shift=1), normal(4, hidden, dtype=weights, shift=1), normal(5, 3, hidden, dtype=block)
    y, h = blank(t, hidden, stream), blank(t, hidden, block)
    block_norm(x.cuda(), branch=b.cuda(), pre_weight=pre.cuda(), post_weight=post.cuda(), gate=gate.cuda(), y=y.t, h=h.t,
               residual_scale=0.75, branch_scale=1.25, eps=N.EPS)
    wy, wh, ey, eh = N.forward(x, b, post, gate, pre, 0.75, 1.25)
    close(y.t, wy, ey, "y")
    close(h.t, wh, eh, "h")
    assert y.intact() and h.intact()
    dy, dh = normal(6, t, hidden, dtype=stream), normal(7, t, hidden, dtype=block)
    got = N.run_gradient(x, dy, dh, b, post, gate, pre, 0.75, 1.25)
    want, bound = N.gradient(x, dy, dh, b, post, gate, pre, 0.75, 1.25)
    for k in want:
        close(got[k].reshape(want[k].shape), want[k], bound[k], k)


def forward(m, n, k, dtype, act):
    x, w = normal(1, m, k, dtype=dtype), normal(2, n, k, dtype=dtype, scale=k ** -0.5)
    bias, times, residual = normal(3, n, dtype=dtype), normal(4, m, n, dtype=dtype), normal(5, m, n, dtype=dtype)
    out, pre = blank(m, n, dtype), blank(m, n, dtype)
    linear(x.cuda(), w.cuda(), out.t, bias=bias.cuda(), activation=act, times=times.cuda(), residual=residual.cuda(), pre=pre.t)
    z, ez, want, eo = L.forward(x, w, bias, act, times, residual)
    close(out.t, want, eo, "out")
    close(pre.t, z, ez, "pre")
    assert out.intact() and pre.intact()


@pytest.mark.parametrize("dtype,kind,shape", PRODUCTS, ids=str)
def test_product(dtype, kind, shape):
    print("product form", dtype, kind, shape, flush=True)
    dtype = DTYPES[dtype]
    m, n, k = linear_sizes(kind, shape)
    if kind == "forward":
        return forward(m, n, k, dtype, "gelu")
    x, w = normal(1, m, k, dtype=dtype), normal(2, n, k, dtype=dtype, scale=n ** -0.5)
    dout, times, pre = normal(3, m, n, dtype=dtype), normal(4, m, n, dtype=dtype), normal(5, m, n, dtype=dtype, scale=1.5)
    got = {kind: blank(*((m, k) if kind == "dx" else (n, k)), dtype), "dbias": blank(None, n, dtype), "dtimes": blank(m, n, dtype)}
    linear_backward(dout.cuda(), x.cuda(), w.cuda(), activation="silu", pre=pre.cuda(), times=times.cuda(),
                    **{q: v.t for q, v in got.items()})
    want, bound = L.gradient(dout, x, w, "silu", pre, times)
    for q, v in got.items():
        close(v.t, want[q], bound[q], q)
        assert v.intact()


@pytest.mark.parametrize("dtype,m,n,k", ROWS, ids=str)
def test_rows(dtype, m, n, k):
    print("rows form", dtype, m, n, k, flush=True)
    forward(m, n, k, DTYPES[dtype], "silu")


@pytest.mark.parametrize("case", DISTILLS, ids=str)
def test_distill(case):
    print("distill form", case, flush=True)
    dtype, tokens, vocab, top = case
    dtype = DTYPES[dtype]
    tau = 1.5
    logits, values, ids, _ = D.make(11, tokens, vocab, top, dtype, torch.float32)
    ids[1, 3:], ids[2] = -1, -1
    ids[3, 1] = ids[3, 0]
    dloss = normal(13, tokens)
    gl, gt, gi, gd = Mat(logits).t, values.cuda(), ids.cuda(), dloss.cuda()
    loss, lse, alone = (blank(None, tokens, torch.float32) for _ in range(3))
    dl, back = blank(tokens, vocab, dtype), blank(tokens, vocab, dtype)
    distill_loss(gl, gt, gi, loss.t, lse.t, temperature=tau, dloss=gd, dlogits=dl.t)
    distill_loss(gl, gt, gi, alone.t, temperature=tau)
    distill_loss_backward(gd, gl, gt, gi, lse.t, back.t, temperature=tau)
    wl, we, wg, el, ee, eg = D.reference(logits, values, ids, tau, None, dloss)
    close(loss.t, wl, el, "loss")
    close(alone.t, wl, el, "loss alone")
    close(lse.t, we, ee, "lse")
    close(dl.t, wg, eg, "dlogits")
    _, _, wg, _, _, eg = D.reference(logits, values, ids, tau, None, dloss, lse.t.cpu())
    close(back.t, wg, eg, "dlogits from lse")
    assert all(v.intact() for v in (loss, lse, alone, dl, back))
