"""The step's operators as a program runs them: the example's step against
autograd, captured into a graph, from several threads on streams of their own,
and without memory for a workspace."""

from __future__ import annotations

import importlib.util
import math
import os
import threading

import pytest
import torch

from block_util import normal
from paper_2411_00284_amd import (Checkpoint, block_norm, checkpoint_restore, checkpoint_save, gated_linear, gated_linear_backward, linear,
                                  linear_backward, policy_loss, policy_loss_backward)

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Layer:
    """The operators forward and backward, at sizes that take workspaces
    (operands off the grid, parts of k, column sums)."""

    def __init__(self, seed, tokens=70, hidden=515, wide=1201, dtype=torch.bfloat16):
        def put(i, *shape, **kw):
            return normal(100 * seed + i, *shape, dtype=dtype, **kw).cuda()

        self.x, self.norm = put(1, tokens, hidden), put(2, hidden, shift=1)
        self.gate, self.up, self.down = (put(i, *s, scale=hidden ** -0.5) for i, s in ((3, (wide, hidden)), (4, (wide, hidden)), (5, (hidden, wide))))
        g = torch.Generator().manual_seed(seed)
        self.actions = torch.randint(0, hidden, (tokens,), generator=g).cuda()
        self.actions[::7] = -1
        self.old, self.adv, self.ref = (torch.randn(tokens, generator=g).sub(s).cuda() for s in (6.0, 0.0, 6.0))
        self.weight = torch.full((tokens,), 1 / tokens, device="cuda")
        like, t = torch.empty_like, self.x.new_empty(tokens, wide)
        self.saved = {"h": Checkpoint.empty(tokens, hidden), "gate": Checkpoint.empty(tokens, wide), "up": Checkpoint.empty(tokens, wide)}
        self.out = {"h": like(self.x), "act": like(t), "one": t.new_empty(1, wide), "logits": like(self.x), "loss": like(self.weight),
                    "logp": like(self.weight), "lse": like(self.weight), "dlogits": like(self.x), "again": like(self.x), "dact": like(t),
                    "ddown": like(self.down), "dh": like(self.x), "dgate": like(self.gate), "dup": like(self.up), "back": like(self.x),
                    "dx": like(self.x), "dw": like(self.gate)}
        self.out |= {f"{k}.{n}": v for k, c in self.saved.items() for n, v in zip(c._fields, c)}

    def run(self, stream=None):
        o, c, s = self.out, self.saved, dict(stream=stream)
        opt = dict(ref_logp=self.ref, kl_weight=0.05, temperature=0.9)
        block_norm(self.x, pre_weight=self.norm, h=o["h"], **s)
        checkpoint_save(o["h"], c["h"], **s)
        gated_linear(o["h"], self.gate, self.up, o["act"], gate=c["gate"], up=c["up"], **s)
        gated_linear(o["h"][:1], self.gate, self.up, o["one"], activation="gelu", **s)
        linear(o["act"], self.down, o["logits"], **s)
        policy_loss(o["logits"], self.actions, self.old, self.adv, o["loss"], o["logp"], o["lse"], dloss=self.weight,
                    dlogits=o["dlogits"], **opt, **s)
        policy_loss_backward(self.weight, o["logits"], self.actions, self.old, self.adv, o["lse"], o["again"], **opt, **s)
        linear_backward(o["dlogits"], o["act"], self.down, dx=o["dact"], dweight=o["ddown"], **s)
        linear_backward(o["dact"], c["h"], self.gate, activation="gelu", pre=c["gate"], dx=o["dx"], dweight=o["dw"], **s)
        gated_linear_backward(o["dact"], c["h"], self.gate, self.up, c["gate"], c["up"], out=o["dact"], dx=o["dh"],
                              dgate_weight=o["dgate"], dup_weight=o["dup"], **s)
        checkpoint_restore(c["h"], o["back"], **s)

    def poison(self):
        for v in self.out.values():
            v.view(torch.uint8).fill_(0xFF)

    def same(self, want):
        return [k for k, v in self.out.items() if not torch.equal(v.view(torch.uint8), want[k].view(torch.uint8))]


def eager(layer):
    layer.run()
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in layer.out.items()}
    assert all(bool(v.isfinite().all()) for v in want.values())
    return want


def captured(layer):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run()
    torch.cuda.synchronize()
    return graph


def test_replayed_from_graphs():
    """Two graphs, whose workspaces come from pools of their own, replayed in
    turn with eager work between them."""
    layers = [Layer(1), Layer(2, tokens=90)]
    wants = [eager(layer) for layer in layers]
    print("step operators: capture", flush=True)
    graphs = [captured(layer) for layer in layers]
    for rep in range(4):
        for i in (0, 1):
            layers[i].poison()
            junk = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(4)]
            torch.cuda.synchronize()
            print("step operators: replay", rep, i, flush=True)
            graphs[i].replay()
            layers[1 - i].run()
            torch.cuda.synchronize()
            assert not layers[i].same(wants[i]) and not layers[1 - i].same(wants[1 - i]), (rep, i)
            del junk


def test_threads_and_streams():
    """Each thread its own stream and buffers; the workspaces come from one
    allocator."""
    layers = [Layer(3 + i, tokens=64 + 10 * i) for i in range(4)]
    wants = [eager(layer) for layer in layers]
    for layer in layers:
        layer.poison()
    torch.cuda.synchronize()
    errors = []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            for rep in range(20):
                if rep % 2:
                    with torch.cuda.stream(stream):
                        layers[i].run()
                else:
                    layers[i].run(stream)
            stream.synchronize()
            if layers[i].same(wants[i]):
                errors.append((i, layers[i].same(wants[i])))
        except Exception as e:  # noqa: BLE001
            errors.append((i, repr(e)))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not errors and not any(t.is_alive() for t in threads), errors


def test_out_of_memory():
    """torch's own error, before anything is enqueued."""
    m = 4096
    new = lambda *s: torch.full(s, 3.0, dtype=torch.float16, device="cuda")  # noqa: E731
    x, w, out, dx, dw = new(m, 2501), new(m, 2501), new(m, m), new(m, 2501), new(m, 2501)
    held = Checkpoint.empty(m, 2501)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    torch.cuda.set_per_process_memory_fraction(0.0)
    try:
        with pytest.raises(torch.OutOfMemoryError):
            gated_linear(x, w, w, out)
        with pytest.raises(torch.OutOfMemoryError):
            gated_linear_backward(out, x, w, w, out, out, dx=dx)
        with pytest.raises(torch.OutOfMemoryError):
            linear_backward(out, held, w, dweight=dw)
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert all(bool((v == 3).all()) for v in (out, dx, dw))


# ------------------------------------------------------------------ the example


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("policy_step", os.path.join(ROOT, "examples", "policy_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def reference(student, params, x, rollout, actions, kl, tau):
    """Losses and gradients by autograd, in 64 bits."""
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in params.items()}
    old, adv, ref = (v.cpu().double() for v in rollout)
    actions = actions.cpu().long()

    def rms(v):
        return v * (v.pow(2).mean(1, keepdim=True) + 1e-5).rsqrt()

    stream = x.cpu().double()
    h = rms(stream) * p["0.ffn_norm"]
    for b in range(student.blocks):
        z = h @ p[f"{b}.w1"].t()
        out = (z * torch.sigmoid(z) * (h @ p[f"{b}.w3"].t())) @ p[f"{b}.w2"].t()
        stream = stream + p[f"{b}.gate"] * rms(out) * p[f"{b}.post_norm"]
        h = rms(stream) * p[f"{b + 1}.ffn_norm" if b + 1 < student.blocks else "norm"]
    logp = torch.log_softmax(h @ p["output"].t() / tau, 1).gather(1, actions.clamp(min=0)[:, None])[:, 0]
    r, d = torch.exp(logp - old), ref - logp
    loss = -torch.minimum(r * adv, r.clamp(0.8, 1.2) * adv) + kl * (torch.exp(d) - d - 1)
    loss = torch.where(actions >= 0, loss, 0.0)
    loss.mean().backward()
    return loss.detach(), {k: v.grad for k, v in p.items()}, logp.detach() - old


def test_example_against_autograd(example):
    """What is kept in 8 bits is off by half a step of at most 2^-6 of its group's
    largest magnitude: evenly spread, 2^-6 / sqrt(12) of some three times its own
    size, 1.4 %, in each of a few factors of a gradient, beside some twenty roundings
    to bf16 of 0.2 %: less than 8 % of it in the 2-norm.  Ratios lie far from the
    clip's borders (the old policy is set so), or their roundings would decide."""
    g = torch.Generator().manual_seed(3)
    student = example.Policy(96, 200, 1000, 2)
    ranks = example.Ranks(student, 3, g)
    S = ranks.plan.chunk_elems
    for r in range(3):
        ranks.plan.ag_pack(r, ranks.shards[r], ranks.gathered[r * S:(r + 1) * S])
    ranks.plan.ag_unpack(ranks.gathered, ranks.flat)
    x, rollout, actions = example.batch(student, 130, g)
    _, _, gap = reference(student, ranks.params, x, rollout, actions, 0.0, 1.0)
    rollout = ((rollout[0].cpu() + gap.float() + math.log(1.05)).cuda(), rollout[1], rollout[2])
    weight = torch.full((130,), 1 / 130, device="cuda")
    loss = student.loss_and_gradients(ranks.params, ranks.grads, x, rollout, actions, weight, 1.0)
    want, grads, _ = reference(student, ranks.params, x, rollout, actions, example.KL_WEIGHT, 1.0)
    assert (loss.cpu().double() - want).norm() <= 0.02 * want.norm()
    for k, v in grads.items():
        off = (ranks.grads[k].cpu().double() - v).norm() / v.norm()
        assert off <= 0.08, (k, off)


def test_example_runs(example):
    losses = example.main(steps=3, tokens=256, vocab=1024)
    assert all(math.isfinite(v) for v in losses)
