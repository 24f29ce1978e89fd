"""Data-parallel distillation steps over one FSDP bucket, on one GPU.

A small student (gated feed-forward blocks between norms, and an output head)
learns a teacher's top logits.  Its parameters live as fp32 ``Shard(0)`` shards
of W ranks in one bucket; the ranks take their turns on the GPU, and the
collectives are copies between their buffers.  Every rank's step:

    ag_pack, [all-gather], ag_unpack        the parameters, in bf16
    block_norm, linear                      the blocks, forward
    distill_loss                            loss and gradient of the logits in one pass
    linear_backward, block_norm_backward    the blocks, backward, straight into the gradients
    rs_pack, [exchange], rs_reduce          the averaged fp32 gradient shards

Run: ``python examples/distill_step.py``.
"""

from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2411_00284_amd import (BucketPlan, block_norm, block_norm_backward, distill_loss, linear,  # noqa: E402
                                  linear_backward)

BF16 = torch.bfloat16


class Student:
    """Sizes, the bucket's order of parameters, and the step between the
    copy-out and the copy-in."""

    def __init__(self, hidden: int, ffn: int, vocab: int, blocks: int):
        self.hidden, self.ffn, self.vocab, self.blocks = hidden, ffn, vocab, blocks
        self.names, self.shapes = [], []
        for b in range(blocks):
            for name, shape in (("w1", (ffn, hidden)), ("w3", (ffn, hidden)), ("w2", (hidden, ffn)),
                                ("ffn_norm", (hidden,)), ("post_norm", (hidden,)), ("gate", (hidden,))):
                self.names.append(f"{b}.{name}")
                self.shapes.append(shape)
        self.names += ["norm", "output"]
        self.shapes += [(hidden,), (vocab, hidden)]

    def init(self, generator) -> list[torch.Tensor]:
        """Full fp32 parameters."""
        out = []
        for name, shape in zip(self.names, self.shapes):
            if len(shape) == 1:
                out.append(torch.full(shape, 0.5 if name.endswith("gate") else 1.0))
            else:
                out.append(torch.randn(shape, generator=generator) * shape[1] ** -0.5)
        return out

    def loss_and_gradients(self, params: dict, grads: dict, x, teacher, ids, weight, temperature):
        """One forward and backward: every token's loss; the gradients of
        ``weight``-ed losses go to ``grads``."""
        t, dev = x.shape[0], x.device

        def empty(columns):
            return torch.empty(t, columns, dtype=BF16, device=dev)

        # forward: the norm before a block is made with the residual add before it
        kept, h = [], empty(self.hidden)
        block_norm(x, pre_weight=params["0.ffn_norm"], h=h)
        stream = x
        for b in range(self.blocks):
            up, pre, act, out = empty(self.ffn), empty(self.ffn), empty(self.ffn), empty(self.hidden)
            linear(h, params[f"{b}.w3"], up)
            linear(h, params[f"{b}.w1"], act, activation="silu", times=up, pre=pre)
            linear(act, params[f"{b}.w2"], out)
            after = params[f"{b + 1}.ffn_norm" if b + 1 < self.blocks else "norm"]
            y, next_h = empty(self.hidden), empty(self.hidden)
            block_norm(stream, branch=out, post_weight=params[f"{b}.post_norm"], gate=params[f"{b}.gate"], pre_weight=after,
                       y=y, h=next_h)
            kept.append((h, up, pre, act, out, y))
            stream, h = y, next_h
        logits = empty(self.vocab)
        linear(h, params["output"], logits)

        # the loss, and the logits' gradient in their place
        loss = torch.empty(t, device=dev)
        distill_loss(logits, teacher, ids, loss, temperature=temperature, dloss=weight, dlogits=logits)

        # backward
        dh, dstream = empty(self.hidden), None
        linear_backward(logits, h, params["output"], dx=dh, dweight=grads["output"])
        for b in reversed(range(self.blocks)):
            h, up, pre, act, out, y = kept[b]
            after = f"{b + 1}.ffn_norm" if b + 1 < self.blocks else "norm"
            dx, dout = empty(self.hidden), empty(self.hidden)
            block_norm_backward(y, dy=dstream, dh=dh, branch=out, post_weight=params[f"{b}.post_norm"],
                                gate=params[f"{b}.gate"], pre_weight=params[after], dx=dx, dbranch=dout,
                                dpre_weight=grads[after], dpost_weight=grads[f"{b}.post_norm"], dgate=grads[f"{b}.gate"])
            dact, dup, dh3 = empty(self.ffn), empty(self.ffn), empty(self.hidden)
            linear_backward(dout, act, params[f"{b}.w2"], dx=dact, dweight=grads[f"{b}.w2"])
            linear_backward(dact, h, params[f"{b}.w1"], activation="silu", pre=pre, times=up, dx=dh, dweight=grads[f"{b}.w1"],
                            dtimes=dup)
            linear_backward(dup, h, params[f"{b}.w3"], dx=dh3, dweight=grads[f"{b}.w3"])
            dh.add_(dh3)
            dstream = dx
        block_norm_backward(x, dy=dstream, dh=dh, pre_weight=params["0.ffn_norm"], dpre_weight=grads["0.ffn_norm"])
        return loss


class Ranks:
    """W ranks of one bucket on one GPU: their shards and buffers."""

    def __init__(self, student: Student, world: int, generator, device="cuda"):
        self.student, self.world = student, world
        self.plan = BucketPlan(world, student.shapes)
        S, n = self.plan.chunk_elems, len(student.shapes)
        full = student.init(generator)
        self.shards = []
        for r in range(world):
            own = []
            for p, w in enumerate(full):
                rows, first = self.plan.local_rows(p, r), r * self.plan.rows_per_rank(p)
                own.append(w[first:first + rows].reshape(-1).contiguous().to(device))
            self.shards.append(own)
        self.gathered = torch.empty(world * S, dtype=BF16, device=device)
        self.sent = [torch.empty(world * S, dtype=BF16, device=device) for _ in range(world)]
        self.received = torch.empty(world * S, dtype=BF16, device=device)
        flat = [torch.empty(self.plan.full_elems(p), dtype=BF16, device=device) for p in range(n)]
        self.flat, self.grad = flat, [torch.empty_like(f) for f in flat]
        self.params = {k: f.view(s) for k, f, s in zip(student.names, flat, student.shapes)}
        self.grads = {k: f.view(s) for k, f, s in zip(student.names, self.grad, student.shapes)}
        self.grad_shards = [[torch.empty_like(s) for s in own] for own in self.shards]

    def step(self, batches, temperature: float, rate: float) -> float:
        """One step of all ranks, a batch (x, teacher, ids) each; the mean loss."""
        S, total = self.plan.chunk_elems, 0.0
        for r in range(self.world):                                     # copy-in; the all-gather lays chunks side by side
            self.plan.ag_pack(r, self.shards[r], self.gathered[r * S:(r + 1) * S])
        for r, (x, teacher, ids) in enumerate(batches):
            self.plan.ag_unpack(self.gathered, self.flat)
            weight = torch.full((x.shape[0],), 1.0 / x.shape[0], device=x.device)
            loss = self.student.loss_and_gradients(self.params, self.grads, x, teacher, ids, weight, temperature)
            self.plan.rs_pack(self.grad, self.sent[r])
            total += float(loss.mean())
        for r in range(self.world):                                     # the exchange: chunk r of every rank
            for i in range(self.world):
                self.received[i * S:(i + 1) * S].copy_(self.sent[i][r * S:(r + 1) * S])
            self.plan.rs_reduce(r, self.received, self.grad_shards[r])
            for w, g in zip(self.shards[r], self.grad_shards[r]):
                w.sub_(g, alpha=rate)
        return total / self.world


def batch(student: Student, tokens: int, top: int, generator, device="cuda"):
    """Activations, and the top logits of a teacher that is a fixed function of them."""
    x = torch.randn(tokens, student.hidden, generator=generator)
    mix = torch.randn(student.hidden, student.vocab, generator=torch.Generator().manual_seed(7)) * 3 * student.hidden ** -0.5
    teacher, ids = (x @ mix).topk(top, 1)
    return x.to(BF16).to(device), teacher.to(device), ids.to(torch.int32).to(device)


def main(steps: int = 8, world: int = 4, hidden: int = 256, ffn: int = 688, vocab: int = 4096, blocks: int = 2,
         tokens: int = 512, top: int = 64) -> list[float]:
    g = torch.Generator().manual_seed(0)
    student = Student(hidden, ffn, vocab, blocks)
    ranks = Ranks(student, world, g)
    batches = [batch(student, tokens, top, g) for _ in range(world)]
    losses = []
    for k in range(steps):
        losses.append(ranks.step(batches, temperature=2.0, rate=10.0))
        print(f"step {k}: loss {losses[-1]:.4f}", flush=True)
    return losses


if __name__ == "__main__":
    main()
