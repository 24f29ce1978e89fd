"""Data-parallel policy steps over one FSDP bucket, on one GPU.

The student of ``distill_step.py`` as a policy: it takes one action per state, and
learns from the advantages of actions that were sampled before, under the
clipped policy loss with a KL term to a reference.  What a block's backward pass
needs is kept in 8 bits: the normed input, both projections of the gated
feed-forward and the block's output; the feed-forward's product is made again from
the projections.  Every rank's step:

    ag_pack, [all-gather], ag_unpack                      the parameters, in bf16
    block_norm, checkpoint_save, gated_linear, linear     the blocks, forward
    policy_loss                                           loss and gradient of the logits in one pass
    linear_backward, gated_linear_backward,
    checkpoint_restore, block_norm_backward               the blocks, backward, straight into the gradients
    rs_pack, [exchange], rs_reduce                        the averaged fp32 gradient shards

Run: ``python examples/policy_step.py``.
"""

from __future__ import annotations

import os
import sys

import torch

sys.path[:0] = [os.path.dirname(os.path.dirname(os.path.abspath(__file__))), os.path.dirname(os.path.abspath(__file__))]
from distill_step import BF16, Ranks, Student  # noqa: E402
from paper_2411_00284_amd import (Checkpoint, block_norm, block_norm_backward, checkpoint_restore, checkpoint_save,  # noqa: E402
                                  gated_linear, gated_linear_backward, linear, linear_backward, policy_loss)

KL_WEIGHT = 0.02


class Policy(Student):
    """The step between the copy-out and the copy-in, from ``rollout`` (the
    actions' log probabilities when they were taken, their advantages, and their
    log probabilities under the reference) and ``actions``."""

    def loss_and_gradients(self, params: dict, grads: dict, x, rollout, actions, weight, temperature):
        t, dev = x.shape[0], x.device
        old, advantages, reference = rollout

        def empty(columns):
            return torch.empty(t, columns, dtype=BF16, device=dev)

        def saved(values):
            kept = Checkpoint.empty(*values.shape, device=dev)
            checkpoint_save(values, kept)
            return kept

        # forward
        kept, h = [], empty(self.hidden)
        block_norm(x, pre_weight=params["0.ffn_norm"], h=h)
        stream = x
        for b in range(self.blocks):
            gate, up = Checkpoint.empty(t, self.ffn, device=dev), Checkpoint.empty(t, self.ffn, device=dev)
            act, out = empty(self.ffn), empty(self.hidden)
            gated_linear(h, params[f"{b}.w1"], params[f"{b}.w3"], act, gate=gate, up=up)
            linear(act, params[f"{b}.w2"], out)
            after = params[f"{b + 1}.ffn_norm" if b + 1 < self.blocks else "norm"]
            y, next_h = empty(self.hidden), empty(self.hidden)
            block_norm(stream, branch=out, post_weight=params[f"{b}.post_norm"], gate=params[f"{b}.gate"], pre_weight=after,
                       y=y, h=next_h)
            kept.append((saved(h), gate, up, saved(out), y))
            stream, h = y, next_h
        logits = empty(self.vocab)
        linear(h, params["output"], logits)

        # the loss, and the logits' gradient in their place
        loss = torch.empty(t, device=dev)
        policy_loss(logits, actions, old, advantages, loss, ref_logp=reference, kl_weight=KL_WEIGHT, temperature=temperature,
                    dloss=weight, dlogits=logits)

        # backward
        dh, dstream = empty(self.hidden), None
        linear_backward(logits, saved(h), params["output"], dx=dh, dweight=grads["output"])
        for b in reversed(range(self.blocks)):
            h8, gate, up, out8, y = kept[b]
            after = f"{b + 1}.ffn_norm" if b + 1 < self.blocks else "norm"
            dx, dout, out, act, dact = empty(self.hidden), empty(self.hidden), empty(self.hidden), empty(self.ffn), empty(self.ffn)
            checkpoint_restore(out8, out)
            block_norm_backward(y, dy=dstream, dh=dh, branch=out, post_weight=params[f"{b}.post_norm"],
                                gate=params[f"{b}.gate"], pre_weight=params[after], dx=dx, dbranch=dout,
                                dpre_weight=grads[after], dpost_weight=grads[f"{b}.post_norm"], dgate=grads[f"{b}.gate"])
            linear_backward(dout, act, params[f"{b}.w2"], dx=dact)
            # The feed-forward's product again, for w2's gradient.
            gated_linear_backward(dact, h8, params[f"{b}.w1"], params[f"{b}.w3"], gate, up, out=act, dx=dh,
                                  dgate_weight=grads[f"{b}.w1"], dup_weight=grads[f"{b}.w3"])
            linear_backward(dout, act, params[f"{b}.w2"], dweight=grads[f"{b}.w2"])
            dstream = dx
        block_norm_backward(x, dy=dstream, dh=dh, pre_weight=params["0.ffn_norm"], dpre_weight=grads["0.ffn_norm"])
        return loss


def batch(student: Student, tokens: int, generator, device="cuda"):
    """States, the log probabilities and advantages of actions sampled evenly
    (better where a fixed function of the state says so), and the actions; the
    first tenth of the states are a prompt's and count for nothing."""
    x = torch.randn(tokens, student.hidden, generator=generator)
    mix = torch.randn(student.hidden, student.vocab, generator=torch.Generator().manual_seed(7)) * student.hidden ** -0.5
    actions = torch.randint(0, student.vocab, (tokens,), generator=generator)
    advantages = (x @ mix).gather(1, actions[:, None])[:, 0]
    actions[:tokens // 10] = -1
    even = torch.full((tokens,), -torch.log(torch.tensor(float(student.vocab))).item())
    return x.to(BF16).to(device), tuple(v.to(device) for v in (even, advantages, even)), actions.to(torch.int32).to(device)


def main(steps: int = 8, world: int = 4, hidden: int = 256, ffn: int = 688, vocab: int = 4096, blocks: int = 2,
         tokens: int = 512) -> list[float]:
    g = torch.Generator().manual_seed(0)
    policy = Policy(hidden, ffn, vocab, blocks)
    ranks = Ranks(policy, world, g)
    batches = [batch(policy, tokens, g) for _ in range(world)]
    losses = []
    for k in range(steps):
        losses.append(ranks.step(batches, temperature=1.0, rate=0.5))
        print(f"step {k}: loss {losses[-1]:.4f}", flush=True)
    return losses


if __name__ == "__main__":
    main()
