"""A worker's training steps on the samples that its stream says come next.

The job is planned as any other (the streams R of all workers). Its samples are
token sequences of unequal length, held in blocks of a resident token buffer;
with each token the sample stores a teacher's top logits. One step of worker 0:

  batch_tables        where the tokens of the next batch lie, for all workers
  packed_attention    one causal attention layer over the packed samples
  topk_distill        loss and gradient against the teacher's top logits

and the gradients go back through packed_attention_grad to the weights.

Usage: python examples/token_step.py [--steps 40]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2101_08734_amd import nopfs  # noqa: E402

VOCAB, TOP, HEADS, KV_HEADS, WIDTH = 503, 4, 4, 2, 32
BLOCK, LONGEST, CAP = 16, 90, 1_024


class Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, qkv, start):
        q, k, v = _heads(qkv)
        o, lse = nopfs.packed_attention(q, k, v, start)
        ctx.save_for_backward(qkv, o, lse, start)
        return o

    @staticmethod
    def backward(ctx, do):
        qkv, o, lse, start = ctx.saved_tensors
        grad = torch.empty_like(qkv)  # dq, dk and dv side by side, as the projection wrote them
        nopfs.packed_attention_grad(do.contiguous(), *_heads(qkv), o, lse, start,
                                    **dict(zip(("dq", "dk", "dv"), _heads(grad))))
        return grad, None


class Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, index, teacher, tau, weight):
        loss, grad = nopfs.topk_distill(logits, index, teacher, tau, weight=weight)
        ctx.save_for_backward(grad)
        return loss.sum()

    @staticmethod
    def backward(ctx, g):
        return ctx.saved_tensors[0] * g, None, None, None, None


def _heads(qkv):
    return qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:]


class Model(torch.nn.Module):
    def __init__(self):
        super().__init__()
        g = torch.Generator().manual_seed(0)
        dim = HEADS * WIDTH

        def weight(*shape):
            return torch.nn.Parameter(torch.randn(shape, generator=g) * shape[0] ** -0.5)

        self.embed = torch.nn.Parameter(torch.randn((VOCAB, dim), generator=g) * 0.5)
        self.qkv = weight(dim, (HEADS + 2 * KV_HEADS) * WIDTH)
        self.out, self.head = weight(dim, dim), weight(dim, VOCAB)

    def forward(self, tokens, start):
        x = self.embed[tokens].bfloat16()
        qkv = (x @ self.qkv.bfloat16()).view(-1, HEADS + 2 * KV_HEADS, WIDTH)
        o = Attention.apply(qkv, start)
        return (x + o.reshape(x.shape) @ self.out.bfloat16()) @ self.head.bfloat16()


def sample_tokens(ids, pos):
    """The content of the samples: token `pos` of sample `id`."""
    return (ids * 31 + pos * 17 + (ids * pos) % 7) % VOCAB


def teacher_entries(tokens, previous):
    """A teacher that goes by the token, and less by the one before it: its top
    classes and their logits."""
    index = torch.stack([tokens * 3 % VOCAB, (tokens * 3 + 101) % VOCAB, (previous * 5 + 7) % VOCAB,
                         (tokens * 3 + 303) % VOCAB], 1)
    logits = torch.tensor([6.0, 4.0, 3.0, 2.0], device=tokens.device).expand(len(tokens), TOP)
    return index.int(), logits.half().contiguous()


def main(steps=40):
    job = nopfs.Job(F=2_000, E=4, N=4, B=16, drop_last=1, seed=42)
    R = nopfs.access_streams(job)
    gen = torch.Generator(device="cuda").manual_seed(1)
    lengths = torch.randint(1, LONGEST + 1, (job.F,), generator=gen, device="cuda", dtype=torch.int32)
    blocks = CAP // BLOCK + job.B
    buffer = torch.zeros(job.N * blocks * BLOCK, dtype=torch.int64, device="cuda")
    free = torch.arange(job.N * blocks, dtype=torch.int32, device="cuda").view(job.N, blocks)
    model = Model().cuda()
    optimizer = torch.optim.Adam(model.parameters(), lr=1e-2)
    losses, tables = [], None
    for step in range(steps):
        at = step * job.B % (R.shape[1] - job.B + 1)
        ids = R[:, at:at + job.B]
        tables = nopfs.batch_tables(ids, lengths, free, BLOCK, -(-LONGEST // BLOCK), CAP, out=tables)
        slot, row, pos, start = (tables[x][0] for x in ("slot", "row", "pos", "start"))
        # what a prefetcher does: the samples' tokens into their blocks
        there = slot >= 0
        buffer[slot[there]] = sample_tokens(ids[0].long()[row[there].long()], pos[there].long())
        # the step, on every packed token and the padding behind them
        tokens = torch.where(there, buffer[slot.clamp(min=0)], 0)
        index, teacher = teacher_entries(tokens, torch.where(pos > 0, tokens.roll(1), 0))
        weight = there.float() / there.sum()
        loss = Distill.apply(model(tokens, start), index, teacher, 1.0, weight)
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    losses = torch.stack(losses).tolist()
    used = tables["used"][0].tolist()
    print(f"worker 0: {used[0]} samples, {used[1]} tokens in {used[2]} blocks in the last step; "
          f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {steps} steps")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=40)
    main(ap.parse_args().steps)
