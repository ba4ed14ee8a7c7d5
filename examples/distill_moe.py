"""A data-parallel distillation of a small mixture-of-experts student, with every operator of the package in its place:

  teacher   its logits -> top_logits -> a payload of K columns, K logits and one entry for the rest per token
  worker    its tokens and payload -> student -> distill_forward / distill_backward (the divergence) and
            balance_forward / balance_backward (the router), whose counts are summed over the workers before the
            gradient is taken: a balance over the global batch
  exchange  the worker's flat gradient -> binding.payload_encode; all payloads -> binding.payload_decode_sum
  update    plain gradient descent; what a payload did not carry stays with its worker for the next step

    python examples/distill_moe.py [--workers 2] [--steps 40]

The workers take turns on one GPU.  On several, each is a process: the two sums of counts become an all-reduce and the
payloads an all-gather.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2102_03112_amd import binding as B  # noqa: E402
from paper_2102_03112_amd import losses as L  # noqa: E402


class Distill(torch.autograd.Function):
    """Per row, weight * KL(teacher || student)"""

    @staticmethod
    def forward(ctx, logits, teacher, temperature, weight):
        rows, cols = logits.shape
        loss = torch.empty(rows, device=logits.device)
        stats = torch.empty(rows, L.STATS, device=logits.device)
        ws = L.workspace(rows, cols, teacher.idx.shape[1], logits.device)
        L.distill_forward(logits, teacher, temperature, weight, loss, stats, ws)
        ctx.save_for_backward(logits, weight, stats)
        ctx.teacher, ctx.temperature = teacher, temperature
        return loss

    @staticmethod
    def backward(ctx, upstream):
        logits, weight, stats = ctx.saved_tensors
        grad = torch.empty_like(logits)
        L.distill_backward(logits, ctx.teacher, ctx.temperature, weight, upstream, stats, grad)
        return grad, None, None, None


class Balance(torch.autograd.Function):
    """The balance loss of one group; `share` collects a worker's counts, and returns the sums over all workers when
    the gradient is taken."""

    @staticmethod
    def forward(ctx, logits, experts, coef, share):
        rows, E = logits.shape
        counts = torch.empty(1, E, dtype=torch.int32, device=logits.device)
        n = torch.empty(1, dtype=torch.int32, device=logits.device)
        loss = torch.empty(1, device=logits.device)
        L.balance_forward(logits, experts, None, rows, coef, counts, n, None, loss,
                          L.workspace(rows, E, 1, logits.device))
        share.add(counts, n)
        ctx.save_for_backward(logits, n)
        ctx.k, ctx.coef, ctx.share = experts.shape[1], coef, share
        return loss

    @staticmethod
    def backward(ctx, upstream):
        logits, n = ctx.saved_tensors
        grad = torch.empty_like(logits)
        L.balance_backward(logits, ctx.k, None, logits.shape[0], ctx.coef, ctx.share.counts, ctx.share.rows, n,
                           upstream.contiguous(), grad)
        return grad, None, None, None


class Share:
    """Counts and rows summed over the workers (an all-reduce, were they processes)."""

    def __init__(self):
        self.counts = self.rows = 0

    def add(self, counts, rows):
        self.counts, self.rows = self.counts + counts, self.rows + rows


class Student(torch.nn.Module):
    def __init__(self, vocab, dim, experts, chosen):
        super().__init__()
        self.embed = torch.nn.Embedding(vocab, dim)
        self.router = torch.nn.Linear(dim, experts, bias=False)
        self.up = torch.nn.Parameter(torch.randn(experts, dim, dim) * dim ** -0.5)
        self.head = torch.nn.Linear(dim, vocab, bias=False)
        self.chosen = chosen

    def forward(self, tokens):
        """(logits, router logits, chosen experts)"""
        x = self.embed(tokens)
        route = self.router(x)
        weight, experts = torch.topk(torch.softmax(route, 1), self.chosen, 1)
        y = x
        for e in range(self.up.shape[0]):
            row, slot = torch.nonzero(experts == e, as_tuple=True)
            y = y.index_add(0, row, weight[row, slot, None] * torch.tanh(x[row] @ self.up[e]))
        return self.head(y), route, experts


def teacher_payload(logits, k, temperature):
    rows, cols = logits.shape
    idx = torch.empty(rows, k, dtype=torch.int32, device=logits.device)
    val = torch.empty(rows, k, device=logits.device)
    rest = torch.empty(rows, device=logits.device)
    L.top_logits(logits, k, temperature, idx, val, rest, L.workspace(rows, cols, k, logits.device))
    return L.Teacher(idx, val, rest)


def flat_gradient(student):
    return torch.cat([p.grad.flatten() for p in student.parameters()])


def worker_losses(student, tokens, teacher, temperature, coef, share):
    """(divergence averaged over the tokens, balance loss), both with their graphs"""
    logits, route, experts = student(tokens)
    n = tokens.numel()
    weight = torch.full((n,), temperature * temperature / n, device=tokens.device)
    return Distill.apply(logits, teacher, temperature, weight).sum(), Balance.apply(route, experts, coef, share)


def train(workers=2, steps=40, rows=256, vocab=2000, dim=32, experts=8, chosen=2, kept=32, temperature=2.0, coef=0.01,
          rate=30.0, seed=0, say=None):
    """The divergence of every step, averaged over the workers."""
    torch.manual_seed(seed)
    dev = "cuda"
    table = torch.randn(vocab, 16, device=dev) @ torch.randn(16, vocab, device=dev)  # the teacher's logits by token
    student = Student(vocab, dim, experts, chosen).to(dev)
    params = list(student.parameters())
    d = sum(p.numel() for p in params)
    offsets = [0]
    for p in params:
        offsets.append(offsets[-1] + p.numel())
    cfg = B.Config(offsets, (1, 20), 1e-3, 5, 8, value_source=B.VALUES_SPARSE)
    total, _ = B.payload_layout(cfg)
    ws = B.workspace(d, cfg.n_tensors)
    payloads = [torch.empty(total, dtype=torch.uint8, device=dev) for _ in range(workers)]
    kept_back = [torch.zeros(d, device=dev) for _ in range(workers)]
    own, mean = torch.empty(d, device=dev), torch.empty(d, device=dev)
    seen = []
    for step in range(steps):
        share, losses = Share(), []
        for w in range(workers):
            gen = torch.Generator(device=dev).manual_seed(seed + 1 + step * workers + w)
            tokens = torch.randint(0, vocab, (rows,), generator=gen, device=dev)
            teacher = teacher_payload(table[tokens], kept, temperature)
            losses.append(worker_losses(student, tokens, teacher, temperature, coef, share))
        for w, (divergence, balance) in enumerate(losses):  # the counts are complete now
            student.zero_grad()
            (divergence + balance.sum()).backward()
            kept_back[w] += flat_gradient(student)
            B.payload_encode(kept_back[w], cfg, payloads[w], None, ws)
            B.payload_decode(payloads[w], cfg, own, None, None, None, ws)
            kept_back[w] -= own
        B.payload_decode_sum(payloads, cfg, 1.0 / workers, mean, None, ws)
        with torch.no_grad():
            for p, a, b in zip(params, offsets, offsets[1:]):
                p -= rate * mean[a:b].view_as(p)
        seen.append(float(sum(x.detach() for x, _ in losses)) / workers)
        if say and (step % 10 == 0 or step == steps - 1):
            say(f"step {step:3d}  divergence {seen[-1]:.4f}  choices per expert {share.counts[0].tolist()}")
    return seen


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--workers", type=int, default=2)
    ap.add_argument("--steps", type=int, default=40)
    a = ap.parse_args()
    train(a.workers, a.steps, say=lambda s: print(s, flush=True))
