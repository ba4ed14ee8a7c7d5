"""The distillation example: its gradient against torch's own derivatives of
the definitions, and its loss over a few steps through the codec."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("distill_moe", os.path.join(ROOT, "examples", "distill_moe.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_gradient_of_a_step_matches_torch(example):
    torch.manual_seed(3)
    vocab, rows, k, t, coef = 1000, 64, 12, 2.0, 0.1
    student = example.Student(vocab, 32, 4, 2).cuda()
    tokens = torch.randint(0, vocab, (rows,), device="cuda")
    x = 4.0 * torch.randn(rows, vocab, device="cuda")
    teacher = example.teacher_payload(x, k, t)
    share = example.Share()
    a, b = example.worker_losses(student, tokens, teacher, t, coef, share)
    student.zero_grad()
    (a + b.sum()).backward()
    got = example.flat_gradient(student).double()

    # the same from torch's operations, in 32 bits where the student's are
    val, idx = torch.topk(x, k, 1)
    assert torch.equal(idx, teacher.idx.long())
    logits, route, experts = student(tokens)
    others = torch.ones_like(x, dtype=torch.bool).scatter(1, idx, False)
    rest = torch.logsumexp(torch.where(others, x / t, -math.inf), 1, keepdim=True)
    log_p = torch.log_softmax(torch.cat([val / t, rest], 1), 1)
    log_q = torch.log_softmax(logits / t, 1)
    tail = torch.logsumexp(torch.where(others, log_q, -math.inf), 1, keepdim=True)
    kl = (log_p.exp() * (log_p - torch.cat([log_q.gather(1, idx), tail], 1))).sum(1)
    want_a = t * t * kl.mean()
    f = 4.0 * torch.bincount(experts.flatten(), minlength=4) / (2 * rows)
    want_b = coef * (f * torch.softmax(route, 1).mean(0)).sum()
    student.zero_grad()
    (want_a + want_b).backward()
    want = example.flat_gradient(student).double()
    a, b, want_a, want_b = (float(v.detach()) for v in (a, b, want_a, want_b))
    assert abs(a - want_a) <= 1e-5 * (1 + want_a)
    assert abs(b - want_b) <= 1e-5 * want_b
    # both sides are sums of some hundred terms in 32 bits
    assert float((got - want).abs().max()) <= 1e-5 * float(want.abs().max())


def test_divergence_falls(example):
    seen = example.train(workers=2, steps=30, rows=128, vocab=2000, dim=32, experts=4)
    assert all(math.isfinite(x) for x in seen)
    assert sum(seen[-5:]) < 0.8 * sum(seen[:5])
