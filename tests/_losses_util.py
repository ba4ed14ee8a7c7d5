"""The loss operators from their definitions, in 64 bits on the CPU, and the
error bounds that the GPU's 32-bit sums keep (not collected by pytest).

Bounds.  A sum of exponentials is off by at most SUM of itself: each thread
adds up to 64 terms one after the other (64 x 2^-24), some 20 further additions
join threads, waves, blocks and slices, and an exponential of an argument
rounded at up to 30 is off by 30 x 2^-23.  Together 9e-6; SUM is 1.5e-5.
"""
from __future__ import annotations

import math

import torch

SUM = 1.5e-5
# half a unit in the last place, twice over: the exact value may round the other way
ROUND = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def top(x, k, t):
    """(columns, values, rest) of each row: by value descending, ties to the lowest column, -inf never kept."""
    x = x.double()
    rows, cols = x.shape
    val, at = torch.sort(x, dim=1, descending=True, stable=True)
    n = min(k, cols)
    idx = torch.full((rows, k), -1, dtype=torch.int64)
    out = torch.full((rows, k), -math.inf, dtype=torch.float64)
    out[:, :n] = val[:, :n]
    idx[:, :n] = torch.where(val[:, :n] == -math.inf, -1, at[:, :n])
    rest = torch.full((rows,), -math.inf, dtype=torch.float64)
    if cols > k:
        rest = torch.logsumexp(val[:, k:] / t, 1)
    return idx, out, rest


def distill(z, idx, val, rest, t, weight=None, upstream=None):
    """(loss per row, gradient at z, the gradient's error scale) from the definition."""
    z = z.double()
    rows, cols = z.shape
    loss = torch.zeros(rows, dtype=torch.float64)
    grad = torch.zeros_like(z)
    scale = torch.zeros_like(z)
    for r in range(rows):
        w = 1.0 if weight is None else float(weight[r])
        u = 1.0 if upstream is None else float(upstream[r])
        if w == 0:
            continue
        there = (idx[r] >= 0) & (idx[r] < cols)
        j = idx[r][there].long()
        b = -math.inf if rest is None else float(rest[r])
        entries = torch.cat([val[r][there].double() / t, torch.tensor([b], dtype=torch.float64)])
        if bool((entries == -math.inf).all()):
            continue
        p_all = torch.softmax(entries, 0)
        p, p_rest = p_all[:-1], float(p_all[-1])
        x = z[r] / t
        none = bool((x == -math.inf).all())
        q = torch.zeros_like(x) if none else torch.softmax(x, 0)
        log_q = torch.full_like(x, -math.inf) if none else torch.log_softmax(x, 0)
        kept = torch.zeros(cols, dtype=torch.bool)
        kept[j] = True
        others = log_q[~kept]
        log_tail = float(torch.logsumexp(others, 0)) if others.numel() else -math.inf
        kl = torch.where(p > 0, p * (torch.log(p) - log_q[j]), 0.0).sum()
        if p_rest > 0:
            kl = kl + p_rest * (math.log(p_rest) - log_tail) if log_tail > -math.inf else torch.tensor(math.inf)
        loss[r] = w * float(kl)
        if u == 0:
            continue
        g = torch.zeros_like(x)
        s = torch.zeros_like(x)
        g[j] = q[j] - p
        s[j] = q[j] + p
        share = torch.zeros_like(x)
        if log_tail > -math.inf:
            share[~kept] = torch.softmax(x[~kept], 0)
            tail = math.exp(log_tail) - p_rest
            g = torch.where(kept, g, share * tail)
            s = torch.where(kept, s, share * (math.exp(log_tail) + p_rest))
        grad[r] = u * w / t * g
        scale[r] = abs(u * w / t) * s
    return loss, grad, scale


def balance(z, experts, k, mask, group, coef, upstream=1.0, counts=None, count_rows=None):
    """(counts, rows, mean probabilities, loss, gradient, the gradient's error scale) from the definition."""
    z = z.double()
    T, E = z.shape
    G = -(-T // group)
    valid = torch.ones(T, dtype=torch.bool) if mask is None else mask.bool()
    own = torch.zeros(G, E, dtype=torch.int64)
    n = torch.zeros(G, dtype=torch.int64)
    prob = torch.zeros(G, E, dtype=torch.float64)
    p = torch.zeros_like(z)
    some = valid & ~(z == -math.inf).all(1)
    p[some] = torch.softmax(z[some], 1)
    for g in range(G):
        part = torch.arange(g * group, min(T, (g + 1) * group))
        part = part[valid[part]]
        n[g] = part.numel()
        if experts is not None:
            e = experts[part].flatten().long()
            own[g] = torch.bincount(e[(e >= 0) & (e < E)], minlength=E)
        if part.numel():
            prob[g] = p[part].sum(0) / part.numel()
    c = own if counts is None else counts.long()
    cn = n if count_rows is None else count_rows.long()
    f = torch.where(cn[:, None] > 0, E * c.double() / (k * cn.clamp(min=1)[:, None].double()), 0.0)
    loss = float(coef / max(G, 1) * (f * prob).sum())
    grad, scale = torch.zeros_like(z), torch.zeros_like(z)
    for r in range(T):
        g = r // group
        if valid[r]:
            s = upstream * coef / (G * int(n[g]))
            dot = (f[g] * p[r]).sum()
            grad[r] = s * p[r] * (f[g] - dot)
            scale[r] = abs(s) * p[r] * (f[g] + dot)
    return own, n, prob, loss, grad, scale


def kept_columns(rows, cols, k, gen):
    return torch.stack([torch.randperm(cols, generator=gen)[:k] for _ in range(rows)])


def student(rows, cols, k, dtype, seed, t=1.0, spread=2.0):
    """(z, idx, val, rest) of ordinary shape: kept columns high in both, the rest a few percent."""
    gen = torch.Generator().manual_seed(seed)
    k = min(k, cols)
    z = spread * torch.randn(rows, cols, generator=gen)
    idx = kept_columns(rows, cols, k, gen)
    v = 8.0 - 1.5 * torch.log1p(torch.arange(k).float()) + 0.3 * torch.randn(rows, k, generator=gen)
    z.scatter_(1, idx, 0.85 * v + torch.randn(rows, k, generator=gen))
    rest = torch.logsumexp(v.double() / t, 1) + torch.log(0.003 + 0.3 * torch.rand(rows, generator=gen).double())
    return z.to(dtype), idx.to(torch.int32), v, rest.float()
