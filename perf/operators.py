"""The losses of a data-parallel distillation step as their users call them: what is timed, on which inputs, and
what the answers are.

A case is one call (or two in a row) of the package's loss operators:

  top          a teacher's logits into its k largest and one logit that stands for the rest (the payload it sends)
  forward      the divergence of a student from such a payload, per row
  backward     its gradient, from what the forward pass saved
  step         both in one call, which reads the logits once
  balance      a router's per-expert counts, mean probabilities and balance loss
  balance_bwd  the loss's gradient from counts that are at hand (those of all workers, say)
  balance_both a training step's two calls, forward and backward

With v the teacher's kept logits, rest its last entry, t the temperature and z the student's row, and w the row's
weight, the divergence of a row is

  p = softmax(v / t, rest)        q = softmax(z / t), and q_rest = the sum of q over the columns not kept
  loss = w (sum_k p_k (ln p_k - ln q_k) + p_rest (ln p_rest - ln q_rest))
  dloss / dz_j = (w / t) (q_j - p_j) for a kept column, (w / t) q_j (1 - p_rest / q_rest) for another one

and the balance loss of a group's n valid rows, each with K chosen experts of E,

  f_e = E count_e / (K n)        P_e = the mean of softmax(z)_e        loss = coef / groups  sum_groups sum_e f_e P_e
  dloss / dz_j = (coef / (groups n)) p_j (f_j - sum_e f_e p_e)
"""
from __future__ import annotations

import math

import torch

own = False  # false: the plain form; true: the package's operators

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
STATS = 8  # floats saved per row by the forward pass
DISTILL = ("forward", "backward", "step")


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------


def _logits(kind, rows, cols, k, **kw):
    c = {"kind": kind, "rows": rows, "cols": cols, "k": k, "type": "bf16", "temperature": 1.0, "pad": 0,
         "padded_rows": kind != "top", "ragged": False, "masked": 0, "index": "i32", "values": "f32"}
    c.update(kw)
    return c


def _router(kind, rows, experts, k, **kw):
    c = {"kind": kind, "rows": rows, "cols": experts, "k": k, "type": "bf16", "group": rows, "padded_rows": False,
         "dropped": False, "index": "i64", "pad": 0}
    c.update(kw)
    return c


def listed():
    cases = [
        # a teacher that answers a few tokens at a time: launches and latency count
        ("top_8x32000", _logits("top", 8, 32_000, 50)),
        # an odd vocabulary in 32 bits whose last columns are masked out
        ("top_777x50001_f32", _logits("top", 777, 50_001, 100, type="f32", temperature=2.0, masked=65)),
        # a teacher's pass over one batch
        ("top_2048x131072", _logits("top", 2048, 131_072, 64)),
        # a short validation batch
        ("forward_16x32000", _logits("forward", 16, 32_000, 50, padded_rows=False)),
        # an odd vocabulary in half precision, rows cut out of a wider matrix, teachers that keep differently many
        ("forward_1500x100003_f16", _logits("forward", 1500, 100_003, 100, type="f16", temperature=2.0, pad=5,
                                            ragged=True, index="i64", values="f16")),
        # the backward pass of a framework that keeps the two apart
        ("backward_2048x65536", _logits("backward", 2048, 65_536, 32)),
        # a small student's step in 32 bits
        ("step_256x32000_f32", _logits("step", 256, 32_000, 64, type="f32")),
        # a student's step over a batch of 4096 tokens
        ("step_4096x131072", _logits("step", 4096, 131_072, 64)),
        # one worker's small router: launches and latency count
        ("balance_512x8", _router("balance", 512, 8, 2)),
        # a router of 64 experts, six chosen, over a batch with padding; some choices were dropped for capacity
        ("balance_16384x64", _router("balance", 16_384, 64, 6, padded_rows=True, dropped=True)),
        # its backward pass
        ("balance_bwd_16384x64", _router("balance_bwd", 16_384, 64, 6, padded_rows=True)),
        # 32 sequences balanced one by one over 256 experts, router logits in 32 bits, both directions
        ("balance_both_131072x256", _router("balance_both", 131_072, 256, 8, type="f32", group=4096, index="i32")),
    ]
    return [dict(c, name=n) for n, c in cases]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: every call, size, type and option of the listed ones, mixed."""
    kind = rng.choice(["top", "top", "forward", "backward", "step", "step", "balance", "balance_bwd", "balance_both"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    index = rng.choice(["i32", "i64"])
    pad = rng.choice([0, 0, 0, rng.randint(1, 70)])
    if kind.startswith("balance"):
        experts = rng.choice([8, 16, 32, 64, 128, 256, rng.randint(4, 300)])
        rows = _log_int(rng, 200, min(262_144, 33_000_000 // experts))
        group = rng.choice([rows, rows, rng.randint(max(1, rows // 64), rows)])
        return _router(kind, rows, experts, rng.randint(1, min(8, experts)), type=dtype, group=group,
                       padded_rows=rng.random() < 0.5, dropped=rng.random() < 0.3, index=index, pad=pad)
    cols = rng.choice([_log_int(rng, 2_000, 200_000), _log_int(rng, 2_000, 200_000) | 1, 32_000, 65_536, 131_072])
    rows = _log_int(rng, 4, max(5, (1 << 27) // cols))
    k = _log_int(rng, 1, 256)
    return _logits(kind, rows, cols, k, type=dtype, temperature=rng.choice([1.0, 1.0, 0.7, 2.0, 4.0]), pad=pad,
                   padded_rows=kind != "top" and rng.random() < 0.5, ragged=rng.random() < 0.3,
                   masked=rng.choice([0, 0, rng.randint(1, cols // 20)]) if kind == "top" else 0, index=index,
                   values=rng.choice(["f32", "f32", dtype]))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1_000_003 * seed + 29)
    return gen


def _matrix(c, gen, scale):
    """rows x cols normal numbers of the case's type, cut out of a matrix that is `pad` columns wider."""
    rows, cols = c["rows"], c["cols"]
    full = torch.empty(rows, cols + c["pad"], dtype=DTYPE[c["type"]], device="cuda")
    step = max(1, (1 << 26) // (cols + c["pad"]))
    for a in range(0, rows, step):
        n = min(step, rows - a)
        full[a:a + n] = torch.randn(n, cols + c["pad"], generator=gen, device="cuda") * scale
    return full[:, :cols]


def _kept(c, gen):
    """rows x k distinct columns in no order: random gaps from a random start."""
    rows, cols, k = c["rows"], c["cols"], c["k"]
    gap = torch.randint(1, cols // k + 1, (rows, k), generator=gen, device="cuda")
    idx = torch.cumsum(gap, 1) - 1
    order = torch.argsort(torch.rand(rows, k, generator=gen, device="cuda"), 1)
    return torch.gather(idx, 1, order)


def _heights(c, gen):
    """Kept logits as a language model's are: a few high ones, a slow fall."""
    fall = 13.0 - 2.5 * torch.log1p(torch.arange(c["k"], device="cuda", dtype=torch.float32))
    return fall + 0.3 * torch.randn(c["rows"], c["k"], generator=gen, device="cuda")


def _valid_rows(c):
    """Rows that are not padding: sequences of 64 tokens that end after 60."""
    r = torch.arange(c["rows"], device="cuda")
    return (r % 64 < 60) if c["padded_rows"] else torch.ones_like(r, dtype=torch.bool)


def _index(c, x):
    return x.to(torch.int32 if c["index"] == "i32" else torch.int64).contiguous()


def _inputs(c, seed):
    gen = _generator(seed)
    rows, cols, k = c["rows"], c["cols"], c["k"]
    s = {"case": c}
    if c["kind"] == "top":
        s["logits"] = _matrix(c, gen, 2.0)
        idx = _kept(c, gen)
        s["logits"].scatter_(1, idx, _heights(c, gen).to(s["logits"].dtype))
        if c["masked"]:
            s["logits"][:, cols - c["masked"]:] = float("-inf")
        return s
    valid = _valid_rows(c)
    if c["kind"] in DISTILL:
        t = c["temperature"]
        z = _matrix(c, gen, 2.0)
        idx, v = _kept(c, gen), _heights(c, gen)
        student = 0.85 * v + torch.randn(rows, k, generator=gen, device="cuda")
        z.scatter_(1, idx, student.to(z.dtype))
        v = v.to(DTYPE[c["values"]])
        share = torch.exp(torch.empty(rows, device="cuda").uniform_(math.log(3e-3), math.log(0.3), generator=gen))
        if c["ragged"]:
            keep = torch.randint((k + 1) // 2, k + 1, (rows, 1), generator=gen, device="cuda")
            idx = torch.where(torch.arange(k, device="cuda") < keep, idx, -1)
        heights = torch.where(idx >= 0, v.float() / t, float("-inf"))
        s["rest"] = torch.logsumexp(heights, 1) + torch.log(share)
        s["logits"], s["idx"], s["val"] = z, _index(c, idx), v
        scale = 4096.0 if c["type"] == "f16" else 1.0  # a loss scale keeps half precision's gradients in range
        s["weight"] = torch.where(valid, scale * t * t / valid.sum(), 0.0).float()
        if c["kind"] == "backward":
            s["upstream"] = torch.rand(rows, generator=gen, device="cuda") + 0.5
            s["stats"] = _saved(s)
        return s
    z = _matrix(c, gen, 1.0)
    noisy = z.float() + 0.5 * torch.randn(cols, generator=gen, device="cuda")
    idx = torch.topk(noisy, k, 1).indices
    if c["dropped"]:
        idx = torch.where(torch.rand(rows, k, generator=gen, device="cuda") < 0.03, -1, idx)
    s["logits"], s["experts"], s["coef"] = z, _index(c, idx), 0.01
    s["mask"] = valid if c["padded_rows"] else None
    if c["kind"] == "balance_bwd":
        s["counts"], s["n"] = _counts(s)
    if c["kind"] != "balance":
        scale = 65536.0 if c["type"] == "f16" else 1.0  # as above
        s["upstream"] = scale * (torch.rand(1, generator=gen, device="cuda") + 0.5)
    return s


def _groups(c):
    return -(-c["rows"] // c["group"])


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    rows, cols, k = c["rows"], c["cols"], c["k"]
    z = lambda n, t: torch.zeros(n, dtype=t, device="cuda")  # noqa: E731
    if c["kind"] == "top":
        s["idx"], s["val"], s["rest"] = z((rows, k), torch.int32), z((rows, k), torch.float32), z(rows, torch.float32)
    if c["kind"] in ("forward", "step"):
        s["loss"] = z(rows, torch.float32)
    if c["kind"] == "forward":
        s["stats"] = z((rows, STATS), torch.float32)
    if c["kind"] in ("backward", "step", "balance_bwd", "balance_both"):
        s["grad"] = z((rows, cols), DTYPE[c["type"]])
    if c["kind"] in ("balance", "balance_both"):
        G = _groups(c)
        s["counts"], s["n"] = z((G, cols), torch.int32), z(G, torch.int32)
        s["prob"], s["loss"] = z((G, cols), torch.float32), z(1, torch.float32)
    if own:
        from paper_2102_03112_amd import losses as L

        s["ws"] = L.workspace(rows, cols, k)
        if c["kind"] in DISTILL:
            s["teacher"] = L.Teacher(s["idx"], s["val"], s["rest"])
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2102_03112_amd import losses as L

    c = s["case"]
    kind = c["kind"]
    if kind == "top":
        L.top_logits(s["logits"], c["k"], c["temperature"], s["idx"], s["val"], s["rest"], s["ws"])
        return {"idx": s["idx"], "val": s["val"], "rest": s["rest"]}
    if kind == "forward":
        L.distill_forward(s["logits"], s["teacher"], c["temperature"], s["weight"], s["loss"], s["stats"], s["ws"])
        return {"loss": s["loss"], "stats": s["stats"]}
    if kind == "backward":
        L.distill_backward(s["logits"], s["teacher"], c["temperature"], s["weight"], s["upstream"], s["stats"],
                           s["grad"])
        return {"grad": s["grad"]}
    if kind == "step":
        L.distill_step(s["logits"], s["teacher"], c["temperature"], s["weight"], s["loss"], s["grad"], s["ws"])
        return {"loss": s["loss"], "grad": s["grad"]}
    out = {}
    if kind != "balance_bwd":
        L.balance_forward(s["logits"], s["experts"], s["mask"], c["group"], s["coef"], s["counts"], s["n"], s["prob"],
                          s["loss"], s["ws"])
        out = {"counts": s["counts"], "rows": s["n"], "prob": s["prob"], "loss": s["loss"]}
    if kind != "balance":
        L.balance_backward(s["logits"], c["k"], s["mask"], c["group"], s["coef"], s["counts"], s["n"], s["n"],
                           s["upstream"], s["grad"])
        out["grad"] = s["grad"]
    return out


def _row_softmax(x):
    m = x.max(1, keepdim=True).values
    e = torch.exp(x - m)
    n = e.sum(1, keepdim=True)
    return e / n, m[:, 0], n[:, 0]


def _teacher(s):
    """(the kept entries' places with a last column for none, p, p_rest, the largest entry, the sum of exponentials)"""
    c = s["case"]
    idx = s["idx"].long()
    place = torch.where(idx >= 0, idx, c["cols"])
    entry = torch.where(idx >= 0, s["val"].float() / c["temperature"], float("-inf"))
    p, m, n = _row_softmax(torch.cat([entry, s["rest"][:, None]], 1))
    return place, p[:, :-1], p[:, -1], m, n


def _spread(c, place, value, like):
    """A matrix with `value` at `place`."""
    out = torch.zeros(c["rows"], c["cols"] + 1, dtype=like, device="cuda")
    return out.scatter_(1, place, value)[:, :-1]


def _student(s, place, p_rest):
    """(the exponentials of the row's logits less the largest one, their sum, the sum over the columns not kept, the
    largest logit, the largest one not kept, what a column not kept has for a gradient per exp((z - that) / t))"""
    t = s["case"]["temperature"]
    z = s["logits"].float()
    kept = _spread(s["case"], place, torch.ones_like(place, dtype=torch.bool), torch.bool)
    m = z.max(1).values
    e = torch.exp((z - m[:, None]) / t)
    n = e.sum(1)
    others = torch.where(kept, float("-inf"), z)
    m_tail = others.max(1).values
    tail = torch.exp((others - m_tail[:, None]) / t).sum(1)
    factor = torch.exp((m_tail - m) / t) / n - p_rest / tail
    return kept, m, n, m_tail, tail, factor


def _stats(s, m, n, m_tail, factor, m_t, n_t):
    """What the forward pass saves per row."""
    stats = torch.zeros(s["case"]["rows"], STATS, device="cuda")
    for i, x in enumerate((m, 1.0 / n, m_tail, factor, m_t, 1.0 / n_t)):
        stats[:, i] = torch.where(s["weight"] == 0, 0.0, x)
    return stats


def _saved(s):
    """The saved numbers of a backward pass that is measured by itself."""
    place, _, p_rest, m_t, n_t = _teacher(s)
    _, m, n, m_tail, _, factor = _student(s, place, p_rest)
    return _stats(s, m, n, m_tail, factor, m_t, n_t)


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "top":
        return _plain_top(s)
    if kind in DISTILL:
        return _plain_distill(s)
    out = {}
    counts, n = s.get("counts"), s.get("n")
    if kind != "balance_bwd":
        counts, n = _counts(s)
    p, _, _ = _row_softmax(s["logits"].float())
    f = c["cols"] * counts.float() / (c["k"] * n.clamp(min=1)[:, None])
    if kind != "balance_bwd":
        prob = _group_sum(s, p) / n.clamp(min=1)[:, None]
        loss = s["coef"] / _groups(c) * (f * prob).sum()
        out = {"counts": counts, "rows": n, "prob": prob, "loss": loss[None]}
    if kind != "balance":
        group = torch.arange(c["rows"], device="cuda") // c["group"]
        fr = f[group]
        scale = s["coef"] / (_groups(c) * n.clamp(min=1)) * s["upstream"]
        g = scale[group][:, None] * p * (fr - (fr * p).sum(1, keepdim=True))
        if s["mask"] is not None:
            g = torch.where(s["mask"][:, None], g, 0.0)
        out["grad"] = g.to(DTYPE[c["type"]])
    return out


def _plain_top(s):
    c = s["case"]
    x = s["logits"].float()
    bits = x.contiguous().view(torch.int32).long()
    order = torch.where(x == 0, 0, torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits))  # as the numbers are ordered
    key = order * (1 << 31) + ((1 << 31) - 1 - torch.arange(c["cols"], device="cuda"))  # then the lower column
    idx = torch.topk(key, min(c["k"], c["cols"]), 1).indices
    val = torch.gather(x, 1, idx)
    rest = x.scatter(1, idx, float("-inf")) / c["temperature"]
    m = rest.max(1).values
    rest = m + torch.log(torch.exp(rest - m[:, None]).sum(1))
    return {"idx": torch.where(val == float("-inf"), -1, idx).to(torch.int32), "val": val, "rest": rest}


def _plain_distill(s):
    c = s["case"]
    t, w = c["temperature"], s["weight"]
    out = {}
    place, p, p_rest, m_t, n_t = _teacher(s)
    z = s["logits"].float()
    if c["kind"] == "backward":
        m, inv_n, m_tail, factor = (s["stats"][:, i] for i in range(4))
        kept = _spread(c, place, torch.ones_like(place, dtype=torch.bool), torch.bool)
        w = w * s["upstream"]
    else:
        kept, m, n, m_tail, tail, factor = _student(s, place, p_rest)
        inv_n = 1.0 / n
        there = place < c["cols"]
        zk = torch.gather(z, 1, torch.where(there, place, 0))
        log_n, log_t = torch.log(n), m_t + torch.log(n_t)
        log_q = (zk - m[:, None]) / t - log_n[:, None]
        log_p = torch.where(there, s["val"].float() / t, float("-inf")) - log_t[:, None]
        terms = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
        last = p_rest * (s["rest"] - log_t - (torch.log(tail) + (m_tail - m) / t - log_n))
        out["loss"] = torch.where(w == 0, 0.0, w * (terms + torch.where(p_rest > 0, last, 0.0)))
    if c["kind"] == "forward":
        out["stats"] = _stats(s, m, n, m_tail, factor, m_t, n_t)
        return out
    q = torch.exp((z - m[:, None]) / t) * inv_n[:, None] - _spread(c, place, p, torch.float32)
    others = torch.exp((z - m_tail[:, None]) / t) * factor[:, None]
    g = torch.where(kept, q, others) * (w / t)[:, None]
    out["grad"] = torch.where((w == 0)[:, None], 0.0, g).to(DTYPE[c["type"]])
    return out


def _counts(s):
    """Chosen experts and valid rows of every group."""
    c = s["case"]
    G, E = _groups(c), c["cols"]
    group = torch.arange(c["rows"], device="cuda") // c["group"]
    valid = torch.ones_like(group, dtype=torch.bool) if s["mask"] is None else s["mask"]
    e = s["experts"].long()
    cell = torch.where((e >= 0) & valid[:, None], group[:, None] * E + e, G * E)
    counts = torch.bincount(cell.flatten(), minlength=G * E + 1)[:-1].reshape(G, E)
    return counts.to(torch.int32), torch.bincount(group, valid.double(), minlength=G).to(torch.int32)


def _group_sum(s, p):
    c = s["case"]
    if s["mask"] is not None:
        p = torch.where(s["mask"][:, None], p, 0.0)
    G, short = _groups(c), _groups(c) * c["group"] - c["rows"]
    if short:
        p = torch.cat([p, torch.zeros(short, c["cols"], dtype=p.dtype, device="cuda")])
    return p.reshape(G, c["group"], c["cols"]).sum(1)


def work(case):
    """Bytes that one pass cannot do without, each input read once and each output written once, and the operations
    of its exponentials, sums and products (four for each logit of a softmax, four for its gradient)."""
    c = case
    rows, cols, k, size = c["rows"], c["cols"], c["k"], BYTES[c["type"]]
    live = sum(1 for r in range(rows) if r % 64 < 60) if c["padded_rows"] else rows
    index = 4 if c["index"] == "i32" else 8
    n = float(live) * cols
    if c["kind"] == "top":
        return {"bytes": n * size + rows * (8.0 * k + 4), "flops": 5 * n}
    if c["kind"] in DISTILL:
        payload = live * (k * (index + BYTES[c["values"]]) + 4.0) + 4.0 * rows
        if c["kind"] == "forward":
            return {"bytes": n * size + payload + 4.0 * rows * (1 + STATS), "flops": 4 * n}
        grad = float(rows) * cols * size
        if c["kind"] == "backward":
            return {"bytes": n * size + payload + 4.0 * rows * (1 + STATS) + grad, "flops": 4 * n}
        return {"bytes": n * size + payload + 4.0 * rows + grad, "flops": 8 * n}
    G = _groups(c)
    chosen = float(live) * k * index + (rows if c["padded_rows"] else 0)
    outs = 4.0 * G * (2 * cols + 1)
    grad = float(rows) * cols * size
    if c["kind"] == "balance":
        return {"bytes": n * size + chosen + outs, "flops": 5 * n}
    if c["kind"] == "balance_bwd":
        return {"bytes": n * size + 4.0 * G * (cols + 1) + (rows if c["padded_rows"] else 0) + grad, "flops": 8 * n}
    return {"bytes": n * size + chosen + outs + grad, "flops": 9 * n}


# ---------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["kind"].startswith("balance"):
        return _exact_balance(s)
    parts = []
    step = max(1, (1 << 26) // c["cols"])
    for a in range(0, c["rows"], step):
        part = slice(a, min(c["rows"], a + step))
        parts.append(_exact_top(s, part) if c["kind"] == "top" else _exact_distill(s, part))
    return {key: None if parts[0][key] is None else torch.cat([p[key] for p in parts]) for key in parts[0]}


def _exact_top(s, part):
    c = s["case"]
    x = s["logits"][part].double()
    val, at = torch.sort(x, dim=1, descending=True, stable=True)
    rest = torch.logsumexp(val[:, c["k"]:] / c["temperature"], 1)
    return {"idx": None, "val": val[:, :c["k"]], "rest": rest}


def _exact_distill(s, part):
    c = s["case"]
    t = c["temperature"]
    z = s["logits"][part].double() / t
    idx, w = s["idx"][part].long(), s["weight"][part].double()
    there = idx >= 0
    entry = torch.where(there, s["val"][part].double() / t, float("-inf"))
    log_p = torch.log_softmax(torch.cat([entry, s["rest"][part].double()[:, None]], 1), 1)
    kept = torch.zeros_like(z, dtype=torch.bool)
    target = torch.zeros_like(z)
    row, slot = torch.nonzero(there, as_tuple=True)
    kept[row, idx[row, slot]] = True
    target[row, idx[row, slot]] = torch.exp(log_p[row, slot])
    log_q = torch.log_softmax(z, 1)
    log_tail = torch.logsumexp(torch.where(kept, float("-inf"), log_q), 1)
    p_rest = torch.exp(log_p[:, -1])
    factor = 1.0 - torch.exp(log_p[:, -1] - log_tail)
    live = w != 0
    out = {}
    if c["kind"] != "backward":
        kl = torch.zeros_like(z)
        kl[row, idx[row, slot]] = target[row, idx[row, slot]] * (log_p[row, slot] - log_q[row, idx[row, slot]])
        loss = w * (kl.sum(1) + p_rest * (log_p[:, -1] - log_tail))
        out["loss"] = torch.where(live, loss, 0.0)
    if c["kind"] == "forward":
        m, m_t = z.max(1).values, torch.maximum(entry.max(1).values, s["rest"][part].double())
        log_sum = torch.logsumexp(torch.cat([entry, s["rest"][part].double()[:, None]], 1), 1)
        m_tail = torch.where(kept, float("-inf"), z).max(1).values
        tail = torch.exp(torch.where(kept, float("-inf"), z) - m_tail[:, None]).sum(1)
        cols = [m * t, torch.exp(m - torch.logsumexp(z, 1)), m_tail * t, (torch.exp(log_tail) - p_rest) / tail, m_t,
                torch.exp(m_t - log_sum)]
        stats = torch.stack(cols + [torch.zeros_like(m)] * (STATS - len(cols)), 1)
        out["stats"] = torch.where(live[:, None], stats, 0.0)
        return out
    if c["kind"] == "backward":
        w = w * s["upstream"][part].double()
    q = torch.exp(log_q)
    grad = (w / t)[:, None] * torch.where(kept, q - target, q * factor[:, None])
    out["grad"] = torch.where(live[:, None], grad, 0.0)
    return out


def _exact_balance(s):
    c = s["case"]
    E, k, size, G = c["cols"], c["k"], c["group"], _groups(c)
    valid = torch.ones(c["rows"], dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"]
    prob, loss, grads = [], torch.zeros((), dtype=torch.float64, device="cuda"), []
    for g in range(G):
        part = slice(g * size, min(c["rows"], (g + 1) * size))
        live = valid[part]
        n = max(1, int(live.sum()))
        p = torch.softmax(s["logits"][part].double(), 1)
        p = torch.where(live[:, None], p, 0.0)
        chosen = s["experts"][part][live].flatten()
        f = torch.bincount(chosen[chosen >= 0].long(), minlength=E).double() * E / (k * n)
        prob.append(p.sum(0) / n)
        loss += s["coef"] / G * (f * prob[-1]).sum()
        if c["kind"] != "balance":
            up = s["upstream"].double()
            grads.append(up * s["coef"] / (G * n) * p * (f - (p * f).sum(1, keepdim=True)))
    out = {}
    if c["kind"] != "balance_bwd":
        out = {"counts": None, "rows": None, "prob": torch.stack(prob), "loss": loss[None]}
    if c["kind"] != "balance":
        out["grad"] = torch.cat(grads)
    return out
