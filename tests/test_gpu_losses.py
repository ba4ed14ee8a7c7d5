"""The loss operators on the GPU against their definitions in 64 bits
(tests/_losses_util.py, which also derives the error bounds)."""
import math

import pytest
import torch

import _losses_util as R
from _gpu_util import log
from paper_2102_03112_amd import losses as L

pytestmark = pytest.mark.gpu


def dev(t):
    return None if t is None else t.cuda()


def run_top(x, k, t=1.0, stream=None):
    rows, cols = x.shape
    idx = torch.full((rows, k), -7, dtype=torch.int32, device="cuda")
    val = torch.full((rows, k), 7.0, device="cuda")
    rest = torch.full((rows,), 7.0, device="cuda")
    L.top_logits(x, k, t, idx, val, rest, L.workspace(rows, cols, k), stream)
    return idx, val, rest


def check_top(x, k, t=1.0):
    idx, val, rest = (y.cpu() for y in run_top(x, k, t))
    ridx, rval, rrest = R.top(x.cpu(), k, t)
    assert torch.equal(idx.long(), ridx)
    assert torch.equal(val.double(), rval)
    bound = R.SUM + 2.0 ** -22 * rrest.abs()
    both = torch.isinf(rrest) & (rest.double() == rrest)
    err = torch.where(both, 0.0, (rest.double() - rrest).abs())
    assert bool((err <= torch.where(both, 0.0, bound)).all()), float(err.max())


TOP_SHAPES = [
    (1, 1, 1), (2, 1, 3), (3, 2, 1), (3, 7, 5), (2, 9, 9), (1, 63, 10), (2, 65, 64), (5, 257, 16), (3, 1000, 256),
    (2, 4095, 50), (2, 4096, 50), (2, 4097, 50), (1, 8193, 1), (2, 16385, 100), (1, 33000, 256), (3, 50001, 64),
    (600, 700, 20), (530, 5001, 33), (1, 131073, 64), (1, 300007, 256),
    # rows enough for small blocks
    (512, 3000, 60), (513, 9001, 64), (515, 9001, 65), (512, 13000, 128), (520, 14001, 200),
]


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("rows,cols,k", TOP_SHAPES)
def test_top_logits(rows, cols, k, dtype):
    log("top", rows, cols, k, dtype)
    gen = torch.Generator().manual_seed(rows * 7 + cols)
    check_top((3.0 * torch.randn(rows, cols, generator=gen)).to(dtype).cuda(), k, 0.8 if cols % 2 else 1.0)


# slices of every length, full and nearly so, alone in their row and with others
@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("cols,k", [(18000, 30), (20480, 7), (24577, 100), (32768, 64), (32769, 256), (40960, 50),
                                    (50257, 200), (65535, 1), (65536, 128), (65537, 128), (98000, 64)])
def test_top_long_slices(cols, k, dtype):
    log("top long slices", cols, k, dtype)
    gen = torch.Generator().manual_seed(cols)
    z = (3 * torch.randn(4, cols, generator=gen)).to(dtype)
    z[1, : cols - k // 2] = -math.inf  # fewer than k left, at the row's end
    z[2] = z[2, 0]
    z[3, 1000:] = -math.inf
    check_top(z.cuda(), k, 1.5)


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("kind", ["equal", "few", "zeros", "rising", "falling", "high", "blocks", "peaked", "wide",
                                  "strides"])
@pytest.mark.parametrize("cols,k", [(20, 8), (5003, 64), (40009, 256)])
def test_top_logits_of_awkward_rows(cols, k, kind, dtype):
    """Ties, signed zeros, sorted rows, numbers that crowd into one block's or one wave's part, wide ranges."""
    log("top", kind, cols, k, dtype)
    gen = torch.Generator().manual_seed(5)
    j = torch.arange(cols)
    if kind == "equal":
        x = torch.full((2, cols), 1.25)
    elif kind == "few":  # five values
        x = torch.randint(-2, 3, (2, cols), generator=gen).float()
    elif kind == "zeros":
        x = torch.where(torch.rand(2, cols, generator=gen) < 0.5, 0.0, -0.0)
        x[:, 3::7] = -1.0
    elif kind == "rising":
        x = (j.float() / cols * 8).repeat(2, 1)
    elif kind == "falling":
        x = (-j.float() / cols * 8).repeat(2, 1)
    elif kind == "high":  # a run of high logits
        x = torch.randn(2, cols, generator=gen)
        x[:, cols // 3: cols // 3 + cols // 5] += 20.0
    elif kind == "blocks":  # high ones where one thread or one wave sits
        x = torch.randn(2, cols, generator=gen)
        x[:, (j // 8) % 64 == 5] += 20.0
    elif kind == "peaked":
        x = torch.randn(2, cols, generator=gen) - 300.0
        x[:, : min(cols, k)] += 300.0
    elif kind == "wide":
        x = 1000.0 * torch.randn(2, cols, generator=gen)
    else:
        x = torch.randn(2, cols, generator=gen)
        x[:, ::64] += 10.0
    check_top(x.to(dtype).cuda(), k)


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("cols,k", [(11, 4), (4500, 64), (70001, 100)])
def test_top_logits_of_masked_rows(cols, k, dtype):
    """Rows that a mask leaves nothing, less than k or only one logit, and the type's lowest value as a mask."""
    gen = torch.Generator().manual_seed(9)
    x = torch.randn(7, cols, generator=gen).to(dtype)
    x[0] = -math.inf
    x[1, 1:] = -math.inf
    x[2, : cols - 1] = -math.inf
    x[3, torch.rand(cols, generator=gen) < 0.9] = -math.inf
    x[4] = torch.finfo(dtype).min
    x[5, k // 2:] = torch.finfo(dtype).min
    check_top(x.cuda(), k)


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (3, 5), (0, 1), (7, 64)])
def test_top_logits_of_strided_rows(offset, pad, dtype):
    gen = torch.Generator().manual_seed(11)
    full = torch.randn(6, offset + 5003 + pad, generator=gen).to(dtype).cuda()
    full[:, offset + 5003:] = 1000.0  # never to be seen
    if offset:
        full[:, :offset] = 1000.0
    check_top(full[:, offset:offset + 5003], 40)


def test_top_logits_keep_nonfinite_rows_apart():
    gen = torch.Generator().manual_seed(12)
    for cols in (100, 9000, 70000):
        x = torch.randn(4, cols, generator=gen)
        clean = [y.clone() for y in run_top(x.cuda(), 16)]
        x[1, 5] = math.nan
        x[1, ::3] = math.nan
        x[2] = math.inf
        for got, want in zip(run_top(x.cuda(), 16), clean):
            assert torch.equal(got[[0, 3]], want[[0, 3]])


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------


def loss_bound(w, z, val, t):
    """SUM in each of two logarithms, and 32-bit reciprocals of the temperature times the logits."""
    z = z.double()
    top = val.double().abs().max() + torch.where(torch.isfinite(z), z, 0.0).abs().max()
    return w * (2 * R.SUM + 2.0 ** -22 * top / t)


def check_grad(got, want, scale, dtype, what):
    got, want = got.double().cpu(), want
    bound = 2 * R.SUM * scale + R.ROUND[dtype] * want.abs() + R.TINY[dtype]
    err = (got - want).abs()
    assert bool((err <= bound).all()), (what, float((err - bound).max()), float(want.abs().max()))


def run_distill(z, idx, val, rest, t, weight, upstream=None, place=False):
    """(loss, gradient by forward and backward, loss and gradient by the step)"""
    rows, cols = z.shape
    teacher = L.Teacher(dev(idx), dev(val), dev(rest))
    w, ws = dev(weight), L.workspace(rows, cols, idx.shape[1])
    loss = torch.full((rows,), 7.0, device="cuda")
    stats = torch.full((rows, L.STATS), 7.0, device="cuda")
    L.distill_forward(z, teacher, t, w, loss, stats, ws)
    grad = torch.full_like(z, 7.0, memory_format=torch.contiguous_format)
    L.distill_backward(z, teacher, t, w, dev(upstream), stats, grad)
    loss2 = torch.full((rows,), 7.0, device="cuda")
    if place:
        grad2 = z.clone(memory_format=torch.contiguous_format)
        L.distill_step(grad2, teacher, t, w, loss2, grad2, ws)
        back = z.clone(memory_format=torch.contiguous_format)
        L.distill_backward(back, teacher, t, w, dev(upstream), stats, back)
        assert torch.equal(back, grad)
    else:
        grad2 = torch.full_like(z, 7.0, memory_format=torch.contiguous_format)
        L.distill_step(z, teacher, t, w, loss2, grad2, ws)
    return loss, grad, loss2, grad2


def check_distill(z, idx, val, rest, t, weight=None, upstream=None, place=False):
    dtype = z.dtype
    loss, grad, loss2, grad2 = run_distill(z.cuda() if not z.is_cuda else z, idx, val, rest, t, weight, upstream, place)
    zc = z.cpu()
    want, g1, s1 = R.distill(zc, idx, val, rest, t, weight)
    w = torch.ones(zc.shape[0]) if weight is None else weight.abs()
    bound = loss_bound(w.double(), zc, torch.where((idx >= 0) & torch.isfinite(val.float()), val.float(), 0.0), t)
    for got in (loss, loss2):
        got = got.double().cpu()
        inf = torch.isinf(want)
        assert torch.equal(got[inf], want[inf])
        err = (got - want).abs()[~inf]
        assert bool((err <= bound[~inf] + 2.0 ** -23 * want[~inf].abs()).all()), (float(err.max()), float(bound.max()))
    check_grad(grad2, g1, s1, dtype, "step")
    if upstream is not None:
        _, g1, s1 = R.distill(zc, idx, val, rest, t, weight, upstream)
    check_grad(grad, g1, s1, dtype, "backward")


DISTILL_SHAPES = [
    (1, 1, 1), (2, 2, 1), (3, 5, 5), (4, 9, 3), (2, 64, 8), (3, 255, 255), (2, 1000, 64), (3, 2047, 100),
    (3, 2048, 100), (3, 2049, 100), (2, 16384, 50), (2, 16385, 50), (5, 20011, 256), (300, 300, 20), (260, 2100, 7),
    (2, 40000, 1000), (1, 131072, 64), (2, 140001, 32),
    # rows enough for a block each, of lengths that take other blocks, one and several rounds of them
    (130, 520, 9), (128, 4097, 30), (131, 8200, 16), (128, 16400, 300), (129, 33000, 12), (128, 70003, 40),
]


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("rows,cols,k", DISTILL_SHAPES)
def test_distill(rows, cols, k, dtype):
    log("distill", rows, cols, k, dtype)
    t = [1.0, 2.0, 0.7][(rows + cols) % 3]
    z, idx, val, rest = R.student(rows, cols, k, dtype, 31 + rows + cols, t)
    gen = torch.Generator().manual_seed(3)
    weight = torch.rand(rows, generator=gen) + 0.25
    weight[rows // 2:: 5] = 0.0
    check_distill(z, idx, val, rest, t, weight, torch.rand(rows, generator=gen) + 0.5, place=cols % 2 == 0)


@pytest.mark.parametrize("index", [torch.int32, torch.int64])
@pytest.mark.parametrize("values", R.TYPES)
def test_distill_types_of_the_payload(values, index):
    z, idx, val, rest = R.student(6, 3001, 40, torch.bfloat16, 17)
    wide_idx = torch.zeros(6, 47, dtype=index)
    wide_idx[:, :40] = idx
    wide_val = torch.zeros(6, 53, dtype=values)
    wide_val[:, :40] = val
    idx_d, val_d = wide_idx.cuda()[:, :40], wide_val.cuda()[:, :40]
    zd = z.cuda()
    loss = torch.zeros(6, device="cuda")
    grad = torch.zeros_like(zd)
    L.distill_step(zd, L.Teacher(idx_d, val_d, rest.cuda()), 1.0, None, loss, grad, L.workspace(6, 3001, 40))
    want, g, s = R.distill(z, idx, val.to(values), rest, 1.0)
    assert bool(((loss.double().cpu() - want).abs() <= loss_bound(1.0, z, val, 1.0)).all())
    check_grad(grad, g, s, torch.bfloat16, "payload types")


@pytest.mark.parametrize("dtype", R.TYPES)
def test_distill_rows_with_missing_entries(dtype):
    """Ragged and empty payloads, no rest, columns out of range in both directions, kept columns of no probability."""
    rows, cols, k = 9, 2500, 24
    z, idx, val, rest = R.student(rows, cols, k, dtype, 23)
    idx[0, 5:] = -1
    idx[1] = -1                      # no entry, a finite rest: p_rest = q_rest = 1
    idx[2] = -1
    rest[2] = -math.inf              # no distribution at all
    rest[3] = -math.inf              # the kept ones are everything
    idx[4, 3], idx[4, 4] = cols, cols + 100
    val[5, 0] = -math.inf            # a kept column of p = 0
    val[6, 7:] = math.nan            # not entries: their logits are not used
    idx[6, 7:] = -3
    rest[7] = 60.0                   # nearly all in the rest
    check_distill(z, idx, val, rest, 1.0)
    rest[:] = -math.inf
    check_distill(z, idx, val, rest, 2.0)
    loss, grad, _, _ = run_distill(z.cuda(), idx, val, None, 2.0, None)
    again, g2, _, _ = run_distill(z.cuda(), idx, val, rest, 2.0, None)
    assert torch.equal(loss, again) and torch.equal(grad, g2)


@pytest.mark.parametrize("dtype", R.TYPES)
def test_distill_masked_students(dtype):
    """-inf and the type's lowest value in a student's row: columns not kept, kept ones, whole rows."""
    rows, cols, k = 8, 3000, 16
    z, idx, val, rest = R.student(rows, cols, k, dtype, 29)
    low = torch.finfo(dtype).min
    kept = torch.zeros(rows, cols, dtype=torch.bool).scatter_(1, idx.long(), True)
    others = torch.nonzero(~kept[0])[:, 0]
    z[0, others[::2]] = -math.inf
    z[1, ~kept[1]] = low
    z[2, ~kept[2]] = -math.inf       # q_rest = 0 with p_rest > 0: loss +inf
    z[3, idx[3, 2].long()] = -math.inf  # a kept column without probability: loss +inf
    z[4] = -math.inf                 # nothing left
    z[5] = low                       # all alike
    z[6, ~kept[6]] = -math.inf
    rest[6] = -math.inf              # q_rest = p_rest = 0: finite
    check_distill(z, idx, val, rest, 1.0)


def test_distill_where_the_kept_columns_hold_nearly_everything():
    """q_rest far below a 32-bit sum's last place, and below the smallest number: no difference of sums takes part."""
    for gap in (15.0, 60.0, 200.0):
        z, idx, val, rest = R.student(4, 5000, 8, torch.float32, 37)
        kept = torch.zeros(4, 5000, dtype=torch.bool).scatter_(1, idx.long(), True)
        z = torch.where(kept, z + gap, z)
        check_distill(z, idx, val, rest, 1.0)


def test_distill_does_not_read_rows_of_no_weight():
    z, idx, val, rest = R.student(6, 2300, 20, torch.bfloat16, 41)
    weight = torch.tensor([1.0, 0.0, 0.5, 0.0, -0.0, 2.0])
    z[weight == 0] = math.nan
    val[weight == 0] = math.nan
    rest[weight == 0] = math.nan
    check_distill(z, idx, val, rest, 1.0, weight, place=True)
    loss, grad, loss2, grad2 = run_distill(z.cuda(), idx, val, rest, 1.0, weight)
    for x in (loss, loss2):
        assert torch.equal(x[[1, 3, 4]].cpu(), torch.zeros(3))
    for g in (grad, grad2):
        assert bool((g[[1, 3, 4]] == 0).all())


def test_distill_keeps_nonfinite_rows_apart():
    z, idx, val, rest = R.student(5, 2600, 20, torch.float32, 43)
    clean = run_distill(z.cuda(), idx, val, rest, 1.0, None)
    z[1, ::5] = math.nan
    z[3, 7] = math.inf
    for got, want in zip(run_distill(z.cuda(), idx, val, rest, 1.0, None), clean):
        assert torch.equal(got[[0, 2, 4]], want[[0, 2, 4]])


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("offset,pad", [(1, 0), (0, 3), (5, 6)])
def test_distill_strided(offset, pad, dtype):
    """Rows cut out of wider matrices, and gradients written into one: nothing beside the rows changes."""
    z, idx, val, rest = R.student(5, 2501, 30, dtype, 47)
    full = torch.full((5, offset + 2501 + pad), math.nan, dtype=dtype, device="cuda")
    full[:, offset:offset + 2501] = z.cuda()
    view = full[:, offset:offset + 2501]
    check_distill(view, idx, val, rest, 1.0)
    out = torch.full((5, 3 + 2501 + 2), 5.0, dtype=dtype, device="cuda")
    loss = torch.zeros(5, device="cuda")
    teacher = L.Teacher(idx.cuda(), val.cuda(), rest.cuda())
    L.distill_step(view, teacher, 1.0, None, loss, out[:, 3:2504], L.workspace(5, 2501, 30))
    _, g, s = R.distill(z, idx, val, rest, 1.0)
    check_grad(out[:, 3:2504], g, s, dtype, "strided")
    assert bool((out[:, :3] == 5).all()) and bool((out[:, 2504:] == 5).all())
    stats = torch.zeros(5, L.STATS, device="cuda")
    L.distill_forward(view, teacher, 1.0, None, loss, stats, L.workspace(5, 2501, 30))
    L.distill_backward(view, teacher, 1.0, None, None, stats, view)  # in its own place
    check_grad(view, g, s, dtype, "in place")
    assert bool(torch.isnan(full[:, :offset]).all()) and bool(torch.isnan(full[:, offset + 2501:]).all())


def test_distill_upstream_may_be_an_expanded_scalar():
    z, idx, val, rest = R.student(7, 900, 12, torch.float32, 53)
    zd = z.cuda()
    teacher = L.Teacher(idx.cuda(), val.cuda(), rest.cuda())
    loss, stats = torch.zeros(7, device="cuda"), torch.zeros(7, L.STATS, device="cuda")
    L.distill_forward(zd, teacher, 1.0, None, loss, stats, L.workspace(7, 900, 12))
    a, b = torch.zeros_like(zd), torch.zeros_like(zd)
    L.distill_backward(zd, teacher, 1.0, None, torch.full((7,), 0.3, device="cuda"), stats, a)
    L.distill_backward(zd, teacher, 1.0, None, torch.full((1,), 0.3, device="cuda").expand(7), stats, b)
    assert torch.equal(a, b)
    strided = torch.full((14,), 9.0, device="cuda")
    strided[::2] = 0.3
    L.distill_backward(zd, teacher, 1.0, None, strided[::2], stats, b)
    assert torch.equal(a, b)


def test_distill_gradient_against_differences():
    """The kernel's gradient against differences of the kernel's loss along random directions."""
    rows, cols, k = 4, 700, 16
    z, idx, val, rest = R.student(rows, cols, k, torch.float32, 59)
    loss, grad, _, _ = run_distill(z.cuda(), idx, val, rest, 1.0, None)
    gen = torch.Generator().manual_seed(61)
    for _ in range(4):
        d = torch.randn(rows, cols, generator=gen)
        h = 2.0 ** -5
        up = run_distill((z + h * d).cuda(), idx, val, rest, 1.0, None)[0].double()
        down = run_distill((z - h * d).cuda(), idx, val, rest, 1.0, None)[0].double()
        slope = ((up - down) / (2 * h)).cpu()
        want = (grad.double().cpu() * d).sum(1)
        # third derivatives of a log-sum-exp along d are at most 4 max|d|^3 E|d - E d|...: below 1 x spread^3
        # for the q- and p-weighted spreads here; the loss's own error is 2 SUM + 2^-22 x 20 at each end
        third = 8.0
        assert bool(((slope - want).abs() <= h * h / 6 * third + (2 * R.SUM + 5e-6) / h).all())


def test_one_label_is_cross_entropy():
    gen = torch.Generator().manual_seed(67)
    z = torch.randn(50, 1003, generator=gen)
    label = torch.randint(0, 1003, (50,), generator=gen)
    loss, grad, _, _ = run_distill(z.cuda(), label[:, None], torch.zeros(50, 1), None, 1.0, None)
    want = torch.nn.functional.cross_entropy(z.double(), label, reduction="none")
    assert bool(((loss.double().cpu() - want).abs() <= 2 * R.SUM + 5e-6).all())
    p = torch.softmax(z.double(), 1)
    g = p - torch.nn.functional.one_hot(label, 1003)
    assert bool(((grad.double().cpu() - g).abs() <= 4 * R.SUM * p + 2e-7).all())


def test_a_teachers_payload_against_its_full_distribution():
    """The payload of dr_top_logits gives a student the exact coarse divergence, 0 for the teacher itself."""
    gen = torch.Generator().manual_seed(71)
    x = (3.0 * torch.randn(20, 5000, generator=gen)).to(torch.bfloat16).cuda()
    idx, val, rest = run_top(x, 50, 2.0)
    loss, grad, _, _ = run_distill(x, idx.cpu(), val.cpu(), rest.cpu(), 2.0, None)
    assert float(loss.abs().max()) <= 2 * R.SUM + 5e-6
    assert float(grad.abs().max()) <= 4 * R.SUM


# ---------------------------------------------------------------------------
# balance loss
# ---------------------------------------------------------------------------


def run_balance(z, experts, mask, group, coef, upstream=None):
    T, E = z.shape
    G = -(-T // group)
    counts = torch.full((G, E), -7, dtype=torch.int32, device="cuda")
    n = torch.full((G,), -7, dtype=torch.int32, device="cuda")
    prob = torch.full((G, E), 7.0, device="cuda")
    loss = torch.full((1,), 7.0, device="cuda")
    L.balance_forward(z, dev(experts), dev(mask), group, coef, counts, n, prob, loss, L.workspace(T, E, 1))
    grad = torch.full_like(z, 7.0, memory_format=torch.contiguous_format)
    L.balance_backward(z, experts.shape[1], dev(mask), group, coef, counts, n, n, dev(upstream), grad)
    return counts, n, prob, loss, grad


def check_balance(z, experts, mask, group, coef=0.01, upstream=None):
    k = experts.shape[1]
    counts, n, prob, loss, grad = run_balance(z, experts, mask, group, coef, upstream)
    u = 1.0 if upstream is None else float(upstream)
    c, rn, p, l, g, s = R.balance(z.cpu(), experts, k, mask, group, coef, u)
    assert torch.equal(counts.long().cpu(), c) and torch.equal(n.long().cpu(), rn)
    assert bool(((prob.double().cpu() - p).abs() <= 2 * R.SUM * p + 1e-37).all())
    assert abs(float(loss) - l) <= 3 * R.SUM * abs(l)
    check_grad(grad, g, s, z.dtype, "balance")


BALANCE_SHAPES = [  # rows, experts, chosen, rows a group
    (1, 1, 1, 1), (5, 1, 1, 2), (7, 3, 2, 7), (64, 8, 2, 64), (65, 8, 8, 64), (130, 16, 4, 33), (257, 60, 6, 257),
    (1000, 64, 6, 1000), (999, 100, 3, 100), (300, 256, 8, 300), (700, 257, 5, 64), (120, 520, 7, 120),
    (90, 1024, 16, 45), (5000, 8, 2, 5000), (4100, 128, 4, 1025), (3000, 32, 4, 7), (2500, 5, 2, 1),
]


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("T,E,k,group", BALANCE_SHAPES)
def test_balance(T, E, k, group, dtype):
    log("balance", T, E, k, group, dtype)
    gen = torch.Generator().manual_seed(T + E)
    z = (1.5 * torch.randn(T, E, generator=gen)).to(dtype)
    experts = torch.topk(z.float() + torch.randn(E, generator=gen), k, 1).indices
    mask = torch.rand(T, generator=gen) < 0.8 if T % 2 else None
    if T % 3 == 0:
        experts = torch.where(torch.rand(T, k, generator=gen) < 0.1, -1, experts)
    # half precision: coef such that gradients stay in range
    coef = 100.0 if dtype == torch.float16 else 0.01
    check_balance(z.cuda(), experts if E % 2 else experts.int(), mask, group, coef, torch.tensor([0.7]))


# every way that a row's vectors lie over lanes; one group, and several of which each has blocks of its own
@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("group", [611, 150])
@pytest.mark.parametrize("E", [40, 90, 120, 180, 250, 380, 500, 700, 768, 1000])
def test_balance_layouts(E, group, dtype):
    log("balance layouts", E, group, dtype)
    gen = torch.Generator().manual_seed(E + group)
    z = (1.5 * torch.randn(611, E, generator=gen)).to(dtype)
    experts = torch.topk(z.float() + torch.randn(E, generator=gen), 4, 1).indices
    coef = 100.0 if dtype == torch.float16 else 0.01
    check_balance(z.cuda(), experts, torch.rand(611, generator=gen) < 0.9, group, coef, torch.tensor([0.7]))


@pytest.mark.parametrize("dtype", R.TYPES)
def test_balance_masks(dtype):
    """Padding that holds NaN, whole groups of padding, masked experts, rows without any expert."""
    gen = torch.Generator().manual_seed(73)
    T, E, group = 200, 24, 40
    z = torch.randn(T, E, generator=gen).to(dtype)
    experts = torch.randint(0, E, (T, 3), generator=gen)
    mask = torch.rand(T, generator=gen) < 0.7
    mask[80:120] = False
    z[~mask] = math.nan
    z[:, 5] = torch.where(mask, -math.inf, math.nan).to(dtype)
    live = torch.nonzero(mask)[:, 0]
    z[live[3]] = -math.inf
    z[live[4]] = torch.finfo(dtype).min
    z[live[5], 1:] = torch.finfo(dtype).min
    experts[live[6]] = torch.tensor([-1, E, E + 1000])  # none of them an expert
    check_balance(z.cuda(), experts, mask, group, 1.0)
    check_balance(z.cuda(), experts, mask.to(torch.uint8) * 3, T, 1.0)
    check_balance(z.cuda(), experts, torch.zeros(T, dtype=torch.bool), group, 1.0)


def test_balance_strided():
    gen = torch.Generator().manual_seed(79)
    for dtype in R.TYPES:
        full = torch.randn(150, 75, generator=gen).to(dtype).cuda()
        full[:, 65:] = math.nan
        full[:, 0] = math.nan
        wide = torch.randint(0, 64, (150, 9), generator=gen).cuda()
        z, experts = full[:, 1:65], wide[:, 2:6]
        counts = torch.zeros(1, 64, dtype=torch.int32, device="cuda")
        n, loss = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda")
        L.balance_forward(z, experts, None, 150, 1.0, counts, n, None, loss, L.workspace(150, 64, 1))
        c, rn, _, l, g, s = R.balance(z.cpu(), experts.cpu(), 4, None, 150, 1.0)
        assert torch.equal(counts.long().cpu(), c) and abs(float(loss) - l) <= 3 * R.SUM * abs(l)
        out = torch.full((150, 80), 5.0, dtype=dtype, device="cuda")
        L.balance_backward(z, 4, None, 150, 1.0, counts, n, n, None, out[:, 7:71])
        check_grad(out[:, 7:71], g, s, dtype, "strided")
        assert bool((out[:, :7] == 5).all()) and bool((out[:, 71:] == 5).all())
        L.balance_backward(z, 4, None, 150, 1.0, counts, n, n, None, z)  # in its own place
        check_grad(z, g, s, dtype, "in place")
        assert bool(torch.isnan(full[:, 65:]).all()) and bool(torch.isnan(full[:, 0]).all())


def test_balance_over_the_global_batch():
    """Two workers' rows with summed counts: the mean of their gradients is the joint batch's."""
    gen = torch.Generator().manual_seed(83)
    z = torch.randn(400, 32, generator=gen)
    experts = torch.randint(0, 32, (400, 4), generator=gen)
    halves = [run_balance(z[h].cuda(), experts[h], None, 200, 1.0) for h in (slice(0, 200), slice(200, 400))]
    counts = halves[0][0] + halves[1][0]
    rows = halves[0][1] + halves[1][1]
    _, _, _, want, g, s = R.balance(z, experts, 4, None, 400, 1.0)
    f = 32.0 * counts.double() / (4 * rows.double())
    loss = sum((f * h[2].double()).sum() for h in halves) / 2
    assert abs(float(loss) - want) <= 3 * R.SUM * abs(want)
    for i, h in enumerate((slice(0, 200), slice(200, 400))):
        grad = torch.zeros(200, 32, device="cuda")
        L.balance_backward(z[h].cuda(), 4, None, 200, 1.0, counts, rows, halves[i][1], None, grad)
        check_grad(grad / 2, g[h], s[h], torch.float32, "global")


def test_balance_gradient_against_differences():
    """Against differences of the definition's loss in 64 bits, the counts held."""
    gen = torch.Generator().manual_seed(89)
    z = torch.randn(30, 12, generator=gen)
    experts = torch.randint(0, 12, (30, 3), generator=gen)
    grad = run_balance(z.cuda(), experts, None, 11, 1.0)[4].double().cpu()
    for _ in range(4):
        d = torch.randn(30, 12, generator=gen).double()
        h = 1e-4
        up, down = (R.balance(z.double() + s * h * d, experts, 3, None, 11, 1.0)[3] for s in (1, -1))
        # a difference in 64 bits is off by h^2 times third derivatives (below 10 here) and 1e-16 / h
        assert abs((up - down) / (2 * h) - float((grad * d).sum())) <= 1e-7 + R.SUM * float((grad * d).abs().sum())


# ---------------------------------------------------------------------------
# streams, graphs, repeated calls
# ---------------------------------------------------------------------------


def _everything(seed):
    """Inputs, and a call of every operator on them into fixed buffers."""
    z, idx, val, rest = R.student(40, 9001, 32, torch.bfloat16, seed)
    gen = torch.Generator().manual_seed(seed)
    zd = z.cuda()
    router = torch.randn(4000, 64, generator=gen).cuda()
    experts = torch.randint(0, 64, (4000, 4), generator=gen).cuda()
    weight = torch.rand(40, generator=gen).cuda()
    teacher = L.Teacher(idx.cuda(), val.cuda(), rest.cuda())
    e = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    out = dict(tidx=e(40, 32, t=torch.int32), tval=e(40, 32), trest=e(40), loss=e(40), stats=e(40, L.STATS),
               grad=torch.zeros_like(zd), loss2=e(40), grad2=torch.zeros_like(zd), counts=e(4, 64, t=torch.int32),
               n=e(4, t=torch.int32), prob=e(4, 64), bal=e(1), rgrad=torch.zeros_like(router))
    ws = [L.workspace(40, 9001, 32), L.workspace(4000, 64, 1)]

    def call(stream=None):
        L.top_logits(zd, 32, 1.0, out["tidx"], out["tval"], out["trest"], ws[0], stream)
        L.distill_forward(zd, teacher, 1.0, weight, out["loss"], out["stats"], ws[0], stream)
        L.distill_backward(zd, teacher, 1.0, weight, None, out["stats"], out["grad"], stream)
        L.distill_step(zd, teacher, 1.0, weight, out["loss2"], out["grad2"], ws[0], stream)
        L.balance_forward(router, experts, None, 1000, 0.1, out["counts"], out["n"], out["prob"], out["bal"], ws[1],
                          stream)
        L.balance_backward(router, 4, None, 1000, 0.1, out["counts"], out["n"], out["n"], None, out["rgrad"], stream)

    return call, out, zd, router


def test_calls_repeat_bit_for_bit():
    call, out, _, _ = _everything(97)
    call()
    first = {k: v.clone() for k, v in out.items()}
    for _ in range(3):
        for v in out.values():
            v.fill_(3)
        call()
        for k, v in out.items():
            assert torch.equal(v, first[k]), k


def test_calls_on_a_stream_of_their_own():
    call, out, _, _ = _everything(101)
    call()
    torch.cuda.synchronize()
    first = {k: v.clone() for k, v in out.items()}
    for v in out.values():
        v.fill_(3)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    call(s)
    s.synchronize()
    for k, v in out.items():
        assert torch.equal(v, first[k]), k


def test_calls_replayed_from_a_graph():
    call, out, zd, router = _everything(103)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        zd.add_(0.125 * i)
        zd[:, i::7] -= 0.5
        router.mul_(1.0 + 0.1 * i)
        for v in out.values():
            v.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in out.items()}
        call()
        torch.cuda.synchronize()
        for k, v in out.items():
            assert torch.equal(v, got[k]), (i, k)


def test_no_rows():
    z = torch.zeros(0, 100, device="cuda")
    empty = torch.zeros(0, 4, device="cuda")
    L.top_logits(z, 4, 1.0, empty.int(), empty, empty[:, 0].contiguous(), L.workspace(0, 100, 4))
    teacher = L.Teacher(empty.int(), empty, None)
    L.distill_step(z, teacher, 1.0, None, empty[:, 0].contiguous(), z, L.workspace(0, 100, 4))
    loss = torch.full((1,), 7.0, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    L.balance_forward(z, empty.int(), None, 5, 1.0, none, none, None, loss, L.workspace(0, 100, 1))
    L.balance_backward(z, 4, None, 5, 1.0, none, none, none, None, z)
    assert float(loss) == 0.0


def test_results_do_not_hang_on_the_workspace():
    """Scratch is undefined between calls: filled with what would show."""
    z, idx, val, rest = R.student(30, 40000, 20, torch.float16, 107)
    zd, teacher = z.cuda(), L.Teacher(idx.cuda(), val.cuda(), rest.cuda())
    ws = L.workspace(30, 40000, 20)
    seen = []
    for fill in (0, 255, 127):
        ws.fill_(fill)
        loss, grad = torch.zeros(30, device="cuda"), torch.zeros_like(zd)
        L.distill_step(zd, teacher, 1.0, None, loss, grad, ws)
        ws.fill_(fill)
        ti, tv, tr = torch.zeros(30, 20, dtype=torch.int32, device="cuda"), torch.zeros(30, 20, device="cuda"), loss * 0
        L.top_logits(zd, 20, 1.0, ti, tv, tr, ws)
        seen.append((loss, grad, ti, tv, tr))
    for other in seen[1:]:
        for a, b in zip(seen[0], other):
            assert torch.equal(a, b)


def test_matrices_of_more_than_2_to_the_32_numbers():
    """The last rows of a matrix whose offsets pass 32 bits, against the same rows by themselves: the same kernels, so
    the same bits."""
    rows, cols, k, few = 33_000, 131_072, 8, 200
    gen = torch.Generator(device="cuda").manual_seed(109)
    z = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    assert rows * cols > 1 << 32
    z[-few:] = 3.0 * torch.randn(few, cols, generator=gen, device="cuda")
    z[:few] = torch.randn(few, cols, generator=gen, device="cuda")
    last = z[-few:].clone()
    big, small = run_top(z, k), run_top(last, k)
    for a, b in zip(big, small):
        assert torch.equal(a[-few:], b)
    weight = torch.zeros(rows, device="cuda")
    weight[-few:] = 1.0
    loss, part = torch.full((rows,), 7.0, device="cuda"), torch.full((few,), 7.0, device="cuda")
    grad = torch.zeros_like(last)
    L.distill_step(last, L.Teacher(*small), 1.0, None, part, grad, L.workspace(few, cols, k))
    L.distill_step(z, L.Teacher(*big), 1.0, weight, loss, z, L.workspace(rows, cols, k))
    assert torch.equal(loss[-few:], part) and torch.equal(z[-few:], grad)
    assert float(loss[:-few].abs().max()) == 0.0 and float(z[:few].abs().max()) == 0.0
