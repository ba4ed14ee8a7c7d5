"""The loss operators at the edges of their contract: logits near a type's
largest numbers, masks of its lowest one, sizes at the ends of their ranges,
sums of very different parts.  Definitions and bounds: tests/_losses_util.py."""
import math

import pytest
import torch

import _losses_util as R
from _gpu_util import log
from paper_2102_03112_amd import losses as L
from test_gpu_losses import check_balance, check_distill, check_grad, check_top, run_balance, run_distill, run_top

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("cols", [1, 2, 7, 31, 33, 65, 255, 257, 513, 1025, 2049, 4100])
def test_distill_short_rows_of_one_entry(cols, dtype):
    """Rows that end anywhere in a block's step, with one kept column: the bitmap's last step and nearly no entries
    behind it."""
    log("short rows", cols, dtype)
    z, idx, val, rest = R.student(200, cols, 1, dtype, 211 + cols)
    check_distill(z, idx, val, rest if cols > 1 else None, 1.0)


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("cols,k", [(40_000, 2), (131_072, 8), (200_001, 64), (300_007, 12)])
@pytest.mark.parametrize("background", [0.0, -math.inf])
def test_top_rest_far_below_kept_logits_of_every_slice(cols, k, background, dtype):
    """K high logits spread evenly, so that every slice keeps its share, and the next ones far below them: what the
    slices' lists hold beyond the K is nearly nothing beside them, and all that the rest is made of."""
    log("top spread", cols, k, background, dtype)
    for gap, t in ((100.0, 1.0), (150.0, 1.0), (300.0, 1.0), (30.0, 0.1), (600.0, 2.0)):
        x = torch.full((3, cols), background)
        x[:, ((torch.arange(k) + 0.5) * cols / k).long()] = 400.0
        x[0, 1] = 400.0 - gap
        x[1, 1], x[1, cols - 1] = 400.0 - gap, 399.0 - gap
        x[2, torch.arange(k) * (cols // k) + 1] = 400.0 - gap  # one more in every part
        check_top(x.to(dtype).cuda(), k, t)


LARGE = [2.7e36, 3e36, 5e36, 1e37, 4e37, 4.3e37, 1e38, 3.38e38]


@pytest.mark.parametrize("cols,k", [(11, 4), (4500, 64), (70_001, 100)])
def test_top_of_large_bfloat16(cols, k):
    """Magnitudes whose bits would be no numbers in float16: rows of one, of several, among ordinary ones, and of
    either sign."""
    log("top large", cols, k)
    gen = torch.Generator().manual_seed(311)
    size = torch.tensor(LARGE)
    rows = [torch.full((cols,), s * v) for v in LARGE for s in (1.0, -1.0)]
    pick = size[torch.randint(0, len(LARGE), (6, cols), generator=gen)]
    sign = torch.where(torch.rand(6, cols, generator=gen) < 0.5, -1.0, 1.0)
    small = 3.0 * torch.randn(6, cols, generator=gen)
    rows += [pick[0], -pick[1], pick[2] * sign[2], torch.where(sign[3] > 0, pick[3], small[3]),
             torch.where(sign[4] > 0, -pick[4], small[4]), 2.0 ** (120 + 7 * torch.rand(cols, generator=gen))]
    check_top(torch.stack(rows).to(BF16).cuda(), k)


def check_step(z, idx, val, rest, t, size, weight=None):
    """Losses and gradients of all calls against the definition; size: the magnitude of the logits that the loss is
    made of, masked ones apart."""
    loss, grad, loss2, grad2 = run_distill(z.cuda(), idx, val, rest, t, weight)
    want, g, s = R.distill(z, idx, val, rest, t, weight)
    w = 1.0 if weight is None else weight.abs().double()
    bound = w * (2 * R.SUM + 2.0 ** -22 * size / t) + (2 * R.SUM + 2.0 ** -22) * want.abs()
    for got in (loss, loss2):
        got = got.double().cpu()
        inf = torch.isinf(want)
        assert torch.equal(got[inf], want[inf])
        assert bool(((got - want).abs()[~inf] <= bound.expand_as(want)[~inf]).all()), (got, want)
    check_grad(grad, g, s, z.dtype, "backward")
    check_grad(grad2, g, s, z.dtype, "step")


@pytest.mark.parametrize("rows,cols", [(3, 3000), (3, 20_000), (2, 70_001), (130, 20_000)])
def test_distill_bfloat16_masked_with_large_numbers(rows, cols):
    """Columns masked with a large negative number, among them the last ones of every thread."""
    log("distill masked with large", rows, cols)
    z, idx, val, rest = R.student(rows, cols, 20, BF16, 313)
    weight = torch.zeros(rows)
    weight[:3] = 1.0
    for mask in [-1e9, -1e30] + [-v for v in LARGE] + [torch.finfo(BF16).min]:
        x = z.clone()
        kept = torch.zeros(rows, cols, dtype=torch.bool).scatter_(1, idx.long(), True)
        x[:, -2048:] = torch.where(kept, x, mask)[:, -2048:].to(BF16)
        x[0] = torch.where(kept[0] | (torch.arange(cols) % 3 == 0), x[0].float(), mask).to(BF16)
        check_step(x, idx, val, rest, 1.0, 40.0, weight)


@pytest.mark.parametrize("cols", [3000, 20_000, 70_001])
def test_distill_large_bfloat16(cols):
    """Large numbers on both sides: kept ones, others, all."""
    log("distill large", cols)
    gen = torch.Generator().manual_seed(317)
    for v in LARGE[:6]:
        z, idx, val, rest = R.student(4, cols, 20, BF16, 319)
        kept = torch.zeros(4, cols, dtype=torch.bool).scatter_(1, idx.long(), True)
        z[0, 5 if not kept[0, 5] else 6] = v
        z[1] = torch.where(kept[1], z[1].float(), -v * (0.5 + 0.5 * torch.rand(cols, generator=gen))).to(BF16)
        z[2] = torch.where(kept[2], z[2].float(), v * torch.ones(cols)).to(BF16)
        z[3] = -v
        check_step(z, idx, val, rest, 1.0, 2 * v)


def test_distill_row_of_more_than_2_to_the_32_bytes():
    """One fp32 row of 2^30 and some columns, whose bytes pass 32 bits: loss and gradient against sums in 64 bits."""
    cols, parts = (1 << 30) + 5, 64
    gen = torch.Generator(device="cuda").manual_seed(331)
    z = torch.empty(1, cols, device="cuda")
    for a in range(0, cols, 1 << 26):
        n = min(1 << 26, cols - a)
        z[0, a:a + n] = torch.randn(n, generator=gen, device="cuda")
    idx = torch.tensor([[3, 1 << 29, cols - 1]], dtype=torch.int32, device="cuda")
    z[0, idx[0].long()] = torch.tensor([20.0, 19.0, 21.5], device="cuda")
    val, rest = torch.tensor([[5.0, 4.0, 6.0]], device="cuda"), torch.tensor([4.5], device="cuda")
    log("2^30 columns")
    loss, stats = torch.zeros(1, device="cuda"), torch.zeros(1, L.STATS, device="cuda")
    grad, ws, teacher = torch.empty_like(z), L.workspace(1, cols, 3), L.Teacher(idx, val, rest)
    L.distill_forward(z, teacher, 1.0, None, loss, stats, ws)
    L.distill_step(z, teacher, 1.0, None, loss, grad, ws)
    total = sum(float(torch.exp(c.double()).sum()) for c in torch.chunk(z[0], parts))
    kept = z[0, idx[0].long()].double().cpu()
    tail = total - float(torch.exp(kept).sum())
    p = torch.softmax(torch.cat([val[0], rest]).double().cpu(), 0)
    q = torch.cat([torch.exp(kept), torch.tensor([tail], dtype=torch.float64)]) / total
    assert abs(float(loss) - float((p * (torch.log(p) - torch.log(q))).sum())) <= 2 * R.SUM + 2.0 ** -22 * 22
    got = grad[0, idx[0].long()].double().cpu()
    assert bool(((got - (q - p)[:3]).abs() <= 2 * R.SUM * (q + p)[:3] + 2.0 ** -23).all())
    factor = (float(q[3]) - float(p[3])) / tail
    for a in (0, 4, (1 << 29) + 1, cols - 1001):  # where no column is kept
        want = torch.exp(z[0, a:a + 1000].double()) * factor
        if a == 0:
            want[3] = grad[0, 3].double()
        bound = 2 * R.SUM * torch.exp(z[0, a:a + 1000].double()) * (float(q[3]) + float(p[3])) / tail
        assert bool(((grad[0, a:a + 1000].double() - want).abs() <= bound + 2.0 ** -23 * want.abs()).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [900, 9000, 20_000])
def test_distill_where_a_kept_logit_is_large(cols, dtype):
    """A kept logit so large that no other has a probability: the loss is finite, p_rest times the distance."""
    log("large kept", cols, dtype)
    for v in (1e31, 3e36, 1e37):
        z, idx, val, rest = R.student(130, cols, 20, dtype, 337)
        z.scatter_(1, idx[:, :1].long(), v)
        weight = torch.zeros(130)
        weight[:4] = 1.0
        z[1] = z[1].float().abs().clamp(max=3.0).to(dtype)  # and one row as usual
        z[2, idx[2, 1].long()] = v / 2
        check_step(z, idx, val, rest, 1.0, 40.0, weight)


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("values", R.TYPES)
@pytest.mark.parametrize("cols", [700, 40_000])
def test_distill_of_rows_masked_with_the_lowest_number(cols, values, dtype):
    """A whole row of a teacher's, of a student's or of both masked with the type's lowest number is a uniform
    distribution, and its loss a few nats: no difference of such numbers shows."""
    log("lowest", cols, values, dtype)
    low = torch.finfo(values).min
    for t in (0.7, 1.0, 2.0):
        z, idx, val, rest = R.student(6, cols, 20, dtype, 347, t)
        val = val.to(values)
        val[0], val[1], val[4] = low, low, low
        val[5, 1:] = low
        rest[0] = rest[4] = -math.inf
        rest[1] = low / t if t >= 1.0 else -math.inf  # a float, and the quotient's very number
        z[2] = z[3] = z[4] = torch.finfo(dtype).min
        rest[3] = -math.inf
        check_step(z, idx, val, rest, t, 40.0)


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("rows,cols", [(5, 600), (5, 40_000), (130, 20_000)])
def test_distill_of_a_teachers_row_of_minus_infinity(rows, cols, dtype):
    """Entries whose logits are all -inf, and no rest: no distribution, loss 0 and gradient 0, as without entries."""
    z, idx, val, rest = R.student(rows, cols, 20, dtype, 349)
    weight = torch.zeros(rows)
    weight[:5] = 1.0
    val[1], rest[1] = -math.inf, -math.inf
    val[2, 3:], rest[2] = -math.inf, -math.inf
    val[3] = -math.inf
    idx[4], rest[4] = -1, -math.inf
    check_step(z, idx, val, rest, 1.0, 40.0, weight)
    loss, grad, loss2, grad2 = run_distill(z.cuda(), idx, val, rest, 1.0, weight)
    for x in (loss, loss2, grad, grad2):
        assert float(x[[1, 4]].abs().max()) == 0.0


# one block, one joining block, 3 .. 64 of them, and more
BALANCE_ROUTES = [(60, 8, 60), (4000, 64, 4000), (4000, 200, 4000), (6000, 40, 2000), (4000, 256, 1000),
                  (3000, 1000, 3000), (9000, 256, 900)]


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("gap", [4.0, 14.0, 30.0, 60.0])
@pytest.mark.parametrize("T,E,group", BALANCE_ROUTES)
def test_balance_loss_of_improbable_choices(T, E, group, gap, dtype):
    """Experts chosen whose probability is next to nothing: a loss far below 1, as exact as any other."""
    log("improbable", T, E, group, gap, dtype)
    gen = torch.Generator().manual_seed(353)
    z = torch.randn(T, E, generator=gen)
    z[:, E // 2:] -= gap
    experts = torch.randint(E // 2, E, (T, 2), generator=gen)
    check_balance(z.to(dtype).cuda(), experts, None, group, 1.0)


@pytest.mark.parametrize("T,E,group", BALANCE_ROUTES)
def test_balance_loss_shows_a_nan(T, E, group):
    """A router that has gone NaN has no finite loss, whichever blocks join it."""
    gen = torch.Generator().manual_seed(359)
    z = torch.randn(T, E, generator=gen)
    z[T // 2, 3] = math.nan
    experts = torch.randint(0, E, (T, 2), generator=gen)
    assert math.isnan(float(run_balance(z.cuda(), experts, None, group, 1.0)[3]))


def test_balance_of_many_long_groups():
    """More than 512 groups have a block each, whose lanes add thousands of rows: equal logits, so that every one of
    those additions rounds the same way."""
    group, E, G = 4096 * 128, 5, 513
    log("long groups")
    z = torch.zeros(group * G, E, device="cuda")
    experts = torch.zeros(group * G, 1, dtype=torch.int32, device="cuda")
    counts, n = torch.zeros(G, E, dtype=torch.int32, device="cuda"), torch.zeros(G, dtype=torch.int32, device="cuda")
    prob, loss = torch.zeros(G, E, device="cuda"), torch.zeros(1, device="cuda")
    L.balance_forward(z, experts, None, group, 1.0, counts, n, prob, loss, L.workspace(group * G, E, 1))
    assert bool((counts[:, 0] == group).all()) and bool((n == group).all()) and int(counts.sum()) == group * G
    assert bool(((prob.double() - 0.2).abs() <= 2 * R.SUM * 0.2).all())
    assert abs(float(loss) - 1.0) <= 3 * R.SUM


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("E,rows", [(7, 70_001), (60, 20_001), (300, 1500), (1000, 700)])
def test_balance_of_groups_in_one_block(E, rows, dtype):
    """Groups of some hundred rows a lane, a block each, against sums in 64 bits."""
    G = 513
    log("one block a group", E, rows, dtype)
    gen = torch.Generator(device="cuda").manual_seed(367)
    few = 3  # the groups that are looked at; the others are copies of the last
    part = torch.randn(few * rows, E, generator=gen, device="cuda").to(dtype)
    z = torch.cat([part, part[-rows:].repeat(G - few, 1)])
    choice = torch.randint(0, E, (few * rows, 2), generator=gen, device="cuda", dtype=torch.int32)
    experts = torch.cat([choice, choice[-rows:].repeat(G - few, 1)])
    counts, n = torch.zeros(G, E, dtype=torch.int32, device="cuda"), torch.zeros(G, dtype=torch.int32, device="cuda")
    prob, loss = torch.zeros(G, E, device="cuda"), torch.zeros(1, device="cuda")
    L.balance_forward(z, experts, None, rows, 1.0, counts, n, prob, loss, L.workspace(G * rows, E, 1))
    p = torch.softmax(part.double(), 1).reshape(few, rows, E).mean(1)
    c = torch.stack([torch.bincount(choice[g * rows:(g + 1) * rows].flatten().long(), minlength=E)
                     for g in range(few)])
    assert torch.equal(counts[:few].long(), c) and bool((counts[few:] == counts[few - 1]).all())
    assert bool((n == rows).all())
    assert bool(((prob[:few].double() - p).abs() <= 2 * R.SUM * p).all())
    assert torch.equal(prob[few:], prob[few - 1:few].expand(G - few, E))
    per_group = (E * c.double() / (2 * rows) * p).sum(1)
    want = float(per_group[:few - 1].sum() + per_group[-1] * (G - few + 1)) / G
    assert abs(float(loss) - want) <= 3 * R.SUM * want


@pytest.mark.parametrize("dtype", R.TYPES)
def test_distill_of_the_longest_rows_of_one_block(dtype):
    """Rows of 2^18 columns, whose threads add more numbers one after the other than any: equal ones, which all round
    the same way, and others."""
    cols, rows, k = 1 << 18, 128, 20
    log("2^18 columns", dtype)
    z, idx, val, rest = R.student(rows, cols, k, dtype, 373)
    z[0] = 0.3
    z[1] = torch.where(torch.arange(cols) % 3 == 0, 0.7, -0.4).to(dtype)
    weight = torch.zeros(rows)
    weight[:4] = 1.0
    check_step(z, idx, val, rest, 1.0, 40.0, weight)


@pytest.mark.parametrize("dtype", R.TYPES)
def test_top_rest_of_equal_numbers(dtype):
    """Slices of sixteen vectors a thread whose exponentials all round the same way."""
    for cols in (65_536, 131_072):
        log("equal numbers", cols, dtype)
        x = torch.full((3, cols), -1.3)
        x[:, :100] = torch.linspace(0.0, 5.0, 100)
        x[1, 200:] = torch.where(torch.arange(cols - 200) % 5 == 0, -0.7, -2.1)
        x[2, 1000:] += torch.arange(cols - 1000) * -1e-5
        check_top(x.to(dtype).cuda(), 64)


@pytest.mark.parametrize("dtype", R.TYPES)
def test_a_workspace_of_the_longest_batch_serves_shorter_ones(dtype):
    rows, cols, k = 512, 40_000, 20
    z, idx, val, rest = (x.cuda() for x in R.student(8, cols, k, dtype, 379))
    ws = L.workspace(rows, cols, k)
    many = [x.repeat(rows // 8, *[1] * (x.dim() - 1)) for x in (z, idx, val, rest)]
    seen = {}
    for n in (512, 511, 300, 100, 8, 1):
        zn, teacher = many[0][:n], L.Teacher(*(x[:n] for x in many[1:]))
        loss, loss2 = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        stats = torch.zeros(n, L.STATS, device="cuda")
        grad = torch.zeros_like(zn)
        L.distill_forward(zn, teacher, 1.0, None, loss, stats, ws)
        L.distill_step(zn, teacher, 1.0, None, loss2, grad, ws)
        seen[n] = loss[0].item(), loss2[0].item()
    want = float(R.distill(z[:1].cpu(), idx.cpu(), val.cpu(), rest.cpu(), 1.0)[0])
    assert all(abs(x - want) <= 2 * R.SUM + 2.0 ** -22 * 40 for pair in seen.values() for x in pair)


def test_numbers_that_a_c_integer_would_cut_are_refused():
    z = torch.zeros(6, 8, device="cuda")
    e = torch.zeros(6, 2, dtype=torch.int32, device="cuda")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    loss, ws = torch.zeros(1, device="cuda"), L.workspace(6, 8, 2)
    for group in (0, -1, (1 << 64) + 3):
        with pytest.raises(ValueError):
            L.balance_forward(z, e, None, group, 1.0, i32(1, 8), i32(1), None, loss, ws)
        with pytest.raises(ValueError):
            L.balance_backward(z, 2, None, group, 1.0, i32(1, 8), i32(1), i32(1), None, z)
    for k in (-1, (1 << 32) + 2):
        with pytest.raises(ValueError):
            L.balance_backward(z, k, None, 6, 1.0, i32(1, 8), i32(1), i32(1), None, z)
        with pytest.raises(ValueError):
            L.top_logits(z, k, 1.0, None, None, None, ws)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [50, 9000, 70_001])
def test_top_rest_beyond_a_floats_range(cols, dtype):
    """Rows masked with the lowest number, over a temperature below 1: the rest is as low as a float goes, and not the
    -inf that says that nothing is left; a student of such a payload has a finite loss and gradient."""
    log("rest beyond", cols, dtype)
    low, top = torch.finfo(dtype).min, torch.finfo(dtype).max
    gen = torch.Generator().manual_seed(383)
    x = torch.randn(4, cols, generator=gen)
    x[0], x[1], x[2, 8:] = low, top, -math.inf
    x = x.to(dtype).cuda()
    idx, val, rest = run_top(x, 8, 0.7)
    f32 = torch.finfo(F32)
    assert rest.tolist()[:3] == [f32.min, f32.max, -math.inf] and abs(float(rest[3])) < 100.0
    z = torch.randn(4, cols, generator=gen).to(dtype).cuda()
    keep = torch.tensor([0, 2, 3])
    for out in run_distill(z[keep], idx.cpu()[keep], val.cpu()[keep], rest.cpu()[keep], 0.7, None):
        assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [900, 5000, 30_000])
@pytest.mark.parametrize("gap,weight", [(30.0, 1.0), (45.0, 1.0), (55.0, 1.0), (-50.0, 1e-9), (-65.0, 1e-9)])
def test_distill_gradients_of_a_tail_far_from_the_kept_logits(cols, gap, weight, dtype):
    """The small gradients of a tail that lies far below the kept logits, or far above them, are as exact as others."""
    log("far tail", cols, gap, dtype)
    z, idx, val, rest = R.student(130, cols, 8, dtype, 389, spread=6.0)
    kept = torch.zeros(130, cols, dtype=torch.bool).scatter_(1, idx.long(), True)
    z = torch.where(kept, z.float() + gap, z.float()).to(dtype)
    w = torch.zeros(130)
    w[:4] = weight
    check_step(z, idx, val, rest, 1.0, 130.0, w)


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("t", [0.05, 0.3, 10.0, 50.0])
@pytest.mark.parametrize("rows,cols,k", [(3, 3000, 30), (130, 20_000, 64), (3, 40_000, 200)])
def test_distill_temperatures(rows, cols, k, t, dtype):
    log("temperatures", rows, cols, k, t, dtype)
    z, idx, val, rest = R.student(rows, cols, k, dtype, 397, t)
    weight = torch.zeros(rows)
    weight[:3] = t * t
    check_step(z, idx, val, rest, t, 40.0, weight)


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("t", [0.05, 0.3, 10.0, 50.0])
@pytest.mark.parametrize("cols,k", [(3000, 30), (70_001, 200), (140_000, 256)])
def test_top_temperatures(cols, k, t, dtype):
    log("top temperatures", cols, k, t, dtype)
    gen = torch.Generator().manual_seed(401)
    check_top((3.0 * torch.randn(3, cols, generator=gen)).to(dtype).cuda(), k, t)


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("cols,k", [(50_001, 1024), (150_000, 700), (262_143, 1024)])
def test_distill_long_rows_of_many_entries(cols, k, dtype):
    """Rows of one block that take several rounds beyond its registers, with as many entries as a row may have."""
    log("long rows, many entries", cols, k, dtype)
    z, idx, val, rest = R.student(128, cols, k, dtype, 409)
    weight = torch.zeros(128)
    weight[[0, 1, 127]] = 1.0
    check_step(z, idx, val, rest, 1.0, 40.0, weight)


@pytest.mark.parametrize("k", [257, 1000])
def test_distill_short_rows_of_many_entries(k):
    """More entries than a wave, or than a block has threads, at every size of block."""
    for cols in (1001, 2500, 5000, 9000, 20_000, 40_000):
        log("many entries", cols, k)
        z, idx, val, rest = R.student(128, cols, k, BF16, 419)
        weight = torch.zeros(128)
        weight[:3] = 1.0
        check_step(z, idx, val, rest, 1.0, 40.0, weight)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("values", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(8, 700), (8, 40_000), (130, 20_000)])
def test_distill_of_large_teachers(rows, cols, values, dtype):
    """Teachers' logits of any size, over temperatures whose quotients a float rounds by more than an exponent takes:
    whole rows of one number, one that stands out, two near each other."""
    log("large teachers", rows, cols, values, dtype)
    near = 1.0 - 2.0 ** -8
    for t in (0.7, 1.0, 1.5, 3.0, 50.0):
        for size in (2e7, 3e9, 3e20, 1e37, torch.finfo(values).max):
            z, idx, val, rest = R.student(rows, cols, 20, dtype, 421, t)
            val[0], val[1] = -size, size
            val[2, :], val[2, 3] = -size, -size * near
            val[3, :], val[3, 5] = size * near, size
            val[4, 1:] = -size
            val[5, 1:] = -size
            val[6] = -size
            val[7, 7], val[7, 8] = 1e9, 1e9
            rest[:4] = -math.inf
            rest[5] = -math.inf
            weight = torch.zeros(rows)
            weight[:8] = 1.0
            check_step(z, idx, val.to(values), rest, t, 40.0, weight)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(8, 700), (8, 40_000), (130, 20_000)])
def test_distill_of_students_of_every_size(rows, cols, dtype):
    """Student's logits of any size: whole rows, whole tails and single columns masked with a large number, tails and
    kept columns that differ little beside it."""
    log("large students", rows, cols, dtype)
    near = 1.0 - 2.0 ** -8
    for t in (0.7, 1.0, 3.0):
        for size in (1e6, 7e7, 2e8, 1e9, 3e9, 1e10, 1e12, 3e20, 1e29, 2e30, 1e37):
            z, idx, val, rest = R.student(rows, cols, 20, dtype, 431, t)
            kept = torch.zeros(rows, cols, dtype=torch.bool).scatter_(1, idx.long(), True)
            third = torch.arange(cols) % 3 == 0
            f = z.float()
            f[0] = -size
            f[1] = torch.where(kept[1], f[1], -size)
            f[2] = torch.where(kept[2], f[2], torch.where(third, -size, -size * near))
            f[3] = torch.where(kept[3], -size, f[3])
            f[4] = torch.where(third, -size * near, -size)
            f[5] = size
            f[6] = torch.where(third & ~kept[6], -size, f[6])
            f[7] = torch.where(kept[7], f[7], torch.where(third, size, size * near))
            rest[[0, 1]] = -math.inf
            weight = torch.zeros(rows)
            weight[:8] = 1.0
            check_step(f.to(dtype), idx, val, rest, t, 40.0, weight)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols,k", [(60, 8), (9000, 64), (140_000, 100)])
def test_top_logits_of_every_size(cols, k, dtype):
    log("top of every size", cols, k, dtype)
    third = torch.arange(cols) % 3 == 0
    gen = torch.Generator().manual_seed(433)
    x = torch.randn(1, cols, generator=gen)[0]
    for t in (0.7, 1.0, 3.0):
        for size in (1e6, 7e7, 2e8, 1e9, 3e9, 1e10, 1e12, 3e20, 1e29, 2e30, 1e37):
            near = size * (1.0 - 2.0 ** -8)
            rows = [torch.full((cols,), -size), torch.full((cols,), size), torch.where(third, size, near),
                    torch.where(third, -size, -near), torch.where(third, -size, x), torch.where(third, size, x)]
            check_top(torch.stack(rows).to(dtype).cuda(), k, t)
