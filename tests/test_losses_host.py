"""Host-side checks of the loss operators' C ABI (no GPU needed, nothing is
launched): exports, refusals before any device work, workspace needs; and the
definitions that the GPU tests compare with, against differences of themselves.
"""
import ctypes
import math
import os
import re

import pytest
import torch

import _losses_util as R
from paper_2102_03112_amd import binding as B
from paper_2102_03112_amd import losses as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "deepreduce_losses.h")
FAKE = 1 << 20  # never dereferenced: the checks fail first
BIG = 1 << 50


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2102_03112_amd import build

        build.build()
    return L.lib()


def test_every_declared_symbol_is_exported(lib):
    names = re.findall(r"DR_EXPORT\s+[\w\s\*]+?\b(dr_\w+)\s*\(", open(HEADER).read())
    assert sorted(names) == sorted(L.EXPORTS) and len(set(names)) == 7
    for n in names:
        assert hasattr(lib, n), n


def test_limits_match_the_header():
    text = open(HEADER).read()
    for name, value in [("DR_MAX_TOP", L.MAX_TOP), ("DR_MAX_TEACHER", L.MAX_TEACHER), ("DR_MAX_EXPERTS", L.MAX_EXPERTS),
                        ("DR_DISTILL_STATS", L.STATS)]:
        assert re.search(rf"#define {name} {value}u", text), name


def logits(**kw):
    c = dict(data=FAKE, rows=10, cols=100, row_stride=100, type=0)
    c.update(kw)
    return L.DrLogits(c["data"], c["rows"], c["cols"], c["row_stride"], c["type"])


def teacher(**kw):
    c = dict(idx=FAKE, val=FAKE, rest=None, idx_stride=8, val_stride=8, k=8, idx_type=0, val_type=0)
    c.update(kw)
    return L.DrTeacher(c["idx"], c["val"], c["rest"], c["idx_stride"], c["val_stride"], c["k"], c["idx_type"],
                       c["val_type"])


def routes(**kw):
    c = dict(idx=FAKE, idx_stride=4, k=4, idx_type=0, row_mask=None, group_rows=5)
    c.update(kw)
    return L.DrRoutes(c["idx"], c["idx_stride"], c["k"], c["idx_type"], c["row_mask"], c["group_rows"])


BAD_LOGITS = [dict(data=None), dict(rows=1 << 31), dict(cols=0), dict(cols=1 << 31, row_stride=1 << 31),
              dict(row_stride=99), dict(row_stride=1 << 62), dict(type=3), dict(data=FAKE + 2)]


ALL = ("top", "forward", "backward", "step", "balance", "balance_bwd")
DISTILL, GRAD, BALANCE = ("forward", "backward", "step"), ("backward", "step", "balance_bwd"), ("balance", "balance_bwd")


def refused(lib, names, lg, te=None, ro=None, t=1.0, coef=0.1, ws=FAKE, n=BIG, out=FAKE, grad=FAKE, gs=100, k=4):
    """Makes the named calls (those that the arguments are wrong for, and no others: nothing may be launched)."""
    te, ro = te or teacher(), ro or routes()
    ref = lambda x: ctypes.byref(x) if x != "null" else None  # noqa: E731
    lg, te, ro = ref(lg), ref(te), ref(ro)
    calls = {
        "top": lambda: lib.dr_top_logits(lg, k, t, out, out, None, ws, n, None),
        "forward": lambda: lib.dr_distill_forward(lg, te, t, None, out, None, ws, n, None),
        "backward": lambda: lib.dr_distill_backward(lg, te, t, None, None, 0, out, grad, gs, None),
        "step": lambda: lib.dr_distill_step(lg, te, t, None, out, grad, gs, ws, n, None),
        "balance": lambda: lib.dr_balance_forward(lg, ro, coef, out, out, None, out, ws, n, None),
        "balance_bwd": lambda: lib.dr_balance_backward(lg, ro, coef, out, out, out, None, grad, gs, None),
    }
    for name in names:
        assert calls[name]() == B.DR_EINVAL, name
        assert B.last_error()


@pytest.mark.parametrize("bad", BAD_LOGITS + [None])
def test_bad_logits_are_refused(lib, bad):
    refused(lib, ALL, "null" if bad is None else logits(**bad))


@pytest.mark.parametrize("bad", [dict(k=0), dict(k=1025, idx_stride=2000, val_stride=2000), dict(idx=None),
                                 dict(val=None), dict(idx_stride=7), dict(val_stride=7), dict(idx_type=2),
                                 dict(val_type=3), dict(idx=FAKE + 4, idx_type=1), dict(val=FAKE + 1, val_type=1),
                                 dict(rest=FAKE + 2), dict(idx_stride=1 << 60), None])
def test_bad_teachers_are_refused(lib, bad):
    refused(lib, DISTILL, logits(), te="null" if bad is None else teacher(**bad))


@pytest.mark.parametrize("bad", [dict(k=0), dict(k=101, idx_stride=200), dict(group_rows=0), dict(group_rows=1 << 31),
                                 None])
def test_bad_routes_are_refused(lib, bad):
    refused(lib, BALANCE, logits(), ro="null" if bad is None else routes(**bad))


@pytest.mark.parametrize("bad", [dict(idx_stride=3), dict(idx_type=2), dict(idx=None), dict(idx=FAKE + 2)])
def test_bad_choices_are_refused(lib, bad):
    refused(lib, ["balance"], logits(), ro=routes(**bad))


def test_too_many_experts_or_choices_are_refused(lib):
    refused(lib, BALANCE, logits(cols=1025, row_stride=1025), gs=1025)
    refused(lib, BALANCE, logits(rows=1 << 29))


@pytest.mark.parametrize("t", [0.0, -1.0, math.nan, math.inf, 1e-39])
def test_bad_temperatures_are_refused(lib, t):
    refused(lib, ("top",) + DISTILL, logits(), t=t)


@pytest.mark.parametrize("coef", [math.nan, math.inf])
def test_bad_coefficients_are_refused(lib, coef):
    refused(lib, BALANCE, logits(), coef=coef)


@pytest.mark.parametrize("k", [0, 257])
def test_bad_numbers_of_kept_logits_are_refused(lib, k):
    refused(lib, ["top"], logits(), k=k)


def test_missing_and_bad_outputs_are_refused(lib):
    refused(lib, ALL, logits(), out=None)
    refused(lib, GRAD, logits(), grad=None)
    for gs, grad in ((99, FAKE), (1 << 62, FAKE), (100, FAKE + 2)):
        refused(lib, GRAD, logits(), gs=gs, grad=grad)
    refused(lib, GRAD, logits(data=FAKE), gs=128, grad=FAKE)  # in place with another stride


def test_calls_too_large_for_one_grid_are_refused(lib):
    lg = logits(rows=1 << 20, cols=1 << 28, row_stride=1 << 28)
    refused(lib, ("top",) + DISTILL, lg, gs=1 << 28)
    refused(lib, ("top",) + DISTILL, logits(rows=1 << 30, cols=8, row_stride=8), gs=8)
    refused(lib, BALANCE, logits(rows=1 << 28), ro=routes(group_rows=1))


def test_small_workspaces_are_refused(lib):
    lg = logits(rows=10, cols=50_000, row_stride=50_000)
    assert lib.dr_losses_workspace_bytes(10, 50_000, 4) > 0
    for ws, n in ((FAKE, 64), (None, BIG), (FAKE + 128, BIG)):
        for name in ("top", "forward", "step"):
            refused(lib, [name], lg, ws=ws, n=n, gs=50_000)
            assert "workspace" in B.last_error()
        refused(lib, ["balance"], logits(), ws=ws, n=n)
        assert "workspace" in B.last_error()


def test_workspace_bytes(lib):
    f = lib.dr_losses_workspace_bytes
    assert f(1 << 31, 10, 1) == f(10, 0, 1) == f(10, 1 << 31, 1) == 0
    with pytest.raises(B.DeepReduceError):
        L.workspace_bytes(10, 0)
    assert 0 < f(0, 10, 1) <= f(100, 100_000, 64) <= f(4096, 131_072, 256)
    # small beside the logits, also where they are 16 bits wide
    assert f(4096, 131_072, 64) < 4096 * 131_072 * 2 // 20
    assert f(131_072, 256, 8) < 16 << 20


def test_a_workspace_serves_smaller_calls(lib):
    """Bytes never fall as rows, columns or kept logits grow: what serves a batch serves a shorter one."""
    f = lib.dr_losses_workspace_bytes
    rows = list(range(1, 70)) + [100, 127, 128, 129, 255, 256, 257, 300, 511, 512, 513, 1000, 1023, 1024, 1025, 4096]
    cols = [1, 8, 300, 1024, 1025, 2000, 8192, 16384, 16385, 32000, 40_000, 65536, 65537, 131_072, 1 << 20]
    for k in (0, 1, 64, 256, 257, 1024):
        for c in cols:
            need = [f(r, c, k) for r in rows]
            assert need == sorted(need), (c, k)
        for r in rows[::9]:
            need = [f(r, c, k) for c in cols]
            assert need == sorted(need), (r, k)
    for r in rows[::9]:
        for c in cols:
            need = [f(r, c, k) for k in (0, 1, 2, 8, 50, 64, 200, 256, 257, 1024)]
            assert need == sorted(need), (r, c)


def test_python_checks():
    z = torch.zeros(4, 10)
    with pytest.raises(ValueError):  # not on a GPU
        L.distill_backward(z, L.Teacher(torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)), 1.0, None, None,
                           torch.zeros(4, 8), z)
    with pytest.raises(ValueError):
        L.Teacher(torch.zeros(4, 2, dtype=torch.int16), torch.zeros(4, 2))
    with pytest.raises(ValueError):
        L.Teacher(torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 3))
    with pytest.raises(ValueError):
        L.Teacher(torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), torch.zeros(3))
    with pytest.raises(ValueError):
        L.Teacher(torch.zeros(2, 4, dtype=torch.int32).t(), torch.zeros(4, 2))


def test_the_definitions_gradients_against_differences():
    z, idx, val, rest = R.student(3, 40, 6, torch.float64, 5, 1.3)
    w, u = torch.tensor([0.5, 0.0, 2.0]), torch.tensor([1.0, 1.0, 0.25])
    _, grad, _ = R.distill(z, idx, val, rest, 1.3, w, u)
    h = 1e-5
    for r in range(3):
        for j in (0, 7, 21, int(idx[r, 0]), int(idx[r, 5])):
            up, down = z.clone(), z.clone()
            up[r, j] += h
            down[r, j] -= h
            d = (R.distill(up, idx, val, rest, 1.3, w)[0] - R.distill(down, idx, val, rest, 1.3, w)[0])[r] / (2 * h)
            assert abs(float(u[r] * d) - float(grad[r, j])) < 1e-9
    gen = torch.Generator().manual_seed(2)
    z = torch.randn(20, 9, generator=gen).double()
    experts = torch.randint(0, 9, (20, 2), generator=gen)
    _, _, _, _, grad, _ = R.balance(z, experts, 2, None, 7, 0.3)
    for r, j in ((0, 0), (8, 3), (19, 8)):
        up, down = z.clone(), z.clone()
        up[r, j] += h
        down[r, j] -= h
        d = (R.balance(up, experts, 2, None, 7, 0.3)[3] - R.balance(down, experts, 2, None, 7, 0.3)[3]) / (2 * h)
        assert abs(d - float(grad[r, j])) < 1e-9


@pytest.mark.parametrize("bad", [-1, 1 << 64, (1 << 64) + 5])
def test_python_refuses_numbers_that_a_c_integer_would_cut(bad):
    """Before the call: a number of group rows cut to 64 bits would have more groups than the outputs are checked for."""
    with pytest.raises(ValueError):
        L._groups(10, bad)
    with pytest.raises(ValueError):
        L.workspace_bytes(bad, 10)
    with pytest.raises(ValueError):
        L.workspace_bytes(10, bad)
    with pytest.raises(ValueError):
        L.workspace_bytes(10, 10, bad)
