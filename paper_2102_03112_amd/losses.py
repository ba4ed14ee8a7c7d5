"""ctypes binding of the loss operators (include/deepreduce_losses.h).

The losses of a data-parallel training step, next to the codec that sends its
gradient: a teacher's top logits, the distillation loss from them and its
gradient, and a router's balance loss with per-expert counts and its gradient.
Argument marshalling only, as in ``binding``: every function passes torch
device tensors' pointers and the current HIP stream to the C ABI entry point of
the same name and raises ``DeepReduceError`` on a non-OK status.  What the C
ABI cannot see (sizes, types, devices) is checked here and raises ValueError.

Logits are 2-D tensors of float32, bfloat16 or float16 whose rows are
contiguous; rows may be strided (a view of a wider matrix).
"""
from __future__ import annotations

import ctypes

import torch

from .binding import DR_EINVAL, DR_OK, DeepReduceError, last_error
from .binding import lib as _base_lib

TYPE_F32, TYPE_BF16, TYPE_F16 = 0, 1, 2
INDEX_I32, INDEX_I64 = 0, 1
MAX_TOP, MAX_TEACHER, MAX_EXPERTS, STATS = 256, 1024, 1024, 8

EXPORTS = [
    "dr_losses_workspace_bytes", "dr_top_logits", "dr_distill_forward", "dr_distill_backward", "dr_distill_step",
    "dr_balance_forward", "dr_balance_backward",
]


class DrLogits(ctypes.Structure):
    _fields_ = [
        ("data", ctypes.c_void_p),
        ("rows", ctypes.c_uint64),
        ("cols", ctypes.c_uint64),
        ("row_stride", ctypes.c_uint64),
        ("type", ctypes.c_uint32),
    ]


class DrTeacher(ctypes.Structure):
    _fields_ = [
        ("idx", ctypes.c_void_p),
        ("val", ctypes.c_void_p),
        ("rest", ctypes.c_void_p),
        ("idx_stride", ctypes.c_uint64),
        ("val_stride", ctypes.c_uint64),
        ("k", ctypes.c_uint32),
        ("idx_type", ctypes.c_uint32),
        ("val_type", ctypes.c_uint32),
    ]


class DrRoutes(ctypes.Structure):
    _fields_ = [
        ("idx", ctypes.c_void_p),
        ("idx_stride", ctypes.c_uint64),
        ("k", ctypes.c_uint32),
        ("idx_type", ctypes.c_uint32),
        ("row_mask", ctypes.c_void_p),
        ("group_rows", ctypes.c_uint64),
    ]


_lib = None


def lib():
    """The loaded library with the loss operators' signatures."""
    global _lib
    if _lib is not None:
        return _lib
    L = _base_lib()
    vp, u32, u64, sz, st, f32 = (ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_size_t, ctypes.c_int,
                                 ctypes.c_float)
    lg, te, ro = ctypes.POINTER(DrLogits), ctypes.POINTER(DrTeacher), ctypes.POINTER(DrRoutes)
    sig = {
        "dr_losses_workspace_bytes": (sz, [u64, u64, u32]),
        "dr_top_logits": (st, [lg, u32, f32, vp, vp, vp, vp, sz, vp]),
        "dr_distill_forward": (st, [lg, te, f32, vp, vp, vp, vp, sz, vp]),
        "dr_distill_backward": (st, [lg, te, f32, vp, vp, u64, vp, vp, u64, vp]),
        "dr_distill_step": (st, [lg, te, f32, vp, vp, vp, u64, vp, sz, vp]),
        "dr_balance_forward": (st, [lg, ro, f32, vp, vp, vp, vp, vp, sz, vp]),
        "dr_balance_backward": (st, [lg, ro, f32, vp, vp, vp, vp, vp, u64, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


# ---------------------------------------------------------------------------
# what the C ABI cannot check.  A small call's time on the GPU is a few
# microseconds, so these stay at about two in all.
# ---------------------------------------------------------------------------

_NUMBER = {torch.float32: TYPE_F32, torch.bfloat16: TYPE_BF16, torch.float16: TYPE_F16}
_INDEX = {torch.int32: INDEX_I32, torch.int64: INDEX_I64}
_F32, _I32 = torch.float32, torch.int32


def _type(table, t, what: str) -> int:
    kind = table.get(t.dtype)
    if kind is None:
        raise ValueError(f"{what}: one of {', '.join(str(d) for d in table)} expected, got {t.dtype}")
    return kind


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _row_stride(t, what: str) -> int:
    """Numbers between row starts of a 2-D tensor whose rows are contiguous."""
    if t.dim() != 2:
        raise ValueError(f"{what}: a 2-D tensor expected")
    rows, cols = t.shape
    row, col = t.stride()
    if col != 1 and cols > 1:
        raise ValueError(f"{what}: rows must be contiguous")
    return row if rows > 1 else cols


def _flat(t, n: int, dtype, dev: int, what: str):
    """The address of a contiguous tensor of n elements of a type on device dev, or None for None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{what}: {n} contiguous elements of {dtype} on cuda:{dev} expected, got {tuple(t.shape)} of "
                         f"{t.dtype} on {t.device}")
    return t.data_ptr()


def _logits(t):
    """(descriptor, rows, cols, device)"""
    dev = t.get_device()
    if dev < 0 or dev != torch.cuda.current_device():
        raise ValueError("logits: on the current device expected")
    stride = _row_stride(t, "logits")
    rows, cols = t.shape
    return DrLogits(t.data_ptr(), rows, cols, stride, _type(_NUMBER, t, "logits")), rows, cols, dev


def _grad(grad, logits, dev: int) -> int:
    if grad.shape != logits.shape or grad.dtype is not logits.dtype or grad.get_device() != dev:
        raise ValueError("grad_out: the logits' shape, type and device expected")
    return _row_stride(grad, "grad_out")


def _scratch(ws, dev: int):
    if ws.dtype is not torch.uint8 or ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError("ws: contiguous bytes on the logits' device expected")
    return ws.data_ptr()


def _stream(stream, dev: int):
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _check(fn: str, status: int):
    if status != DR_OK:
        raise DeepReduceError(fn, status, last_error())


def workspace_bytes(rows: int, cols: int, k: int = 1) -> int:
    """Scratch bytes for any call below on at most rows x cols logits with at most k kept ones."""
    _need(0 <= rows < 1 << 64 and 0 <= cols < 1 << 64 and 0 <= k < 1 << 32, "rows, cols or k out of range")
    n = int(lib().dr_losses_workspace_bytes(rows, cols, k))
    if n == 0:
        raise DeepReduceError("dr_losses_workspace_bytes", DR_EINVAL, last_error())
    return n


def workspace(rows: int, cols: int, k: int = 1, device="cuda"):
    """A device scratch buffer of workspace_bytes(rows, cols, k) bytes."""
    n = workspace_bytes(rows, cols, k)
    ws = torch.empty(n + 256, dtype=torch.uint8, device=device)
    off = (-ws.data_ptr()) % 256
    return ws[off:off + n]


# ---------------------------------------------------------------------------
# a teacher's logits into a payload
# ---------------------------------------------------------------------------


def top_logits(logits, k: int, temperature: float, idx_out, val_out, rest_out, ws, stream=None):
    """The k largest logits of each row and the entry for the rest (dr_top_logits)."""
    m, rows, _, dev = _logits(logits)
    _need(0 <= k < 1 << 32, "k out of range")
    _check("dr_top_logits", lib().dr_top_logits(
        ctypes.byref(m), k, temperature, _flat(idx_out, rows * k, _I32, dev, "idx_out"),
        _flat(val_out, rows * k, _F32, dev, "val_out"), _flat(rest_out, rows, _F32, dev, "rest_out"),
        _scratch(ws, dev), ws.numel(), _stream(stream, dev)))


class Teacher:
    """A teacher's payload: idx (rows x k, int32 or int64; outside the columns: no entry), val (rows x k logits) and
    rest (per row, or None: the kept logits are the whole distribution).  Rows may be strided.  It keeps the tensors
    alive."""

    def __init__(self, idx, val, rest=None):
        _need(idx.dim() == 2 and idx.shape == val.shape, "teacher: idx and val of one 2-D shape expected")
        self.rows, k = idx.shape
        self.dev = idx.get_device()
        _need(val.get_device() == self.dev, "teacher: idx and val on one device expected")
        self.idx, self.val, self.rest = idx, val, rest
        self.c = DrTeacher(idx.data_ptr(), val.data_ptr(), _flat(rest, self.rows, _F32, self.dev, "rest"),
                           _row_stride(idx, "idx"), _row_stride(val, "val"), k, _type(_INDEX, idx, "idx"),
                           _type(_NUMBER, val, "val"))

    def _for(self, rows: int, dev: int):
        if self.rows != rows or self.dev != dev:
            raise ValueError("teacher: one row per row of logits, on their device, expected")
        return ctypes.byref(self.c)


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------


def distill_forward(logits, teacher: Teacher, temperature: float, weight, loss_out, stats_out, ws, stream=None):
    """Per row, weight * KL(teacher || student); stats_out (rows x STATS, or None) is for distill_backward."""
    m, rows, _, dev = _logits(logits)
    _check("dr_distill_forward", lib().dr_distill_forward(
        ctypes.byref(m), teacher._for(rows, dev), temperature, _flat(weight, rows, _F32, dev, "weight"),
        _flat(loss_out, rows, _F32, dev, "loss_out"), _flat(stats_out, rows * STATS, _F32, dev, "stats_out"),
        _scratch(ws, dev), ws.numel(), _stream(stream, dev)))


def distill_backward(logits, teacher: Teacher, temperature: float, weight, upstream, stats, grad_out, stream=None):
    """The gradient at the logits; upstream (the loss's gradient per row, or None for ones) may be an expanded
    scalar.  grad_out may be the logits themselves."""
    m, rows, _, dev = _logits(logits)
    up, stride = None, 0
    if upstream is not None:
        if upstream.dtype is not _F32 or upstream.dim() != 1 or upstream.shape[0] != rows or \
                upstream.get_device() != dev:
            raise ValueError("upstream: one float32 per row on the logits' device expected")
        up, stride = upstream.data_ptr(), upstream.stride(0) if rows > 1 else 0
    _check("dr_distill_backward", lib().dr_distill_backward(
        ctypes.byref(m), teacher._for(rows, dev), temperature, _flat(weight, rows, _F32, dev, "weight"), up, stride,
        _flat(stats, rows * STATS, _F32, dev, "stats"), grad_out.data_ptr(), _grad(grad_out, logits, dev),
        _stream(stream, dev)))


def distill_step(logits, teacher: Teacher, temperature: float, weight, loss_out, grad_out, ws, stream=None):
    """Loss and gradient in one call; grad_out may be the logits themselves."""
    m, rows, _, dev = _logits(logits)
    _check("dr_distill_step", lib().dr_distill_step(
        ctypes.byref(m), teacher._for(rows, dev), temperature, _flat(weight, rows, _F32, dev, "weight"),
        _flat(loss_out, rows, _F32, dev, "loss_out"), grad_out.data_ptr(), _grad(grad_out, logits, dev),
        _scratch(ws, dev), ws.numel(), _stream(stream, dev)))


# ---------------------------------------------------------------------------
# balance loss
# ---------------------------------------------------------------------------


def _mask(mask, rows: int, dev: int):
    if mask is None:
        return None
    _need(mask.dtype is torch.bool or mask.dtype is torch.uint8, "row_mask: bool or uint8 expected")
    return _flat(mask, rows, mask.dtype, dev, "row_mask")


def _groups(rows: int, group_rows: int) -> int:
    # cut to 64 bits, it would have more groups than the outputs are checked for here
    _need(1 <= group_rows < 1 << 64, "group_rows out of range")
    return -(-rows // group_rows)


def balance_forward(logits, experts, row_mask, group_rows: int, coef: float, counts_out, rows_out, prob_out, loss_out,
                    ws, stream=None):
    """Per group of group_rows rows: choices per expert, valid rows, mean probabilities (prob_out may be None); and the
    balance loss.  experts: rows x k chosen ones (int32 or int64), negative where dropped."""
    m, rows, E, dev = _logits(logits)
    G = _groups(rows, group_rows)
    stride = _row_stride(experts, "experts")
    if experts.shape[0] != rows or experts.get_device() != dev:
        raise ValueError("experts: one row per row of logits, on their device, expected")
    r = DrRoutes(experts.data_ptr(), stride, experts.shape[1], _type(_INDEX, experts, "experts"),
                 _mask(row_mask, rows, dev), group_rows)
    _check("dr_balance_forward", lib().dr_balance_forward(
        ctypes.byref(m), ctypes.byref(r), coef, _flat(counts_out, G * E, _I32, dev, "counts_out"),
        _flat(rows_out, G, _I32, dev, "rows_out"), _flat(prob_out, G * E, _F32, dev, "prob_out"),
        _flat(loss_out, 1, _F32, dev, "loss_out"), _scratch(ws, dev), ws.numel(), _stream(stream, dev)))


def balance_backward(logits, k: int, row_mask, group_rows: int, coef: float, counts, count_rows, rows_in, upstream,
                     grad_out, stream=None):
    """The balance loss's gradient at the router's logits.  counts and count_rows: a worker's own (count_rows is
    rows_in then) or the sums over all workers; upstream: one float32, or None for 1."""
    m, rows, E, dev = _logits(logits)
    G = _groups(rows, group_rows)
    _need(0 <= k < 1 << 32, "k out of range")
    r = DrRoutes(None, 0, k, INDEX_I32, _mask(row_mask, rows, dev), group_rows)
    _check("dr_balance_backward", lib().dr_balance_backward(
        ctypes.byref(m), ctypes.byref(r), coef, _flat(counts, G * E, _I32, dev, "counts"),
        _flat(count_rows, G, _I32, dev, "count_rows"), _flat(rows_in, G, _I32, dev, "rows_in"),
        _flat(upstream, 1, _F32, dev, "upstream"), grad_out.data_ptr(), _grad(grad_out, logits, dev),
        _stream(stream, dev)))
