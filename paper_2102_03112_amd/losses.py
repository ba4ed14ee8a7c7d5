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

from .binding import DR_EINVAL, DeepReduceError, _check, _ptr, _stream, last_error
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
# what the C ABI cannot check
# ---------------------------------------------------------------------------


def _number_type(t, what: str) -> int:
    import torch

    types = {torch.float32: TYPE_F32, torch.bfloat16: TYPE_BF16, torch.float16: TYPE_F16}
    if t.dtype not in types:
        raise ValueError(f"{what}: float32, bfloat16 or float16 expected, got {t.dtype}")
    return types[t.dtype]


def _index_type(t, what: str) -> int:
    import torch

    types = {torch.int32: INDEX_I32, torch.int64: INDEX_I64}
    if t.dtype not in types:
        raise ValueError(f"{what}: int32 or int64 expected, got {t.dtype}")
    return types[t.dtype]


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _row_stride(t, what: str) -> int:
    """Numbers between row starts of a 2-D tensor whose rows are contiguous and do not overlap."""
    _need(t.dim() == 2, f"{what}: a 2-D tensor expected")
    rows, cols = t.shape
    _need(cols <= 1 or t.stride(1) == 1, f"{what}: rows must be contiguous")
    return int(t.stride(0)) if rows > 1 else int(cols)


def _scratch(ws, like):
    import torch

    _place(ws, like, "ws")
    _need(ws.dtype == torch.uint8 and ws.is_contiguous(), "ws: contiguous bytes expected")


def _place(t, like, what: str):
    _need(t.device == like.device, f"{what}: on {t.device}, the logits are on {like.device}")


def _flat(t, n: int, dtype, like, what: str):
    """A contiguous tensor of n elements of a type, or None."""
    if t is None:
        return
    _place(t, like, what)
    _need(t.dtype == dtype, f"{what}: {dtype} expected, got {t.dtype}")
    _need(t.is_contiguous() and t.numel() == n, f"{what}: {n} contiguous elements expected")


def _logits(t) -> DrLogits:
    import torch

    _need(t.is_cuda and t.device.index == torch.cuda.current_device(), "logits: on the current device expected")
    stride = _row_stride(t, "logits")
    return DrLogits(_ptr(t), t.shape[0], t.shape[1], stride, _number_type(t, "logits"))


def _grad(grad, logits) -> int:
    _need(tuple(grad.shape) == tuple(logits.shape) and grad.dtype == logits.dtype,
          "grad_out: the logits' shape and type expected")
    _place(grad, logits, "grad_out")
    return _row_stride(grad, "grad_out")


def workspace_bytes(rows: int, cols: int, k: int = 1) -> int:
    """Scratch bytes for any call below on rows x cols logits with k kept ones."""
    n = int(lib().dr_losses_workspace_bytes(rows, cols, k))
    if n == 0:
        raise DeepReduceError("dr_losses_workspace_bytes", DR_EINVAL, last_error())
    return n


def workspace(rows: int, cols: int, k: int = 1, device="cuda"):
    """A device scratch buffer of workspace_bytes(rows, cols, k) bytes."""
    import torch

    n = workspace_bytes(rows, cols, k)
    ws = torch.empty(n + 256, dtype=torch.uint8, device=device)
    off = (-ws.data_ptr()) % 256
    return ws[off:off + n]


# ---------------------------------------------------------------------------
# a teacher's logits into a payload
# ---------------------------------------------------------------------------


def top_logits(logits, k: int, temperature: float, idx_out, val_out, rest_out, ws, stream=None):
    """The k largest logits of each row and the entry for the rest (dr_top_logits)."""
    import torch

    m = _logits(logits)
    rows = logits.shape[0]
    _flat(idx_out, rows * k, torch.int32, logits, "idx_out")
    _flat(val_out, rows * k, torch.float32, logits, "val_out")
    _flat(rest_out, rows, torch.float32, logits, "rest_out")
    _scratch(ws, logits)
    _check("dr_top_logits", lib().dr_top_logits(
        ctypes.byref(m), k, temperature, _ptr(idx_out), _ptr(val_out), _ptr(rest_out), _ptr(ws), ws.numel(),
        _stream(stream)))


class Teacher:
    """A teacher's payload: idx (rows x k, int32 or int64; outside the columns: no entry), val (rows x k logits) and
    rest (per row, or None: the kept logits are the whole distribution).  Rows may be strided.  It keeps the tensors
    alive."""

    def __init__(self, idx, val, rest=None):
        import torch

        _need(idx.dim() == 2 and tuple(idx.shape) == tuple(val.shape), "teacher: idx and val of one 2-D shape expected")
        _place(val, idx, "val")
        _flat(rest, idx.shape[0], torch.float32, idx, "rest")
        self.idx, self.val, self.rest = idx, val, rest
        self.c = DrTeacher(_ptr(idx), _ptr(val), _ptr(rest), _row_stride(idx, "idx"), _row_stride(val, "val"),
                           idx.shape[1], _index_type(idx, "idx"), _number_type(val, "val"))

    def _for(self, logits):
        _need(self.idx.shape[0] == logits.shape[0], "teacher: one row per row of logits expected")
        _place(self.idx, logits, "teacher")
        return ctypes.byref(self.c)


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------


def distill_forward(logits, teacher: Teacher, temperature: float, weight, loss_out, stats_out, ws, stream=None):
    """Per row, weight * KL(teacher || student); stats_out (rows x STATS, or None) is for distill_backward."""
    import torch

    m = _logits(logits)
    rows = logits.shape[0]
    _flat(weight, rows, torch.float32, logits, "weight")
    _flat(loss_out, rows, torch.float32, logits, "loss_out")
    _flat(stats_out, rows * STATS, torch.float32, logits, "stats_out")
    _scratch(ws, logits)
    _check("dr_distill_forward", lib().dr_distill_forward(
        ctypes.byref(m), teacher._for(logits), temperature, _ptr(weight), _ptr(loss_out), _ptr(stats_out), _ptr(ws),
        ws.numel(), _stream(stream)))


def distill_backward(logits, teacher: Teacher, temperature: float, weight, upstream, stats, grad_out, stream=None):
    """The gradient at the logits; upstream (the loss's gradient per row, or None for ones) may be an expanded
    scalar.  grad_out may be the logits themselves."""
    import torch

    m = _logits(logits)
    rows = logits.shape[0]
    stride = 0
    if upstream is not None:
        _place(upstream, logits, "upstream")
        _need(upstream.dtype == torch.float32 and tuple(upstream.shape) == (rows,) and (rows <= 1 or
              upstream.stride(0) >= 0), "upstream: one float32 per row expected")
        stride = int(upstream.stride(0)) if rows > 1 else 0
    _flat(weight, rows, torch.float32, logits, "weight")
    _flat(stats, rows * STATS, torch.float32, logits, "stats")
    grad_stride = _grad(grad_out, logits)
    _check("dr_distill_backward", lib().dr_distill_backward(
        ctypes.byref(m), teacher._for(logits), temperature, _ptr(weight), _ptr(upstream), stride, _ptr(stats),
        _ptr(grad_out), grad_stride, _stream(stream)))


def distill_step(logits, teacher: Teacher, temperature: float, weight, loss_out, grad_out, ws, stream=None):
    """Loss and gradient in one call; grad_out may be the logits themselves."""
    import torch

    m = _logits(logits)
    rows = logits.shape[0]
    _flat(weight, rows, torch.float32, logits, "weight")
    _flat(loss_out, rows, torch.float32, logits, "loss_out")
    grad_stride = _grad(grad_out, logits)
    _scratch(ws, logits)
    _check("dr_distill_step", lib().dr_distill_step(
        ctypes.byref(m), teacher._for(logits), temperature, _ptr(weight), _ptr(loss_out), _ptr(grad_out), grad_stride,
        _ptr(ws), ws.numel(), _stream(stream)))


# ---------------------------------------------------------------------------
# balance loss
# ---------------------------------------------------------------------------


def _mask(mask, rows: int, logits):
    import torch

    if mask is not None:
        _need(mask.dtype in (torch.bool, torch.uint8), "row_mask: bool or uint8 expected")
        _flat(mask, rows, mask.dtype, logits, "row_mask")
    return _ptr(mask)


def balance_forward(logits, experts, row_mask, group_rows: int, coef: float, counts_out, rows_out, prob_out, loss_out,
                    ws, stream=None):
    """Per group of group_rows rows: choices per expert, valid rows, mean probabilities (prob_out may be None); and the
    balance loss.  experts: rows x k chosen ones (int32 or int64), negative where dropped."""
    import torch

    m = _logits(logits)
    rows, E = logits.shape
    _need(experts.dim() == 2 and experts.shape[0] == rows, "experts: one row per row of logits expected")
    _place(experts, logits, "experts")
    _need(group_rows >= 1, "group_rows must be at least 1")
    G = -(-rows // group_rows)
    _flat(counts_out, G * E, torch.int32, logits, "counts_out")
    _flat(rows_out, G, torch.int32, logits, "rows_out")
    _flat(prob_out, G * E, torch.float32, logits, "prob_out")
    _flat(loss_out, 1, torch.float32, logits, "loss_out")
    _scratch(ws, logits)
    r = DrRoutes(_ptr(experts), _row_stride(experts, "experts"), experts.shape[1], _index_type(experts, "experts"),
                 _mask(row_mask, rows, logits), group_rows)
    _check("dr_balance_forward", lib().dr_balance_forward(
        ctypes.byref(m), ctypes.byref(r), coef, _ptr(counts_out), _ptr(rows_out), _ptr(prob_out), _ptr(loss_out),
        _ptr(ws), ws.numel(), _stream(stream)))


def balance_backward(logits, k: int, row_mask, group_rows: int, coef: float, counts, count_rows, rows_in, upstream,
                     grad_out, stream=None):
    """The balance loss's gradient at the router's logits.  counts and count_rows: a worker's own (count_rows is
    rows_in then) or the sums over all workers; upstream: one float32, or None for 1."""
    import torch

    m = _logits(logits)
    rows, E = logits.shape
    _need(group_rows >= 1, "group_rows must be at least 1")
    G = -(-rows // group_rows)
    _flat(counts, G * E, torch.int32, logits, "counts")
    _flat(count_rows, G, torch.int32, logits, "count_rows")
    _flat(rows_in, G, torch.int32, logits, "rows_in")
    _flat(upstream, 1, torch.float32, logits, "upstream")
    grad_stride = _grad(grad_out, logits)
    r = DrRoutes(None, 0, k, INDEX_I32, _mask(row_mask, rows, logits), group_rows)
    _check("dr_balance_backward", lib().dr_balance_backward(
        ctypes.byref(m), ctypes.byref(r), coef, _ptr(counts), _ptr(count_rows), _ptr(rows_in), _ptr(upstream),
        _ptr(grad_out), grad_stride, _stream(stream)))
