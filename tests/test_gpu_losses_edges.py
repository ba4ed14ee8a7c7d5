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
