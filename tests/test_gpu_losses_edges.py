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
