"""Grouped products and gradients in every tile and every way in which rows are loaded and stored: layers with few columns out (a map's
coordinates), whose gradients' tiles are 128 columns by 16, and wide ones with rows that are no whole 16-byte chunks; groups in parts, short
and empty ones.  What is checked, and its bounds, is in test_gpu_map_operators."""
import pytest
import torch

import test_gpu_map_operators as operators

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16

#: (groups, rows, in, out, type, how rows fall into groups)
NARROW = [(4, 3000, 65, 2, F32, "ragged"), (3, 2500, 128, 1, F32, "ragged"), (5, 4000, 256, 2, F32, "ragged"), (1, 20_000, 256, 2, F32, "one"), (5, 4000, 256, 16, F32, "ragged"),
          (2, 2100, 129, 3, F32, "ragged"), (300, 900, 128, 2, F32, "ragged"), (3, 64, 132, 2, F32, "empty"), (2, 1, 68, 16, F32, "one"),
          (3, 3000, 256, 16, BF16, "ragged"), (4, 3000, 128, 2, BF16, "ragged"), (3, 2000, 129, 3, BF16, "ragged"), (2, 2000, 65, 1, BF16, "ragged"), (1, 9000, 264, 2, BF16, "one"),
          (3, 3000, 264, 16, F16, "ragged"), (4, 3000, 128, 2, F16, "ragged"), (3, 2000, 129, 3, F16, "ragged"), (2, 2000, 66, 16, F16, "ragged"), (90, 700, 72, 8, F16, "ragged")]

WIDE = [(3, 900, 50, 256, F32, "ragged"), (2, 1100, 129, 250, F32, "ragged"), (3, 900, 52, 256, BF16, "ragged"), (2, 1100, 129, 250, F16, "ragged"),
        (2, 700, 256, 200, F32, "ragged"), (2, 700, 250, 200, BF16, "ragged"), (2, 700, 256, 120, F16, "ragged"), (2, 900, 124, 252, F32, "ragged"), (1, 5000, 250, 256, BF16, "one"),
        (2, 900, 60, 64, F32, "ragged"), (2, 900, 64, 60, BF16, "ragged"), (2, 900, 62, 64, BF16, "ragged"), (2, 900, 64, 63, F32, "ragged"), (2, 900, 61, 64, F32, "ragged"),
        (2, 900, 256, 250, F32, "ragged"), (2, 900, 256, 250, BF16, "ragged")]


@pytest.mark.parametrize("groups,total,inner,out,dtype,kind", NARROW + WIDE)
@pytest.mark.parametrize("gathered", [False, True])
def test_weight_gradient(groups, total, inner, out, dtype, kind, gathered):
    operators.test_weight_gradient(groups, total, inner, out, dtype, kind, gathered)


@pytest.mark.parametrize("groups,total,inner,out,dtype,kind", NARROW + WIDE)
@pytest.mark.parametrize("turned", [False, True])
def test_product(groups, total, inner, out, dtype, kind, turned):
    operators.test_product(groups, total, inner, out, dtype, kind, turned, True)
