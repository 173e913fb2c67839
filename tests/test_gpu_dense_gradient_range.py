"""Gradients of a dense layer whose dy comes near float16's end: slopes of SiLU and GELU are above 1 in places, dz = dy act'(z) is kept in float16, and results that
float16 holds have to be finite.

Tolerances as in tests/test_gpu_more_operators.py: a sum's K roundings of 2^-24, dz's own rounding (half a unit of 2^-10, or of the smallest step, 2^-24, which a
dz that is kept as 7/8 of itself has as 8/7 of that), and the result's."""
import numpy as np
import pytest
import torch

import paper_2505_15511_amd as nomad
from oracle import map_oracle as mo
from test_gpu_map_operators import F16, F32, U32, UNIT, host, near, note, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,inner,out", [(3, 16, 5), (300, 24, 40), (700, 264, 272), (33_000, 72, 136), (9000, 512, 256)])
@pytest.mark.parametrize("activation", ["silu", "gelu", "relu"])
def test_dy_near_float16_s_end(rows, inner, out, activation):
    note(f"dy near the end rows={rows} {inner}->{out} {activation}")
    rng = np.random.default_rng(rows + inner)
    x, w = randn((rows, inner), F16, rng, 0.25 / rows), randn((out, inner), F16, rng, 2.0 ** -10 / out ** 0.5)
    dy, z = randn((rows, out), F16, rng), randn((rows, out), F16, rng, 2.0)
    there = torch.from_numpy(rng.random((rows, out)) < 0.05).cuda()
    there[0, 0] = True                                                    # (at least one)
    dy[there] = torch.where(dy[there] > 0, 65504.0, -65504.0).to(F16)
    z[there] = 1.5                                                        # slopes of 1.04 and 1.13
    want_dx, want_dw, want_db, dz = mo.dense_gradient(host(dy), host(x), host(w), activation, host(z))
    assert np.abs(want_dx).max() < 65504 and np.abs(want_dw).max() < 65504 and (activation == "relu" or np.abs(dz).max() > 65520)
    slope = (16 * U32 * (1 + np.abs(host(z))) + 2.0 ** -16) * np.abs(host(dy))
    off = slope + UNIT[F16] * np.abs(dz) + 2.0 ** -25 * 8 / 7
    for ww in (w, w.t().contiguous().t()):
        for wide in (F16, F32):
            dx, dw, db = nomad.dense_gradient(dy, x, ww, activation, z, out_dtype=wide)
            assert torch.isfinite(dx).all() and torch.isfinite(dw).all()
            near(dx, want_dx, (out + 8) * U32 * (np.abs(dz) @ np.abs(host(w))) + 1.01 * off @ np.abs(host(w)), F16, "dx")
            near(dw, want_dw, (rows + 8) * U32 * (np.abs(dz).T @ np.abs(host(x))) + 1.01 * off.T @ np.abs(host(x)), wide, "dw")
            near(db, want_db, (rows + 8) * U32 * np.abs(dz).sum(0) + slope.sum(0), F32, "db")
