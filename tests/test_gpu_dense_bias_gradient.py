"""The bias' gradient of a dense layer is float32, whatever the operands' type: so are the slopes that it is summed from."""
import numpy as np
import pytest
import torch

import paper_2505_15511_amd as nomad
from oracle import map_oracle as mo
from test_gpu_map_operators import BF16, F16, F32, U32, host, near, note, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("out", [4096, 4097])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("activation", ["silu", "gelu"])
def test_one_row_s_slopes(out, dtype, activation):
    """Of one row db is dy act'(z). A slope is made of a fit good to 2.2 units of 2^-24, an exponential whose argument's rounding counts x e^-x <= 0.37 units of twice 2^-24,
    reciprocals and half a dozen roundings: 8 (1 + |z|) units hold them."""
    note(f"slopes {out} {dtype} {activation}")
    rng = np.random.default_rng(out)
    x, dy, w = randn((1, 8), dtype, rng), randn((1, out), dtype, rng), randn((out, 8), dtype, rng)
    z = torch.linspace(-6.0, 6.0, out, device="cuda").to(dtype)[None]
    want = mo.dense_gradient(host(dy), host(x), host(w), activation, host(z))[2]
    db = nomad.dense_gradient(dy, x, w, activation, z)[2]
    near(db, want, (8 * U32 * (1 + np.abs(host(z))) * np.abs(host(dy)))[0] + 2 * U32 * np.abs(want), F32, "db")
