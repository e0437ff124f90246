"""Products at the edges of their forms, against 64 bits (tolerances: ``test_gpu_linear.close``) or bit by bit."""
import pytest
import torch

from test_gpu_linear import BF, F, KINDS, close, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,out", KINDS)
def test_residuals_by_boxes_and_outputs_by_elements_over_many_tiles(dtype, out):
    from paper_2609_31938_b200 import tokens as tk
    # (several whole tiles for each pair of SMs, the last features of a tile in some lanes only)
    x, w, b, r = inputs(5000, 4200, 200, dtype, False, out, seed=3)
    want = tk.linear(x, w, b, activation="silu", residual=r, out_dtype=out)
    close(want, x, w, b, "silu", False, r)
    wide = torch.full((5000, 4203), -3.0, device="cuda", dtype=out)
    off = torch.empty((5000, 4209), device="cuda", dtype=out)
    off[:, 7:4207] = r
    for _ in range(3):
        for res in (r, off[:, 7:4207]):
            tk.linear(x, w, b, activation="silu", residual=res, out=wide[:, 1:4201])
            assert torch.equal(wide[:, 1:4201], want) and bool((wide[:, 0] == -3).all()) and bool((wide[:, 4201:] == -3).all())
    assert tk.status() == 0
