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


FIRST_IN_A_CAPTURE = """
import torch
import paper_2609_31938_b200 as ccv
from paper_2609_31938_b200 import tokens as tk

x, w = torch.randn(40, 64, device="cuda"), torch.randn(24, 64, device="cuda")
given, call = [], ccv.lib.ccv3d_linear
class Library:
    def __getattr__(self, name):
        return getattr(ccv.lib, name)
    def ccv3d_linear(self, *a):
        given.append(a[-2])
        return call(*a)
tk.lib = Library()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    y = tk.linear(x, w)                                     # the process's first product
graph.replay()
assert tk.status() == 0 and torch.equal(y, tk.linear(x, w)) and given[0] and given[0] == given[1], given
# what is reported there is read
memory = tk.DecayMemory.empty(1, 1, 64, 64)
q = torch.zeros(1, 1, 64, device="cuda")
ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
batch, h, g = tk.StreamBatch(ints(0, 1), ints(5), 1), ccv.Heads(q.data_ptr(), 64, 64), torch.zeros(1, 1, device="cuda")
out = torch.zeros_like(q)
assert ccv.ccv3d_decay_attend(memory.c, batch.c(1), h, h, h, g.data_ptr(), 1, 1, ccv.Heads(out.data_ptr(), 64, 64), 1, ccv.F32, 1.0, status=given[0],
                              stream=torch.cuda.current_stream().cuda_stream) == ccv.OK
assert tk.status() == ccv.TOKENS_BAD_SLOT and tk.status() == 0
"""


def test_a_first_product_inside_a_capture_has_a_word_to_report_in():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_IN_A_CAPTURE], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
