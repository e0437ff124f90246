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


@pytest.mark.parametrize("rows", [40, 500, 3000])
def test_long_sums_into_f32_are_cut_no_more_than_within_512_terms(rows):
    """Sums of positive products show every cut.  Of 32 partial sums s1 < s2 < .. < s32 of 16 products each, a cut takes half a last bit in the mean,
    2^-24 of the sum at most; s1 + .. + s32 are 16.5 s32: 16.5 2^-24 in the mean, and a rounding or two of a whole sum."""
    from paper_2609_31938_b200 import tokens as tk
    g = torch.Generator(device="cuda").manual_seed(9)
    x, w = (torch.randn(n, 1024, generator=g, device="cuda").exp() for n in (rows, 500))       # (with bits far below the sums')
    x, w = x.to(BF), w.to(BF)
    want = x.double() @ w.double().T
    off = (tk.linear(x, w, out_dtype=F).double() / want - 1).abs().mean().item()
    assert off <= 18 * 2.0 ** -24, f"{off * 2 ** 24:.1f} x 2^-24 in the mean"


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("m,k", [(5, 1024), (5, 1025), (64, 1088), (16, 20000), (300, 40000), (33, 65536)])
def test_depths_around_a_hand_over(m, k, gated, act):
    from paper_2609_31938_b200 import tokens as tk
    for dtype, out in KINDS:
        x, w, b, r = inputs(m, 130, k, dtype, gated, out, seed=k + m)
        close(tk.linear(x, w, b, activation=act, gated=gated, residual=r, out_dtype=out), x, w, b, act, gated, r)
    assert tk.status() == 0


@pytest.mark.parametrize("dtype,out", KINDS)
@pytest.mark.parametrize("m,n,k,gated", [(5, 3000, 4096, False), (100, 2500, 4096, True), (600, 700, 6144, False)])
def test_in_place_on_the_residual_of_a_product_cut_along_its_depth(m, n, k, gated, dtype, out):
    from paper_2609_31938_b200 import tokens as tk
    x, w, b, r = inputs(m, n, k, dtype, gated, out, seed=11)
    want = tk.linear(x, w, b, activation="gelu", gated=gated, residual=r, out_dtype=out)
    close(want, x, w, b, "gelu", gated, r)
    wide = torch.zeros(m, n + 9, device="cuda", dtype=out)
    for there in (r.clone(), wide[:, 3:n + 3]):
        there.copy_(r)
        assert torch.equal(tk.linear(x, w, b, activation="gelu", gated=gated, residual=there, out=there), want)


@pytest.mark.parametrize("rows", [20, 70])
def test_large_and_small_f32_by_either_form(rows):
    """In plain arithmetic (few rows), and split into BF16 parts."""
    from paper_2609_31938_b200 import tokens as tk
    x, w, _, _ = inputs(rows, 40, 64, F, seed=3)
    for f in (2.0 ** 60, 2.0 ** -60):
        assert torch.equal(tk.linear(x * f, w), tk.linear(x, w) * f)
    top = torch.full((rows, 64), torch.finfo(F).max, device="cuda")
    top[1::2] *= -1
    one = torch.zeros(64, 64, device="cuda")
    one.fill_diagonal_(0.5)
    assert torch.equal(tk.linear(top, one), top * 0.5)
    # numbers next to the largest of BF16, 3.3895e38, and the three parts of a number of 24 bits
    top = torch.full((rows, 64), 3.39e38, device="cuda")
    top[:, 1], top[:, 2], top[:, 3] = 3.3895e38, 3.3896e38, 1.0 + 2.0 ** -23
    assert torch.equal(tk.linear(top, one), top * 0.5)
