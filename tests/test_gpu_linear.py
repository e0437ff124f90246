"""Products with their epilogue against 64 bits.

Tolerances, for a sum of products with magnitudes `mass`: the tensor cores add 16 products at a time and cut the sum at its last bit
(2^-23), k / 16 times in a row for BF16 outputs, some 28 times and then, rounded, k / 256 (F32: k / 64) times for F32 ones; the parts of an
F32 operand that are left out are under 2^-23.  An activation from approximations adds 2^-19 of itself, and the output half a step of its
type (with a residual: of the sum)."""
import pytest
import torch

import _operators_ref as ref

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def inputs(m, n, k, dtype, gated=False, out=None, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    rows = n * (1 + gated)
    # rows of x and weights lie in wider ones, whose rest is NaN: nothing behind k counts
    pad = -(-(k + 3) // 8) * 8
    x, w = torch.full((m, pad), float("nan"), device="cuda", dtype=dtype), torch.full((rows, pad), float("nan"), device="cuda", dtype=dtype)
    x[:, :k], w[:, :k] = r(m, k).to(dtype), (r(rows, k) * k ** -0.5).to(dtype)
    return x[:, :k], w[:, :k], (0.5 * r(rows)).to(dtype), (2 * r(m, n)).to(out or dtype)


def close(y, x, w, bias, act, gated, residual):
    want, mass, part = ref.linear(x, w, bias, act, gated, residual)
    k = x.shape[1]
    cuts = k / 16 + 4 if y.dtype == BF else 32 + k / 64
    tol = cuts * 2.0 ** -23 * mass + 2.0 ** -19 * part + ref.half_step(y.dtype) * want.abs() * 1.01 + 1e-30
    if residual is not None and y.dtype == BF:
        tol = tol + 2.0 ** -20 * residual.double().abs()
    bad = (y.double() - want).abs() - tol
    assert bool(torch.isfinite(y).all()) and bad.max().item() <= 0, f"off by {bad.max().item():.3g} more than allowed"


KINDS = [(BF, BF), (BF, F), (F, F)]


@pytest.mark.parametrize("dtype,out", KINDS)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 700, 200), (3, 257, 1160), (16, 255, 64), (17, 96, 72), (64, 300, 520), (65, 130, 33), (128, 128, 128),
                                   (129, 513, 95), (300, 64, 1000), (777, 391, 264)])
def test_against_64_bits(m, n, k, gated, dtype, out):
    from paper_2609_31938_b200 import tokens as tk
    x, w, b, r = inputs(m, n, k, dtype, gated, out, seed=m + n + k)
    for act, bias, res in (("none", None, None), ("silu", b, r), ("gelu", b, None), ("gelu_tanh", None, r)):
        close(tk.linear(x, w, bias, activation=act, gated=gated, residual=res, out_dtype=out), x, w, bias, act, gated, res)


@pytest.mark.parametrize("dtype,out", KINDS)
@pytest.mark.parametrize("m,n,k,gated", [(5, 3000, 4096, False), (100, 2500, 4096, True), (2, 512, 16384, False), (600, 700, 6144, False), (2500, 1600, 1024, True),
                                         (5000, 4200, 512, False)])
def test_larger_cut_along_k(m, n, k, gated, dtype, out):
    from paper_2609_31938_b200 import tokens as tk
    x, w, b, r = inputs(m, n, k, dtype, gated, out, seed=7)
    y = tk.linear(x, w, b, activation="silu", gated=gated, residual=r, out_dtype=out)
    close(y, x, w, b, "silu", gated, r)
    assert torch.equal(y, tk.linear(x, w, b, activation="silu", gated=gated, residual=r, out_dtype=out))      # the same bits again
    assert tk.status() == 0


@pytest.mark.parametrize("dtype,out", KINDS)
def test_output_strides_and_in_place(dtype, out):
    from paper_2609_31938_b200 import tokens as tk
    x, w, b, r = inputs(70, 45, 96, dtype, False, out, seed=1)
    want = tk.linear(x, w, b, residual=r, out_dtype=out)
    close(want, x, w, b, "none", False, r)
    wide = torch.full((70, 53), -3.0, device="cuda", dtype=out)
    tk.linear(x, w, b, residual=r, out=wide[:, 3:48])
    assert torch.equal(wide[:, 3:48], want) and bool((wide[:, :3] == -3).all()) and bool((wide[:, 48:] == -3).all())
    again = r.clone()
    assert torch.equal(tk.linear(x, w, b, residual=again, out=again), want)
    # residuals and outputs as boxes, by elements, and one of each: the same bits
    for rows in (40, 600):
        x, w, b, r = inputs(rows, 160, 96, dtype, False, out, seed=2)
        want = tk.linear(x, w, b, residual=r, out_dtype=out, activation="silu")
        close(want, x, w, b, "silu", False, r)
        wide, off = (torch.zeros((rows, 177), device="cuda", dtype=out) for _ in range(2))
        wide[:, 5:165] = r
        for res in (r, wide[:, 5:165]):
            for to in (torch.empty_like(r), off[:, 9:169]):
                assert torch.equal(tk.linear(x, w, b, residual=res, out=to, activation="silu"), want)
    x, w, b, r = inputs(70, 45, 96, dtype, False, out, seed=1)
    close(tk.linear(x, w, b, residual=r[:1].expand(70, -1), out_dtype=out), x, w, b, "none", False, r[:1].expand(70, -1))
    one = x[:1].expand(70, -1)
    if dtype == BF:                                              # (rows on one another: any stride)
        with pytest.raises(Exception):
            tk.linear(one, w, b)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("m", [3, 70, 300])
def test_what_is_not_finite_stays_in_its_row_and_column(m, dtype):
    from paper_2609_31938_b200 import tokens as tk
    x, w, b, _ = inputs(m, 300, 130, dtype, seed=2)
    want = tk.linear(x, w, b)
    x[1, 5], w[7, 3], w[299, 129] = float("nan"), float("inf"), float("nan")
    y = tk.linear(x, w, b)
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[1], keep[:, 7], keep[:, 299] = False, False, False
    assert torch.equal(y[keep], want[keep]) and torch.isnan(y[1]).all() and torch.isnan(y[:, 299]).all()
    assert not torch.isfinite(y[:, 7]).any()
    if dtype == BF:
        assert torch.isinf(y[torch.arange(m, device="cuda") != 1, 7]).all()


def test_large_and_small_f32():
    from paper_2609_31938_b200 import tokens as tk
    x, w, _, _ = inputs(20, 40, 64, F, seed=3)
    for f in (2.0 ** 60, 2.0 ** -60):
        torch.testing.assert_close(tk.linear(x * f, w), tk.linear(x, w) * f, rtol=0, atol=0)
    top = torch.full((1, 64), torch.finfo(F).max, device="cuda")
    one = torch.zeros(64, 64, device="cuda")
    one.fill_diagonal_(0.5)
    assert torch.equal(tk.linear(top, one), top * 0.5)


@pytest.mark.parametrize("dtype", [BF, F])
def test_streams_and_graphs(dtype):
    from paper_2609_31938_b200 import tokens as tk
    x, w, b, _ = inputs(90, 1100, 2048, dtype, seed=4)
    want = tk.linear(x, w, b, activation="gelu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = [tk.linear(x, w, b, activation="gelu") for _ in range(3)]
    side.synchronize()
    assert all(torch.equal(v, want) for v in y)
    still = x.clone(memory_format=torch.contiguous_format)
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(tk.linear(still, w, b, activation="gelu"))
    still.copy_(x.flip(0))
    for gr in graphs:
        gr.replay()
    assert all(torch.equal(o, want.flip(0)) for o in outs)


def test_far_offsets():
    from paper_2609_31938_b200 import tokens as tk
    m, n = 140_001, 16_400                                       # 2.3e9 outputs
    x, w = torch.zeros(m, 16, device="cuda", dtype=BF), torch.zeros(n, 16, device="cuda", dtype=BF)
    x[-3:] = torch.randn(3, 16, device="cuda").to(BF)
    w[-5:] = torch.randn(5, 16, device="cuda").to(BF)
    y = tk.linear(x, w)
    close(y[-3:, -5:], x[-3:], w[-5:], None, "none", False, None)
    assert bool((y[:-3, ::97] == 0).all()) and bool((y[-3:, :-5] == 0).all())


def test_no_rows():
    from paper_2609_31938_b200 import tokens as tk
    assert tk.linear(torch.empty(0, 64, device="cuda"), torch.empty(5, 64, device="cuda")).shape == (0, 5)
