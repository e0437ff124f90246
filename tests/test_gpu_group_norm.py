"""Group norms on channels-last activations against 64 bits.

Tolerances: half a step of the output's type, and what ``_operators_ref.group_norm`` says of the statistics: sums run in chains of some
hundred additions, whose random roundings come to less than 2^-18 of the mean magnitude.  BF16 outputs have activations from approximations
good to 2^-20."""
import pytest
import torch

import _operators_ref as ref

pytestmark = pytest.mark.gpu
ACTS = ("none", "silu", "gelu", "gelu_tanh")


def inputs(s, p, c, dtype, seed=0, mean=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *n: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    return (r(s, p, c) + mean * r(c)).to(dtype), 1 + 0.2 * r(c), 0.3 * r(c), 0.3 * r(s, c), 0.3 * r(s, c)


def close(y, want, err):
    tol = err + (ref.half_step(y.dtype) + 2.0 ** -20) * want.abs() + 1e-30
    bad = (y.double() - want).abs() - tol
    assert bool(torch.isfinite(y).all()) and bad.max().item() <= 0, f"off by {bad.max().item():.3g} more than allowed"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("s,p,c,groups", [
    (1, 16, 8, 1), (3, 1, 64, 2), (2, 5, 200, 25), (1, 97, 192, 32), (2, 301, 96, 96), (7, 63, 6, 3), (1, 7040, 96, 32), (2, 1100, 130, 13), (1, 40, 5000, 8),
    (2, 3, 16384, 4), (1, 30011, 40, 5), (1, 70001, 33, 3), (1, 300, 4104, 3)])
def test_against_64_bits(s, p, c, groups, dtype):
    from paper_2609_31938_b200 import tokens as tk
    x, w, b, sc, sh = inputs(s, p, c, dtype)
    for i, act in enumerate(ACTS):
        mod = i % 2 == 0
        y = tk.group_norm(x, groups, w, b, scale=sc if mod else None, shift=sh if mod else None, eps=1e-5, activation=act)
        close(y, *ref.group_norm(x, groups, w, b, sc if mod else None, sh if mod else None, 1e-5, act))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_alignment_and_in_place(dtype):
    from paper_2609_31938_b200 import tokens as tk
    x, w, b, sc, sh = inputs(3, 50, 48, dtype, seed=1)
    want = ref.group_norm(x, 6, w, b, sc, sh, 1e-6, "silu")
    wide = torch.full((3, 53, 61), float("nan"), device="cuda", dtype=dtype)
    wide[:, 2:52, 5:53] = x                                               # rows start off 16 bytes
    out = torch.full((50, 3, 96), -7.0, device="cuda", dtype=dtype)       # pixel by pixel, samples between
    y = tk.group_norm(wide[:, 2:52, 5:53], 6, w, b, scale=sc, shift=sh, activation="silu", out=out.transpose(0, 1)[..., 16:64])
    close(y, *want)
    assert bool((out[..., :16] == -7).all()) and bool((out[..., 64:] == -7).all())
    mod = torch.randn(3, 2, 48, device="cuda")
    mod[:, 0], mod[:, 1] = sc, sh
    z = x.clone()
    assert tk.group_norm(z, 6, w, b, scale=mod[:, 0], shift=mod[:, 1], activation="silu", out=z) is z
    close(z, *want)
    one = x[:1].expand(3, -1, -1)                                         # a broadcast sample
    close(tk.group_norm(one, 6, w, b), *ref.group_norm(one.contiguous(), 6, w, b, None, None, 1e-6, "none"))


@pytest.mark.parametrize("p", [9, 40000])
def test_large_mean_constant_and_not_finite(p):
    from paper_2609_31938_b200 import tokens as tk
    x, w, b, _, _ = inputs(4, p, 32, torch.float32, seed=2)
    x[1] += 1000.0
    x[2, :, :4] = 3.0                                                     # a group without spread
    want, err = ref.group_norm(x, 8, w, b, None, None, 1e-6, "none")
    x[3, 3, 9] = float("nan")
    x[3, 1, 30] = float("inf")
    y = tk.group_norm(x, 8, w, b)
    close(y[:3], want[:3], err[:3])
    torch.testing.assert_close(y[2, :, :4], b[:4].expand(p, -1), rtol=0, atol=1e-2 if p > 100 else 1e-3)   # (sqrt(eps) of the mean's last bit)
    bad = torch.isnan(y[3]).all(0)
    assert bad[8:12].all() and bad[28:].all() and not torch.isnan(y[3, :, :8]).any() and not torch.isnan(y[3, :, 12:28]).any()


@pytest.mark.parametrize("c,h,w,groups", [(96, 9, 13, 32), (192, 44, 80, 32), (96, 150, 150, 8), (64, 1, 1, 4)])
def test_rings(c, h, w, groups):
    import paper_2609_31938_b200 as ccv
    n, t = 2, 3
    x = (torch.randn(n, c, t, h, w, device="cuda") + torch.randn(c, 1, 1, 1, device="cuda")).bfloat16()
    g = torch.Generator(device="cuda").manual_seed(3)
    wt, b = 1 + 0.2 * torch.randn(c, generator=g, device="cuda"), torch.randn(c, generator=g, device="cuda")
    sc, sh = (0.3 * torch.randn(n * t, c, generator=g, device="cuda") for _ in range(2))
    a, o = ccv.FrameRing(n, c, 5, h, w, zero=True), ccv.FrameRing(n, c, 4, h, w, zero=True)
    a.load(3, x)                                                          # slots 3, 4, 0
    a.group_norm(3, t, groups, wt, b, scale=sc, shift=sh, activation="silu", out_ring=o, out_slot=2)
    rows = x.permute(0, 2, 3, 4, 1).reshape(n * t, h * w, c)
    want, err = ref.group_norm(rows, groups, wt, b, sc, sh, 1e-6, "silu")
    back = lambda r, s: r.store(s, t).permute(0, 2, 3, 4, 1).reshape(n * t, h * w, c)  # noqa: E731
    close(back(o, 2), want, err)
    assert bool((o.buf[:, 1] == 0).all()) and torch.equal(a.store(3, t), x)
    whole = back(o, 2)
    # a frame by itself has the same bits, and so has the norm in place
    for i in range(t):
        a.group_norm((3 + i) % 5, 1, groups, wt, b, scale=sc[i::t], shift=sh[i::t], activation="silu", out_ring=o, out_slot=i)
    assert torch.equal(back(o, 0), whole)
    a.group_norm(3, t, groups, wt, b, scale=sc, shift=sh, activation="silu")
    assert torch.equal(back(a, 3), whole)


def test_streams_and_graphs():
    from paper_2609_31938_b200 import tokens as tk
    x, w, b, _, _ = inputs(2, 40000, 64, torch.bfloat16, seed=4)
    want = tk.group_norm(x, 8, w, b, activation="silu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = tk.group_norm(x, 8, w, b, activation="silu")
    side.synchronize()
    assert torch.equal(y, want)
    graph, still = torch.cuda.CUDAGraph(), x.clone()
    with torch.cuda.graph(graph):
        z = tk.group_norm(still, 8, w, b, activation="silu")
    still.copy_(x.flip(0))
    graph.replay()
    assert torch.equal(z, want.flip(0))


def test_far_offsets():
    from paper_2609_31938_b200 import tokens as tk
    x = torch.zeros(2, 1 << 21, 544, device="cuda", dtype=torch.bfloat16)        # 2.28e9 elements
    x[1, -1] = torch.randn(544, device="cuda").bfloat16()
    x[1, 0] = -x[1, -1]
    edge = x[1, -1].clone()
    y = tk.group_norm(x, 1, out=x)
    std = (2 * edge.double().square().sum() / (1 << 21) / 544 + 1e-6).sqrt()
    torch.testing.assert_close(y[1, -1].double(), edge.double() / std, rtol=2.0 ** -8, atol=0)
    torch.testing.assert_close(y[1, 0].double(), -edge.double() / std, rtol=2.0 ** -8, atol=0)
    # the mean is zero but for the rounding of the tiles' means: 2^-18 of the mean magnitude, as everywhere here, in units of the deviation
    off = 2.0 ** -18 * 2 * edge.double().abs().sum() / (1 << 21) / 544 / std
    assert bool((y[0] == 0).all()) and bool((y[1, 1:-1:997].abs() <= off).all())


def test_nothing_to_do():
    from paper_2609_31938_b200 import tokens as tk
    for shape in ((0, 5, 8), (3, 0, 8)):
        x = torch.empty(shape, device="cuda")
        assert tk.group_norm(x, 2).shape == shape
