"""Activations far from zero, through products and group norms, against their formulas in 64 bits.

Tolerances: half a step of the output's type; 2^-19 of the result for BF16 outputs, whose activations are made of approximations; and 2^-53
absolutely, under which the header lets SiLU and tanh-GELU of BF16 outputs come out as zero.  (erf-GELU is a difference of ones, each good to
2^-24: 2^-23 of the argument.)"""
import pytest
import torch

import _operators_ref as ref

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
INF = float("inf")
ARGS = (-45.0, 3.0, -1e2, -90.0, -1e6, 0.5, -1e18, 1e20, -1e20, -3.3e38, 1.0, INF, -INF, float("nan"), -41.0, 88.0)


def formula(v, kind):
    """The header's, at its limits: what exp sends to zero is zero, both infinities are as 64 bits have them."""
    return ref.activate(v, kind) if kind != "gelu" else v * torch.special.ndtr(v)


def close(y, v, kind):
    """y [..., n] against the activation of v [n]."""
    want = formula(v.double(), kind).expand(y.shape)
    assert torch.equal(torch.isnan(y), torch.isnan(want)), f"{kind}: {y} for {v}"
    tol = (ref.half_step(y.dtype) + 2.0 ** -19) * want.abs() + 2.0 ** -53 + (2.0 ** -23 * v.double().abs() if kind == "gelu" else 0.0)
    same, seen = y.double() == want, ~torch.isnan(want)
    bad = ((y.double() - want).abs() - tol)[seen & ~same]
    assert bad.numel() == 0 or bad.max().item() <= 0, f"{kind}: {y[0].tolist()} instead of {want[0].tolist()}"


@pytest.mark.parametrize("dtype,out", [(BF, BF), (BF, F), (F, F)])
@pytest.mark.parametrize("kind", ["silu", "gelu_tanh", "gelu"])
@pytest.mark.parametrize("rows,k", [(3, 16), (70, 16), (300, 16), (3, 8192)])              # (the last: cut along K)
def test_products(rows, k, kind, dtype, out):
    from paper_2609_31938_b200 import tokens as tk
    bias = torch.tensor(ARGS, device="cuda").clamp(torch.finfo(dtype).min, INF) if dtype == F else torch.tensor(ARGS, device="cuda")
    bias = bias.to(dtype)
    x, w = torch.zeros(rows, k, device="cuda", dtype=dtype), torch.zeros(len(ARGS), k, device="cuda", dtype=dtype)
    close(tk.linear(x, w, bias, activation=kind, out_dtype=out), bias, kind)
    # the gate of a pair: what it closes stays closed
    w2, b2 = torch.cat([w, w]), torch.cat([bias, torch.full_like(bias, 64.0)])
    y = tk.linear(x, w2, b2, activation=kind, gated=True, out_dtype=out)
    closed = (bias <= -45) & torch.isfinite(bias)
    assert bool((y[:, closed].abs() <= 64 * (2.0 ** -53 + (2.0 ** -23 * bias[closed].double().abs() if kind == "gelu" else 0.0))).all())


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("kind", ["silu", "gelu_tanh", "gelu"])
@pytest.mark.parametrize("pixels", [1, 40, 30000])
@pytest.mark.parametrize("off", [0, 3])                                  # rows on 16 bytes, and not
def test_group_norms(off, pixels, kind, dtype):
    from paper_2609_31938_b200 import tokens as tk
    c = len(ARGS)
    wide = torch.randn(2, pixels, c + 8, device="cuda").to(dtype)
    bias = torch.tensor(ARGS, device="cuda")
    x, weight = wide[..., off:off + c], torch.zeros(c, device="cuda")
    for shift in (None, bias.expand(2, -1).contiguous()):
        y = tk.group_norm(x, 2, weight, bias if shift is None else None, shift=shift, activation=kind)
        close(y.flatten(0, 1)[::997], bias, kind)


@pytest.mark.parametrize("kind", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("gated", [False, True])
def test_a_row_has_the_same_bits_beside_other_contents(gated, kind):
    from paper_2609_31938_b200 import tokens as tk
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF)  # noqa: E731
    for rows in (16, 1000):
        w, x = r(3000 * (1 + gated), 64) * 0.25, r(rows, 64)
        y = tk.linear(x, w, activation=kind, gated=gated)
        x[1::2] = r(rows // 2, 64)
        assert torch.equal(tk.linear(x, w, activation=kind, gated=gated)[::2], y[::2])
