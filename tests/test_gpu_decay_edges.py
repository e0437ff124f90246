"""Attention with decaying states at the edges of what its calls may hold, against 64 bits token by token."""
import pytest
import torch

import _operators_ref as ref
from test_gpu_decay import BF, F, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n", [5, 24, 200, 1300])
def test_states_that_grow(n, dtype):
    """Tolerance, beside those of ``test_gpu_decay``: token by token, each of 64 tokens of a chunk rounds a state twice (2^-24) and its factor
    once or twice (2^-23): 2^-16 of the magnitudes."""
    c = Case([n, 0], 3, 3, 64, 64, dtype, seed=21)
    c.fresh = torch.tensor([1, 0], device="cuda").int()
    m = min(n, 40)
    # head 0: nothing is remembered yet while the decays add up to 5 m; head 1: a state fades by exp(-60) and comes back; head 2: a little at a time
    c.g[:m, 0], c.k[:m - 1, 0] = 5.0, 0.0
    c.g[1, 1], c.g[2:m, 1] = -60.0, 60.0 / (m - 2)
    c.g[:, 2] = 0.2 - 0.4 * (torch.arange(n, device="cuda") % 2)
    if n > 200:                                                           # ... a segment's decay beyond FP32, onto a state of zeros
        c.g[:400, 0], c.k[:399, 0] = 2.0, 0.0
    out, memory = c.run()
    want, states, big_out, big = ref.decay(c.q, c.k, c.v, c.g, c.starts, c.slot.tolist(), c.fresh.tolist(), c.states, c.scale)
    assert torch.isfinite(big).all() and torch.isfinite(out).all()
    bad = (out.double() - want).abs() - ((2.0 ** -14 if dtype == BF else 2.0 ** -16) * big_out + ref.half_step(dtype) * want.abs() + 1e-30)
    assert bad.max().item() <= 0, f"out is off by {bad.max().item():.3g} more than allowed"
    bad = (memory.states.double() - states).abs() - (2.0 ** -16 * big + 1e-30)
    assert bad.max().item() <= 0, f"a state is off by {bad.max().item():.3g} more than allowed"


def test_a_small_state_and_a_large_decay_of_a_segment():
    """exp(t) beyond FP32, its product with the state within: what the scan over segments makes of it."""
    n = 1300
    c = Case([n], 1, 1, 64, 64, F, seed=22)
    c.states *= 1e-30
    c.k[:] = 0.0
    c.g[:] = 0.0
    c.g[:256] = 100.0 / 256
    out, memory = c.run()
    want, states, _, _ = ref.decay(c.q, c.k, c.v, c.g, c.starts, c.slot.tolist(), None, c.states, c.scale)
    # (a factor of exp(t) in FP32 is good to |t| 2^-24 and some roundings, a step to 2^-22, 1300 of them in a row in the worst way)
    torch.testing.assert_close(memory.states.double(), states, rtol=1300 * 2.0 ** -22, atol=0)
    torch.testing.assert_close(out.double(), want, rtol=1300 * 2.0 ** -22, atol=1300 * 2.0 ** -22 * want.abs().max().item())


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n", [6, 200, 1300])
@pytest.mark.parametrize("at", [3, 4])
def test_a_decay_of_nan_reaches_only_what_follows(at, n, dtype):
    c = Case([n], 2, 2, 64, 64, dtype, seed=23)
    clean, _ = c.run()
    bad = at if n < 100 else 64 + at
    c.g[bad, 0] = float("nan")
    out, m = c.run()
    tol = dict(rtol=2.0 ** -6 if dtype == BF else 2.0 ** -16, atol=1e-4)
    torch.testing.assert_close(out[:bad], clean[:bad], **tol)
    torch.testing.assert_close(out[:, 1], clean[:, 1], **tol)
    assert torch.isnan(out[bad:, 0]).all() and torch.isnan(m.states[c.slot[0], 0]).all() and torch.isfinite(m.states[c.slot[0], 1]).all()
    # ... and is forgotten, in the same segment of a cut sequence too
    c.g[bad + 1, 0] = -float("inf")
    out, m = c.run()
    assert torch.isnan(out[bad, 0]).all() and torch.isfinite(out[bad + 1:]).all() and torch.isfinite(m.states[c.slot[0]]).all()
    c.g[bad, 0] = 0.0
    want, w = c.run()
    torch.testing.assert_close(out[bad + 1:], want[bad + 1:], **tol)
    torch.testing.assert_close(m.states, w.states, rtol=2.0 ** -16, atol=1e-5)
