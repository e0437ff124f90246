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


def attend(c, max_new):
    from paper_2609_31938_b200 import tokens as tk
    m = tk.DecayMemory(c.states.clone())
    return m.attend(c.q, c.k, c.v, c.g, tk.StreamBatch(c.starts, c.slot, max_new, fresh=c.fresh)), m


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("new,heads", [([1] * 200 + [3000] + [1] * 200, 4), ([2, 1500, 0, 30, 900, 257, 256, 1], 2), ([1] * 40 + [2100], 1)])
def test_single_tokens_beside_long_prompts(new, heads, dtype):
    c = Case(new, heads, 1, 64, 64, dtype, seed=31, rate=0.02)
    g = torch.Generator(device="cuda").manual_seed(1)
    c.fresh = (torch.rand(len(new), generator=g, device="cuda") < 0.3).int()
    out, m = c.run()
    c.check(out, m)
    assert m.status() == 0
    again, other = c.run()
    assert torch.equal(out, again) and torch.equal(m.states, other.states)
    # a bound that is far off: the same
    out, m = attend(c, 100_000)
    c.check(out, m)
    assert m.status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("new,heads", [([200] * 40, 8), ([200], 2), ([150, 140], 1)])
def test_a_loose_bound_does_not_change_a_bit(new, heads, dtype):
    c = Case(new, heads, heads, 64, 128, dtype, seed=32)
    out, m = attend(c, max(new))
    loose, other = attend(c, 1 << 30)
    assert torch.equal(out, loose) and torch.equal(m.states, other.states) and m.status() == other.status() == 0
    c.check(out, m)


@pytest.mark.parametrize("singles,prompt", [(256, 4000), (1024, 28000), (65000, 1000)])
def test_scratch_goes_by_what_is_cut(singles, prompt):
    """No more than the states of two segments for each 256 tokens, however many sequences there are."""
    import paper_2609_31938_b200 as ccv
    some = torch.zeros(16, device="cuda")
    at = some.data_ptr()
    for dtype in (ccv.BF16, ccv.F32):
        memory = ccv.DecayMemoryC(at, singles + 1, 32, 128, 128)
        tokens = singles + prompt
        for bound in (prompt, 1 << 30):
            s, n = ccv.ccv3d_decay_attend_workspace(memory, ccv.StreamBatchC(at, at, None, singles + 1, tokens, bound), 32, dtype)
            assert s == ccv.OK and n <= 2 * (tokens / 256 + 1) * 32 * (128 * 128 + 1) * 4 + 512


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n", [4, 100, 1000])
def test_bad_offsets_leave_other_sequences_and_states_alone(n, dtype):
    from paper_2609_31938_b200 import TOKENS_BAD_LENGTH, TOKENS_BAD_SLOT
    c = Case([n, 3, n, 2], 2, 2, 64, 64, dtype, seed=33)
    want, w = c.run()
    for starts, untouched in (([0, n, 10 * n, 2 * n + 3, 2 * n + 5], [0, 3]),      # one ends past the rows, the next begins there
                              ([0, n, -7, 2 * n + 3, 2 * n + 5], [3])):            # ... or below the first, whose rows are then written twice
        good = c.starts.clone()
        c.starts[:] = torch.tensor(starts, device="cuda")
        out, m = attend(c, max(c.new))
        assert m.status() & TOKENS_BAD_LENGTH
        c.starts = good
        for b in (0, 3):
            rows = slice(int(good[b]), int(good[b + 1]))
            tol = dict(rtol=2.0 ** -6 if dtype == BF else 2.0 ** -16, atol=1e-3)
            if b in untouched:
                torch.testing.assert_close(out[rows], want[rows], **tol)
            torch.testing.assert_close(m.states[c.slot[b]], w.states[c.slot[b]], rtol=2.0 ** -16, atol=1e-4)
        free = torch.ones(len(c.states), dtype=torch.bool, device="cuda")
        free[c.slot.long()] = False
        assert torch.equal(m.states[free], c.states[free])
    # a slot outside the pool: no state changes but those of the others
    slot, c.slot = c.slot.clone(), c.slot.clone()
    c.slot[0], c.slot[2] = -1, 1 << 30
    out, m = attend(c, max(c.new))
    assert m.status() == TOKENS_BAD_SLOT
    lost = slot[[0, 2]].long()
    assert torch.equal(m.states[lost], c.states[lost])
    torch.testing.assert_close(m.states[slot[1]], w.states[slot[1]], rtol=2.0 ** -16, atol=1e-4)
    torch.testing.assert_close(m.states[slot[3]], w.states[slot[3]], rtol=2.0 ** -16, atol=1e-4)
