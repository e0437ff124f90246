"""Attention with decaying states against 64 bits, token by token.

Tolerances, in terms of the same recurrence with magnitudes throughout (`big`): outputs of BF16 inputs 2^-14 of it (scores, states and decayed
values as BF16 numbers of 16 bits and more, each product within 2^-16, sums cut at 2^-23 some ten times) and half a step of BF16; states, and
outputs of F32 inputs, 2^-19 (24 bits, some thirty cuts of 2^-23)."""
import pytest
import torch

import _operators_ref as ref

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


class Case:
    def __init__(self, new, heads, qk_heads, dk, dv, dtype, seed=0, rate=0.05, slots=None, rows_behind=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.new, n = list(new), sum(new) + rows_behind
        slots = slots or len(new) + 2
        fused = r(n, 2 * qk_heads * dk + heads * dv)
        fused[:, qk_heads * dk:2 * qk_heads * dk] *= dk ** -0.5
        fused = fused.to(dtype)
        self.q, self.k = fused[:, :qk_heads * dk].view(n, qk_heads, dk), fused[:, qk_heads * dk:2 * qk_heads * dk].view(n, qk_heads, dk)
        self.v = fused[:, 2 * qk_heads * dk:].view(n, heads, dv)
        self.g = -rate * torch.exp(r(n, heads))
        self.states = r(slots, heads, dk, dv)
        self.slot = torch.randperm(slots, generator=g, device="cuda")[:len(new)].int()
        self.starts = torch.tensor([0] + self.new, device="cuda").cumsum(0).int()
        self.scale = dk ** -0.5
        self.fresh = None

    def run(self, **kw):
        from paper_2609_31938_b200 import tokens as tk
        m = tk.DecayMemory(self.states.clone())
        out = m.attend(self.q, self.k, self.v, self.g, tk.StreamBatch(self.starts, self.slot, max(self.new + [1]), fresh=self.fresh), **kw)
        return out, m

    def check(self, out, m, rows=None):
        want, states, big_out, big = ref.decay(self.q, self.k, self.v, self.g, self.starts, self.slot.tolist(),
                                               None if self.fresh is None else self.fresh.tolist(), self.states, self.scale)
        n = sum(self.new) if rows is None else rows
        part = 2.0 ** -14 if out.dtype == BF else 2.0 ** -19
        bad = (out[:n].double() - want[:n]).abs() - (part * big_out[:n] + ref.half_step(out.dtype) * want[:n].abs() + 1e-30)
        assert n == 0 or bad.max().item() <= 0, f"out is off by {bad.max().item():.3g} more than allowed"
        bad = (m.states.double() - states).abs() - (2.0 ** -19 * big + 1e-30)
        assert bad.max().item() <= 0, f"a state is off by {bad.max().item():.3g} more than allowed"


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (64, 192), (128, 256), (64, 512)])
@pytest.mark.parametrize("new", [[1], [1, 0, 3, 8], [9], [64, 1, 65], [130, 0, 63, 17]])
def test_against_64_bits(new, dk, dv, dtype):
    c = Case(new, 4, 2, dk, dv, dtype, seed=dk + dv)
    out, m = c.run()
    c.check(out, m)
    assert m.status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("new,heads,dk,dv", [([1500], 3, 64, 64), ([700, 5, 0, 1201], 2, 128, 128), ([33] * 40, 8, 64, 64), ([3000], 1, 64, 64), ([6000], 1, 128, 64),
                                             ([1300] * 9, 16, 128, 128)])
def test_long_and_many(new, heads, dk, dv, dtype):
    c = Case(new, heads, 1, dk, dv, dtype, seed=5, rate=0.01)
    out, m = c.run()
    c.check(out, m)
    assert m.status() == 0
    again, other = c.run()
    assert torch.equal(out, again) and torch.equal(m.states, other.states)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n", [5, 200, 1300])
def test_strong_decays_and_forgetting(n, dtype):
    c = Case([n], 2, 2, 64, 64, dtype, seed=6)
    c.g[::3] *= 400                                                       # some forget nearly all, next to some that forget little
    c.g[3] = -float("inf")
    if n > 100:
        c.g[70:75, 0] = -float("inf")
        c.g[64, 1] = -3e38
        c.g[128:140] = 0.0
    out, m = c.run()
    c.check(out, m)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n", [6, 200, 900])
def test_what_is_not_finite_reaches_only_what_sees_it(n, dtype):
    c = Case([n], 2, 2, 64, 64, dtype, seed=7)
    clean, _ = c.run()
    bad = n - 3
    c.v[bad, 0, 5], c.k[bad, 1, 3] = float("nan"), float("inf")
    out, m = c.run()
    tol = dict(rtol=2.0 ** -6 if dtype == BF else 2.0 ** -16, atol=1e-4)
    torch.testing.assert_close(out[:bad], clean[:bad], **tol)             # earlier tokens
    assert torch.isnan(out[bad:, 0, 5]).all() and not torch.isnan(out[:, 0, :5]).any()
    assert not torch.isfinite(out[bad, 1]).any() and not torch.isfinite(m.states[c.slot[0], 1, 3]).any()
    assert m.status() == 0
    # all that went wrong is forgotten at once
    c.g[bad + 1] = -float("inf")
    out, m = c.run()
    assert torch.isfinite(out[bad + 1:]).all() and torch.isfinite(m.states).all()
    k, v = c.k.double(), c.v.double()
    want = torch.einsum("hk,hk,hv->hv", c.q[bad + 1].double(), k[bad + 1], v[bad + 1]) * c.scale
    torch.testing.assert_close(out[bad + 1].double(), want, rtol=2.0 ** -6, atol=1e-3)


def test_states_that_are_not_finite_are_left_behind():
    c = Case([3, 70], 2, 1, 64, 64, BF, seed=8)
    c.states[:] = float("nan")
    c.fresh = torch.tensor([1, 1], device="cuda").int()
    out, m = c.run()
    free = torch.ones(len(c.states), dtype=torch.bool, device="cuda")
    free[c.slot.long()] = False
    assert torch.isfinite(out).all() and torch.isfinite(m.states[~free]).all() and torch.isnan(m.states[free]).all()
    c.states[:] = 0
    want, w = c.run()
    assert torch.equal(out, want) and torch.equal(m.states[~free], w.states[~free])


@pytest.mark.parametrize("n", [4, 100, 1000])
def test_bad_slots_and_offsets(n):
    from paper_2609_31938_b200 import TOKENS_BAD_LENGTH, TOKENS_BAD_SLOT
    c = Case([n, 2, n, 0], 2, 2, 64, 64, BF, seed=9)
    good = c.slot.clone()
    c.slot[2] = c.slot[0]                                                 # twice: the second starts from zeros and is lost
    c.slot[3] = c.slot[0]                                                 # (no tokens: no matter)
    c.slot[1] = 99
    out, m = c.run()
    assert m.status() == TOKENS_BAD_SLOT and m.status() == 0
    c.slot, c.fresh = good, torch.tensor([0, 1, 1, 0], device="cuda").int()
    want, w = c.run()
    assert torch.equal(out, want) and torch.equal(m.states[good[0]], w.states[good[0]])
    rest = [s for s in range(len(c.states)) if s != good[0].item()]
    assert torch.equal(m.states[rest], c.states[rest])
    c.starts[2] = 5 * n                                                   # past the rows
    before = c.states.clone()
    out, m = c.run()
    assert m.status() & TOKENS_BAD_LENGTH and torch.equal(c.states, before)
    c.starts[:] = torch.tensor([n, -4, 2 * n, 0, 2 * n], device="cuda")   # falling, and tokens named twice
    out, m = c.run()
    assert m.status() & TOKENS_BAD_LENGTH


@pytest.mark.parametrize("new", [[2, 3], [90, 40], [1400]])
def test_rows_behind_and_outputs_of_ones_own(new):
    c = Case(new, 2, 1, 64, 128, BF, seed=10, rows_behind=9)
    c.g = c.g[:1].expand(len(c.g), -1)                                    # one decay for each head
    out = torch.full((len(c.q), 2, 192), -5.0, device="cuda", dtype=BF)
    got, m = c.run(out=out[..., 32:160])
    c.check(got, m)
    assert bool((out[sum(new):] == -5).all()) and bool((out[..., :32] == -5).all()) and bool((out[..., 160:] == -5).all())


@pytest.mark.parametrize("dtype", [BF, F])
def test_a_stream_in_pieces_is_the_stream(dtype):
    from paper_2609_31938_b200 import tokens as tk
    c = Case([300], 2, 2, 128, 64, dtype, seed=11)
    whole, m = c.run()
    pieces, at = tk.DecayMemory(c.states.clone()), 0
    outs = []
    for n in (1, 64, 3, 100, 132):
        s = slice(at, at + n)
        outs.append(pieces.attend(c.q[s], c.k[s], c.v[s], c.g[s], tk.StreamBatch(torch.tensor([0, n], device="cuda").int(), c.slot, n)))
        at += n
    c.check(torch.cat(outs), pieces)
    c.check(whole, m)


def test_streams_and_graphs():
    from paper_2609_31938_b200 import tokens as tk
    for n in (2, 100, 1500):
        c = Case([n, n], 2, 2, 64, 64, BF, seed=12)
        want, m = c.run()
        still, batch = tk.DecayMemory(c.states.clone()), tk.StreamBatch(c.starts, c.slot, n)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            out = still.attend(c.q, c.k, c.v, c.g, batch)
        side.synchronize()
        assert torch.equal(out, want) and torch.equal(still.states, m.states)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = still.attend(c.q, c.k, c.v, c.g, batch)
        still.states.copy_(c.states)
        out.zero_()
        graph.replay()
        assert torch.equal(out, want) and torch.equal(still.states, m.states)
        graph.replay()                                                    # goes on from the states it left
        c.states = m.states.clone()
        want, m = c.run()
        assert torch.equal(out, want) and torch.equal(still.states, m.states)


def test_types_in_turn_and_two_memories():
    from paper_2609_31938_b200 import tokens as tk
    cases = [Case([700, 20], 2, 2, 64, 64, t, seed=13) for t in (BF, F, BF, F)]
    for c in cases:                                                       # (calls of one geometry and two types)
        c.check(*c.run())
    a, b = cases[0], cases[2]
    streams, memories, outs = [torch.cuda.Stream() for _ in range(2)], [], []
    for c, s in zip((a, b), streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            memories.append(tk.DecayMemory(c.states.clone()))
            outs.append(memories[-1].attend(c.q, c.k, c.v, c.g, tk.StreamBatch(c.starts, c.slot, 700)))
    torch.cuda.synchronize()
    for c, m, o in zip((a, b), memories, outs):
        c.check(o, m)


def test_nothing_to_do():
    from paper_2609_31938_b200 import tokens as tk
    c = Case([0, 0], 2, 2, 64, 64, BF)
    out, m = c.run()
    assert out.shape[0] == 0 and torch.equal(m.states, c.states)
    empty = torch.zeros(0, dtype=torch.int32, device="cuda")
    m.attend(c.q, c.k, c.v, c.g, tk.StreamBatch(torch.zeros(1, dtype=torch.int32, device="cuda"), empty, 0))
