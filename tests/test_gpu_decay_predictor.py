"""The products, decaying states and group norms together: a predictor of fixed memory and a decoder chain with normed blocks."""
import pytest
import torch

import _operators_ref as ref
from _tokens_ref import norm

pytestmark = pytest.mark.gpu


def plain_step(m, x, condition, states):
    """DecayPredictor.step in 64 bits."""
    d = lambda t: t.double()  # noqa: E731
    n, c, hk, hv = m.n, m.c, m.heads * m.dk, m.heads * m.dv
    mod = (d(condition) @ d(m.modulation)).view(len(m.blocks), 2, 2, 1, c)
    r = d(x)
    starts = torch.tensor([0, n])
    for i, b in enumerate(m.blocks):
        h = norm(r, "rms", 1e-6) * d(b["w"][0]) * (1 + mod[i, 0, 0]) + mod[i, 0, 1]
        qkv = h @ d(b["qkv"]).T
        g = -torch.nn.functional.softplus(h @ d(b["decay"]).T + d(b["rate"]))
        q, k, v = qkv[:, :hk].view(n, m.heads, m.dk), qkv[:, hk:2 * hk].view(n, m.heads, m.dk), qkv[:, 2 * hk:].view(n, m.heads, m.dv)
        o, states[i], _, _ = ref.decay(q, k, v, g, starts, [0], None, states[i], m.dk ** -0.5)
        o, _ = ref.group_norm(o.view(n, 1, hv), m.heads, *b["head"], None, None, 1e-6, "none")
        r = r + o.view(n, hv) @ d(b["out"]).T
        h = norm(r, "rms", 1e-6) * d(b["w"][1]) * (1 + mod[i, 1, 0]) + mod[i, 1, 1]
        z = h @ d(b["up"]).T
        r = r + (ref.activate(z[:, :4 * c], "silu") * z[:, 4 * c:]) @ d(b["down"]).T
    return r


# F32: the norms divide by deviations of about 0.1 in places, so that a step's own errors (2^-20) grow some fivefold from block to block: 2^-12 is
# ten times that of four norms.  BF16: a rounding of 2^-9 at each of the eight operators of a block instead, in the mean over the outputs.
@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2.0 ** -12), (torch.bfloat16, 2.0 ** -4)])
def test_predictor_against_64_bits(dtype, tol):
    from paper_2609_31938_b200.predictor import DecayPredictor
    m = DecayPredictor(channels=64, heads=2, key_dim=64, value_dim=128, blocks=2, height=9, width=17, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(5)
    states = [torch.zeros(1, m.heads, m.dk, m.dv, dtype=torch.float64, device="cuda") for _ in m.blocks]
    firsts = []
    for f in range(3):
        x, condition = torch.randn(m.n, 64, generator=g, device="cuda"), torch.randn(64, generator=g, device="cuda")
        y, want = m.step(x, condition), plain_step(m, x, condition, states)
        assert ((y.double() - want).norm() / want.norm()).item() < tol
        firsts.append((x, condition, y))
    assert not any(m.status())
    m.reset()
    x, condition, y = firsts[0]
    assert torch.equal(m.step(x, condition), y)


def layers(seed=1):
    from paper_2609_31938_b200.chain import LAYERS
    g = torch.Generator(device="cuda").manual_seed(seed)
    ca, cb, cc = 64, 32, 32
    shapes = {"A1": (ca, ca, 3), "A2": (ca, ca, 3), "PA": (cb, ca, 1), "B1": (cb, cb, 3), "B2": (cb, cb, 3), "PB": (cc, cb, 1), "C1": (cc, cc, 3), "C2": (cc, cc, 3)}
    w = {k: (torch.randn((co, ci, n, n, n), generator=g, device="cuda") * (ci * n ** 3) ** -0.5).bfloat16() for k, (co, ci, n) in shapes.items()}
    b = {k: (0.1 * torch.randn(w[k].shape[0], generator=g, device="cuda")).bfloat16() for k in LAYERS}
    norms = {k: (1 + 0.2 * torch.randn(s[1], generator=g, device="cuda"), 0.2 * torch.randn(s[1], generator=g, device="cuda")) for k, s in shapes.items() if k[0] != "P"}
    return w, b, norms


def test_normed_chain_streams_and_matches_its_plain_form():
    from paper_2609_31938_b200.chain import NormedDecoderChain
    w, b, norms = layers()
    x = torch.randn(1, 64, 4, 16, 24, device="cuda").bfloat16()
    chain = NormedDecoderChain(w, b, norms, groups=8)
    whole = chain.step(x)
    chain.reset()
    assert torch.equal(torch.cat([chain.step(x[:, :, t:t + 1].contiguous()) for t in range(4)], 2), whole)

    def conv(name, t):                                           # cached causal convolution of the whole stream, zero history
        k = w[name].shape[2]
        t = torch.nn.functional.pad(t, (k // 2,) * 4 + (k - 1, 0))
        return torch.nn.functional.conv3d(t.double(), w[name].double(), b[name].double()).bfloat16()

    def normed(name, t):
        n, c, f, h, wd = t.shape
        rows = t.permute(0, 2, 3, 4, 1).reshape(n * f, h * wd, c)
        y = ref.group_norm(rows, 8, *norms[name], None, None, 1e-6, "silu")[0].bfloat16()
        return y.view(n, f, h, wd, c).permute(0, 4, 1, 2, 3)

    def block(one, two, t):
        return (t.double() + conv(two, normed(two, conv(one, normed(one, t)))).double()).bfloat16()

    up = lambda t, rt: t.repeat_interleave(rt, 2).repeat_interleave(2, 3).repeat_interleave(2, 4)  # noqa: E731
    a = block("A1", "A2", x)
    c = block("B1", "B2", up(conv("PA", a), 4))
    want = block("C1", "C2", up(conv("PB", c), 1))
    # twelve roundings to BF16 (2^-9 each in the mean) on the longest way
    assert ((whole.double() - want.double()).norm() / want.double().norm()).item() < 12 * 2.0 ** -9
    chain.close()


def test_command_runs():
    from paper_2609_31938_b200 import predictor
    predictor.main(2, "decay")
