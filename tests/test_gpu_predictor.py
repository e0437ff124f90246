"""The latent predictor: the token operators run together over a stream of frames whose old pages are given back.

Held to a plain 64-bit run of the same network on the same rounded weights, cache quantisation included.  Two 64-bit-near
runs part where a key or value falls on the other side of an E4M3 rounding (a step of 2^-4 to 2^-3 of it), and every
BF16 tensor in between rounds by 2^-8; a frame passes about twenty of those.  Root mean square of the difference over that
of the frame: 20 roundings of 2^-9 (root mean square of a rounding is below half its bound) in quadrature are 0.9 %, and
the changed codes (a few in a thousand, averaged by the softmax) stay under that: 3 % is allowed.
"""
import pytest

import _tokens_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def plain_step(m, x, condition, seen):
    """One frame of LatentPredictor in 64 bits on the CPU; `seen`: quantised keys and values [frame][block] so far."""
    n, c, d = m.n, m.c, m.d
    f = len(seen)
    cpu = lambda t: t.double().cpu()  # noqa: E731
    mod = (cpu(condition) @ cpu(m.modulation)).view(len(m.blocks), 2, 3, 1, c)
    t = torch.arange(n)
    pos = torch.stack([torch.full_like(t, f), t // m.w, t % m.w], 1)
    sections = tuple(m.rotary.c.section)
    pre = lambda r, w, s, h: ref.norm(r, "rms", 1e-6) * cpu(w) * (1 + s) + h  # noqa: E731
    r = cpu(x.float())
    h = pre(r, m.blocks[0]["w"][0], mod[0, 0, 1], mod[0, 0, 2])
    seen.append([])
    for i, b in enumerate(m.blocks):
        qkv = (h @ cpu(b["qkv"])).view(n, -1, d)
        q, k, v = qkv[:, :m.hq], qkv[:, m.hq:m.hq + m.hk], qkv[:, m.hq + m.hk:]
        q = ref.rotate(q, m.rotary.cos, m.rotary.sin, pos, sections, False)[0]
        k = ref.rotate(k, m.rotary.cos, m.rotary.sin, pos, sections, False)[0]
        # pages begin at whole numbers of tokens from the stream's start here (n is a multiple of the page)
        quant = []
        for u in (k, v):
            p = u.view(n // m.page, m.page, m.hk, d)
            s = torch.exp2(torch.ceil(torch.log2(p.abs().amax((1, 3), keepdim=True) / 448.0)))
            quant.append((ref.e4m3(p / s) * s).view(n, m.hk, d))
        seen[-1].append(quant)
        lo = max(0, f - m.window)
        kk = torch.cat([seen[j][i][0] for j in range(lo, f + 1)]).repeat_interleave(m.hq // m.hk, 1)
        vv = torch.cat([seen[j][i][1] for j in range(lo, f + 1)]).repeat_interleave(m.hq // m.hk, 1)
        p = torch.softmax(torch.einsum("nhd,thd->hnt", q, kk) * d ** -0.5, -1)
        a = torch.einsum("hnt,thd->nhd", p, vv).reshape(n, -1)
        r = r + mod[i, 0, 0] * (ref.norm(a @ cpu(b["out"]), "rms", 1e-6) * cpu(b["w"][1]))
        h = pre(r, b["w"][2], mod[i, 1, 1], mod[i, 1, 2])
        y = torch.nn.functional.silu(h @ cpu(b["up"])) @ cpu(b["down"])
        r = r + mod[i, 1, 0] * (ref.norm(y, "rms", 1e-6) * cpu(b["w"][3]))
        if i + 1 < len(m.blocks):
            h = pre(r, m.blocks[i + 1]["w"][0], mod[i + 1, 0, 1], mod[i + 1, 0, 2])
    return r


def test_stream_of_frames_against_a_plain_run():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_31938_b200.predictor import LatentPredictor
    m = LatentPredictor(channels=96, heads=6, kv_heads=2, head_dim=64, blocks=2, height=8, width=16, window_frames=2, page_tokens=32)
    g = torch.Generator(device="cuda").manual_seed(5)
    seen = []
    for f in range(6):
        x, cond = torch.randn(m.n, 96, generator=g, device="cuda"), torch.randn(96, generator=g, device="cuda")
        want = plain_step(m, x, cond, seen)
        got = m.step(x, cond).double().cpu()
        rel = ((got - want).square().mean() / want.square().mean()).sqrt().item()
        assert rel <= 0.03, (f, rel)
        assert len(m.held) * m.page <= (m.window + 2) * m.n           # old frames' pages went back
    assert all(c.status() == 0 for c in m.caches)


def test_stream_restarts_and_frames_that_cut_pages():
    """The same frames after a reset give the same bits; frames that are no whole number of pages run as well."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_31938_b200.predictor import LatentPredictor
    m = LatentPredictor(channels=64, heads=4, kv_heads=1, head_dim=64, blocks=1, height=5, width=7, window_frames=3, page_tokens=64)
    g = torch.Generator(device="cuda").manual_seed(6)
    xs = [(torch.randn(35, 64, generator=g, device="cuda"), torch.randn(64, generator=g, device="cuda")) for _ in range(7)]
    first = [m.step(x, c).clone() for x, c in xs]
    m.reset()
    again = [m.step(x, c) for x, c in xs]
    assert all(torch.equal(a, b) for a, b in zip(first, again)) and all(torch.isfinite(a).all() for a in first)
    assert all(c.status() == 0 for c in m.caches)


def test_stream_past_the_end_of_the_rotation_tables():
    """A stream that begins some frames before its tables wrap predicts what one beginning at frame 0 does: attention only
    knows the distance of two frames."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_31938_b200.predictor import LatentPredictor
    m = LatentPredictor(channels=96, heads=6, kv_heads=2, head_dim=64, blocks=2, height=8, width=16, window_frames=2, page_tokens=32)
    m.frame = m.origin = m.rows - 3
    g = torch.Generator(device="cuda").manual_seed(5)
    seen = []
    for f in range(8):
        x, cond = torch.randn(m.n, 96, generator=g, device="cuda"), torch.randn(96, generator=g, device="cuda")
        want = plain_step(m, x, cond, seen)                # (counts its frames from 0)
        got = m.step(x, cond).double().cpu()
        rel = ((got - want).square().mean() / want.square().mean()).sqrt().item()
        assert rel <= 0.03, (f, rel)
    assert all(c.status() == 0 for c in m.caches)


def test_frame_axis_turns_whole_times_in_a_table():
    """Rows 1 .. rows - 1 and 0 again: the tables' period is their length, and no pair of the frame axis stands still."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_31938_b200.predictor import LatentPredictor
    m = LatentPredictor(channels=64, heads=2, kv_heads=1, head_dim=64, blocks=1, height=4, width=8, window_frames=70)
    n = m.rotary.c.section[0]
    assert m.rows > 2 * (m.window + 1)
    z = torch.complex(m.rotary.cos[:, :n].double(), m.rotary.sin[:, :n].double()).cpu()
    step = z[1:] / z[:-1]
    assert (step - step[0]).abs().max() <= 2e-6 and (z[0] / z[-1] - step[0]).abs().max() <= 2e-6
    assert ((step[0] - 1).abs() > 1e-3).all()


def test_reports_outlive_a_pool_that_grows(monkeypatch, capsys):
    """What a block's cache reported is told once, also after the pool grew, and main names the bits."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_31938_b200 as ccv
    from paper_2609_31938_b200 import predictor
    m = predictor.LatentPredictor(channels=64, heads=4, kv_heads=1, head_dim=64, blocks=2, height=5, width=7, window_frames=3, page_tokens=64)
    g = torch.Generator(device="cuda").manual_seed(6)
    m.caches[1]._status.fill_(ccv.TOKENS_BAD_POSITION)
    small = m.caches[1].pages
    for _ in range(12):
        m.step(torch.randn(35, 64, generator=g, device="cuda"), torch.randn(64, generator=g, device="cuda"))
    assert m.caches[1].pages > small
    assert m.status() == [0, ccv.TOKENS_BAD_POSITION]
    assert m.status() == [0, 0]

    class Reporting(predictor.LatentPredictor):
        def step(self, x, condition):
            self.caches[0]._status.fill_(ccv.TOKENS_BAD_PAGE)
            return super().step(x, condition)

    monkeypatch.setattr(predictor, "LatentPredictor", Reporting)
    with pytest.raises(SystemExit) as e:
        predictor.main(1)
    assert "0x1" in str(e.value)
