"""How the token operators are called: outputs among the slices of one projection, threads, streams, reports."""
import pytest

import _tokens_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("new", [[19, 2], [1]])
def test_append_among_slices_that_do_not_overlap(new):
    """Ranges of q_out, q, k and v lie in one another, elements do not: the same bits as with tensors of their own."""
    from paper_2609_31938_b200 import tokens as tk
    c = ref.Case(new, [5] * len(new), 4, 2, 64, 32, BF16, seed=4)
    rot = ref.tables(64, 32)
    rotary, pos = tk.Rotary(rot[0].cuda(), rot[1].cuda()), c.pos.int()[:, None].cuda()
    want, batch = c.on_gpu()
    q = want.append(c.k.cuda(), c.v.cuda(), batch, rotary, pos, q=c.q.cuda())
    wide = torch.zeros(c.tokens, 12, 64, dtype=BF16, device="cuda")                # q, q_out, k, v side by side
    apart = torch.zeros(c.tokens, 16, 64, dtype=BF16, device="cuda")               # on every other head, k and v between q's
    for q_in, q_out, k, v in ((wide[:, :4], wide[:, 4:8], wide[:, 8:10], wide[:, 10:]), (apart[:, 0:8:2],) * 2 + (apart[:, 1:5:2], apart[:, 5:9:2])):
        q_in.copy_(c.q.cuda()), k.copy_(c.k.cuda()), v.copy_(c.v.cuda())
        cache, batch = c.on_gpu()
        assert cache.append(k, v, batch, rotary, pos, q=q_in, q_out=q_out) is q_out
        assert torch.equal(q_out, q) and torch.equal(cache.scales, want.scales) and torch.equal(cache.codes, want.codes)
        assert torch.equal(k.cpu(), c.k) and torch.equal(v.cpu(), c.v)
