"""F32 attention is as exact as 32-bit operations: its error, in norm and against 64 bits, is at most 2^-20 of the outputs or one and
a half times that of elementary FP32 operations on the same inputs, whichever is larger.

Derivation: queries and weights carry 22 bits (2^-22 each); what the outputs' sums lose is to stay under that of a sum rounded
at every step, for which some hundred tokens of like size give 2^-21 and thousands more than 2^-20."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def inputs(batch, new, old, h, g, dim, seed):
    from paper_2609_31938_b200 import tokens as tk
    gen = torch.Generator(device="cuda").manual_seed(seed)
    page, total = 64, old + new
    need = -(-total // page)
    codes = torch.empty(batch * need, 2, h, page, dim, dtype=torch.uint8, device="cuda")
    scales = torch.empty(batch * need, 2, h, device="cuda")
    for b in range(batch):
        at = slice(b * need, (b + 1) * need)
        x = torch.randn((need, 2, h, page, dim), generator=gen, device="cuda")
        m, e = torch.frexp(x.abs().amax((3, 4)))
        scales[at] = torch.ldexp(torch.ones_like(m), torch.where(m <= 0.875, e - 9, e - 8))
        codes[at] = (x / scales[at][..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.arange(batch * need, dtype=torch.int32, device="cuda").view(batch, need)
    call = tk.TokenBatch(ints([b * new for b in range(batch + 1)]), ints([total] * batch), table, new)
    return tk.PagedCache(codes, scales), call, torch.randn((batch * new, h * g, dim), generator=gen, device="cuda")


def plain(cache, q, b, new, old, g, causal, dtype):
    """Elementary operations in `dtype` for one sequence."""
    need = -(-(old + new) // 64)
    at = slice(b * need, (b + 1) * need)
    k, v = ((cache.codes[at, j].view(torch.float8_e4m3fn).to(dtype) * cache.scales[at, j].to(dtype)[..., None, None]).transpose(0, 1).flatten(1, 2)[:, :old + new]
            for j in range(2))                                                            # [heads, tokens, dim]
    h = k.shape[0]
    x = q[b * new:(b + 1) * new].to(dtype).view(new, h, g, -1).permute(1, 2, 0, 3).reshape(h, g * new, -1) @ k.transpose(1, 2) * k.shape[2] ** -0.5
    if causal:
        hidden = torch.arange(old + new, device="cuda") > old + torch.arange(new, device="cuda")[:, None]
        x.view(h, g, new, -1).masked_fill_(hidden, -torch.inf)
    p = (x - x.amax(-1, keepdim=True)).exp()
    return (p @ v / p.sum(-1, keepdim=True)).view(h, g, new, -1).permute(2, 0, 1, 3).reshape(new, h * g, -1)


CASES = [  # batch, new, old, kv heads, heads of each, head size, causal
    (64, 1, 31000, 1, 2, 128, True),              # step kernel, 8 rows: long shares
    (64, 1, 31000, 1, 4, 64, True),
    (16, 4, 31000, 4, 2, 128, True),
    (32, 2, 31000, 2, 8, 64, True),               # 16 rows
    (16, 4, 31000, 4, 8, 128, True),
    (2, 580, 46, 3, 8, 64, False),                # tile kernel: prompts that all see all
    (1, 340, 42, 2, 8, 128, False),
    (1, 500, 3580, 3, 4, 64, True),
    (1, 380, 12300, 2, 1, 128, True),
]


@pytest.mark.parametrize("batch,new,old,h,g,dim,causal", CASES)
def test_f32_attention_is_as_exact_as_fp32(batch, new, old, h, g, dim, causal):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    assert not torch.backends.cuda.matmul.allow_tf32
    cache, call, q = inputs(batch, new, old, h, g, dim, seed=batch + new)
    got = cache.attend(q, call, frame=1 if causal else 0)
    assert cache.status() == 0
    ours = theirs = size = 0.0
    for b in range(batch):
        want = plain(cache, q, b, new, old, g, causal, torch.float64)
        ours += (got[b * new:(b + 1) * new].double() - want).square().sum().item()
        theirs += (plain(cache, q, b, new, old, g, causal, torch.float32).double() - want).square().sum().item()
        size += want.square().sum().item()
    ours, theirs = (ours / size) ** 0.5, (theirs / size) ** 0.5
    assert ours <= max(2.0 ** -20, 1.5 * theirs), (ours, theirs)
