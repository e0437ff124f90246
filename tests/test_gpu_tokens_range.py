"""Attention where scores leave the range in which floats are closer than a unit.

With e = head_dim * 2^-24 * sum |q||k| the error of a score (a sum of exact products in FP32), a row whose best token leads by
more than 2 e + 100 has every other weight under e^-100 of it: its output is that token's value within the roundings of
weights (2^-11 BF16, 2^-20 F32) and output, its lse that token's score within e and FP32.  Of any other row no more is
known than that its output is an average of values it sees.
"""
import math

import pytest

import _tokens_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def scores_of(c, frame=1, window=-1):
    """Per row: scores [rows, heads, tokens] in 64 bits (-inf where unseen), the sums of magnitudes, and the values."""
    kv = ref.decode(c.codes, c.scales)
    H, P, D = kv.shape[2], kv.shape[3], kv.shape[4]
    G = c.q.shape[1] // H
    out = []
    for b, n in enumerate(c.new):
        total = int(c.total[b])
        pages = c.table[b, :-(-total // P)].long()
        k, v = (kv[pages, j].transpose(0, 1).reshape(H, -1, D)[:, :total].repeat_interleave(G, 0) for j in range(2))
        q = c.q[int(c.starts[b]):int(c.starts[b]) + n].double()
        x = torch.einsum("nhd,htd->nht", q, k) * D ** -0.5
        size = (torch.einsum("nhd,htd->nht", q.abs(), k.abs()) * D ** -0.5).amax(-1)
        for i in range(n):
            lo, hi = ref.visible(total - n + i, total, frame, window)
            x[i, :, :lo], x[i, :, hi:] = -math.inf, -math.inf
        out.append((x, size, v))
    return out


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new,dim", [(1, 128), (5, 64), (150, 128), (150, 64)])
@pytest.mark.parametrize("size", [3e6, 3e7, 1e8, 2e8, 1e10, 1e12, 1e20, 1e30])
def test_attend_far_scores(size, new, dim, dtype):
    c = ref.Case([new, 2], [200, 90], 4, 2, dim, 32, dtype, seed=41, stale=0x7F)
    c.q = (c.q.float() * size).to(dtype)
    cache, batch = c.on_gpu()
    got, lse = cache.attend(c.q.cuda(), batch, want_lse=True)
    assert cache.status() == 0
    got, lse = got.cpu().double(), lse.cpu().double()
    led = rows = 0
    for b, (x, mag, v) in enumerate(scores_of(c)):
        at = slice(int(c.starts[b]), int(c.starts[b + 1]))
        e = dim * U * mag
        top, best = x.max(-1)
        lead = top - x.scatter(-1, best[..., None], -math.inf).amax(-1) > 2 * e + 100
        want = torch.stack([v[h, best[:, h]] for h in range(4)], 1)
        tol = ((2.0 ** -8 if dtype == BF16 else U) + (2.0 ** -11 if dtype == BF16 else 2.0 ** -20)) * want.abs()
        assert ((got[at] - want).abs() <= tol)[lead].all()
        assert ((lse[at] - top).abs() <= e + 2.0 ** -20 * (1 + top.abs()))[lead].all()
        most = v.abs().amax((1, 2))[None, :, None] * (1 + 2.0 ** -7)
        assert torch.isfinite(got[at]).all() and (got[at].abs() <= most).all() and torch.isfinite(lse[at]).all()
        led, rows = led + int(lead.sum()), rows + lead.numel()
    assert led >= 0.8 * rows or size < 1e8               # (smaller scores lead by less)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 150])
def test_attend_far_scores_of_some_rows_and_of_later_tokens(new, dtype):
    """Rows with ordinary scores next to rows with far ones; scores that become far, and stop being so, along the cache."""
    c = ref.Case([new], [700], 4, 2, 128, 64, dtype, seed=43, stale=0x7F)
    c.q[:, ::2] *= 2.0 ** 20
    for j, power in ((3, 12), (4, 20), (5, -30), (8, 24)):
        c.scales[int(c.table[0, j]), 0, 0] *= 2.0 ** power
    cache, batch = c.on_gpu()
    got = cache.attend(c.q.cuda(), batch).cpu().double()
    assert cache.status() == 0
    (x, mag, v), = scores_of(c)
    p = torch.softmax(x, -1)
    want, mass = torch.einsum("nht,htd->nhd", p, v), torch.einsum("nht,htd->nhd", p, v.abs())
    far = 128 * U * mag > 1e-2                           # rows whose scores are uncertain: hold for those that lead
    top, best = x.max(-1)
    lead = top - x.scatter(-1, best[..., None], -math.inf).amax(-1) > 2 * 128 * U * mag + 100
    tol = (2.0 ** -8 if dtype == BF16 else U) * want.abs() + mass * (2.0 ** -11 if dtype == BF16 else 2.0 ** -20)
    assert lead[far].double().mean() >= 0.5
    assert ((got - want).abs() <= tol)[lead & far].all()
    tol = tol + mass * (2 * 128 * U * mag)[..., None]
    assert ((got - want).abs() <= tol)[~far].all()
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 150])
def test_attend_scores_past_the_largest_float(new, dtype):
    """A row one of whose scores passes the largest float is NaN, as infinity minus infinity is; below the smallest it weighs nothing."""
    c = ref.Case([new], [120], 2, 1, 64, 32, dtype, seed=44, stale=0x7F)
    c.q = (c.q.float() * (4e31 if new == 1 else 2.5e31)).to(dtype)
    c.scales[:, 0] *= 2.0 ** 20
    cache, batch = c.on_gpu()
    got, lse = cache.attend(c.q.cuda(), batch, want_lse=True)
    (x, _, _), = scores_of(c)
    largest = 3.402823466e38 * math.log(2.0)             # (scores are kept in units of log2)
    over, under = (x > 1.01 * largest).any(-1), (x < 0.99 * largest).all(-1)
    assert over.any() and under.any()
    assert torch.isnan(got.cpu()[over]).all() and torch.isnan(lse.cpu()[over]).all()
    assert torch.isfinite(got.cpu()[under]).all()
    assert cache.status() == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new,dim", [(1, 64), (5, 128), (70, 128), (150, 64)])
def test_attend_infinite_and_nan_queries(new, dim, dtype):
    """A query with an infinity has infinite scores (NaN where the key is zero).  A row whose scores are all -infinity weighs nothing:
    zeros, lse -infinity; one that has +infinity or NaN among them is NaN.  The rows beside it are right (with the bounds of
    ordinary scores: a product per channel, weights as halves)."""
    c = ref.Case([new], [150], 4, 2, dim, 32, dtype, seed=51, stale=0x7F)
    total = 150 + new
    clean = c.q.clone()
    for j in range(c.table.shape[1]):                    # keys: channel 3 negative, 5 positive, 7 zero before token 100, channel 9 mixed
        page = int(c.table[0, j])
        held = max(0, min(32, total - 32 * j))
        c.codes[page, 0, :, :held, 3] |= 0x80
        c.codes[page, 0, :, :held, 3] = c.codes[page, 0, :, :held, 3].clamp_min(0x90)
        c.codes[page, 0, :, :held, 5] = (c.codes[page, 0, :, :held, 5] & 0x7F).clamp_min(0x10)
        for t in range(held):
            if 32 * j + t < 100:
                c.codes[page, 0, :, t, 7] = 0
            else:
                c.codes[page, 0, :, t, 7] = 0xA0
    kinds = [(3, math.inf), (5, -math.inf), (3, -math.inf), (7, math.inf), (9, math.inf), (0, math.nan)]
    rows = {}
    for n, i in enumerate(range(0, new * 4, 3)):
        rows[i // 4, i % 4] = kinds[n % 6]
        c.q[i // 4, i % 4, kinds[n % 6][0]] = kinds[n % 6][1]
        c.q[i // 4, i % 4, 20] = 3e38 * (-1) ** n        # next to an infinity, the largest finite number is one of many
    for window in (-1, 40):
        cache, batch = c.on_gpu()
        got, lse = cache.attend(c.q.cuda(), batch, window=window, want_lse=True)
        assert cache.status() == 0
        (x, _, _), = scores_of(c, window=window)
        got, lse = got.cpu(), lse.cpu()
        for (i, h), _ in rows.items():
            lo, hi = ref.visible(total - new + i, total, 1, window)
            seen = x[i, h, lo:hi]
            if bool((seen == -math.inf).all()):
                assert (got[i, h] == 0).all() and lse[i, h] == -math.inf, (i, h, window)
            else:
                assert torch.isnan(got[i, h]).all() and torch.isnan(lse[i, h]), (i, h, window)
        same = torch.ones(new, 4, dtype=torch.bool)
        for i, h in rows:
            same[i, h] = False
        want, _, mass, spread = ref.attend(clean, c.codes, c.scales, c.starts, c.total, c.table, dim ** -0.5, 1, window)
        tol = (2.0 ** -8 if dtype == BF16 else U) * want.abs() + mass * (2.0 ** -11 if dtype == BF16 else 2.0 ** -20)
        assert ((got.double() - want).abs() <= tol + mass * (2 * dim * U * spread)[..., None])[same].all()


@pytest.mark.parametrize("dtype,new,dim,power", [
    (BF16, 1, 128, 22), (BF16, 5, 64, 22), (F32, 1, 64, 22), (F32, 5, 128, 22), (F32, 70, 128, 22), (F32, 70, 64, 10), (BF16, 70, 128, 16)])
def test_attend_queries_with_one_large_channel(dtype, new, dim, power):
    """One channel of the queries is 2^power times the others, and the keys are zero there: the scores are made of the others.
    Bounds as for ordinary scores (spread, the sum of |q||k|, does not see the large channel)."""
    c = ref.Case([new], [150], 4, 2, dim, 32, dtype, seed=61, stale=0x7F)
    c.q[:, :, 11] *= 2.0 ** power
    c.codes[:, 0, :, :, 11] = 0
    cache, batch = c.on_gpu()
    got, lse = cache.attend(c.q.cuda(), batch, want_lse=True)
    assert cache.status() == 0
    want, want_lse, mass, spread = ref.attend(c.q, c.codes, c.scales, c.starts, c.total, c.table, dim ** -0.5, 1, -1)
    e = dim * U * spread
    tol = (2.0 ** -8 if dtype == BF16 else U) * want.abs() + mass * ((2.0 ** -11 if dtype == BF16 else 2.0 ** -20) + 2 * e)[..., None]
    assert ((got.cpu().double() - want).abs() <= tol).all()
    assert ((lse.cpu().double() - want_lse).abs() <= e + 2.0 ** -20 * (1 + want_lse.abs())).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 5, 100])
@pytest.mark.parametrize("power", [10, 16, 20, 24])
def test_attend_page_whose_scale_is_far_above_the_others(power, new, dtype):
    """A page whose value scale is 2^power times the others' and whose own codes are small (a token that no row sees may have raised
    it).  Weights are halves (F32: two) of exp(score) times value scale.  With W the largest of those products of a row, each is
    within 2^-11 (2^-22) of itself and 2^-32 W: half of the halves' smallest step, 2^-25, where W is 2^7 at least.  So outputs are
    within that of mass, and within 2^-32 W sum |code| over the softmax's sum."""
    c = ref.Case([new], [200], 4, 2, 64, 32, dtype, seed=71, stale=0x7F)
    big = int(c.table[0, 2])
    c.scales[big, 1] *= 2.0 ** power
    c.codes[big, 1] = torch.where(c.codes[big, 1] % 2 == 0, 0, 1).to(torch.uint8)         # zeros and the smallest number
    c.codes[big, 1, :, :, :32] = 0
    cache, batch = c.on_gpu()
    got = cache.attend(c.q.cuda(), batch).cpu().double()
    assert cache.status() == 0
    want, _, mass, spread = ref.attend(c.q, c.codes, c.scales, c.starts, c.total, c.table, 64 ** -0.5, 1, -1)
    (x, _, _), = scores_of(c)
    p = torch.softmax(x, -1)
    pages = c.table[0].long()
    scale = c.scales[pages, 1].double().repeat_interleave(32, 0)[:200 + new].T.repeat_interleave(2, 0)           # [heads, tokens]
    codes = c.codes[pages, 1].view(torch.float8_e4m3fn).double().transpose(0, 1).flatten(1, 2)[:, :200 + new].abs()
    codes = torch.where(torch.isfinite(codes), codes, torch.zeros_like(codes)).sum(1).repeat_interleave(2, 0)    # [heads, dim]
    most = (p * scale).amax(-1)
    tol = (2.0 ** -8 if dtype == BF16 else U) * want.abs() + mass * ((2.0 ** -11 if dtype == BF16 else 2.0 ** -20) + 2 * 64 * U * spread)[..., None]
    assert ((got - want).abs() <= tol + 2.0 ** -32 * most[..., None] * codes).all()
