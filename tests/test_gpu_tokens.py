"""The token operators (paged E4M3 cache: append and attend; gated norms) against plain 64-bit implementations.

Tolerances, derived before the first run (u = 2^-24, the half-step of FP32, 2^-8 that of BF16):

* append: rotated values carry three FP32 roundings, 3u of their terms' magnitudes; a code is then within half a step of
  E4M3 of that.  Scales are equal (the inputs' largest magnitudes are no nearer than 3u to a power-of-two border).
* attend: a score is a sum of head_dim exact products in FP32, off by at most head_dim * u * sum |q||k|, which is the
  relative error of its exponential; numerator and denominator both carry it.  Weights go into the product as halves
  (half-step 2^-12, 2^-11 allowed: two roundings) for BF16 and in two pieces (2^-20 allowed) for F32.  The bound scales
  with sum p |v|; the output's own rounding adds 2^-8 (BF16) or u of the output.
* gated norm: the row sums run over at most 32 terms in a thread and a tree, so norms are good to 2^-20; r is within
  2^-20 of its terms' magnitudes, h within 2^-18 of the row's largest.
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


# ------------------------------------------------------------------------------------------------ append
def check_append(c, cache, rot=None, positions=None, sections=None, interleaved=False):
    """The cache after an append of c.k, c.v against the definition on what the cache held before."""
    P = c.codes.shape[3]
    k, big = (ref.rotate(c.k, *rot, positions, sections, interleaved) if rot else (c.k.double(), c.k.double().abs()))
    v = c.v.double()
    want_codes, want_scales = c.codes.clone(), c.scales.clone()
    got_codes, got_scales = cache.codes.cpu(), cache.scales.cpu()
    got = ref.decode(got_codes, got_scales)
    touched = torch.zeros(c.codes.shape[0], P, dtype=torch.bool)
    for b, n in enumerate(c.new):
        total = int(c.total[b])
        n0 = max(0, n - total)                       # tokens without a place
        first, old, n = int(c.starts[b]) + n0, total - (n - n0), n - n0
        for j in range(old // P, -(-total // P) if n else 0):
            t0, t1 = max(0, old - j * P), min(P, total - j * P)
            page, rows = int(c.table[b, j]), slice(first + j * P + t0 - old, first + j * P + t1 - old)
            touched[page, t0:t1] = True
            for w, (x, m) in enumerate(((k, big), (v, v.abs()))):
                x, m = x[rows].transpose(0, 1), m[rows].transpose(0, 1)             # [heads, tokens, dim]
                most = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax((1, 2))
                e = torch.ceil(torch.log2(most / 448.0)).clamp_min(-64.0)
                scale = torch.exp2(e)
                if t0:
                    scale = torch.maximum(scale, c.scales[page, w].double())
                assert torch.equal(got_scales[page, w].double(), scale)
                s = scale[:, None, None]
                assert torch.equal(torch.isnan(got[page, w, :, t0:t1]), torch.isnan(x))
                cut = torch.nan_to_num((x / s).clamp(-448.0, 448.0))
                err = (torch.nan_to_num(got[page, w, :, t0:t1] / s) - cut).abs()
                assert (err <= 0.5 * ref.e4m3_step(cut) + torch.nan_to_num(3 * U * m / s, posinf=0.0)).all()
                was = ref.decode(c.codes, c.scales)[page, w, :, :t0]                # older tokens: moved exactly
                assert torch.equal(got[page, w, :, :t0] / s, ref.e4m3(was / s))
                want_scales[page, w] = scale.float()
    same = ~touched[:, None, None, :, None].expand_as(want_codes)
    moved = (got_scales != c.scales)[..., None, None].expand_as(want_codes)
    assert torch.equal(want_codes[same & ~moved], got_codes[same & ~moved])         # nothing else changed
    assert torch.equal(want_scales, got_scales)
    assert cache.status() == 0


APPENDS = [  # new, old, q_heads, kv_heads, dim, page, dtype, rotary pairs, axes, interleaved
    ([1], [0], 1, 1, 64, 16, BF16, 0, 1, False),
    ([1, 1, 1], [0, 15, 64], 4, 2, 128, 64, BF16, 64, 1, False),
    ([5, 0, 33, 16], [3, 7, 16, 31], 6, 3, 64, 16, BF16, 16, 1, True),
    ([200], [77], 8, 1, 128, 128, F32, 64, 3, False),
    ([129, 1, 64], [127, 128, 0], 5, 5, 128, 32, BF16, 60, 3, True),
    ([31, 17], [1, 0], 7, 1, 64, 128, F32, 32, 1, False),
    ([1, 2], [63, 63], 2, 2, 64, 64, F32, 4, 1, True),
]


@pytest.mark.parametrize("new,old,hq,h,d,page,dtype,pairs,axes,inter", APPENDS)
def test_append(new, old, hq, h, d, page, dtype, pairs, axes, inter):
    from paper_2609_31938_b200 import tokens as tk
    c = ref.Case(new, old, hq, h, d, page, dtype, seed=len(new) + d + page)
    cache, batch = c.on_gpu()
    rot = sections = positions = None
    rotary = None
    if pairs:
        rot = ref.tables(int(c.total.max()) + 1, pairs)
        sections = (pairs,) if axes == 1 else (pairs // 2 - 1, pairs // 4, pairs - pairs // 2 + 1 - pairs // 4)
        positions = c.pos.clamp_min(0)[:, None] if axes == 1 else torch.stack([c.pos // 7, c.pos % 7, c.pos % 5], 1)
        positions = positions.int()
        rotary = tk.Rotary(rot[0].cuda(), rot[1].cuda(), sections, interleaved=inter)
    q = cache.append(c.k.cuda(), c.v.cuda(), batch, rotary, None if positions is None else positions.cuda(), q=c.q.cuda())
    check_append(c, cache, rot, positions, sections, inter)
    want, big = ref.rotate(c.q, *rot, positions, sections, inter) if rot else (c.q.double(), c.q.double().abs())
    tol = 3 * U * big + (2.0 ** -8 if dtype == BF16 else U) * want.abs()
    assert ((q.cpu().double() - want).abs() <= tol).all()


def test_append_strided_slices_and_in_place_queries():
    """q, k and v as slices of one fused projection, q rotated in place; odd strides that keep 16 bytes."""
    from paper_2609_31938_b200 import tokens as tk
    for dtype in (BF16, F32):
        c = ref.Case([19, 2], [5, 40], 4, 2, 64, 32, dtype, seed=4)
        cache, batch = c.on_gpu()
        fused = torch.zeros(c.tokens, 9, 72, dtype=dtype, device="cuda")
        fused[:, :4, :64], fused[:, 4:6, :64], fused[:, 6:8, :64] = c.q.cuda(), c.k.cuda(), c.v.cuda()
        q, k, v = fused[:, :4, :64], fused[:, 4:6, :64], fused[:, 6:8, :64]
        rot = ref.tables(64, 32)
        pos = c.pos.int()[:, None]
        before = fused.clone()
        out = cache.append(k, v, batch, tk.Rotary(rot[0].cuda(), rot[1].cuda()), pos.cuda(), q=q, q_out=q)
        assert out is q
        check_append(c, cache, rot, pos, (32,), False)
        want, big = ref.rotate(c.q, *rot, pos, (32,), False)
        assert ((q.cpu().double() - want).abs() <= 3 * U * big + (2.0 ** -8 if dtype == BF16 else U) * want.abs()).all()
        q.copy_(c.q.cuda())
        assert torch.equal(fused, before)                # nothing outside q was touched


@pytest.mark.parametrize("page", [16, 64])
def test_append_token_by_token_equals_one_call(page):
    """Scales equal; codes equal but for those under the smallest normal number, which may have been rounded twice."""
    from paper_2609_31938_b200 import tokens as tk
    n = 70
    c = ref.Case([n], [0], 2, 2, 64, page, BF16, seed=9)
    c.v *= torch.exp2(torch.linspace(-9, 9, n)).view(n, 1, 1).bfloat16()     # scales that grow all the way
    whole, batch = c.on_gpu()
    whole.append(c.k.cuda(), c.v.cuda(), batch)
    steps = tk.PagedCache(torch.randint(0, 255, c.codes.shape, dtype=torch.uint8).cuda(), c.scales.cuda() * 1e6)
    for t in range(n):
        one = tk.TokenBatch(torch.tensor([0, 1], dtype=torch.int32).cuda(), torch.tensor([t + 1], dtype=torch.int32).cuda(),
                            c.table.cuda(), 1)
        steps.append(c.k[t:t + 1].cuda(), c.v[t:t + 1].cuda(), one)
    ids = c.table[0].long()
    assert torch.equal(whole.scales[ids.cuda()], steps.scales[ids.cuda()])
    a, b = (x.codes.cpu()[ids].view(torch.float8_e4m3fn).double().permute(0, 3, 1, 2, 4).flatten(0, 1)[:n] for x in (whole, steps))
    normal = a.abs() >= 2.0 ** -6
    assert torch.equal(a[normal], b[normal]) and ((a - b).abs() <= 2.0 ** -9).all()


def test_append_infinities_nan_zeros_and_extremes():
    c = ref.Case([8, 3, 2], [0, 9, 0], 1, 1, 64, 16, F32, seed=5)
    c.k[0, 0, 3], c.k[1, 0, 5], c.v[2, 0, 7] = math.inf, math.nan, -math.inf
    c.v[8:11] = 0.0                                      # zeros behind older tokens keep the old scale
    c.k[11:13] = 0.0                                     # a fresh page of zeros: the smallest scale
    c.v[11], c.v[12] = 3.0e38, 1.0e-38                   # the largest scale, and a value far under it
    cache, batch = c.on_gpu()
    cache.append(c.k.cuda(), c.v.cuda(), batch)
    check_append(c, cache)


def test_append_more_new_tokens_than_places_is_reported_and_cut():
    import paper_2609_31938_b200 as ccv
    c = ref.Case([6, 4], [0, 3], 1, 1, 64, 16, F32, seed=6, short=2)        # total 4 of 6 new tokens
    cache, batch = c.on_gpu()
    cache.append(c.k.cuda(), c.v.cuda(), batch)
    assert cache.status() == ccv.TOKENS_BAD_LENGTH and cache.status() == 0
    check_append(c, cache)


def test_append_bad_pages_and_positions_are_reported_and_skipped():
    from paper_2609_31938_b200 import tokens as tk
    import paper_2609_31938_b200 as ccv
    c = ref.Case([20, 5], [0, 0], 2, 2, 64, 16, BF16, seed=7)
    c.table[0, 1] = c.codes.shape[0]                     # one past the pool
    cache, batch = c.on_gpu()
    rot = ref.tables(4, 32)
    pos = torch.zeros(25, 1, dtype=torch.int32)
    pos[3], pos[4] = 4, -1
    cache.append(c.k.cuda(), c.v.cuda(), batch, tk.Rotary(rot[0].cuda(), rot[1].cuda()), pos.cuda())
    assert cache.status() == ccv.TOKENS_BAD_PAGE | ccv.TOKENS_BAD_POSITION
    first = c.codes.clone()
    held = c.table[[0, 1], [0, 0]].long()
    first[held] = cache.codes.cpu()[held]
    assert torch.equal(first, cache.codes.cpu())         # only the two good pages were written
    c = ref.Case([20, 5], [0, 0], 2, 2, 64, 16, BF16, seed=7)
    c.starts[1] = 40                                     # offsets past the rows, then falling
    cache, batch = c.on_gpu()
    cache.append(c.k.cuda(), c.v.cuda(), batch)
    assert cache.status() == ccv.TOKENS_BAD_LENGTH


# ------------------------------------------------------------------------------------------------ attend
def check_attend(c, cache, batch, frame=1, window=-1, scale=None, q=None, out=None):
    D = c.codes.shape[4]
    q = c.q.cuda() if q is None else q
    got, lse = cache.attend(q, batch, scale=scale, frame=frame, window=window, out=out, want_lse=True)
    scale = D ** -0.5 if scale is None else scale
    want, want_lse, mass, spread = ref.attend(c.q, cache.codes, cache.scales, c.starts, c.total, c.table, scale, frame, window)
    bf16 = c.q.dtype == BF16
    e_score = D * U * spread
    tol = (2.0 ** -8 if bf16 else U) * want.abs() + mass * ((2.0 ** -11 if bf16 else 2.0 ** -20) + 2 * e_score)[..., None]
    err = (got.cpu().double() - want).abs()
    assert (err <= tol).all(), f"worst {float((err / tol.clamp_min(1e-300)).max()):.3g} of the tolerance"
    empty = want_lse == -math.inf
    assert torch.equal(lse.cpu() == -math.inf, empty) and (got.cpu()[empty] == 0).all()
    err = (lse.cpu().double() - want_lse)[~empty].abs()
    assert (err <= (e_score + 2.0 ** -20 * (1 + want_lse.abs()))[~empty]).all()
    assert cache.status() == 0
    return got


ATTENDS = [  # new, old, q_heads, kv_heads, dim, page, dtype, frame, window
    ([1], [0], 1, 1, 64, 16, BF16, 1, -1),                               # one token that sees itself
    ([1, 1, 1, 1], [0, 15, 16, 300], 16, 2, 128, 16, BF16, 1, -1),
    ([1, 1], [700, 33], 7, 1, 64, 64, F32, 1, -1),                       # seven heads on one, 32 bits
    ([1, 1, 1], [127, 128, 129], 3, 3, 128, 128, BF16, 1, 100),
    ([2, 1, 0, 5], [40, 200, 9, 0], 8, 2, 64, 32, BF16, 1, -1),          # a sequence without new tokens
    ([4, 3], [250, 61], 24, 8, 128, 32, F32, 1, 17),
    ([17], [111], 40, 2, 64, 16, BF16, 1, -1),                           # rows of a tile that end inside a token
    ([100, 37, 1], [0, 300, 64], 4, 2, 128, 64, BF16, 1, -1),
    ([130], [200], 3, 1, 128, 128, BF16, 0, -1),                         # all see all
    ([96, 60], [96, 12], 2, 2, 64, 16, BF16, 24, -1),                    # whole frames
    ([90], [70], 2, 1, 128, 32, BF16, 20, 45),                           # frames that the chunk cuts, with a window
    ([75, 20], [33, 190], 5, 1, 64, 64, F32, 1, 40),
    ([140], [30], 2, 2, 128, 16, F32, 35, -1),
    ([64], [0], 2, 1, 64, 64, BF16, 0, 5),
    ([3, 40], [500, 0], 6, 2, 128, 16, BF16, 1, 0),                      # each token sees itself alone
]


@pytest.mark.parametrize("new,old,hq,h,d,page,dtype,frame,window", ATTENDS)
def test_attend(new, old, hq, h, d, page, dtype, frame, window):
    c = ref.Case(new, old, hq, h, d, page, dtype, seed=sum(new) + d, stale=0x7F)       # NaN in every slot nobody holds
    cache, batch = c.on_gpu()
    check_attend(c, cache, batch, frame, window)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 3, 150])
def test_attend_rows_without_any_token(new, dtype):
    """More new tokens than the cache holds: the first see nothing and get zeros and -infinity; so does an empty cache."""
    c = ref.Case([new, 1], [0, 5], 4, 2, 64, 16, dtype, seed=new, short=1 + new // 2, stale=0xFF)
    cache, batch = c.on_gpu()
    check_attend(c, cache, batch)
    c = ref.Case([new, 2], [0, 0], 4, 2, 128, 32, dtype, seed=new, short=new, stale=0xFF)
    cache, batch = c.on_gpu()
    check_attend(c, cache, batch, frame=0)


@pytest.mark.parametrize("new,frame", [(1, 1), (4, 1), (64, 16), (64, 1)])
def test_attend_nan_that_some_rows_do_not_see(new, frame):
    """A NaN value in the cache reaches the rows that see it, in its own channel, and no other row."""
    c = ref.Case([new], [100], 2, 1, 64, 16, BF16, seed=3)
    t, d = 100 + new - 1, 11                             # the last token's value, channel 11
    page = int(c.table[0, t // 16])
    c.codes[page, 1, 0, t % 16, d] = 0x7F
    cache, batch = c.on_gpu()
    got = cache.attend(c.q.cuda(), batch, frame=frame).cpu().float()
    want = ref.attend(c.q, c.codes, c.scales, c.starts, c.total, c.table, 64 ** -0.5, frame, -1)[0]
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.isnan(want).any()
    fine = ~torch.isnan(want)
    assert ((got.double() - want)[fine].abs() <= 2.0 ** -8 * (1 + want[fine].abs())).all()
    # a NaN key: every row that sees it, whole; no other
    c.codes[page, 1, 0, t % 16, d] = 0
    c.codes[page, 0, 0, t % 16, d] = 0xFF
    cache, batch = c.on_gpu()
    got = cache.attend(c.q.cuda(), batch, frame=frame).cpu().float()
    want = ref.attend(c.q, c.codes, c.scales, c.starts, c.total, c.table, 64 ** -0.5, frame, -1)[0]
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.isnan(want).any()


@pytest.mark.parametrize("new", [1, 130])
def test_attend_scores_and_scales_of_any_size(new):
    """Queries far outside the range of halves, page scales from tiny to huge, scores that differ by thousands."""
    for dtype, qs, ks, vs in ((BF16, 1e-30, 1e30, 2.0 ** -40), (BF16, 1e30, 1e-31, 2.0 ** 60), (F32, 300.0, 1.0, 1.0),
                              (F32, 1e-30, 2.0 ** 100, 1.0), (BF16, 100.0, 10.0, 2.0 ** -60)):
        c = ref.Case([new], [190], 4, 2, 64, 32, dtype, seed=12)
        c.q = (c.q.float() * qs).to(dtype)
        c.scales[:, 0] *= 2.0 ** round(math.log2(ks))
        c.scales[:, 1] *= vs
        c.scales[::3, 1] *= 2.0 ** -20                   # some pages' values are a million times smaller
        cache, batch = c.on_gpu()
        check_attend(c, cache, batch)


@pytest.mark.parametrize("new,old,hq,h", [(1, 9000, 8, 1), (2, 5000, 4, 4), (200, 3000, 2, 1)])
def test_attend_long_cache_split_over_blocks(new, old, hq, h):
    c = ref.Case([new, 1], [old, 3], hq, h, 128, 64, BF16, seed=8, stale=0x7F)
    cache, batch = c.on_gpu()
    a = check_attend(c, cache, batch)
    for _ in range(3):                                   # the same bits whichever block ends first
        assert torch.equal(a, cache.attend(c.q.cuda(), batch))


def test_attend_many_sequences_and_shared_pages():
    """More sequences than a warp scans at once, of unlike length; two of them read the same prefix pages."""
    new, old = [1 + i % 2 for i in range(70)], [(i * 37) % 150 for i in range(70)]
    old[5] = old[6] = 96
    c = ref.Case(new, old, 4, 2, 64, 32, BF16, seed=2, stale=0x7F)
    c.table[6, :3] = c.table[5, :3]
    cache, batch = c.on_gpu()
    check_attend(c, cache, batch)


def long_items(dtype, d, rising):
    """So many items that a block walks over more than 2000 tokens of one, also with scores that rise all along."""
    c = ref.Case([5] * 4, [5000, 4900, 5100, 5050], 14 * 16, 16, d, 64, dtype, seed=31, stale=0x7F)
    if rising:
        for b in range(4):
            for j in range(0, 75, 15):
                c.scales[c.table[b, j:].long().clamp_min(0).unique(), 0] *= 2
    return c


@pytest.mark.parametrize("dtype,d,rising", [(F32, 64, False), (BF16, 64, True)])
def test_attend_long_stretches_of_one_item(dtype, d, rising):
    c = long_items(dtype, d, rising)
    cache, batch = c.on_gpu()
    check_attend(c, cache, batch)


def test_attend_rising_scores_over_a_long_stretch():
    """Scores up to 500 000: where the one token that counts has a value of zero, an output is made of weights under e^-90
    of the largest (an exact output of 1.6e-51 is among them).  Weights are halves, 2^8 for the largest and 2^-24 their
    smallest step, so each may be off by 2^-33 of the largest besides what the other tests allow."""
    c = long_items(F32, 128, True)
    cache, batch = c.on_gpu()
    got = cache.attend(c.q.cuda(), batch).cpu().double()
    want, _, mass, spread = ref.attend(c.q, cache.codes, cache.scales, c.starts, c.total, c.table, 128 ** -0.5, 1, -1)
    kv = ref.decode(cache.codes, cache.scales)[:, 1]
    kv[~torch.isfinite(kv)] = 0.0                                                           # (slots nobody holds)
    magnitudes = torch.stack([kv[c.table[b, :-(-int(c.total[b]) // 64)].long()].abs().sum((0, 2)) for b in range(4)])
    floor = 2.0 ** -33 * magnitudes.repeat_interleave(5, 0).repeat_interleave(14, 1)        # of a token's every head
    tol = U * want.abs() + mass * (2.0 ** -20 + 2 * 128 * U * spread)[..., None] + floor
    assert ((got - want).abs() <= tol).all()
    assert cache.status() == 0


@pytest.mark.parametrize("new", [1, 40])
def test_pool_beyond_32_bit_offsets(new):
    """The same sequence at the two ends of a pool of 5.3 GB: the same bits, appended and read."""
    from paper_2609_31938_b200 import tokens as tk
    c = ref.Case([new], [300], 16, 8, 128, 64, BF16, seed=21)
    need = -(-(300 + new) // 64)
    pages = 40500
    codes = torch.zeros(pages, 2, 8, 64, 128, dtype=torch.uint8, device="cuda")
    assert codes.numel() > 1 << 32
    scales = torch.ones(pages, 2, 8, device="cuda")
    held = c.table[0, :need].long()
    outs = []
    for first in (0, pages - need):
        codes[first:first + need], scales[first:first + need] = c.codes[held].cuda(), c.scales[held].cuda()
        cache = tk.PagedCache(codes, scales)
        batch = tk.TokenBatch(c.starts.cuda(), c.total.cuda(), torch.arange(first, first + need, dtype=torch.int32).cuda()[None], new)
        cache.append(c.k.cuda(), c.v.cuda(), batch)
        outs.append((cache.attend(c.q.cuda(), batch), codes[first:first + need].clone(), scales[first:first + need].clone()))
        assert cache.status() == 0
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    small, batch = c.on_gpu()
    small.append(c.k.cuda(), c.v.cuda(), batch)
    assert torch.equal(small.codes.cpu()[held], outs[0][1].cpu()) and torch.equal(small.attend(c.q.cuda(), batch), outs[0][0])
    del codes, outs
    torch.cuda.empty_cache()


def test_attend_strides_and_given_output():
    c = ref.Case([9, 50], [20, 80], 6, 2, 64, 16, BF16, seed=14)
    cache, batch = c.on_gpu()
    wide = torch.zeros(c.tokens, 7, 88, dtype=BF16, device="cuda")
    wide[:, 1:, :64] = c.q.cuda()
    out = torch.full((c.tokens, 8, 80), 7.0, dtype=BF16, device="cuda")
    check_attend(c, cache, batch, q=wide[:, 1:, :64], out=out[:, 2:, 8:72])
    out[:, 2:, 8:72] = 7.0
    assert (out == 7.0).all()                            # nothing outside the view was written


def test_attend_bad_indices_are_reported_and_skipped():
    import paper_2609_31938_b200 as ccv
    for new in (1, 60):
        c = ref.Case([new, new], [100, 40], 4, 2, 64, 16, BF16, seed=15)
        c.table[0, 2] = c.codes.shape[0] + 5
        cache, batch = c.on_gpu()
        out = cache.attend(c.q.cuda(), batch)
        assert cache.status() == ccv.TOKENS_BAD_PAGE
        want = ref.attend(c.q, c.codes, c.scales, c.starts, c.total, c.table.clamp(-1, c.codes.shape[0] - 1), 0.125, 1, -1)[0]
        a, b = out.cpu().double()[new:], want[new:]      # the other sequence is whole
        assert ((a - b).abs() <= 2.0 ** -7 * (1 + b.abs())).all()
        c = ref.Case([new, new], [100, 40], 4, 2, 64, 16, BF16, seed=15)
        c.total[1] = 100000                              # more than the table's pages hold
        cache, batch = c.on_gpu()
        cache.attend(c.q.cuda(), batch)
        assert cache.status() & ccv.TOKENS_BAD_LENGTH


def test_side_stream_and_captured_graph():
    """The operators run on the current stream and inside a capture; a replay follows what the length arrays hold then."""
    from paper_2609_31938_b200 import tokens as tk
    c = ref.Case([1, 1], [60, 30], 4, 2, 64, 16, BF16, seed=16)
    cache, batch = c.on_gpu()
    q, k, v = c.q.cuda(), c.k.cuda(), c.v.cuda()
    x = torch.randn(2, 128, device="cuda", dtype=BF16)

    def step():
        cache.append(k, v, batch)
        return cache.attend(q, batch), tk.gated_norm(x, x * 2)[1]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, h = step()
    batch.total.copy_(torch.tensor([50, 20], dtype=torch.int32))            # the streams were cut back
    graph.replay()
    torch.cuda.synchronize()
    c.total = batch.total.cpu()
    c.codes, c.scales = cache.codes.cpu(), cache.scales.cpu()
    want, _, mass, spread = ref.attend(c.q, c.codes, c.scales, c.starts, c.total, c.table, 0.125, 1, -1)
    assert ((out.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + mass * (2.0 ** -11 + 128 * U * spread[..., None])).all()
    assert torch.equal(h, tk.gated_norm(x, x * 2)[1])


# ------------------------------------------------------------------------------------------------ gated norm
NORMS = [  # rows, channels, groups, res, act, weights, mod, post, pre, parts
    (1, 1, 1, BF16, BF16, F32, F32, "rms", "rms", "ywgs"),
    (3, 64, 3, F32, BF16, BF16, BF16, "rms", "layer", "ywbgs"),
    (130, 192, 2, BF16, BF16, F32, BF16, "layer", "rms", "ywg"),
    (7, 1000, 1, F32, F32, F32, F32, "none", "layer", "yws"),
    (33, 1153, 4, F32, F32, BF16, F32, "rms", "rms", "ywgs"),
    (5, 2050, 2, BF16, F32, F32, BF16, "rms", "layer", "yb"),
    (9, 4096, 3, BF16, BF16, BF16, BF16, "rms", "rms", "ywbgs"),
    (2, 8191, 1, F32, BF16, F32, F32, "layer", "layer", "ywbgs"),
    (3, 16384, 1, F32, F32, F32, F32, "rms", "layer", "ywgs"),
    (17, 384, 5, BF16, BF16, F32, F32, "rms", "rms", "w"),                # no block output: the residual's own norm
    (6, 512, 1, F32, BF16, F32, F32, "layer", "none", "yg"),
]


def norm_inputs(rows, ch, groups, res, act, wd, md, parts, seed=0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s, m=0.0, a=1.0: m + a * torch.randn(s, generator=g)  # noqa: E731
    x, y = rnd(rows, ch, m=0.3, a=3.0).to(res), (rnd(rows, ch, m=-0.2).to(act) if "y" in parts else None)
    w = [rnd(ch, m=1.0, a=0.2).to(wd) if "w" in parts else None for _ in range(2)]
    b = [rnd(ch, a=0.3).to(wd) if "b" in parts else None for _ in range(2)]
    mods = rnd(groups, 3, ch, a=0.5).to(md)
    gate = mods[:, 0] if "g" in parts else None
    scale, shift = (mods[:, 1], mods[:, 2]) if "s" in parts else (None, None)
    return x, y, gate, w[0], b[0], w[1], b[1], scale, shift


def check_norm(args, per, a, eps, post, pre, r, h):
    want_r, want_h, size = ref.gated_norm(args[0], args[1], per, *args[2:], a, eps, post, pre)
    half = lambda t: 2.0 ** -8 if t.dtype == BF16 else U  # noqa: E731
    if r is not None:
        assert ((r.cpu().double() - want_r).abs() <= half(r) * want_r.abs() + 2.0 ** -20 * size + 1e-37).all()
    if h is not None:
        big = want_h.abs().amax(-1, keepdim=True) + 1
        assert ((h.cpu().double() - want_h).abs() <= half(h) * want_h.abs() + 2.0 ** -18 * big).all()


@pytest.mark.parametrize("rows,ch,groups,res,act,wd,md,post,pre,parts", NORMS)
def test_gated_norm(rows, ch, groups, res, act, wd, md, post, pre, parts):
    from paper_2609_31938_b200 import tokens as tk
    args = norm_inputs(rows, ch, groups, res, act, wd, md, parts, seed=rows + ch)
    x, y, gate, pw, pb, qw, qb, scale, shift = (None if t is None else t.cuda() for t in args)
    per = -(-rows // groups)
    r, h = tk.gated_norm(x, y, gate=gate, post_weight=pw, post_bias=pb, pre_weight=qw, pre_bias=qb, scale=scale, shift=shift,
                         residual_scale=0.75, eps=1e-5, post_kind=post, pre_kind=pre, act_dtype=act)
    assert r.dtype == res and h.dtype == act
    check_norm(args, per, 0.75, 1e-5, post, pre, r, h)


MANY = [  # stretches of rows that cross the groups, channels that no access or team divides
    (3001, 64, 7, BF16, BF16, F32, BF16, "rms", "layer", "ywbgs"),
    (700, 192, 3, F32, BF16, BF16, F32, "layer", "rms", "ywbgs"),
    (901, 390, 1, F32, F32, F32, F32, "rms", "layer", "w"),
    (640, 1000, 64, BF16, F32, F32, F32, "rms", "layer", "ywgs"),
    (517, 1153, 5, F32, F32, F32, BF16, "layer", "rms", "ywgs"),
    (299, 1536, 2, F32, BF16, BF16, BF16, "rms", "layer", "ywbgs"),
    (333, 4096, 2, BF16, BF16, F32, F32, "rms", "none", "yws"),
    (305, 3001, 1, F32, BF16, F32, F32, "none", "rms", "yg"),
    (300, 6001, 2, F32, F32, F32, F32, "rms", "layer", "ywgs"),
]


@pytest.mark.parametrize("rows,ch,groups,res,act,wd,md,post,pre,parts", MANY)
def test_gated_norm_of_many_rows(rows, ch, groups, res, act, wd, md, post, pre, parts):
    """As above, with r's terms counted down to what the post norm adds up: with n = (y - mean) f, f = 1 / rms, a sum
    a x + gate (w n + b) is within 2^-20 of |a x| + |gate| (|w| (|y| + |mean|) f + |b|), which may be far over the sum itself."""
    from paper_2609_31938_b200 import tokens as tk
    args = norm_inputs(rows, ch, groups, res, act, wd, md, parts, seed=rows + ch)
    x, y, gate, pw, pb, qw, qb, scale, shift = (None if t is None else t.cuda() for t in args)
    per = -(-rows // groups)
    r, h = tk.gated_norm(x, y, gate=gate, post_weight=pw, post_bias=pb, pre_weight=qw, pre_bias=qb, scale=scale, shift=shift,
                         residual_scale=0.75, eps=1e-5, post_kind=post, pre_kind=pre, act_dtype=act)
    want_r, want_h, size = ref.gated_norm(args[0], args[1], per, *args[2:], 0.75, 1e-5, post, pre)
    if y is not None:
        z = args[1].double()
        mean = z.mean(-1, keepdim=True) if post == "layer" else torch.zeros(rows, 1, dtype=torch.float64)
        f = 1.0 if post == "none" else ((z - mean).square().mean(-1, keepdim=True) + 1e-5).rsqrt()
        z = (z.abs() + mean.abs()) * f
        z = z * args[3].double().abs() if args[3] is not None else z
        z = z + args[4].double().abs() if args[4] is not None else z
        z = z * args[2].double().abs()[torch.arange(rows) // per] if args[2] is not None else z
        size = (0.75 * args[0].double()).abs() + z
    half = lambda t: 2.0 ** -8 if t.dtype == BF16 else U  # noqa: E731
    assert ((r.cpu().double() - want_r).abs() <= half(r) * want_r.abs() + 2.0 ** -20 * size).all()
    big = want_h.abs().amax(-1, keepdim=True) + 1
    assert ((h.cpu().double() - want_h).abs() <= half(h) * want_h.abs() + 2.0 ** -18 * big).all()


def test_gated_norm_strides_in_place_and_single_outputs():
    from paper_2609_31938_b200 import tokens as tk
    for ch, wide in ((192, 200), (193, 201)):
        args = norm_inputs(21, ch, 3, BF16, BF16, F32, BF16, "ywgs", seed=ch)
        gx, gy = torch.zeros(21, wide, dtype=BF16, device="cuda"), torch.zeros(21, wide + 8, dtype=BF16, device="cuda")
        gx[:, :ch], gy[:, 4:4 + ch] = args[0].cuda(), args[1].cuda()
        x, y = gx[:, :ch], gy[:, 4:4 + ch]
        rest = [None if t is None else t.cuda() for t in args[2:]]
        kw = dict(zip(("gate", "post_weight", "post_bias", "pre_weight", "pre_bias", "scale", "shift"), rest))
        r0, h0 = tk.gated_norm(x, y, post_kind="rms", pre_kind="layer", **kw)
        check_norm(args, 7, 1.0, 1e-6, "rms", "layer", r0, h0)
        r1, none = tk.gated_norm(x, y, post_kind="rms", pre_kind="layer", want_h=False, **kw)
        assert none is None and torch.equal(r0, r1)
        none, h1 = tk.gated_norm(x, y, post_kind="rms", pre_kind="layer", want_r=False, **kw)
        assert none is None and torch.equal(h0, h1)
        r2, h2 = tk.gated_norm(x, y, post_kind="rms", pre_kind="layer", out_r=x, out_h=y, **kw)
        assert r2 is x and h2 is y and torch.equal(x, r0) and torch.equal(y, h0)
        x.zero_(), y.zero_()
        assert not gx.any() and not gy.any()             # nothing outside the rows was written


def test_gated_norm_empty_zero_and_non_finite_rows():
    from paper_2609_31938_b200 import tokens as tk
    r, h = tk.gated_norm(torch.zeros(0, 64, device="cuda"), torch.zeros(0, 64, device="cuda"))
    assert r.shape == h.shape == (0, 64)
    x = torch.randn(4, 96, device="cuda")
    y = torch.randn(4, 96, device="cuda")
    x[0], y[0] = 0.0, 0.0
    y[1, 5], x[2, 7] = math.nan, math.inf
    r, h = tk.gated_norm(x, y, post_kind="rms", pre_kind="rms")
    assert (r[0] == 0).all() and (h[0] == 0).all()
    assert torch.isnan(r[1]).all() and torch.isnan(h[1]).all()
    assert r[2, 7] == math.inf and torch.isfinite(r[2]).sum() == 95
    check_norm([t[3:].cpu() if t is not None else None for t in (x, y)] + [None] * 7, 1, 1.0, 1e-6, "rms", "rms", r[3:], h[3:])
