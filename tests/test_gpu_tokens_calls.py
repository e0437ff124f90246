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


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attend_prompt_beside_single_tokens_with_wide_tables(dtype):
    """One prompt of 8192 tokens beside 63 streams of one, tables for 131072 tokens: every stream, and rows all over the prompt."""
    n = [1] * 40 + [8192] + [1] * 23
    c = ref.Case(n, [(i * 37) % 150 for i in range(40)] + [0] + [5 * i for i in range(23)], 32, 8, 64, 64, dtype, seed=11, stale=0x7F)
    c.table = torch.nn.functional.pad(c.table, (0, 2048 - c.table.shape[1]), value=-1)
    cache, batch = c.on_gpu()
    got = cache.attend(c.q.cuda(), batch).cpu().double()
    assert cache.status() == 0
    kv = ref.decode(c.codes, c.scales)
    for b, new in enumerate(n):
        total, first = int(c.total[b]), int(c.starts[b])
        pages = c.table[b, :-(-total // 64)].long()
        k, v = (kv[pages, j].transpose(0, 1).reshape(8, -1, 64) for j in range(2))
        for i in [0] if new == 1 else [0, 1, 63, 64, 127, 128, 1000, 4097, 8190, 8191]:
            upto = total - new + i + 1
            q = c.q[first + i].double().view(8, 4, 64)
            x = torch.einsum("hgd,htd->hgt", q, k[:, :upto]) / 8
            p = torch.softmax(x, -1)
            want, mass = (torch.einsum("hgt,htd->hgd", p, u).reshape(32, 64) for u in (v[:, :upto], v[:, :upto].abs()))
            spread = (torch.einsum("hgd,htd->hgt", q.abs(), k[:, :upto].abs()) / 8).amax(-1).reshape(32, 1)
            u = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
            tol = u * want.abs() + mass * ((2.0 ** -11 if dtype == BF16 else 2.0 ** -20) + 2 * 64 * 2.0 ** -24 * spread)
            assert ((got[first + i] - want).abs() <= tol).all(), (b, i)


@pytest.mark.parametrize("new", [1, 60])
def test_offsets_that_fall_are_reported(new):
    import paper_2609_31938_b200 as ccv
    c = ref.Case([new] * 6, [100] * 6, 4, 2, 64, 16, BF16, seed=15)
    c.starts[2], c.starts[4] = 0, 0                      # rows named again and again
    cache, batch = c.on_gpu()
    cache.attend(c.q.cuda(), batch)
    cache.append(c.k.cuda(), c.v.cuda(), batch)
    assert cache.status() == ccv.TOKENS_BAD_LENGTH


def test_attend_from_threads_on_one_stream():
    """Eight threads on the default stream, each with queries of its own, all items split over blocks: the bits of calls in turn."""
    import threading
    c = ref.Case([1, 1], [3000, 2500], 8, 2, 64, 32, BF16, seed=19)
    cache, batch = c.on_gpu()
    g = torch.Generator(device="cuda").manual_seed(1)
    qs = [torch.randn(2, 8, 64, generator=g, device="cuda").to(BF16) for _ in range(8)]
    want = [cache.attend(q, batch) for q in qs]
    got = [[] for _ in qs]

    def work(i):
        for _ in range(50):
            got[i].append(cache.attend(qs[i], batch))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert all(len(a) == 50 and all(torch.equal(o, w) for o in a) for a, w in zip(got, want))
    assert cache.status() == 0


def test_status_covers_calls_on_other_streams():
    """A bad page reported behind half a second of other work on a side stream, asked for from the default stream."""
    import paper_2609_31938_b200 as ccv
    c = ref.Case([1], [100], 4, 2, 64, 16, BF16, seed=15)
    c.table[0, 2] = c.codes.shape[0] + 5
    cache, batch = c.on_gpu()
    q = c.q.cuda()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)
        cache.attend(q, batch)
    assert cache.status() == ccv.TOKENS_BAD_PAGE
    assert cache.status() == 0


def test_cache_object_made_inside_a_capture():
    """The handle of a cache whose memory is there may be made in a captured function; a replay starts with no reports."""
    import paper_2609_31938_b200 as ccv
    from paper_2609_31938_b200 import tokens as tk
    c = ref.Case([1], [100], 4, 2, 64, 16, BF16, seed=15)
    outside, batch = c.on_gpu()
    q = c.q.cuda()
    want = outside.attend(q, batch)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        inside = tk.PagedCache(outside.codes, outside.scales)
        out = inside.attend(q, batch)
    graph.replay()
    assert inside.status() == 0 and torch.equal(out, want)
    batch.page_table[0, 2] = c.codes.shape[0]
    graph.replay()
    assert inside.status() == ccv.TOKENS_BAD_PAGE
