"""Plain 64-bit implementations of the token operators (torch, CPU) and the inputs of their tests."""
import math

import torch


def decode(codes, scales):
    """E4M3 codes [pages, 2, heads, tokens, dim] and scales to the values they stand for."""
    return codes.cpu().view(torch.float8_e4m3fn).double() * scales.cpu().double()[..., None, None]


def e4m3(x):
    """Nearest E4M3 value (ties to even), cut to +-448; NaN stays."""
    x = x.clamp(-448.0, 448.0)
    e = torch.frexp(x)[1]
    step = torch.ldexp(torch.ones_like(x), (e - 1).clamp_min(-6) - 3)
    return torch.round(x / step) * step


def e4m3_step(x):
    """Distance between neighbouring E4M3 values at x."""
    e = torch.frexp(x.abs().clamp(2.0 ** -9, 448.0))[1]
    return torch.ldexp(torch.ones_like(x), (e - 1).clamp_min(-6) - 3)


def visible(pos, total, frame, window):
    start = pos // frame * frame if frame > 0 else pos
    hi = min(total, start + frame) if frame > 0 else total
    lo = 0 if window < 0 else max(0, start - window)
    return (0, 0) if pos < 0 else (lo, max(lo, hi))


def rotate(x, cos, sin, positions, sections, interleaved):
    """x [tokens, heads, dim] in 64 bits; also the sum of the magnitudes that each output is made of."""
    x = x.double().cpu().clone()
    big = x.abs()
    pairs = cos.shape[1]
    axis = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)])
    rows = positions.cpu().long()[:, axis]
    c = cos.cpu().double()[rows, torch.arange(pairs)][:, None]
    s = sin.cpu().double()[rows, torch.arange(pairs)][:, None]
    i = torch.arange(pairs)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
    xa, xb = x[..., a].clone(), x[..., b].clone()
    x[..., a], x[..., b] = xa * c - xb * s, xb * c + xa * s
    big[..., a], big[..., b] = (xa * c).abs() + (xb * s).abs(), (xb * c).abs() + (xa * s).abs()
    return x, big


def attend(q, codes, scales, new_start, total, table, scale, frame, window):
    """out, lse, and for the tolerances: sum p |v| for each output and the largest scale * sum |q| |k| of each row."""
    kv = decode(codes, scales)
    H, P, D = kv.shape[2], kv.shape[3], kv.shape[4]
    T, Hq = q.shape[0], q.shape[1]
    q = q.cpu().double()
    out, mass = torch.zeros(T, Hq, D, dtype=torch.float64), torch.zeros(T, Hq, D, dtype=torch.float64)
    lse, spread = torch.full((T, Hq), -math.inf, dtype=torch.float64), torch.zeros(T, Hq, dtype=torch.float64)
    new_start, total, table = new_start.tolist(), total.tolist(), table.cpu()
    for b in range(len(total)):
        n = new_start[b + 1] - new_start[b]
        pages = table[b, :-(-total[b] // P)].long()
        k = kv[pages, 0].transpose(0, 1).reshape(H, -1, D)
        v = kv[pages, 1].transpose(0, 1).reshape(H, -1, D)
        for i in range(n):
            lo, hi = visible(total[b] - n + i, total[b], frame, window)
            if hi <= lo:
                continue
            t = new_start[b] + i
            for h in range(Hq):
                g = h // (Hq // H)
                kk, vv = k[g, lo:hi], v[g, lo:hi]
                x = kk @ q[t, h] * scale
                p = torch.softmax(x, 0)
                out[t, h], mass[t, h], lse[t, h] = p @ vv, p @ vv.abs(), torch.logsumexp(x, 0)
                spread[t, h] = (kk.abs() @ q[t, h].abs()).max() * abs(scale)
    return out, lse, mass, spread


def norm(x, kind, eps):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    return x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)


def gated_norm(x, y, per, gate, pw, pb, qw, qb, scale, shift, a, eps, post, pre):
    """(r, h, size of r's terms) in 64 bits."""
    d = lambda t: None if t is None else t.cpu().double()  # noqa: E731
    x, y, gate, pw, pb, qw, qb, scale, shift = map(d, (x, y, gate, pw, pb, qw, qb, scale, shift))
    g = torch.arange(x.shape[0]) // per
    r, size = a * x, (a * x).abs()
    if y is not None:
        z = norm(y, post, eps)
        z = z * pw if pw is not None else z
        z = z + pb if pb is not None else z
        z = z * gate[g] if gate is not None else z
        r, size = r + z, size + z.abs()
    h = norm(r, pre, eps)
    h = h * qw if qw is not None else h
    h = h + qb if qb is not None else h
    h = h * (1 + scale[g]) if scale is not None else h
    h = h + shift[g] if shift is not None else h
    return r, h, size


class Case:
    """A batch on a pool of scattered pages, with the cache filled with ordinary keys and values."""

    def __init__(self, new, old, q_heads, kv_heads, dim, page, dtype, seed=0, short=0, stale=None):
        """short: how many of the first sequence's new tokens have no place in the cache (total < new)."""
        g = torch.Generator().manual_seed(seed)
        self.new, self.old = list(new), list(old)
        total = [n + o for n, o in zip(new, old)]
        total[0] -= short
        need = [-(-t // page) for t in total]
        pages = sum(need) + 2
        order = torch.randperm(pages, generator=g)
        width = max(1, max(need))
        self.table = torch.full((len(new), width), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n].int()
            at += n
        self.starts = torch.tensor([0] + list(new)).cumsum(0).int()
        self.total = torch.tensor(total, dtype=torch.int32)
        self.tokens, self.max_new = sum(new), max(new)
        x = torch.randn((pages, 2, kv_heads, page, dim), generator=g) * (1 + 3 * torch.rand((pages, 2, kv_heads, 1, 1), generator=g))
        m, e = torch.frexp(x.abs().amax((3, 4)))
        self.scales = torch.ldexp(torch.ones_like(m), torch.where(m <= 0.875, e - 9, e - 8))
        self.codes = (x / self.scales[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        if stale is not None:                    # what no sequence holds
            held = torch.zeros(pages, page, dtype=torch.bool)
            for b, t in enumerate(total):
                for j in range(need[b]):
                    held[self.table[b, j], :max(0, min(page, t - j * page))] = True
            self.codes.permute(0, 3, 1, 2, 4)[~held] = stale
        self.q = torch.randn((self.tokens, q_heads, dim), generator=g).to(dtype)
        self.k = torch.randn((self.tokens, kv_heads, dim), generator=g).to(dtype)
        self.v = (2 * torch.randn((self.tokens, kv_heads, dim), generator=g)).to(dtype)
        self.pos = torch.cat([torch.arange(t - n, t) for n, t in zip(new, total)])

    def on_gpu(self):
        from paper_2609_31938_b200 import tokens as tk
        cache = tk.PagedCache(self.codes.cuda(), self.scales.cuda())
        batch = tk.TokenBatch(self.starts.cuda(), self.total.cuda(), self.table.cuda(), self.max_new)
        return cache, batch


def tables(rows, pairs):
    a = torch.arange(rows, dtype=torch.float64)[:, None] * 1000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)
    return a.cos().float(), a.sin().float()
