"""Cases of the token operators: the paged 8-bit cache of keys and values (append, attend) and the gated norms.

They are what a streaming world model runs in front of a causal video decoder: a transformer predicts the next latent
frame token by token or frame by frame, its keys and values stay in a paged cache held in E4M3 with one power-of-two
scale for each page and head, and every block's output passes through a norm, a gate and the residual sum into the
next block's norm.  Latent frames are the decoder chain's, 44 x 80 pixels (3520 tokens, or 880 in patches of 2 x 2).

`run` with `own` false computes the operators in their plain form: elementary torch operations in 32 bits, rounded once.
"""
import math
import random

import torch

own = False

DEV = "cuda"
E4M3_MAX = 448.0
MIN_EXP = -64            # smallest exponent of a page's scale
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one new token for each of 64 streams of unlike age: q, k and v are slices of one fused projection
        dict(name="append-step-b64", op="append", dtype="bf16", batch=64, new_lo=1, new_hi=1, old_lo=0, old_hi=1500,
             q_heads=32, kv_heads=8, dim=128, page=64, rot=128, axes=1, interleaved=False),
        # one latent frame of 44 x 80 tokens behind another, rotated by (frame, row, column); a page is half full
        dict(name="append-latent-frame", op="append", dtype="bf16", batch=1, new_lo=3520, new_hi=3520, old_lo=3520,
             old_hi=3520, q_heads=12, kv_heads=12, dim=128, page=128, rot=128, axes=3, interleaved=True),
        # prompts of unlike length in 32 bits, half of each head rotated, small pages
        dict(name="append-ragged-f32", op="append", dtype="f32", batch=24, new_lo=1, new_hi=2500, old_lo=0, old_hi=700,
             q_heads=14, kv_heads=2, dim=64, page=16, rot=32, axes=1, interleaved=False),
        # the smallest call: three young streams, latency is all there is
        dict(name="attend-step-small", op="attend", dtype="bf16", batch=3, new_lo=1, new_hi=1, old_lo=0, old_hi=300,
             q_heads=16, kv_heads=16, dim=64, page=16, frame=1, window=-1),
        # one token for each of 64 streams of unlike length: bound by the cache's bytes
        dict(name="attend-step-b64", op="attend", dtype="bf16", batch=64, new_lo=1, new_hi=1, old_lo=500, old_hi=8000,
             q_heads=32, kv_heads=8, dim=128, page=64, frame=1, window=-1),
        # one token of one stream behind a long cache: few rows, split over the cache
        dict(name="attend-step-long", op="attend", dtype="bf16", batch=1, new_lo=1, new_hi=1, old_lo=131070,
             old_hi=131070, q_heads=56, kv_heads=8, dim=128, page=64, frame=1, window=-1),
        # a few drafted tokens for each stream, in 32 bits
        dict(name="attend-draft-f32", op="attend", dtype="f32", batch=6, new_lo=1, new_hi=5, old_lo=100, old_hi=6000,
             q_heads=8, kv_heads=2, dim=64, page=32, frame=1, window=-1),
        # the largest: a latent frame of 44 x 80 tokens that sees itself and the seven frames before it
        dict(name="attend-latent-frame", op="attend", dtype="bf16", batch=1, new_lo=3520, new_hi=3520, old_lo=28160,
             old_hi=28160, q_heads=12, kv_heads=12, dim=128, page=128, frame=3520, window=24640),
        # prompts of unlike length, some behind a cached prefix, causal with a window
        dict(name="attend-ragged-causal", op="attend", dtype="bf16", batch=8, new_lo=3, new_hi=2047, old_lo=0, old_hi=1900,
             q_heads=28, kv_heads=4, dim=128, page=64, frame=1, window=1023),
        # one token for each of 64 streams between two blocks
        dict(name="norm-step-b64", op="norm", res="bf16", act="bf16", mod="bf16", rows=64, groups=1, channels=4096,
             kind="rms", scale=1.0, gate=False, shift=False),
        # eight latent frames of 44 x 80 tokens, residual in 32 bits, gate, scale and shift for each frame
        dict(name="norm-latent-frames", op="norm", res="f32", act="bf16", mod="f32", rows=28160, groups=8, channels=1536,
             kind="layer", scale=1.0, gate=True, shift=True),
        # odd rows of an odd number of channels in 32 bits, residual scaled down
        dict(name="norm-odd-f32", op="norm", res="f32", act="f32", mod="f32", rows=5001, groups=3, channels=1153,
             kind="rms", scale=0.7071, gate=True, shift=False),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    v = min(hi, max(lo, v))
    return v + 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(["append", "attend-step", "attend", "attend", "norm"])
    if op == "norm":
        rows = _log(rng, 1, 30000)
        channels = _log(rng, 64, min(8192, max(64, 43_000_000 // rows)))
        channels = channels if rng.random() < 0.3 else max(64, channels // 64 * 64)
        channels += 64 if channels == 3072 else 0
        res, act = rng.choice([("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
        return dict(op="norm", res=res, act=act, mod=rng.choice(["bf16", "f32"]), rows=rows, groups=rng.randint(1, min(8, rows)),
                    channels=channels, kind=rng.choice(["rms", "layer"]), scale=rng.choice([1.0, 0.5]),
                    gate=rng.random() < 0.6, shift=rng.random() < 0.6)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    dim = rng.choice([64, 128])
    page = rng.choice([16, 32, 64, 128])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    group = rng.choice([1, 2, 3, 4, 7, 8])
    if op == "append":
        batch = _log(rng, 1, 64)
        new_hi = _log(rng, 1, max(1, 40000 // batch // (kv_heads * group * dim // 128 or 1)))
        old_hi = _log(rng, 1, 1500)
        return dict(op="append", dtype=dtype, batch=batch, new_lo=rng.randint(1, new_hi), new_hi=new_hi,
                    old_lo=rng.randint(0, old_hi), old_hi=old_hi, q_heads=kv_heads * group, kv_heads=kv_heads, dim=dim,
                    page=page, rot=rng.choice([dim // 2, dim]), axes=rng.choice([1, 3]), interleaved=rng.random() < 0.5)
    if op == "attend-step":
        batch = _log(rng, 1, 64)
        new_hi = rng.choice([1, 1, 1, 2, 4])
        old_hi = _log(rng, 1, max(1, 250_000 * 8 // (batch * kv_heads)))
        old_hi = min(old_hi, 131000)
    else:
        batch = _log(rng, 1, 8)
        new_hi = _log(rng, 8, 3000)
        old_hi = _log(rng, 1, 28000 // batch)
    old_lo = rng.randint(0, old_hi)
    # the plain form holds all scores of a padded batch in 32 bits: keep them under some 4 GB
    while batch * kv_heads * group * new_hi * (old_hi + new_hi) > 1_000_000_000:
        batch, new_hi, old_hi = max(1, batch // 2), max(1, new_hi * 3 // 4), max(1, old_hi * 3 // 4)
        old_lo = min(old_lo, old_hi)
    frame = rng.choice([0, 1, 1, 880])
    return dict(op="attend", dtype=dtype, batch=batch, new_lo=rng.randint(1, new_hi), new_hi=new_hi, old_lo=old_lo,
                old_hi=old_hi, q_heads=kv_heads * group, kv_heads=kv_heads, dim=dim, page=page, frame=frame,
                window=rng.choice([-1, -1, _log(rng, 16, 4000)]))


def _lengths(case):
    """(new tokens, cached tokens before them) of each sequence: spread over the case's ranges, the same for every seed."""
    rng = random.Random(case["batch"] * 1000003 + case["new_hi"] * 1009 + case["old_hi"])
    new, old = [], []
    for i in range(case["batch"]):
        new.append(rng.randint(case["new_lo"], case["new_hi"]))
        old.append(rng.randint(case["old_lo"], case["old_hi"]))
    new[rng.randrange(case["batch"])] = case["new_hi"]
    return new, old


def _visible(case, p, total):
    """Range of cached tokens that the token at position p sees."""
    f, w = case["frame"], case["window"]
    start = p // f * f if f > 0 else p
    return (0 if w < 0 else max(0, start - w)), (min(total, start + f) if f > 0 else total)


# ------------------------------------------------------------------------------------------------------- the work
def work(case):
    if case["op"] == "norm":
        n, s = case["rows"] * case["channels"], {"bf16": 2, "f32": 4}
        mods = (case["gate"] + 2 * case["shift"]) * case["groups"] * case["channels"] + 2 * case["channels"]
        return {"bytes": n * 2 * (s[case["res"]] + s[case["act"]]) + mods * s[case["mod"]], "flops": 14 * n}
    new, old = _lengths(case)
    e = 2 if case["dtype"] == "bf16" else 4
    d, h, hq = case["dim"], case["kv_heads"], case["q_heads"]
    tokens = sum(new)
    if case["op"] == "append":
        pages = sum((o + n - 1) // case["page"] - o // case["page"] + 1 for n, o in zip(new, old))
        table = min(tokens, 256 if case["axes"] == 3 else max(o + n for n, o in zip(new, old))) * case["rot"] * 4
        moved = tokens * (2 * hq * d * e + 2 * h * d * e + 2 * h * d) + pages * 2 * h * 4 + table + tokens * 4 * case["axes"]
        return {"bytes": moved, "flops": tokens * (3 * case["rot"] * (hq + h) + 4 * h * d)}
    seen, pairs = 0, 0
    for n, o in zip(new, old):
        lo, hi = _visible(case, o, o + n)[0], _visible(case, o + n - 1, o + n)[1]
        seen += hi - lo
        for i in range(n):
            a, b = _visible(case, o + i, o + n)
            pairs += b - a
    return {"bytes": 2 * tokens * hq * d * e + 4 * tokens * hq + 2 * seen * h * d + 8 * h * -(-seen // case["page"]),
            "flops": 4 * pairs * hq * d}


# ----------------------------------------------------------------------------------------------------- the inputs
def _normal(g, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def _fill(g, pages, case):
    """A pool of pages as earlier appends left it: codes of normal keys (a few strong channels) and values, and their scales."""
    h, p, d = case["kv_heads"], case["page"], case["dim"]
    codes = torch.empty(pages, 2, h, p, d, dtype=torch.uint8, device=DEV)
    scales = torch.empty(pages, 2, h, device=DEV)
    strong = torch.ones(2, 1, 1, d, device=DEV)
    strong[0, ..., torch.randperm(d, generator=g, device=DEV)[: d // 32]] = 4.0
    step = max(1, (1 << 26) // (2 * h * p * d))
    for i in range(0, pages, step):
        n = min(step, pages - i)
        x = torch.randn((n, 2, h, p, d), generator=g, device=DEV) * strong
        m, e = torch.frexp(x.abs().amax((3, 4)))
        s = torch.ldexp(torch.ones_like(m), torch.where(m <= 0.875, e - 9, e - 8))
        codes[i:i + n] = (x / s[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        scales[i:i + n] = s
    return codes, scales


def _batch(g, case):
    """Packed offsets, lengths and page table of a batch whose pages lie scattered over the pool."""
    new, old = _lengths(case)
    need = [-(-(n + o) // case["page"]) for n, o in zip(new, old)]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=g, device=DEV).int()
    table = torch.full((case["batch"], max(need)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    starts = torch.tensor([0] + new).cumsum(0).int().to(DEV)
    lens = torch.tensor([n + o for n, o in zip(new, old)], dtype=torch.int32, device=DEV)
    return starts, lens, table, pages, new, old


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    if case["op"] == "norm":
        r, c, k = case["rows"], case["channels"], case["groups"]
        res, act, mod = DTYPES[case["res"]], DTYPES[case["act"]], DTYPES[case["mod"]]
        per = -(-r // k)
        m = _normal(g, k, 3, c, scale=0.5, dtype=mod)           # gate, scale and shift as one projection gives them
        return {"case": case, "x": _normal(g, r, c, scale=3.0, dtype=res), "y": _normal(g, r, c, scale=0.7, dtype=act),
                "post": 1 + _normal(g, c, scale=0.1), "pre": 1 + _normal(g, c, scale=0.1), "per": per,
                "gate": m[:, 0] if case["gate"] else None, "scale": m[:, 1] if case["shift"] else None,
                "shift": m[:, 2] if case["shift"] else None}
    starts, lens, table, pages, new, old = _batch(g, case)
    codes, scales = _fill(g, pages, case)
    dtype, d, h, hq = DTYPES[case["dtype"]], case["dim"], case["kv_heads"], case["q_heads"]
    tokens = sum(new)
    s = {"case": case, "starts": starts, "lens": lens, "table": table, "codes": codes, "scales": scales,
         "tokens": tokens, "max_new": max(new)}
    if case["op"] == "attend":
        s["q"] = _normal(g, tokens, hq, d, dtype=dtype)
    else:
        fused = _normal(g, tokens, hq + 2 * h, d, dtype=dtype)
        s["q"], s["k"], s["v"] = fused[:, :hq], fused[:, hq:hq + h], fused[:, hq + h:]
        pos = torch.cat([torch.arange(o, o + n) for n, o in zip(new, old)])
        if case["axes"] == 3:                                   # (frame, row, column) on the 44 x 80 grid
            pos = torch.stack([pos // 3520 % 256, pos % 3520 // 80, pos % 80], 1)
            pairs = case["rot"] // 2
            s["sections"] = (pairs - 2 * (pairs * 3 // 8), pairs * 3 // 8, pairs * 3 // 8)
        else:
            pos, s["sections"] = pos[:, None], (case["rot"] // 2,)
        s["pos"] = pos.int().to(DEV)
        angle = torch.arange(int(pos.max()) + 1, dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(case["rot"] // 2, dtype=torch.float64) / (case["rot"] // 2))
        s["cos"], s["sin"] = angle.cos().float().to(DEV), angle.sin().float().to(DEV)
    if own:                                                     # the cache's handle, the batch and the rotation, as a program keeps them
        from paper_2609_31938_b200 import tokens as tk
        s["cache"] = tk.PagedCache(codes, scales)
        s["batch"] = tk.TokenBatch(starts, lens, table, max_new=s["max_new"])
        if case["op"] == "append":
            s["rotary"] = tk.Rotary(s["cos"], s["sin"], s["sections"], interleaved=case["interleaved"])
    return s


# -------------------------------------------------------------------------------------------------- the plain forms
def _rotate(x, s, case):
    """Position rotation of [tokens, heads, dim] in 32 bits."""
    r = case["rot"]
    axis = torch.repeat_interleave(torch.arange(len(s["sections"]), device=DEV), torch.tensor(s["sections"], device=DEV))
    rows = s["pos"].long()[:, axis]                              # [tokens, r / 2]
    cols = torch.arange(r // 2, device=DEV)
    c, n = s["cos"][rows, cols][:, None], s["sin"][rows, cols][:, None]
    x = x.float()
    if case["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * c - b * n, b * c + a * n], -1)
    return torch.cat([y, x[..., r:]], -1)


def _append_plain(s):
    case = s["case"]
    P = case["page"]
    starts, lens, table, codes, scales = s["starts"].long(), s["lens"].long(), s["table"].long(), s["codes"], s["scales"]
    n = starts[1:] - starts[:-1]
    tok = torch.arange(s["tokens"], device=DEV)
    seq = torch.searchsorted(starts, tok, right=True) - 1
    pos = (lens - n)[seq] + tok - starts[seq]
    page, slot = table[seq, pos // P], pos % P
    kv = torch.stack([_rotate(s["k"], s, case), s["v"].float()], 1)          # [tokens, 2, heads, dim]
    most = torch.zeros_like(scales).index_reduce_(0, page, kv.abs().amax(-1), "amax")
    m, e = torch.frexp(most)
    e = torch.where(most > 0, torch.where(m <= 0.875, e - 9, e - 8), torch.full_like(e, MIN_EXP)).clamp_min(MIN_EXP)
    need = torch.ldexp(torch.ones_like(m), e)
    touched = torch.zeros(scales.shape[0], dtype=torch.bool, device=DEV).index_fill_(0, page, True)
    fresh = torch.zeros_like(touched).index_fill_(0, torch.where(slot == 0, page, page[:1].expand_as(page)), True)
    fresh[page[0]] = slot[0] == 0
    kept = torch.where(fresh[:, None, None], need, torch.maximum(scales, need))
    now = torch.where(touched[:, None, None], kept, scales)
    # the page that a sequence's new tokens begin in holds older ones: their codes move to the page's new scale
    first = (lens - n)[n > 0]
    head = table[n > 0].gather(1, (first // P)[:, None])[:, 0]
    was = codes[head].view(torch.float8_e4m3fn).float()
    moved = (was * (scales[head] / now[head])[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    older = torch.arange(P, device=DEV)[None] < (first % P)[:, None]
    codes[head] = torch.where(older[:, None, None, :, None], moved, codes[head])
    scales.copy_(now)
    x = (kv / now[page][..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
    codes[page, :, :, slot] = x
    return {"q": _rotate(s["q"], s, case).to(s["q"].dtype), "codes": codes.view(torch.float8_e4m3fn), "scales": scales}


def _attend_plain(s):
    case = s["case"]
    B, P, D, H, G = case["batch"], case["page"], case["dim"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    starts, lens, table = s["starts"].long(), s["lens"].long(), s["table"].long().clamp_min(0)
    n, most = starts[1:] - starts[:-1], s["max_new"]
    kv = s["codes"][table].view(torch.float8_e4m3fn).float() * s["scales"][table][..., None, None]
    kv = kv.permute(2, 0, 3, 1, 4, 5).reshape(2, B, H, -1, D)                # [2, batch, heads, tokens, dim]
    t, i = torch.arange(kv.shape[3], device=DEV), torch.arange(most, device=DEV)
    pos = (lens - n)[:, None] + i                                            # [batch, most]
    f, w = case["frame"], case["window"]
    at = pos // f * f if f > 0 else pos
    hi = torch.minimum(at + f, lens[:, None]) if f > 0 else lens[:, None].expand_as(at)
    sees = (t < hi[..., None]) & (t < lens[:, None, None])
    if w >= 0:
        sees &= t >= (at - w)[..., None]
    valid = i < n[:, None]                                                   # [batch, most]
    q = torch.zeros(B, most, H, G, D, device=DEV)
    q[valid] = s["q"].float().view(-1, H, G, D)
    q = q.permute(0, 2, 3, 1, 4).reshape(B, H, G * most, D)
    x = torch.matmul(q, kv[0].transpose(-1, -2)).mul_(D ** -0.5).view(B, H, G, most, -1)
    x.masked_fill_(~sees[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = x.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, H, G * most, -1), kv[1]).view(B, H, G, most, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    o = o.permute(0, 3, 1, 2, 4)[valid].reshape(-1, H * G, D).to(s["q"].dtype)
    lse = (m + total.log())[..., 0].permute(0, 3, 1, 2)[valid].reshape(-1, H * G)
    return {"out": o, "lse": lse}


def _norm(x, kind):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)


def _norm_plain(s):
    case = s["case"]
    group = torch.arange(case["rows"], device=DEV) // s["per"]
    r = _norm(s["y"].float(), "rms") * s["post"]
    if s["gate"] is not None:
        r = r * s["gate"].float()[group]
    r = case["scale"] * s["x"].float() + r
    h = _norm(r, case["kind"]) * s["pre"]
    if s["scale"] is not None:
        h = h * (1 + s["scale"].float()[group]) + s["shift"].float()[group]
    return {"r": r.to(s["x"].dtype), "h": h.to(s["y"].dtype)}


def run(s):
    case = s["case"]
    if not own:
        return {"append": _append_plain, "attend": _attend_plain, "norm": _norm_plain}[case["op"]](s)
    from paper_2609_31938_b200 import tokens as tk
    if case["op"] == "append":
        q = s["cache"].append(s["k"], s["v"], s["batch"], rotary=s["rotary"], positions=s["pos"], q=s["q"])
        return {"q": q, "codes": s["codes"].view(torch.float8_e4m3fn), "scales": s["scales"]}
    if case["op"] == "attend":
        out, lse = s["cache"].attend(s["q"], s["batch"], frame=case["frame"], window=case["window"], want_lse=True)
        return {"out": out, "lse": lse}
    r, h = tk.gated_norm(s["x"], s["y"], gate=s["gate"], post_weight=s["post"], pre_weight=s["pre"], scale=s["scale"],
                         shift=s["shift"], rows_per_group=s["per"], residual_scale=case["scale"], eps=1e-6,
                         post_kind="rms", pre_kind=case["kind"])
    return {"r": r, "h": h}


# ------------------------------------------------------------------------------------------- the definitions in 64 bits
def _e4m3(x):
    """Nearest E4M3 value (ties to even), magnitudes beyond the largest cut to it."""
    x = x.clamp(-E4M3_MAX, E4M3_MAX)
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 1).clamp_min(-6) - 3)
    return torch.round(x / step) * step


def _exact_append(s):
    case = s["case"]
    P, r = case["page"], case["rot"]
    codes, scales = s["codes"].view(torch.float8_e4m3fn).double(), s["scales"].double()
    starts, lens, table = s["starts"].tolist(), s["lens"].tolist(), s["table"].tolist()
    axis = [a for a, m in enumerate(s["sections"]) for _ in range(m)]
    cos = torch.stack([s["cos"].double()[s["pos"][:, a].long(), j] for j, a in enumerate(axis)], 1)
    sin = torch.stack([s["sin"].double()[s["pos"][:, a].long(), j] for j, a in enumerate(axis)], 1)

    def turn(x):
        x = x.double().clone()
        first, second = (slice(0, r, 2), slice(1, r, 2)) if case["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
        z = torch.complex(x[..., first], x[..., second]) * torch.complex(cos, sin)[:, None]
        x[..., first], x[..., second] = z.real, z.imag
        return x

    k, v = turn(s["k"]), s["v"].double()
    for b in range(case["batch"]):
        n = starts[b + 1] - starts[b]
        old = lens[b] - n
        lead = old % P
        count = -(-(lead + n) // P) if n else 0
        if not count:
            continue
        ids = torch.tensor(table[b][old // P:old // P + count], device=DEV)
        new = torch.zeros(2, case["kv_heads"], count * P, case["dim"], dtype=torch.float64, device=DEV)
        new[0, :, lead:lead + n] = k[starts[b]:starts[b + 1]].transpose(0, 1)
        new[1, :, lead:lead + n] = v[starts[b]:starts[b + 1]].transpose(0, 1)
        new = new.view(2, case["kv_heads"], count, P, case["dim"]).permute(2, 0, 1, 3, 4)
        most = new.abs().amax((3, 4))
        need = torch.exp2(torch.ceil(torch.log2(most.clamp_min(1e-300) / E4M3_MAX)).clamp_min(MIN_EXP))
        if lead:
            need[0] = torch.maximum(need[0], scales[ids[0]])
        at = torch.arange(count * P, device=DEV).view(count, 1, 1, P, 1)
        was = codes[ids]
        back = _e4m3(was * (scales[ids] / need)[..., None, None])
        codes[ids] = torch.where(at < lead, back, torch.where(at < lead + n, _e4m3(new / need[..., None, None]), was))
        scales[ids] = need
    return {"q": turn(s["q"]), "codes": codes, "scales": scales}


def _exact_attend(s):
    case = s["case"]
    G = case["q_heads"] // case["kv_heads"]
    starts, lens, table = s["starts"].tolist(), s["lens"].tolist(), s["table"]
    out = torch.zeros(s["tokens"], case["q_heads"], case["dim"], dtype=torch.float64, device=DEV)
    lse = torch.full((s["tokens"], case["q_heads"]), -math.inf, dtype=torch.float64, device=DEV)
    for b in range(case["batch"]):
        n = starts[b + 1] - starts[b]
        ids = table[b, :-(-lens[b] // case["page"])].long()
        lohi = torch.tensor([_visible(case, lens[b] - n + i, lens[b]) for i in range(n)], device=DEV)
        t = torch.arange(lens[b], device=DEV)
        hidden = (t < lohi[:, :1]) | (t >= lohi[:, 1:])
        for h in range(case["kv_heads"]):
            k, v = ((s["codes"][ids, j, h].view(torch.float8_e4m3fn).double() * s["scales"][ids, j, h].double()[:, None, None])
                    .flatten(0, 1)[:lens[b]] for j in range(2))
            for i in range(h * G, h * G + G):
                x = (s["q"][starts[b]:starts[b + 1], i].double() @ k.T) / math.sqrt(case["dim"])
                x[hidden] = -math.inf
                lse[starts[b]:starts[b + 1], i] = torch.logsumexp(x, 1)
                out[starts[b]:starts[b + 1], i] = torch.nan_to_num(torch.softmax(x, 1)) @ v
    return {"out": out, "lse": lse}


def _exact_norm(s):
    case = s["case"]
    r, h = (torch.empty(case["rows"], case["channels"], dtype=torch.float64, device=DEV) for _ in range(2))
    for g in range(case["groups"]):
        at = slice(g * s["per"], min(case["rows"], (g + 1) * s["per"]))
        y = s["y"][at].double()
        z = y / (y.square().mean(1, keepdim=True) + 1e-6).sqrt() * s["post"].double()
        if s["gate"] is not None:
            z *= s["gate"][g].double()
        z = case["scale"] * s["x"][at].double() + z
        r[at] = z
        if case["kind"] == "layer":
            z = (z - z.mean(1, keepdim=True)) / (z.var(1, unbiased=False, keepdim=True) + 1e-6).sqrt()
        else:
            z = z / (z.square().mean(1, keepdim=True) + 1e-6).sqrt()
        z = z * s["pre"].double()
        if s["scale"] is not None:
            z = z * (1 + s["scale"][g].double()) + s["shift"][g].double()
        h[at] = z
    return {"r": r, "h": h}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "norm": _exact_norm}[case["op"]](s)
