"""Cases of the operators of a latent predictor with a memory of fixed size and of a decoder with normed blocks: matrix
products with their epilogue, attention with decaying states, and group norms on channels-last activations.

A world model that streams for hours keeps, instead of a growing cache of keys and values, one state for each head that
old tokens fade from.  Around it stand the products of its projections and feed-forward blocks (with bias, activation or
gated pair, and residual), the norm of each head's output, and in the decoder behind it the group norms with an activation
in front of the convolutions, on frame rings.  Latent frames are the decoder chain's, 44 x 80 pixels.

`run` with `own` false computes the operators in their plain form: elementary torch operations in 32 bits (sums of log
decays in 64), rounded once.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one latent frame in front of a convolution of the decoder's first stage, on its ring: latency
        dict(name="group-norm-latent-ring", op="group_norm", form="ring", dtype="bf16", n=1, frames=1, h=44, w=80, channels=192,
             groups=32, act="silu", mod=False),
        # four output-size frames of the decoder's last stage: bound by memory
        dict(name="group-norm-output-ring", op="group_norm", form="ring", dtype="bf16", n=1, frames=4, h=352, w=640, channels=96,
             groups=32, act="silu", mod=False),
        # samples of an odd size in 32 bits, with a scale and shift for each
        dict(name="group-norm-odd-f32", op="group_norm", form="rows", dtype="f32", samples=3, pixels=6527, channels=200, groups=25,
             act="gelu_tanh", mod=True),
        # the output of every head of every token of a latent frame, behind the decaying attention
        dict(name="group-norm-heads", op="group_norm", form="rows", dtype="bf16", samples=3520, pixels=1, channels=1536, groups=12,
             act="none", mod=False),
        # queries, keys and values of four streams' next tokens
        dict(name="linear-step", op="linear", dtype="bf16", out="bf16", rows=4, k=1536, n=4608, bias=True, act="none", gated=False,
             residual=False),
        # a gated feed-forward block's first half for one token of each of 64 streams: bound by the weights' bytes
        dict(name="linear-gated-b64", op="linear", dtype="bf16", out="bf16", rows=64, k=4096, n=11008, bias=False, act="silu", gated=True,
             residual=False),
        # a feed-forward block's first half for a latent frame
        dict(name="linear-frame-gelu", op="linear", dtype="bf16", out="bf16", rows=3520, k=1536, n=6144, bias=True, act="gelu_tanh",
             gated=False, residual=False),
        # the largest: its second half for eight latent frames, onto the residual stream in 32 bits
        dict(name="linear-frames-residual", op="linear", dtype="bf16", out="f32", rows=28160, k=6144, n=1536, bias=False, act="none",
             gated=False, residual=True),
        # odd sizes in 32 bits
        dict(name="linear-odd-f32", op="linear", dtype="f32", out="f32", rows=1501, k=1160, n=1153, bias=True, act="silu", gated=False,
             residual=True),
        # one token for each of 64 streams: bound by the states' bytes
        dict(name="decay-step-b64", op="decay", dtype="bf16", batch=64, new_lo=1, new_hi=1, heads=32, qk_heads=32, dk=128, dv=128),
        # eight latent frames of one stream
        dict(name="decay-frames", op="decay", dtype="bf16", batch=1, new_lo=28160, new_hi=28160, heads=12, qk_heads=12, dk=128, dv=128),
        # prompts of unlike length in 32 bits, queries and keys shared by pairs of heads
        dict(name="decay-ragged-f32", op="decay", dtype="f32", batch=24, new_lo=1, new_hi=700, heads=14, qk_heads=7, dk=64, dv=128),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["group_norm", "linear", "linear", "decay"])
    act = rng.choice(["none", "silu", "gelu", "gelu_tanh"])
    if op == "group_norm":
        if rng.random() < 0.5:
            channels = 32 * rng.randint(1, 16)
            h, w = _log(rng, 5, 352), _log(rng, 5, 640)
            n, frames = rng.randint(1, 2), _log(rng, 1, 8)
            while n * frames * h * w * channels > 80_000_000:
                n, frames, h, w = 1, max(1, frames - 1), max(5, h * 3 // 4), max(5, w * 3 // 4)
            return dict(op=op, form="ring", dtype="bf16", n=n, frames=frames, h=h, w=w, channels=channels,
                        groups=rng.choice([g for g in (1, 8, 16, 32) if channels % g == 0]), act=act, mod=rng.random() < 0.3)
        groups = rng.choice([1, 4, 5, 8, 12, 25, 32])
        channels = groups * _log(rng, 1, 2048 // groups)
        samples = _log(rng, 1, 5000)
        pixels = _log(rng, 1, min(60000, max(1, 40_000_000 // (samples * channels))))
        if pixels * channels // groups < 16:         # (a group of a few values is no norm)
            pixels = -(-16 * groups // channels)
        return dict(op=op, form="rows", dtype=rng.choice(["bf16", "f32"]), samples=samples, pixels=pixels, channels=channels, groups=groups,
                    act=act, mod=rng.random() < 0.5)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "linear":
        k, n = 8 * _log(rng, 8, 1024), _log(rng, 1, 12288)
        gated = rng.random() < 0.3
        most = 250_000_000_000 // (1 + gated) // (1 if dtype == "bf16" else 8)
        return dict(op=op, dtype=dtype, out="f32" if dtype == "f32" else rng.choice(["bf16", "bf16", "f32"]), rows=_log(rng, 1, min(30000, most // (k * n))),
                    k=k, n=n, bias=rng.random() < 0.5, act=act, gated=gated, residual=rng.random() < 0.5)
    batch = _log(rng, 1, 64)
    heads, dk, dv = rng.choice([1, 4, 6, 12, 16, 32]), rng.choice([64, 128]), rng.choice([64, 128, 192, 256])
    new_hi = rng.choice([1, 2, 4]) if rng.random() < 0.4 else _log(rng, 5, max(6, min(28000, 2_500_000 // (batch * heads * dv // 16))))
    return dict(op=op, dtype=dtype, batch=batch, new_lo=rng.randint(1, new_hi), new_hi=new_hi, heads=heads,
                qk_heads=rng.choice([q for q in (1, 2, 4, 6, 12, 16, 32) if heads % q == 0]), dk=dk, dv=dv)


def _lengths(case):
    """New tokens of each sequence: spread over the case's range, the same for every seed."""
    rng = random.Random(case["batch"] * 1000003 + case["new_hi"])
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["batch"])]
    new[rng.randrange(case["batch"])] = case["new_hi"]
    return new


# ------------------------------------------------------------------------------------------------------- the work
def work(case):
    size = {"bf16": 2, "f32": 4}
    e = size[case["dtype"]]
    if case["op"] == "group_norm":
        if case["form"] == "ring":
            samples, pixels = case["n"] * case["frames"], case["h"] * case["w"]
        else:
            samples, pixels = case["samples"], case["pixels"]
        values, c = samples * pixels * case["channels"], case["channels"]
        return {"bytes": 2 * values * e + 8 * c + (8 * samples * c if case["mod"] else 0), "flops": 8 * values}
    if case["op"] == "linear":
        m, k, n, pair = case["rows"], case["k"], case["n"], 1 + case["gated"]
        o = size[case["out"]] * m * n
        return {"bytes": m * k * e + pair * n * k * e + o * (1 + case["residual"]) + (pair * n * e if case["bias"] else 0),
                "flops": 2 * m * n * k * pair}
    tokens, h, q, dk, dv = sum(_lengths(case)), case["heads"], case["qk_heads"], case["dk"], case["dv"]
    # the recurrence's operations: the state's decay and update, and its product with the query
    return {"bytes": tokens * (2 * q * dk + 2 * h * dv) * e + 4 * tokens * h + 8 * case["batch"] * h * dk * dv,
            "flops": 5 * tokens * h * dk * dv}


# ----------------------------------------------------------------------------------------------------- the inputs
def _normal(g, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "group_norm":
        c = case["channels"]
        # activations: channels of unlike mean and spread
        mean, spread = _normal(g, c, scale=0.5), 0.5 + torch.rand(c, generator=g, device=DEV)
        s = {"case": case, "weight": 1 + _normal(g, c, scale=0.2), "bias": _normal(g, c, scale=0.2)}
        if case["form"] == "ring":
            n, t, h, w, kb = case["n"], case["frames"], case["h"], case["w"], 64 if c % 64 == 0 else 32
            x = torch.randn((n, t, c // kb, h, w, kb), generator=g, device=DEV)
            s["x"] = (x * spread.view(c // kb, 1, 1, kb) + mean.view(c // kb, 1, 1, kb)).to(dtype)
            samples = n * t
        else:
            samples = case["samples"]
            s["x"] = (torch.randn((samples, case["pixels"], c), generator=g, device=DEV) * spread + mean).to(dtype)
        m = _normal(g, samples, 2, c, scale=0.3)                # scale and shift as one projection gives them
        s["scale"], s["shift"] = (m[:, 0], m[:, 1]) if case["mod"] else (None, None)
        if own and case["form"] == "ring":                      # the decoder's rings
            import paper_2609_31938_b200 as ccv
            s["ring"], s["to"] = (ccv.FrameRing(n, c, t, h, w) for _ in range(2))
            s["ring"].buf.copy_(s["x"])
        return s
    if case["op"] == "linear":
        m, k, n, pair = case["rows"], case["k"], case["n"], 1 + case["gated"]
        return {"case": case, "x": _normal(g, m, k, dtype=dtype), "weight": _normal(g, pair * n, k, scale=k ** -0.5, dtype=dtype),
                "bias": _normal(g, pair * n, scale=0.5, dtype=dtype) if case["bias"] else None,
                "residual": _normal(g, m, n, scale=2.0, dtype=DTYPES[case["out"]]) if case["residual"] else None}
    new = _lengths(case)
    tokens, b, h, q, dk, dv = sum(new), case["batch"], case["heads"], case["qk_heads"], case["dk"], case["dv"]
    fused = _normal(g, tokens, 2 * q * dk + h * dv)             # queries, keys and values as one projection gives them
    fused[:, q * dk:2 * q * dk] *= dk ** -0.5
    fused = fused.to(dtype)
    # heads that remember from five tokens to a thousand, tokens that let more or less of it go
    rate = torch.exp(torch.linspace(math.log(0.2), math.log(0.001), h, device=DEV))
    s = {"case": case, "new": new, "q": fused[:, :q * dk].unflatten(1, (q, dk)), "k": fused[:, q * dk:2 * q * dk].unflatten(1, (q, dk)),
         "v": fused[:, 2 * q * dk:].unflatten(1, (h, dv)), "decay": -rate * torch.exp(_normal(g, tokens, h, scale=0.7)),
         "starts": torch.tensor([0] + new).cumsum(0).int().to(DEV), "state": _normal(g, b + 2, h, dk, dv),
         "slot": torch.randperm(b + 2, generator=g, device=DEV)[:b].int()}
    if own:                                                     # the memory's handle and the batch, as a program keeps them
        from paper_2609_31938_b200 import tokens as tk
        s["memory"] = tk.DecayMemory(s["state"])
        s["batch"] = tk.StreamBatch(s["starts"], s["slot"], max_new=max(new))
    return s


# -------------------------------------------------------------------------------------------------- the plain forms
def _act(x, kind):
    if kind == "silu":
        return x / (1 + torch.exp(-x))
    if kind == "gelu":
        return 0.5 * x * (1 + torch.erf(x * 0.5 ** 0.5))
    if kind == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh((2 / math.pi) ** 0.5 * (x + 0.044715 * x * x * x)))
    return x


def _group_norm_plain(s):
    case, x = s["case"], s["x"]
    c, groups = case["channels"], case["groups"]
    if case["form"] == "ring":
        x = x.permute(0, 1, 3, 4, 2, 5)                          # [n, frames, h, w, blocks, channels of a block]
    y = x.float().reshape(-1, x.shape[2] * x.shape[3] if case["form"] == "ring" else case["pixels"], groups, c // groups)
    y = y - y.mean((1, 3), keepdim=True)
    y = y * torch.rsqrt((y * y).mean((1, 3), keepdim=True) + EPS)
    y = y.flatten(2) * s["weight"] + s["bias"]
    if s["scale"] is not None:
        y = y * (1 + s["scale"][:, None]) + s["shift"][:, None]
    y = _act(y, case["act"]).to(x.dtype).view(x.shape)
    return y.permute(0, 1, 4, 2, 3, 5).contiguous() if case["form"] == "ring" else y


def _linear_plain(s):
    case = s["case"]
    y = torch.matmul(s["x"].float(), s["weight"].float().T)
    if s["bias"] is not None:
        y = y + s["bias"].float()
    y = _act(y[:, :case["n"]], case["act"]) * y[:, case["n"]:] if case["gated"] else _act(y, case["act"])
    if s["residual"] is not None:
        y = s["residual"].float() + y
    return y.to(DTYPES[case["out"]])


CHUNK = 64


def _decay_plain(s):
    """The recurrence in chunks of tokens, the batch padded with tokens that do nothing."""
    case = s["case"]
    h, per, most = case["heads"], case["heads"] // case["qk_heads"], -(-case["new_hi"] // CHUNK) * CHUNK
    starts = s["starts"].long()
    at = torch.arange(most, device=DEV)
    valid = at < (starts[1:] - starts[:-1])[:, None]            # [batch, most]
    rows = (starts[:-1, None] + at)[valid]

    def padded(x):                                               # [tokens, heads, dim] -> [batch, heads, chunks, CHUNK, dim]
        y = torch.zeros(valid.shape + x.shape[1:], dtype=x.dtype, device=DEV)
        y[valid] = x[rows]
        return y.transpose(1, 2).unflatten(2, (-1, CHUNK))

    q, k, v = padded(s["q"].float()), padded(s["k"].float()), padded(s["v"].float())
    q, k = q.repeat_interleave(per, 1) * case["dk"] ** -0.5, k.repeat_interleave(per, 1)
    total = padded(s["decay"].double()[..., None])[..., 0].cumsum(-1)                # [batch, heads, chunks, CHUNK]
    slot = s["slot"].long()
    state = s["state"][slot]
    later = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=DEV).triu(1)
    out = torch.empty(v.shape, device=DEV)
    for i in range(v.shape[2]):
        qi, ki, vi, t = q[:, :, i], k[:, :, i], v[:, :, i], total[:, :, i]
        fade = torch.exp((t[..., :, None] - t[..., None, :]).masked_fill(later, -math.inf)).float()
        out[:, :, i] = torch.matmul(torch.matmul(qi, ki.transpose(-1, -2)) * fade, vi) + torch.matmul(qi * torch.exp(t).float()[..., None], state)
        last = t[..., -1:]
        state = state * torch.exp(last).float()[..., None] + torch.matmul((ki * torch.exp(last - t).float()[..., None]).transpose(-1, -2), vi)
    s["state"][slot] = state
    out = out.flatten(2, 3).transpose(1, 2)[valid]
    return {"out": out.to(s["q"].dtype), "state": s["state"]}


def run(s):
    case = s["case"]
    if not own:
        return {"group_norm": _group_norm_plain, "linear": _linear_plain, "decay": _decay_plain}[case["op"]](s)
    from paper_2609_31938_b200 import tokens as tk
    if case["op"] == "group_norm":
        if case["form"] == "ring":
            s["ring"].group_norm(0, case["frames"], case["groups"], s["weight"], s["bias"], scale=s["scale"], shift=s["shift"], eps=EPS,
                                 activation=case["act"], out_ring=s["to"])
            return s["to"].buf
        return tk.group_norm(s["x"], case["groups"], s["weight"], s["bias"], scale=s["scale"], shift=s["shift"], eps=EPS, activation=case["act"])
    if case["op"] == "linear":
        return tk.linear(s["x"], s["weight"], s["bias"], activation=case["act"], gated=case["gated"], residual=s["residual"],
                         out_dtype=DTYPES[case["out"]])
    return {"out": s["memory"].attend(s["q"], s["k"], s["v"], s["decay"], s["batch"]), "state": s["state"]}


# ------------------------------------------------------------------------------------------- the definitions in 64 bits
def _exact_act(x, kind):
    if kind == "silu":
        return x * torch.special.expit(x)
    if kind == "gelu":
        return x * torch.special.ndtr(x)
    if kind == "gelu_tanh":
        return x * torch.special.expit(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))
    return x


def _exact_group_norm(s):
    case = s["case"]
    x = s["x"].flatten(0, 1) if case["form"] == "ring" else s["x"]     # [samples, blocks, h, w, kb], or [samples, pixels, channels]
    out = torch.empty(x.shape, dtype=torch.float64, device=DEV)
    c, per = case["channels"], case["channels"] // case["groups"]
    blocks, kb = (x.shape[1], x.shape[4]) if case["form"] == "ring" else (1, c)
    step = max(1, 60_000_000 // (x.numel() // x.shape[0]))
    for i in range(0, x.shape[0], step):
        z = x[i:i + step].double().reshape(-1, blocks, x[0].numel() // c, kb).movedim(2, 3).flatten(1, 2)    # [samples, channels, pixels]
        zg = z.unflatten(1, (-1, per)).flatten(2)
        m, v = zg.mean(2), zg.var(2, unbiased=False)
        a = (v + EPS).sqrt().reciprocal().repeat_interleave(per, 1)
        z = (z - m.repeat_interleave(per, 1)[..., None]) * (a * s["weight"].double())[..., None] + s["bias"].double()[:, None]
        if s["scale"] is not None:
            z = z * (1 + s["scale"][i:i + step].double())[..., None] + s["shift"][i:i + step].double()[..., None]
        z = _exact_act(z, case["act"])
        out[i:i + step] = z.unflatten(1, (blocks, kb)).movedim(3, 2).reshape(x[i:i + step].shape)
    return out.view(s["x"].shape)


def _exact_linear(s):
    case, n = s["case"], s["case"]["n"]
    w = s["weight"].double()
    out = torch.empty(case["rows"], n, dtype=torch.float64, device=DEV)
    for i in range(0, case["rows"], 4096):
        x = s["x"][i:i + 4096].double()
        z = [x @ w[j:j + n].T + (0 if s["bias"] is None else s["bias"][j:j + n].double()) for j in range(0, w.shape[0], n)]
        y = _exact_act(z[0], case["act"])
        for u in z[1:]:
            y = y * u
        out[i:i + 4096] = y if s["residual"] is None else y + s["residual"][i:i + 4096].double()
    return out


def _exact_decay(s):
    """Token by token, all sequences side by side."""
    case, new = s["case"], torch.tensor(s["new"], device=DEV)
    per = case["heads"] // case["qk_heads"]
    begin, slot = s["starts"][:-1].long(), s["slot"].long()
    state = s["state"].double()
    out = torch.empty(s["v"].shape, dtype=torch.float64, device=DEV)
    q, k = (x.double().repeat_interleave(per, 1) for x in (s["q"], s["k"]))
    v, keep = s["v"].double(), torch.exp(s["decay"].double())
    shortest = min(s["new"])
    for i in range(case["new_hi"]):
        live = slice(None) if i < shortest else new > i
        row, at = begin[live] + i, slot[live]
        now = state[at] * keep[row][..., None, None]
        now.addcmul_(k[row][..., :, None], v[row][..., None, :])
        out[row] = torch.matmul(q[row][..., None, :], now)[..., 0, :]
        state[at] = now
    return {"out": out * case["dk"] ** -0.5, "state": state}


def exact(case, seed):
    s = prepare(case, seed)
    return {"group_norm": _exact_group_norm, "linear": _exact_linear, "decay": _exact_decay}[case["op"]](s)
