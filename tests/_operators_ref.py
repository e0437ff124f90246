"""Plain 64-bit implementations of the products, decaying states and group norms, with the sizes that their tolerances go by."""
import math

import torch


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def activate(x, kind):
    if kind == "silu":
        return x / (1 + torch.exp(-x))
    if kind == "gelu":
        return x * torch.special.ndtr(x)
    if kind == "gelu_tanh":
        return x / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    return x


def linear(x, w, bias, kind, gated, residual):
    """(result, sum of the magnitudes that a result's own errors scale with)."""
    d = lambda t: t.double()  # noqa: E731
    n = w.shape[0] // 2 if gated else w.shape[0]
    z, mass = d(x) @ d(w).T, d(x).abs() @ d(w).abs().T
    if bias is not None:
        z, mass = z + d(bias), mass + d(bias).abs()
    a = activate(z[:, :n], kind)
    if gated:
        a, mass = a * z[:, n:], 1.2 * mass[:, :n] * z[:, n:].abs() + a.abs() * mass[:, n:]      # (no activation is steeper than 1.2)
    else:
        mass = 1.2 * mass
    return (a if residual is None else a + d(residual)), mass, a.abs()


def decay(q, k, v, g, starts, slot, fresh, states, scale):
    """(out, states, and both with magnitudes throughout), token by token."""
    q, k, v, g, states = (t.double() for t in (q, k, v, g, states))
    out, big_out = torch.zeros_like(v), torch.zeros_like(v)
    states = states.clone()
    big = states.abs()
    per = v.shape[1] // q.shape[1]
    q, k = q.repeat_interleave(per, 1), k.repeat_interleave(per, 1)
    starts = starts.tolist()
    for b in range(len(starts) - 1):
        s, m = states[slot[b]], big[slot[b]]
        if starts[b + 1] == starts[b]:
            continue
        if fresh is not None and fresh[b]:
            s, m = torch.zeros_like(s), torch.zeros_like(m)
        for t in range(starts[b], starts[b + 1]):
            f = torch.exp(g[t])[:, None, None]
            gone = f == 0
            s = torch.where(gone, torch.zeros_like(s), s * f) + k[t][:, :, None] * v[t][:, None, :]
            m = torch.where(gone, torch.zeros_like(m), m * f) + k[t][:, :, None].abs() * v[t][:, None, :].abs()
            out[t] = scale * torch.einsum("hk,hkv->hv", q[t], s)
            big_out[t] = abs(scale) * torch.einsum("hk,hkv->hv", q[t].abs(), m)
        states[slot[b]], big[slot[b]] = s, m
    return out, states, big_out, big


def group_norm(x, groups, weight, bias, scale, shift, eps, kind):
    """x [samples, pixels, channels] -> (result, size of what the errors scale with)."""
    s, p, c = x.shape
    x = x.double()
    y = x.view(s, p, groups, c // groups)
    mean = y.mean((1, 3), keepdim=True)
    std = (y.var((1, 3), unbiased=False, keepdim=True) + eps).sqrt()
    most = y.abs().mean((1, 3), keepdim=True)
    n, off = ((y - mean) / std).reshape(s, p, c), ((most / std).expand_as(y)).reshape(s, p, c)
    a, b = torch.ones(s, 1, c, dtype=torch.float64, device=x.device), torch.zeros(s, 1, c, dtype=torch.float64, device=x.device)
    if weight is not None:
        a = a * weight.double()
    if bias is not None:
        b = b + bias.double()
    if scale is not None:
        a, b = a * (1 + scale.double())[:, None], b * (1 + scale.double())[:, None]
    if shift is not None:
        b = b + shift.double()[:, None]
    z = n * a + b
    # the mean's rounding, 2^-18 of the mean magnitude, and of the deviation, 2^-18 of the normed value; a few roundings of the terms
    err = 2.0 ** -18 * (off + n.abs()) * a.abs() + 2.0 ** -21 * (n.abs() * a.abs() + b.abs())
    return activate(z, kind), 1.2 * err
