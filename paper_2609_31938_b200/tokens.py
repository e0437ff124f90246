"""Token operators on torch tensors: a paged E4M3 cache of keys and values, and the gated norms between blocks.

What a transformer that predicts the latents of a streamed decoder needs next to its matrix products.  torch owns the
memory and the stream (its current one); every step runs in ``libccv3d.so`` (``ccv3d_kv_append``, ``ccv3d_kv_attend``,
``ccv3d_gated_norm``, declared with their rules in ``include/ccv3d.h``).
"""
from __future__ import annotations

import ctypes

import torch

from . import (BF16, F32, NORM_LAYER, NORM_NONE, NORM_RMS, OK, Ccv3dError, Heads, KvCache, NormDesc, RotaryC, TokenBatchC,
               ccv3d_kv_attend_workspace, lib)

_DTYPES = {torch.bfloat16: BF16, torch.float32: F32}
_KINDS = {"none": NORM_NONE, "rms": NORM_RMS, "layer": NORM_LAYER}


def _dtype(t: torch.Tensor, what: str) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise TypeError(f"{what}: {t.dtype} is neither bfloat16 nor float32")
    return d


def _on_device(t: torch.Tensor, what: str, dev: int) -> None:
    if t.get_device() != dev:
        raise ValueError(f"{what} is on {t.device}, not on the current CUDA device cuda:{dev}")


def _heads(t: torch.Tensor, what: str, tokens: int, dim: int, dev: int) -> Heads:
    if t.dim() != 3 or t.shape[0] != tokens or t.shape[2] != dim:
        raise ValueError(f"{what} has shape {tuple(t.shape)}: [{tokens}, heads, {dim}] is wanted")
    _on_device(t, what, dev)
    ts, hs, es = t.stride()
    if es != 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    if t.shape[1] == 1:
        hs = dim             # torch gives a dimension of one any stride
    if tokens == 1:
        ts = t.shape[1] * hs
    return Heads(t.data_ptr(), ts, hs)


def _int_array(t: torch.Tensor, what: str, shape, dev: int) -> None:
    if t.dtype != torch.int32 or not t.is_contiguous() or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} must be a contiguous int32 tensor of shape {tuple(shape)}, not {t.dtype} {tuple(t.shape)}")
    _on_device(t, what, dev)


class TokenBatch:
    """The sequences of a call (``ccv3d_token_batch``): packed offsets of their new tokens [batch + 1], their lengths
    with the new tokens [batch], and their page tables [batch, max_pages], int32 on the device.  The arrays may be
    changed in place between calls (a captured graph replays with what they hold then); ``max_new`` bounds the new
    tokens of any sequence, ``tokens`` (default: what the call's tensors hold) the rows."""

    def __init__(self, new_start, total, page_table, max_new: int):
        dev = torch.cuda.current_device()
        b = total.shape[0]
        _int_array(new_start, "new_start", (b + 1,), dev)
        _int_array(total, "total", (b,), dev)
        _int_array(page_table, "page_table", (b, page_table.shape[1]), dev)
        self.new_start, self.total, self.page_table, self.max_new = new_start, total, page_table, int(max_new)
        self.device = dev
        self.c = TokenBatchC(new_start.data_ptr(), total.data_ptr(), page_table.data_ptr(), b, page_table.shape[1], 0,
                             self.max_new)


class Rotary:
    """Position rotation (``ccv3d_rotary``): FP32 tables of cosines and sines [rows, pairs]; ``sections`` splits the
    pairs among the axes of ``positions`` (default: one axis)."""

    def __init__(self, cos, sin, sections=None, interleaved=False):
        dev = torch.cuda.current_device()
        for t, what in ((cos, "cos"), (sin, "sin")):
            if t.dtype != torch.float32 or t.dim() != 2 or not t.is_contiguous() or t.shape != cos.shape:
                raise ValueError(f"{what} must be a contiguous float32 table [rows, pairs]")
            _on_device(t, what, dev)
        sections = tuple(int(s) for s in (sections or (cos.shape[1],)))
        if not 1 <= len(sections) <= 3 or sum(sections) != cos.shape[1]:
            raise ValueError(f"sections {sections} do not split {cos.shape[1]} pairs among one to three axes")
        self.cos, self.sin, self.axes = cos, sin, len(sections)
        self.c = RotaryC(cos.data_ptr(), sin.data_ptr(), None, cos.shape[0], cos.shape[1], len(sections),
                         (ctypes.c_int32 * 3)(*sections, *([0] * (3 - len(sections)))), int(bool(interleaved)))


class PagedCache:
    """A paged cache of keys and values in E4M3 with a power-of-two scale for each page and head.

    ``codes`` uint8 [pages, 2, kv_heads, page_tokens, head_dim] (keys, then values), ``scales`` float32
    [pages, 2, kv_heads]; ``PagedCache.empty`` allocates them."""

    def __init__(self, codes, scales):
        dev = torch.cuda.current_device()
        if codes.dtype != torch.uint8 or codes.dim() != 5 or codes.shape[1] != 2 or not codes.is_contiguous():
            raise ValueError("codes must be a contiguous uint8 tensor [pages, 2, kv_heads, page_tokens, head_dim]")
        if scales.dtype != torch.float32 or scales.shape != codes.shape[:3] or not scales.is_contiguous():
            raise ValueError(f"scales must be a contiguous float32 tensor {tuple(codes.shape[:3])}")
        _on_device(codes, "codes", dev)
        _on_device(scales, "scales", dev)
        self.codes, self.scales, self.device = codes, scales, dev
        self.pages, _, self.kv_heads, self.page_tokens, self.head_dim = codes.shape
        self.c = KvCache(codes.data_ptr(), scales.data_ptr(), self.pages, self.kv_heads, self.page_tokens, self.head_dim)
        self._status = torch.zeros(1, dtype=torch.int32, device=codes.device)
        self._status_ptr = self._status.data_ptr()

    @classmethod
    def empty(cls, pages, kv_heads, head_dim, page_tokens=64):
        return cls(torch.empty((pages, 2, kv_heads, page_tokens, head_dim), dtype=torch.uint8, device="cuda"),
                   torch.zeros((pages, 2, kv_heads), dtype=torch.float32, device="cuda"))

    def status(self) -> int:
        """TOKENS_* bits that the calls so far have reported (waits for them), cleared by reading."""
        bits = int(self._status.item())
        if bits:
            self._status.zero_()
        return bits

    def _batch(self, batch: TokenBatch, tokens: int) -> TokenBatchC:
        if batch.device != self.device:
            raise ValueError("the batch lies on another device than the cache")
        if torch.cuda.current_device() != self.device:
            raise ValueError(f"the cache lies on cuda:{self.device}, which is not the current device")
        batch.c.tokens = tokens
        return batch.c

    def append(self, k, v, batch: TokenBatch, rotary: Rotary | None = None, positions=None, q=None, q_out=None):
        """Writes the new keys (rotated) and values [tokens, kv_heads, head_dim] into the cache; returns ``q`` rotated
        (a new tensor, or ``q_out``, which may be ``q`` itself), None without ``q``."""
        tokens, dim, dev = k.shape[0], self.head_dim, self.device
        c = self._batch(batch, tokens)
        dt = _dtype(k, "k")
        if k.shape != v.shape or k.shape[1] != self.kv_heads:
            raise ValueError(f"k {tuple(k.shape)} and v {tuple(v.shape)} must be [tokens, {self.kv_heads}, {dim}]")
        if v.dtype != k.dtype or (q is not None and q.dtype != k.dtype):
            raise TypeError("q, k and v must have one type")
        ck, cv = _heads(k, "k", tokens, dim, dev), _heads(v, "v", tokens, dim, dev)
        r = None
        if rotary is not None:
            if positions is None:
                raise ValueError("a rotation needs positions")
            if positions.dim() == 1:
                positions = positions[:, None]
            _int_array(positions, "positions", (tokens, rotary.axes), dev)
            r = rotary.c
            r.positions = positions.data_ptr()
        cq = cqo = None
        heads = 0
        if q is not None:
            heads = q.shape[1]
            cq = _heads(q, "q", tokens, dim, dev)
            if q_out is None:
                q_out = torch.empty((tokens, heads, dim), dtype=q.dtype, device=q.device)
            elif q_out.dtype != q.dtype or q_out.shape != q.shape:
                raise ValueError("q_out must have q's shape and type")
            cqo = _heads(q_out, "q_out", tokens, dim, dev)
        elif q_out is not None:
            raise ValueError("q_out without q")
        s = lib.ccv3d_kv_append(self.c, c, ck, cv, r, cq, cqo, heads, dt, self._status_ptr,
                                torch.cuda.current_stream().cuda_stream)
        if s != OK:
            raise Ccv3dError(s, "ccv3d_kv_append")
        return q_out

    def attend(self, q, batch: TokenBatch, scale: float | None = None, frame: int = 1, window: int = -1, out=None,
               want_lse: bool = False):
        """Attention of q [tokens, q_heads, head_dim] over the cache (``frame``, ``window``: who sees what, as
        ``ccv3d_kv_attend`` says); ``scale`` defaults to head_dim ** -0.5.  Returns out, or (out, lse)."""
        tokens, heads = q.shape[0], q.shape[1]
        c = self._batch(batch, tokens)
        dt = _dtype(q, "q")
        cq = _heads(q, "q", tokens, self.head_dim, self.device)
        if out is None:
            out = torch.empty((tokens, heads, self.head_dim), dtype=q.dtype, device=q.device)
        elif out.dtype != q.dtype or out.shape != q.shape:
            raise ValueError("out must have q's shape and type")
        co = _heads(out, "out", tokens, self.head_dim, self.device)
        lse = torch.empty((tokens, heads), dtype=torch.float32, device=q.device) if want_lse else None
        s, need = ccv3d_kv_attend_workspace(self.c, c, heads, dt)
        if s != OK:
            raise Ccv3dError(s, "ccv3d_kv_attend_workspace")
        # scratch from torch's allocator: on the current stream, so calls on other streams never share it
        ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
        s = lib.ccv3d_kv_attend(self.c, c, cq, co, None if lse is None else lse.data_ptr(), heads, dt,
                                self.head_dim ** -0.5 if scale is None else scale, frame, window,
                                None if ws is None else ws.data_ptr(), need, self._status_ptr,
                                torch.cuda.current_stream().cuda_stream)
        if s != OK:
            raise Ccv3dError(s, "ccv3d_kv_attend")
        return (out, lse) if want_lse else out


def _rows(t, what, shape, dev):
    if t.dim() != 2 or tuple(t.shape) != shape:
        raise ValueError(f"{what} has shape {tuple(t.shape)}: {list(shape)} is wanted")
    _on_device(t, what, dev)
    rs, es = t.stride()
    if es != 1 and shape[1] > 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    return rs if shape[0] > 1 else shape[1]


def gated_norm(x, y=None, *, gate=None, post_weight=None, post_bias=None, pre_weight=None, pre_bias=None, scale=None,
               shift=None, rows_per_group: int | None = None, residual_scale: float = 1.0, eps: float = 1e-6,
               post_kind: str = "none", pre_kind: str = "rms", out_r=None, out_h=None, act_dtype=None, want_r: bool = True,
               want_h: bool = True):
    """(r, h): r = residual_scale x + gate * post(y), h = pre(r) * (1 + scale) + shift (``ccv3d_gated_norm``).

    x [rows, channels] is the residual stream (r has its type), y the block's output (h has its type; without y, or to
    ask for another, ``act_dtype``).  gate, scale and shift are [groups, channels]; row i reads group
    i // rows_per_group (default: the rows split evenly).  Weights and biases [channels] share one type, as do gate,
    scale and shift.  ``out_r`` may be x and ``out_h`` y.  An output not wanted is None."""
    if x.dim() != 2:
        raise ValueError("x must be [rows, channels]")
    rows, ch = x.shape
    shape = (rows, ch)
    dev = torch.cuda.current_device()
    d = NormDesc()
    d.rows, d.channels, d.residual_scale, d.eps = rows, ch, residual_scale, eps
    d.post_kind, d.pre_kind = _KINDS[post_kind], _KINDS[pre_kind]
    d.res_dtype = _dtype(x, "x")
    d.x_stride = _rows(x, "x", shape, dev)
    if y is not None:
        if act_dtype is not None and act_dtype != y.dtype:
            raise TypeError("act_dtype differs from y's type")
        act_dtype = y.dtype
        d.y_stride = _rows(y, "y", shape, dev)
    act_dtype = act_dtype or x.dtype
    if act_dtype not in _DTYPES:
        raise TypeError(f"act_dtype {act_dtype} is neither bfloat16 nor float32")
    d.act_dtype = _DTYPES[act_dtype]
    groups, mod, weight = None, None, None
    for t, what, field in ((gate, "gate", "gate_stride"), (scale, "scale", "scale_stride"), (shift, "shift", "shift_stride")):
        if t is None:
            continue
        if t.dim() != 2 or t.shape[1] != ch or (groups is not None and t.shape[0] != groups) or (mod is not None and t.dtype != mod):
            raise ValueError(f"{what} must be [groups, {ch}], with one type and number of groups for gate, scale and shift")
        groups, mod = t.shape[0], t.dtype
        setattr(d, field, _rows(t, what, (groups, ch), dev))
    d.mod_dtype = F32 if mod is None else _DTYPES.get(mod, -1)
    if rows_per_group is None:
        rows_per_group = max(1, -(-rows // groups)) if groups else max(1, rows)
    if groups is not None and rows > groups * rows_per_group:
        raise ValueError(f"{groups} groups of {rows_per_group} rows do not cover {rows} rows")
    d.rows_per_group = rows_per_group
    for t, what in ((post_weight, "post_weight"), (post_bias, "post_bias"), (pre_weight, "pre_weight"), (pre_bias, "pre_bias")):
        if t is None:
            continue
        if t.shape != (ch,) or not t.is_contiguous() or (weight is not None and t.dtype != weight):
            raise ValueError(f"{what} must be a contiguous [{ch}], with one type for all weights and biases")
        _on_device(t, what, dev)
        weight = t.dtype
    d.weight_dtype = F32 if weight is None else _DTYPES.get(weight, -1)
    if out_r is None and want_r:
        out_r = torch.empty(shape, dtype=x.dtype, device=x.device)
    if out_h is None and want_h:
        out_h = torch.empty(shape, dtype=act_dtype, device=x.device)
    for t, what, dt, field in ((out_r, "out_r", x.dtype, "r_stride"), (out_h, "out_h", act_dtype, "h_stride")):
        if t is not None:
            if t.dtype != dt:
                raise TypeError(f"{what} must be {dt}")
            setattr(d, field, _rows(t, what, shape, dev))
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    s = lib.ccv3d_gated_norm(d, x.data_ptr(), ptr(y), ptr(post_weight), ptr(post_bias), ptr(gate), ptr(pre_weight),
                             ptr(pre_bias), ptr(scale), ptr(shift), ptr(out_r), ptr(out_h),
                             torch.cuda.current_stream().cuda_stream)
    if s != OK:
        raise Ccv3dError(s, "ccv3d_gated_norm")
    return out_r, out_h
