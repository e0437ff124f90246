"""Token operators on torch tensors: a paged E4M3 cache of keys and values, and the gated norms between blocks.

What a transformer that predicts the latents of a streamed decoder needs next to its matrix products.  torch owns the
memory and the stream (its current one); every step runs in ``libccv3d.so`` (``ccv3d_kv_append``, ``ccv3d_kv_attend``,
``ccv3d_gated_norm``, declared with their rules in ``include/ccv3d.h``).
"""
from __future__ import annotations

import ctypes
import threading

import torch

from . import (ACTIVATIONS, BF16, F32, NORM_LAYER, NORM_NONE, NORM_RMS, OK, Ccv3dError, DecayMemoryC, GroupNormDesc, Heads, KvCache,
               LinearDesc, NormDesc, RotaryC, StreamBatchC, TokenBatchC, ccv3d_decay_attend_workspace, ccv3d_group_norm_ring_workspace,
               ccv3d_group_norm_workspace, ccv3d_kv_attend_workspace, ccv3d_linear_status_word, ccv3d_linear_workspace, ccv3d_take_status, lib)

_DTYPES = {torch.bfloat16: BF16, torch.float32: F32}
_KINDS = {"none": NORM_NONE, "rms": NORM_RMS, "layer": NORM_LAYER}
# current device and stream as plain numbers: the calls below are short enough for the objects around them to matter
_device = torch.cuda.current_device
_stream = torch._C._cuda_getCurrentRawStream
_like = torch.empty_like
_capturing = torch._C._cuda_isCurrentStreamCapturing
_synchronize = torch.cuda.synchronize
_DENSE = torch.contiguous_format


def _dtype(t: torch.Tensor, what: str) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise TypeError(f"{what}: {t.dtype} is neither bfloat16 nor float32")
    return d


def _int32(v: int, what: str) -> int:
    if not -0x80000000 <= v <= 0x7FFFFFFF:
        raise ValueError(f"{what} {v} does not fit 32 bits")
    return v


def _elsewhere(t: torch.Tensor, what: str, dev: int):
    return ValueError(f"{what} is on {t.device}, not on the current CUDA device cuda:{dev}")


def _on_device(t: torch.Tensor, what: str, dev: int) -> None:
    if t.get_device() != dev:
        raise _elsewhere(t, what, dev)


def _heads(t: torch.Tensor, what: str, tokens: int, dim: int, dev: int) -> Heads:
    shape = t.shape
    if len(shape) != 3 or shape[0] != tokens or shape[2] != dim:
        raise ValueError(f"{what} has shape {tuple(shape)}: [{tokens}, heads, {dim}] is wanted")
    if t.get_device() != dev:
        raise _elsewhere(t, what, dev)
    ts, hs, es = t.stride()
    if es != 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    if shape[1] == 1:
        hs = dim             # torch gives a dimension of one any stride
    if tokens == 1:
        ts = shape[1] * hs
    return Heads(t.data_ptr(), ts, hs)


def _int_array(t: torch.Tensor, what: str, shape, dev: int) -> None:
    if t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous int32 tensor of shape {tuple(shape)}, not {t.dtype} {tuple(t.shape)}")
    _on_device(t, what, dev)


class TokenBatch:
    """The sequences of a call (``ccv3d_token_batch``): packed offsets of their new tokens [batch + 1], their lengths
    with the new tokens [batch], and their page tables [batch, max_pages], int32 on the device.  The arrays may be
    changed in place between calls (a captured graph replays with what they hold then); ``max_new`` bounds the new
    tokens of any sequence.  A batch and a rotation may serve several calls at a time: no call writes to them."""

    def __init__(self, new_start, total, page_table, max_new: int):
        dev = _device()
        b = total.shape[0]
        _int_array(new_start, "new_start", (b + 1,), dev)
        _int_array(total, "total", (b,), dev)
        _int_array(page_table, "page_table", (b, page_table.shape[1]), dev)
        self.new_start, self.total, self.page_table, self.max_new = new_start, total, page_table, _int32(int(max_new), "max_new")
        self.device = dev
        self._at = (new_start.data_ptr(), total.data_ptr(), page_table.data_ptr(), b, page_table.shape[1])
        self._c = {}

    def c(self, tokens: int) -> TokenBatchC:
        """The struct of a call with so many rows (kept, and not written again)."""
        c = self._c.get(tokens)
        if c is None:
            if len(self._c) >= 64:
                self._c = {}
            c = self._c[tokens] = TokenBatchC(*self._at, tokens, self.max_new)
        return c


class Rotary:
    """Position rotation (``ccv3d_rotary``): FP32 tables of cosines and sines [rows, pairs]; ``sections`` splits the
    pairs among the axes of ``positions`` (default: one axis)."""

    def __init__(self, cos, sin, sections=None, interleaved=False):
        dev = _device()
        for t, what in ((cos, "cos"), (sin, "sin")):
            if t.dtype != torch.float32 or t.dim() != 2 or not t.is_contiguous() or t.shape != cos.shape:
                raise ValueError(f"{what} must be a contiguous float32 table [rows, pairs]")
            _on_device(t, what, dev)
        sections = tuple(int(s) for s in (sections or (cos.shape[1],)))
        if not 1 <= len(sections) <= 3 or sum(sections) != cos.shape[1]:
            raise ValueError(f"sections {sections} do not split {cos.shape[1]} pairs among one to three axes")
        self.cos, self.sin, self.axes = cos, sin, len(sections)      # (the struct without positions: `at` adds a call's)
        self.c = RotaryC(cos.data_ptr(), sin.data_ptr(), None, cos.shape[0], cos.shape[1], len(sections),
                         (ctypes.c_int32 * 3)(*sections, *([0] * (3 - len(sections)))), int(bool(interleaved)))

    def at(self, positions: torch.Tensor) -> RotaryC:
        """The struct of a call with these positions: its own, as several calls may be made at a time."""
        r = RotaryC.from_buffer_copy(self.c)
        r.positions = positions.data_ptr()
        return r


class PagedCache:
    """A paged cache of keys and values in E4M3 with a power-of-two scale for each page and head.

    ``codes`` uint8 [pages, 2, kv_heads, page_tokens, head_dim] (keys, then values), ``scales`` float32
    [pages, 2, kv_heads]; ``PagedCache.empty`` allocates them."""

    def __init__(self, codes, scales):
        dev = _device()
        if codes.dtype != torch.uint8 or codes.dim() != 5 or codes.shape[1] != 2 or not codes.is_contiguous():
            raise ValueError("codes must be a contiguous uint8 tensor [pages, 2, kv_heads, page_tokens, head_dim]")
        if scales.dtype != torch.float32 or scales.shape != codes.shape[:3] or not scales.is_contiguous():
            raise ValueError(f"scales must be a contiguous float32 tensor {tuple(codes.shape[:3])}")
        _on_device(codes, "codes", dev)
        _on_device(scales, "scales", dev)
        self.codes, self.scales, self.device = codes, scales, dev
        self.pages, _, self.kv_heads, self.page_tokens, self.head_dim = codes.shape
        self.c = KvCache(codes.data_ptr(), scales.data_ptr(), self.pages, self.kv_heads, self.page_tokens, self.head_dim)
        # there for every stream when this returns (in a capture, whose every replay zeroes it: for what follows there)
        self._status = torch.zeros(1, dtype=torch.int32, device=codes.device if _capturing() else None).to(codes.device)
        self._status_ptr = self._status.data_ptr()
        self._needs = {}         # geometry of a call -> bytes of scratch
        self._scratch = {}       # stream -> scratch of attend calls on it
        self._lock = threading.Lock()

    @classmethod
    def empty(cls, pages, kv_heads, head_dim, page_tokens=64):
        return cls(torch.empty((pages, 2, kv_heads, page_tokens, head_dim), dtype=torch.uint8, device="cuda"),
                   torch.zeros((pages, 2, kv_heads), dtype=torch.float32, device="cuda"))

    def status(self) -> int:
        """TOKENS_* bits that the calls so far have reported, cleared by reading.  Waits for the device, as the calls may have
        gone to any of its streams, and holds back calls of other threads meanwhile (not replays of their graphs)."""
        with self._lock:
            _synchronize(self.device)
            bits = int(self._status.item())
            if bits:
                self._status.zero_()
                _synchronize(self.device)
        return bits

    def _batch(self, batch: TokenBatch, tokens: int) -> TokenBatchC:
        if batch.device != self.device:
            raise ValueError("the batch lies on another device than the cache")
        if _device() != self.device:
            raise ValueError(f"the cache lies on cuda:{self.device}, which is not the current device")
        return batch.c(tokens)

    def _workspace(self, c: TokenBatchC, heads: int, dt: int, stream: int):
        """Scratch for an attend call on `stream`: kept for the next call on it, so calls on other streams never share it.
        A captured call gets its own, which belongs to the graph.  Called, and the scratch put to use, under the lock: an
        attend call is two launches, and those of two host threads on one stream must not come in between."""
        key = (c.max_new, c.batch, c.max_pages, c.tokens, heads, dt)
        need = self._needs.get(key)
        if need is None:
            s, need = ccv3d_kv_attend_workspace(self.c, c, heads, dt)
            if s != OK:
                raise Ccv3dError(s, "ccv3d_kv_attend_workspace")
            if len(self._needs) > 4096:
                self._needs.clear()
            self._needs[key] = need
        if _capturing():
            return torch.empty(need, dtype=torch.uint8, device=self.codes.device), need
        ws = self._scratch.get(stream)
        if ws is None or ws.shape[0] < need:
            ws = self._scratch[stream] = torch.empty(need, dtype=torch.uint8, device=self.codes.device)
        return ws, need

    def append(self, k, v, batch: TokenBatch, rotary: Rotary | None = None, positions=None, q=None, q_out=None):
        """Writes the new keys (rotated) and values [tokens, kv_heads, head_dim] into the cache; returns ``q`` rotated
        (a new tensor, or ``q_out``, which may be ``q`` itself), None without ``q``."""
        shape = k.shape
        tokens, dim, dev = shape[0], self.head_dim, self.device
        c = self._batch(batch, tokens)
        dt = _dtype(k, "k")
        if shape != v.shape or len(shape) != 3 or shape[1] != self.kv_heads:
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
            if rotary.cos.get_device() != dev:
                raise ValueError("the rotation lies on another device than the cache")
            r = rotary.at(positions)
        cq = cqo = None
        heads = 0
        if q is not None:
            cq = _heads(q, "q", tokens, dim, dev)
            heads = q.shape[1]
            if q_out is None:
                q_out = _like(q, memory_format=_DENSE)
                cqo = Heads(q_out.data_ptr(), heads * dim, dim)
            elif q_out.dtype != q.dtype or q_out.shape != q.shape:
                raise ValueError("q_out must have q's shape and type")
            else:
                cqo = _heads(q_out, "q_out", tokens, dim, dev)
        elif q_out is not None:
            raise ValueError("q_out without q")
        with self._lock:         # (see status)
            s = lib.ccv3d_kv_append(self.c, c, ck, cv, r, cq, cqo, heads, dt, self._status_ptr, _stream(dev))
        if s != OK:
            raise Ccv3dError(s, "ccv3d_kv_append")
        return q_out

    def attend(self, q, batch: TokenBatch, scale: float | None = None, frame: int = 1, window: int = -1, out=None,
               want_lse: bool = False):
        """Attention of q [tokens, q_heads, head_dim] over the cache (``frame``, ``window``: who sees what, as
        ``ccv3d_kv_attend`` says); ``scale`` defaults to head_dim ** -0.5.  Returns out, or (out, lse); rows behind the
        last sequence's are not written."""
        tokens, dim, dev = q.shape[0], self.head_dim, self.device
        c = self._batch(batch, tokens)
        dt = _dtype(q, "q")
        cq = _heads(q, "q", tokens, dim, dev)
        heads = q.shape[1]
        _int32(frame, "frame")
        _int32(window, "window")
        if out is None:
            out = _like(q, memory_format=_DENSE)
            co = Heads(out.data_ptr(), heads * dim, dim)
        elif out.dtype != q.dtype or out.shape != q.shape:
            raise ValueError("out must have q's shape and type")
        else:
            co = _heads(out, "out", tokens, dim, dev)
        lse = q.new_empty((tokens, heads), dtype=torch.float32) if want_lse else None
        stream = _stream(dev)
        with self._lock:
            ws, need = self._workspace(c, heads, dt, stream)
            s = lib.ccv3d_kv_attend(self.c, c, cq, co, None if lse is None else lse.data_ptr(), heads, dt,
                                    dim ** -0.5 if scale is None else scale, frame, window, ws.data_ptr(), need,
                                    self._status_ptr, stream)
        if s != OK:
            raise Ccv3dError(s, "ccv3d_kv_attend")
        return (out, lse) if want_lse else out


def _rows(t, what, rows, ch, dev):
    """Elements between the rows of a [rows, ch] tensor."""
    if t.shape != (rows, ch):
        raise ValueError(f"{what} has shape {tuple(t.shape)}: {[rows, ch]} is wanted")
    if t.get_device() != dev:
        raise _elsewhere(t, what, dev)
    rs, es = t.stride()
    if es != 1 and ch > 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    return rs if rows > 1 else ch


def _ptr(t):
    return None if t is None else t.data_ptr()


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
    _int32(rows, "the number of rows")
    dev = _device()
    res = _dtype(x, "x")
    xs, ys = _rows(x, "x", rows, ch, dev), 0
    if y is not None:
        if act_dtype is not None and act_dtype != y.dtype:
            raise TypeError("act_dtype differs from y's type")
        act_dtype = y.dtype
        ys = _rows(y, "y", rows, ch, dev)
    elif act_dtype is None:
        act_dtype = x.dtype
    act = _DTYPES.get(act_dtype)
    if act is None:
        raise TypeError(f"{act_dtype} is neither bfloat16 nor float32")
    groups, mod, strides = None, torch.float32, [0, 0, 0]
    for i, t in enumerate((gate, scale, shift)):
        if t is None:
            continue
        if groups is None:
            groups, mod = t.shape[0], t.dtype
        elif t.dtype != mod:
            raise TypeError("gate, scale and shift must have one type")
        strides[i] = _rows(t, ("gate", "scale", "shift")[i], groups, ch, dev)
    if rows_per_group is None:
        rows_per_group = max(1, -(-rows // groups)) if groups else max(1, rows)
    _int32(rows_per_group, "rows_per_group")
    if groups is not None and rows > groups * rows_per_group:
        raise ValueError(f"{groups} groups of {rows_per_group} rows do not cover {rows} rows")
    weight = None
    for t in (post_weight, post_bias, pre_weight, pre_bias):
        if t is None:
            continue
        if weight is None:
            weight = t.dtype
        if t.shape != (ch,) or t.dtype != weight or not t.is_contiguous():
            raise ValueError(f"weights and biases must be contiguous [{ch}] tensors of one type")
        if t.get_device() != dev:
            raise _elsewhere(t, "a weight or bias", dev)
    rs = hs = ch
    if out_r is not None:
        if out_r.dtype != x.dtype:
            raise TypeError(f"out_r must be {x.dtype}")
        rs = _rows(out_r, "out_r", rows, ch, dev)
    elif want_r:
        out_r = _like(x, memory_format=_DENSE)
    if out_h is not None:
        if out_h.dtype != act_dtype:
            raise TypeError(f"out_h must be {act_dtype}")
        hs = _rows(out_h, "out_h", rows, ch, dev)
    elif want_h:
        out_h = _like(x if y is None else y, dtype=act_dtype, memory_format=_DENSE)
    d = NormDesc(rows, ch, rows_per_group, _KINDS[post_kind], _KINDS[pre_kind], res, act,
                 F32 if weight is None else _DTYPES.get(weight, -1), _DTYPES.get(mod, -1), residual_scale, eps, xs, ys, rs, hs,
                 *strides)
    s = lib.ccv3d_gated_norm(d, x.data_ptr(), _ptr(y), _ptr(post_weight), _ptr(post_bias), _ptr(gate), _ptr(pre_weight),
                             _ptr(pre_bias), _ptr(scale), _ptr(shift), _ptr(out_r), _ptr(out_h), _stream(dev))
    if s != OK:
        raise Ccv3dError(s, "ccv3d_gated_norm")
    return out_r, out_h


# ---- scratch of a call: taken from torch's allocator on the current stream and given back when the call has been made, so that what
# ---- follows on the stream may have it next (and a captured call's belongs to its graph)
_needs = {}


def _scratch(key, ask, what, *args):
    """(tensor or None, address, bytes) of scratch for a call; `key` says what the size depends on."""
    need = _needs.get(key)
    if need is None:
        s, need = ask(*args)
        if s != OK:
            raise Ccv3dError(s, what)
        if len(_needs) > 4096:
            _needs.clear()
        _needs[key] = need
    if need == 0:
        return None, None, 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    return ws, ws.data_ptr(), need


def _vector(t, what, n, dtype, dev):
    if t is None:
        return None
    if t.shape != (n,) or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous [{n}] tensor of {dtype}, not {t.dtype} {tuple(t.shape)}")
    if t.get_device() != dev:
        raise _elsewhere(t, what, dev)
    return t.data_ptr()


def _per_sample(t, what, samples, ch, dev):
    """(address, elements between rows) of a float32 [samples, channels] tensor, which may be a slice."""
    if t is None:
        return None, 0
    if t.dtype != torch.float32:
        raise TypeError(f"{what} must be float32")
    return t.data_ptr(), _rows(t, what, samples, ch, dev)


def _activation(name):
    kind = ACTIVATIONS.get(name)
    if kind is None:
        raise ValueError(f"activation {name!r} is none of {', '.join(ACTIVATIONS)}")
    return kind


def group_norm(x, groups: int, weight=None, bias=None, *, scale=None, shift=None, eps: float = 1e-6, activation: str = "none", out=None):
    """act((norm(x) * weight + bias) * (1 + scale) + shift), as ``ccv3d_group_norm`` says: x [samples, pixels, channels] (channels dense, any
    strides), normed for each sample and group of channels over all pixels.  weight and bias are [channels], scale
    and shift [samples, channels], all float32.  ``out`` may be x."""
    if x.dim() != 3:
        raise ValueError("x must be [samples, pixels, channels]")
    samples, pixels, ch = x.shape
    dt, dev = _dtype(x, "x"), _device()
    for n, what in ((samples, "the number of samples"), (pixels, "the number of pixels"), (ch, "the number of channels")):
        _int32(n, what)
    _int32(groups, "groups")
    if out is None:
        out = _like(x, memory_format=_DENSE)
    elif out.dtype != x.dtype or out.shape != x.shape:
        raise ValueError("out must have x's shape and type")
    for t, what in ((x, "x"), (out, "out")):
        if t.get_device() != dev:
            raise _elsewhere(t, what, dev)
        if t.stride(2) != 1 and ch > 1:
            raise ValueError(f"{what}: the last dimension must be contiguous")
    sc, sc_stride = _per_sample(scale, "scale", samples, ch, dev)
    sh, sh_stride = _per_sample(shift, "shift", samples, ch, dev)
    w, b = _vector(weight, "weight", ch, torch.float32, dev), _vector(bias, "bias", ch, torch.float32, dev)
    d = GroupNormDesc(samples, pixels, ch, groups, _activation(activation), dt, eps, x.stride(0), x.stride(1), out.stride(0), out.stride(1),
                      sc_stride, sh_stride)
    keep, ws, need = _scratch(("group_norm", samples, pixels, ch, groups, dt), ccv3d_group_norm_workspace, "ccv3d_group_norm_workspace", d)
    s = lib.ccv3d_group_norm(d, x.data_ptr(), w, b, sc, sh, out.data_ptr(), ws, need, _stream(dev))
    if s != OK:
        raise Ccv3dError(s, "ccv3d_group_norm")
    return out


def ring_group_norm(ring, slot, T, groups, weight, bias, scale, shift, eps, activation, out_ring, out_slot):
    """``FrameRing.group_norm``."""
    dev = _device()
    for r in (ring, out_ring):
        if r.buf.get_device() != dev:
            raise _elsewhere(r.buf, "the ring", dev)
    for n, what in ((slot, "slot"), (out_slot, "out_slot"), (T, "T"), (groups, "groups")):
        _int32(n, what)
    samples = ring.N * T
    sc, sc_stride = _per_sample(scale, "scale", samples, ring.C, dev)
    sh, sh_stride = _per_sample(shift, "shift", samples, ring.C, dev)
    w, b = _vector(weight, "weight", ring.C, torch.float32, dev), _vector(bias, "bias", ring.C, torch.float32, dev)
    keep, ws, need = _scratch(("ring", ring.N, ring.C, ring.F, ring.H, ring.W, T, groups), ccv3d_group_norm_ring_workspace,
                              "ccv3d_group_norm_ring_workspace", ring.c, T, groups)
    s = lib.ccv3d_group_norm_ring(ring.c, slot, out_ring.c, out_slot, T, groups, w, b, sc, sc_stride, sh, sh_stride, eps,
                                  _activation(activation), ws, need, _stream(dev))
    if s != OK:
        raise Ccv3dError(s, "ccv3d_group_norm_ring")


_words = {}              # device -> address of the library's word that products report in
_reports = threading.Lock()


def _word(dev):
    w = _words.get(dev)
    if w is None:
        s, w = ccv3d_linear_status_word()
        if s != OK:
            raise Ccv3dError(s, "ccv3d_linear_status_word")
        _words[dev] = w
    return w


def status() -> int:
    """TOKENS_* bits that products (``linear``) on the current device have reported, replays of captured ones too, cleared by reading.
    Waits for the device, and holds back products of other threads meanwhile (not replays of their graphs)."""
    with _reports:
        s, bits = ccv3d_take_status(_word(_device()))
    if s != OK:
        raise Ccv3dError(s, "ccv3d_take_status")
    return bits


def linear(x, weight, bias=None, *, activation: str = "none", gated: bool = False, residual=None, out=None, out_dtype=None):
    """residual + act(x weight^T + bias), or gated: residual + act(x w1^T + b1) * (x w2^T + b2) for weight [w1; w2] and bias [b1; b2]
    (``ccv3d_linear``).

    x [rows, k] and weight [n, k] (gated [2 n, k]) have one type, rows dense and on 16 bytes; bias has it too.  out [rows, n] has x's
    type, or ``out_dtype`` (float32), which residual has as well; it may be residual."""
    if x.dim() != 2 or weight.dim() != 2 or weight.shape[1] != x.shape[1]:
        raise ValueError(f"x {tuple(x.shape)} and weight {tuple(weight.shape)} must be [rows, k] and [n, k]")
    rows, k = x.shape
    n, dev = weight.shape[0], _device()
    dt = _dtype(x, "x")
    if weight.dtype != x.dtype:
        raise TypeError("x and weight must have one type")
    if gated:
        if n % 2:
            raise ValueError("a gated pair has an even number of rows of weights")
        n //= 2
    for v, what in ((rows, "the number of rows"), (k, "k"), (2 * n, "the number of features")):
        _int32(v, what)
    if out is not None:
        if out_dtype is not None and out_dtype != out.dtype:
            raise TypeError("out_dtype differs from out's type")
        out_dtype = out.dtype
    elif out_dtype is None:
        out_dtype = x.dtype
    od = _DTYPES.get(out_dtype)
    if od is None:
        raise TypeError(f"{out_dtype} is neither bfloat16 nor float32")
    if dt == F32 and od != F32:
        raise TypeError("a product of float32 is float32")
    xs, ws_ = _rows(x, "x", rows, k, dev), _rows(weight, "weight", weight.shape[0], k, dev)
    b = _vector(bias, "bias", weight.shape[0], x.dtype, dev)
    rs = n
    if residual is not None:
        if residual.dtype != out_dtype:
            raise TypeError(f"residual must be {out_dtype}")
        rs = _rows(residual, "residual", rows, n, dev)
    if out is None:
        out, os_ = x.new_empty((rows, n), dtype=out_dtype), n
    else:
        os_ = _rows(out, "out", rows, n, dev)
    if rows == 0 or n == 0:
        return out
    d = LinearDesc(rows, n, k, bool(gated), _activation(activation), dt, od, xs, ws_, os_, rs)
    keep, ws, need = _scratch(("linear", dev, rows, n, k, bool(gated), dt), ccv3d_linear_workspace, "ccv3d_linear_workspace", d)
    with _reports:           # (see status)
        s = lib.ccv3d_linear(d, x.data_ptr(), weight.data_ptr(), b, _ptr(residual), out.data_ptr(), ws, need, _word(dev), _stream(dev))
    if s != OK:
        raise Ccv3dError(s, "ccv3d_linear")
    return out


class StreamBatch:
    """The sequences of a call on decaying states (``ccv3d_stream_batch``): packed offsets of their new tokens [batch + 1], the
    slots of their states [batch], and, where given, which of them start anew (``fresh`` [batch], not 0), int32 on the device.  The arrays
    may be changed in place between calls; ``max_new`` bounds the new tokens of any sequence.  May serve several calls at a time."""

    def __init__(self, new_start, slot, max_new: int, fresh=None):
        dev = _device()
        b = slot.shape[0]
        _int_array(new_start, "new_start", (b + 1,), dev)
        _int_array(slot, "slot", (b,), dev)
        if fresh is not None:
            _int_array(fresh, "fresh", (b,), dev)
        self.new_start, self.slot, self.fresh, self.max_new = new_start, slot, fresh, _int32(int(max_new), "max_new")
        self.device = dev
        self._at = (new_start.data_ptr(), slot.data_ptr(), _ptr(fresh), b)
        self._c = {}

    def c(self, tokens: int) -> StreamBatchC:
        """The struct of a call with so many rows (kept, and not written again)."""
        c = self._c.get(tokens)
        if c is None:
            if len(self._c) >= 64:
                self._c = {}
            c = self._c[tokens] = StreamBatchC(*self._at, tokens, self.max_new)
        return c


class DecayMemory:
    """States of fixed size from which old tokens fade, one for each slot and head: float32 [slots, heads, key_dim, value_dim].

    ``DecayMemory.empty`` allocates them (zeros)."""

    def __init__(self, states):
        dev = _device()
        if states.dtype != torch.float32 or states.dim() != 4 or not states.is_contiguous():
            raise ValueError("states must be a contiguous float32 tensor [slots, heads, key_dim, value_dim]")
        _on_device(states, "states", dev)
        self.states, self.device = states, dev
        self.slots, self.heads, self.key_dim, self.value_dim = states.shape
        self.c = DecayMemoryC(states.data_ptr(), *states.shape)
        # there for every stream when this returns (in a capture, whose every replay zeroes it: for what follows there)
        self._status = torch.zeros(1, dtype=torch.int32, device=states.device if _capturing() else None).to(states.device)
        self._status_ptr = self._status.data_ptr()
        self._lock = threading.Lock()

    @classmethod
    def empty(cls, slots, heads, key_dim, value_dim):
        return cls(torch.zeros((slots, heads, key_dim, value_dim), dtype=torch.float32, device="cuda"))

    def status(self) -> int:
        """TOKENS_* bits that the calls so far have reported, cleared by reading.  Waits for the device, and holds back calls of other
        threads meanwhile (not replays of their graphs)."""
        with self._lock:
            _synchronize(self.device)
            bits = int(self._status.item())
            if bits:
                self._status.zero_()
                _synchronize(self.device)
        return bits

    def attend(self, q, k, v, log_decay, batch: StreamBatch, scale: float | None = None, out=None):
        """Takes the new tokens' keys and values into the states of their sequences, each after the states have faded by
        exp(log_decay), and reads them with the queries (``ccv3d_decay_attend``): q, k [tokens, qk_heads, key_dim], v, out [tokens, heads,
        value_dim], log_decay [tokens, heads] float32; ``scale`` defaults to key_dim ** -0.5.  Rows behind the last sequence's are not written."""
        tokens, dev, heads = q.shape[0], self.device, self.heads
        if batch.device != dev:
            raise ValueError("the batch lies on another device than the states")
        if _device() != dev:
            raise ValueError(f"the states lie on cuda:{dev}, which is not the current device")
        c = batch.c(tokens)
        dt = _dtype(q, "q")
        if k.dtype != q.dtype or v.dtype != q.dtype:
            raise TypeError("q, k and v must have one type")
        if k.shape != q.shape:
            raise ValueError(f"q {tuple(q.shape)} and k {tuple(k.shape)} must have one shape")
        cq, ck = _heads(q, "q", tokens, self.key_dim, dev), _heads(k, "k", tokens, self.key_dim, dev)
        cv = _heads(v, "v", tokens, self.value_dim, dev)
        if v.shape[1] != heads:
            raise ValueError(f"v has {v.shape[1]} heads, the states {heads}")
        if log_decay.dtype != torch.float32 or log_decay.shape != (tokens, heads):
            raise ValueError(f"log_decay must be float32 [{tokens}, {heads}], not {log_decay.dtype} {tuple(log_decay.shape)}")
        _on_device(log_decay, "log_decay", dev)
        if out is None:
            out = _like(v, memory_format=_DENSE)
            co = Heads(out.data_ptr(), heads * self.value_dim, self.value_dim)
        elif out.dtype != v.dtype or out.shape != v.shape:
            raise ValueError("out must have v's shape and type")
        else:
            co = _heads(out, "out", tokens, self.value_dim, dev)
        qk_heads = q.shape[1]
        keep, ws, need = _scratch(("decay", dev, c.batch, tokens, c.max_new, heads, self.key_dim, self.value_dim, dt),
                                  ccv3d_decay_attend_workspace, "ccv3d_decay_attend_workspace", self.c, c, qk_heads, dt)
        with self._lock:         # (see status)
            s = lib.ccv3d_decay_attend(self.c, c, cq, ck, cv, log_decay.data_ptr(), log_decay.stride(0), log_decay.stride(1), co, qk_heads,
                                       dt, self.key_dim ** -0.5 if scale is None else scale, ws, need, self._status_ptr, _stream(dev))
        if s != OK:
            raise Ccv3dError(s, "ccv3d_decay_attend")
        return out
