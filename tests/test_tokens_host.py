"""Refusals of the token operators' C entry points: everything here is turned down before a device is touched."""
import ctypes

import pytest

import paper_2609_31938_b200 as ccv

K = 1 << 20


def cache(**kw):
    d = dict(codes=16 * K, scales=8 * K, pages=4, kv_heads=2, page_tokens=16, head_dim=64)
    d.update(kw)
    return ccv.KvCache(*d.values())


def batch(**kw):
    d = dict(new_start=K, total=K + 64, page_table=K + 128, batch=2, max_pages=2, tokens=3, max_new=2)
    d.update(kw)
    return ccv.TokenBatchC(*d.values())


def heads(at, ts=128, hs=64):
    return ccv.Heads(at, ts, hs)


def rotary(**kw):
    d = dict(cos=2 * K, sin=3 * K, positions=K + 256, rows=8, pairs=32, axes=1, section=(ctypes.c_int32 * 3)(32, 0, 0), inter=0)
    d.update(kw)
    return ccv.RotaryC(*d.values())


def append(c=None, b=None, k=None, v=None, rot=None, q=None, qo=None, hq=2, dt=ccv.BF16):
    return ccv.ccv3d_kv_append(c or cache(), b or batch(), k or heads(4 * K), v or heads(5 * K), rot, q, qo, hq, dt)


def attend(c=None, b=None, q=None, o=None, lse=None, hq=2, dt=ccv.BF16, frame=1, window=-1, ws=32 * K, n=1 << 40):
    return ccv.ccv3d_kv_attend(c or cache(), b or batch(), q or heads(4 * K), o or heads(5 * K), lse, hq, dt, 1.0, frame,
                               window, ws, n)


def test_struct_sizes():
    assert ctypes.sizeof(ccv.KvCache) == 2 * 8 + 4 * 4
    assert ctypes.sizeof(ccv.TokenBatchC) == 3 * 8 + 4 * 4
    assert ctypes.sizeof(ccv.Heads) == 3 * 8
    assert ctypes.sizeof(ccv.RotaryC) == 3 * 8 + 7 * 4 + 4
    assert ctypes.sizeof(ccv.NormDesc) == 9 * 4 + 2 * 4 + 4 + 7 * 8


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("bad,expected", [
    (dict(c=cache(codes=None)), ccv.ERR_INVALID_ARG),
    (dict(c=cache(scales=None)), ccv.ERR_INVALID_ARG),
    (dict(c=cache(pages=0)), ccv.ERR_INVALID_ARG),
    (dict(c=cache(kv_heads=0)), ccv.ERR_INVALID_ARG),
    (dict(c=cache(page_tokens=48)), ccv.ERR_UNSUPPORTED),
    (dict(c=cache(head_dim=96)), ccv.ERR_UNSUPPORTED),
    (dict(c=cache(codes=16 * K + 8)), ccv.ERR_ALIGNMENT),
    (dict(b=batch(new_start=None)), ccv.ERR_INVALID_ARG),
    (dict(b=batch(page_table=None)), ccv.ERR_INVALID_ARG),
    (dict(b=batch(batch=0)), ccv.ERR_INVALID_ARG),
    (dict(b=batch(tokens=-1)), ccv.ERR_INVALID_ARG),
    (dict(b=batch(max_pages=1 << 28)), ccv.ERR_UNSUPPORTED),
    (dict(b=batch(total=K + 2)), ccv.ERR_ALIGNMENT),
    (dict(dt=7), ccv.ERR_INVALID_ARG),
])
def test_bad_cache_batch_and_type(call, bad, expected):
    assert call(**bad) == expected


@pytest.mark.parametrize("bad,expected", [
    (dict(k=heads(None)), ccv.ERR_INVALID_ARG),
    (dict(k=heads(4 * K + 8)), ccv.ERR_ALIGNMENT),
    (dict(v=heads(5 * K, ts=132)), ccv.ERR_ALIGNMENT),
    (dict(v=heads(5 * K, ts=-128)), ccv.ERR_INVALID_ARG),
    (dict(k=heads(16 * K + 64)), ccv.ERR_ALIAS),                                  # keys inside the pool
    (dict(q=heads(6 * K)), ccv.ERR_INVALID_ARG),                                  # q without q_out
    (dict(q=heads(6 * K), qo=heads(7 * K), hq=0), ccv.ERR_INVALID_ARG),
    (dict(q=heads(6 * K), qo=heads(6 * K + 16)), ccv.ERR_ALIAS),
    (dict(q=heads(6 * K), qo=heads(4 * K)), ccv.ERR_ALIAS),                       # q_out on k
    (dict(q=heads(6 * K), qo=heads(7 * K, ts=64)), ccv.ERR_INVALID_ARG),          # output rows that lie on one another
    (dict(q=heads(6 * K), qo=heads(7 * K, hs=0)), ccv.ERR_INVALID_ARG),
    (dict(rot=rotary(cos=None)), ccv.ERR_INVALID_ARG),
    (dict(rot=rotary(positions=None)), ccv.ERR_INVALID_ARG),
    (dict(rot=rotary(axes=4)), ccv.ERR_INVALID_ARG),
    (dict(rot=rotary(pairs=30)), ccv.ERR_UNSUPPORTED),
    (dict(rot=rotary(pairs=36)), ccv.ERR_UNSUPPORTED),
    (dict(rot=rotary(pairs=16)), ccv.ERR_INVALID_ARG),                            # sections do not sum to the pairs
    (dict(rot=rotary(cos=2 * K + 4)), ccv.ERR_ALIGNMENT),
])
def test_append_refuses(bad, expected):
    assert append(**bad) == expected


@pytest.mark.parametrize("bad,expected", [
    (dict(q=heads(None)), ccv.ERR_INVALID_ARG),
    (dict(hq=3), ccv.ERR_INVALID_ARG),                                            # not a multiple of the kv heads
    (dict(hq=0), ccv.ERR_INVALID_ARG),
    (dict(frame=-1), ccv.ERR_INVALID_ARG),
    (dict(window=-2), ccv.ERR_INVALID_ARG),
    (dict(o=heads(4 * K + 32)), ccv.ERR_ALIAS),
    (dict(o=heads(16 * K)), ccv.ERR_ALIAS),
    (dict(o=heads(5 * K, ts=64)), ccv.ERR_INVALID_ARG),
    (dict(lse=5 * K + 64), ccv.ERR_ALIAS),
    (dict(lse=6 * K + 2), ccv.ERR_ALIGNMENT),
    (dict(ws=32 * K + 16), ccv.ERR_ALIGNMENT),
    (dict(ws=None), ccv.ERR_NOMEM),
    (dict(n=0), ccv.ERR_NOMEM),
])
def test_attend_refuses(bad, expected):
    assert attend(**bad) == expected


def test_calls_without_tokens_need_no_device():
    assert append(b=batch(tokens=0)) == ccv.OK
    assert attend(b=batch(tokens=0)) == ccv.OK
    assert norm(rows=0) == ccv.OK


def norm(x=K, y=2 * K, r=3 * K, h=4 * K, gate=None, pw=None, **kw):
    d = dict(rows=4, channels=64, rows_per_group=1, post_kind=1, pre_kind=2, res_dtype=ccv.F32, act_dtype=ccv.BF16,
             weight_dtype=ccv.F32, mod_dtype=ccv.F32, residual_scale=1.0, eps=1e-6, x_stride=64, y_stride=64, r_stride=64,
             h_stride=64, gate_stride=64, scale_stride=0, shift_stride=0)
    d.update(kw)
    return ccv.ccv3d_gated_norm(ccv.NormDesc(*d.values()), x, y, pw, None, gate, None, None, None, None, r, h)


@pytest.mark.parametrize("bad,expected", [
    (dict(x=None), ccv.ERR_INVALID_ARG),
    (dict(r=None, h=None), ccv.ERR_INVALID_ARG),
    (dict(rows=-1), ccv.ERR_INVALID_ARG),
    (dict(channels=0), ccv.ERR_INVALID_ARG),
    (dict(channels=16385, x_stride=16385, y_stride=16385, r_stride=16385, h_stride=16385), ccv.ERR_UNSUPPORTED),
    (dict(rows_per_group=0), ccv.ERR_INVALID_ARG),
    (dict(post_kind=3), ccv.ERR_INVALID_ARG),
    (dict(pre_kind=-1), ccv.ERR_INVALID_ARG),
    (dict(act_dtype=2), ccv.ERR_INVALID_ARG),
    (dict(r_stride=63), ccv.ERR_INVALID_ARG),
    (dict(x_stride=-64), ccv.ERR_INVALID_ARG),
    (dict(x=K + 2), ccv.ERR_ALIGNMENT),
    (dict(r=K + 256), ccv.ERR_ALIAS),                                             # r one row below x
    (dict(r=K, r_stride=128), ccv.ERR_ALIAS),                                     # r on x with other strides
    (dict(h=K + 256), ccv.ERR_ALIAS),
    (dict(h=3 * K + 64), ccv.ERR_ALIAS),
    (dict(pw=3 * K), ccv.ERR_ALIAS),
    (dict(gate=4 * K), ccv.ERR_ALIAS),
])
def test_gated_norm_refuses(bad, expected):
    assert norm(**bad) == expected


def test_null_structs():
    assert ccv.lib.ccv3d_kv_append(None, None, None, None, None, None, None, 0, 0, None, None) == ccv.ERR_INVALID_ARG
    assert ccv.lib.ccv3d_kv_append(cache(), None, None, None, None, None, None, 0, 0, None, None) == ccv.ERR_INVALID_ARG
    assert ccv.lib.ccv3d_gated_norm(None, *[None] * 12) == ccv.ERR_INVALID_ARG
    assert ccv.lib.ccv3d_kv_attend_workspace(cache(), batch(), 2, ccv.BF16, None) == ccv.ERR_INVALID_ARG
