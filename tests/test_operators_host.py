"""Refusals of the products', decaying states' and group norms' C entry points: turned down before a device is touched."""
import ctypes

import pytest

import paper_2609_31938_b200 as ccv

K = 1 << 20


def test_struct_sizes():
    assert ctypes.sizeof(ccv.LinearDesc) == 7 * 4 + 4 + 4 * 8
    assert ctypes.sizeof(ccv.DecayMemoryC) == 8 + 4 * 4
    assert ctypes.sizeof(ccv.StreamBatchC) == 3 * 8 + 3 * 4 + 4
    assert ctypes.sizeof(ccv.GroupNormDesc) == 7 * 4 + 4 + 6 * 8


def linear(x=4 * K, w=8 * K, bias=None, res=None, out=16 * K, ws=None, n=0, status=None, **kw):
    d = dict(rows=4, n_out=32, k=64, gated=0, activation=0, dtype=ccv.BF16, out_dtype=ccv.BF16, x_stride=64, w_stride=64, out_stride=32,
             residual_stride=32)
    d.update(kw)
    return ccv.ccv3d_linear(ccv.LinearDesc(*d.values()), x, w, bias, res, out, ws, n, status)


@pytest.mark.parametrize("bad,expected", [
    (dict(rows=-1), ccv.ERR_INVALID_ARG), (dict(n_out=0), ccv.ERR_INVALID_ARG), (dict(k=0), ccv.ERR_INVALID_ARG), (dict(gated=2), ccv.ERR_INVALID_ARG),
    (dict(activation=4), ccv.ERR_INVALID_ARG), (dict(activation=-1), ccv.ERR_INVALID_ARG), (dict(dtype=2), ccv.ERR_INVALID_ARG),
    (dict(dtype=ccv.F32), ccv.ERR_INVALID_ARG),                                   # F32 into BF16
    (dict(k=65544, x_stride=65544, w_stride=65544), ccv.ERR_UNSUPPORTED), (dict(n_out=0x7FFFFFF0), ccv.ERR_UNSUPPORTED), (dict(rows=0x7FFFFFF0), ccv.ERR_UNSUPPORTED),
    (dict(rows=800_000_000, dtype=ccv.F32, out_dtype=ccv.F32), ccv.ERR_UNSUPPORTED),
    (dict(x=None), ccv.ERR_INVALID_ARG), (dict(w=None), ccv.ERR_INVALID_ARG), (dict(out=None), ccv.ERR_INVALID_ARG),
    (dict(x_stride=56), ccv.ERR_INVALID_ARG), (dict(w_stride=8), ccv.ERR_INVALID_ARG), (dict(out_stride=31), ccv.ERR_INVALID_ARG),
    (dict(res=20 * K, residual_stride=-1), ccv.ERR_INVALID_ARG),
    (dict(x=4 * K + 8), ccv.ERR_ALIGNMENT), (dict(w=8 * K + 2), ccv.ERR_ALIGNMENT), (dict(x_stride=68), ccv.ERR_ALIGNMENT), (dict(w_stride=65), ccv.ERR_ALIGNMENT),
    (dict(bias=K + 1), ccv.ERR_ALIGNMENT), (dict(out=16 * K + 1), ccv.ERR_ALIGNMENT), (dict(res=20 * K + 1), ccv.ERR_ALIGNMENT), (dict(status=6), ccv.ERR_ALIGNMENT),
    (dict(out=4 * K + 64), ccv.ERR_ALIAS), (dict(out=8 * K + 2), ccv.ERR_ALIAS), (dict(bias=16 * K + 8), ccv.ERR_ALIAS),
    (dict(res=16 * K + 2), ccv.ERR_ALIAS), (dict(res=16 * K, residual_stride=33), ccv.ERR_ALIAS),
])
def test_linear_refusals(bad, expected):
    assert linear(**bad) == expected


def test_linear_without_rows():
    assert linear(rows=0, x=None, out=None) == ccv.OK
    assert ccv.ccv3d_linear_workspace(ccv.LinearDesc(0, 32, 64, 0, 0, ccv.BF16, ccv.BF16, 64, 64, 32, 32)) == (ccv.OK, 0)
    assert ccv.ccv3d_linear_workspace(ccv.LinearDesc(0, 0, 64, 0, 0, ccv.BF16, ccv.BF16, 64, 64, 32, 32))[0] == ccv.ERR_INVALID_ARG
    assert linear(rows=0, activation=9) == ccv.ERR_INVALID_ARG


def memory(**kw):
    d = dict(states=64 * K, slots=4, heads=2, key_dim=64, value_dim=64)
    d.update(kw)
    return ccv.DecayMemoryC(*d.values())


def batch(**kw):
    d = dict(new_start=K, slot=K + 64, fresh=None, batch=2, tokens=3, max_new=2)
    d.update(kw)
    return ccv.StreamBatchC(*d.values())


def heads(at, ts=128, hs=64):
    return ccv.Heads(at, ts, hs)


def decay(m=None, b=None, q=None, k=None, v=None, g=2 * K, gt=2, gh=1, o=None, qk=2, dt=ccv.BF16):
    return ccv.ccv3d_decay_attend(m or memory(), b or batch(), q or heads(4 * K), k or heads(5 * K), v or heads(6 * K), g, gt, gh,
                                  o or heads(7 * K), qk, dt, 1.0)


@pytest.mark.parametrize("bad,expected", [
    (dict(m=memory(states=None)), ccv.ERR_INVALID_ARG), (dict(m=memory(slots=0)), ccv.ERR_INVALID_ARG), (dict(m=memory(heads=0)), ccv.ERR_INVALID_ARG),
    (dict(m=memory(key_dim=96)), ccv.ERR_UNSUPPORTED), (dict(m=memory(value_dim=96)), ccv.ERR_UNSUPPORTED), (dict(m=memory(value_dim=576)), ccv.ERR_UNSUPPORTED),
    (dict(m=memory(heads=8192)), ccv.ERR_UNSUPPORTED), (dict(m=memory(states=64 * K + 8)), ccv.ERR_ALIGNMENT),
    (dict(b=batch(batch=-1)), ccv.ERR_INVALID_ARG), (dict(b=batch(tokens=-1)), ccv.ERR_INVALID_ARG), (dict(b=batch(max_new=-1)), ccv.ERR_INVALID_ARG),
    (dict(b=batch(batch=0)), ccv.ERR_INVALID_ARG), (dict(b=batch(batch=70000)), ccv.ERR_UNSUPPORTED), (dict(b=batch(tokens=0x7FFFFFFF)), ccv.ERR_UNSUPPORTED),
    (dict(b=batch(new_start=None)), ccv.ERR_INVALID_ARG), (dict(b=batch(slot=None)), ccv.ERR_INVALID_ARG),
    (dict(b=batch(slot=K + 2)), ccv.ERR_ALIGNMENT), (dict(b=batch(fresh=K + 1)), ccv.ERR_ALIGNMENT),
    (dict(qk=0), ccv.ERR_INVALID_ARG), (dict(m=memory(heads=3)), ccv.ERR_INVALID_ARG), (dict(dt=5), ccv.ERR_INVALID_ARG),
    (dict(g=None), ccv.ERR_INVALID_ARG), (dict(gt=-1), ccv.ERR_INVALID_ARG), (dict(g=2 * K + 2), ccv.ERR_ALIGNMENT),
    (dict(q=heads(None)), ccv.ERR_INVALID_ARG), (dict(q=heads(4 * K + 8)), ccv.ERR_ALIGNMENT), (dict(k=heads(5 * K, ts=132)), ccv.ERR_ALIGNMENT),
    (dict(v=heads(6 * K, hs=-64)), ccv.ERR_INVALID_ARG),
    (dict(o=heads(7 * K, ts=64)), ccv.ERR_INVALID_ARG),                           # rows of out on one another
])
def test_decay_refusals(bad, expected):
    assert decay(**bad) == expected


def test_decay_without_work():
    assert decay(b=batch(tokens=0)) == ccv.OK
    assert decay(b=batch(max_new=0)) == ccv.OK
    assert decay(b=batch(batch=0, tokens=0, new_start=None, slot=None)) == ccv.OK
    assert ccv.ccv3d_decay_attend_workspace(memory(), batch(batch=0, tokens=0), 2, ccv.BF16) == (ccv.OK, 0)


def norm(x=4 * K, y=8 * K, w=None, b=None, scale=None, shift=None, ws=None, n=0, **kw):
    d = dict(samples=2, pixels=3, channels=32, groups=4, activation=0, dtype=ccv.BF16, eps=1e-6, xs=96, xp=32, ys=96, yp=32, scs=32, shs=32)
    d.update(kw)
    return ccv.ccv3d_group_norm(ccv.GroupNormDesc(*d.values()), x, w, b, scale, shift, y, ws, n)


@pytest.mark.parametrize("bad,expected", [
    (dict(samples=-1), ccv.ERR_INVALID_ARG), (dict(pixels=-1), ccv.ERR_INVALID_ARG), (dict(channels=0), ccv.ERR_INVALID_ARG), (dict(groups=0), ccv.ERR_INVALID_ARG),
    (dict(groups=5), ccv.ERR_INVALID_ARG), (dict(activation=4), ccv.ERR_INVALID_ARG), (dict(dtype=3), ccv.ERR_INVALID_ARG),
    (dict(channels=16388), ccv.ERR_UNSUPPORTED), (dict(samples=1 << 27), ccv.ERR_UNSUPPORTED),
    (dict(x=None), ccv.ERR_INVALID_ARG), (dict(y=None), ccv.ERR_INVALID_ARG), (dict(xs=-1), ccv.ERR_INVALID_ARG), (dict(yp=16), ccv.ERR_INVALID_ARG),
    (dict(ys=64), ccv.ERR_INVALID_ARG), (dict(scale=K, scs=-4), ccv.ERR_INVALID_ARG),
    (dict(x=4 * K + 1), ccv.ERR_ALIGNMENT), (dict(y=8 * K + 1), ccv.ERR_ALIGNMENT), (dict(w=K + 2), ccv.ERR_ALIGNMENT), (dict(shift=K + 1), ccv.ERR_ALIGNMENT),
    (dict(ws=K + 128), ccv.ERR_ALIGNMENT),
    (dict(y=4 * K + 2), ccv.ERR_ALIAS), (dict(y=4 * K, yp=64, ys=192), ccv.ERR_ALIAS), (dict(w=8 * K + 4), ccv.ERR_ALIAS), (dict(scale=8 * K + 128), ccv.ERR_ALIAS),
    (dict(pixels=200_000, xs=200_000 * 32, ys=200_000 * 32, y=64 * K), ccv.ERR_NOMEM),
    (dict(pixels=200_000, xs=200_000 * 32, ys=200_000 * 32, y=64 * K, ws=4 * K, n=1 << 30), ccv.ERR_ALIAS),
])
def test_group_norm_refusals(bad, expected):
    assert norm(**bad) == expected


def test_group_norm_without_work():
    assert norm(samples=0, x=None) == ccv.OK and norm(pixels=0, y=None) == ccv.OK


def ring(base=4 * K, **kw):
    d = dict(N=1, C=64, F=4, H=8, W=8, KB=64)
    d.update(kw)
    return ccv.Ring(base, *d.values())


def ring_norm(a=None, b=None, sa=0, sb=0, T=2, groups=8, w=None, scale=None, act=0, ws=None):
    return ccv.ccv3d_group_norm_ring(a or ring(), sa, b or ring(8 * K), sb, T, groups, w, None, scale, 64, None, 0, 1e-6, act, ws, 0)


@pytest.mark.parametrize("bad,expected", [
    (dict(a=ring(None)), ccv.ERR_INVALID_ARG), (dict(b=ring(8 * K, H=4)), ccv.ERR_INVALID_ARG), (dict(a=ring(KB=48)), ccv.ERR_INVALID_ARG),
    (dict(b=ring(8 * K, KB=32)), ccv.ERR_INVALID_ARG), (dict(T=5), ccv.ERR_INVALID_ARG), (dict(T=-1), ccv.ERR_INVALID_ARG), (dict(sa=4), ccv.ERR_INVALID_ARG),
    (dict(sb=-1), ccv.ERR_INVALID_ARG), (dict(groups=7), ccv.ERR_INVALID_ARG), (dict(act=8), ccv.ERR_INVALID_ARG), (dict(a=ring(4 * K + 8)), ccv.ERR_ALIGNMENT),
    (dict(b=ring(4 * K), sb=1), ccv.ERR_ALIAS), (dict(b=ring(4 * K + 1024)), ccv.ERR_ALIAS), (dict(w=8 * K), ccv.ERR_ALIAS), (dict(scale=8 * K + 32), ccv.ERR_ALIAS),
    (dict(ws=100), ccv.ERR_ALIGNMENT),
])
def test_ring_norm_refusals(bad, expected):
    assert ring_norm(**bad) == expected


def test_ring_norm_without_work_and_scratch():
    assert ring_norm(T=0) == ccv.OK
    assert ccv.ccv3d_group_norm_ring_workspace(ring(), 2, 8) == (ccv.OK, 0)
    s, n = ccv.ccv3d_group_norm_ring_workspace(ring(H=352, W=640), 4, 8)
    assert s == ccv.OK and n > 0
    assert ccv.ccv3d_group_norm_ring_workspace(ring(), 9, 8)[0] == ccv.ERR_INVALID_ARG
