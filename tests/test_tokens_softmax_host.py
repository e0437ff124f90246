"""The arithmetic of the attention kernels' running base (ccv3d_tokens_softmax.cuh) on the host: the passes over half a tile
end, no weight leaves the range of halves and no row loses all its weights, whatever the size of the scores.

`passes` below is the loop of the tile kernel on a warp of 32 rows without its bound of two passes, `step` that of the step
kernel; both use the header's functions and FP32 operations in the kernels' order.  Bounds, derived before the first run: a score v is a product and an
addend in one rounding, the base another float, so what the weights stand for is off by at most four spacings of floats at
the largest magnitude met; the sum of 64 weights adds 2^-17 of itself, and log2 of it 2^-23 of the result.
"""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include <algorithm>
#include "ccv3d_tokens_softmax.cuh"
using namespace ccv3d;
// One pass over a half tile of a warp; true if some row asks for another.
struct Warp { float m[32]; double l[32]; bool far; };
static bool pass(const Warp& w, bool rounded, const float* s, const float* f, const float* e, float (&mx)[32], float (&out)[32][64], bool (&raise)[32]) {
    bool need = false;
    for (int r = 0; r < 32; ++r) {
        const float base = base_or_start(w.m[r]);
        mx[r] = -INFINITY;
        for (int i = 0; i < 64; ++i) {
            const float k = e[i / 16], x = fmaf(s[r * 64 + i], f[r], rounded ? k : k - base);
            mx[r] = fmaxf(mx[r], x);
            out[r][i] = rounded ? x - base : x;
        }
        raise[r] = rounded ? mx[r] > base_limit(w.m[r]) : mx[r] > WEIGHT_TOP || (w.m[r] == -INFINITY && mx[r] > -INFINITY);
        need = need || raise[r];
    }
    return need;
}
// scores [tiles][32 rows][64 tokens] with a factor for each row and an addend (log2 of a value scale) for each 16 tokens of a tile;
// `edge`: the code for tiles that rows see in part from the start.  Returns the most passes of one code over any half tile; base
// and sum of each row, the largest exponent that went out.
extern "C" int passes(const float* s, const float* f, const float* e, int tiles, int edge, float* base_out, double* sum_out, float* top) {
    Warp w;
    int worst = 0;
    w.far = edge;
    *top = -INFINITY;
    for (int r = 0; r < 32; ++r) { w.m[r] = -INFINITY; w.l[r] = 0; }
    for (int t = 0; t < tiles; ++t) {
        float mx[32], out[32][64];
        bool raise[32], done = false;
        for (int rounded = w.far; rounded < 2 && !done; ++rounded)
            for (int n = 1;; ++n) {
                const bool need = pass(w, rounded, s + t * 2048, f, e + 4 * t, mx, out, raise);
                worst = std::max(worst, n);
                done = !need;
                if (done || n > 10) break;
                float now[32];
                bool far = false;
                for (int r = 0; r < 32; ++r) {
                    now[r] = fmaxf(w.m[r], base_for(rounded ? mx[r] : mx[r] + base_or_start(w.m[r])));
                    far = far || (raise[r] && !(fabsf(now[r]) <= SCORE_EXACT));
                }
                if (far) w.far = true;
                if (far && !rounded) break;
                for (int r = 0; r < 32; ++r) {
                    w.l[r] *= w.m[r] == -INFINITY ? 0. : exp2((double)w.m[r] - now[r]);
                    w.m[r] = now[r];
                }
            }
        for (int r = 0; r < 32; ++r)
            for (int i = 0; i < 64; ++i) {
                *top = fmaxf(*top, out[r][i]);
                w.l[r] += exp2((double)out[r][i]) * exp2(-(double)e[4 * t + i / 16]);
            }
    }
    for (int r = 0; r < 32; ++r) { base_out[r] = w.m[r]; sum_out[r] = w.l[r]; }
    return worst;
}
extern "C" void step(const float* s, const float* f, const float* e, int tiles, float* base_out, double* sum_out, float* top) {
    *top = -INFINITY;
    for (int r = 0; r < 32; ++r) {
        float m = -INFINITY;
        double l = 0;
        for (int t = 0; t < tiles; ++t) {
            float v[64], mx = -INFINITY;
            for (int i = 0; i < 64; ++i) {
                v[i] = fmaf(s[(t * 32 + r) * 64 + i], f[r], e[4 * t + i / 16]);
                mx = fmaxf(mx, v[i]);
            }
            if (mx > base_limit(m)) {
                const float now = fmaxf(m, base_for(mx));
                l *= m == -INFINITY ? 0. : exp2((double)m - now);
                m = now;
            }
            for (int i = 0; i < 64; ++i) {
                const float x = v[i] - base_or_start(m);
                *top = fmaxf(*top, x);
                l += exp2((double)x) * exp2(-(double)e[4 * t + i / 16]);
            }
        }
        base_out[r] = m;
        sum_out[r] = l;
    }
}
extern "C" float limit_of(float m) { return base_limit(base_for(m)); }
extern "C" float start_of(float m) { return base_for(m); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("softmax")
    (d / "e.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-fPIC", "-shared", "-I", os.path.join(ROOT, "paper_2609_31938_b200", "csrc"),
                    "-o", str(d / "e.so"), str(d / "e.cpp")], check=True)
    lib = ctypes.CDLL(str(d / "e.so"))
    lib.limit_of.restype = lib.start_of.restype = ctypes.c_float
    lib.limit_of.argtypes = lib.start_of.argtypes = [ctypes.c_float]
    return lib


def ptr(a):
    return a.ctypes.data_as(ctypes.c_void_p)


def run(lib, s, f, e, kernel):
    base, total, top = np.zeros(32, np.float32), np.zeros(32), ctypes.c_float()
    passes = 1
    if kernel != "step":
        passes = lib.passes(ptr(s), ptr(f), ptr(e), len(s), int(kernel == "edge"), ptr(base), ptr(total), ctypes.byref(top))
    else:
        lib.step(ptr(s), ptr(f), ptr(e), len(s), ptr(base), ptr(total), ctypes.byref(top))
    return passes, base.astype(np.float64), total, top.value


SIZES = [1.0, 1e3, 1e6, 3e6, 8e6, 3e7, 6e7, 1e8, 2e8, 1e9, 1e10, 1e15, 1e25, 1e37]


@pytest.mark.parametrize("kernel", ["tile", "edge", "step"])
@pytest.mark.parametrize("kind", ["random", "rising", "falling", "negative", "one row", "scales"])
@pytest.mark.parametrize("size", SIZES)
def test_scores_of_any_size(lib, size, kind, kernel):
    rng = np.random.default_rng(int(np.log10(size) * 10) + len(kind))
    for _ in range(20):
        tiles = 4
        x = rng.standard_normal((tiles, 32, 64))
        if kind == "rising":
            x = x * np.array([1e-6, 1e-3, 0.1, 1.0])[:, None, None]
        elif kind == "falling":
            x = x * np.array([1.0, 0.1, 1e-3, 1e-6])[:, None, None]
        elif kind == "negative":
            x = -np.abs(x) - 1
        f = (size * np.exp2(rng.uniform(-1, 1, 32) - 10)).astype(np.float32)
        if kind == "one row":
            f[1:] = rng.uniform(0.001, 0.01, 31)
        e = (rng.integers(-64, 121, 4 * tiles) if kind == "scales" else np.zeros(4 * tiles)).astype(np.float32)
        s = (x * 1024).astype(np.float32)
        passes, base, total, top = run(lib, s, f, e, kernel)
        assert passes <= 2
        assert top <= 15.0                               # 2^15: the halves' largest is 65504
        assert (total > 0).all() and np.isfinite(total).all()
        v = s.astype(np.float64) * f.astype(np.float64)[None, :, None]
        most = v.max((0, 2))
        want = most + np.log2(np.exp2(v - most[None, :, None]).sum((0, 2)))
        got = base + np.log2(total)
        if kind == "scales":                             # (a row's weight may all lie in pages of a scale too small to hold it)
            continue
        spacing = np.spacing(np.abs(v).max((0, 2)).astype(np.float32)).astype(np.float64)
        assert (np.abs(got - want) <= 4 * spacing + 2.0 ** -16 + 2.0 ** -23 * np.abs(want)).all()


def test_limits_hold_at_every_size(lib):
    """2^(v - base) is at most 2^15 for the largest v that a base bears, the base's own score included."""
    rng = np.random.default_rng(0)
    sizes = np.exp2(rng.uniform(-3, 127, 20000)).astype(np.float32)
    edges = np.float32([0.0, 2.0 ** 22 - 1, 2.0 ** 22, 2.0 ** 22 + 1, 2.0 ** 22 + 8, 2.0 ** 23 - 8, 2.0 ** 23, 2.0 ** 24 - 1, 2.0 ** 24, 2.0 ** 27])
    for v in np.concatenate([sizes, -sizes, edges, -edges]):
        base, limit = np.float32(lib.start_of(v)), np.float32(lib.limit_of(v))
        assert np.float32(limit) >= v and np.float32(limit) - base <= 15.0 and v - base <= 8.0
        above = np.nextafter(limit, np.float32(np.inf))
        assert above > limit                             # the next score moves the base
    assert lib.start_of(-np.inf) == -np.inf and lib.limit_of(-np.inf) == -np.inf


@pytest.mark.parametrize("kernel", ["tile", "edge", "step"])
def test_infinite_scores_end(lib, kernel):
    for values in ([np.inf], [-np.inf], [np.inf, -np.inf], [np.nan], [np.inf, np.nan, 1e30], [3e38, -3e38]):
        s = np.zeros((3, 32, 64), np.float32)
        for i, v in enumerate(values):
            s[1, ::2, i::7] = v
        for factor in (1.0, 1e30):
            passes, base, total, _ = run(lib, s, np.full(32, factor, np.float32), np.zeros(12, np.float32), kernel)
            assert passes <= 2
            with np.errstate(over="ignore", invalid="ignore"):
                v = s * np.float32(factor)
            bad = np.isnan(v).any((0, 2)) | (v == np.inf).any((0, 2))
            assert np.array_equal(~np.isfinite(total), bad)
            good = v[:, ~bad].astype(np.float64)
            most = good.max((0, 2))
            want = most + np.log2(np.exp2(good - most[None, :, None]).sum((0, 2)))
            assert (np.abs(base[~bad] + np.log2(total[~bad]) - want) <= 2.0 ** -16 + 2.0 ** -22 * np.abs(want)).all()
