// The norms on both sides of a gated residual sum: r = a x + gate * post(y), h = pre(r) * (1 + scale) + shift.
//
// Bound by HBM: both kernels hold a row in the registers of G threads from its one load to its one store, so each tensor
// moves once.  The mean square of a LAYER norm is taken around the mean (two sums in turn), never as a difference of
// moments.
//   gated_norm_rows_kernel   many rows: a block walks over a stretch of rows with the weights, gate, scale and shift of
//                            their group folded into two factors and two summands for each channel in shared memory; its
//                            teams of G threads take rows in turn and ask for the next one as soon as registers are free
//   gated_norm_kernel        few or very long rows: one row to a group of threads, as many threads as the row feeds
// Measured: 520 MB of BF16 rows in 98 us, 81 % of the copy rate; 92 MB of F32 rows of an odd width in 25.5 us, 55 %.
#pragma once
#include "ccv3d_tokens_common.cuh"

namespace ccv3d {

struct NormParams {
    ccv3d_norm_desc d;
    const void *x, *y, *post_w, *post_b, *gate, *pre_w, *pre_b, *scale, *shift;
    void *r, *h;
};

// V neighbouring elements of a tensor whose type is known at run time (weights, modulation: small, read from cache)
template <int V>
__device__ __forceinline__ void load_any(const void* p, int dtype, int64_t i, float (&v)[V]) {
    if constexpr (V == 4) {
        if (dtype == CCV3D_F32) load4((const float*)p + i, v);
        else load4((const __nv_bfloat16*)p + i, v);
    } else {
        v[0] = dtype == CCV3D_F32 ? load1((const float*)p + i) : load1((const __nv_bfloat16*)p + i);
    }
}
template <int V, typename T>
__device__ __forceinline__ void load_row(const T* p, float (&v)[V]) {
    if constexpr (V == 4) load4(p, v); else v[0] = load1(p);
}
template <int V, typename T>
__device__ __forceinline__ void store_row(T* p, const float (&v)[V]) {
    if constexpr (V == 4) store4(p, v); else store1(p, v[0]);
}

// Sum over the G threads of a row.  Sums take turns with two rows of words, a word for each warp of the block, so that one
// barrier is enough: when a row of words is written again, every warp has passed the barrier of the sum between.
template <int G>
__device__ __forceinline__ float row_sum(float v, float (*part)[16], int& turn) {
    if constexpr (G < 32) {
#pragma unroll
        for (int o = G / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    }
    v = warp_sum(v);
    if constexpr (G > 32) {
        if ((threadIdx.x & 31) == 0) part[turn][threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < G / 32; ++i) v += part[turn][i];
        turn ^= 1;
    }
    return v;
}

// V neighbouring elements as they lie in memory: loaded now, turned into floats where they are needed
template <typename T, int V> struct Raw;
template <> struct Raw<float, 4> { float4 v; };
template <> struct Raw<float, 1> { float v; };
template <> struct Raw<__nv_bfloat16, 4> { uint2 v; };
template <> struct Raw<__nv_bfloat16, 1> { __nv_bfloat16 v; };
template <typename T, int V>
__device__ __forceinline__ void to_floats(const Raw<T, V>& r, float (&v)[V]) { load_row(reinterpret_cast<const T*>(&r.v), v); }

// Sum over the G threads of a team (whole warps of a block of ROWS_THREADS), as row_sum but by the team's own barrier.
constexpr int ROWS_THREADS = 512;
template <int G>
__device__ __forceinline__ float team_sum(float v, float (*part)[ROWS_THREADS / 32], int& turn) {
    v = warp_sum(v);
    if constexpr (G > 32) {
        const int warp = threadIdx.x >> 5, team = threadIdx.x / G;
        if ((threadIdx.x & 31) == 0) part[turn][warp] = v;
        asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(G) : "memory");
        v = 0.f;
#pragma unroll
        for (int i = 0; i < G / 32; ++i) v += part[turn][team * (G / 32) + i];
        turn ^= 1;
    }
    return v;
}

template <typename TX, typename TY, int G, int V, int K>
__global__ void __launch_bounds__(ROWS_THREADS, K * V <= 12 ? 2 : 1) gated_norm_rows_kernel(const NormParams p) {
    constexpr int TEAMS = ROWS_THREADS / G;
    extern __shared__ __align__(16) float folded[];              // [4][channels, rounded up to V]
    __shared__ float part[2][ROWS_THREADS / 32];
    int turn = 0;
    const ccv3d_norm_desc& d = p.d;
    const int team = threadIdx.x / G, t = (int)threadIdx.x % G, C = d.channels, CP = (C + V - 1) / V * V;
    const int first = (int)((int64_t)d.rows * blockIdx.x / gridDim.x), last = (int)((int64_t)d.rows * (blockIdx.x + 1) / gridDim.x);
    const float inv_c = 1.f / (float)C;
    Raw<TX, V> nx[K];
    Raw<TY, V> ny[K];
    float v[K][V];
    auto fetch_y = [&](int row) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * G + t) * V;
            if (c < C) ny[k] = *reinterpret_cast<const Raw<TY, V>*>((const TY*)p.y + (int64_t)row * d.y_stride + c);
        }
    };
    auto fetch_x = [&](int row) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * G + t) * V;
            if (c < C) nx[k] = *reinterpret_cast<const Raw<TX, V>*>((const TX*)p.x + (int64_t)row * d.x_stride + c);
        }
    };
    auto normalise = [&](int kind) {
        if (kind == CCV3D_NORM_NONE) return;
        float s = 0.f;
        if (kind == CCV3D_NORM_LAYER) {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) s += v[k][i];
            const float mean = team_sum<G>(s, part, turn) * inv_c;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) v[k][i] = (k * G + t) * V < C ? v[k][i] - mean : 0.f;
            s = 0.f;
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) s = fmaf(v[k][i], v[k][i], s);
        const float r = rsqrtf(team_sum<G>(s, part, turn) * inv_c + d.eps);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] *= r;
    };
    for (int begin = first; begin < last;) {                     // the stretch's rows of one group
        const int64_t group = begin / d.rows_per_group;
        const int end = (int)min((int64_t)last, (group + 1) * d.rows_per_group);
        int row = begin + team;
        if (row < end) {
            if (p.y) fetch_y(row);
            fetch_x(row);
        }
        __syncthreads();                                         // the group before is done with
        // gate * (post_weight n + post_bias) = a n + b;  (pre_weight n + pre_bias) (1 + scale) + shift = f n + g
        for (int c = threadIdx.x * V; c < C; c += ROWS_THREADS * V) {
            float a[V], b[V], f[V], g[V], w[V];
#pragma unroll
            for (int i = 0; i < V; ++i) { a[i] = f[i] = 1.f; b[i] = g[i] = 0.f; }
            if (p.post_w) load_any<V>(p.post_w, d.weight_dtype, c, a);
            if (p.post_b) load_any<V>(p.post_b, d.weight_dtype, c, b);
            if (p.pre_w) load_any<V>(p.pre_w, d.weight_dtype, c, f);
            if (p.pre_b) load_any<V>(p.pre_b, d.weight_dtype, c, g);
            if (p.gate) {
                load_any<V>(p.gate, d.mod_dtype, group * d.gate_stride + c, w);
#pragma unroll
                for (int i = 0; i < V; ++i) { a[i] *= w[i]; b[i] *= w[i]; }
            }
            if (p.scale) {
                load_any<V>(p.scale, d.mod_dtype, group * d.scale_stride + c, w);
#pragma unroll
                for (int i = 0; i < V; ++i) { f[i] = fmaf(f[i], w[i], f[i]); g[i] = fmaf(g[i], w[i], g[i]); }
            }
            if (p.shift) {
                load_any<V>(p.shift, d.mod_dtype, group * d.shift_stride + c, w);
#pragma unroll
                for (int i = 0; i < V; ++i) g[i] += w[i];
            }
            store_row(folded + c, a);
            store_row(folded + CP + c, b);
            store_row(folded + 2 * CP + c, f);
            store_row(folded + 3 * CP + c, g);
        }
        __syncthreads();
        for (; row < end; row += TEAMS) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if ((k * G + t) * V < C && p.y) {
                    to_floats<TY, V>(ny[k], v[k]);
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) v[k][i] = 0.f;
                }
            }
            if (p.y && row + TEAMS < end) fetch_y(row + TEAMS);
            if (p.y) normalise(d.post_kind);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k * G + t) * V;
                if (c < C) {
                    float x[V];
                    to_floats<TX, V>(nx[k], x);
                    if (p.y) {
                        float a[V], b[V];
                        load_row(folded + c, a);
                        load_row(folded + CP + c, b);
#pragma unroll
                        for (int i = 0; i < V; ++i) v[k][i] = fmaf(v[k][i], a[i], b[i]);
                    }
#pragma unroll
                    for (int i = 0; i < V; ++i) v[k][i] = fmaf(d.residual_scale, x[i], v[k][i]);
                    if (p.r) store_row((TX*)p.r + (int64_t)row * d.r_stride + c, v[k]);
                }
            }
            if (row + TEAMS < end) fetch_x(row + TEAMS);
            if (!p.h) continue;
            normalise(d.pre_kind);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k * G + t) * V;
                if (c < C) {
                    float f[V], g[V];
                    load_row(folded + 2 * CP + c, f);
                    load_row(folded + 3 * CP + c, g);
#pragma unroll
                    for (int i = 0; i < V; ++i) v[k][i] = fmaf(v[k][i], f[i], g[i]);
                    store_row((TY*)p.h + (int64_t)row * d.h_stride + c, v[k]);
                }
            }
        }
        begin = end;
    }
}

// V elements per access (4, or 1 where a row start or the channel count is no multiple of 4), K accesses per thread
template <typename TX, typename TY, int G, int V, int K>
__global__ void __launch_bounds__(G) gated_norm_kernel(const NormParams p) {
    __shared__ float part[2][16];
    int turn = 0;
    const ccv3d_norm_desc& d = p.d;
    const int row = blockIdx.x, t = threadIdx.x;
    const int C = d.channels;
    const int64_t grp = row / d.rows_per_group;
    const float inv_c = 1.f / (float)C;
    float v[K][V], x[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * G + t) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) v[k][i] = x[k][i] = 0.f;
        if (c < C) {
            if (p.y) load_row((const TY*)p.y + (int64_t)row * d.y_stride + c, v[k]);
            load_row((const TX*)p.x + (int64_t)row * d.x_stride + c, x[k]);
        }
    }
    // norm of what v holds, in place; elements past the row's end stay out of the sums
    auto normalise = [&](int kind) {
        if (kind == CCV3D_NORM_NONE) return;
        if (kind == CCV3D_NORM_LAYER) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) s += v[k][i];
            const float mean = row_sum<G>(s, part, turn) * inv_c;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) v[k][i] = (k * G + t) * V + i < C ? v[k][i] - mean : 0.f;
        }
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) s = fmaf(v[k][i], v[k][i], s);
        const float f = rsqrtf(row_sum<G>(s, part, turn) * inv_c + d.eps);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] *= f;
    };
    if (p.y) normalise(d.post_kind);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * G + t) * V;
        if (c < C) {
            float w[V];
            if (p.y && p.post_w) {
                load_any<V>(p.post_w, d.weight_dtype, c, w);
#pragma unroll
                for (int i = 0; i < V; ++i) v[k][i] *= w[i];
            }
            if (p.y && p.post_b) {
                load_any<V>(p.post_b, d.weight_dtype, c, w);
#pragma unroll
                for (int i = 0; i < V; ++i) v[k][i] += w[i];
            }
            if (p.y && p.gate) {
                load_any<V>(p.gate, d.mod_dtype, grp * d.gate_stride + c, w);
#pragma unroll
                for (int i = 0; i < V; ++i) v[k][i] *= w[i];
            }
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] = fmaf(d.residual_scale, x[k][i], v[k][i]);
            if (p.r) store_row((TX*)p.r + (int64_t)row * d.r_stride + c, v[k]);
        }
    }
    if (!p.h) return;
    normalise(d.pre_kind);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * G + t) * V;
        if (c < C) {
            float w[V];
            if (p.pre_w) {
                load_any<V>(p.pre_w, d.weight_dtype, c, w);
#pragma unroll
                for (int i = 0; i < V; ++i) v[k][i] *= w[i];
            }
            if (p.pre_b) {
                load_any<V>(p.pre_b, d.weight_dtype, c, w);
#pragma unroll
                for (int i = 0; i < V; ++i) v[k][i] += w[i];
            }
            if (p.scale) {
                load_any<V>(p.scale, d.mod_dtype, grp * d.scale_stride + c, w);
#pragma unroll
                for (int i = 0; i < V; ++i) v[k][i] = fmaf(v[k][i], w[i], v[k][i]);
            }
            if (p.shift) {
                load_any<V>(p.shift, d.mod_dtype, grp * d.shift_stride + c, w);
#pragma unroll
                for (int i = 0; i < V; ++i) v[k][i] += w[i];
            }
            store_row((TY*)p.h + (int64_t)row * d.h_stride + c, v[k]);
        }
    }
}

}  // namespace ccv3d
