// The norms on both sides of a gated residual sum: r = a x + gate * post(y), h = pre(r) * (1 + scale) + shift.
//
// A group of G threads holds one row in registers from its one load to its one store, so the kernel moves each tensor
// once; the mean square of a LAYER norm is taken around the mean (two sums in turn), never as a difference of moments.
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

// Sum over the G threads of a row; `part` holds a word for each warp of the block.  All threads of the block call it.
template <int G>
__device__ __forceinline__ float row_sum(float v, float* part) {
    if constexpr (G < 32) {
#pragma unroll
        for (int o = G / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    }
    v = warp_sum(v);
    if constexpr (G > 32) {
    const int warp = threadIdx.x >> 5;
    __syncthreads();                            // the words of the sum before have been read
    if ((threadIdx.x & 31) == 0) part[warp] = v;
    __syncthreads();
    constexpr int W = G / 32;
    const int w0 = warp / W * W;
    v = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) v += part[w0 + i];
    }
    return v;
}

// V elements per access (4, or 1 where a row start or the channel count is no multiple of 4), K accesses per thread
template <typename TX, typename TY, int G, int V, int K>
__global__ void __launch_bounds__(G < 128 ? 128 : G) gated_norm_kernel(const NormParams p) {
    constexpr int NT = G < 128 ? 128 : G;
    __shared__ float part[NT / 32];
    const ccv3d_norm_desc& d = p.d;
    const int row = blockIdx.x * (NT / G) + (int)threadIdx.x / G, t = (int)threadIdx.x % G;
    const bool live = row < d.rows;
    const int C = d.channels;
    const int64_t grp = live ? row / d.rows_per_group : 0;
    const float inv_c = 1.f / (float)C;
    float v[K][V], x[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * G + t) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) v[k][i] = x[k][i] = 0.f;
        if (live && c < C) {
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
            const float mean = row_sum<G>(s, part) * inv_c;
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
        const float f = rsqrtf(row_sum<G>(s, part) * inv_c + d.eps);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] *= f;
    };
    if (p.y) normalise(d.post_kind);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * G + t) * V;
        if (live && c < C) {
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
        if (live && c < C) {
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
