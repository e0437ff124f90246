// Group norm with an activation on channels-last activations (packed rows, or the blocks of a frame ring).
//
// Bound by HBM.  A thread keeps to one column of V channels (16 bytes) and walks over pixels, so that mean, factor and summand of its
// channels stay in registers.  Samples that fit into the registers of a cluster of up to 16 blocks are read once
// (group_norm_whole_kernel: mean, then the variance around it, over the cluster's shared memory).  Larger ones are read twice, the second
// time mostly from L2 (group_norm_stats_kernel, group_norm_apply_kernel): every thread counts mean and squared deviations of each of its
// channels by batches that are joined by their exact formula, never as a difference of moments.  No atomics: sums have one order.
#pragma once
#include "ccv3d_tokens_activation.cuh"
#include "ccv3d_tokens_common.cuh"

namespace ccv3d {

constexpr int GN_THREADS = 512;

// where a tensor's samples, pixels and blocks of channels lie, in elements
struct GroupNormView {
    int64_t n_stride, f_stride, pixel_stride, block_stride;
    int F, slot;                 // sample n * T + t is at n * n_stride + (slot + t) mod F * f_stride
};
struct GroupNormParams {
    const void* x;
    void* y;
    const float *weight, *bias, *scale, *shift;
    int64_t scale_stride, shift_stride;
    GroupNormView xv, yv;
    int T, samples, pixels, C, groups, per, KB;      // per: channels of a group; KB: channels of a block
    int columns, lanes;                              // of a thread block: columns of V channels, pixels side by side
    float eps;
    int act;
    // two-kernel form
    float2* part;                                    // [sample][tile][chunk of columns][group]: mean, squared deviations
    int tiles, chunks, tile_pixels, first;           // first: sample of the launch's first
};

__device__ __forceinline__ int64_t sample_at(const GroupNormView& v, int s, int T) {
    const int n = s / T, t = s - n * T;
    int f = v.slot + t;
    if (f >= v.F) f -= v.F;
    return n * v.n_stride + f * v.f_stride;
}

// V elements as they lie in memory
template <typename T, int V> struct Piece;
template <> struct Piece<__nv_bfloat16, 8> { uint4 v; };
template <> struct Piece<float, 4> { float4 v; };
template <> struct Piece<__nv_bfloat16, 1> { __nv_bfloat16 v; };
template <> struct Piece<float, 1> { float v; };
template <typename T, int V>
__device__ __forceinline__ void unpack(const Piece<T, V>& p, float (&v)[V]) {
    if constexpr (V == 1) v[0] = load1(&p.v);
    else if constexpr (V == 4) { v[0] = p.v.x; v[1] = p.v.y; v[2] = p.v.z; v[3] = p.v.w; }
    else {
        const uint32_t w[4] = {p.v.x, p.v.y, p.v.z, p.v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_piece(T* at, const float (&v)[V]) {
    if constexpr (V == 1) store1(at, v[0]);
    else if constexpr (V == 4) store4(at, v);
    else *reinterpret_cast<uint4*>(at) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// Sums over the lanes and channels of each group of what the threads hold for their channels; `out` [groups of the block's columns].
// c0: first channel of the block's columns, n_ch their number, g0 .. g1: groups that have channels there.
template <int V>
__device__ __forceinline__ void group_sums(const GroupNormParams& p, const float (&v)[V], bool live, int lane, int col, int c0, int n_ch, int g0, int g1,
                                           float* buf, float* out) {
    if (live) {
#pragma unroll
        for (int i = 0; i < V; ++i) buf[lane * n_ch + col * V + i] = v[i];
    }
    __syncthreads();
    if (p.lanes > 1) {
        for (int c = threadIdx.x; c < n_ch; c += blockDim.x) {
            float s = buf[c];
            for (int l = 1; l < p.lanes; ++l) s += buf[l * n_ch + c];
            buf[c] = s;
        }
        __syncthreads();
    }
    for (int g = g0 + (threadIdx.x >> 5); g < g1; g += blockDim.x >> 5) {
        const int lo = max(g * p.per, c0), hi = min((g + 1) * p.per, c0 + n_ch);
        float s = 0.f;
        for (int c = lo + (threadIdx.x & 31); c < hi; c += 32) s += buf[c - c0];
        s = warp_sum(s);
        if ((threadIdx.x & 31) == 0) out[g - g0] = s;
    }
    __syncthreads();
}

// y = act((x - mean) * a + b): a thread's channels c .. c + V - 1
template <int V>
__device__ __forceinline__ void fold_affine(const GroupNormParams& p, int s, int c, const float (&rstd)[V], float (&a)[V], float (&b)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        a[i] = p.weight ? rstd[i] * __ldg(p.weight + c + i) : rstd[i];
        b[i] = p.bias ? __ldg(p.bias + c + i) : 0.f;
        if (p.scale) {
            const float f = __ldg(p.scale + s * p.scale_stride + c + i);
            a[i] = fmaf(a[i], f, a[i]);
            b[i] = fmaf(b[i], f, b[i]);
        }
        if (p.shift) b[i] += __ldg(p.shift + s * p.shift_stride + c + i);
    }
}

__device__ __forceinline__ float remote_float(const float* p, uint32_t rank) {
    uint32_t a;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void group_cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// One sample to a cluster, R pieces to a thread.  Its columns cover all channels (columns * V = C).
template <typename T, int V, int R>
__global__ void __launch_bounds__(GN_THREADS) group_norm_whole_kernel(const __grid_constant__ GroupNormParams p) {
    extern __shared__ float gn_smem[];
    uint32_t rank, ranks;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    float* buf = gn_smem;                                   // [lanes][C]
    float *sum = buf + p.lanes * p.C, *dev = sum + p.groups, *mean = dev + p.groups, *rstd = mean + p.groups;
    const int s = blockIdx.x / ranks, t = threadIdx.x, lane = t / p.columns, col = t - lane * p.columns, c = col * V;
    const bool live = lane < p.lanes;
    const int p0 = (int)((int64_t)p.pixels * rank / ranks), p1 = (int)((int64_t)p.pixels * (rank + 1) / ranks);
    const T* x = (const T*)p.x + sample_at(p.xv, s, p.T) + c / p.KB * p.xv.block_stride + c % p.KB;
    T* y = (T*)p.y + sample_at(p.yv, s, p.T) + c / p.KB * p.yv.block_stride + c % p.KB;
    Piece<T, V> raw[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int px = p0 + lane + r * p.lanes;
        if (live && px < p1) raw[r] = *reinterpret_cast<const Piece<T, V>*>(x + px * p.xv.pixel_stride);
    }
    const float inv = 1.f / ((float)p.pixels * (float)p.per);
    float v[V], acc[V], m[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (live && p0 + lane + r * p.lanes < p1) {
            unpack<T, V>(raw[r], v);
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] += v[i];
        }
    group_sums<V>(p, acc, live, lane, col, 0, p.C, 0, p.groups, buf, sum);
    if (ranks > 1) group_cluster_sync();
    for (int g = t; g < p.groups; g += blockDim.x) {
        float w = 0.f;
        if (ranks > 1) for (uint32_t k = 0; k < ranks; ++k) w += remote_float(sum + g, k);
        else w = sum[g];
        mean[g] = w * inv;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) { acc[i] = 0.f; m[i] = live ? mean[(c + i) / p.per] : 0.f; }
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (live && p0 + lane + r * p.lanes < p1) {
            unpack<T, V>(raw[r], v);
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] = fmaf(v[i] - m[i], v[i] - m[i], acc[i]);
        }
    group_sums<V>(p, acc, live, lane, col, 0, p.C, 0, p.groups, buf, dev);
    if (ranks > 1) group_cluster_sync();
    for (int g = t; g < p.groups; g += blockDim.x) {
        float w = 0.f;
        if (ranks > 1) for (uint32_t k = 0; k < ranks; ++k) w += remote_float(dev + g, k);
        else w = dev[g];
        rstd[g] = rsqrtf(fmaf(w, inv, p.eps));
    }
    __syncthreads();
    if (live) {
        float a[V], b[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = rstd[(c + i) / p.per];
        fold_affine<V>(p, s, c, v, a, b);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int px = p0 + lane + r * p.lanes;
            if (px < p1) {
                unpack<T, V>(raw[r], v);
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = activate<sizeof(T) == 4>(fmaf(v[i] - m[i], a[i], b[i]), p.act);
                store_piece<T, V>(y + px * p.yv.pixel_stride, v);
            }
        }
    }
    if (ranks > 1) group_cluster_sync();                    // a block's sums are there until the others have read them
}

constexpr int GN_BATCH = 8;      // pieces in flight of a thread

// Mean and squared deviations of the groups over one tile of pixels (x), one chunk of columns (y) of one sample (z).
template <typename T, int V>
__global__ void __launch_bounds__(GN_THREADS, 2) group_norm_stats_kernel(const __grid_constant__ GroupNormParams p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    extern __shared__ float gn_smem[];
    const int s = p.first + blockIdx.z, t = threadIdx.x, lane = t / p.columns, col = t - lane * p.columns;
    const int c0 = blockIdx.y * p.columns * V, n_ch = min(p.columns * V, p.C - c0), c = c0 + col * V;
    const bool live = lane < p.lanes && c < p.C;
    const int g0 = c0 / p.per, g1 = (c0 + n_ch - 1) / p.per + 1;
    float* buf = gn_smem;                                   // [lanes][n_ch]
    float *sum = buf + p.lanes * p.columns * V, *dev = sum + (g1 - g0);
    const int p0 = (int)min((int64_t)blockIdx.x * p.tile_pixels, (int64_t)p.pixels), p1 = (int)min((int64_t)p0 + p.tile_pixels, (int64_t)p.pixels);
    const T* x = (const T*)p.x + sample_at(p.xv, s, p.T) + c / p.KB * p.xv.block_stride + c % p.KB;
    float mean[V], m2[V], n = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) mean[i] = m2[i] = 0.f;
    const int step = GN_BATCH * p.lanes;
    if (live) {
        for (int px = p0 + lane; px < p1; px += step) {
            Piece<T, V> raw[GN_BATCH];
#pragma unroll
            for (int r = 0; r < GN_BATCH; ++r)
                if (px + r * p.lanes < p1) raw[r] = *reinterpret_cast<const Piece<T, V>*>(x + (px + r * p.lanes) * p.xv.pixel_stride);
            const int have = min(GN_BATCH, (p1 - px + p.lanes - 1) / p.lanes);
            float b[V], v[V], q[V];
            const float inv = 1.f / (float)have;
#pragma unroll
            for (int i = 0; i < V; ++i) b[i] = q[i] = 0.f;
#pragma unroll
            for (int r = 0; r < GN_BATCH; ++r)
                if (r < have) {
                    unpack<T, V>(raw[r], v);
#pragma unroll
                    for (int i = 0; i < V; ++i) b[i] += v[i];
                }
#pragma unroll
            for (int i = 0; i < V; ++i) b[i] *= inv;
#pragma unroll
            for (int r = 0; r < GN_BATCH; ++r)
                if (r < have) {
                    unpack<T, V>(raw[r], v);
#pragma unroll
                    for (int i = 0; i < V; ++i) q[i] = fmaf(v[i] - b[i], v[i] - b[i], q[i]);
                }
            const float total = n + (float)have, share = (float)have / total, w = n * share;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = b[i] - mean[i];
                mean[i] = fmaf(d, share, mean[i]);
                m2[i] += fmaf(d * d, w, q[i]);
            }
            n = total;
        }
    }
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = n * mean[i];
    group_sums<V>(p, v, live, lane, col, c0, n_ch, g0, g1, buf, sum);
    for (int g = g0 + t; g < g1; g += blockDim.x) {
        const int ch = min((g + 1) * p.per, c0 + n_ch) - max(g * p.per, c0);
        sum[g - g0] /= (float)(p1 - p0) * (float)ch;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float d = live ? mean[i] - sum[(c + i) / p.per - g0] : 0.f;
        v[i] = n > 0.f ? fmaf(n * d, d, m2[i]) : 0.f;
    }
    group_sums<V>(p, v, live, lane, col, c0, n_ch, g0, g1, buf, dev);
    float2* part = p.part + ((int64_t)(blockIdx.z * p.tiles + blockIdx.x) * p.chunks + blockIdx.y) * p.groups;
    for (int g = g0 + t; g < g1; g += blockDim.x) part[g] = make_float2(sum[g - g0], dev[g - g0]);
}

// The norm itself, from the tiles' means and deviations; blocks go over the samples backwards, as what was read last is still in L2.
template <typename T, int V>
__global__ void __launch_bounds__(GN_THREADS, 2) group_norm_apply_kernel(const __grid_constant__ GroupNormParams p) {
    extern __shared__ float gn_smem[];
    const int z = gridDim.z - 1 - blockIdx.z, tile = gridDim.x - 1 - blockIdx.x;
    const int s = p.first + z, t = threadIdx.x, lane = t / p.columns, col = t - lane * p.columns;
    const int c0 = blockIdx.y * p.columns * V, n_ch = min(p.columns * V, p.C - c0), c = c0 + col * V;
    const bool live = lane < p.lanes && c < p.C;
    const int g0 = c0 / p.per, g1 = (c0 + n_ch - 1) / p.per + 1;
    float *mean = gn_smem, *rstd = mean + (g1 - g0);
    const int p0 = (int)min((int64_t)tile * p.tile_pixels, (int64_t)p.pixels), p1 = (int)min((int64_t)p0 + p.tile_pixels, (int64_t)p.pixels);
    const T* x = (const T*)p.x + sample_at(p.xv, s, p.T) + c / p.KB * p.xv.block_stride + c % p.KB;
    T* y = (T*)p.y + sample_at(p.yv, s, p.T) + c / p.KB * p.yv.block_stride + c % p.KB;
    Piece<T, V> raw[GN_BATCH];
    const int step = GN_BATCH * p.lanes;
    auto fetch = [&](int px) {
#pragma unroll
        for (int r = 0; r < GN_BATCH; ++r)
            if (live && px + r * p.lanes < p1) raw[r] = *reinterpret_cast<const Piece<T, V>*>(x + (px + r * p.lanes) * p.xv.pixel_stride);
    };
    fetch(p0 + lane);                                       // (x was there before the statistics began)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const float inv = 1.f / ((float)p.pixels * (float)p.per);
    for (int g = g0 + (t >> 5); g < g1; g += blockDim.x >> 5) {
        const float2* part = p.part + (int64_t)z * p.tiles * p.chunks * p.groups + g;
        // chunks that have channels of the group
        const int k0 = g * p.per / (p.columns * V), k1 = ((g + 1) * p.per - 1) / (p.columns * V) + 1, n_k = k1 - k0;
        float w = 0.f, d = 0.f;
        auto count = [&](int i, int k) {
            const int px = min(p.tile_pixels, p.pixels - i * p.tile_pixels);
            return (float)px * (float)(min((g + 1) * p.per, (k + 1) * p.columns * V) - max(g * p.per, k * p.columns * V));
        };
        for (int j = t & 31; j < p.tiles * n_k; j += 32) {
            const int i = j / n_k, k = k0 + j - i * n_k;
            w = fmaf(count(i, k), part[((int64_t)i * p.chunks + k) * p.groups].x, w);
        }
        w = warp_sum(w) * inv;
        for (int j = t & 31; j < p.tiles * n_k; j += 32) {
            const int i = j / n_k, k = k0 + j - i * n_k;
            const float2 o = part[((int64_t)i * p.chunks + k) * p.groups];
            d += fmaf(count(i, k) * (o.x - w), o.x - w, o.y);
        }
        d = warp_sum(d);
        if ((t & 31) == 0) { mean[g - g0] = w; rstd[g - g0] = rsqrtf(fmaf(d, inv, p.eps)); }
    }
    __syncthreads();
    if (!live) return;
    float v[V], m[V], a[V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) { m[i] = mean[(c + i) / p.per - g0]; v[i] = rstd[(c + i) / p.per - g0]; }
    fold_affine<V>(p, s, c, v, a, b);
    for (int px = p0 + lane; px < p1; px += step) {
        if (px > p0 + lane) fetch(px);
#pragma unroll
        for (int r = 0; r < GN_BATCH; ++r) {
            if (px + r * p.lanes < p1) {
                unpack<T, V>(raw[r], v);
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = activate<sizeof(T) == 4>(fmaf(v[i] - m[i], a[i], b[i]), p.act);
                store_piece<T, V>(y + (px + r * p.lanes) * p.yv.pixel_stride, v);
            }
        }
    }
}

}  // namespace ccv3d
