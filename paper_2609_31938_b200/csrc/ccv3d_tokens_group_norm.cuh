// Group norm with an activation on channels-last activations (packed rows, or the blocks of a frame ring).
//
// Bound by HBM.  A thread keeps to one column of V channels (16 bytes) and walks over pixels, so that mean, factor and summand of its
// channels stay in registers.
//   group_norm_token_kernel   samples of one pixel (the heads of a token): a group lies in neighbouring lanes
//   group_norm_whole_kernel   samples that fit into the registers of a cluster of up to eight blocks are read once: mean, then the variance
//                             around it, over the cluster's shared memory
//   group_norm_stats_kernel, group_norm_fold_kernel, group_norm_apply_kernel   larger ones are read twice, the second time from L2: every
//                             thread counts mean and squared deviations of each of its channels by batches that are joined by their
//                             exact formula, never as a difference of moments; the tiles' are joined, and folded with weights and
//                             modulation into two factors for each channel, by a kernel between
// No atomics: sums have one order.
// Measured (BF16): four frames of 352 x 640 x 96 on a ring with SiLU 118 us (346 MB: 45 % of the copy rate; 14 us of statistics and 16 us of the
// norm for each frame, whose 2^x and 1 / x alone take 7.5); replayed in a graph, one of 44 x 80 x 192 9.3 us, 3520 tokens of 12 heads 6.4 us.
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
    int T, samples, pixels, C, groups, per;          // per: channels of a group
    int block_shift;                                 // channels of a block: 2^block_shift (packed rows: one block)
    int columns, lanes;                              // of a thread block: columns of V channels, pixels side by side
    float eps;
    int act;
    int vec_affine;                                  // weight, bias, scale and shift can be read four at a time
    // three-kernel form
    float2* part;                                    // [sample][tile][unit]: mean, squared deviations
    float* factors;                                  // [sample][3][C]: mean, factor, summand of each channel
    int tiles, tile_pixels, unit, first;             // unit: channels that a tile's statistics are for; first: sample of the launch's first
};

__device__ __forceinline__ int64_t sample_at(const GroupNormView& v, int s, int T) {      // (packed rows: T = samples)
    const int n = s / T, t = s - n * T;
    int f = v.slot + t;
    if (f >= v.F) f -= v.F;
    return n * v.n_stride + f * v.f_stride;
}

__device__ __forceinline__ int64_t channel_at(const GroupNormParams& p, const GroupNormView& v, int c) {
    return (c >> p.block_shift) * v.block_stride + (c & ((1 << p.block_shift) - 1));
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

// Sums over the lanes and over each `unit` channels of what the threads hold for their V channels each, n_ch of a block; `out` [n_ch / unit].
template <int V>
__device__ __forceinline__ void unit_sums(const float (&v)[V], bool live, int lanes, int lane, int col, int n_ch, int unit, float* buf, float* out) {
    if (live) {
        float* at = buf + lane * n_ch + col * V;
        if constexpr (V == 1) at[0] = v[0];
        else {
#pragma unroll
            for (int i = 0; i < V; i += 4) *reinterpret_cast<float4*>(at + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        }
    }
    __syncthreads();
    if (lanes > 1 || unit == 1) {
        float* to = unit == 1 ? out : buf;
        for (int c = threadIdx.x; c < n_ch; c += blockDim.x) {
            float s = buf[c];
#pragma unroll 8
            for (int l = 1; l < lanes; ++l) s += buf[l * n_ch + c];
            to[c] = s;
        }
        __syncthreads();
        if (unit == 1) return;
    }
    if (unit <= 32) {
        for (int u = threadIdx.x; u * unit < n_ch; u += blockDim.x) {
            float s = buf[u * unit];
            for (int c = 1; c < unit; ++c) s += buf[u * unit + c];
            out[u] = s;
        }
    } else {
        for (int u = threadIdx.x >> 5; u * unit < n_ch; u += blockDim.x >> 5) {
            float s = 0.f;
            for (int c = threadIdx.x & 31; c < unit; c += 32) s += buf[u * unit + c];
            s = warp_sum(s);
            if ((threadIdx.x & 31) == 0) out[u] = s;
        }
    }
    __syncthreads();
}

// What stands for the units of channels c .. c + V - 1.
template <int V>
__device__ __forceinline__ void of_units(const float* values, int unit, int c, float (&v)[V]) {
    int u = c / unit, r = c - u * unit;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (r == unit) { r = 0; ++u; }
        v[i] = values[u];
        ++r;
    }
}

// act((x - m) a + b) of V values.  BF16: m is zero, and -m a is in b; what that costs, 2^-24 of m a, is far under the rounding of x itself.
template <typename T, int V, typename K>
__device__ __forceinline__ void finish(float (&v)[V], const float (&m)[V], const float (&a)[V], const float (&b)[V], K) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = sizeof(T) == 4 ? fmaf(v[i] - m[i], a[i], b[i]) : fmaf(v[i], a[i], b[i]);
    activate_all<sizeof(T) == 4, K::value>(v);
}
template <typename T, int V>
__device__ __forceinline__ void fold_mean(const float (&m)[V], const float (&a)[V], float (&b)[V]) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < V; ++i) b[i] = fmaf(-m[i], a[i], b[i]);
    }
}

// Factors and summands of a thread's channels c .. c + V - 1
template <int V>
__device__ __forceinline__ void load_affine(const float* at, bool vec, float (&v)[V]) {
    if (V > 1 && vec) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 t = *reinterpret_cast<const float4*>(at + i);
            v[i] = t.x; v[i + (V > 1)] = t.y; v[i + 2 * (V > 1)] = t.z; v[i + 3 * (V > 1)] = t.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = at[i];
    }
}
template <int V>
__device__ __forceinline__ void fold_affine(const GroupNormParams& p, int s, int c, const float (&rstd)[V], float (&a)[V], float (&b)[V]) {
    float w[V];
#pragma unroll
    for (int i = 0; i < V; ++i) { a[i] = rstd[i]; b[i] = 0.f; }
    if (p.weight) {
        load_affine<V>(p.weight + c, p.vec_affine, w);
#pragma unroll
        for (int i = 0; i < V; ++i) a[i] *= w[i];
    }
    if (p.bias) load_affine<V>(p.bias + c, p.vec_affine, b);
    if (p.scale) {
        load_affine<V>(p.scale + s * p.scale_stride + c, p.vec_affine, w);
#pragma unroll
        for (int i = 0; i < V; ++i) { a[i] = fmaf(a[i], w[i], a[i]); b[i] = fmaf(b[i], w[i], b[i]); }
    }
    if (p.shift) {
        load_affine<V>(p.shift + s * p.shift_stride + c, p.vec_affine, w);
#pragma unroll
        for (int i = 0; i < V; ++i) b[i] += w[i];
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
// Sums of n values over the blocks of the cluster (eight at most), a lane to a block; f(i, sum) is called by one lane for each.
// All threads; the values are there until the next barrier of the cluster.
template <typename F>
__device__ __forceinline__ void cluster_sums(const float* values, int n, uint32_t ranks, F&& f) {
    if (ranks > 1) group_cluster_sync();
    const int r = threadIdx.x & 7, step = blockDim.x >> 3;
    for (int i = threadIdx.x >> 3; i < (n + 3) / 4 * 4; i += step) {      // (all quarters of a warp stay)
        float v = i < n && r < (int)ranks ? (ranks > 1 ? remote_float(values + i, r) : values[i]) : 0.f;
#pragma unroll
        for (int o = 4; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (r == 0 && i < n) f(i, v);
    }
    __syncthreads();
}

// Samples of one pixel whose groups are 2^k pieces wide (32 at most): a thread to a piece, a group in neighbouring lanes.  A block has
// `lanes` samples side by side (or a part of a long one, blockIdx.y), four times, all on their way at once.
constexpr int GN_TOKENS = 4;
template <typename T, int V>
__global__ void __launch_bounds__(GN_THREADS, 2) group_norm_token_kernel(const __grid_constant__ GroupNormParams p) {
    const int lane = threadIdx.x / p.columns, col = threadIdx.x - lane * p.columns, c = (blockIdx.y * p.columns + col) * V, wide = p.per / V;
    const int first = blockIdx.x * (GN_TOKENS * p.lanes) + lane;
    const int have = lane < p.lanes && c < p.C && first < p.samples ? (p.samples - first + p.lanes - 1) / p.lanes : 0;
    const T* x = (const T*)p.x + first * p.xv.f_stride + c;     // (packed rows: a sample is a frame of one pixel)
    T* y = (T*)p.y + first * p.yv.f_stride + c;
    const int64_t xs = p.lanes * p.xv.f_stride, ys = p.lanes * p.yv.f_stride;
    Piece<T, V> raw[GN_TOKENS] = {};
#pragma unroll
    for (int r = 0; r < GN_TOKENS; ++r)
        if (r < have) raw[r] = *reinterpret_cast<const Piece<T, V>*>(x + r * xs);
    float v[V], a[V], b[V], one[V];
#pragma unroll
    for (int j = 0; j < V; ++j) { one[j] = a[j] = 1.f; b[j] = 0.f; }
    const float inv = 1.f / (float)p.per;
    const bool moded = p.scale || p.shift;
    if (have && !moded) fold_affine<V>(p, 0, c, one, a, b);
    const auto group_sum = [&](float v) {
#pragma unroll
        for (int o = 1; o < 32; o *= 2)
            if (o < wide) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    };
    with_activation(p.act, [&](auto kind) {
#pragma unroll
        for (int r = 0; r < GN_TOKENS; ++r) {
            if (first - lane + r * p.lanes >= p.samples) break;          // (whole blocks)
            unpack<T, V>(raw[r], v);
            if (r < have && moded) fold_affine<V>(p, first + r * p.lanes, c, one, a, b);
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) sum += v[j];
            const float mean = group_sum(sum) * inv;
            sum = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) { v[j] -= mean; sum = fmaf(v[j], v[j], sum); }
            const float rstd = rsqrtf(fmaf(group_sum(sum), inv, p.eps));
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = fmaf(v[j] * rstd, a[j], b[j]);
            activate_all<sizeof(T) == 4, decltype(kind)::value>(v);
            if (r < have) store_piece<T, V>(y + r * ys, v);
        }
    });
}

// One sample to a cluster, R pieces to a thread.  Its columns cover all channels (columns * V = C).
template <typename T, int V, int R>
__global__ void __launch_bounds__(GN_THREADS) group_norm_whole_kernel(const __grid_constant__ GroupNormParams p) {
    extern __shared__ __align__(16) float gn_smem[];
    uint32_t rank, ranks;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    float* buf = gn_smem;                                   // [lanes][C]
    float *sum = buf + p.lanes * p.C, *dev = sum + p.groups, *mean = dev + p.groups, *rstd = mean + p.groups;
    const int s = blockIdx.x / ranks, t = threadIdx.x, lane = t / p.columns, col = t - lane * p.columns, c = col * V;
    const bool live = lane < p.lanes;
    const int p0 = (int)((int64_t)p.pixels * rank / ranks), p1 = live ? (int)((int64_t)p.pixels * (rank + 1) / ranks) : 0;
    const int64_t xs = p.lanes * p.xv.pixel_stride, ys = p.lanes * p.yv.pixel_stride;
    const T* x = (const T*)p.x + sample_at(p.xv, s, p.T) + channel_at(p, p.xv, c) + (p0 + lane) * p.xv.pixel_stride;
    T* y = (T*)p.y + sample_at(p.yv, s, p.T) + channel_at(p, p.yv, c) + (p0 + lane) * p.yv.pixel_stride;
    const int have = p0 + lane < p1 ? (p1 - p0 - lane + p.lanes - 1) / p.lanes : 0;      // pieces of this thread
    Piece<T, V> raw[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (r < have) raw[r] = *reinterpret_cast<const Piece<T, V>*>(x + r * xs);
    const float inv = 1.f / ((float)p.pixels * (float)p.per);
    float v[V], acc[V], m[V], a[V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) { acc[i] = 0.f; a[i] = 1.f; }
    if (live) fold_affine<V>(p, s, c, a, m, b);             // (m: the factors, until the deviation is known)
#pragma unroll
    for (int i = 0; i < V; ++i) a[i] = m[i];
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (r < have) {
            unpack<T, V>(raw[r], v);
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] += v[i];
        }
    unit_sums<V>(acc, live, p.lanes, lane, col, p.C, p.per, buf, sum);
    cluster_sums(sum, p.groups, ranks, [&](int g, float w) { mean[g] = w * inv; });
#pragma unroll
    for (int i = 0; i < V; ++i) { acc[i] = 0.f; m[i] = 0.f; }
    if (live) of_units<V>(mean, p.per, c, m);
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (r < have) {
            unpack<T, V>(raw[r], v);
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] = fmaf(v[i] - m[i], v[i] - m[i], acc[i]);
        }
    unit_sums<V>(acc, live, p.lanes, lane, col, p.C, p.per, buf, dev);
    cluster_sums(dev, p.groups, ranks, [&](int g, float w) { rstd[g] = rsqrtf(fmaf(w, inv, p.eps)); });
    if (ranks > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // this block has read the others' sums
    if (live) {
        of_units<V>(rstd, p.per, c, v);
#pragma unroll
        for (int i = 0; i < V; ++i) a[i] *= v[i];
        fold_mean<T>(m, a, b);
        with_activation(p.act, [&](auto kind) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (r < have) {
                    unpack<T, V>(raw[r], v);
                    finish<T>(v, m, a, b, kind);
                    store_piece<T, V>(y + r * ys, v);
                }
        });
    }
    if (ranks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");        // a block's sums are there until the others have read them
}

constexpr int GN_BIG_THREADS = 256;
constexpr int GN_BATCH = 8;      // pieces in flight of a thread

// Mean and squared deviations of the units of channels over one tile of pixels (x), one chunk of columns (y) of one sample (z).
template <typename T, int V>
__global__ void __launch_bounds__(GN_BIG_THREADS, 2) group_norm_stats_kernel(const __grid_constant__ GroupNormParams p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    extern __shared__ __align__(16) float gn_smem[];
    const int s = p.first + blockIdx.z, t = threadIdx.x, lane = t / p.columns, col = t - lane * p.columns;
    const int c0 = blockIdx.y * p.columns * V, n_ch = min(p.columns * V, p.C - c0), c = c0 + col * V;
    const bool live = lane < p.lanes && c < p.C;
    float* buf = gn_smem;                                   // [lanes][n_ch]
    float *sum = buf + p.lanes * p.columns * V, *dev = sum + p.columns * V / p.unit;
    const int p0 = (int)((int64_t)blockIdx.x * p.tile_pixels), p1 = (int)min((int64_t)p0 + p.tile_pixels, (int64_t)p.pixels);
    const T* x = (const T*)p.x + sample_at(p.xv, s, p.T) + channel_at(p, p.xv, c) + (p0 + lane) * p.xv.pixel_stride;
    const int64_t xs = p.lanes * p.xv.pixel_stride;
    int left = live && p0 + lane < p1 ? (p1 - p0 - lane + p.lanes - 1) / p.lanes : 0;      // pieces of this thread
    float mean[V], m2[V], n = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) mean[i] = m2[i] = 0.f;
    auto batch = [&](auto all) {
        const int most = decltype(all)::value ? GN_BATCH : left;
        Piece<T, V> raw[GN_BATCH];
#pragma unroll
        for (int r = 0; r < GN_BATCH; ++r)
            if (r < most) raw[r] = *reinterpret_cast<const Piece<T, V>*>(x + r * xs);
        x += GN_BATCH * xs;
        const float have = (float)most, inv = 1.f / have, total = n + have, share = __fdividef(have, total), w = n * share;
        float b[V], v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) b[i] = 0.f;
#pragma unroll
        for (int r = 0; r < GN_BATCH; ++r)
            if (r < most) {
                unpack<T, V>(raw[r], v);
#pragma unroll
                for (int i = 0; i < V; ++i) b[i] += v[i];
            }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            b[i] *= inv;
            const float d = b[i] - mean[i];
            mean[i] = fmaf(d, share, mean[i]);
            m2[i] = fmaf(d * d, w, m2[i]);
        }
#pragma unroll
        for (int r = 0; r < GN_BATCH; ++r)
            if (r < most) {
                unpack<T, V>(raw[r], v);
#pragma unroll
                for (int i = 0; i < V; ++i) m2[i] = fmaf(v[i] - b[i], v[i] - b[i], m2[i]);
            }
        n = total;
    };
#pragma unroll 1
    for (; left >= GN_BATCH; left -= GN_BATCH) batch(std::true_type());
    if (left > 0) batch(std::false_type());
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = n * mean[i];
    unit_sums<V>(v, live, p.lanes, lane, col, n_ch, p.unit, buf, sum);
    const float inv = 1.f / ((float)(p1 - p0) * (float)p.unit);
    if (live) of_units<V>(sum, p.unit, col * V, v);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float d = mean[i] - v[i] * inv;
        v[i] = n > 0.f ? fmaf(n * d, d, m2[i]) : 0.f;
    }
    unit_sums<V>(v, live, p.lanes, lane, col, n_ch, p.unit, buf, dev);
    asm volatile("griddepcontrol.wait;" ::: "memory");      // (what was here for the samples before has been used)
    float2* part = p.part + ((int64_t)blockIdx.z * p.tiles + blockIdx.x) * (p.C / p.unit) + c0 / p.unit;
    for (int u = t; u * p.unit < n_ch; u += blockDim.x) part[u] = make_float2(sum[u] * inv, dev[u]);
}

// The tiles' statistics of one group (x) of one sample (y), and the factors of its channels.
constexpr int GN_FOLD_THREADS = 256, GN_FOLD_AHEAD = 4;
__global__ void __launch_bounds__(GN_FOLD_THREADS) group_norm_fold_kernel(const __grid_constant__ GroupNormParams p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float part_sum[2][GN_FOLD_THREADS / 32];
    const int g = blockIdx.x, t = threadIdx.x, units = p.C / p.unit, mine = p.per / p.unit, items = p.tiles * mine;
    const float2* part = p.part + (int64_t)blockIdx.y * p.tiles * units + (int64_t)g * mine;
    const float full = (float)p.tile_pixels * (float)p.unit, rest = (float)(p.pixels - (p.tiles - 1) * (int64_t)p.tile_pixels) * (float)p.unit;
    const float inv = 1.f / ((float)p.pixels * (float)p.per);
    auto all = [&](float w, int turn) {
        w = warp_sum(w);
        if ((t & 31) == 0) part_sum[turn][t >> 5] = w;
        __syncthreads();
        w = 0.f;
#pragma unroll
        for (int i = 0; i < GN_FOLD_THREADS / 32; ++i) w += part_sum[turn][i];
        return w;
    };
    float w = 0.f, d = 0.f;
    float2 o[GN_FOLD_AHEAD];
    float n[GN_FOLD_AHEAD];
    auto fetch = [&](int j) {
#pragma unroll
        for (int i = 0; i < GN_FOLD_AHEAD; ++i) {
            const int item = j + i * GN_FOLD_THREADS, tile = mine == 1 ? item : item / mine;
            n[i] = item < items ? (tile + 1 == p.tiles ? rest : full) : 0.f;
            o[i] = item < items ? part[(int64_t)tile * units + (item - tile * mine)] : make_float2(0.f, 0.f);
        }
    };
    for (int j = t; j < items; j += GN_FOLD_AHEAD * GN_FOLD_THREADS) {
        fetch(j);
#pragma unroll
        for (int i = 0; i < GN_FOLD_AHEAD; ++i) w = fmaf(n[i], o[i].x, w);
    }
    w = all(w, 0) * inv;
    for (int j = t; j < items; j += GN_FOLD_AHEAD * GN_FOLD_THREADS) {
        if (items > GN_FOLD_AHEAD * GN_FOLD_THREADS) fetch(j);          // (else they are still here)
#pragma unroll
        for (int i = 0; i < GN_FOLD_AHEAD; ++i) d += n[i] > 0.f ? fmaf(n[i] * (o[i].x - w), o[i].x - w, o[i].y) : 0.f;
    }
    const float rstd[1] = {rsqrtf(fmaf(all(d, 1), inv, p.eps))};
    float* to = p.factors + (int64_t)blockIdx.y * 3 * p.C;
    for (int c = g * p.per + t; c < (g + 1) * p.per; c += GN_FOLD_THREADS) {
        float a[1], b[1];
        fold_affine<1>(p, p.first + blockIdx.y, c, rstd, a, b);
        to[c] = w;
        to[p.C + c] = a[0];
        to[2 * p.C + c] = b[0];
    }
}

// The norm itself; blocks go over a launch's samples backwards, as what was read last is still in L2.
template <typename T, int V>
__global__ void __launch_bounds__(GN_BIG_THREADS, 2) group_norm_apply_kernel(const __grid_constant__ GroupNormParams p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int z = gridDim.z - 1 - blockIdx.z, tile = gridDim.x - 1 - blockIdx.x;
    const int s = p.first + z, t = threadIdx.x, lane = t / p.columns, col = t - lane * p.columns;
    const int c = (blockIdx.y * p.columns + col) * V;
    const bool live = lane < p.lanes && c < p.C;
    const int p0 = (int)((int64_t)tile * p.tile_pixels), p1 = (int)min((int64_t)p0 + p.tile_pixels, (int64_t)p.pixels);
    const T* x = (const T*)p.x + sample_at(p.xv, s, p.T) + channel_at(p, p.xv, c) + (p0 + lane) * p.xv.pixel_stride;
    T* y = (T*)p.y + sample_at(p.yv, s, p.T) + channel_at(p, p.yv, c) + (p0 + lane) * p.yv.pixel_stride;
    const int64_t xs = p.lanes * p.xv.pixel_stride, ys = p.lanes * p.yv.pixel_stride;
    int left = live && p0 + lane < p1 ? (p1 - p0 - lane + p.lanes - 1) / p.lanes : 0;
    Piece<T, V> raw[GN_BATCH];
    auto fetch = [&]() {
#pragma unroll
        for (int r = 0; r < GN_BATCH; ++r)
            if (r < left) raw[r] = *reinterpret_cast<const Piece<T, V>*>(x + r * xs);
        x += GN_BATCH * xs;
    };
    fetch();                                                // (x was there before the statistics began)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (!live) return;
    float v[V], m[V], a[V], b[V];
    const float* from = p.factors + (int64_t)z * 3 * p.C + c;
    const bool vec = p.C % 4 == 0;
    load_affine<V>(from, vec, m);
    load_affine<V>(from + p.C, vec, a);
    load_affine<V>(from + 2 * p.C, vec, b);
    fold_mean<T>(m, a, b);
    with_activation(p.act, [&](auto kind) {
        auto one = [&](int r) {
            unpack<T, V>(raw[r], v);
            finish<T>(v, m, a, b, kind);
            store_piece<T, V>(y + r * ys, v);
        };
#pragma unroll 1
        for (; left >= GN_BATCH;) {
#pragma unroll
            for (int r = 0; r < GN_BATCH; ++r) one(r);
            left -= GN_BATCH;
            y += GN_BATCH * ys;
            fetch();
        }
#pragma unroll
        for (int r = 0; r < GN_BATCH; ++r)
            if (r < left) one(r);
    });
}

}  // namespace ccv3d
