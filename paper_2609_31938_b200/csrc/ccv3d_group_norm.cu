// C entry points of the group norms: argument checks, kernel choice, launches.
#include "ccv3d_tokens_group_norm.cuh"
#include "ccv3d_tokens_host.cuh"

using namespace ccv3d;

namespace {

constexpr int GN_SMEM = 100 * 1024;
constexpr int GN_PIECES = 8;             // most pieces of a thread in the one-pass form

// How a call is cut up.  It goes by the sample's size and type alone, not by how many samples there are (but for how many go at once), so that
// a stream of frames has the same bits however it is cut into calls; nor by the device, whose 148 SMs and L2 stand here as numbers.
struct GnPlan {
    bool vec, token, whole;
    int V, columns, lanes, chunks;       // chunks: of columns (token and three-kernel forms)
    int cluster, pieces;                 // one-pass form
    int tile_pixels, tiles, unit, at_once;   // three-kernel form: pixels of a block, channels of a unit, samples of a turn of launches
    uint64_t factors_at;
    uint64_t bytes;
};

GnPlan gn_plan(int64_t samples, int64_t pixels, int C, int groups, int dtype, bool vec, bool ring = false) {
    GnPlan q = {};
    q.vec = vec;
    q.V = vec ? 16 / (int)esize(dtype) : 1;
    const int VC = C / q.V, wide = C / groups / q.V;
    if (pixels == 1 && !ring && C / groups % q.V == 0 && wide <= 32 && (wide & (wide - 1)) == 0) {
        // (a block's columns are whole groups)
        q.token = true;
        q.columns = VC < GN_THREADS ? VC : GN_THREADS / wide * wide;
        q.chunks = (VC + q.columns - 1) / q.columns;
        q.lanes = q.columns < 256 ? 256 / q.columns : 1;
        return q;
    }
    if (VC <= GN_THREADS) {
        // the fewest blocks that leave a thread four pieces at most, eight blocks where that takes more
        const int lanes = GN_THREADS / VC;
        for (q.cluster = 1; q.cluster < 8 && pixels > (int64_t)4 * q.cluster * lanes; q.cluster *= 2) {}
        const int64_t share = (pixels + q.cluster - 1) / q.cluster;
        q.lanes = (int)(share < lanes ? share : lanes);
        const int64_t pieces = (share + q.lanes - 1) / q.lanes;
        if (pieces <= GN_PIECES) {
            q.whole = true;
            q.columns = VC;
            q.chunks = 1;
            for (q.pieces = 1; q.pieces < pieces; q.pieces *= 2) {}
            return q;
        }
    }
    q.columns = VC < GN_BIG_THREADS ? VC : GN_BIG_THREADS;
    q.chunks = (VC + q.columns - 1) / q.columns;
    q.lanes = GN_BIG_THREADS / q.columns;
    // A block to each half of an SM, or as many as have sixteen pieces for a thread.  (Four frames of 43 MB, us: 296 blocks 117, 576 136, 1152 140;
    // three samples of 5 MB, with pieces for a thread: 8 20, 16 17, 24 19.)
    const int64_t blocks = 296 / q.chunks > 1 ? 296 / q.chunks : 1, share = (pixels + blocks - 1) / blocks, least = (int64_t)q.lanes * 16;
    q.tile_pixels = (int)(share > least ? share : least);
    q.tiles = (int)((pixels + q.tile_pixels - 1) / q.tile_pixels);
    // statistics go by whole groups, or by what divides groups and chunks of columns
    q.unit = C / groups;
    if (q.chunks > 1)
        for (int a = q.unit, b = q.columns * q.V; b; q.unit = a) { const int r = a % b; a = b; b = r; }
    const int64_t size = pixels * C * esize(dtype), fit = (48ll << 20) / size;      // what is read again shall still be in L2
    const int64_t most = 65535;
    q.at_once = (int)(fit < 1 ? 1 : fit < samples ? (fit < most ? fit : most) : (samples < most ? samples : most));
    q.factors_at = ((uint64_t)q.at_once * q.tiles * (C / q.unit) * sizeof(float2) + 255) / 256 * 256;
    q.bytes = q.factors_at + ((uint64_t)q.at_once * 3 * C * sizeof(float) + 255) / 256 * 256;
    return q;
}

template <typename T, int V, int R>
ccv3d_status launch_whole(GroupNormParams& p, const GnPlan& q, const Device& dev, cudaStream_t st) {
    static std::atomic<uint64_t> done{0};
    auto* kernel = group_norm_whole_kernel<T, V, R>;
    if (!allow_smem(kernel, GN_SMEM, dev.index, done)) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = q.cluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.samples * q.cluster);
    cfg.blockDim = dim3((q.columns * q.lanes + 31) / 32 * 32);
    cfg.dynamicSmemBytes = (size_t)(q.lanes * p.C + 4 * p.groups) * 4;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, p) != cudaSuccess) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    return CCV3D_OK;
}

template <typename T, int V>
ccv3d_status launch_group_norm(GroupNormParams& p, const GnPlan& q, void* ws, const Device& dev, cudaStream_t st) {
    if (q.token) {
        const int per = GN_TOKENS * q.lanes;
        group_norm_token_kernel<T, V><<<dim3((p.samples + per - 1) / per, q.chunks), (q.columns * q.lanes + 31) / 32 * 32, 0, st>>>(p);
        return launched();
    }
    if (q.whole) {
        if (q.pieces == 1) return launch_whole<T, V, 1>(p, q, dev, st);
        if (q.pieces == 2) return launch_whole<T, V, 2>(p, q, dev, st);
        if (q.pieces == 4) return launch_whole<T, V, 4>(p, q, dev, st);
        return launch_whole<T, V, 8>(p, q, dev, st);
    }
    p.part = (float2*)ws;
    p.factors = (float*)((char*)ws + q.factors_at);
    p.tiles = q.tiles;
    p.tile_pixels = q.tile_pixels;
    p.unit = q.unit;
    // each kernel is resident when the one before it ends; the first of a turn reads while the last turn's outputs go out
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    for (int first = 0; first < p.samples; first += q.at_once) {
        p.first = first;
        const int now = min(q.at_once, p.samples - first);
        cudaLaunchConfig_t cfg = {};
        cfg.stream = st;
        cfg.attrs = at;
        cfg.numAttrs = first ? 1 : 0;
        cfg.gridDim = dim3(q.tiles, q.chunks, now);
        cfg.blockDim = dim3((q.columns * q.lanes + 31) / 32 * 32);
        cfg.dynamicSmemBytes = (size_t)(q.lanes * q.columns * V + 2 * (q.columns * V / q.unit)) * 4;
        if (cudaLaunchKernelEx(&cfg, group_norm_stats_kernel<T, V>, p) != cudaSuccess) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
        cfg.dynamicSmemBytes = 0;
        cfg.numAttrs = 1;
        const dim3 tiles = cfg.gridDim, threads = cfg.blockDim;
        cfg.gridDim = dim3(p.groups, now);
        cfg.blockDim = dim3(GN_FOLD_THREADS);
        if (cudaLaunchKernelEx(&cfg, group_norm_fold_kernel, p) != cudaSuccess) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
        cfg.gridDim = tiles;
        cfg.blockDim = threads;
        if (cudaLaunchKernelEx(&cfg, group_norm_apply_kernel<T, V>, p) != cudaSuccess) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    }
    return CCV3D_OK;
}

ccv3d_status run_group_norm(GroupNormParams& p, const GnPlan& q, int dtype, void* ws, cudaStream_t st) {
    Device dev;
    const ccv3d_status s = current_device(&dev);
    if (s != CCV3D_OK) return s;
    if (dtype == CCV3D_BF16) return q.vec ? launch_group_norm<__nv_bfloat16, 8>(p, q, ws, dev, st) : launch_group_norm<__nv_bfloat16, 1>(p, q, ws, dev, st);
    return q.vec ? launch_group_norm<float, 4>(p, q, ws, dev, st) : launch_group_norm<float, 1>(p, q, ws, dev, st);
}

// Sizes and kinds that do not need tensors.
ccv3d_status check_group_norm(int64_t samples, int64_t pixels, int channels, int groups, int activation, int dtype) {
    if (samples < 0 || pixels < 0 || channels < 1 || groups < 1 || channels % groups || !dtype_ok(dtype)) return CCV3D_ERR_INVALID_ARG;
    if (activation < CCV3D_ACT_NONE || activation > CCV3D_ACT_GELU_TANH) return CCV3D_ERR_INVALID_ARG;
    if (channels > 16384 || samples > (1 << 26) || pixels > (1 << 30)) return CCV3D_ERR_UNSUPPORTED;
    return CCV3D_OK;
}

// Whether a tensor [samples, pixels, channels] writes no element twice.
bool apart(int64_t samples, int64_t pixels, int64_t C, int64_t ss, int64_t ps) {
    if (pixels > 1 && samples > 1)
        return (ps >= C && ss >= (pixels - 1) * ps + C) || (ss >= C && ps >= (samples - 1) * ss + C);
    return (pixels <= 1 || ps >= C) && (samples <= 1 || ss >= C);
}

bool whole_vectors(const void* p, int dtype, int64_t a, int64_t b) {
    const int64_t V = 16 / esize(dtype);
    return !misaligned(p, 16) && a % V == 0 && b % V == 0;
}

bool affine_vectors(const GroupNormParams& p) {
    return !misaligned(p.weight, 16) && !misaligned(p.bias, 16) && !misaligned(p.scale, 16) && !misaligned(p.shift, 16) &&
           (!p.scale || p.scale_stride % 4 == 0) && (!p.shift || p.shift_stride % 4 == 0);
}

}  // namespace

extern "C" {

ccv3d_status ccv3d_group_norm_workspace(const ccv3d_group_norm_desc* d, uint64_t* bytes_host) {
    if (!d || !bytes_host) return CCV3D_ERR_INVALID_ARG;
    const ccv3d_status s = check_group_norm(d->samples, d->pixels, d->channels, d->groups, d->activation, d->dtype);
    if (s != CCV3D_OK) return s;
    *bytes_host = 0;
    if (d->samples == 0 || d->pixels == 0) return CCV3D_OK;
    // either form of access (the addresses are not known here)
    for (int vec = 0; vec < 2; ++vec) {
        if (vec && d->channels % (16 / esize(d->dtype))) continue;
        const uint64_t n = gn_plan(d->samples, d->pixels, d->channels, d->groups, d->dtype, vec).bytes;
        if (n > *bytes_host) *bytes_host = n;
    }
    return CCV3D_OK;
}

ccv3d_status ccv3d_group_norm(const ccv3d_group_norm_desc* d, const void* x, const float* weight, const float* bias,
                              const float* scale, const float* shift, void* y, void* ws, uint64_t ws_bytes, void* stream) {
    if (!d) return CCV3D_ERR_INVALID_ARG;
    ccv3d_status s = check_group_norm(d->samples, d->pixels, d->channels, d->groups, d->activation, d->dtype);
    if (s != CCV3D_OK) return s;
    if (d->samples == 0 || d->pixels == 0) return CCV3D_OK;
    if (!x || !y) return CCV3D_ERR_INVALID_ARG;
    if (d->x_sample_stride < 0 || d->x_pixel_stride < 0 || d->y_sample_stride < 0 || d->y_pixel_stride < 0 || (scale && d->scale_stride < 0) ||
        (shift && d->shift_stride < 0))
        return CCV3D_ERR_INVALID_ARG;
    const int64_t S = d->samples, P = d->pixels, C = d->channels, e = esize(d->dtype);
    if (!apart(S, P, C, d->y_sample_stride, d->y_pixel_stride)) return CCV3D_ERR_INVALID_ARG;
    if (misaligned(x, e) || misaligned(y, e) || misaligned(weight, 4) || misaligned(bias, 4) || misaligned(scale, 4) || misaligned(shift, 4))
        return CCV3D_ERR_ALIGNMENT;
    // strides of dimensions of one are anything
    const int64_t xs = S > 1 ? d->x_sample_stride : 0, xp = P > 1 ? d->x_pixel_stride : 0, ys = S > 1 ? d->y_sample_stride : 0, yp = P > 1 ? d->y_pixel_stride : 0;
    const bool vec = C % (16 / e) == 0 && whole_vectors(x, d->dtype, xs, xp) && whole_vectors(y, d->dtype, ys, yp);
    const GnPlan q = gn_plan(S, P, (int)C, d->groups, d->dtype, vec);
    if ((s = check_ws(ws, ws_bytes, q.bytes)) != CCV3D_OK) return s;
    const Span in = span_of(x, ((S - 1) * xs + (P - 1) * xp + C) * e), out = span_of(y, ((S - 1) * ys + (P - 1) * yp + C) * e);
    if (meet(in, out) && !(x == y && xs == ys && xp == yp)) return CCV3D_ERR_ALIAS;
    const Span small[] = {span_of(weight, weight ? C * 4 : 0), span_of(bias, bias ? C * 4 : 0),
                          span_of(scale, scale ? ((S - 1) * d->scale_stride + C) * 4 : 0), span_of(shift, shift ? ((S - 1) * d->shift_stride + C) * 4 : 0)};
    const Span w = span_of(ws, q.bytes);
    for (const Span& t : small)
        if (t.a != t.b && (meet(t, out) || (q.bytes && meet(t, w)))) return CCV3D_ERR_ALIAS;
    if (q.bytes && (meet(w, in) || meet(w, out))) return CCV3D_ERR_ALIAS;
    GroupNormParams p = {};
    p.x = x; p.y = y; p.weight = weight; p.bias = bias; p.scale = scale; p.shift = shift;
    p.scale_stride = d->scale_stride; p.shift_stride = d->shift_stride;
    p.xv = {0, xs, xp, 0, (int)S, 0};
    p.yv = {0, ys, yp, 0, (int)S, 0};
    p.T = (int)S; p.samples = (int)S; p.pixels = (int)P; p.C = (int)C; p.groups = d->groups; p.per = (int)C / d->groups; p.block_shift = 30;
    p.columns = q.columns; p.lanes = q.lanes; p.eps = d->eps; p.act = d->activation;
    p.vec_affine = affine_vectors(p);
    return run_group_norm(p, q, d->dtype, ws, (cudaStream_t)stream);
}

ccv3d_status ccv3d_group_norm_ring_workspace(const ccv3d_ring* in, int32_t T, int32_t groups, uint64_t* bytes_host) {
    if (!in || !bytes_host || ccv3d_ring_bytes(in) == 0 || T < 0 || T > in->F) return CCV3D_ERR_INVALID_ARG;
    const ccv3d_status s = check_group_norm((int64_t)in->N * T, (int64_t)in->H * in->W, in->C, groups, CCV3D_ACT_NONE, CCV3D_BF16);
    if (s != CCV3D_OK) return s;
    *bytes_host = T == 0 ? 0 : gn_plan((int64_t)in->N * T, (int64_t)in->H * in->W, in->C, groups, CCV3D_BF16, true, true).bytes;
    return CCV3D_OK;
}

ccv3d_status ccv3d_group_norm_ring(const ccv3d_ring* in, int32_t in_slot, const ccv3d_ring* out, int32_t out_slot, int32_t T,
                                   int32_t groups, const float* weight, const float* bias, const float* scale, int64_t scale_stride,
                                   const float* shift, int64_t shift_stride, float eps, int32_t activation, void* ws,
                                   uint64_t ws_bytes, void* stream) {
    if (!in || !out || !in->base || !out->base || ccv3d_ring_bytes(in) == 0 || ccv3d_ring_bytes(out) == 0) return CCV3D_ERR_INVALID_ARG;
    if (T < 0 || T > in->F || T > out->F || in_slot < 0 || in_slot >= in->F || out_slot < 0 || out_slot >= out->F) return CCV3D_ERR_INVALID_ARG;
    if (in->N != out->N || in->C != out->C || in->H != out->H || in->W != out->W || in->KB != out->KB) return CCV3D_ERR_INVALID_ARG;
    if ((scale && scale_stride < 0) || (shift && shift_stride < 0)) return CCV3D_ERR_INVALID_ARG;
    const int64_t S = (int64_t)in->N * T, P = (int64_t)in->H * in->W;
    const int C = in->C;
    ccv3d_status s = check_group_norm(S, P, C, groups, activation, CCV3D_BF16);
    if (s != CCV3D_OK) return s;
    if (S == 0) return CCV3D_OK;
    if (misaligned(in->base, 16) || misaligned(out->base, 16) || misaligned(weight, 4) || misaligned(bias, 4) || misaligned(scale, 4) || misaligned(shift, 4))
        return CCV3D_ERR_ALIGNMENT;
    const GnPlan q = gn_plan(S, P, C, groups, CCV3D_BF16, true, true);
    if ((s = check_ws(ws, ws_bytes, q.bytes)) != CCV3D_OK) return s;
    const Span a = span_of(in->base, (int64_t)ccv3d_ring_bytes(in)), b = span_of(out->base, (int64_t)ccv3d_ring_bytes(out)), w = span_of(ws, q.bytes);
    if (meet(a, b) && !(in->base == out->base && in->F == out->F && in_slot == out_slot)) return CCV3D_ERR_ALIAS;
    const Span small[] = {span_of(weight, weight ? C * 4 : 0), span_of(bias, bias ? C * 4 : 0),
                          span_of(scale, scale ? ((S - 1) * scale_stride + C) * 4 : 0), span_of(shift, shift ? ((S - 1) * shift_stride + C) * 4 : 0)};
    for (const Span& t : small)
        if (t.a != t.b && (meet(t, b) || (q.bytes && meet(t, w)))) return CCV3D_ERR_ALIAS;
    if (q.bytes && (meet(w, a) || meet(w, b))) return CCV3D_ERR_ALIAS;
    GroupNormParams p = {};
    p.x = in->base; p.y = out->base; p.weight = weight; p.bias = bias; p.scale = scale; p.shift = shift;
    p.scale_stride = scale_stride; p.shift_stride = shift_stride;
    const int64_t frame = P * C;
    p.xv = {in->F * frame, frame, in->KB, P * in->KB, in->F, in_slot};
    p.yv = {out->F * frame, frame, in->KB, P * in->KB, out->F, out_slot};
    p.T = T; p.samples = (int)S; p.pixels = (int)P; p.C = C; p.groups = groups; p.per = C / groups; p.block_shift = in->KB == 64 ? 6 : 5;
    p.columns = q.columns; p.lanes = q.lanes; p.eps = eps; p.act = activation;
    p.vec_affine = affine_vectors(p);
    return run_group_norm(p, q, CCV3D_BF16, ws, (cudaStream_t)stream);
}

}  // extern "C"
