// C entry points of the products: argument checks, cutting into tiles, launches.
#include "ccv3d_tokens_linear.cuh"
#include "ccv3d_tokens_host.cuh"

using namespace ccv3d;

namespace {

__device__ uint32_t linear_status_word;      // (lent to calls that have none of their own)

// Tokens of a tile, and how its tiles fall to the pairs of SMs.
struct LinearPlan {
    Device dev;
    bool few;                    // F32 without the tensor cores
    int BT, kblocks, n_tiles, whole, tail, sharers, pairs;      // pairs: of SMs (few: blocks)
    int64_t t_tiles, pitch, x_at, w_at, part_at;      // F32: elements between rows of a split operand; bytes in the scratch
    uint64_t bytes;
};

ccv3d_status check_linear(const ccv3d_linear_desc* d) {
    if (!d || d->rows < 0 || d->n_out < 1 || d->k < 1 || (d->gated != 0 && d->gated != 1)) return CCV3D_ERR_INVALID_ARG;
    if (!dtype_ok(d->dtype) || !dtype_ok(d->out_dtype) || (d->dtype == CCV3D_F32 && d->out_dtype != CCV3D_F32)) return CCV3D_ERR_INVALID_ARG;
    if (d->activation < CCV3D_ACT_NONE || d->activation > CCV3D_ACT_GELU_TANH) return CCV3D_ERR_INVALID_ARG;
    const int64_t most = 0x7FFF0000, parts = d->dtype == CCV3D_F32 ? 3 : 1;
    if (d->k > (1 << 16) || parts * (d->rows + 256LL) > most || parts * (d->n_out * (1LL + d->gated) + 256) > most) return CCV3D_ERR_UNSUPPORTED;
    return CCV3D_OK;
}

// F32 rows that go without the tensor cores.  us, 4096 -> 9472, without / with them: 16 rows 59 / 146, 32 rows 96 / 145, 64 rows 175 / 149;
// gated 16 rows 120 / 275.
int few_rows(bool gated) { return gated ? 16 : 32; }

// Microseconds of a K block of a tile with every pair of SMs at work (measured with one tile for each: the way from L2, at 12 to 14 TB/s,
// bounds narrow tiles, so that one of 128 tokens takes as long as one of 16), and of a tile's end.
double block_us(int BT, bool gated, bool f32) {
    if (f32) return (gated ? 2.0 : 1.0) * (BT == 16 ? 0.60 : BT == 64 ? 0.65 : BT == 128 ? 0.75 : 1.15);
    return gated ? (BT == 128 ? 0.55 : 0.47) : BT == 256 ? 0.35 : 0.26;
}

ccv3d_status plan_linear(const ccv3d_linear_desc* d, LinearPlan* q) {
    ccv3d_status s = check_linear(d);
    if (s != CCV3D_OK) return s;
    if ((s = current_device(&q->dev)) != CCV3D_OK) return s;
    const bool f32 = d->dtype == CCV3D_F32;
    q->few = f32 && d->rows <= few_rows(d->gated);
    const int kb = f32 ? 32 : 64;
    q->kblocks = (d->k + kb - 1) / kb;
    q->n_tiles = (d->n_out + 255) / 256;
    q->pairs = q->few ? (d->gated ? 1 : 2) * q->dev.sm_count : q->dev.sm_count / 2;
    // Tokens of a tile, and whether the tiles of the last, unfilled turn are cut along K: by the time that the call would take.  It is not under
    // that of the weights' bytes; cutting costs a launch, and the sums' way through memory.
    const double bytes_us = (double)d->n_out * (1 + d->gated) * d->k * esize(d->dtype) / 5.6e6;
    double best = 1e30;
    for (const int BT : {16, 32, 64, 128, 256}) {
        if (q->few ? BT > few_rows(d->gated) : BT == 32 || (BT == 256 && d->gated)) continue;
        const int64_t t_tiles = ((int64_t)d->rows + BT - 1) / BT, tiles = q->n_tiles * t_tiles, turns = tiles / q->pairs;
        if (tiles > 0x3FFFFFFF) continue;
        const double tile_us = q->kblocks * (q->few ? (BT == 32 ? 1.5 : 1.0) : block_us(BT, d->gated, f32)), end_us = BT * (1 + d->gated) / 85.0;
        const int left = (int)(tiles % q->pairs);
        const auto longer = [](double a, double b) { return a > b ? a : b; };
        double us = longer((turns + (left > 0)) * tile_us, bytes_us) + end_us;
        if (us < best) {
            best = us;
            q->BT = BT;
            q->t_tiles = t_tiles;
            q->whole = (int)tiles;
            q->tail = q->sharers = 0;
        }
        const int64_t shares = (int64_t)left * q->kblocks / 4;         // of four K blocks at least
        const int sharers = (int)(shares < q->pairs ? shares : q->pairs);
        if (left == 0 || sharers <= left) continue;
        const double sums = 2.0 * (sharers + left) * BT * (1 + d->gated) * 1024;
        us = longer(turns * tile_us + left * tile_us / sharers, bytes_us) + end_us + 5.0 + sums / 4e6;
        if (us < best) {
            best = us;
            q->BT = BT;
            q->t_tiles = t_tiles;
            q->whole = (int)(tiles - left);
            q->tail = left;
            q->sharers = sharers;
        }
    }
    if (best == 1e30) return CCV3D_ERR_UNSUPPORTED;
    const auto up = [](int64_t n) { return (n + 255) / 256 * 256; };
    q->pitch = (d->k + 7LL) / 8 * 8;
    q->x_at = 0;
    const bool split = f32 && !q->few;
    q->w_at = split ? up(3 * q->pitch * d->rows * 2) : 0;
    q->part_at = q->w_at + (split ? up(3 * q->pitch * d->n_out * (1 + d->gated) * 2) : 0);
    q->bytes = q->part_at + 2LL * q->sharers * q->BT * (1 + d->gated) * 256 * 4;
    return CCV3D_OK;
}

// A matrix of `rows` rows of k elements of `size` bytes, in boxes of box_k elements of box_rows rows.
ccv3d_status encode_rows(CUtensorMap* tm, const void* at, int size, int64_t rows, int64_t k, int64_t stride, int box_k, int box_rows, CUtensorMapSwizzle swizzle) {
    const EncodeTiledFn fn = encode_tiled();
    if (!fn) return CCV3D_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)(stride * size)};
    const cuuint32_t box[2] = {(cuuint32_t)box_k, (cuuint32_t)box_rows}, es[2] = {1, 1};
    const CUresult r = fn(tm, size == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, const_cast<void*>(at), dims, strides, box, es,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? CCV3D_OK : CCV3D_ERR_CUDA;
}

// The sums of tiles that were cut, launched so that it is resident when the kernel before it ends.
template <typename TO, bool GATED>
ccv3d_status launch_join(const LinearParams& p, int BT, cudaStream_t st) {
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.tail, BT / LINEAR_JOIN_TOKENS);
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, linear_join_kernel<TO, GATED>, p, BT) != cudaSuccess) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    return CCV3D_OK;
}

template <typename S, typename TO>
ccv3d_status launch_linear_as(LinearParams& p, const LinearPlan& q, const void* x, int64_t x_rows, int64_t x_stride, const void* w, int64_t w_rows,
                              int64_t w_stride, int k, cudaStream_t st) {
    static std::atomic<uint64_t> done{0};
    if (!allow_smem(linear_tile_kernel<S, TO>, S::SMEM, q.dev.index, done)) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    constexpr CUtensorMapSwizzle swizzle = S::ROWB == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B;
    CUtensorMap tw, tx, to = {}, tr = {};
    ccv3d_status s = encode_rows(&tw, w, 2, w_rows, k, w_stride, S::KB, 128, swizzle);
    if (s == CCV3D_OK) s = encode_rows(&tx, x, 2, x_rows, k, x_stride, S::KB, S::BT / 2, swizzle);
    if (s == CCV3D_OK && p.boxes) s = encode_rows(&to, p.out, sizeof(TO), p.rows, p.n_out, p.out_stride, 32, S::CH, CU_TENSOR_MAP_SWIZZLE_NONE);
    if (s == CCV3D_OK && p.res_boxes) s = encode_rows(&tr, p.res, sizeof(TO), p.rows, p.n_out, p.res_stride, 32, S::CH, CU_TENSOR_MAP_SWIZZLE_NONE);
    if (s != CCV3D_OK) return s;
    const int used = p.tail ? p.pairs : (p.whole < p.pairs ? p.whole : p.pairs);
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * used);
    cfg.blockDim = dim3(S::THREADS);
    cfg.dynamicSmemBytes = S::SMEM;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = S::PARTS == 3 ? 1 : 0;            // behind the kernels that split the operands
    if (cudaLaunchKernelEx(&cfg, linear_tile_kernel<S, TO>, tw, tx, to, tr, p) != cudaSuccess) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    return p.tail ? launch_join<TO, S::GATED>(p, S::BT, st) : CCV3D_OK;
}

template <bool GATED, int BT>
ccv3d_status launch_few(LinearParams& p, const LinearPlan& q, const float* x, int64_t x_stride, const float* w, int64_t w_stride, int k, cudaStream_t st) {
    constexpr int bytes = (LINEAR_FEW_STAGES * (GATED ? 2 : 1) * 256 + 2 * BT) * LINEAR_FEW_K * 4;
    static std::atomic<uint64_t> done{0};
    if (!allow_smem(linear_few_kernel<GATED, BT>, bytes, q.dev.index, done)) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    const int used = p.tail ? p.pairs : (p.whole < p.pairs ? p.whole : p.pairs);
    linear_few_kernel<GATED, BT><<<used, LINEAR_FEW_THREADS, bytes, st>>>(p, x, x_stride, w, w_stride, k);
    const ccv3d_status s = launched();
    return s == CCV3D_OK && p.tail ? launch_join<float, GATED>(p, BT, st) : s;
}

template <int PARTS, typename TO, typename... A>
ccv3d_status launch_linear(bool gated, int BT, A&&... a) {
    constexpr bool F = sizeof(TO) == 4;
    if (gated) {
        if (BT == 16) return launch_linear_as<LinearShape<16, true, PARTS, F>, TO>(a...);
        if (BT == 64) return launch_linear_as<LinearShape<64, true, PARTS, F>, TO>(a...);
        return launch_linear_as<LinearShape<128, true, PARTS, F>, TO>(a...);
    }
    if (BT == 16) return launch_linear_as<LinearShape<16, false, PARTS, F>, TO>(a...);
    if (BT == 64) return launch_linear_as<LinearShape<64, false, PARTS, F>, TO>(a...);
    if (BT == 128) return launch_linear_as<LinearShape<128, false, PARTS, F>, TO>(a...);
    return launch_linear_as<LinearShape<256, false, PARTS, F>, TO>(a...);
}

}  // namespace

extern "C" {

ccv3d_status ccv3d_linear_status_word(uint32_t** word_host) {
    if (!word_host) return CCV3D_ERR_INVALID_ARG;
    Device dev;
    const ccv3d_status s = current_device(&dev);
    if (s != CCV3D_OK) return s;
    // (the first asking may load the code, which a capture of this thread would not allow)
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    void* at = nullptr;
    if (cudaThreadExchangeStreamCaptureMode(&mode) != cudaSuccess) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    const bool found = cudaGetSymbolAddress(&at, linear_status_word) == cudaSuccess;
    if (!found) cudaGetLastError();
    if (cudaThreadExchangeStreamCaptureMode(&mode) != cudaSuccess || !found) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    *word_host = (uint32_t*)at;
    return CCV3D_OK;
}

ccv3d_status ccv3d_take_status(uint32_t* status, uint32_t* bits_host) {
    if (!status || !bits_host) return CCV3D_ERR_INVALID_ARG;
    if (misaligned(status, 4)) return CCV3D_ERR_ALIGNMENT;
    uint32_t bits = 0;
    bool ok = cudaDeviceSynchronize() == cudaSuccess && cudaMemcpy(&bits, status, 4, cudaMemcpyDeviceToHost) == cudaSuccess;
    if (ok && bits) ok = cudaMemset(status, 0, 4) == cudaSuccess && cudaDeviceSynchronize() == cudaSuccess;
    if (!ok) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    *bits_host = bits;
    return CCV3D_OK;
}

ccv3d_status ccv3d_linear_workspace(const ccv3d_linear_desc* d, uint64_t* bytes_host) {
    if (!bytes_host) return CCV3D_ERR_INVALID_ARG;
    LinearPlan q;
    ccv3d_status s = check_linear(d);
    if (s == CCV3D_OK && d->rows == 0) {
        *bytes_host = 0;
        return s;
    }
    if (s == CCV3D_OK) s = plan_linear(d, &q);
    if (s == CCV3D_OK) *bytes_host = q.bytes;
    return s;
}

ccv3d_status ccv3d_linear(const ccv3d_linear_desc* d, const void* x, const void* w, const void* bias, const void* residual,
                          void* out, void* ws, uint64_t ws_bytes, uint32_t* status, void* stream) {
    ccv3d_status s = check_linear(d);
    if (s != CCV3D_OK) return s;
    if (d->rows == 0) return CCV3D_OK;
    if (!x || !w || !out) return CCV3D_ERR_INVALID_ARG;
    const int64_t M = d->rows, N = d->n_out, K = d->k, NW = N * (1 + d->gated), e = esize(d->dtype), eo = esize(d->out_dtype);
    // strides of a single row are anything
    const int64_t xs = M > 1 ? d->x_stride : (K * e + 15) / 16 * 16 / e, wst = NW > 1 ? d->w_stride : (K * e + 15) / 16 * 16 / e;
    if (xs < K || wst < K || (M > 1 && d->out_stride < N) || (M > 1 && residual && d->residual_stride < 0)) return CCV3D_ERR_INVALID_ARG;
    if (misaligned(x, 16) || misaligned(w, 16) || xs * e % 16 || wst * e % 16 || misaligned(bias, e) || misaligned(residual, eo) || misaligned(out, eo) ||
        misaligned(status, 4))
        return CCV3D_ERR_ALIGNMENT;
    const Span so = span_of(out, ((M - 1) * d->out_stride + N) * eo);
    const Span in[] = {span_of(x, ((M - 1) * xs + K) * e), span_of(w, ((NW - 1) * wst + K) * e), span_of(bias, bias ? NW * e : 0),
                       span_of(residual, residual ? ((M - 1) * d->residual_stride + N) * eo : 0)};
    for (int i = 0; i < 4; ++i)
        if (in[i].a != in[i].b && meet(so, in[i]) && !(i == 3 && out == residual && (M == 1 || d->out_stride == d->residual_stride))) return CCV3D_ERR_ALIAS;
    LinearPlan q;
    if ((s = plan_linear(d, &q)) != CCV3D_OK) return s;
    if ((s = check_ws(ws, ws_bytes, q.bytes)) != CCV3D_OK) return s;
    const Span sw = span_of(ws, (int64_t)q.bytes);
    if (q.bytes) {
        if (meet(sw, so)) return CCV3D_ERR_ALIAS;
        for (const Span& t : in)
            if (t.a != t.b && meet(sw, t)) return CCV3D_ERR_ALIAS;
    }
    cudaStream_t st = (cudaStream_t)stream;
    LinearParams p = {};
    p.bias = bias;
    p.res = residual;
    p.out = out;
    p.out_stride = d->out_stride;
    p.res_stride = d->residual_stride;
    p.rows = d->rows;
    p.n_out = d->n_out;
    p.act = d->activation;
    p.bias_f32 = d->dtype == CCV3D_F32;
    p.n_tiles = q.n_tiles;
    p.kblocks = q.kblocks;
    p.whole = q.whole;
    p.tail = q.tail;
    p.sharers = q.sharers;
    p.pairs = q.pairs;
    p.part = (float*)((char*)ws + q.part_at);
    p.boxes = !misaligned(out, 16) && (M == 1 ? (N * eo) % 16 == 0 : d->out_stride * eo % 16 == 0);
    if (M == 1) p.out_stride = p.res_stride = N;
    // (rows on one another, a broadcast residual, have no map)
    p.res_boxes = residual && !misaligned(residual, 16) && p.res_stride >= N && p.res_stride * eo % 16 == 0;
    p.status = status;
    p.wait_clk = q.dev.wait_clk;
    if (q.few) {
        const float *xf = (const float*)x, *wf = (const float*)w;
        if (d->gated) return launch_few<true, 16>(p, q, xf, xs, wf, wst, d->k, st);
        return q.BT == 16 ? launch_few<false, 16>(p, q, xf, xs, wf, wst, d->k, st) : launch_few<false, 32>(p, q, xf, xs, wf, wst, d->k, st);
    }
    if (d->dtype == CCV3D_F32) {
        void *px = (char*)ws + q.x_at, *pw = (char*)ws + q.w_at;
        const int64_t blocks = ((NW + M) * (q.pitch / 4) + 255) / 256;
        linear_split_kernel<<<(unsigned)(blocks < 16 * q.dev.sm_count ? blocks : 16 * q.dev.sm_count), 256, 0, st>>>(
            (const float*)w, wst, (int)NW, (__nv_bfloat16*)pw, (const float*)x, xs, d->rows, (__nv_bfloat16*)px, d->k, (int)q.pitch);
        if ((s = launched()) != CCV3D_OK) return s;
        p.x_plane = d->rows;
        p.w_plane = (int)NW;
        return launch_linear<3, float>(d->gated, q.BT, p, q, px, 3 * M, q.pitch, pw, 3 * NW, q.pitch, d->k, st);
    }
    if (d->out_dtype == CCV3D_F32) return launch_linear<1, float>(d->gated, q.BT, p, q, x, M, xs, w, NW, wst, d->k, st);
    return launch_linear<1, __nv_bfloat16>(d->gated, q.BT, p, q, x, M, xs, w, NW, wst, d->k, st);
}

}  // extern "C"
