// Host side of the token operators, the shared part: argument checks, spans, what is known of a device, tensor maps.
#pragma once
#include "../../include/ccv3d.h"

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <cstdlib>

// (each source that includes this uses a part of it)
#pragma nv_diag_suppress 177

namespace {

inline int64_t esize(int dt) { return dt == CCV3D_BF16 ? 2 : 4; }
inline bool dtype_ok(int dt) { return dt == CCV3D_F32 || dt == CCV3D_BF16; }
inline bool misaligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

ccv3d_status launched() {
    if (cudaGetLastError() == cudaSuccess) return CCV3D_OK;
    return CCV3D_ERR_CUDA;
}

// What the launches need to know of the current device, looked up once for each.
struct Device { int index, sm_count; long long wait_clk; };
constexpr int MAX_DEVICES = 64;
std::atomic<int> g_sms[MAX_DEVICES];     // 0: not looked up, < 0: not compute capability 10.x

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// CCV3D_WAIT_LIMIT_MS (1..10000) bounds the waits inside the kernels; default about a second at the highest SM clock.
long long wait_limit_clk() {
    static const long long clk = [] {
        const char* e = getenv("CCV3D_WAIT_LIMIT_MS");
        const int ms = e ? atoi(e) : 0;
        return 2000000LL * (ms >= 1 && ms <= 10000 ? ms : 1000);
    }();
    return clk;
}

ccv3d_status current_device(Device* d) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    int sms = g_sms[dev].load(std::memory_order_relaxed);
    if (!sms) {
        int major = 0;
        if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
            cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
            cudaGetLastError();
            return CCV3D_ERR_CUDA;
        }
        if (major != 10) sms = -1;
        g_sms[dev].store(sms, std::memory_order_relaxed);
    }
    if (sms < 0) return CCV3D_ERR_ARCH;
    d->index = dev;
    d->sm_count = sms;
    d->wait_clk = wait_limit_clk();
    return CCV3D_OK;
}

// Byte range of a strided tensor: rows (and heads) with non-negative strides.
struct Span { uintptr_t a, b; };
inline Span span_of(const void* p, int64_t bytes) { return {(uintptr_t)p, (uintptr_t)p + (uint64_t)bytes}; }
inline Span span_of(const ccv3d_heads& h, int64_t tokens, int heads, int dim, int dt) {
    return span_of(h.data, ((tokens - 1) * h.token_stride + (heads - 1) * h.head_stride + dim) * esize(dt));
}
inline bool meet(const Span& x, const Span& y) { return x.a < y.b && y.a < x.b; }

// Whether two packed tensors of the same tokens share an element.  Slices of one projection have ranges that lie in one another
// without sharing any: with one token stride, heads are compared within a token's stretch.  Unlike strides count as shared
// where the ranges meet.
bool share(const ccv3d_heads& x, int x_heads, const ccv3d_heads& y, int y_heads, int64_t tokens, int dim, int dt) {
    if (!meet(span_of(x, tokens, x_heads, dim, dt), span_of(y, tokens, y_heads, dim, dt))) return false;
    const int64_t e = esize(dt), len = dim * e, xs = x.head_stride * e, ys = y.head_stride * e;
    const int64_t x_far = (x_heads - 1) * xs + len, y_far = (y_heads - 1) * ys + len;
    const int64_t first = (int64_t)((uintptr_t)y.data - (uintptr_t)x.data), stretch = tokens > 1 ? x.token_stride * e : x_far + y_far;
    if (tokens > 1 && (x.token_stride != y.token_stride || x_far > stretch || y_far > stretch)) return true;
    const int64_t at = tokens > 1 ? (first % stretch + stretch) % stretch : first;     // of y in x's stretch (one token: anywhere)
    // heads that follow one another closely are one piece
    const int64_t x_len = xs <= len ? x_far : len, y_len = ys <= len ? y_far : len;
    for (int i = 0; i < (xs <= len ? 1 : x_heads); ++i)
        for (int j = 0; j < (ys <= len ? 1 : y_heads); ++j)
            for (int64_t a = at + j * ys - i * xs - (tokens > 1 ? stretch : 0), turn = 0; turn < (tokens > 1 ? 3 : 1); ++turn, a += stretch)
                if (a < x_len && a + y_len > 0) return true;     // (the stretch before, this one, the one behind)
    return false;
}

// `tokens` > 0: an output, whose rows must not lie on one another (token by token or head by head); an input's may (a
// broadcast head or token).
ccv3d_status check_heads(const ccv3d_heads* h, int heads, int dim, int dt, int64_t tokens = 0) {
    if (!h || !h->data || h->token_stride < 0 || h->head_stride < 0) return CCV3D_ERR_INVALID_ARG;
    if (tokens) {
        const int64_t ts = tokens > 1 ? h->token_stride : INT64_MAX, hs = heads > 1 ? h->head_stride : INT64_MAX;
        const bool by_token = hs >= dim && ts >= (heads > 1 ? (heads - 1) * hs : 0) + dim;
        const bool by_head = ts >= dim && hs >= (tokens > 1 ? (tokens - 1) * ts : 0) + dim;
        if (!by_token && !by_head) return CCV3D_ERR_INVALID_ARG;
    }
    const int64_t unit = 16 / esize(dt);
    if (misaligned(h->data, 16) || h->token_stride % unit || h->head_stride % unit) return CCV3D_ERR_ALIGNMENT;
    return CCV3D_OK;
}

// Opts a kernel into its dynamic shared memory, once for each device.
template <typename F>
bool allow_smem(F* kernel, int bytes, int dev, std::atomic<uint64_t>& done) {
    if (done.load(std::memory_order_relaxed) >> dev & 1) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
    done.fetch_or(1ull << dev, std::memory_order_relaxed);
    return true;
}

// cuTensorMapEncodeTiled, looked up once.
EncodeTiledFn encode_tiled() {
    static std::atomic<EncodeTiledFn> encode{nullptr};
    EncodeTiledFn fn = encode.load(std::memory_order_relaxed);
    if (!fn) {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &qres) != cudaSuccess || !f || qres != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        fn = (EncodeTiledFn)f;
        encode.store(fn, std::memory_order_relaxed);
    }
    return fn;
}

ccv3d_status check_ws(const void* ws, uint64_t have, uint64_t need) {
    if (misaligned(ws, 256)) return CCV3D_ERR_ALIGNMENT;
    return need && (!ws || have < need) ? CCV3D_ERR_NOMEM : CCV3D_OK;
}

}  // namespace
