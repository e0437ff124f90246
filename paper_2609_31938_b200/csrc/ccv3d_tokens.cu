// C entry points of the token operators: argument checks, kernel choice, launches.
#include "../../include/ccv3d.h"

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdlib>

#include "ccv3d_tokens_append.cuh"
#include "ccv3d_tokens_attend_step.cuh"
#include "ccv3d_tokens_attend_tile.cuh"
#include "ccv3d_tokens_norm.cuh"

using namespace ccv3d;

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

ccv3d_status check_cache(const ccv3d_kv_cache* c) {
    if (!c || !c->codes || !c->scales || c->pages < 1 || c->kv_heads < 1) return CCV3D_ERR_INVALID_ARG;
    if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128) return CCV3D_ERR_UNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128) return CCV3D_ERR_UNSUPPORTED;
    if (c->kv_heads > 65536) return CCV3D_ERR_UNSUPPORTED;
    if (misaligned(c->codes, 16) || misaligned(c->scales, 4)) return CCV3D_ERR_ALIGNMENT;
    return CCV3D_OK;
}

ccv3d_status check_batch(const ccv3d_token_batch* b, int page_tokens) {
    if (!b || b->batch < 0 || b->max_pages < 0 || b->tokens < 0 || b->max_new < 0) return CCV3D_ERR_INVALID_ARG;
    if (b->batch == 0) return b->tokens == 0 ? CCV3D_OK : CCV3D_ERR_INVALID_ARG;      // nobody: no arrays, no rows
    if (!b->new_start || !b->total) return CCV3D_ERR_INVALID_ARG;
    if (!b->page_table && b->max_pages > 0) return CCV3D_ERR_INVALID_ARG;
    if ((int64_t)b->max_pages * page_tokens > 0x7FFFFF00 || b->batch > 65536) return CCV3D_ERR_UNSUPPORTED;    // (room for a unit more)
    if (misaligned(b->new_start, 4) || misaligned(b->total, 4) || misaligned(b->page_table, 4)) return CCV3D_ERR_ALIGNMENT;
    return CCV3D_OK;
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

Span codes_span(const ccv3d_kv_cache* c) {
    return span_of(c->codes, (int64_t)c->pages * 2 * c->kv_heads * c->page_tokens * c->head_dim);
}
Span scales_span(const ccv3d_kv_cache* c) { return span_of(c->scales, (int64_t)c->pages * 2 * c->kv_heads * 4); }
bool meets_batch(const Span& x, const ccv3d_token_batch* b) {
    return meet(x, span_of(b->new_start, (b->batch + 1LL) * 4)) || meet(x, span_of(b->total, b->batch * 4LL)) ||
           meet(x, span_of(b->page_table, (int64_t)b->batch * b->max_pages * 4));
}
bool meets_rotary(const Span& x, const ccv3d_rotary* r, int64_t tokens) {
    const int64_t table = (int64_t)r->rows * r->pairs * 4;
    return meet(x, span_of(r->cos_table, table)) || meet(x, span_of(r->sin_table, table)) || meet(x, span_of(r->positions, tokens * r->axes * 4));
}

template <typename T, int D, int P, bool FEW>
ccv3d_status launch_append_as(AppendParams& p, cudaStream_t st) {
    using S = AppendShape<D, P, FEW>;
    // pages that n new tokens can touch: one for n = 1, else up to (n - 1) / P + 2
    const int64_t by_tokens = (int64_t)p.bt.tokens / P + 2LL * p.bt.batch;
    const int64_t by_batch = (int64_t)p.bt.batch * (p.bt.max_new <= 1 ? 1 : (p.bt.max_new - 1) / P + 2);
    const bool one = p.bt.max_new <= 1;            // (then a block's number names its sequence)
    const int64_t kv = (one || by_batch < by_tokens ? by_batch : by_tokens) * p.c.kv_heads;
    const int64_t items = p.q.data ? (int64_t)p.bt.tokens * ((p.q_heads + QUERY_HEADS - 1) / QUERY_HEADS) : 0;
    const int64_t q_blocks = ((items + S::TPI - 1) / S::TPI + S::CLUSTER - 1) / S::CLUSTER * S::CLUSTER;
    const int64_t all = kv * S::CLUSTER + q_blocks;
    if (all > 0x7FFFFFFF || items > 0xF0000000LL) return CCV3D_ERR_UNSUPPORTED;
    p.kv_blocks = (unsigned)(kv * S::CLUSTER);
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = S::CLUSTER;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)all);
    cfg.blockDim = dim3(S::THREADS);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = S::CLUSTER > 1 ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kv_append_kernel<T, D, P, FEW>, p) != cudaSuccess) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    return CCV3D_OK;
}

template <typename T>
ccv3d_status launch_append(AppendParams& p, cudaStream_t st) {
    const int D = p.c.head_dim, P = p.c.page_tokens;
    const bool few = p.bt.max_new <= 128 / (D / 4);
#define CCV3D_APPEND(d, pg) \
    if (D == d && P == pg) return few ? launch_append_as<T, d, pg, true>(p, st) : launch_append_as<T, d, pg, false>(p, st);
    CCV3D_APPEND(64, 16) CCV3D_APPEND(64, 32) CCV3D_APPEND(64, 64) CCV3D_APPEND(64, 128)
    CCV3D_APPEND(128, 16) CCV3D_APPEND(128, 32) CCV3D_APPEND(128, 64) CCV3D_APPEND(128, 128)
#undef CCV3D_APPEND
    return CCV3D_ERR_UNSUPPORTED;
}

// Opts a kernel into its dynamic shared memory, once for each device.
template <typename F>
bool allow_smem(F* kernel, int bytes, int dev, std::atomic<uint64_t>& done) {
    if (done.load(std::memory_order_relaxed) >> dev & 1) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
    done.fetch_or(1ull << dev, std::memory_order_relaxed);
    return true;
}

template <typename TX, typename TY, int G, int V, int K>
ccv3d_status launch_norm_rows(const NormParams& p, const Device& dev, cudaStream_t st) {
    constexpr int most_smem = 4 * G * V * K * 4;   // of the widest rows it takes; the blocks of an SM below have room for theirs
    static std::atomic<uint64_t> done{0};
    if (!allow_smem(gated_norm_rows_kernel<TX, TY, G, V, K>, most_smem, dev.index, done)) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    const int C = p.d.channels, smem = 4 * ((C + V - 1) / V * V) * 4, teams = ROWS_THREADS / G;
    const int most = (p.d.rows + teams - 1) / teams, wave = (K * V <= 12 ? 2 : 1) * dev.sm_count;
    gated_norm_rows_kernel<TX, TY, G, V, K><<<most < wave ? most : wave, ROWS_THREADS, smem, st>>>(p);
    return launched();
}

// Threads to a row (g), elements of an access (v), accesses of a thread (k).
template <typename TX, typename TY>
ccv3d_status launch_norm(const NormParams& p, bool vec, const Device& dev, cudaStream_t st) {
    const int C = p.d.channels, rows = p.d.rows;
#define CCV3D_ROWS(g, v, k) \
    if (C <= (g) * (v) * (k)) return launch_norm_rows<TX, TY, g, v, k>(p, dev, st);
#define CCV3D_NORM(g, v, k) \
    if (C <= (g) * (v) * (k)) { \
        gated_norm_kernel<TX, TY, g, v, k><<<rows, g, 0, st>>>(p); \
        return launched(); \
    }
    // more than two rows to an SM: rows by stretches, where a thread's share of the channels fits into its registers
    if (rows > 2 * dev.sm_count) {
        if (vec) {
            CCV3D_ROWS(32, 4, 1) CCV3D_ROWS(32, 4, 2) CCV3D_ROWS(32, 4, 3) CCV3D_ROWS(64, 4, 3) CCV3D_ROWS(128, 4, 2) CCV3D_ROWS(128, 4, 3)
            CCV3D_ROWS(256, 4, 2) CCV3D_ROWS(256, 4, 3) CCV3D_ROWS(512, 4, 2)
        } else {
            CCV3D_ROWS(32, 1, 4) CCV3D_ROWS(32, 1, 12) CCV3D_ROWS(128, 1, 5) CCV3D_ROWS(128, 1, 10) CCV3D_ROWS(256, 1, 8) CCV3D_ROWS(256, 1, 12)
            CCV3D_ROWS(512, 1, 8)
        }
    }
    if (vec) {
        CCV3D_NORM(128, 4, 1) CCV3D_NORM(512, 4, 1) CCV3D_NORM(512, 4, 2) CCV3D_NORM(512, 4, 4) CCV3D_NORM(512, 4, 8)
    } else {
        CCV3D_NORM(512, 1, 1) CCV3D_NORM(512, 1, 4) CCV3D_NORM(512, 1, 16) CCV3D_NORM(512, 1, 32)
    }
#undef CCV3D_NORM
#undef CCV3D_ROWS
    return CCV3D_ERR_UNSUPPORTED;
}

// Query rows of an item (8 or 16: step kernel, 128 or 256: tile kernel) where the sequences of a call have up to `rows` of a kv head.
// The step kernel reads the cache once for every 8 or 16 rows, the tile kernel once for all but always in products of 128
// rows.  Device time, us, BF16 (F32), 16 heads on 4, 64 streams of 2000 tokens, 8-row items / 16-row items / tiles:
//   8 rows 43 (49) / 51 (66) / 96 (131);  16 rows - / 55 (70) / 98 (133);  32 rows - / 92 (121) / 98 (137);
//   48 rows - / 127 (168) / 100 (139);  128 rows - / 297 (402) / 107 (145)
// (one stream of 32768: 32 rows 33 (41) / 37 (45), 48 rows 43 (55) / 37 (45); two of 500, 48 to 128 rows: 16 to 21 (18 to 25) / 27 (29 to
// 33): there the rule, which goes by rows alone, gives a quarter and more away)
int rows_per_item(int64_t rows, int dtype) { return rows <= 8 ? 8 : rows <= 32 ? 16 : dtype == CCV3D_BF16 ? 256 : 128; }

ccv3d_status check_attend(const ccv3d_kv_cache* cache, const ccv3d_token_batch* batch, int q_heads, int dtype) {
    ccv3d_status s = check_cache(cache);
    if (s != CCV3D_OK) return s;
    if ((s = check_batch(batch, cache->page_tokens)) != CCV3D_OK) return s;
    if (!dtype_ok(dtype) || q_heads < 1 || q_heads % cache->kv_heads) return CCV3D_ERR_INVALID_ARG;
    const int64_t group = q_heads / cache->kv_heads;
    // 32-bit row numbers (TMA coordinates, query rows) and unit numbers
    if ((int64_t)cache->pages * 2 * cache->kv_heads * cache->page_tokens > 0x7FFFFFFF) return CCV3D_ERR_UNSUPPORTED;
    if ((int64_t)batch->tokens * q_heads > 0x7FFFFFFF) return CCV3D_ERR_UNSUPPORTED;
    // items of `per` rows: of a batch whose sequences all bring max_new tokens, and of all the rows there are, whichever is fewer
    const int64_t units = (int64_t)batch->max_pages * cache->page_tokens / STEP_UNIT + 1, per = rows_per_item(batch->max_new * group, dtype);
    const int64_t by_batch = batch->batch * ((batch->max_new * group + per - 1) / per), by_rows = batch->tokens * group / per + batch->batch;
    if ((double)(by_batch < by_rows ? by_batch : by_rows) * cache->kv_heads * units > MAX_UNITS) return CCV3D_ERR_UNSUPPORTED;
    return CCV3D_OK;
}

// Kernel, grid and scratch of a call.
struct Plan {
    Device dev;
    int rows_per_item;       // query rows of an item: 8 or 16 (step kernel), 128 or 256 (tile kernel)
    int blocks, slot_rows;
    uint64_t ml_at, join_at, bytes;
};

ccv3d_status plan_attend(const ccv3d_kv_cache* cache, const ccv3d_token_batch* batch, int q_heads, int dtype, Plan* pl) {
    ccv3d_status s = check_attend(cache, batch, q_heads, dtype);
    if (s != CCV3D_OK) return s;
    if ((s = current_device(&pl->dev)) != CCV3D_OK) return s;
    const int64_t rows = (int64_t)batch->max_new * (q_heads / cache->kv_heads);
    pl->rows_per_item = rows_per_item(rows, dtype);
    const bool tile = pl->rows_per_item >= 128;
    pl->blocks = (tile ? 1 : step_blocks(dtype == CCV3D_F32, cache->head_dim, pl->rows_per_item)) * pl->dev.sm_count;
    if (pl->blocks > JOIN_PARTS) pl->blocks = JOIN_PARTS;
    pl->slot_rows = tile ? pl->rows_per_item : 16;
    pl->ml_at = (uint64_t)2 * pl->blocks * pl->slot_rows * cache->head_dim * 4;
    pl->join_at = pl->ml_at + (uint64_t)2 * pl->blocks * pl->slot_rows * sizeof(float2);
    pl->bytes = (pl->join_at + pl->blocks * sizeof(Join) + 255) / 256 * 256;
    return CCV3D_OK;
}

// The cache as a matrix of rows of head_dim codes, read in boxes of 32 tokens (16 where a page holds no more).
ccv3d_status encode_cache_map(const ccv3d_kv_cache& c, CUtensorMap* tm, int box_rows) {
    static std::atomic<EncodeTiledFn> encode{nullptr};
    EncodeTiledFn fn = encode.load(std::memory_order_relaxed);
    if (!fn) {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &qres) != cudaSuccess || !f || qres != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return CCV3D_ERR_CUDA;
        }
        fn = (EncodeTiledFn)f;
        encode.store(fn, std::memory_order_relaxed);
    }
    const cuuint64_t dims[2] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.pages * 2 * c.kv_heads * c.page_tokens};
    const cuuint64_t strides[1] = {(cuuint64_t)c.head_dim};
    const cuuint32_t box[2] = {(cuuint32_t)c.head_dim, (cuuint32_t)box_rows}, es[2] = {1, 1};
    const CUresult r = fn(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, c.codes, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          c.head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? CCV3D_OK : CCV3D_ERR_CUDA;
}

template <typename T, int D, int NT>
ccv3d_status launch_step(const AttendParams& p, const Plan& pl, cudaStream_t st) {
    static std::atomic<uint64_t> done{0};
    using S = StepShape<D>;
    if (!allow_smem(kv_attend_step_kernel<T, D, NT>, S::BYTES, pl.dev.index, done)) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    CUtensorMap tm;
    const ccv3d_status s = encode_cache_map(p.c, &tm, p.c.page_tokens < STEP_TILE ? p.c.page_tokens : STEP_TILE);
    if (s != CCV3D_OK) return s;
    kv_attend_step_kernel<T, D, NT><<<pl.blocks, 32 * STEP_WARPS, S::BYTES, st>>>(tm, p);
    return launched();
}

// The sum over parts, launched so that it is resident when the attention kernel ends.
template <typename T, int D>
ccv3d_status launch_join(const AttendParams& p, const Plan& pl, cudaStream_t st) {
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(pl.blocks, pl.slot_rows <= 16 ? pl.rows_per_item : 64);
    cfg.blockDim = dim3(JOIN_THREADS);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, attend_join_kernel<T, D>, p) != cudaSuccess) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
    return CCV3D_OK;
}

template <typename T, int D>
ccv3d_status launch_attend(const AttendParams& p, const Plan& pl, cudaStream_t st) {
    if (pl.rows_per_item >= 128) {
        static std::atomic<uint64_t> done{0};
        constexpr int bytes = TileShape<T, D>::END + sizeof(TileShared);
        static_assert(bytes <= 232448, "shared memory of a block");
        if (!allow_smem(kv_attend_tile_kernel<T, D>, bytes, pl.dev.index, done)) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
        kv_attend_tile_kernel<T, D><<<pl.blocks, TILE_THREADS, bytes, st>>>(p);
        const ccv3d_status s = launched();
        return s == CCV3D_OK ? launch_join<T, D>(p, pl, st) : s;
    }
    const ccv3d_status s = pl.rows_per_item == 8 ? launch_step<T, D, 1>(p, pl, st) : launch_step<T, D, 2>(p, pl, st);
    return s == CCV3D_OK ? launch_join<T, D>(p, pl, st) : s;
}

}  // namespace

extern "C" {

ccv3d_status ccv3d_kv_append(const ccv3d_kv_cache* cache, const ccv3d_token_batch* batch, const ccv3d_heads* k,
                             const ccv3d_heads* v, const ccv3d_rotary* rot, const ccv3d_heads* q,
                             const ccv3d_heads* q_out, int32_t q_heads, int32_t dtype, uint32_t* status, void* stream) {
    ccv3d_status s = check_cache(cache);
    if (s != CCV3D_OK) return s;
    if ((s = check_batch(batch, cache->page_tokens)) != CCV3D_OK) return s;
    if (!dtype_ok(dtype) || (!q != !q_out) || (q && q_heads < 1)) return CCV3D_ERR_INVALID_ARG;
    const int D = cache->head_dim, H = cache->kv_heads, tokens = batch->tokens;
    if (tokens == 0) return CCV3D_OK;
    if ((s = check_heads(k, H, D, dtype)) != CCV3D_OK || (s = check_heads(v, H, D, dtype)) != CCV3D_OK) return s;
    if (rot) {
        if (!rot->cos_table || !rot->sin_table || !rot->positions || rot->rows < 1 || rot->axes < 1 || rot->axes > 3) return CCV3D_ERR_INVALID_ARG;
        if (rot->pairs < 4 || rot->pairs % 4 || rot->pairs > D / 2) return CCV3D_ERR_UNSUPPORTED;
        int sum = 0;
        for (int a = 0; a < 3; ++a) {
            if (a < rot->axes && rot->section[a] < 0) return CCV3D_ERR_INVALID_ARG;
            if (a < rot->axes) sum += rot->section[a];
        }
        if (sum != rot->pairs) return CCV3D_ERR_INVALID_ARG;
        if (misaligned(rot->cos_table, 16) || misaligned(rot->sin_table, 16) || misaligned(rot->positions, 4)) return CCV3D_ERR_ALIGNMENT;
    }
    const Span sc = codes_span(cache), ss = scales_span(cache), sk = span_of(*k, tokens, H, D, dtype), sv = span_of(*v, tokens, H, D, dtype);
    if (meet(sc, ss) || meet(sc, sk) || meet(sc, sv) || meet(ss, sk) || meet(ss, sv)) return CCV3D_ERR_ALIAS;
    if (meets_batch(sc, batch) || meets_batch(ss, batch) || (rot && (meets_rotary(sc, rot, tokens) || meets_rotary(ss, rot, tokens)))) return CCV3D_ERR_ALIAS;
    if (q) {
        if ((s = check_heads(q, q_heads, D, dtype)) != CCV3D_OK || (s = check_heads(q_out, q_heads, D, dtype, tokens)) != CCV3D_OK) return s;
        const Span a = span_of(*q, tokens, q_heads, D, dtype), b = span_of(*q_out, tokens, q_heads, D, dtype);
        const bool self = q->data == q_out->data && q->token_stride == q_out->token_stride && q->head_stride == q_out->head_stride;
        if (!self && share(*q, q_heads, *q_out, q_heads, tokens, D, dtype)) return CCV3D_ERR_ALIAS;
        if (share(*k, H, *q_out, q_heads, tokens, D, dtype) || share(*v, H, *q_out, q_heads, tokens, D, dtype)) return CCV3D_ERR_ALIAS;
        if (meet(b, sc) || meet(b, ss) || meet(a, sc) || meet(a, ss)) return CCV3D_ERR_ALIAS;
        if (meets_batch(b, batch) || (rot && meets_rotary(b, rot, tokens))) return CCV3D_ERR_ALIAS;
    }
    Device dev;
    if ((s = current_device(&dev)) != CCV3D_OK) return s;
    AppendParams p = {};
    p.c = *cache;
    p.bt = *batch;
    p.k = *k;
    p.v = *v;
    if (q) { p.q = *q; p.qo = *q_out; p.q_heads = q_heads; }
    if (rot) {
        p.rot = *rot;
        for (int a = rot->axes; a < 3; ++a) p.rot.section[a] = 0;
    }
    p.status = status;
    return dtype == CCV3D_BF16 ? launch_append<__nv_bfloat16>(p, (cudaStream_t)stream) : launch_append<float>(p, (cudaStream_t)stream);
}

ccv3d_status ccv3d_kv_attend_workspace(const ccv3d_kv_cache* cache, const ccv3d_token_batch* batch, int32_t q_heads,
                                       int32_t dtype, uint64_t* bytes_host) {
    if (!bytes_host) return CCV3D_ERR_INVALID_ARG;
    Plan pl;
    ccv3d_status s = check_attend(cache, batch, q_heads, dtype);
    if (s == CCV3D_OK && batch->batch == 0) {
        *bytes_host = 0;
        return s;
    }
    if (s == CCV3D_OK) s = plan_attend(cache, batch, q_heads, dtype, &pl);
    if (s == CCV3D_OK) *bytes_host = pl.bytes;
    return s;
}

ccv3d_status ccv3d_kv_attend(const ccv3d_kv_cache* cache, const ccv3d_token_batch* batch, const ccv3d_heads* q,
                             const ccv3d_heads* out, float* lse, int32_t q_heads, int32_t dtype, float scale,
                             int32_t frame, int32_t window, void* ws, uint64_t ws_bytes, uint32_t* status, void* stream) {
    Plan pl;
    ccv3d_status s = check_attend(cache, batch, q_heads, dtype);
    if (s != CCV3D_OK) return s;
    if (frame < 0 || window < -1) return CCV3D_ERR_INVALID_ARG;
    if (batch->tokens == 0 || batch->max_new == 0) return CCV3D_OK;
    const int D = cache->head_dim, tokens = batch->tokens;
    if ((s = check_heads(q, q_heads, D, dtype)) != CCV3D_OK || (s = check_heads(out, q_heads, D, dtype, tokens)) != CCV3D_OK) return s;
    if (misaligned(lse, 4) || misaligned(ws, 256)) return CCV3D_ERR_ALIGNMENT;
    const Span a = span_of(*q, tokens, q_heads, D, dtype), o = span_of(*out, tokens, q_heads, D, dtype), sc = codes_span(cache), ss = scales_span(cache);
    if (meet(a, o) || meet(o, sc) || meet(o, ss) || meets_batch(o, batch)) return CCV3D_ERR_ALIAS;
    if (lse) {
        const Span l = span_of(lse, (int64_t)tokens * q_heads * 4);
        if (meet(l, a) || meet(l, o) || meet(l, sc) || meet(l, ss) || meets_batch(l, batch)) return CCV3D_ERR_ALIAS;
    }
    if (!ws || ws_bytes == 0) return CCV3D_ERR_NOMEM;
    if ((s = plan_attend(cache, batch, q_heads, dtype, &pl)) != CCV3D_OK) return s;
    if (ws_bytes < pl.bytes) return CCV3D_ERR_NOMEM;
    const Span w = span_of(ws, (int64_t)pl.bytes);
    if (meet(w, a) || meet(w, o) || meet(w, sc) || meet(w, ss) || meets_batch(w, batch)) return CCV3D_ERR_ALIAS;
    if (lse && meet(w, span_of(lse, (int64_t)tokens * q_heads * 4))) return CCV3D_ERR_ALIAS;
    AttendParams p = {};
    p.c = *cache;
    p.bt = *batch;
    p.q = *q;
    p.o = *out;
    p.lse = lse;
    p.q_heads = q_heads;
    p.group = q_heads / cache->kv_heads;
    p.scale = scale;
    p.frame = frame;
    p.window = window;
    p.status = status;
    p.wait_clk = pl.dev.wait_clk;
    p.part = (float*)ws;
    p.part_ml = (float2*)((char*)ws + pl.ml_at);
    p.join = (Join*)((char*)ws + pl.join_at);
    p.slot_rows = pl.slot_rows;
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == CCV3D_BF16)
        return D == 64 ? launch_attend<__nv_bfloat16, 64>(p, pl, st) : launch_attend<__nv_bfloat16, 128>(p, pl, st);
    return D == 64 ? launch_attend<float, 64>(p, pl, st) : launch_attend<float, 128>(p, pl, st);
}

ccv3d_status ccv3d_gated_norm(const ccv3d_norm_desc* d, const void* x, const void* y, const void* post_weight,
                              const void* post_bias, const void* gate, const void* pre_weight, const void* pre_bias,
                              const void* scale, const void* shift, void* r, void* h, void* stream) {
    if (!d || d->rows < 0 || d->channels < 1 || d->rows_per_group < 1) return CCV3D_ERR_INVALID_ARG;
    if (!dtype_ok(d->res_dtype) || !dtype_ok(d->act_dtype) || !dtype_ok(d->weight_dtype) || !dtype_ok(d->mod_dtype)) return CCV3D_ERR_INVALID_ARG;
    if (d->post_kind < 0 || d->post_kind > 2 || d->pre_kind < 0 || d->pre_kind > 2) return CCV3D_ERR_INVALID_ARG;
    if (d->channels > 16384) return CCV3D_ERR_UNSUPPORTED;
    if (d->rows == 0) return CCV3D_OK;
    if (!x || (!r && !h)) return CCV3D_ERR_INVALID_ARG;
    const int64_t C = d->channels, last = d->rows - 1, er = esize(d->res_dtype), ea = esize(d->act_dtype);
    if (d->x_stride < 0 || (y && d->y_stride < 0) || (r && d->r_stride < C) || (h && d->h_stride < C)) return CCV3D_ERR_INVALID_ARG;
    if ((gate && d->gate_stride < 0) || (scale && d->scale_stride < 0) || (shift && d->shift_stride < 0)) return CCV3D_ERR_INVALID_ARG;
    const int64_t em = esize(d->mod_dtype), ew = esize(d->weight_dtype);
    if (misaligned(x, er) || misaligned(r, er) || misaligned(y, ea) || misaligned(h, ea) || misaligned(gate, em) || misaligned(scale, em) ||
        misaligned(shift, em) || misaligned(post_weight, ew) || misaligned(post_bias, ew) || misaligned(pre_weight, ew) || misaligned(pre_bias, ew))
        return CCV3D_ERR_ALIGNMENT;
    // outputs against every input (and one another); r on x and h on y are allowed row for row
    const Span in[] = {span_of(x, (last * d->x_stride + C) * er), y ? span_of(y, (last * d->y_stride + C) * ea) : Span{0, 0},
                       span_of(post_weight, post_weight ? C * ew : 0), span_of(post_bias, post_bias ? C * ew : 0),
                       span_of(pre_weight, pre_weight ? C * ew : 0), span_of(pre_bias, pre_bias ? C * ew : 0),
                       span_of(gate, gate ? (last / d->rows_per_group * d->gate_stride + C) * em : 0),
                       span_of(scale, scale ? (last / d->rows_per_group * d->scale_stride + C) * em : 0),
                       span_of(shift, shift ? (last / d->rows_per_group * d->shift_stride + C) * em : 0)};
    const Span sr = span_of(r, r ? (last * d->r_stride + C) * er : 0), sh = span_of(h, h ? (last * d->h_stride + C) * ea : 0);
    if (r && h && meet(sr, sh)) return CCV3D_ERR_ALIAS;
    for (int i = 0; i < 9; ++i) {
        if (in[i].a == in[i].b) continue;
        if (r && meet(sr, in[i]) && !(i == 0 && r == x && d->r_stride == d->x_stride)) return CCV3D_ERR_ALIAS;
        if (h && meet(sh, in[i]) && !(i == 1 && h == y && d->h_stride == d->y_stride)) return CCV3D_ERR_ALIAS;
    }
    Device dev;
    const ccv3d_status s = current_device(&dev);
    if (s != CCV3D_OK) return s;
    NormParams p = {*d, x, y, post_weight, post_bias, gate, pre_weight, pre_bias, scale, shift, r, h};
    // four elements per access where every row and vector starts on a multiple of four
    const auto whole = [](const void* t, int64_t stride, int64_t e) { return !t || (!misaligned(t, 4 * e) && stride % 4 == 0); };
    const bool vec = C % 4 == 0 && whole(x, d->x_stride, er) && whole(y, d->y_stride, ea) && whole(r, d->r_stride, er) && whole(h, d->h_stride, ea) &&
                     whole(gate, d->gate_stride, em) && whole(scale, d->scale_stride, em) && whole(shift, d->shift_stride, em) &&
                     whole(post_weight, 0, ew) && whole(post_bias, 0, ew) && whole(pre_weight, 0, ew) && whole(pre_bias, 0, ew);
    cudaStream_t st = (cudaStream_t)stream;
    if (d->res_dtype == CCV3D_BF16)
        return d->act_dtype == CCV3D_BF16 ? launch_norm<__nv_bfloat16, __nv_bfloat16>(p, vec, dev, st) : launch_norm<__nv_bfloat16, float>(p, vec, dev, st);
    return d->act_dtype == CCV3D_BF16 ? launch_norm<float, __nv_bfloat16>(p, vec, dev, st) : launch_norm<float, float>(p, vec, dev, st);
}

}  // extern "C"
