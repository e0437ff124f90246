// Attention of many query rows (frames, prompts) over the paged E4M3 cache, on tcgen05.
//
// Bound by the tensor cores.  An item is a block of 256 query rows of one kv head (F32: 128), rows being (token, head of
// the group) so that grouped heads share the keys they share; a unit is 128 cached tokens.  12 warps (at 168 registers), one block to an SM:
//   warps 0-3, 4-7   softmax of the first and second 128 rows, a thread to a row: scores from TMEM, weights back as halves
//                    over them, sums in registers, the output from TMEM at the end; they also stage the queries
//   warps 8-10       fetch pages and turn codes into halves in shared memory (exact), keys and values in two slots each
//   warp 11          issues the MMAs: S = Q K^T from shared memory, O += P V with P in TMEM
// Two row blocks in turn keep the tensor cores busy: while one is in its softmax the other's products run.
//
// Keys and values are staged alike, rows of 64 channels (128 bytes, 128-byte swizzle) token by token: K-major for the
// scores and, read the other way, MN-major for the outputs.  The softmax maximum is only raised when a score passes it
// by more than 2^7 (then the sums in TMEM are scaled down): weights stay under 2^15 and a tile needs one pass.
// For F32 queries and weights go in as two halves each (value and remainder): about 22 bits, at twice the MMAs.
#pragma once
#include "ccv3d_tokens_attend_step.cuh"

namespace ccv3d {

constexpr int TILE_UNIT = 128, TILE_THREADS = 384, TILE_BATCH = 1024;
constexpr float TILE_SHIFT = 8.f, TILE_TOP = 15.f;      // weights start at 2^8 for the maximum and may reach 2^15

template <typename T, int D> struct TileShape {
    static constexpr int TERMS = sizeof(T) == 4 ? 2 : 1, NQ = sizeof(T) == 4 ? 1 : 2, ROWS = 128 * NQ;
    static constexpr uint32_t HALF = 128 * 128;                       // 128 rows of 64 channels
    static constexpr uint32_t KV = HALF * (D / 64), Q = KV * TERMS;   // one staged tile; one row block's queries
    static constexpr uint32_t Q_AT = 0, K_AT = NQ * Q, V_AT = K_AT + 2 * KV, END = V_AT + 2 * KV;
    // TMEM columns: scores (and weights over them) of the row blocks, then outputs; F32 has weights of its own
    static constexpr uint32_t S_COL = 0, P_COL = NQ == 2 ? 0 : 128, O_COL = 256;
};

struct TileShared {
    float4 group[4][8];      // per staged tile and 16 tokens: key scale, log2 and reciprocal of the value scale
    int cost[TILE_BATCH];    // units of a sequence
    uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], q_full[2], s_full[2], p_full[2], o_full[2], o_empty[2];
    uint32_t tmem;
    int abort_flag, nan_found;
};

// An item: rows row0 .. row0 + nrows - 1 of sequence s, kv head h, cached tokens [lo, hi) that any of its rows sees,
// [lo_all, hi_all) that all of them see.
struct TileItem { int row0, nrows, lo, hi, lo_all, hi_all, base, units; };

template <int ROWS>
__device__ __forceinline__ TileItem tile_item(const AttendParams& p, const Seq& s, int rb) {
    TileItem t;
    const int rows = s.n * p.group;
    t.row0 = rb * ROWS;
    t.nrows = min(ROWS, rows - t.row0);
    const int first = s.total - s.n + t.row0 / p.group, last = s.total - s.n + (t.row0 + t.nrows - 1) / p.group;
    int skip;
    t.lo = t.hi = t.lo_all = t.hi_all = 0;
    if (last >= 0) {
        visible(p, max(first, 0), s.total, t.lo, skip);
        visible(p, last, s.total, t.lo_all, t.hi);
        visible(p, first, s.total, skip, t.hi_all);
    }
    t.base = t.lo / TILE_UNIT * TILE_UNIT;
    t.units = max(1, (t.hi - t.base + TILE_UNIT - 1) / TILE_UNIT);
    return t;
}

// The walk over a block's share: segments of items, the same for every role.
template <int ROWS>
struct TileWalk {
    int u, u1, b, rb, h, unit;
    int64_t total, blocks;
    Seq s;
    TileItem t;
    __device__ __forceinline__ bool done() const { return u >= u1; }
    __device__ __forceinline__ int length() const { return min(t.units - unit, u1 - u); }       // units of this segment
    __device__ __forceinline__ void next(const AttendParams& p) {
        u += length();
        if (u >= u1) return;
        unit = 0;
        if (++h < p.c.kv_heads) return;
        h = 0;
        if ((++rb) * ROWS >= s.n * p.group) {
            rb = 0;
            do {
                if (++b >= p.bt.batch) { u1 = u; return; }          // (only if the arrays changed under the kernel)
                s = load_seq(p.bt, p.c.page_tokens, b, nullptr);
            } while (s.n == 0);
        }
        t = tile_item<ROWS>(p, s, rb);
    }
};

// Finds this block's share.  All threads of the block call it: costs of up to TILE_BATCH sequences at a time, a warp each.
template <int ROWS>
__device__ __forceinline__ TileWalk<ROWS> tile_share(const AttendParams& p, TileShared* sh) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    TileWalk<ROWS> w;
    w.u = w.u1 = w.b = w.rb = w.h = w.unit = 0;
    w.total = 0;
    w.s = {0, 0, 0};
    w.t = {0, 0, 0, 0, 0, 0, 0, 0};
    bool found = false;
    int64_t before = 0;
    for (int pass = 0; pass < 2; ++pass) {
        for (int c0 = 0; c0 < p.bt.batch; c0 += TILE_BATCH) {
            const int n = min(TILE_BATCH, p.bt.batch - c0);
            if (pass == 0 || p.bt.batch > TILE_BATCH) {
                __syncthreads();
                for (int b = warp; b < n; b += warps) {
                    const Seq s = load_seq(p.bt, p.c.page_tokens, c0 + b, pass == 0 ? p.status : nullptr);
                    const int blocks = (s.n * p.group + ROWS - 1) / ROWS;
                    int units = 0;
                    for (int rb = lane; rb < blocks; rb += 32) units += tile_item<ROWS>(p, s, rb).units;
                    units = __reduce_add_sync(0xffffffffu, units);
                    if (lane == 0) sh->cost[b] = units * p.c.kv_heads;
                }
                __syncthreads();
            }
            for (int b0 = 0; b0 < n && !found; b0 += 32) {
                const int mine = b0 + lane < n ? sh->cost[b0 + lane] : 0;
                const int upto = warp_scan(mine), all = __shfl_sync(0xffffffffu, upto, 31);
                if (pass == 0) { w.total += all; continue; }
                const unsigned hit = __ballot_sync(0xffffffffu, mine > 0 && (int64_t)w.u < before + upto);
                if (!hit) { before += all; continue; }
                const int who = __ffs(hit) - 1;
                int at = w.u - (int)(before + __shfl_sync(0xffffffffu, upto - mine, who));
                w.b = c0 + b0 + who;
                w.s = load_seq(p.bt, p.c.page_tokens, w.b, nullptr);
                const int blocks = (w.s.n * p.group + ROWS - 1) / ROWS;
                for (int r0 = 0; r0 < blocks && !found; r0 += 32) {
                    const int cost = r0 + lane < blocks ? tile_item<ROWS>(p, w.s, r0 + lane).units * p.c.kv_heads : 0;
                    const int to = warp_scan(cost);
                    const unsigned in = __ballot_sync(0xffffffffu, cost > 0 && at < to);
                    if (!in) { at -= __shfl_sync(0xffffffffu, to, 31); continue; }
                    const int r = __ffs(in) - 1;
                    at -= __shfl_sync(0xffffffffu, to - cost, r);
                    w.rb = r0 + r;
                    w.t = tile_item<ROWS>(p, w.s, w.rb);
                    w.h = at / w.t.units;
                    w.unit = at % w.t.units;
                    found = true;
                }
            }
        }
        if (pass == 0) {
            w.blocks = min((int64_t)gridDim.x, w.total);
            if ((int64_t)blockIdx.x < w.blocks) {
                w.u = (int)(w.total * blockIdx.x / w.blocks);
                w.u1 = (int)(w.total * (blockIdx.x + 1) / w.blocks);
            }
            found = w.done();                                       // (nothing to look for)
        }
    }
    if (!found) w.u1 = w.u;
    return w;
}

// Bounded wait; false when it gave up or another role did.
__device__ __forceinline__ bool tile_wait(uint64_t* bar, uint32_t parity, TileShared* sh, const AttendParams& p) {
    const uint32_t b = smem_u32(bar);
    if (mbar_try_wait(b, parity)) return true;
    long long since = 0;
    for (uint32_t it = 1;; ++it) {
        if (mbar_try_wait(b, parity)) return true;
        if ((it & 63u) == 0u) {
            if (*(volatile int*)&sh->abort_flag) return false;
            const long long now = clock64();
            if (!since) since = now;
            else if (now - since > p.wait_clk) {
                *(volatile int*)&sh->abort_flag = 1;
                report(p.status, CCV3D_TOKENS_TIMEOUT);
                return false;
            }
        }
    }
}

__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, TileShared* sh, const AttendParams& p) {
    return __all_sync(0xffffffffu, tile_wait(bar, parity, sh, p));
}

// upper word of a shared-memory operand descriptor: stride-dimension offset, version 1, 128-byte swizzle
__device__ __forceinline__ uint32_t tile_desc_hi(uint32_t sbo) { return ((sbo >> 4) & 0x3FFFu) | (1u << 14) | (2u << 29); }

__device__ __forceinline__ void tc_mma_f16_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 da, {%1, %3};\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(acc)
        : "memory");
}
__device__ __forceinline__ void tc_mma_f16_ts(uint32_t d, uint32_t a_tmem, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}" ::"r"(d), "r"(a_tmem), "r"(b_lo), "r"(hi), "r"(idesc), "r"(acc)
        : "memory");
}
template <int N>
__device__ __forceinline__ void tc_st(uint32_t taddr, const uint32_t* v) {
    static_assert(N == 16 || N == 32, "");
    if constexpr (N == 32)
        asm volatile(
            "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
            "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
            "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
            "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]),
            "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]),
            "r"(v[31])
            : "memory");
    else
        asm volatile(
            "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
            "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
            "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
            : "memory");
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// What a softmax thread knows of its row.
struct TileRow {
    int lo, hi;              // cached tokens it sees
    float factor;            // of its scores: softmax scale, log2(e), the power of two taken off its queries
    int token, head;         // packed token, query head; token < 0: no row
};

// Stages the queries of one row (each thread its own) and returns what the row needs to know.
template <typename T, int D, int ROWS>
__device__ __forceinline__ TileRow stage_row(const AttendParams& p, const TileWalk<ROWS>& w, int r, int tid, uint8_t* q) {
    using S = TileShape<T, D>;
    TileRow row = {0, 0, 0.f, -1, 0};
    float most = 0.f;
    const T* src = nullptr;
    if (r < w.t.nrows) {
        const int at = w.t.row0 + r;
        row.token = w.s.first + at / p.group;
        row.head = w.h * p.group + at % p.group;
        visible(p, w.s.total - w.s.n + at / p.group, w.s.total, row.lo, row.hi);
        src = (const T*)p.q.data + row.token * p.q.token_stride + row.head * p.q.head_stride;
    }
    if constexpr (sizeof(T) == 2) {
        uint4 x[D / 8];
#pragma unroll
        for (int i = 0; i < D / 8; ++i) x[i] = src ? *reinterpret_cast<const uint4*>(src + 8 * i) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            const uint32_t e[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k)
                most = fmaxf(most, fmaxf(fabsf(__uint_as_float(e[k] << 16)), fabsf(__uint_as_float(e[k] & 0xFFFF0000u))));
        }
        float down, up;
        row_power(most, down, up);
        row.factor = up * (p.scale * LOG2E);
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            const uint32_t e[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
            uint32_t y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = pack_half(__uint_as_float(e[k] << 16) * down, __uint_as_float(e[k] & 0xFFFF0000u) * down);
            *reinterpret_cast<uint4*>(q + (i / 8) * S::HALF + tid * 128 + ((i % 8) ^ (tid & 7)) * 16) = make_uint4(y[0], y[1], y[2], y[3]);
        }
    } else {
        for (int i = 0; i < D / 4; ++i) {
            float x[4] = {0.f, 0.f, 0.f, 0.f};
            if (src) load4(src + 4 * i, x);
            most = fmaxf(fmaxf(most, fmaxf(fabsf(x[0]), fabsf(x[1]))), fmaxf(fabsf(x[2]), fabsf(x[3])));
        }
        float down, up;
        row_power(most, down, up);
        row.factor = up * (p.scale * LOG2E);
        for (int i = 0; i < D / 8; ++i) {
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = 0.f;
            if (src) {
                float a[4];
                load4(src + 8 * i, a);
                x[0] = a[0]; x[1] = a[1]; x[2] = a[2]; x[3] = a[3];
                load4(src + 8 * i + 4, a);
                x[4] = a[0]; x[5] = a[1]; x[6] = a[2]; x[7] = a[3];
            }
            uint32_t y[4], z[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                y[k] = pack_half(x[2 * k] * down, x[2 * k + 1] * down);
                z[k] = pack_rest(x[2 * k] * down, x[2 * k + 1] * down, y[k]);
            }
            uint8_t* dst = q + (i / 8) * S::HALF + tid * 128 + ((i % 8) ^ (tid & 7)) * 16;
            *reinterpret_cast<uint4*>(dst) = make_uint4(y[0], y[1], y[2], y[3]);
            *reinterpret_cast<uint4*>(dst + S::KV) = make_uint4(z[0], z[1], z[2], z[3]);
        }
    }
    return row;
}

// One tile's scores to weights.  On return l holds the row's weight sum, mx the largest exponent met (before the shift's
// bound is checked); pr the packed weights (BF16), or they lie in TMEM already (F32).
template <typename T, bool EDGE>
__device__ __forceinline__ float tile_weights(uint32_t t_s, uint32_t t_p, const float4* group, const TileRow& row, float m_use, int t0,
                                              uint32_t (&pr)[64], float& sum) {
    float mx = -INFINITY;
    sum = 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        uint32_t v[32];
        tc_ld32(t_s + 32 * c, v);
        tc_wait_ld();
        uint32_t lo16[16], hi16[16];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const float4 k = group[2 * c + g];
            const float f = k.x * row.factor, a = k.y - m_use;
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                float t[2], e[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    t[j] = fmaf(__uint_as_float(v[16 * g + i + j]), f, a);
                    if (EDGE) {
                        const int at = t0 + 32 * c + 16 * g + i + j;
                        if (at < row.lo || at >= row.hi || k.y == -INFINITY) t[j] = -INFINITY;
                    }
                    mx = fmaxf(mx, t[j]);
                    e[j] = exp2_fast(t[j]);
                    part += e[j];
                }
                const uint32_t h = pack_half(e[0], e[1]);
                if constexpr (sizeof(T) == 2) pr[16 * c + 8 * g + i / 2] = h;
                else { hi16[8 * g + i / 2] = h; lo16[8 * g + i / 2] = pack_rest(e[0], e[1], h); }
            }
            sum = fmaf(part, k.z, sum);
        }
        if constexpr (sizeof(T) == 4) {
            tc_st<16>(t_p + 16 * c, hi16);
            tc_st<16>(t_p + 64 + 16 * c, lo16);
        }
    }
    return mx;
}

template <typename T, int D>
__global__ void __launch_bounds__(TILE_THREADS, 1) kv_attend_tile_kernel(const AttendParams p) {
    using S = TileShape<T, D>;
    constexpr int ROWS = S::ROWS, NQ = S::NQ, TERMS = S::TERMS;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    TileShared* sh = reinterpret_cast<TileShared*>(smem + S::END);
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int P = p.c.page_tokens, H = p.c.kv_heads;

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh->k_full[i]), 3); mbar_init(smem_u32(&sh->k_empty[i]), 1);
            mbar_init(smem_u32(&sh->v_full[i]), 3); mbar_init(smem_u32(&sh->v_empty[i]), 1);
            mbar_init(smem_u32(&sh->q_full[i]), 4); mbar_init(smem_u32(&sh->s_full[i]), 1);
            mbar_init(smem_u32(&sh->p_full[i]), 4); mbar_init(smem_u32(&sh->o_full[i]), 1);
            mbar_init(smem_u32(&sh->o_empty[i]), 4);
        }
        sh->abort_flag = 0;
        sh->nan_found = 0;
        p.join[blockIdx.x] = {0, 0, 0, 0};
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 11) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    TileWalk<ROWS> w = tile_share<ROWS>(p, sh);      // (synchronises the block)
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem;
    bool ok = true;

    if (warp < 4 * NQ) {
        // ------------------------------------------------------------------------------------------ softmax
        const int qt = warp >> 2, tid = threadIdx.x & 127;
        uint8_t* q = smem + S::Q_AT + qt * S::Q;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + lanes + S::S_COL + qt * 128, t_p = tmem + lanes + S::P_COL + qt * 128;
        const uint32_t t_o = tmem + lanes + S::O_COL + qt * D;
        uint32_t s_ph = 0, o_ph = 0;
        int tile = 0;                                // tiles staged so far, over all segments (for the group ring)
        auto mine = [&](const TileWalk<ROWS>& x) { return !x.done() && x.t.nrows > 128 * qt; };
        auto stage = [&](const TileWalk<ROWS>& x) {
            const TileRow r = stage_row<T, D, ROWS>(p, x, 128 * qt + tid, tid, q);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->q_full[qt]));
            return r;
        };
        TileRow row = {0, 0, 0.f, -1, 0};
        bool staged = false;
        while (ok && !w.done()) {
            const int n = w.length();
            if (!mine(w)) { tile += n; w.next(p); continue; }
            if (!staged) row = stage(w);
            float m = -INFINITY, l = 0.f;
            for (int i = 0; i < n; ++i, ++tile) {
                if (!(ok = warp_wait(&sh->s_full[qt], s_ph, sh, p))) break;
                s_ph ^= 1;
                tc_fence_after();
                const int t0 = w.t.base + (w.unit + i) * TILE_UNIT;
                const float4* group = sh->group[tile & 3];
                bool edge = t0 < w.t.lo_all || t0 + TILE_UNIT > w.t.hi_all;
#pragma unroll
                for (int g = 0; g < 8; ++g) edge = edge || group[g].w != 0.f;      // (a page that is not there)
                uint32_t pr[64];
                float sum, m_use = (m == -INFINITY ? 0.f : m) - TILE_SHIFT;
                float mx = edge ? tile_weights<T, true>(t_s, t_p, group, row, m_use, t0, pr, sum)
                                : tile_weights<T, false>(t_s, t_p, group, row, m_use, t0, pr, sum);
                const bool raise = mx > TILE_TOP || (m == -INFINITY && mx > -INFINITY);
                if (__any_sync(0xffffffffu, raise)) {
                    if (sizeof(T) == 4) tc_wait_st();
                    const float now = fmaxf(m, mx + m_use);                      // (mx = -inf leaves m)
                    const float corr = m == -INFINITY ? 0.f : exp2_fast(m - now);
                    if (i > 0)                                                   // (the scores' arrival says that the last sum is complete)
                        for (int c = 0; c < D; c += 32) {
                            uint32_t v[32];
                            tc_ld32(t_o + c, v);
                            tc_wait_ld();
#pragma unroll
                            for (int k = 0; k < 32; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * corr);
                            tc_st<32>(t_o + c, v);
                        }
                    l *= corr;
                    m = now;
                    m_use = (m == -INFINITY ? 0.f : m) - TILE_SHIFT;
                    if (edge) tile_weights<T, true>(t_s, t_p, group, row, m_use, t0, pr, sum);
                    else tile_weights<T, false>(t_s, t_p, group, row, m_use, t0, pr, sum);
                }
                l += sum;
                if constexpr (sizeof(T) == 2) {
                    tc_st<32>(t_p, pr);
                    tc_st<32>(t_p + 32, pr + 32);
                }
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->p_full[qt]));
            }
            if (!ok) break;
            // the next segment's queries go in before this one's output is complete
            TileWalk<ROWS> nx = w;
            nx.next(p);
            staged = mine(nx);
            TileRow nrow = row;
            if (staged) nrow = stage(nx);
            if (!(ok = warp_wait(&sh->o_full[qt], o_ph, sh, p))) break;
            o_ph ^= 1;
            tc_fence_after();
            const bool starts = w.unit == 0, ends = w.unit + n == w.t.units, whole = starts && ends;
            const int64_t slot = (2 * (int64_t)blockIdx.x + (starts ? 1 : 0)) * p.slot_rows + 128 * qt + tid;
            const float inv = l != 0.f ? 1.f / l : 0.f;
            const bool nan = *(volatile int*)&sh->nan_found != 0;
            for (int c = 0; c < D; c += 32) {
                uint32_t v[32];
                tc_ld32(t_o + c, v);
                tc_wait_ld();
                if (nan) {
                    // values that are NaN were staged as zeros where some rows do not see them: find those this row sees
                    for (int i = 0; i < n; ++i) {
                        const int t0 = w.t.base + (w.unit + i) * TILE_UNIT;
                        if (t0 >= w.t.lo_all && t0 + TILE_UNIT <= w.t.hi_all) continue;
                        for (int t = max(t0, row.lo); t < min(t0 + TILE_UNIT, row.hi); ++t) {
                            const int page = load_page(p.bt, p.c, w.b, t / P, nullptr);
                            if (page < 0) continue;
                            const uint8_t* src = (const uint8_t*)p.c.codes + ((((int64_t)page * 2 + 1) * H + w.h) * P + t % P) * D + c;
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if ((src[k] & 0x7F) == 0x7F) v[k] = 0x7FFFFFFFu;
                        }
                    }
                }
                if (row.token >= 0) {
#pragma unroll
                    for (int k = 0; k < 32; k += 4) {
                        float x[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(v[k + e]);
                        if (whole) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) x[e] = l != 0.f ? x[e] * inv : 0.f;
                            store_out<T>(p, row.token, row.head, c + k, x);
                        } else {
                            store4(p.part + slot * D + c + k, x);
                        }
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->o_empty[qt]));
            if (row.token >= 0) {
                if (!whole) p.part_ml[slot] = make_float2(m, l);
                else if (p.lse) p.lse[(int64_t)row.token * p.q_heads + row.head] = lse_of(m, l, TILE_SHIFT);
            }
            if (starts && !ends && threadIdx.x == 0) {
                const int64_t x = (int64_t)w.u + w.t.units - 1;               // the item's last unit, and the block that takes it
                const int z = (int)(((x + 1) * w.blocks - 1) / w.total);
                p.join[blockIdx.x] = {z - (int)blockIdx.x + 1, w.s.first * p.group + w.t.row0, w.t.nrows, w.h * p.group};
            }
            row = nrow;
            w = nx;
        }
    } else if (warp >= 8 && warp < 11) {
        // ------------------------------------------------------------------------------------------ codes to halves
        // a warp moves eight rows by 64 codes at a time, a thread 16 of a row, so that the eight lanes of a store phase
        // meet eight different banks; the pieces of a tile go around the three warps
        const int cw = warp - 8, rl = lane >> 2, piece = lane & 3;
        constexpr int HALVES = D / 64, PIECES = 16 * HALVES, ROUNDS = (PIECES + 2) / 3;
        uint32_t ks = 0, kp = 1, vs = 0, vp = 1;                                // slots and parities (the first use passes at once)
        int tile = 0;
        // pages and scales of a tile: lane g < 8 holds those of its 16 tokens [16 g, 16 g + 16)
        auto find = [&](const TileWalk<ROWS>& x, int unit) {
            int page = -1;
            const int th = x.t.base + unit * TILE_UNIT + (lane & 7) * 16;
            if (th < x.t.hi && th + 16 > x.t.lo) page = load_page(p.bt, p.c, x.b, th / P, lane < 8 && cw == 0 ? p.status : nullptr);
            return page;
        };
        auto fetch = [&](const TileWalk<ROWS>& x, int unit, int page, int j, uint4 (&raw)[ROUNDS]) {
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r) {
                const int u = 3 * r + cw, at = u / HALVES * 8 + rl, t = x.t.base + unit * TILE_UNIT + at;
                const int pg = __shfl_sync(0xffffffffu, page, (u / HALVES / 2) & 7);
                raw[r] = make_uint4(0, 0, 0, 0);
                if (u < PIECES && pg >= 0 && t >= x.t.lo && t < x.t.hi)
                    raw[r] = __ldg(reinterpret_cast<const uint4*>((const uint8_t*)p.c.codes + ((((int64_t)pg * 2 + j) * H + x.h) * P + t % P) * D + u % HALVES * 64 + piece * 16));
            }
        };
        auto put = [&](uint8_t* dst, const uint4 (&raw)[ROUNDS]) {
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r) {
                const int u = 3 * r + cw, at = u / HALVES * 8 + rl;
                if (u >= PIECES) break;
                const uint32_t c[4] = {raw[r].x, raw[r].y, raw[r].z, raw[r].w};
                uint32_t y[8];
#pragma unroll
                for (int k = 0; k < 4; ++k) { y[2 * k] = e4m3x2_to_half2(c[k] & 0xFFFFu); y[2 * k + 1] = e4m3x2_to_half2(c[k] >> 16); }
                uint8_t* line = dst + u % HALVES * S::HALF + at * 128;
                *reinterpret_cast<uint4*>(line + ((2 * piece) ^ (at & 7)) * 16) = make_uint4(y[0], y[1], y[2], y[3]);
                *reinterpret_cast<uint4*>(line + ((2 * piece + 1) ^ (at & 7)) * 16) = make_uint4(y[4], y[5], y[6], y[7]);
            }
        };
        uint4 kraw[ROUNDS], vraw[ROUNDS];
        int unit = w.unit, left = w.done() ? 0 : w.length(), page = -1;
        if (left) { page = find(w, unit); fetch(w, unit, page, 0, kraw); }
        while (ok && left) {
            // what comes after this tile
            TileWalk<ROWS> nx = w;
            int nunit = unit + 1, nleft = left - 1;
            if (!nleft) {
                nx.next(p);
                nunit = nx.unit;
                nleft = nx.done() ? 0 : nx.length();
            }
            const int npage = nleft ? find(nx, nunit) : -1;
            fetch(w, unit, page, 1, vraw);
            if (cw == 0 && lane < 8) {
                float4 g = make_float4(0.f, -INFINITY, 0.f, 1.f);                // not there: weighs nothing
                const int th = w.t.base + unit * TILE_UNIT + lane * 16;
                if (page >= 0) {
                    g.x = __ldg(p.c.scales + (int64_t)page * 2 * H + w.h);
                    scale_terms(__ldg(p.c.scales + ((int64_t)page * 2 + 1) * H + w.h), g.y, g.z);
                    g.w = 0.f;
                } else if (th >= w.t.hi || th + 16 <= w.t.lo) g.w = 0.f;         // masked anyway
                sh->group[tile & 3][lane] = g;
            }
            if (!(ok = warp_wait(&sh->k_empty[ks], kp, sh, p))) break;
            put(smem + S::K_AT + ks * S::KV, kraw);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->k_full[ks]));
            if (++ks == 2) { ks = 0; kp ^= 1; }
            if (nleft) fetch(nx, nunit, npage, 0, kraw);
            // NaN values that not every row of the item sees: staged as zeros, put in place at the end
            const int t0 = w.t.base + unit * TILE_UNIT;
            if (t0 < w.t.lo_all || t0 + TILE_UNIT > w.t.hi_all) {
                bool any = false;
#pragma unroll
                for (int r = 0; r < ROUNDS; ++r) {
                    uint32_t* c = reinterpret_cast<uint32_t*>(&vraw[r]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t n4 = __vcmpeq4(c[k] & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
                        any = any || n4;
                        c[k] &= ~n4;
                    }
                }
                if (any) *(volatile int*)&sh->nan_found = 1;
            }
            if (!(ok = warp_wait(&sh->v_empty[vs], vp, sh, p))) break;
            put(smem + S::V_AT + vs * S::KV, vraw);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->v_full[vs]));
            if (++vs == 2) { vs = 0; vp ^= 1; }
            ++tile;
            w = nx; unit = nunit; left = nleft; page = npage;
        }
    } else if (warp == 11) {
        // ------------------------------------------------------------------------------------------ MMAs
        // D = F32, A = B = F16; scores: both K-major; outputs: A in TMEM, B MN-major (bit 16)
        constexpr uint32_t I_S = (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
        constexpr uint32_t I_O = (1u << 4) | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);
        const uint32_t hi = tile_desc_hi(1024);
        const uint32_t q_lo = ((smem_u32(smem + S::Q_AT) & 0x3FFFFu) >> 4) | (1u << 16);
        const uint32_t k_lo = ((smem_u32(smem + S::K_AT) & 0x3FFFFu) >> 4) | (1u << 16);
        const uint32_t v_lo = ((smem_u32(smem + S::V_AT) & 0x3FFFFu) >> 4) | ((S::HALF >> 4) << 16);
        uint32_t ks = 0, kp = 0, vs = 0, vp = 0, q_ph = 0, p_ph[2] = {0, 0}, o_ph[2] = {1, 1}, q1_ph = 0;
        auto scores = [&](int qt, uint32_t slot) {
            if (elect_one()) {
                const uint32_t a0 = q_lo + qt * (S::Q >> 4), b0 = k_lo + slot * (S::KV >> 4), d = tmem + S::S_COL + qt * 128;
#pragma unroll
                for (int t = 0; t < TERMS; ++t)
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off = (k / 4) * (S::HALF >> 4) + (k % 4) * 2;
                        tc_mma_f16_ss(d, a0 + t * (S::KV >> 4) + off, b0 + off, hi, I_S, t + k > 0);
                    }
                tc_commit(smem_u32(&sh->s_full[qt]));
            }
            __syncwarp();
        };
        auto outputs = [&](int qt, uint32_t slot, bool first) {
            if (elect_one()) {
                const uint32_t b0 = v_lo + slot * (S::KV >> 4), d = tmem + S::O_COL + qt * D, a0 = tmem + S::P_COL + qt * 128;
#pragma unroll
                for (int t = 0; t < TERMS; ++t)
#pragma unroll
                    for (int k = 0; k < 8; ++k) tc_mma_f16_ts(d, a0 + 64 * t + 8 * k, b0 + k * (2048 >> 4), hi, I_O, !first || t + k > 0);
            }
            __syncwarp();
        };
        auto commit = [&](uint64_t* bar) {
            if (elect_one()) tc_commit(smem_u32(bar));
            __syncwarp();
        };
        while (ok && !w.done()) {
            const int n = w.length(), nq = w.t.nrows > 128 ? 2 : 1;
            if (!(ok = warp_wait(&sh->q_full[0], q_ph, sh, p))) break;
            q_ph ^= 1;
            if (nq == 2) {
                if (!(ok = warp_wait(&sh->q_full[1], q1_ph, sh, p))) break;
                q1_ph ^= 1;
            }
            if (!(ok = warp_wait(&sh->k_full[ks], kp, sh, p))) break;
            tc_fence_after();
            for (int qt = 0; qt < nq; ++qt) scores(qt, ks);
            commit(&sh->k_empty[ks]);
            if (++ks == 2) { ks = 0; kp ^= 1; }
            for (int i = 0; ok && i < n; ++i) {
                for (int qt = 0; ok && qt < nq; ++qt) {
                    if (i == 0) {
                        if (!(ok = warp_wait(&sh->o_empty[qt], o_ph[qt], sh, p))) break;
                        o_ph[qt] ^= 1;
                    }
                    if (qt == 0 && !(ok = warp_wait(&sh->v_full[vs], vp, sh, p))) break;
                    if (!(ok = warp_wait(&sh->p_full[qt], p_ph[qt], sh, p))) break;
                    p_ph[qt] ^= 1;
                    tc_fence_after();
                    outputs(qt, vs, i == 0);
                    if (qt == nq - 1) commit(&sh->v_empty[vs]);
                    if (i + 1 < n) {
                        if (qt == 0) {
                            if (!(ok = warp_wait(&sh->k_full[ks], kp, sh, p))) break;
                            tc_fence_after();
                        }
                        scores(qt, ks);
                        if (qt == nq - 1) commit(&sh->k_empty[ks]);
                    } else {
                        commit(&sh->o_full[qt]);
                    }
                }
                if (i + 1 < n && ++ks == 2) { ks = 0; kp ^= 1; }
                if (++vs == 2) { vs = 0; vp ^= 1; }
            }
            w.next(p);
        }
    }
    if (!ok) {                                       // MMAs still reading shared memory
        const long long t = clock64();
        while (clock64() - t < 400000) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 11) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

}  // namespace ccv3d
