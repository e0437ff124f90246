// Attention of few query rows (single and drafted tokens) over the paged E4M3 cache.
//
// Bound by the cache's bytes.  Four warps to a block, three blocks to an SM where registers allow (64 streams,
// 8 rows, 146 us at two and 122 at three); a unit is 128 cached tokens of one kv head and
// each warp streams its own 32 of them: keys and values arrive by TMA in a ring of stages that only this warp fills and
// drains, so nothing but the end of an item synchronises the block.  Codes turn into halves (exactly) in registers and
// go straight into mma.sync: scores as K Q^T with the cached tokens as M and up to 8 query rows as N, outputs as V^T P
// with the head's channels as M.  The order of a contraction is free, so each thread takes whole 16-byte pieces of a
// row; the TMA swizzle keeps those reads off one another's banks.
// For F32 the queries and the weights go in as two halves each (value and remainder): about 22 bits.  The tensor cores cut each
// sum they add to instead of rounding it, which over some thousand tokens shrinks the outputs by several 1e-6: products of 16
// tokens start from zero and are added to the rest with rounding.
//
// Measured (BF16): 64 streams, 612 MB of cache, 120 us = 5.1 TB/s, 78 % of the copy rate; one stream of 269 MB, 60 us =
// 4.5 TB/s, of which some 8 us are the start and the join.  What holds it is the latency of a warp's dependent
// instructions (0.47 of a scheduler's slots are used, the tensor pipe 17 % of the time), not one unit.
#pragma once
#include "ccv3d_tokens_attend.cuh"

namespace ccv3d {

// Blocks on an SM.  Three where the registers allow; for F32 and heads of 128 they would spill (64 streams of 8000 tokens 234 us against
// 229 with two blocks, one of 131000 74.5 against 69), and so they would with 16 rows.
constexpr int step_blocks(bool f32, int dim, int rows) { return rows == 8 && !(f32 && dim == 128) ? 3 : 2; }
constexpr int STEP_WARPS = 4, STEP_TILE = 32, STEP_UNIT = STEP_WARPS * STEP_TILE;

template <int D> struct StepShape {
    static constexpr int STAGES = D == 128 ? 2 : 4;
    static constexpr uint32_t HALF = STEP_TILE * D, STAGE = 2 * HALF;             // keys, then values
    static constexpr uint32_t RING = STEP_WARPS * STAGES * STAGE;
    static constexpr uint32_t MERGE = STEP_WARPS / 2 * 8 * D * 4;                 // sums of 8 rows of two warps
    static constexpr uint32_t BYTES = RING + MERGE + STEP_WARPS * (STAGES * (8 + 8 + 16) + 16 * 8) + 64;
};

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* tm, uint32_t bar, int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(tm), "r"(c0), "r"(c1), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {     // an 8 x 8 matrix of halves over the warp
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 t = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}
__device__ __forceinline__ float2 unpack_half(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
// What is left of two floats after their halves were taken (infinities and NaN leave nothing more to add)
__device__ __forceinline__ uint32_t pack_rest(float lo, float hi, uint32_t taken) {
    const float2 t = unpack_half(taken);
    const float a = lo - t.x, b = hi - t.y;
    return pack_half(fabsf(a) <= 65504.f ? a : 0.f, fabsf(b) <= 65504.f ? b : 0.f);
}
// Power of two that brings the row's largest magnitude into [2^14, 2^15), and its reciprocal.  The halves' range lies below: an
// element is off by 2^-40 of the row's largest at most (F32: or 2^-22 of itself), and BF16 ones are exact down to 2^-31 of it.  Rows under
// 2^-112 come as near as powers of two go, beside an infinity every finite number stays finite; a NaN is not counted.
__device__ __forceinline__ void row_power(float most, float& down, float& up) {
    const int d = min(14 + 127 - (int)(__float_as_uint(most) >> 23), 126);
    down = __uint_as_float((uint32_t)(127 + d) << 23);
    up = __uint_as_float((uint32_t)(127 - d) << 23);
}

// A walk over the units of a block's share of the list.  Every member is the same for all lanes.
struct StepWalk {
    int u, u1;               // next unit, end of the share
    int64_t total, blocks;   // units of the whole list, blocks that share it
    int b, h, rb, rbs;       // sequence, kv head, row block, row blocks of the sequence (an item: row blocks fastest)
    int unit, units;         // next unit of the item, its units
    int lo, hi, base;        // cached tokens that any row of the sequence sees; first token of unit 0
    Seq s;

    // geometry of sequence b: items and units
    __device__ __forceinline__ static void measure(const AttendParams& p, int rows_per_item, const Seq& s, int& items, int& units, int& lo, int& hi) {
        lo = hi = 0;
        if (s.n > 0) {
            int t;
            visible(p, max(0, s.total - s.n), s.total, lo, t);
            visible(p, s.total - 1, s.total, t, hi);
        }
        units = max(1, (hi - lo / STEP_UNIT * STEP_UNIT + STEP_UNIT - 1) / STEP_UNIT);
        items = (int)(((int64_t)s.n * p.group + rows_per_item - 1) / rows_per_item) * p.c.kv_heads;
    }
    __device__ __forceinline__ void enter(const AttendParams& p, int rows_per_item) {
        int items;
        measure(p, rows_per_item, s, items, units, lo, hi);
        rbs = items / p.c.kv_heads;
        base = lo / STEP_UNIT * STEP_UNIT;
    }
    __device__ __forceinline__ bool done() const { return u >= u1; }
    __device__ __forceinline__ void next(const AttendParams& p, int rows_per_item) {
        if (++u >= u1) return;
        if (++unit < units) return;
        unit = 0;
        if (++rb < rbs) return;
        rb = 0;
        if (++h < p.c.kv_heads) return;
        h = 0;
        do {
            if (++b >= p.bt.batch) { u1 = u; return; }      // (only if the arrays changed under the kernel)
            s = load_seq(p.bt, p.c.page_tokens, b, nullptr);
            enter(p, rows_per_item);
        } while (rbs == 0);
    }
};

// Finds the share of this block: a scan of the batch by one warp.
__device__ __forceinline__ StepWalk step_share(const AttendParams& p, int rows_per_item) {
    const int lane = threadIdx.x & 31;
    int64_t total = 0;
    for (int b0 = 0; b0 < p.bt.batch; b0 += 32) {
        int items = 0, units = 0, lo, hi;
        if (b0 + lane < p.bt.batch) StepWalk::measure(p, rows_per_item, load_seq(p.bt, p.c.page_tokens, b0 + lane, p.status), items, units, lo, hi);
        total += warp_sum_wide(items * units);
    }
    if (total > MAX_UNITS) {
        report(p.status, CCV3D_TOKENS_BAD_LENGTH);
        total = 0;
    }
    StepWalk w;
    w.total = total;
    w.blocks = min((int64_t)gridDim.x, total);      // every block that takes part has a unit: parts lie in neighbouring blocks
    w.u = w.u1 = 0;
    if ((int64_t)blockIdx.x < w.blocks) {
        w.u = (int)(total * blockIdx.x / w.blocks);
        w.u1 = (int)(total * (blockIdx.x + 1) / w.blocks);
    }
    w.b = w.h = w.rb = w.rbs = w.unit = w.units = w.lo = w.hi = w.base = 0;
    w.s = {0, 0, 0};
    if (w.done()) return w;
    int before = 0;
    for (int b0 = 0; b0 < p.bt.batch; b0 += 32) {
        int items = 0, units = 0, lo, hi;
        if (b0 + lane < p.bt.batch) StepWalk::measure(p, rows_per_item, load_seq(p.bt, p.c.page_tokens, b0 + lane, nullptr), items, units, lo, hi);
        const int mine = items * units, upto = before + warp_scan(mine);
        const unsigned hit = __ballot_sync(0xffffffffu, mine > 0 && w.u < upto);
        if (hit) {
            const int who = __ffs(hit) - 1;
            w.b = b0 + who;
            const int at = w.u - __shfl_sync(0xffffffffu, upto - mine, who);
            w.s = load_seq(p.bt, p.c.page_tokens, w.b, nullptr);
            w.enter(p, rows_per_item);
            w.unit = at % w.units;
            w.rb = at / w.units % w.rbs;
            w.h = at / w.units / w.rbs;
            return w;
        }
        before = __shfl_sync(0xffffffffu, upto, 31);
    }
    w.u1 = w.u;                 // (the arrays changed under the kernel)
    return w;
}

template <typename T, int D, int NT>
__global__ void __launch_bounds__(32 * STEP_WARPS, step_blocks(sizeof(T) == 4, D, 8 * NT)) kv_attend_step_kernel(const __grid_constant__ CUtensorMap tm, const AttendParams p) {
    using S = StepShape<D>;
    constexpr int TERMS = sizeof(T) == 4 ? 2 : 1, ROWS = 8 * NT, CH = D / 64;     // CH: 16-byte pieces of a row for a thread
    extern __shared__ __align__(1024) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r8 = lane >> 2, c4 = lane & 3;
    uint8_t* ring = smem + warp * S::STAGES * S::STAGE;
    float* merge = reinterpret_cast<float*>(smem + S::RING);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S::RING + S::MERGE) + warp * S::STAGES;
    int2* pages = reinterpret_cast<int2*>(smem + S::RING + S::MERGE + STEP_WARPS * S::STAGES * 8) + warp * S::STAGES;
    float4* scales = reinterpret_cast<float4*>(smem + S::RING + S::MERGE + STEP_WARPS * S::STAGES * 16) + warp * S::STAGES;
    float2* stats = reinterpret_cast<float2*>(smem + S::RING + S::MERGE + STEP_WARPS * S::STAGES * 32);     // [warp][16]
    const int P = p.c.page_tokens, H = p.c.kv_heads, pshift = 31 - __clz(P);

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (lane == 0) {
        for (int i = 0; i < S::STAGES; ++i) mbar_init(smem_u32(bars + i), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tm) : "memory");
    }
    __syncwarp();
    StepWalk w = step_share(p, ROWS);
    if (threadIdx.x == 0) p.join[blockIdx.x] = {0, 0, 0, 0};

    // ---- producer side of this warp: the same walk, ahead by up to STAGES tiles
    StepWalk f = w;
    int f_page = -2;             // lanes 0 and 1: page of the halves of the tile f stands on, as the table says (-2: not to be read)
    float f_scale = 0.f;         // lanes 0 .. 3: scales of the tile issued last, still to be left in its stage
    int issued = 0;
    auto seek = [&]() {          // moves f to the next unit in which this warp has tokens to read, and asks for its pages
        while (!f.done()) {
            const int t0 = f.base + f.unit * STEP_UNIT + warp * STEP_TILE;
            if (t0 < f.hi && t0 + STEP_TILE > f.lo) {
                f_page = -2;
                const int th = P < 32 ? t0 + lane * 16 : t0;
                if (lane < 2 && (P >= 32 || (th < f.hi && th + 16 > f.lo)))
                    f_page = __ldg(p.bt.page_table + (size_t)f.b * p.bt.max_pages + (th >> pshift));     // (looked at when the tile is issued)
                return;
            }
            f.next(p, ROWS);
        }
    };
    auto leave_scales = [&]() {  // lanes 0 .. 3 hold (half, keys or values) of the tile issued last
        if (issued > 0 && lane < 4) reinterpret_cast<float*>(scales + (issued - 1) % S::STAGES)[lane] = f_scale;
    };
    auto issue = [&]() {
        if (f.done()) return;
        if ((unsigned)f_page >= (unsigned)p.c.pages) {
            if (f_page != -2) report(p.status, CCV3D_TOKENS_BAD_PAGE);
            f_page = -1;
        }
        const int pg0 = __shfl_sync(0xffffffffu, f_page, 0), pg1 = __shfl_sync(0xffffffffu, f_page, 1);
        const int st = issued % S::STAGES, h = f.h;
        const int t0 = f.base + f.unit * STEP_UNIT + warp * STEP_TILE;
        if (lane < 4) {
            const int pg = lane < 2 ? pg0 : pg1;
            f_scale = pg >= 0 ? __ldg(p.c.scales + ((int64_t)pg * 2 + (lane & 1)) * H + h) : 0.f;
        }
        if (lane == 0) {
            pages[st] = make_int2(pg0, pg1);
            const uint32_t bar = smem_u32(bars + st), dst = smem_u32(ring + st * S::STAGE);
            // pages of 16 tokens: a box for each half
            const int box = P < 32 ? 16 : 32;
            const bool second = P < 32 && pg1 >= 0;
            mbar_expect_tx(bar, ((pg0 >= 0 ? 1u : 0u) + (second ? 1u : 0u)) * 2u * box * D);
            if (pg0 >= 0) {
                const int row = (pg0 * 2 * H + h) * P + (t0 & (P - 1));
                tma_load_2d(dst, &tm, bar, 0, row);
                tma_load_2d(dst + S::HALF, &tm, bar, 0, row + H * P);
            }
            if (second) {
                const int row = (pg1 * 2 * H + h) * P + ((t0 + 16) & (P - 1));
                tma_load_2d(dst + 16 * D, &tm, bar, 0, row);
                tma_load_2d(dst + S::HALF + 16 * D, &tm, bar, 0, row + H * P);
            }
        }
        ++issued;
        f.next(p, ROWS);
        seek();
    };
    seek();
#pragma unroll 1
    for (int i = 0; i < S::STAGES; ++i) {
        leave_scales();
        issue();
    }
    leave_scales();
    __syncwarp();

    bool alive = true;           // false: a wait of this warp gave up (it stays in step with the block and computes nothing)
    int used = 0;
    while (!w.done()) {
        // ---- an item (or this block's share of it)
        const int h = w.h, row0 = w.rb * ROWS;
        const Seq s = w.s;
        const int nrows = min(ROWS, s.n * p.group - row0);
        const int unit0 = w.unit, units = w.units, item_u = w.u - w.unit;        // the item's first unit in the whole list
        const int lo = w.lo, hi = w.hi, base = w.base;
        const int last = min(units, unit0 + (w.u1 - w.u));                       // one past the last unit this block takes
        // queries: row n = 8 i + r8 of the block, this thread's pieces of its channels
        uint32_t qf[NT][TERMS][CH][8];
        float qup[NT][2];        // factors of columns 2 c4 and 2 c4 + 1
        int clo[NT][2], chi[NT][2];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int n = 8 * i + r8;
            float x[CH][16];
            float most = 0.f;
#pragma unroll
            for (int g = 0; g < CH; ++g)
#pragma unroll
                for (int k = 0; k < 16; ++k) x[g][k] = 0.f;
            if (n < nrows) {
                const int token = s.first + (row0 + n) / p.group, head = h * p.group + (row0 + n) % p.group;
                const T* src = (const T*)p.q.data + token * p.q.token_stride + head * p.q.head_stride;
#pragma unroll
                for (int g = 0; g < CH; ++g)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float t[4];
                        load4(src + (c4 * CH + g) * 16 + 4 * k, t);
#pragma unroll
                        for (int e = 0; e < 4; ++e) { x[g][4 * k + e] = t[e]; most = fmaxf(most, fabsf(t[e])); }
                    }
            }
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            float down, up;
            row_power(most, down, up);
#pragma unroll
            for (int g = 0; g < CH; ++g)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float a = x[g][2 * k] * down, b = x[g][2 * k + 1] * down;
                    qf[i][0][g][k] = pack_half(a, b);
                    if (TERMS == 2) qf[i][TERMS - 1][g][k] = pack_rest(a, b, qf[i][0][g][k]);
                }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                qup[i][e] = __shfl_sync(0xffffffffu, up, (2 * c4 + e) * 4) * (p.scale * LOG2E);
                const int n2 = 8 * i + 2 * c4 + e;
                clo[i][e] = chi[i][e] = 0;
                if (n2 < nrows) visible(p, s.total - s.n + (row0 + n2) / p.group, s.total, clo[i][e], chi[i][e]);
            }
        }
        float m[NT][2], l[NT][2], o[NT][D / 16][4];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            m[i][0] = m[i][1] = -INFINITY;
            l[i][0] = l[i][1] = 0.f;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) o[i][k][0] = o[i][k][1] = o[i][k][2] = o[i][k][3] = 0.f;
        }
        const bool one_view = s.n == 1;                                          // all rows see the same tokens

        for (int unit = unit0; unit < last; ++unit) {
            const int t0 = base + unit * STEP_UNIT + warp * STEP_TILE;
            if (t0 >= hi || t0 + STEP_TILE <= lo) continue;
            const int st = used % S::STAGES;
            if (alive) {
                const uint32_t bar = smem_u32(bars + st), ph = (uint32_t)(used / S::STAGES) & 1u;
                long long since = 0;
                for (uint32_t it = 0; !mbar_try_wait(bar, ph); ++it)
                    if ((it & 63u) == 63u) {
                        const long long now = clock64();
                        if (!since) since = now;
                        else if (now - since > p.wait_clk) { alive = false; break; }
                    }
                alive = __all_sync(0xffffffffu, alive);
                if (!alive && lane == 0) report(p.status, CCV3D_TOKENS_TIMEOUT);
            }
            if (!alive) { ++used; continue; }
            const uint8_t* ks = ring + st * S::STAGE;
            int2 pg = pages[st];
            float4 sc = scales[st];
            if (P >= 32) { pg.y = pg.x; sc.z = sc.x; sc.w = sc.y; }
            // a tile that every row sees whole needs no masks
            bool whole = pg.x >= 0 && pg.y >= 0;
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) whole = whole && (8 * i + 2 * c4 + e >= nrows || (t0 >= clo[i][e] && t0 + STEP_TILE <= chi[i][e]));
            whole = __all_sync(0xffffffffu, whole);
            // scores of 2 x 16 tokens; even and odd steps of the contraction in sums of their own, so that four (NT = 1)
            // products are on their way at a time
            float x[NT][2][4], y[NT][2][4];
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[i][j][e] = y[i][j][e] = 0.f;
#pragma unroll
            for (int g = 0; g < CH; ++g) {
                uint4 a[2][2];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int row = 16 * j + 8 * e + r8, piece = c4 * CH + g;
                        const int sw = D == 128 ? (piece ^ (row & 7)) : (piece ^ ((row >> 1) & 3));
                        a[j][e] = *reinterpret_cast<const uint4*>(ks + row * D + sw * 16);
                    }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t a0 = k == 0 ? a[j][0].x : k == 1 ? a[j][0].y : k == 2 ? a[j][0].z : a[j][0].w;
                        const uint32_t a1 = k == 0 ? a[j][1].x : k == 1 ? a[j][1].y : k == 2 ? a[j][1].z : a[j][1].w;
                        const uint32_t af[4] = {e4m3x2_to_half2(a0 & 0xFFFFu), e4m3x2_to_half2(a1 & 0xFFFFu), e4m3x2_to_half2(a0 >> 16), e4m3x2_to_half2(a1 >> 16)};
#pragma unroll
                        for (int i = 0; i < NT; ++i)
#pragma unroll
                            for (int t = 0; t < TERMS; ++t) mma_f16((k + t) & 1 ? y[i][j] : x[i][j], af, qf[i][t][g][2 * k], qf[i][t][g][2 * k + 1]);
                    }
            }
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[i][j][e] += y[i][j][e];
            // ---- softmax: x[i][j] holds tokens 16 j + r8 (elements 0, 1) and 16 j + 8 + r8 (2, 3) of columns 2 c4, 2 c4 + 1
            float ev[2], iv[2];
            scale_terms(sc.y, ev[0], iv[0]);
            scale_terms(sc.w, ev[1], iv[1]);
            const float kf[2] = {sc.x, sc.z};
            // The base is that of earlier tiles until a score passes what it bears: then it moves, by a whole power of two, for
            // all rows.  Most tiles so need no maximum over the lanes.
            bool raise = false;
            float limit[NT][2];
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) limit[i][e] = base_limit(m[i][e]);
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float v = fmaf(x[i][j][e], qup[i][e & 1] * kf[j], ev[j]);
                        if (!whole) {
                            const int t = t0 + 16 * j + 8 * (e >> 1) + r8;
                            if (t < clo[i][e & 1] || t >= chi[i][e & 1] || (j ? pg.y : pg.x) < 0) v = -INFINITY;
                        }
                        x[i][j][e] = v;
                        raise = raise || v > limit[i][e & 1];
                    }
            if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = fmaxf(fmaxf(x[i][0][e], x[i][0][e + 2]), fmaxf(x[i][1][e], x[i][1][e + 2]));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                        mx = fmaxf(m[i][e], base_for(mx));
                        const float corr = m[i][e] == -INFINITY ? 0.f : exp2_fast(m[i][e] - mx);
                        m[i][e] = mx;
                        l[i][e] *= corr;
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) { o[i][k][e] *= corr; o[i][k][e + 2] *= corr; }
                    }
            }
            uint32_t pf[NT][TERMS][2][2];                                        // weights, tokens down the contraction
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const float m_use[2] = {base_or_start(m[i][0]), base_or_start(m[i][1])};
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float w4[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w4[e] = exp2_fast(x[i][j][e] - m_use[e & 1]);
                        l[i][e & 1] = fmaf(w4[e], iv[j], l[i][e & 1]);
                    }
                    const uint32_t a = pack_half(w4[0], w4[1]), b = pack_half(w4[2], w4[3]);
                    pf[i][0][j][0] = transpose8(a);
                    pf[i][0][j][1] = transpose8(b);
                    if (TERMS == 2) {
                        pf[i][TERMS - 1][j][0] = transpose8(pack_rest(w4[0], w4[1], a));
                        pf[i][TERMS - 1][j][1] = transpose8(pack_rest(w4[2], w4[3], b));
                    }
                }
            }
            // ---- outputs: V^T P.  A thread takes channels r8 * D / 8 .. of tokens 2 c4, 2 c4 + 1, 2 c4 + 8, 2 c4 + 9
            const uint8_t* vs = ks + S::HALF;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t v[4][D / 32];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int row = 16 * j + 2 * c4 + (e & 1) + 8 * (e >> 1);
                    if constexpr (D == 128) {
                        const uint4 t = *reinterpret_cast<const uint4*>(vs + row * D + (r8 ^ (row & 7)) * 16);
                        v[e][0] = t.x; v[e][1] = t.y; v[e][2] = t.z; v[e][3] = t.w;
                    } else {
                        const uint2 t = *reinterpret_cast<const uint2*>(vs + row * D + ((r8 >> 1) ^ ((row >> 1) & 3)) * 16 + (r8 & 1) * 8);
                        v[e][0] = t.x; v[e][1] = t.y;
                    }
                    if (!whole) {                                                // what no row sees may hold anything
                        const int t = t0 + row;
                        const bool gone = t < lo || t >= hi || (j ? pg.y : pg.x) < 0;
#pragma unroll
                        for (int k = 0; k < D / 32; ++k) v[e][k] = gone ? 0u : v[e][k];
                    }
                }
                if (!whole && !one_view) {
                    // a NaN among tokens that some rows see and others do not: it would reach them all through a zero
                    // weight.  Its code goes; a product of "is NaN" and "is seen" marks the outputs it belongs to.
                    bool any = false;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int k = 0; k < D / 32; ++k) any = any || __vcmpeq4(v[e][k] & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
                    if (__any_sync(0xffffffffu, any)) {
                        uint32_t nan[4][D / 32];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
#pragma unroll
                            for (int k = 0; k < D / 32; ++k) {
                                nan[e][k] = __vcmpeq4(v[e][k] & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
                                v[e][k] &= ~nan[e][k];
                                nan[e][k] &= 0x38383838u;                        // 1.0
                            }
#pragma unroll
                        for (int i = 0; i < NT; ++i) {
                            float seen[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int t = t0 + 16 * j + 8 * (e >> 1) + r8;
                                seen[e] = t >= clo[i][e & 1] && t < chi[i][e & 1] ? 1.f : 0.f;
                            }
                            const uint32_t b0 = transpose8(pack_half(seen[0], seen[1])), b1 = transpose8(pack_half(seen[2], seen[3]));
#pragma unroll
                            for (int k = 0; k < D / 32; ++k) {
                                const uint32_t p01 = __byte_perm(nan[0][k], nan[1][k], 0x5140), p01h = __byte_perm(nan[0][k], nan[1][k], 0x7362);
                                const uint32_t p23 = __byte_perm(nan[2][k], nan[3][k], 0x5140), p23h = __byte_perm(nan[2][k], nan[3][k], 0x7362);
#pragma unroll
                                for (int half = 0; half < 2; ++half) {
                                    const uint32_t x01 = half ? p01h : p01, x23 = half ? p23h : p23;
                                    const uint32_t af[4] = {e4m3x2_to_half2(x01 & 0xFFFFu), e4m3x2_to_half2(x01 >> 16),
                                                            e4m3x2_to_half2(x23 & 0xFFFFu), e4m3x2_to_half2(x23 >> 16)};
                                    float hit[4] = {0.f, 0.f, 0.f, 0.f};
                                    mma_f16(hit, af, b0, b1);
#pragma unroll
                                    for (int e = 0; e < 4; ++e)
                                        if (hit[e] > 0.f) o[i][2 * k + half][e] = __int_as_float(0x7FFFFFFF);
                                }
                            }
                        }
                    }
                }
#pragma unroll
                for (int k = 0; k < D / 32; ++k) {                               // four channels: two tiles of 16 rows
                    // bytes (token 0, token 1) of channels 0, 1 and 2, 3
                    const uint32_t p01 = __byte_perm(v[0][k], v[1][k], 0x5140), p01h = __byte_perm(v[0][k], v[1][k], 0x7362);
                    const uint32_t p23 = __byte_perm(v[2][k], v[3][k], 0x5140), p23h = __byte_perm(v[2][k], v[3][k], 0x7362);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t x01 = half ? p01h : p01, x23 = half ? p23h : p23;
                        const uint32_t af[4] = {e4m3x2_to_half2(x01 & 0xFFFFu), e4m3x2_to_half2(x01 >> 16),
                                                e4m3x2_to_half2(x23 & 0xFFFFu), e4m3x2_to_half2(x23 >> 16)};
#pragma unroll
                        for (int i = 0; i < NT; ++i) {
                            if constexpr (TERMS == 1) {
                                mma_f16(o[i][2 * k + half], af, pf[i][0][j][0], pf[i][0][j][1]);
                            } else {
                                float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                                for (int t = TERMS - 1; t >= 0; --t) mma_f16(sum, af, pf[i][t][j][0], pf[i][t][j][1]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[i][2 * k + half][e] += sum[e];
                            }
                        }
                    }
                }
            }
            ++used;
            __syncwarp();                                                        // the stage has been read
            leave_scales();                                                      // (of the tile before: they have had a tile's time)
            issue();
            __syncwarp();
        }

        // ---- end of the item here: the four warps' sums into one
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float t = l[i][e];
                t += __shfl_xor_sync(0xffffffffu, t, 4);
                t += __shfl_xor_sync(0xffffffffu, t, 8);
                t += __shfl_xor_sync(0xffffffffu, t, 16);
                if (r8 == 0) stats[warp * 16 + 8 * i + 2 * c4 + e] = make_float2(m[i][e], t);
            }
        __syncthreads();
        const bool starts = unit0 == 0, ends = last == units;
        const int64_t slot = 2 * (int64_t)blockIdx.x + (starts ? 1 : 0);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            float f2[2], inv[2], mm[2], ll[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int n = 8 * i + 2 * c4 + e;
                mm[e] = -INFINITY;
#pragma unroll
                for (int k = 0; k < STEP_WARPS; ++k) mm[e] = fmaxf(mm[e], stats[k * 16 + n].x);
                ll[e] = 0.f;
#pragma unroll
                for (int k = 0; k < STEP_WARPS; ++k) {
                    const float2 a = stats[k * 16 + n];
                    ll[e] = fmaf(a.x == -INFINITY ? 0.f : exp2_fast(a.x - mm[e]), a.y, ll[e]);
                }
                f2[e] = m[i][e] == -INFINITY ? 0.f : exp2_fast(m[i][e] - mm[e]);
                inv[e] = starts && ends ? (ll[e] != 0.f ? 1.f / ll[e] : 0.f) : 1.f;
            }
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][k][e] *= f2[e & 1];
            // warps 2 and 3 to 0 and 1, then 1 to 0
#pragma unroll
            for (int half = STEP_WARPS / 2; half; half >>= 1) {
                if (warp >= half && warp < 2 * half) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        *reinterpret_cast<float4*>(merge + (((warp - half) * (D / 16) + k) * 32 + lane) * 4) = make_float4(o[i][k][0], o[i][k][1], o[i][k][2], o[i][k][3]);
                }
                __syncthreads();
                if (warp < half) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const float4 t = *reinterpret_cast<const float4*>(merge + ((warp * (D / 16) + k) * 32 + lane) * 4);
                        o[i][k][0] += t.x; o[i][k][1] += t.y; o[i][k][2] += t.z; o[i][k][3] += t.w;
                    }
                }
                if (half > 1) __syncthreads();
            }
            if (warp == 0) {
                // this thread: channels r8 * D / 8 + 2 k (elements 0, 1) and + 1 (2, 3) of columns 2 c4, 2 c4 + 1
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int n = 8 * i + 2 * c4 + e;
                    if (n >= nrows) continue;
                    if (starts && ends) {
                        const int token = s.first + (row0 + n) / p.group, head = h * p.group + (row0 + n) % p.group;
#pragma unroll
                        for (int k = 0; k < D / 16; k += 2) {
                            float v[4] = {o[i][k][e], o[i][k][e + 2], o[i][k + 1][e], o[i][k + 1][e + 2]};
#pragma unroll
                            for (int t = 0; t < 4; ++t) v[t] = ll[e] != 0.f ? v[t] * inv[e] : 0.f;
                            store_out<T>(p, token, head, r8 * (D / 8) + 2 * k, v);
                        }
                        if (r8 == 0 && p.lse) p.lse[(int64_t)token * p.q_heads + head] = lse_of(mm[e], ll[e]);
                    } else {
                        float* dst = p.part + (slot * p.slot_rows + n) * D + r8 * (D / 8);
#pragma unroll
                        for (int k = 0; k < D / 16; k += 2)
                            *reinterpret_cast<float4*>(dst + 2 * k) = make_float4(o[i][k][e], o[i][k][e + 2], o[i][k + 1][e], o[i][k + 1][e + 2]);
                        if (r8 == 0) p.part_ml[slot * p.slot_rows + n] = make_float2(mm[e], ll[e]);
                    }
                }
            }
            __syncthreads();
        }
        if (starts && !ends && threadIdx.x == 0) {
            // the block that takes the item's last unit x is the largest i with floor(i U / G) <= x
            const int64_t x = item_u + units - 1;
            const int z = (int)(((x + 1) * w.blocks - 1) / w.total);
            p.join[blockIdx.x] = {z - (int)blockIdx.x + 1, s.first * p.group + row0, nrows, h * p.group};
        }
        for (int i = last - unit0; i > 0; --i) w.next(p, ROWS);
    }
    if (!alive) {                                                                // copies still on their way into this block
        const long long t = clock64();
        while (clock64() - t < 400000) __nanosleep(1000);
    }
}

}  // namespace ccv3d
