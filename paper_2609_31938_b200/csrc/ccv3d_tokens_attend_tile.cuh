// Attention of many query rows (frames, prompts) over the paged E4M3 cache, on tcgen05.
//
// Bound by the tensor cores and, next to them, the exponentials.  An item is a block of 256 query rows of one kv head (F32:
// 128), rows being (token, head of the group) so that grouped heads share the keys they share; a unit is 128 cached tokens.
// 20 warps, one block to an SM:
//   warps 0-3, 4-7   softmax of the first and second 128 rows, a thread to a row: scores from TMEM, weights back as halves
//                    over them, sums in registers, the output from TMEM at the end; they also stage the queries
//   warps 8-11, 12-15  turn codes into halves in shared memory (exact): keys and values, two slots each
//   warps 16, 19     issue the MMAs of one row block each: S = Q K^T from shared memory, O += P V with P in TMEM (an issuer is
//                    held up while the tensor cores work on what it issued: with one for both the blocks waited in line)
//   warp 17          walks the block's share ahead of the others and tells them of it: segments (an item, or the stretch of
//                    it that falls to this block), and pages and scales of up to eight coming tiles
//   warp 18          brings the codes in: bulk copies of 16 tokens into a ring of four half tiles
// Two row blocks in turn keep the tensor cores busy: while one is in its softmax the other's products run.
//
// Keys and values are staged alike, rows of 64 channels (128 bytes, 128-byte swizzle) token by token: K-major for the
// scores and, read the other way, MN-major for the outputs.  The softmax base is only raised when a score passes what it
// bears (then the sums in TMEM are scaled down): weights stay under 2^15 and a tile needs one pass.
// For F32 queries and weights go in as two halves each (value and remainder): about 22 bits, at twice the MMAs.
//
// Measured (BF16): 3520 rows on 28160 tokens, 12 heads of 128, 645 to 665 us = 0.93 PFLOP/s, 56 % of what the tensor cores do
// in a plain product.  A tile of 256 x 128 takes 3.6 k cycles, of which the tensor pipe is busy for 2.05 k and the exponential
// unit for 2.07 k.  Each stretch of an item costs some 25 k cycles more (queries in, outputs out): nine tiles to an item, 260 us
// for 100 GFLOP.
#pragma once
#include "ccv3d_tokens_attend_step.cuh"

namespace ccv3d {

constexpr int TILE_UNIT = 128, TILE_THREADS = 640;
constexpr int TILE_BATCH = 1024;                       // sequences whose costs are counted at a time (in the ring of codes)
constexpr int TILE_MOVERS = 4;                         // warps that turn keys into halves, and as many for values
constexpr int TILE_AHEAD = 8;                          // tiles and segments that may be known ahead
static_assert(TILE_AHEAD >= 8, "news goes out four tiles at a time and comes back two tiles late");
constexpr int TILE_REGS_SOFTMAX = 168, TILE_REGS_REST = 48;   // of 256 and 384 threads: 61440 registers, what 640 threads are launched with at 96
// F32: the tensor cores cut each sum they add to instead of rounding it, which over 20 000 tokens in one stretch costs 5.6e-6 of
// the result.  Every so many tiles the outputs go into sums of their own in TMEM, rounded, and start again from zero.
// Errors of two batches of prompts that see 670 and 380 tokens (32-bit operations: 0.56e-6, 0.69e-6) and time of 1760 rows, 12
// heads, on 15840 tokens: every tile 0.38e-6, 0.43e-6, 445 us; every 2 tiles 0.60e-6, 0.64e-6, 395 us; every 4 tiles 1.1e-6,
// 1.2e-6, 371 us (without the order of the remainders below).
constexpr int TILE_FOLD = 2;

template <typename T, int D> struct TileShape {
    static constexpr int TERMS = sizeof(T) == 4 ? 2 : 1, NQ = sizeof(T) == 4 ? 1 : 2, ROWS = 128 * NQ;
    static constexpr uint32_t HALF = 128 * 128;                       // 128 rows of 64 channels
    static constexpr uint32_t KV = HALF * (D / 64), Q = KV * TERMS;   // one staged tile; one row block's queries
    static constexpr uint32_t Q_AT = 0, K_AT = NQ * Q, V_AT = K_AT + 2 * KV, RAW_AT = V_AT + 2 * KV;
    static constexpr uint32_t RAW = 64 * D, END = RAW_AT + 4 * RAW;      // codes of 64 tokens: keys, keys, values, values
    // TMEM columns: scores of the row blocks, each half's weights over the first of its scores, then outputs; F32 has
    // columns of its own for weights
    static constexpr uint32_t S_COL = 0, P_COL = NQ == 2 ? 0 : 128, P_HALF = NQ == 2 ? 64 : 32, O_COL = 256, FOLD_COL = 384;
};

// A coming tile: what the movers and the softmax need to know of its pages.
struct TileInfo {
    float4 group[8];         // of each 16 tokens: key scale, log2 and reciprocal of the value scale
    int rows[8];             // their rows in the pool in units of 16, -1: not to be read
    int live, edge, t0, lo, hi;     // edge: not every row of the item sees all of it; lo, hi: tokens that any row sees
    int absent;              // a page that should be there is not
};

// A stretch of an item that falls to this block: units unit .. unit + n - 1 of item rows row0 .. row0 + nrows - 1 (of
// sequence b) of kv head h.
struct TileSegment {
    int live, n, starts, ends, parts;        // parts: blocks that an item which starts here reaches into, if it does not end here
    int b, h, row0, nrows, first, before, total;     // before: cached tokens before the sequence's new ones; first: packed token of those
    int t0, lo_all, hi_all;                  // first token of the stretch
};

struct TileShared {
    TileInfo info[TILE_AHEAD];
    TileSegment seg[TILE_AHEAD];
    uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], q_full[2], s_full[2][2], p_full[2][2], h_done[2], o_full[2], o_empty[2];
    uint64_t i_full[TILE_AHEAD], i_empty[TILE_AHEAD], g_full[TILE_AHEAD], g_empty[TILE_AHEAD];
    uint64_t r_full[4], r_empty[4];
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
__device__ __noinline__ TileItem tile_item_call(const AttendParams& p, const Seq& s, int rb) { return tile_item<ROWS>(p, s, rb); }
template <int ROWS>
__device__ __forceinline__ TileWalk<ROWS> tile_share(const AttendParams& p, int* cost_of) {
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
                    for (int rb = lane; rb < blocks; rb += 32) units += tile_item_call<ROWS>(p, s, rb).units;
                    units = __reduce_add_sync(0xffffffffu, units);
                    if (lane == 0) cost_of[b] = units * p.c.kv_heads;
                }
                __syncthreads();
            }
            for (int b0 = 0; b0 < n && !found; b0 += 32) {
                const int mine = b0 + lane < n ? cost_of[b0 + lane] : 0;
                if (pass == 0) { w.total += warp_sum_wide(mine); continue; }
                const int upto = warp_scan(mine), all = __shfl_sync(0xffffffffu, upto, 31);
                const unsigned hit = __ballot_sync(0xffffffffu, mine > 0 && (int64_t)w.u < before + upto);
                if (!hit) { before += all; continue; }
                const int who = __ffs(hit) - 1;
                int at = w.u - (int)(before + __shfl_sync(0xffffffffu, upto - mine, who));
                w.b = c0 + b0 + who;
                w.s = load_seq(p.bt, p.c.page_tokens, w.b, nullptr);
                const int blocks = (w.s.n * p.group + ROWS - 1) / ROWS;
                for (int r0 = 0; r0 < blocks && !found; r0 += 32) {
                    const int cost = r0 + lane < blocks ? tile_item_call<ROWS>(p, w.s, r0 + lane).units * p.c.kv_heads : 0;
                    const int to = warp_scan(cost);
                    const unsigned in = __ballot_sync(0xffffffffu, cost > 0 && at < to);
                    if (!in) { at -= __shfl_sync(0xffffffffu, to, 31); continue; }
                    const int r = __ffs(in) - 1;
                    at -= __shfl_sync(0xffffffffu, to - cost, r);
                    w.rb = r0 + r;
                    w.t = tile_item_call<ROWS>(p, w.s, w.rb);
                    w.h = at / w.t.units;
                    w.unit = at % w.t.units;
                    found = true;
                }
            }
        }
        if (pass == 0) {
            if (w.total > MAX_UNITS) {
                if (threadIdx.x == 0) report(p.status, CCV3D_TOKENS_BAD_LENGTH);
                w.total = 0;
            }
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
    const long long since = clock64();
#pragma unroll 1
    while (!mbar_try_wait(b, parity)) {
        if (*(volatile int*)&sh->abort_flag) return false;
        if (clock64() - since > p.wait_clk) {
            *(volatile int*)&sh->abort_flag = 1;
            report(p.status, CCV3D_TOKENS_TIMEOUT);
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, TileShared* sh, const AttendParams& p) {
    return __all_sync(0xffffffffu, tile_wait(bar, parity, sh, p));
}

__device__ __forceinline__ void bulk_prefetch(const void* p, uint32_t bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
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

// 32 elements of a row; zeros without one.
__device__ __forceinline__ void load_row32(const float* src, float (&x)[32]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float4 t = src ? *reinterpret_cast<const float4*>(src + 4 * j) : make_float4(0.f, 0.f, 0.f, 0.f);
        x[4 * j] = t.x; x[4 * j + 1] = t.y; x[4 * j + 2] = t.z; x[4 * j + 3] = t.w;
    }
}
template <typename T>
__device__ __forceinline__ void store_row32(T* dst, const float (&x)[32]) {
#pragma unroll
    for (int j = 0; j < 32; j += sizeof(T) == 2 ? 8 : 4) {
        if constexpr (sizeof(T) == 2)
            *reinterpret_cast<uint4*>(dst + j) = make_uint4(pack_bf16(x[j], x[j + 1]), pack_bf16(x[j + 2], x[j + 3]), pack_bf16(x[j + 4], x[j + 5]), pack_bf16(x[j + 6], x[j + 7]));
        else
            *reinterpret_cast<float4*>(dst + j) = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
    }
}
// Stages the queries of 32 rows (all lanes of the warp call it) and returns what each thread needs to know of its own.
template <typename T, int D>
__device__ __forceinline__ TileRow stage_row(const AttendParams& p, const TileSegment& w, int r, int tid, uint8_t* q) {
    using S = TileShape<T, D>;
    TileRow row = {0, 0, 0.f, -1, 0};
    const T* src = nullptr;
    if (r < w.nrows) {
        const int at = w.row0 + r;
        row.token = w.first + at / p.group;
        row.head = w.h * p.group + at % p.group;
        visible(p, w.before + at / p.group, w.total, row.lo, row.hi);
        src = (const T*)p.q.data + row.token * p.q.token_stride + row.head * p.q.head_stride;
    }
    float up;
    if constexpr (sizeof(T) == 2) {
        // A warp reads its 32 rows together, D / 8 lanes to a row: a thread's own row would take 32 lines for each access.
        constexpr int LPR = D / 8, RPI = 32 / LPR, IT = LPR;     // lanes to a row, rows at a time, rounds
        const int lane = tid & 31, sub = lane / LPR, l = lane % LPR, r0 = r - lane;      // first row of the warp
        const int at = w.row0 + r0 + sub;
        int head = at % p.group;
        const T* from = (const T*)p.q.data + (w.first + at / p.group) * p.q.token_stride + (w.h * p.group + head) * p.q.head_stride + l * 8;
        const int64_t step = RPI * p.q.head_stride, wrap = p.q.token_stride - p.group * p.q.head_stride;
        uint4 x[IT];
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            x[i] = make_uint4(0, 0, 0, 0);
            if (r0 + i * RPI + sub < w.nrows) x[i] = *reinterpret_cast<const uint4*>(from);
            from += step;
            head += RPI;
#pragma unroll
            for (int k = 0; k < RPI; ++k)
                if (head >= p.group) { head -= p.group; from += wrap; }
        }
        // largest magnitudes from the bits, two elements to an instruction; then over a row's lanes, halving the rounds a
        // lane answers for at each step: lane l ends with round l's
        uint32_t big[IT];
#pragma unroll
        for (int i = 0; i < IT; ++i)
            big[i] = __vmaxu2(__vmaxu2(x[i].x & 0x7FFF7FFFu, x[i].y & 0x7FFF7FFFu), __vmaxu2(x[i].z & 0x7FFF7FFFu, x[i].w & 0x7FFF7FFFu));
#pragma unroll
        for (int o = LPR / 2; o; o >>= 1)
#pragma unroll
            for (int i = 0; i < o; ++i) {
                const uint32_t give = l & o ? big[i] : big[i + o], keep = l & o ? big[i + o] : big[i];
                big[i] = __vmaxu2(keep, __shfl_xor_sync(0xffffffffu, give, o));
            }
        // BF16 s eeeeeeee mmmmmmm to a half s eeeee mmm mmmm000 with the row's largest exponent in the place of 2^14: exponents
        // by a subtraction, both elements at once; what lies 2^-28 under the row's largest becomes zero.  The factor puts
        // the exponent back.  Infinities and NaN go over as such if their exponent comes in the place of theirs (31).
        const uint32_t most = max(big[0] & 0xFFFFu, big[0] >> 16);
        const int field = max((int)(most >> 7) - (most >= 0x7F80u ? 31 : 29), 0);
        up = __uint_as_float((uint32_t)(field + 15) << 23);
        up = __shfl_sync(0xffffffffu, up, lane % RPI * LPR + lane / RPI);        // of this thread's own row
        const uint32_t off = (uint32_t)(-(field << 7) & 0xFFFF) * 0x10001u;
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            const int rr = i * RPI + sub;                                        // row of the warp, and of the row block
            const uint32_t o = __shfl_sync(0xffffffffu, off, sub * LPR + i);
            const uint32_t e[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
            uint32_t y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = (__viaddmax_s16x2(e[k] & 0x7FFF7FFFu, o, 0u) << 3) | (e[k] & 0x80008000u);
            *reinterpret_cast<uint4*>(q + (l / 8) * S::HALF + (tid - lane + rr) * 128 + ((l & 7) ^ (rr & 7)) * 16) = make_uint4(y[0], y[1], y[2], y[3]);
        }
    } else {
        float most = 0.f;
#pragma unroll 1
        for (int i = 0; i < D; i += 32) {
            float x[32];
            load_row32(src ? src + i : nullptr, x);
#pragma unroll
            for (int k = 0; k < 32; ++k) most = fmaxf(most, fabsf(x[k]));
        }
        float down;
        row_power(most, down, up);
#pragma unroll 1
        for (int i = 0; i < D; i += 32) {
            float x[32];
            load_row32(src ? src + i : nullptr, x);
            uint8_t* dst = q + (i / 64) * S::HALF + tid * 128;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t y[4], z[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float u = x[8 * j + 2 * k] * down, v = x[8 * j + 2 * k + 1] * down;
                    y[k] = pack_half(u, v);
                    z[k] = pack_rest(u, v, y[k]);
                }
                uint8_t* at = dst + (((i / 8 + j) & 7) ^ (tid & 7)) * 16;
                *reinterpret_cast<uint4*>(at) = make_uint4(y[0], y[1], y[2], y[3]);
                *reinterpret_cast<uint4*>(at + S::KV) = make_uint4(z[0], z[1], z[2], z[3]);
            }
        }
    }
    row.factor = up * (p.scale * LOG2E);
    return row;
}

// two floats to an instruction
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {      // (NaN stays out, as with fmaxf)
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Bits of the tokens [first, end) of 32 that begin at 0.
__device__ __forceinline__ uint32_t bits_between(int first, int end) {
    const uint32_t below_end = end >= 32 ? 0xFFFFFFFFu : (1u << max(end, 0)) - 1u, below_first = first >= 32 ? 0xFFFFFFFFu : (1u << max(first, 0)) - 1u;
    return below_end & ~below_first;
}
// Scores of 32 tokens (two groups of 16) to weights: packed into pr (F32: remainders into rest), sum: what the weights add to the
// row's weight sum.  The exponent comes in one rounding from the product, and mx gathers the largest.  EDGE (tokens that this
// row may not see, and rows with far scores) rounds the score first, and mx gathers the largest score: it then is that of some
// token, and none lies above it, which no longer holds of the other once neighbouring floats are no small part of a unit apart.
template <bool REST, bool EDGE>
__device__ __forceinline__ void chunk_weights(const uint32_t (&v)[32], const float4* group, const TileRow& row, float base, int t0, uint32_t* pr,
                                              uint32_t* rest, float& mx, float& sum) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        const float4 k = group[g];
        const float f = k.x * row.factor, a = EDGE ? k.y : k.y - base;
        const uint64_t f2 = pair(f, f), a2 = pair(a, a), down2 = pair(-base, -base);
        uint64_t part = 0;                                       // two sums: even and odd tokens
        const uint32_t seen = EDGE && k.y != -INFINITY ? bits_between(row.lo - t0 - 16 * g, row.hi - t0 - 16 * g) : 0u;
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            float x, y;
            unpair(fma_pair(pair(__uint_as_float(v[16 * g + i]), __uint_as_float(v[16 * g + i + 1])), f2, a2), x, y);
            if (EDGE) {
                if (!(seen >> i & 1u)) x = -INFINITY;
                if (!(seen >> (i + 1) & 1u)) y = -INFINITY;
            }
            mx = max3(mx, x, y);
            if (EDGE) unpair(add_pair(pair(x, y), down2), x, y);
            const float e0 = exp2_fast(x), e1 = exp2_fast(y);
            part = add_pair(part, pair(e0, e1));
            const uint32_t h = pack_half(e0, e1);
            pr[8 * g + i / 2] = h;
            if (REST) rest[8 * g + i / 2] = pack_rest(e0, e1, h);
        }
        float s0, s1;
        unpair(part, s0, s1);
        sum = fmaf(s0 + s1, k.z, sum);
    }
}
// Scales 32 TMEM columns of this thread's lane: FP32 values or pairs of halves.
__device__ __forceinline__ void scale_columns(uint32_t t, float f) {
    uint32_t v[32];
    tc_ld32(t, v);
    tc_wait_ld();
#pragma unroll
    for (int k = 0; k < 32; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * f);
    tc_st<32>(t, v);
}

// A softmax thread's state: TMEM addresses of its scores, weights and outputs, its running base and sum.
struct TileSoftmax {
    uint32_t t_s, t_p, t_o, t_fold;
    float m, l;
    bool folded;             // (F32) there are sums at t_fold
    bool far;                // (the same for the warp) scores of some row are beyond SCORE_EXACT
};
// Passes over a half tile: the first, and one after the base was raised.  No raise leaves an exponent that asks for another.
constexpr int TILE_PASSES = 2;

// One tile of a row, from `half` on: weights of 64 tokens twice; `scores(1)` waits for the second half's scores (the first half's are
// there), `ready(half)` tells the MMA warp that the weights are in TMEM.  Where a score passes the base by more than the weights
// can hold, the base moves (by a whole power of two, so what has been summed is scaled exactly) and the half is done
// again by the same code; `settled(half)` waits until the outputs hold all weights given before that half.  Returns 2, or -1
// if a wait gave up, or without EDGE the half that turned out to hold far scores (nothing of it has gone out).
template <typename T, int D, bool EDGE, typename Scores, typename Ready, typename Settled>
__device__ __forceinline__ int tile_softmax(TileSoftmax& x, const float4* group, const TileRow& row, int t0, bool first, int half,
                                            const Scores& scores, const Ready& ready, const Settled& settled) {
    constexpr bool REST = sizeof(T) == 4;
    uint32_t pr[32], rest[REST ? 32 : 16];
#pragma unroll 1
    for (; half < 2; ++half) {
        const float4* k = group + 4 * half;
        float sum;
        if (half == 1 && !scores(1)) return -1;
#pragma unroll 1
        for (int pass = 1;; ++pass) {
            float mx = -INFINITY;
            sum = 0.f;
            const float base = base_or_start(x.m);
            // (what tcgen05.ld brings is used, and copied, behind its wait only: nothing of it is carried around a loop)
            uint32_t a[32], b[32];
            tc_ld32(x.t_s + 64 * half, a);
            tc_ld32(x.t_s + 64 * half + 32, b);
            tc_wait_ld();
            chunk_weights<REST, EDGE>(a, k, row, base, t0 + 64 * half, pr, rest, mx, sum);
            chunk_weights<REST, EDGE>(b, k + 2, row, base, t0 + 64 * half + 32, pr + 16, rest + (REST ? 16 : 0), mx, sum);
            const bool raise = mx > (EDGE ? base_limit(x.m) : x.m == -INFINITY ? -INFINITY : WEIGHT_TOP);
            if (pass >= TILE_PASSES || !__any_sync(0xffffffffu, raise)) break;
            const float now = fmaxf(x.m, base_for(EDGE ? mx : mx + base));       // (mx = -inf leaves the base)
            if (__any_sync(0xffffffffu, raise && !(fabsf(now) <= SCORE_EXACT))) {
                x.far = true;
                if (!EDGE) return half;
            }
            const float corr = x.m == -INFINITY ? 0.f : exp2_fast(x.m - now);
            if (!first || half == 1) {
                if (!settled(half)) return -1;
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    scale_columns(x.t_o + c, corr);
                    if (REST && x.folded) scale_columns(x.t_fold + c, corr);
                }
            }
            x.l *= corr;
            x.m = now;
        }
        x.l += sum;
        tc_st<32>(x.t_p + TileShape<T, D>::P_HALF * half, pr);
        if constexpr (REST) tc_st<32>(x.t_p + 64 + TileShape<T, D>::P_HALF * half, rest);
        tc_wait_st();
        ready(half);
    }
    return 2;
}

template <typename T, int D>
__global__ void __launch_bounds__(TILE_THREADS, 1) kv_attend_tile_kernel(const __grid_constant__ AttendParams p) {
    using S = TileShape<T, D>;
    constexpr int ROWS = S::ROWS, NQ = S::NQ, TERMS = S::TERMS;
    extern __shared__ __align__(1024) uint8_t smem[];
    TileShared* sh = reinterpret_cast<TileShared*>(smem + S::END);
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int P = p.c.page_tokens, H = p.c.kv_heads;

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh->k_full[i]), TILE_MOVERS); mbar_init(smem_u32(&sh->k_empty[i]), NQ);
            mbar_init(smem_u32(&sh->v_full[i]), TILE_MOVERS); mbar_init(smem_u32(&sh->v_empty[i]), NQ);
            mbar_init(smem_u32(&sh->q_full[i]), 4); mbar_init(smem_u32(&sh->s_full[i][0]), 1); mbar_init(smem_u32(&sh->s_full[i][1]), 1);
            mbar_init(smem_u32(&sh->p_full[i][0]), 4); mbar_init(smem_u32(&sh->p_full[i][1]), 4);
            mbar_init(smem_u32(&sh->h_done[i]), 1); mbar_init(smem_u32(&sh->o_full[i]), 1);
            mbar_init(smem_u32(&sh->o_empty[i]), 4);
        }
        for (int i = 0; i < TILE_AHEAD; ++i) { mbar_init(smem_u32(&sh->i_full[i]), 1); mbar_init(smem_u32(&sh->i_empty[i]), TILE_MOVERS); }
        for (int i = 0; i < TILE_AHEAD; ++i) { mbar_init(smem_u32(&sh->g_full[i]), 1); mbar_init(smem_u32(&sh->g_empty[i]), 5 * NQ); }
        for (int i = 0; i < 4; ++i) { mbar_init(smem_u32(&sh->r_full[i]), 1); mbar_init(smem_u32(&sh->r_empty[i]), TILE_MOVERS); }
        sh->abort_flag = 0;
        sh->nan_found = 0;
        p.join[blockIdx.x] = {0, 0, 0, 0};
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 16) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    TileWalk<ROWS> w = tile_share<ROWS>(p, reinterpret_cast<int*>(smem + S::RAW_AT));      // (synchronises the block)
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem;
    bool ok = true;
    if (warp < 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(TILE_REGS_SOFTMAX));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TILE_REGS_REST));

    if (warp < 4 * NQ) {
        // ------------------------------------------------------------------------------------------ softmax
        const int qt = warp >> 2, tid = threadIdx.x & 127;
        uint8_t* q = smem + S::Q_AT + qt * S::Q;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + lanes + S::S_COL + qt * 128, t_p = tmem + lanes + S::P_COL + qt * 128;
        const uint32_t t_o = tmem + lanes + S::O_COL + qt * D;
        uint32_t s_ph = 0, o_ph = 0;
        int tile = 0;                                // tiles of the block so far, over all segments
        const int pshift = 31 - __clz(P);
        auto meet = [&](int g) {                     // waits for the news of segment g
            ok = warp_wait(&sh->g_full[g % TILE_AHEAD], (uint32_t)(g / TILE_AHEAD) & 1u, sh, p);
        };
        auto release = [&](int g) {
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->g_empty[g % TILE_AHEAD]));
        };
        auto stage = [&](const TileSegment& x) {
            const TileRow r = stage_row<T, D>(p, x, 128 * qt + tid, tid, q);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->q_full[qt]));
            return r;
        };
        TileRow row = {0, 0, 0.f, -1, 0};
        TileSoftmax x = {t_s, t_p, t_o, tmem + lanes + S::FOLD_COL, 0.f, 0.f, false, false};
        // A turn of the loop: the queries of segment g go in, then the output of the segment before comes out (it may not be
        // complete yet when they do), then g's tiles.  (Each piece of code stands here once: it is long.)
        bool before = false;                         // the segment before had rows here
        for (int g = 0; ok; ++g) {
            meet(g);
            if (!ok) break;
            const TileSegment& w = sh->seg[g % TILE_AHEAD];
            const bool live = w.live, here = live && w.nrows > 128 * qt;
            TileRow nrow = row;
            if (here) nrow = stage(w);
            if (before) {
                const TileSegment& d = sh->seg[(g - 1) % TILE_AHEAD];
                if (!(ok = warp_wait(&sh->o_full[qt], o_ph, sh, p))) break;
                o_ph ^= 1;
                tc_fence_after();
                const bool whole = d.starts && d.ends;
                const int64_t slot = (2 * (int64_t)blockIdx.x + (d.starts ? 1 : 0)) * p.slot_rows + 128 * qt + tid;
                const float inv = x.l != 0.f ? 1.f / x.l : 0.f;
                const bool nan = *(volatile int*)&sh->nan_found != 0;
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t v[32];
                    tc_ld32(t_o + c, v);
                    tc_wait_ld();
                    if (TERMS == 2 && x.folded) {
                        uint32_t u[32];
                        tc_ld32(x.t_fold + c, u);
                        tc_wait_ld();
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) + __uint_as_float(u[k]));
                    }
                    if (nan) {
                        // values that are NaN were staged as zeros where some rows do not see them: find those this row sees
                        for (int i = 0; i < d.n; ++i) {
                            const int t0 = d.t0 + i * TILE_UNIT;
                            if (t0 >= d.lo_all && t0 + TILE_UNIT <= d.hi_all) continue;
                            for (int t = max(t0, row.lo); t < min(t0 + TILE_UNIT, row.hi); ++t) {
                                const int page = load_page(p.bt, p.c, d.b, t >> pshift, nullptr);
                                if (page < 0) continue;
                                const uint32_t* src = reinterpret_cast<const uint32_t*>((const uint8_t*)p.c.codes + ((((int64_t)page * 2 + 1) * H + d.h) * P + (t & (P - 1))) * D + c);
#pragma unroll
                                for (int k = 0; k < 8; ++k) {
                                    const uint32_t n4 = __vcmpeq4(src[k] & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
#pragma unroll
                                    for (int e = 0; e < 4; ++e)
                                        if (n4 >> (8 * e) & 1u) v[4 * k + e] = 0x7FFFFFFFu;
                                }
                            }
                        }
                    }
                    if (row.token >= 0) {
                        float y[32];
#pragma unroll
                        for (int k = 0; k < 32; ++k) y[k] = whole ? (x.l != 0.f ? __uint_as_float(v[k]) * inv : 0.f) : __uint_as_float(v[k]);
                        if (whole) store_row32((T*)p.o.data + row.token * p.o.token_stride + row.head * p.o.head_stride + c, y);
                        else store_row32(p.part + slot * D + c, y);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->o_empty[qt]));
                if (row.token >= 0) {
                    if (!whole) p.part_ml[slot] = make_float2(x.m, x.l);
                    else if (p.lse) p.lse[(int64_t)row.token * p.q_heads + row.head] = lse_of(x.m, x.l);
                }
                if (d.starts && !d.ends && threadIdx.x == 0) p.join[blockIdx.x] = {d.parts, d.first * p.group + d.row0, d.nrows, d.h * p.group};
                release(g - 1);
            }
            if (!live) break;
            before = here;
            const int n = w.n;
            if (!here) {
                tile += n;
                release(g);
                continue;
            }
            row = nrow;
            x.m = -INFINITY;
            x.l = 0.f;
            x.folded = x.far = false;
            for (int i = 0; i < n; ++i, ++tile) {
                const int t0 = w.t0 + i * TILE_UNIT;
                const TileInfo& info = sh->info[tile % TILE_AHEAD];
                auto scores = [&](int half) {
                    const bool there = warp_wait(&sh->s_full[qt][half], s_ph, sh, p);
                    tc_fence_after();
                    return there;
                };
                auto ready = [&](int half) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&sh->p_full[qt][half]));
                };
                // all weights given before are summed: the first half's (half = 1), or the tile before's, whose second half went
                // to the tensor cores ahead of this tile's second scores
                auto settled = [&](int half) {
                    const bool there = warp_wait(half ? &sh->h_done[qt] : &sh->s_full[qt][1], s_ph, sh, p);
                    tc_fence_after();
                    return there;
                };
                // (the first scores' arrival says that the tile's news is there, too: it is not looked at before)
                if (!(ok = scores(0))) break;
                if (TERMS == 2 && i && i % TILE_FOLD == 0) {
                    if (!(ok = settled(0))) break;
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        uint32_t u[32], v[32];
                        tc_ld32(t_o + c, v);
                        tc_ld32(x.t_fold + c, u);
                        tc_wait_ld();
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) + (x.folded ? __uint_as_float(u[k]) : 0.f));
                        tc_st<32>(x.t_fold + c, v);
                    }
                    tc_wait_st();
                    x.folded = true;
                }
                int half = 0;
                if (!(info.edge || info.absent || x.far)) half = tile_softmax<T, D, false>(x, info.group, row, t0, i == 0, 0, scores, ready, settled);
                if (half >= 0 && half < 2) half = tile_softmax<T, D, true>(x, info.group, row, t0, i == 0, half, scores, ready, settled);
                ok = half == 2;
                s_ph ^= 1;
                if (!ok) break;
            }
        }
    } else if (warp == 17) {
        // ------------------------------------------------------------------------------------------ coming tiles
        // four tiles at a time: lane 8 k + g looks after the 16 tokens [16 g, 16 g + 16) of tile k, so that the loads of
        // four tiles (page, then its scales) are on their way together
        const int pshift = 31 - __clz(P), k = lane >> 3, g = lane & 7;
        int unit = 0, left = 0, tile = 0, seg = 0;
        auto begin = [&]() {                     // the segment w stands on: tells of it
            unit = w.unit;
            left = w.done() ? 0 : w.length();
            const int slot = seg % TILE_AHEAD;
            ok = warp_wait(&sh->g_empty[slot], ((uint32_t)(seg / TILE_AHEAD) & 1u) ^ 1u, sh, p);
            if (ok && lane == 0) {
                TileSegment x;
                x.live = left > 0;
                x.n = left;
                x.starts = unit == 0;
                x.ends = unit + left == w.t.units;
                // the block that takes the item's last unit u is the largest i with floor(i U / G) <= u
                const int64_t last = (int64_t)w.u - unit + w.t.units - 1;
                x.parts = w.done() ? 0 : (int)(((last + 1) * w.blocks - 1) / w.total) - (int)blockIdx.x + 1;
                x.b = w.b; x.h = w.h; x.row0 = w.t.row0; x.nrows = w.t.nrows;
                x.first = w.s.first; x.before = w.s.total - w.s.n; x.total = w.s.total;
                x.t0 = w.t.base + unit * TILE_UNIT;
                x.lo_all = w.t.lo_all; x.hi_all = w.t.hi_all;
                sh->seg[slot] = x;
                mbar_arrive(smem_u32(&sh->g_full[slot]));
            }
            __syncwarp();
            ++seg;
        };
        bool fresh = true;
        for (bool more = true; ok && more;) {
            int t0 = 0, lo = 0, hi = 0, b = 0, h = 0;
            bool live = false, edge = false;
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
                if (fresh && ok) begin();
                fresh = false;
                if (i == k) {
                    live = left > 0;
                    t0 = w.t.base + unit * TILE_UNIT;
                    lo = w.t.lo; hi = w.t.hi; b = w.b; h = w.h;
                    edge = t0 < w.t.lo_all || t0 + TILE_UNIT > w.t.hi_all;
                }
                if (left > 0) {
                    ++unit;
                    if (--left == 0) {
                        w.next(p);
                        fresh = true;
                    }
                } else {
                    more = false;                                               // the tile after the last is marked as none
                }
            }
            if (!ok) break;
            const int th = t0 + g * 16;
            const bool wanted = live && th < hi && th + 16 > lo;
            const int page = wanted ? load_page(p.bt, p.c, b, th >> pshift, p.status) : -1;
            float4 c = make_float4(0.f, -INFINITY, 0.f, 0.f);                    // not there: weighs nothing
            int rows = -1;
            if (page >= 0) {
                const int at = page * 2 * H + h;
                c.x = __ldg(p.c.scales + at);
                scale_terms(__ldg(p.c.scales + at + H), c.y, c.z);
                rows = (at << pshift >> 4) + ((th & (P - 1)) >> 4);
                // into L2 already: the ring of codes is not deep enough to wait for HBM
                const uint8_t* codes = (const uint8_t*)p.c.codes + (int64_t)rows * (16 * D);
                bulk_prefetch(codes, 16 * D);
                bulk_prefetch(codes + (int64_t)H * P * D, 16 * D);
            }
            const unsigned gone = __ballot_sync(0xffffffffu, wanted && page < 0);
            const int n = tile + k, slot = n % TILE_AHEAD;
            // (a wait for each of the four slots in turn: a warp's lanes do not wait for different barriers)
            for (int i = 0; i < 4 && ok; ++i) ok = warp_wait(&sh->i_empty[(tile + i) % TILE_AHEAD], ((tile + i) / TILE_AHEAD & 1) ^ 1, sh, p);
            if (!ok) break;
            TileInfo& info = sh->info[slot];
            info.group[g] = c;
            info.rows[g] = rows;
            if (g == 0) {
                info.live = live; info.edge = edge; info.t0 = t0; info.lo = lo; info.hi = hi;
                info.absent = (gone >> (8 * k) & 0xFFu) != 0;
            }
            __syncwarp();
            if (g == 0) mbar_arrive(smem_u32(&sh->i_full[slot]));
            tile += 4;
        }
    } else if (warp == 18) {
        // ------------------------------------------------------------------------------------------ codes in
        const int64_t v_codes = (int64_t)H * P * D;                             // from a key to its value
        for (int tile = 0; ok; ++tile) {
            if (!(ok = warp_wait(&sh->i_full[tile % TILE_AHEAD], (uint32_t)(tile / TILE_AHEAD) & 1u, sh, p))) break;
            const TileInfo& c = sh->info[tile % TILE_AHEAD];
            if (!c.live) break;
            const int rows = c.rows[lane & 7];
            for (int part = 0; part < 4; ++part) {                              // keys, keys, values, values
                if (!(ok = warp_wait(&sh->r_empty[part], ((uint32_t)tile & 1u) ^ 1u, sh, p))) break;
                const int mine = __shfl_sync(0xffffffffu, rows, (part & 1) * 4 + (lane & 3));
                const int n = __popc(__ballot_sync(0xffffffffu, lane < 4 && mine >= 0));
                const uint32_t bar = smem_u32(&sh->r_full[part]);
                if (lane == 0) mbar_expect_tx(bar, n * 16 * D);
                __syncwarp();
                if (lane < 4 && mine >= 0)
                    bulk_load(smem_u32(smem + S::RAW_AT + part * S::RAW + lane * 16 * D), (const uint8_t*)p.c.codes + (int64_t)mine * (16 * D) + (part >= 2 ? v_codes : 0), 16 * D, bar);
            }
        }
    } else if (warp >= 8 && warp < 16) {
        // ------------------------------------------------------------------------------------------ codes to halves
        // A thread takes 16 codes of a row at a time, a warp eight rows by four such pieces: of one half of the channels in
        // even rows and of the other in odd ones (head dimension 128), so that the eight lanes of a phase meet eight
        // different banks both reading and writing.
        const int cw = (warp - 8) & 3, values = warp >= 12, rl = lane >> 2, piece = lane & 3;
        constexpr int ROUNDS = D == 128 ? 4 : 2, STEP = D == 128 ? 16 : 32;      // rows that the four warps take at a time
        const int row_in = D == 128 ? (cw & 1) * 8 + rl : cw * 8 + rl, half = D == 128 ? (cw >> 1) ^ (rl & 1) : 0;
        const uint32_t from = row_in * D + half * 64 + piece * 16;
        const uint32_t line = half * S::HALF + row_in * 128, at0 = line + ((2 * piece) ^ rl) * 16, at1 = line + ((2 * piece + 1) ^ rl) * 16;
        // one half tile from the ring to its place; `masked`: tokens that are not there or that no row sees become zeros, and
        // so do NaN values that not every row sees (they are put in place at the end)
        auto move = [&](const TileInfo& c, int part, uint8_t* dst, bool masked) {
            const uint8_t* src = smem + S::RAW_AT + part * S::RAW + from;
            const int base = (part & 1) * 64;
            dst += base * 128;
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r) {
                uint4 raw = *reinterpret_cast<const uint4*>(src + r * (STEP * D));
                if (masked) {
                    const int at = base + r * STEP + row_in, t = c.t0 + at;
                    if (c.rows[at >> 4] < 0 || t < c.lo || t >= c.hi) raw = make_uint4(0, 0, 0, 0);
                    if (part >= 2 && c.edge) {
                        uint32_t* x = reinterpret_cast<uint32_t*>(&raw);
                        uint32_t any = 0;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t n4 = __vcmpeq4(x[k] & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
                            any |= n4;
                            x[k] &= ~n4;
                        }
                        if (any) *(volatile int*)&sh->nan_found = 1;
                    }
                }
                const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
                uint32_t y[8];
#pragma unroll
                for (int k = 0; k < 4; ++k) { y[2 * k] = e4m3x2_to_half2(w[k] & 0xFFFFu); y[2 * k + 1] = e4m3x2_to_half2(w[k] >> 16); }
                *reinterpret_cast<uint4*>(dst + r * (STEP * 128) + at0) = make_uint4(y[0], y[1], y[2], y[3]);
                *reinterpret_cast<uint4*>(dst + r * (STEP * 128) + at1) = make_uint4(y[4], y[5], y[6], y[7]);
            }
        };
        for (int tile = 0; ok; ++tile) {
            if (!(ok = warp_wait(&sh->i_full[tile % TILE_AHEAD], (uint32_t)(tile / TILE_AHEAD) & 1u, sh, p))) break;
            const TileInfo& c = sh->info[tile % TILE_AHEAD];
            if (!c.live) break;
            const bool masked = c.edge || c.absent;
            const int slot = tile & 1;
            if (!(ok = warp_wait(values ? &sh->v_empty[slot] : &sh->k_empty[slot], ((uint32_t)(tile >> 1) & 1u) ^ 1u, sh, p))) break;   // (the first use passes at once)
            uint8_t* dst = smem + (values ? S::V_AT : S::K_AT) + slot * S::KV;
#pragma unroll 1
            for (int part = 2 * values; part < 2 * values + 2; ++part) {
                if (!(ok = warp_wait(&sh->r_full[part], (uint32_t)tile & 1u, sh, p))) break;
                move(c, part, dst, masked);
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->r_empty[part]));
            }
            fence_async_smem();
            __syncwarp();
            if (ok && lane == 0) {
                mbar_arrive(smem_u32(values ? &sh->v_full[slot] : &sh->k_full[slot]));
                // the slot of values held the tile before last: its softmax is over, its news may go
                if (values && tile >= 2) mbar_arrive(smem_u32(&sh->i_empty[(tile - 2) % TILE_AHEAD]));
            }
        }
    } else if (warp == 16 || (warp == 19 && NQ == 2)) {
        // ------------------------------------------------------------------------------------------ MMAs
        const int qt = warp == 16 ? 0 : 1;
        // D = F32, A = B = F16; scores: both K-major; outputs: A in TMEM, B MN-major (bit 16)
        constexpr uint32_t I_S = (1u << 4) | ((64u >> 3) << 17) | ((128u >> 4) << 24);        // 64 tokens
        constexpr uint32_t I_O = (1u << 4) | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);
        const uint32_t hi = tile_desc_hi(1024);
        const uint32_t q_lo = ((smem_u32(smem + S::Q_AT + qt * S::Q) & 0x3FFFFu) >> 4) | (1u << 16);
        const uint32_t k_lo = ((smem_u32(smem + S::K_AT) & 0x3FFFFu) >> 4) | (1u << 16);
        const uint32_t v_lo = ((smem_u32(smem + S::V_AT) & 0x3FFFFu) >> 4) | ((S::HALF >> 4) << 16);
        const uint32_t d_s = tmem + S::S_COL + qt * 128, d_o = tmem + S::O_COL + qt * D, a_p = tmem + S::P_COL + qt * 128;
        auto scores = [&](uint32_t slot, int half) { // of 64 tokens; with the second half the slot's keys have been used
            if (elect_one()) {
                const uint32_t b0 = k_lo + slot * (S::KV >> 4) + half * (8192 >> 4);
                // (remainders first: a cut is as small as the sum it is made in; in this order 1.5e-6 of a result, else 2e-6)
#pragma unroll
                for (int t = TERMS - 1; t >= 0; --t)
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off = (k / 4) * (S::HALF >> 4) + (k % 4) * 2;
                        tc_mma_f16_ss(d_s + 64 * half, q_lo + t * (S::KV >> 4) + off, b0 + off, hi, I_S, t < TERMS - 1 || k > 0);
                    }
                tc_commit(smem_u32(&sh->s_full[qt][half]));
                if (half) tc_commit(smem_u32(&sh->k_empty[slot]));
            }
            __syncwarp();
        };
        auto outputs = [&](uint32_t slot, int half, bool first, bool last) {    // of the weights of 64 tokens
            if (elect_one()) {
                const uint32_t b0 = v_lo + slot * (S::KV >> 4) + half * (8192 >> 4), a0 = a_p + S::P_HALF * half;
                // (remainders first here, too)
#pragma unroll
                for (int t = TERMS - 1; t >= 0; --t)
#pragma unroll
                    for (int k = 0; k < 4; ++k) tc_mma_f16_ts(d_o, a0 + 64 * t + 8 * k, b0 + k * (2048 >> 4), hi, I_O, !first || t < TERMS - 1 || k > 0);
                tc_commit(smem_u32(half == 0 ? &sh->h_done[qt] : &sh->v_empty[slot]));
                if (half == 1 && last) tc_commit(smem_u32(&sh->o_full[qt]));
            }
            __syncwarp();
        };
        uint32_t q_ph = 0, p_ph = 0, o_ph = 1;
        int kt = 0, vt = 0;                          // tiles whose keys and values were used
        auto keys = [&]() { return ok = warp_wait(&sh->k_full[kt & 1], (uint32_t)(kt >> 1) & 1u, sh, p); };
        auto values = [&]() { return ok = warp_wait(&sh->v_full[vt & 1], (uint32_t)(vt >> 1) & 1u, sh, p); };
        for (int g = 0; ok; ++g) {
            if (!(ok = warp_wait(&sh->g_full[g % TILE_AHEAD], (uint32_t)(g / TILE_AHEAD) & 1u, sh, p))) break;
            const TileSegment& x = sh->seg[g % TILE_AHEAD];
            if (!x.live) break;
            const int n = x.n, nrows = x.nrows;
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->g_empty[g % TILE_AHEAD]));
            if (nrows <= 128 * qt) {                 // no rows here: gives the slots back in step
                for (int i = 0; ok && i < n; ++i, ++kt, ++vt) {
                    if (!keys()) break;
                    if (lane == 0) mbar_arrive(smem_u32(&sh->k_empty[kt & 1]));
                    if (!values()) break;
                    if (lane == 0) mbar_arrive(smem_u32(&sh->v_empty[vt & 1]));
                }
                continue;
            }
            if (!(ok = warp_wait(&sh->q_full[qt], q_ph, sh, p))) break;
            q_ph ^= 1;
            if (!keys()) break;
            tc_fence_after();
            scores(kt & 1, 0);
            scores(kt & 1, 1);
            ++kt;
            if (!(ok = warp_wait(&sh->o_empty[qt], o_ph, sh, p))) break;
            o_ph ^= 1;
            // The next tile's scores of 64 tokens go out behind the outputs of this one's, into the columns that these weights
            // leave: the softmax finds them done when it comes to them, and no product waits for a whole tile.
            for (int i = 0; ok && i < n; ++i, ++vt) {
                const bool more = i + 1 < n;
                if (!values()) break;
                if (!(ok = warp_wait(&sh->p_full[qt][0], p_ph, sh, p))) break;
                tc_fence_after();
                outputs(vt & 1, 0, i == 0 || (TERMS == 2 && i % TILE_FOLD == 0), !more);
                if (more) {
                    if (!keys()) break;
                    tc_fence_after();
                    scores(kt & 1, 0);
                }
                if (!(ok = warp_wait(&sh->p_full[qt][1], p_ph, sh, p))) break;
                p_ph ^= 1;
                tc_fence_after();
                outputs(vt & 1, 1, false, !more);
                if (more) {
                    scores(kt & 1, 1);
                    ++kt;
                }
            }
        }
    }
    if (!ok) {                                       // MMAs still reading shared memory
        const long long t = clock64();
        while (clock64() - t < 400000) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 16) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

}  // namespace ccv3d
