// Products of token rows with weights, with bias, activation or gated pair, and residual in the epilogue, on tcgen05.
//
// Few rows: bound by the weights' bytes.  Many rows: bound by the tensor cores.  One kernel for both, with the weights as the rows of
// the products (M = 256, a pair of CTAs) and BT tokens as their columns (16 for single tokens, up to 256 for frames), so that a lane of
// tensor memory is an output feature: its bias is one register, and a warp's loads and stores of a token's features are contiguous at any
// alignment and any number of features.  A gated pair has two accumulators, of its two rows of weights, side by side.
//
// 12 or 20 warps, persistent, one pair of CTAs to two SMs:
//   warp 0     TMA of weight and token tiles (K blocks of 128 bytes, F32: 64) into a ring of stages; each CTA of a pair loads its own 128
//              weight rows and half of the tokens
//   warp 1     the leader's issues the MMAs of the pair
//   warp 2     tensor memory
//   warps 4..  epilogue of one accumulator while the next is filled: four warps to the 128 lanes, the columns in two or four parts
// Tiles go round the pairs in turn; those of the last, unfilled turn are cut along K into equal shares of K blocks, whose sums
// linear_join_kernel adds in order (no atomics: the same bits every run).
//
// Measured (BF16), in short bursts at up to 1965 MHz: 9472 x 4096 -> 4096 199 us = 1.60 PFLOP/s, 97 % of a plain library product's rate;
// 28160 x 6144 -> 1536 341 us (1.56); 3520 x 1536 -> 6144 with GELU 52 us (1.28: 4.5 turns of tiles take five); gated, with SiLU, 103 us (1.29);
// 64 rows on 180 MB of gated weights 35 us (5.2 TB/s).  Again and again, under the power cap: with GELU 58 us at 1590 MHz, 28160 x 6144 -> 1536 onto an
// F32 residual 495 us (1.07) at 1350 MHz.  Tiles of 256 tokens want 92 GB/s of L2 for each SM, near what all of them get
// at once.
//
// F32 outputs, and few rows: the tensor cores cut what they add to instead of rounding it, which shrinks long sums; so accumulators are
// handed over every few K blocks and summed in registers with rounding.  (BF16 outputs of many rows stay in them; 3520 x 1536 -> 6144
// would take 6 % longer.)  F32 operands are split beforehand into three BF16 numbers each (8 + 8 + 8 bits, exact); six of the nine
// products, smallest first, keep 2^-24.
#pragma once
#include "ccv3d_tc_ptx.cuh"
#include "ccv3d_tokens_activation.cuh"
#include "ccv3d_tokens_common.cuh"

namespace ccv3d {

constexpr int LINEAR_MAX_STAGES = 12;

struct LinearParams {
    const void *bias, *res;
    void* out;
    int64_t out_stride, res_stride;
    int rows, n_out;
    int act, bias_f32;
    int n_tiles, kblocks;        // tiles of 256 features (of a pair of CTAs); K blocks of a tile
    int whole;                   // tiles 0 .. whole - 1 go round the pairs
    int tail, sharers;           // the next `tail` tiles are cut into `sharers` equal runs of K blocks
    int x_plane, w_plane;        // F32: rows between the three parts of an operand
    int pairs;
    int boxes, res_boxes;        // outputs go out, residuals come in as boxes (their rows are on 16 bytes)
    float* part;                 // [2 * sharers][columns][256 features]
    uint32_t* status;
    long long wait_clk;
};

// A piece of work: K blocks kb0 .. kb1 - 1 of a tile; slot >= 0: an unfinished sum.
struct LinearPiece { int tile, kb0, kb1, slot; };
struct LinearWalk {
    int next, pair, pairs, whole, kblocks;
    int64_t u, u1, first;
    __device__ __forceinline__ LinearWalk(const LinearParams& p, int pair_) : next(pair_), pair(pair_), pairs(p.pairs), whole(p.whole), kblocks(p.kblocks) {
        const int64_t units = (int64_t)p.tail * p.kblocks;
        u = u1 = 0;
        if (pair_ < p.sharers) { u = units * pair_ / p.sharers; u1 = units * (pair_ + 1) / p.sharers; }
        first = u;
    }
    __device__ __forceinline__ bool get(LinearPiece& w) {
        if (next < whole) {
            w = {next, 0, kblocks, -1};
            next += pairs;
            return true;
        }
        if (u >= u1) return false;
        const int t = (int)(u / kblocks);
        w.tile = whole + t;
        w.kb0 = (int)(u - (int64_t)t * kblocks);
        w.kb1 = (int)min((int64_t)kblocks, w.kb0 + u1 - u);
        w.slot = w.kb0 == 0 && w.kb1 == kblocks ? -1 : 2 * pair + (u == first ? 0 : 1);
        u += w.kb1 - w.kb0;
        return true;
    }
};

template <int BT_, bool GATED_, int PARTS_, bool F32_OUT> struct LinearShape {
    static constexpr int BT = BT_, PARTS = PARTS_, SETS = GATED_ ? 2 : 1;
    static constexpr bool GATED = GATED_, F32 = F32_OUT, FOLD = F32_OUT || BT_ <= 64;
    static constexpr int COLS = SETS * BT;                                   // of an accumulator
    static constexpr int ROWB = PARTS == 3 ? 64 : 128, KB = ROWB / 2;        // bytes and elements of a row of a stage
    static constexpr uint32_t A_TILE = 128 * ROWB, B_TILE = BT / 2 * ROWB, A_BYTES = PARTS * SETS * A_TILE, STAGE = A_BYTES + PARTS * B_TILE;
    static constexpr int EPI_WARPS = FOLD && COLS == 256 ? 16 : 8, PARTS_OF_COLS = EPI_WARPS / 4, CW = BT / PARTS_OF_COLS;   // CW: tokens of a warp
    static constexpr int LD = CW < 16 ? CW : 16, CH = F32_OUT || CW < 32 ? LD : 32;   // columns read at a time onto rounded sums; finished at a time
    static constexpr int THREADS = 128 + 32 * EPI_WARPS;
    static constexpr uint32_t TMEM = 2 * COLS < 32 ? 32 : 2 * COLS;
    // K blocks between hand-overs of a sum that is kept with rounding: 64 terms of F32 (with their remainders), 512 of BF16 into F32 (errors half to all
    // of those of FP32 arithmetic, which twice as many had more of: 4.5e-7 of the largest listed product against 3.6e-7, now 2.1e-7 at 3 % more
    // time), 1024 into BF16 where rows are few and time goes by the weights' bytes
    static constexpr int HAND = FOLD ? (PARTS == 3 ? 2 : F32_OUT ? 8 : 16) : 1 << 30;
    // outputs on their way: two boxes of 32 features and CH tokens for each warp
    static constexpr uint32_t BOX = 32 * CH * (F32_OUT ? 4 : 2), BOXES = 2 * EPI_WARPS * BOX;
    static constexpr int FIT = (int)((230400 - 1024 - BOXES) / STAGE), STAGES = FIT < LINEAR_MAX_STAGES ? FIT : LINEAR_MAX_STAGES;
    static constexpr uint32_t SMEM = STAGES * STAGE + BOXES + 1024;
    static_assert(STAGES >= 2 && SMEM <= 230400 && BOX % 128 == 0 && (CW == 8 || CW % 32 == 0) && (TMEM & (TMEM - 1)) == 0, "");
};

struct LinearShared {
    uint64_t full[LINEAR_MAX_STAGES], empty[LINEAR_MAX_STAGES], acc_full[2], acc_empty[2], res_full[16][2];
    uint32_t tmem;
    int abort_flag;
};

// Bounded wait; false when it gave up or another role did.
__device__ __forceinline__ bool linear_wait(uint64_t* bar, uint32_t parity, LinearShared* sh, const LinearParams& p) {
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
__device__ __forceinline__ bool linear_warp_wait(uint64_t* bar, uint32_t parity, LinearShared* sh, const LinearParams& p) {
    return __all_sync(0xffffffffu, linear_wait(bar, parity, sh, p));
}

template <int N>
__device__ __forceinline__ void tc_ld(uint32_t at, uint32_t (&v)[32]) {
    if constexpr (N == 32) tc_ld32(at, v);
    else if constexpr (N == 16) tc_ld16(at, v);
    else {
        static_assert(N == 8, "");
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                     : "r"(at)
                     : "memory");
    }
}

__device__ __forceinline__ float bias_at(const LinearParams& p, int i) {
    return p.bias_f32 ? __ldg((const float*)p.bias + i) : __bfloat162float(((const __nv_bfloat16*)p.bias)[i]);
}

__device__ __forceinline__ void tma_store_2d(const CUtensorMap* tm, uint32_t src, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(tm), "r"(src), "r"(c0), "r"(c1) : "memory");
}

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* tm, uint32_t bar, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(tm), "r"(c0),
                 "r"(c1), "r"(bar)
                 : "memory");
}

// The epilogue of N tokens t0 .. of one feature: g (and u) hold the sums, bg and bu the biases; the results are in g.  `box`: where the
// residual lies in shared memory, 0: where p.res says.
template <typename TO, bool GATED, int N>
__device__ __forceinline__ void linear_epilogue(const LinearParams& p, int n, int t0, float (&g)[N], const float (&u)[N], float bg, float bu, uint32_t box = 0) {
    const int live = n < p.n_out ? min(N, p.rows - t0) : 0;
    float r[N];
    if (box) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if constexpr (sizeof(TO) == 4) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(r[j]) : "r"(box + (j * 32 + (threadIdx.x & 31)) * 4) : "memory");
            else {
                unsigned short h;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(box + (j * 32 + (threadIdx.x & 31)) * 2) : "memory");
                r[j] = __uint_as_float((uint32_t)h << 16);
            }
        }
    } else if (p.res) {
        const TO* at = (const TO*)p.res + (int64_t)t0 * p.res_stride + n;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            r[j] = j < live ? load1(at) : 0.f;
            at += p.res_stride;
        }
    }
    with_activation(p.act, [&](auto kind) {
#pragma unroll
        for (int j = 0; j < N; ++j) g[j] += bg;
        // (each value by itself: its neighbours here are other tokens', whose contents must not reach its last bits; 3520 x 1536 -> 6144 with GELU
        // takes as long as with a reciprocal for two)
#pragma unroll
        for (int j = 0; j < N; ++j) g[j] = activate<sizeof(TO) == 4>(g[j], decltype(kind)::value);
        if (GATED) {
#pragma unroll
            for (int j = 0; j < N; ++j) g[j] *= u[j] + bu;
        }
    });
    if (p.res) {
#pragma unroll
        for (int j = 0; j < N; ++j) g[j] += r[j];
    }
}
template <typename TO, int N>
__device__ __forceinline__ void linear_put(const LinearParams& p, int n, int t0, const float (&g)[N]) {
    const int live = n < p.n_out ? min(N, p.rows - t0) : 0;
    TO* at = (TO*)p.out + (int64_t)t0 * p.out_stride + n;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (j < live) store1(at, g[j]);
        at += p.out_stride;
    }
}

template <typename S, typename TO>
__global__ void __launch_bounds__(S::THREADS, 1) __cluster_dims__(2, 1, 1)
linear_tile_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_o,
                   const __grid_constant__ CUtensorMap tm_r, const __grid_constant__ LinearParams p) {
    extern __shared__ uint8_t linear_smem[];
    __shared__ LinearShared shared;
    LinearShared* sh = &shared;
    const uint32_t base = (smem_u32(linear_smem) + 1023u) & ~1023u;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x >> 1;
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::STAGES; ++i) { mbar_init(smem_u32(&sh->full[i]), 1); mbar_init(smem_u32(&sh->empty[i]), 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&sh->acc_full[i]), 1); mbar_init(smem_u32(&sh->acc_empty[i]), 2 * S::EPI_WARPS); }
        for (int i = 0; i < S::EPI_WARPS; ++i) { mbar_init(smem_u32(&sh->res_full[i][0]), 1); mbar_init(smem_u32(&sh->res_full[i][1]), 1); }
        sh->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    cluster_sync_all();                  // both CTAs' barriers exist before anything of the peer can arrive on them
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem)), "r"(S::TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem;
    asm volatile("griddepcontrol.wait;" ::: "memory");               // (the split operands)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    bool ok = true;
    LinearWalk walk(p, pair);
    LinearPiece w;
    if (warp == 0) {
        // ------------------------------------------------------------------------------------------ loads
        if (lane == 0) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_w) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_x) : "memory");
            int s = 0;
            uint32_t ph = 1;
            while (ok && walk.get(w)) {
                const int nt = w.tile % p.n_tiles, f0 = nt * 256 + (int)rank * 128, t0 = w.tile / p.n_tiles * S::BT + (int)rank * (S::BT / 2);
                for (int kb = w.kb0; kb < w.kb1; ++kb) {
                    if (!(ok = linear_wait(&sh->empty[s], ph, sh, p))) break;
                    const uint32_t bar = smem_u32(&sh->full[s]), at = base + s * S::STAGE;
                    if (rank == 0) mbar_expect_tx(bar, 2 * S::STAGE);      // both CTAs' boxes are counted on the leader's barrier
#pragma unroll
                    for (int i = 0; i < S::PARTS; ++i) {
#pragma unroll
                        for (int h = 0; h < S::SETS; ++h)
                            tma_load_2d_pair(at + (i * S::SETS + h) * S::A_TILE, &tm_w, bar, kb * S::KB, i * p.w_plane + h * p.n_out + f0);
                        tma_load_2d_pair(at + S::A_BYTES + i * S::B_TILE, &tm_x, bar, kb * S::KB, i * p.x_plane + t0);
                    }
                    if (++s == S::STAGES) { s = 0; ph ^= 1; }
                }
            }
        }
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------------------------------------------------ MMAs
        // D = F32, A = B = BF16, both K-major, M = 256, N = BT
        constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(S::BT >> 3) << 17) | ((256u >> 4) << 24);
        constexpr uint32_t HI = ((8u * S::ROWB) >> 4) | (1u << 14) | ((S::ROWB == 128 ? 2u : 4u) << 29);
        const uint32_t a0 = ((base & 0x3FFFFu) >> 4) | (1u << 16), b0 = a0 + (S::A_BYTES >> 4);
        int s = 0, acc = 0;
        uint32_t ph = 0, acc_ph = 1;
        while (ok && walk.get(w)) {
            for (int kb = w.kb0; ok && kb < w.kb1;) {
                const int end = min(w.kb1 - kb, S::HAND) + kb;
                if (!(ok = linear_warp_wait(&sh->acc_empty[acc], acc_ph, sh, p))) break;
                tc_fence_after();
                const uint32_t d = tmem + acc * S::COLS;
                uint32_t add = 0;
                for (; kb < end; ++kb) {
                    if (!(ok = linear_warp_wait(&sh->full[s], ph, sh, p))) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t a = a0 + s * (S::STAGE >> 4), b = b0 + s * (S::STAGE >> 4);
#pragma unroll
                        for (int o = S::PARTS - 1; o >= 0; --o)          // products of parts i and o - i: the small ones first
#pragma unroll
                            for (int i = o; i >= 0; --i)
#pragma unroll
                                for (int k = 0; k < S::KB / 16; ++k)
#pragma unroll
                                    for (int h = 0; h < S::SETS; ++h)
                                        tc_mma_bf16_pair(d + h * S::BT, a + (i * S::SETS + h) * (S::A_TILE >> 4) + 2 * k, HI, b + (o - i) * (S::B_TILE >> 4) + 2 * k, HI,
                                                         IDESC, o < S::PARTS - 1 || i < o || k > 0 ? 1u : add);
                        tc_commit_pair(smem_u32(&sh->empty[s]));
                        if (kb + 1 == end) tc_commit_pair(smem_u32(&sh->acc_full[acc]));
                    }
                    __syncwarp();
                    add = 1;
                    if (++s == S::STAGES) { s = 0; ph ^= 1; }
                }
                acc ^= 1;
                if (acc == 0) acc_ph ^= 1;
            }
        }
    } else if (warp >= 4) {
        // ------------------------------------------------------------------------------------------ epilogue
        const int q = warp & 3, half = (warp - 4) >> 2;                 // lanes 32 q .., part of the columns
        const uint32_t mine = tmem + ((uint32_t)q << 21) + half * S::CW;
        const uint32_t box = base + S::STAGES * S::STAGE + (warp - 4) * 2 * S::BOX;
        int acc = 0;
        uint32_t ph = 0, turn = 0, res_ph = 0;
        while (ok && walk.get(w)) {
            const int nt = w.tile % p.n_tiles, f = (int)rank * 128 + q * 32 + lane, n = nt * 256 + f, t0 = w.tile / p.n_tiles * S::BT + half * S::CW;
            float bg = 0.f, bu = 0.f;
            if (p.bias && n < p.n_out) {
                bg = bias_at(p, n);
                if (S::GATED) bu = bias_at(p, p.n_out + n);
            }
            // the residual's first boxes come in while the sums are made, the rest of it comes to L2
            auto ask = [&](int c, uint32_t b) {
                if (lane == 0) {
                    const uint32_t bar = smem_u32(&sh->res_full[warp - 4][b]);
                    mbar_expect_tx(bar, S::BOX);
                    tma_load_2d(box + b * S::BOX, &tm_r, bar, n, t0 + c);
                }
            };
            if (p.res && w.slot < 0) {
                if (p.res_boxes) {
                    // all lanes have read the last tile's residual from the boxes, and its outputs have left them
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) bulk_wait_read<0>();
                    ask(0, turn);
                    if (S::CW > S::CH) ask(S::CH, turn ^ 1);
                }
                if (n - lane < p.n_out && (S::CW > 2 * S::CH || !p.res_boxes))
                    for (int j = lane; j < min(S::CW, p.rows - t0); j += 32)
                        asm volatile("prefetch.global.L2 [%0];" ::"l"((const TO*)p.res + (int64_t)(t0 + j) * p.res_stride + (n - lane)));
            }
            // sums of CH tokens from column c of the warp's on: finished, or put down for the join
            auto leave = [&](int c, float (&g)[S::CH], float (&u)[S::CH]) {
                if (w.slot >= 0) {
                    float* at = p.part + ((int64_t)w.slot * S::COLS + half * S::CW + c) * 256 + f;
#pragma unroll
                    for (int j = 0; j < S::CH; ++j) {
                        at[j * 256] = g[j];
                        if (S::GATED) at[(S::BT + j) * 256] = u[j];
                    }
                    return;
                }
                const uint32_t b = turn, at = box + b * S::BOX;
                const bool by_box = p.res && p.res_boxes;
                if (by_box) {
                    ok = linear_warp_wait(&sh->res_full[warp - 4][b], res_ph >> b & 1u, sh, p) && ok;
                    res_ph ^= 1u << b;
                }
                linear_epilogue<TO, S::GATED, S::CH>(p, n, t0 + c, g, u, bg, bu, by_box ? at : 0u);
                if (p.boxes || by_box) turn ^= 1;
                if (!p.boxes) {
                    linear_put<TO, S::CH>(p, n, t0 + c, g);
                    if (by_box && c + 2 * S::CH < S::CW) {
                        fence_async_smem();                      // (read before it is written again)
                        __syncwarp();
                        ask(c + 2 * S::CH, b);
                    }
                    return;
                }
                if (!by_box) {
                    if (lane == 0) bulk_wait_read<1>();          // the box before the last has left its place
                    __syncwarp();
                }
#pragma unroll
                for (int j = 0; j < S::CH; j += 2) {
                    if constexpr (sizeof(TO) == 4) {
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + (j * 32 + lane) * 4), "f"(g[j]) : "memory");
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + (j * 32 + 32 + lane) * 4), "f"(g[j + 1]) : "memory");
                    } else {
                        const uint32_t two = pack_bf16(g[j], g[j + 1]);
                        asm volatile("st.shared.u16 [%0], %1;" ::"r"(at + (j * 32 + lane) * 2), "h"((unsigned short)two) : "memory");
                        asm volatile("st.shared.u16 [%0], %1;" ::"r"(at + (j * 32 + 32 + lane) * 2), "h"((unsigned short)(two >> 16)) : "memory");
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (n < p.n_out && t0 + c < p.rows) tma_store_2d(&tm_o, at, n, t0 + c);
                    bulk_commit();
                }
                if (by_box && c + 2 * S::CH < S::CW) {           // this box's place takes the residual after next
                    if (lane == 0) bulk_wait_read<0>();
                    ask(c + 2 * S::CH, b);
                }
            };
            // (one accumulator's worth of a BF16 output: straight from tensor memory)
            const bool whole = !S::FOLD || (!S::F32 && w.kb1 - w.kb0 <= S::HAND);
            if constexpr (S::FOLD) {
                if (!whole) {
                    float sum[S::SETS][S::CW];
#pragma unroll
                    for (int h = 0; h < S::SETS; ++h)
#pragma unroll
                        for (int j = 0; j < S::CW; ++j) sum[h][j] = 0.f;
                    for (int kb = w.kb0; kb < w.kb1; kb += S::HAND) {
                        if (!(ok = linear_warp_wait(&sh->acc_full[acc], ph, sh, p))) break;
                        tc_fence_after();
#pragma unroll
                        for (int h = 0; h < S::SETS; ++h)
#pragma unroll
                            for (int c = 0; c < S::CW; c += S::LD) {
                                uint32_t v[32];
                                tc_ld<S::LD>(mine + acc * S::COLS + h * S::BT + c, v);
                                tc_wait_ld();
#pragma unroll
                                for (int j = 0; j < S::LD; ++j) sum[h][c + j] += __uint_as_float(v[j]);
                            }
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_leader(smem_u32(&sh->acc_empty[acc]));
                        acc ^= 1;
                        if (acc == 0) ph ^= 1;
                    }
                    if (ok) {
#pragma unroll
                        for (int c = 0; c < S::CW; c += S::CH) {
                            float g[S::CH], u[S::CH];
#pragma unroll
                            for (int j = 0; j < S::CH; ++j) { g[j] = sum[0][c + j]; u[j] = sum[S::SETS - 1][c + j]; }
                            leave(c, g, u);
                        }
                    }
                }
            }
            if constexpr (!S::FOLD || !S::F32) {
                if (whole) {
                    if (!(ok = linear_warp_wait(&sh->acc_full[acc], ph, sh, p))) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < S::CW; c += S::CH) {
                        uint32_t v[2][32];
#pragma unroll
                        for (int h = 0; h < S::SETS; ++h) tc_ld<S::CH>(mine + acc * S::COLS + h * S::BT + c, v[h]);
                        tc_wait_ld();
                        if (c + S::CH == S::CW) {
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive_leader(smem_u32(&sh->acc_empty[acc]));
                        }
                        float g[S::CH], u[S::CH];
#pragma unroll
                        for (int j = 0; j < S::CH; ++j) { g[j] = __uint_as_float(v[0][j]); u[j] = __uint_as_float(v[S::SETS - 1][j]); }
                        leave(c, g, u);
                    }
                    acc ^= 1;
                    if (acc == 0) ph ^= 1;
                }
            }
        }
        if (lane == 0) bulk_wait_read<0>();          // (the boxes' places are this block's)
    }
    if (!ok) {                                       // loads and MMAs still in flight
        const long long t = clock64();
        while (clock64() - t < 400000) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                              // the leader's MMAs read the peer's shared memory and write its tensor memory
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::TMEM) : "memory");
    }
}

// The sums of the tiles that were cut along K: block (tile of the tail, group of 8 tokens), a thread to a feature.
constexpr int LINEAR_JOIN_TOKENS = 8;
template <typename TO, bool GATED>
__global__ void __launch_bounds__(256) linear_join_kernel(const __grid_constant__ LinearParams p, int BT) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int t = blockIdx.x, c = blockIdx.y * LINEAR_JOIN_TOKENS, f = threadIdx.x, tile = p.whole + t, cols = GATED ? 2 * BT : BT;
    const int n = tile % p.n_tiles * 256 + f, t0 = tile / p.n_tiles * BT + c;
    const int64_t units = (int64_t)p.tail * p.kblocks, begin = (int64_t)t * p.kblocks, end = begin + p.kblocks;
    const int64_t from = ((begin + 1) * p.sharers - 1) / units, to = (end * p.sharers - 1) / units;      // the sharers of the first and last K block
    if (from == to || n >= p.n_out || t0 >= p.rows) return;
    float g[LINEAR_JOIN_TOKENS], u[LINEAR_JOIN_TOKENS];
#pragma unroll
    for (int j = 0; j < LINEAR_JOIN_TOKENS; ++j) g[j] = u[j] = 0.f;
    for (int64_t i = from; i <= to; ++i) {
        const int64_t slot = 2 * i + (units * i / p.sharers >= begin ? 0 : 1);
        const float* at = p.part + (slot * cols + c) * 256 + f;
#pragma unroll
        for (int j = 0; j < LINEAR_JOIN_TOKENS; ++j) {
            g[j] += at[j * 256];
            if (GATED) u[j] += at[(BT + j) * 256];
        }
    }
    float bg = 0.f, bu = 0.f;
    if (p.bias) {
        bg = bias_at(p, n);
        if (GATED) bu = bias_at(p, p.n_out + n);
    }
    linear_epilogue<TO, GATED, LINEAR_JOIN_TOKENS>(p, n, t0, g, u, bg, bu);
    linear_put<TO, LINEAR_JOIN_TOKENS>(p, n, t0, g);
}

// Few rows of F32: bound by the weights' bytes, which splitting them would double and double again; so in plain FP32 arithmetic.  A thread has
// two features of a tile of 256 and BT tokens.  Weights come in by cp.async, K blocks of 32, in rows of 128 bytes whose 16-byte pieces are
// swapped by row so that eight threads read eight banks' worth; tokens through registers, one block ahead.  Sums of 64 terms are added up
// apart (of 256, in the same time, errors were 1.3 to 1.8 times as large).
constexpr int LINEAR_FEW_K = 32, LINEAR_FEW_FOLD = 2, LINEAR_FEW_THREADS = 128, LINEAR_FEW_STAGES = 3;
template <bool GATED, int BT>
__global__ void __launch_bounds__(LINEAR_FEW_THREADS) linear_few_kernel(const __grid_constant__ LinearParams p, const float* x, int64_t x_stride, const float* w,
                                                                        int64_t w_stride, int k) {
    constexpr int SETS = GATED ? 2 : 1, KB = LINEAR_FEW_K, COLS = SETS * BT, ROWS = SETS * 256, XQ = BT * (KB / 4) / LINEAR_FEW_THREADS, NST = LINEAR_FEW_STAGES;
    extern __shared__ __align__(16) float few[];
    float *ws = few, *xs = few + NST * ROWS * KB;                 // weights [stage][row][KB], tokens [2][k][BT]
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int t = threadIdx.x;
    LinearWalk walk(p, blockIdx.x);
    LinearPiece piece;
    while (walk.get(piece)) {
        const int n0 = piece.tile % p.n_tiles * 256, t0 = piece.tile / p.n_tiles * BT, blocks = piece.kb1 - piece.kb0;
        float total[SETS][2][BT], sum[SETS][2][BT], xr[XQ][4];
#pragma unroll
        for (int h = 0; h < SETS; ++h)
#pragma unroll
            for (int j = 0; j < 2 * BT; ++j) total[h][j / BT][j % BT] = sum[h][j / BT][j % BT] = 0.f;
        auto bring = [&](int i) {                                 // weights of the piece's i-th K block; what is not there is zero
            if (i < blocks) {
                const int k0 = (piece.kb0 + i) * KB, c = t & 7, left = max(0, min(16, (k - k0 - 4 * c) * 4));
#pragma unroll 4
                for (int r = t >> 3; r < ROWS; r += LINEAR_FEW_THREADS / 8) {
                    const int f = r & 255, row = (r >> 8) * p.n_out + n0 + f;
                    const int size = n0 + f < p.n_out ? left : 0;
                    const uint32_t dst = smem_u32(ws + (i % NST * ROWS + r) * KB + ((c ^ (r & 7)) << 2));
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(size ? w + row * w_stride + k0 + 4 * c : w), "r"(size) : "memory");
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        auto tokens = [&](int i) {                                // of the i-th, into registers
            const int k0 = (piece.kb0 + i) * KB;
#pragma unroll
            for (int e = 0; e < XQ; ++e) {
                const int at = t + e * LINEAR_FEW_THREADS, r = at / (KB / 4), c = at % (KB / 4) * 4;
                const float* from = x + (int64_t)(t0 + r) * x_stride + k0 + c;
#pragma unroll
                for (int j = 0; j < 4; ++j) xr[e][j] = 0.f;
                if (t0 + r < p.rows && i < blocks) {
                    if (k0 + c + 4 <= k) load4(from, xr[e]);
                    else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) if (k0 + c + j < k) xr[e][j] = from[j];
                    }
                }
            }
        };
        __syncthreads();                                          // the last piece's stages have been read
#pragma unroll
        for (int i = 0; i < NST - 1; ++i) bring(i);
        tokens(0);
        for (int i = 0; i < blocks; ++i) {
            asm volatile("cp.async.wait_group %0;" ::"n"(NST - 2) : "memory");
            float* xb = xs + (i & 1) * KB * BT;
#pragma unroll
            for (int e = 0; e < XQ; ++e) {
                const int at = t + e * LINEAR_FEW_THREADS, r = at / (KB / 4), c = at % (KB / 4) * 4;
#pragma unroll
                for (int j = 0; j < 4; ++j) xb[(c + j) * BT + r] = xr[e][j];
            }
            __syncthreads();
            bring(i + NST - 1);
            tokens(i + 1);
            const float* wb = ws + i % NST * ROWS * KB;
#pragma unroll 2
            for (int c = 0; c < KB; c += 4) {
                float a[SETS][2][4];
#pragma unroll
                for (int h = 0; h < SETS; ++h)
#pragma unroll
                    for (int f = 0; f < 2; ++f) load4(wb + (h * 256 + f * 128 + t) * KB + (((c >> 2) ^ (t & 7)) << 2), a[h][f]);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                    for (int j = 0; j < BT; j += 4) {
                        float v[4];
                        load4(xb + (c + kk) * BT + j, v);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
#pragma unroll
                            for (int h = 0; h < SETS; ++h)
#pragma unroll
                                for (int f = 0; f < 2; ++f) sum[h][f][j + e] = fmaf(a[h][f][kk], v[e], sum[h][f][j + e]);
                    }
            }
            if (i % LINEAR_FEW_FOLD == LINEAR_FEW_FOLD - 1 || i + 1 == blocks) {
#pragma unroll
                for (int h = 0; h < SETS; ++h)
#pragma unroll
                    for (int j = 0; j < 2 * BT; ++j) { total[h][j / BT][j % BT] += sum[h][j / BT][j % BT]; sum[h][j / BT][j % BT] = 0.f; }
            }
        }
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            const int n = n0 + f * 128 + t;
            if (piece.slot >= 0) {
                float* at = p.part + (int64_t)piece.slot * COLS * 256 + f * 128 + t;
#pragma unroll
                for (int h = 0; h < SETS; ++h)
#pragma unroll
                    for (int j = 0; j < BT; ++j) at[(h * BT + j) * 256] = total[h][f][j];
                continue;
            }
            float bg = 0.f, bu = 0.f;
            if (p.bias && n < p.n_out) {
                bg = bias_at(p, n);
                if (GATED) bu = bias_at(p, p.n_out + n);
            }
            linear_epilogue<float, GATED, BT>(p, n, t0, total[0][f], total[SETS - 1][f], bg, bu);
            linear_put<float, BT>(p, n, t0, total[0][f]);
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// F32 rows of both operands as three BF16 numbers each, in three planes [rows][pitch]: rounded to 8 bits, what is left to 8 more, and the
// rest (8 bits: exact).  A thread to four elements.
__global__ void __launch_bounds__(256) linear_split_kernel(const float* w, int64_t w_stride, int w_rows, __nv_bfloat16* w_to, const float* x, int64_t x_stride,
                                                           int x_rows, __nv_bfloat16* x_to, int k, int pitch) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int quads = pitch / 4;
    const int64_t w_all = (int64_t)w_rows * quads, all = w_all + (int64_t)x_rows * quads;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < all; i += (int64_t)gridDim.x * blockDim.x) {
        const bool of_x = i >= w_all;
        const int64_t j0 = of_x ? i - w_all : i, r = j0 / quads, plane = (int64_t)(of_x ? x_rows : w_rows) * pitch;
        const int c = (int)(j0 - r * quads) * 4;
        float v[4] = {0.f, 0.f, 0.f, 0.f}, a[4], b[4], d[4];
        const float* at = of_x ? x + r * x_stride + c : w + r * w_stride + c;
        if (c + 4 <= k) load4(at, v);
        else
            for (int j = 0; c + j < k; ++j) v[j] = at[j];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float whole = 3.38953138925e38f;                        // largest BF16 number: what lies above it must not become an infinity
            a[j] = isinf(v[j]) ? v[j] : __bfloat162float(__float2bfloat16_rn(isnan(v[j]) ? v[j] : fminf(fmaxf(v[j], -whole), whole)));
            const float rest = isfinite(v[j]) ? v[j] - a[j] : 0.f;
            b[j] = __bfloat162float(__float2bfloat16_rn(rest));
            d[j] = rest - b[j];
        }
        __nv_bfloat16* o = (of_x ? x_to : w_to) + r * pitch + c;
        store4(o, a);
        store4(o + plane, b);
        store4(o + 2 * plane, d);
    }
}

}  // namespace ccv3d
