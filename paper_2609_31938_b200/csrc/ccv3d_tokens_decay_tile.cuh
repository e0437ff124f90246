// Attention with decaying states on tcgen05: many tokens, BF16 (the mathematics stand in ccv3d_tokens_decay.cuh).
//
// Bound by the arithmetic around the products: scores and their decay, the values' decay, the state's split into BF16 parts.  A block has 128
// value columns of one state and goes over its tokens in chunks of 64.  With the value columns as the rows of every product (M = 128), a lane of
// tensor memory is a value column throughout:
//   D3 [value, key]   = V'^T K     values with their decay to the chunk's end (three parts), what the state gains
//   D1 [value, token] = S^T Q^T    the state before the chunk (two parts)
//   D2 [value, token] = V^T P^T    scores times decay (two parts)
//   out = scale (exp(G) D1 + D2);  S = exp(G_end) S + D3
// 20 warps:
//   0-7    bring q, k, v in (cp.async, a chunk ahead), decay the values, make scores (mma.sync, 64 x 64) and P
//   8-15   the state in registers (lane: value column; half of the keys each): its update, its parts to shared memory, and the outputs
//   16     issues the MMAs: D3 as soon as the values are there, D1 and D2 when scores and state are
//   17     the sums of log decays, ahead of the others (18, 19: none)
// Measured: one stream of 28160 tokens, 12 heads of 128 x 128, 269 us a call in three kernels (shares: states 31 %, scan 4 %, outputs 65 %; a floor of
// 53 us of bytes).
// A chunk takes 1.9 us where only the state is gained and some 4 us with outputs: the chains front -> products -> state, not the tensor cores
// (0.8 us) nor the issue slots (1.9 us).
#pragma once
#include "ccv3d_tc_ptx.cuh"
#include "ccv3d_tokens_decay.cuh"

namespace ccv3d {

// registers of 256, 256 and 128 threads: 61440, what 640 threads are launched with at 96
constexpr int DECAY_REGS_FRONT = 88, DECAY_REGS_STATE = 128, DECAY_REGS_REST = 48;
constexpr int DECAY_TILE_THREADS = 640, DECAY_TILE_DV = 128, DECAY_TILE_RING = 5;

template <int DK> struct DecayTileShape {
    static constexpr uint32_t HALF = 64 * 128;                            // 64 tokens of 64 channels
    static constexpr uint32_t QK = DK / 64 * HALF, V = 2 * HALF, STAGE = 2 * QK + V;
    static constexpr uint32_t S_HALF = 128 * 128, S_PART = DK / 64 * S_HALF;   // 128 value columns of 64 keys
    static constexpr uint32_t P_AT = 2 * STAGE, VD_AT = P_AT + 2 * HALF, S_AT = VD_AT + 3 * V, SHARED_AT = S_AT + 2 * S_PART;
};

struct DecayTileShared {
    // (a ring of five: the outputs of chunk c - 2 may still be made while the sums of chunk c + 2 are taken)
    float begin[DECAY_TILE_RING][DECAY_CHUNK];      // exp(G_i)
    float last[DECAY_TILE_RING];                    // exp(G_end); -1: log decays that are not for products
    int odd[DECAY_TILE_RING];
    uint32_t tmem;
    int abort_flag;
    alignas(16) float2 g[2][DECAY_CHUNK];           // (read two at a time)
    float end[2][DECAY_CHUNK];
    uint64_t told[4], g_full[2], g_empty[2], v_ready, v_used, ready, used, s_full, out_full[2], out_empty[2], d3_full[2], d3_empty[2], meet_full, meet_empty, odd_done;
};

// Bounded wait of a whole warp; false when it gave up or another did.  Warps that meet at named barriers go on to the end all the same, every
// further wait returning at once, so that none is left waiting there.
__device__ __forceinline__ bool decay_wait(uint64_t* bar, uint32_t parity, DecayTileShared* sh, const DecayParams& p) {
    const uint32_t b = smem_u32(bar);
    bool ok = true;
    if (!mbar_try_wait(b, parity)) {
        const long long since = clock64();
#pragma unroll 1
        while (!mbar_try_wait(b, parity)) {
            if (*(volatile int*)&sh->abort_flag) { ok = false; break; }
            if (clock64() - since > p.wait_clk) {
                *(volatile int*)&sh->abort_flag = 1;
                report(p.status, CCV3D_TOKENS_TIMEOUT);
                ok = false;
                break;
            }
        }
    }
    return __all_sync(0xffffffffu, ok);
}

static_assert(DecayTileShape<128>::SHARED_AT + sizeof(DecayTileShared) <= 232448, "shared memory of a block");

// A position in a matrix of rows of 64 BF16 numbers (128 bytes, 128-byte swizzle): row r, 16-byte piece c.
__device__ __forceinline__ uint32_t swizzled(int r, int c) { return r * 128 + ((c ^ (r & 7)) << 4); }

__device__ __forceinline__ void decay_mma(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t add) {
    constexpr uint32_t HI = (1024u >> 4) | (1u << 14) | (2u << 29);      // eight rows of 128 bytes, 128-byte swizzle
    tc_mma_bf16(d, a_lo, HI, b_lo, HI, idesc, add);
}

template <int DK, int MODE>
__global__ void __launch_bounds__(DECAY_TILE_THREADS, 1) decay_tile_kernel(const __grid_constant__ DecayParams p) {
    using S = DecayTileShape<DK>;
    using T = __nv_bfloat16;
    constexpr int L = DECAY_CHUNK, KH = DK / 2;               // KH: keys of a thread of the state
    constexpr bool OUT = MODE != DECAY_STATES;
    extern __shared__ uint8_t decay_tile_smem[];
    uint8_t* base = decay_tile_smem;                           // (all shared memory there is: on 1024 bytes)
    DecayTileShared* sh = reinterpret_cast<DecayTileShared*>(base + S::SHARED_AT);
    const uint32_t at0 = smem_u32(base);
    const int t = threadIdx.x, warp = __shfl_sync(0xffffffffu, t >> 5, 0), lane = t & 31;
    const int slices = (p.m.value_dim + DECAY_TILE_DV - 1) / DECAY_TILE_DV, slice = blockIdx.y % slices, h = blockIdx.y / slices;
    const int dv0 = slice * DECAY_TILE_DV, dvs = min(DECAY_TILE_DV, p.m.value_dim - dv0);
    DecayWork work;
    if (!decay_work<MODE>(p, h, DK, work, (int*)sh->begin)) return;
    const int first = work.first, n = work.n;
    const int chunks = (n + L - 1) / L;
    if (at0 & 1023u) {                                         // (not so: nothing is touched)
        if (t == 0) report(p.status, CCV3D_TOKENS_TIMEOUT);
        return;
    }
    if (t == 0) {
        for (int i = 0; i < 4; ++i) mbar_init(smem_u32(&sh->told[i]), 1);
        mbar_init(smem_u32(&sh->v_ready), 8);
        mbar_init(smem_u32(&sh->v_used), 1);
        mbar_init(smem_u32(&sh->ready), 8);
        mbar_init(smem_u32(&sh->used), 1);
        mbar_init(smem_u32(&sh->s_full), 8);
        mbar_init(smem_u32(&sh->meet_full), 4);
        mbar_init(smem_u32(&sh->meet_empty), 4);
        mbar_init(smem_u32(&sh->odd_done), 8);
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh->g_full[i]), 1);
            mbar_init(smem_u32(&sh->g_empty[i]), 8);
            mbar_init(smem_u32(&sh->out_full[i]), 1);
            mbar_init(smem_u32(&sh->out_empty[i]), 8);
            mbar_init(smem_u32(&sh->d3_full[i]), 1);
            mbar_init(smem_u32(&sh->d3_empty[i]), 8);
        }
        sh->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 16) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem;
    // columns: D3 0, 128; D1 256, 320; D2 384, 448
    bool ok = true;
    if (warp < 8) {
        // ------------------------------------------------------------------------------------------ tokens in, scores, values
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(DECAY_REGS_FRONT));
        const int g = lane >> 2, tc = lane & 3;
        const T* kp = (const T*)p.k.data + h / p.group * p.k.head_stride;
        const T* qp = (const T*)p.q.data + h / p.group * p.q.head_stride;
        const T* vp = (const T*)p.v.data + h * p.v.head_stride + dv0;
        auto bring = [&](const T* from, int64_t stride, int tok, int live, uint32_t to, int dim, int have) {
            const int per = dim / 8;
            for (int i = t; i < L * per; i += 256) {
                const int r = i / per, c = i - r * per;
                const bool there = r < live && 8 * c < have;
                const T* at = there ? from + (int64_t)(tok + r) * stride + 8 * c : from;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + (c >> 3) * S::HALF + swizzled(r, c & 7)), "l"(at), "r"(there ? 16u : 0u) : "memory");
            }
        };
        auto bring_chunk = [&](int chunk) {
            const uint32_t to = at0 + (chunk & 1) * S::STAGE;
            const int tok = first + chunk * L, live = min(L, n - chunk * L);
            if (OUT) bring(qp, p.q.token_stride, tok, live, to, DK, DK);
            bring(kp, p.k.token_stride, tok, live, to + S::QK, DK, DK);
            bring(vp, p.v.token_stride, tok, live, to + 2 * S::QK, DECAY_TILE_DV, dvs);
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        auto front_sync = [] { asm volatile("bar.sync 1, 256;" ::: "memory"); };
        // the rows of a chunk come to L2 ahead of their turn, a line of 128 bytes to a thread
        auto prefetch = [&](const T* from, int64_t stride, int tok, int live, int have) {
            const int per = (have + 63) / 64;
            for (int i = t; i < live * per; i += 256) {
                const int r = i / per, c = i - r * per;
                asm volatile("prefetch.global.L2 [%0];" ::"l"(from + (int64_t)(tok + r) * stride + 64 * c));
            }
        };
        bring_chunk(0);
        for (int chunk = 0; chunk < chunks; ++chunk) {
            const int ring = chunk % DECAY_TILE_RING, two = chunk & 1;
            const uint8_t* st = base + two * S::STAGE;
            const uint32_t sq_ = smem_u32(st), sk = sq_ + S::QK;
            const float2* gs = sh->g[two];
            if (chunk + 2 < chunks) {
                const int tok = first + (chunk + 2) * L, live = min(L, n - (chunk + 2) * L);
                if (OUT) prefetch(qp, p.q.token_stride, tok, live, DK);
                prefetch(kp, p.k.token_stride, tok, live, DK);
                prefetch(vp, p.v.token_stride, tok, live, dvs);
            }
            if (t == 0) sh->odd[ring] = 0;
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            front_sync();
            // whether all keys and values are finite
            uint32_t most = 0;
            auto look = [&](const uint8_t* at, int bytes) {
                for (int i = t; i < bytes / 16; i += 256) {
                    const uint4 w = *reinterpret_cast<const uint4*>(at + i * 16);
                    most = __vmaxu2(most, __vmaxu2(__vmaxu2(w.x & 0x7FFF7FFFu, w.y & 0x7FFF7FFFu), __vmaxu2(w.z & 0x7FFF7FFFu, w.w & 0x7FFF7FFFu)));
                }
            };
            look(st + S::QK, S::QK + S::V);
            if ((most & 0xFFFFu) >= 0x7F80u || (most >> 16) >= 0x7F80u) sh->odd[ring] = 1;
            // values with their decay to the chunk's end, as parts
            ok = decay_wait(&sh->g_full[two], chunk >> 1 & 1, sh, p) && ok;
            if (chunk) ok = decay_wait(&sh->v_used, (chunk - 1) & 1, sh, p) && ok;
#pragma unroll
            for (int i = 0; i < L * 16 / 256; ++i) {
                const int at = t + 256 * i, r = at >> 4, c = at & 15;
                const uint32_t pos = (c >> 3) * S::HALF + swizzled(r, c & 7);
                const uint4 w = *reinterpret_cast<const uint4*>(st + 2 * S::QK + pos);
                const float e = sh->end[two][r];
                const uint32_t raw[4] = {w.x, w.y, w.z, w.w};
                uint32_t part[4][3];
#pragma unroll
                for (int j = 0; j < 4; ++j) split_pair<3>(__uint_as_float(raw[j] << 16) * e, __uint_as_float(raw[j] & 0xFFFF0000u) * e, part[j]);
#pragma unroll
                for (int z = 0; z < 3; ++z)
                    *reinterpret_cast<uint4*>(base + S::VD_AT + z * S::V + pos) = make_uint4(part[0][z], part[1][z], part[2][z], part[3][z]);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->v_ready));
            if constexpr (OUT) {
                // scores of 16 tokens i with 32 tokens j, times their decay, as parts
                const int i0 = 16 * (warp & 3), j0 = 32 * (warp >> 2);
                float sc[4][4];
#pragma unroll
                for (int j = 0; j < 16; ++j) sc[j >> 2][j & 3] = 0.f;
                if (j0 <= i0 + 15) {
#pragma unroll
                    for (int kt = 0; kt < DK / 16; ++kt) {
                        uint32_t af[4];
                        ldsm(sq_ + (kt >> 2) * S::HALF + swizzled(i0 + (lane & 15), 2 * (kt & 3) + (lane >> 4)), af);
#pragma unroll
                        for (int j = 0; j < 4; j += 2) {
                            if (j0 + 8 * j > i0 + 15) continue;
                            uint32_t bf[4];
                            ldsm(sk + (kt >> 2) * S::HALF + swizzled(j0 + 8 * j + (lane & 7) + (lane >> 4) * 8, 2 * (kt & 3) + (lane >> 3 & 1)), bf);
                            mma_bf16(sc[j], af, bf[0], bf[1]);
                            mma_bf16(sc[j + 1], af, bf[2], bf[3]);
                        }
                    }
                }
                uint32_t pa[4][2], pb[4][2];
                const float2 ga = gs[i0 + g], gb = gs[i0 + g + 8];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = j0 + 8 * j + 2 * tc;
                    const float4 gj = *reinterpret_cast<const float4*>(&gs[c]);
                    const auto weigh = [&](float s, const float2& gi, float hi, float lo, bool seen) {
                        const float w = seen ? __expf((gi.x - hi) + (gi.y - lo)) : 0.f;
                        return w == 0.f ? 0.f : s * w;
                    };
                    split_pair<2>(weigh(sc[j][0], ga, gj.x, gj.y, c <= i0 + g), weigh(sc[j][1], ga, gj.z, gj.w, c + 1 <= i0 + g), pa[j]);
                    split_pair<2>(weigh(sc[j][2], gb, gj.x, gj.y, c <= i0 + g + 8), weigh(sc[j][3], gb, gj.z, gj.w, c + 1 <= i0 + g + 8), pb[j]);
                }
                if (chunk) ok = decay_wait(&sh->used, (chunk - 1) & 1, sh, p) && ok;       // (the products of the chunk before are done)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = j0 + 8 * j + 2 * tc;
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        *reinterpret_cast<uint32_t*>(base + S::P_AT + z * S::HALF + swizzled(i0 + g, c >> 3) + (c & 7) * 2) = pa[j][z];
                        *reinterpret_cast<uint32_t*>(base + S::P_AT + z * S::HALF + swizzled(i0 + g + 8, c >> 3) + (c & 7) * 2) = pb[j][z];
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->ready));
            }
            if (lane == 0) mbar_arrive(smem_u32(&sh->g_empty[two]));
            if (chunk + 1 < chunks) bring_chunk(chunk + 1);      // (into the place of the chunk before, whose products are done)
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp < 16) {
        // ------------------------------------------------------------------------------------------ the state, outputs
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(DECAY_REGS_STATE));
        const int q = warp & 3, half = (warp - 8) >> 2, dv = 32 * q + lane;
        const uint32_t lanes = tmem + ((uint32_t)q << 21);
        const bool mine = dv < dvs;
        float st[KH];                                          // S^T[dv, half * KH ..]
        auto state_at = [&](auto* from, int j) { return from + (int64_t)(half * KH + j) * p.m.value_dim + dv0 + dv; };
#pragma unroll
        for (int j = 0; j < KH; ++j) st[j] = MODE != DECAY_STATES && work.from && mine ? *state_at(work.from, j) : 0.f;
        auto put_state = [&]() {                              // its parts, for the next chunk's products
#pragma unroll
            for (int j = 0; j < KH; j += 8) {
                uint32_t w[4][2];
#pragma unroll
                for (int i = 0; i < 4; ++i) split_pair<2>(st[j + 2 * i], st[j + 2 * i + 1], w[i]);
                const int key = half * KH + j;
#pragma unroll
                for (int z = 0; z < 2; ++z)
                    *reinterpret_cast<uint4*>(base + S::S_AT + z * S::S_PART + (key >> 6) * S::S_HALF + swizzled(dv, (key & 63) >> 3)) =
                        make_uint4(w[0][z], w[1][z], w[2][z], w[3][z]);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->s_full));
        };
        if (OUT) put_state();
        T* op = (T*)p.o.data + h * p.o.head_stride + dv0;
        int turn = 0, met = 0;                                 // chunks that went through the tensor cores, tokens that did not
        for (int chunk = 0; ok && chunk < chunks; ++chunk) {
            const int tok0 = first + chunk * L, live = min(L, n - chunk * L), ring = chunk % DECAY_TILE_RING;
            // (the issuer tells of a chunk; it is never four ahead, while the front may be more than a phase of its barriers ahead of this)
            if (!(ok = decay_wait(&sh->told[chunk & 3], chunk >> 2 & 1, sh, p))) break;
            const bool last_one = chunk + 1 == chunks;
            if (sh->odd[ring] || sh->last[ring] < 0.f) {
                // token by token; the two halves' parts of q S meet in shared memory (the place of P)
                const uint8_t* tok = base + (chunk & 1) * S::STAGE;
                float* meet = reinterpret_cast<float*>(base + S::P_AT);
                auto value = [&](uint32_t at, int r, int c) {
                    return __bfloat162float(*reinterpret_cast<const T*>(tok + at + (c >> 6) * S::HALF + swizzled(r, (c & 63) >> 3) + (c & 7) * 2));
                };
#pragma unroll 1
                for (int i = 0; i < live; ++i) {
                    const float f = expf(__ldg(p.decay + (int64_t)(tok0 + i) * p.d_token + h * p.d_head)), v = value(2 * S::QK, i, dv);
                    float y = 0.f;
#pragma unroll
                    for (int j = 0; j < KH; ++j) {
                        st[j] = fade_add(st[j], f, value(S::QK, i, half * KH + j) * v);
                        if (OUT) y = fmaf(value(0, i, half * KH + j), st[j], y);
                    }
                    if constexpr (OUT) {
                        if (half) {
                            if (met) ok = decay_wait(&sh->meet_empty, (met - 1) & 1, sh, p) && ok;
                            meet[dv] = y;
                        } else {
                            ok = decay_wait(&sh->meet_full, met & 1, sh, p) && ok;
                            if (mine && ok) store1(op + (int64_t)(tok0 + i) * p.o.token_stride + dv, p.scale * (y + meet[dv]));
                        }
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(half ? &sh->meet_full : &sh->meet_empty));
                        ++met;
                    }
                }
                if (OUT && !last_one) put_state();
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // (P's place is the products' again)
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->odd_done));
                continue;
            }
            const int buf = turn & 1;
            const uint32_t ph = turn >> 1 & 1;
            ++turn;
            if (OUT && !(ok = decay_wait(&sh->out_full[buf], ph, sh, p))) break;
            if (work.last || !last_one) {
                if (!(ok = decay_wait(&sh->d3_full[buf], ph, sh, p))) break;
                tc_fence_after();
                const float f = sh->last[ring];
#pragma unroll
                for (int j = 0; j < KH; j += 16) {
                    uint32_t v[32];
                    tc_ld16(lanes + buf * 128 + half * KH + j, v);
                    tc_wait_ld();
                    if (f != 0.f) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) st[j + i] = fmaf(st[j + i], f, __uint_as_float(v[i]));
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) st[j + i] = __uint_as_float(v[i]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->d3_empty[buf]));
                if (OUT && !last_one) put_state();
            }
            if constexpr (OUT) {
                tc_fence_after();
                T* at = op + (int64_t)(tok0 + 32 * half) * p.o.token_stride + dv;
#pragma unroll
                for (int j = 0; j < 32; j += 16) {
                    uint32_t x[32], y[32];
                    tc_ld16(lanes + 256 + buf * 64 + 32 * half + j, x);
                    tc_ld16(lanes + 384 + buf * 64 + 32 * half + j, y);
                    tc_wait_ld();
                    if (j == 16) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&sh->out_empty[buf]));
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float o = p.scale * fade_add(__uint_as_float(x[i]), sh->begin[ring][32 * half + j + i], __uint_as_float(y[i]));
                        if (mine && 32 * half + j + i < live) store1(at, o);
                        at += p.o.token_stride;
                    }
                }
            }
        }
        if (ok && mine && work.to) {
#pragma unroll
            for (int j = 0; j < KH; ++j) *state_at(work.to, j) = st[j];
        }
    } else {
        // ------------------------------------------------------------------------------------------ MMAs
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(DECAY_REGS_REST));
        if (warp == 17) {
            // log decays of tokens 2 lane, 2 lane + 1 of a chunk and their sums, up to two chunks ahead
            double total = 0.0;
            bool gone = false;
            float next[2];
            auto fetch = [&](int chunk) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int r = chunk * L + 2 * lane + i;
                    next[i] = r < n ? __ldg(p.decay + (int64_t)(first + r) * p.d_token + h * p.d_head) : 0.f;
                }
            };
            fetch(0);
            for (int chunk = 0; ok && chunk < chunks; ++chunk) {
                const int two = chunk & 1, ring = chunk % DECAY_TILE_RING;
                double x[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) x[i] = next[i] < DECAY_GONE ? (double)DECAY_FORGET : (double)next[i];
                const bool steep = decay_steep(decay_rise(next[0]) + decay_rise(next[1]));
                gone = __any_sync(0xffffffffu, next[0] < DECAY_GONE || next[1] < DECAY_GONE) || gone;
                if (chunk + 1 < chunks) fetch(chunk + 1);
                double s = x[0] + x[1];
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double y = __shfl_up_sync(0xffffffffu, s, o);
                    if (lane >= o) s += y;
                }
                const double end = __shfl_sync(0xffffffffu, s, 31);
                if (!(ok = decay_wait(&sh->g_empty[two], (chunk >> 1 & 1) ^ 1u, sh, p))) break;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const double at = i ? s : s - x[1];
                    const float hi = (float)at;
                    sh->g[two][2 * lane + i] = make_float2(hi, (float)(at - hi));
                    sh->begin[ring][2 * lane + i] = expf((float)at);
                    sh->end[two][2 * lane + i] = expf((float)(end - at));
                }
                if (lane == 31) sh->last[ring] = steep ? -1.f : expf((float)end);
                total += end;
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->g_full[two]));
            }
            if (MODE == DECAY_STATES && ok && lane == 0 && slice == 0) p.fade[(int64_t)blockIdx.x * p.m.heads + h] = gone ? -INFINITY : (float)total;
        }
        // D = F32, A = B = BF16, M = 128; bits 15, 16: A, B lie with their rows, not K, side by side (tokens are K in D3 and for the values)
        constexpr uint32_t I = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);
        constexpr uint32_t I_D3 = I | (1u << 15) | (1u << 16) | ((uint32_t)(DK >> 3) << 17), I_D1 = I | ((64u >> 3) << 17), I_D2 = I | (1u << 15) | ((64u >> 3) << 17);
        const auto k_major = [&](uint32_t at) { return (((at0 + at) & 0x3FFFFu) >> 4) | (1u << 16); };
        const auto mn_major = [&](uint32_t at) { return (((at0 + at) & 0x3FFFFu) >> 4) | ((S::HALF >> 4) << 16); };
        int turn = 0, s_turn = 0, odd_turn = 0;
        for (int chunk = 0; warp == 16 && ok && chunk < chunks; ++chunk) {
            if (!(ok = decay_wait(&sh->v_ready, chunk & 1, sh, p))) break;
            const bool odd = sh->odd[chunk % DECAY_TILE_RING] || sh->last[chunk % DECAY_TILE_RING] < 0.f;
            if (odd && OUT) {
                // P and the state have been written, and go unused: before the state's warps hear of the chunk and go on
                if (!(ok = decay_wait(&sh->ready, chunk & 1, sh, p))) break;
                if (!(ok = decay_wait(&sh->s_full, s_turn & 1, sh, p))) break;
                ++s_turn;
            }
            if (lane == 0) mbar_arrive(smem_u32(&sh->told[chunk & 3]));
            __syncwarp();
            if (odd) {                                          // token by token
                if (!(ok = decay_wait(&sh->odd_done, odd_turn & 1, sh, p))) break;
                ++odd_turn;
                if (lane == 0) {
                    mbar_arrive(smem_u32(&sh->v_used));
                    if (OUT) mbar_arrive(smem_u32(&sh->used));
                }
                __syncwarp();
                continue;
            }
            const int buf = turn & 1;
            const uint32_t ph = (turn >> 1 & 1) ^ 1u, st = (chunk & 1) * S::STAGE;
            ++turn;
            if (work.last || chunk + 1 < chunks) {
                if (!(ok = decay_wait(&sh->d3_empty[buf], ph, sh, p))) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t a0 = mn_major(S::VD_AT), b0 = mn_major(st + S::QK);
#pragma unroll
                    for (int z = 2; z >= 0; --z)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            decay_mma(tmem + buf * 128, a0 + z * (S::V >> 4) + k * (2048 >> 4), b0 + k * (2048 >> 4), I_D3, z < 2 || k > 0);
                    tc_commit(smem_u32(&sh->d3_full[buf]));
                    tc_commit(smem_u32(&sh->v_used));
                }
                __syncwarp();
            }
            if constexpr (OUT) {
                if (!(ok = decay_wait(&sh->ready, chunk & 1, sh, p))) break;
                if (!(ok = decay_wait(&sh->out_empty[buf], ph, sh, p))) break;
                if (!(ok = decay_wait(&sh->s_full, s_turn & 1, sh, p))) break;
                ++s_turn;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t a1 = k_major(S::S_AT), b1 = k_major(st), a2 = mn_major(st + 2 * S::QK), b2 = k_major(S::P_AT);
#pragma unroll
                    for (int z = 1; z >= 0; --z)
#pragma unroll
                        for (int k = 0; k < DK / 16; ++k)
                            decay_mma(tmem + 256 + buf * 64, a1 + z * (S::S_PART >> 4) + (k >> 2) * (S::S_HALF >> 4) + 2 * (k & 3),
                                      b1 + (k >> 2) * (S::HALF >> 4) + 2 * (k & 3), I_D1, z < 1 || k > 0);
#pragma unroll
                    for (int z = 1; z >= 0; --z)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            decay_mma(tmem + 384 + buf * 64, a2 + k * (2048 >> 4), b2 + z * (S::HALF >> 4) + 2 * k, I_D2, z < 1 || k > 0);
                    tc_commit(smem_u32(&sh->out_full[buf]));
                    tc_commit(smem_u32(&sh->used));
                }
                __syncwarp();
            }
        }
    }
    if (!ok) {                                                  // loads and MMAs still in flight
        const long long since = clock64();
        while (clock64() - since < 400000) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 16) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

}  // namespace ccv3d
