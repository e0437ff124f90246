// Attention with decaying states: S_t = exp(g_t) S_{t-1} + k_t v_t^T, out_t = scale q_t S_t.
//
// Single tokens (decay_step_kernel): bound by the states' bytes.  A block holds a slice of 64 value columns of one state in registers from
// its one load to its one store.
// Measured: 64 streams of one token, 32 heads of 128 x 128, 49 us = 5.5 TB/s, 84 % of the copy rate.
// Many tokens (decay_tile_kernel for BF16; F32: decay_chunk_kernel): in chunks of 64, with G the sum of the log decays from the chunk's start on,
//   out_i = scale (exp(G_i) q_i S + sum_{j <= i} exp(G_i - G_j) (q_i . k_j) v_j)        S' = exp(G_end) S + sum_j exp(G_end - G_j) k_j v_j^T
// decay_chunk_kernel does so as mma.sync products of BF16 with FP32 sums.  A warp owns 16 value columns of S^T, in registers as the products leave them, which is also
// the layout that the next product wants them in as its B operand: the state never leaves the registers.  What is not BF16 already goes in
// as three BF16 numbers, 8 bits each, of whose nine products six are taken (BF16 inputs: scores with their decay and S as two, v with its
// decay as three).  F32, 24 prompts of up to 700 tokens, 14 heads of 64 x 128: 330 us, bound by the latency of eight warps' products.
// G is summed in 64 bits and kept as two floats, so that differences of sums that a strong decay made large still have all their bits.
//
// Where sequences and heads are too few for the machine, sequences of more than a segment are cut: their segments' contributions to the state side by
// side, then a scan over the segments (decay_scan_kernel), then the outputs.  Other sequences of such a call go beside the outputs in one piece.
//
// A chunk in which a key or value is not finite goes token by token (0 times infinity must not reach a token that does not see it), and so does one
// with a log decay of NaN, or whose positive log decays come to more than 16: products of sums would overflow, a state of zeros times infinity, where
// the recurrence does not.
#pragma once
#include "ccv3d_tokens_common.cuh"

namespace ccv3d {

constexpr int DECAY_CHUNK = 64;
constexpr int DECAY_STEP_THREADS = 256;
constexpr float DECAY_GONE = -104.f, DECAY_FORGET = -1e4f;      // exp of what lies below the first is zero: it goes into sums as the second
constexpr float DECAY_RISE = 16.f;

struct DecayParams {
    ccv3d_decay_memory m;
    ccv3d_stream_batch bt;
    ccv3d_heads q, k, v, o;
    const float* decay;
    int64_t d_token, d_head;
    int group;                   // heads that share a q and k
    float scale;
    uint32_t* status;
    int seg;                     // tokens of a segment (0: sequences are not cut)
    float* part;                 // [item][head][key][value]: contributions of cut sequences' segments, then the states they start from
    float* fade;                 // [item][head]: log decay over a whole segment
    int items;                   // room in them; the blocks behind them have the sequences that are not cut
    long long wait_clk;
};

struct DecaySeq { int first, n, slot; bool zero; };     // slot < 0: the state is not kept

__device__ __forceinline__ void decay_span(const ccv3d_stream_batch& bt, int b, int& first, int& n, bool& bad) {
    int s = __ldg(bt.new_start + b), e = __ldg(bt.new_start + b + 1);
    bad = s < 0 || e < s || e > bt.tokens || e - s > bt.max_new;
    if (bad) {
        s = min(max(s, 0), bt.tokens);
        e = min(max(e, s), s + min(bt.tokens - s, bt.max_new));
    }
    first = s;
    n = e - s;
}
// All threads of the block.  A sequence of more than `most` tokens (0: any number) is another block's: without tokens here.
__device__ __forceinline__ DecaySeq decay_seq(const DecayParams& p, int b, bool tell, int most = 0) {
    DecaySeq s;
    bool bad;
    decay_span(p.bt, b, s.first, s.n, bad);
    if (most && s.n > most) return {s.first, 0, -1, true};
    s.slot = __ldg(p.bt.slot + b);
    uint32_t word = bad ? CCV3D_TOKENS_BAD_LENGTH : 0u;
    int taken = 0;
    if ((unsigned)s.slot >= (unsigned)p.m.slots) {
        s.slot = -1;
        if (s.n) word |= CCV3D_TOKENS_BAD_SLOT;
    } else if (s.n) {
        for (int j = threadIdx.x; j < b && !taken; j += blockDim.x)
            if (__ldg(p.bt.slot + j) == s.slot) {
                int f, n;
                decay_span(p.bt, j, f, n, bad);
                taken = n > 0;
            }
    }
    if (__syncthreads_or(taken)) {
        s.slot = -1;
        word |= CCV3D_TOKENS_BAD_SLOT;
    }
    s.zero = s.slot < 0 || (p.bt.fresh && __ldg(p.bt.fresh + b) != 0);
    if (word && tell && threadIdx.x == 0) report(p.status, word);
    return s;
}

// exp(g) S: what is forgotten wholly is zero whatever it was
__device__ __forceinline__ float fade(float s, float f) { return f == 0.f ? 0.f : s * f; }
__device__ __forceinline__ float fade_add(float s, float f, float x) { return f == 0.f ? x : fmaf(s, f, x); }
// exp(t) s + x, where exp(t) may lie beyond FP32 and the product within
__device__ __forceinline__ float grow_add(float s, float t, float x) {
    if (t <= 64.f) return fade_add(s, expf(t), x);
    const float f = expf(0.25f * t);
    return s == 0.f ? x : fmaf(s * f * f * f, f, x);
}

// What a log decay adds to a chunk's rise (NaN stays), and whether all of them (two to a lane) leave the chunk to products.
__device__ __forceinline__ float decay_rise(float g) { return g <= 0.f ? 0.f : g; }
__device__ __forceinline__ bool decay_steep(float rise) {
    if (!__any_sync(0xffffffffu, !(rise <= 0.f))) return false;
    return !(warp_sum(rise) <= DECAY_RISE);
}

// ---------------------------------------------------------------------------------------------------- single tokens
// Block (sequence, head, 64 value columns): thread t has columns 4 (t % 16) .. + 3 of rows R (t / 16) + i, whose keys and queries it reads four at
// a time (one by one, the way to shared memory bounds prompts).  Up to eight tokens are brought in at a time, and their outputs' parts summed together.
constexpr int DECAY_STEP_TOKENS = 8;
template <typename T, int DK>
__global__ void __launch_bounds__(DECAY_STEP_THREADS) decay_step_kernel(const __grid_constant__ DecayParams p) {
    constexpr int R = DK / 16, M = DECAY_STEP_TOKENS;
    __shared__ __align__(16) float ks[M][DK], qs[M][DK], vs[M][64], fs[M];
    __shared__ __align__(16) float part[M][8][64];
    const int slices = p.m.value_dim / 64, t = threadIdx.x, team = t >> 4, row0 = team * R, c4 = (t & 15) * 4;
    const int slice = blockIdx.x % slices, h = blockIdx.x / slices % p.m.heads, b = blockIdx.x / slices / p.m.heads;
    const DecaySeq s = decay_seq(p, b, slice == 0 && h == 0);
    if (s.n == 0) return;
    float* state = p.m.states + ((int64_t)max(s.slot, 0) * p.m.heads + h) * DK * p.m.value_dim + slice * 64 + c4;
    float4 S[R];
#pragma unroll
    for (int i = 0; i < R; ++i) S[i] = s.zero ? make_float4(0.f, 0.f, 0.f, 0.f) : *reinterpret_cast<const float4*>(state + (int64_t)(row0 + i) * p.m.value_dim);
    const T* k = (const T*)p.k.data + h / p.group * p.k.head_stride;
    const T* q = (const T*)p.q.data + h / p.group * p.q.head_stride;
    const T* v = (const T*)p.v.data + h * p.v.head_stride + slice * 64;
    T* o = (T*)p.o.data + h * p.o.head_stride + slice * 64;
    for (int base = 0; base < s.n; base += M) {
        const int m = min(M, s.n - base);
        const int64_t tok = s.first + base;
        for (int i = t; i < m * (DK / 4); i += DECAY_STEP_THREADS) {
            const int r = i / (DK / 4), c = i % (DK / 4) * 4;
            float x[4];
            load4(k + (tok + r) * p.k.token_stride + c, x);
            store4(&ks[r][c], x);
            load4(q + (tok + r) * p.q.token_stride + c, x);
            store4(&qs[r][c], x);
        }
        if (team < m) {
            float x[4];
            load4(v + (tok + team) * p.v.token_stride + c4, x);
            store4(&vs[team][c4], x);
        }
        if (t < m) fs[t] = expf(__ldg(p.decay + (tok + t) * p.d_token + h * p.d_head));
        __syncthreads();
        for (int i = 0; i < m; ++i) {
            const float4 x = *reinterpret_cast<const float4*>(&vs[i][c4]);
            const float f = fs[i];
            float y[4] = {0.f, 0.f, 0.f, 0.f};
            if (f == 0.f) {                                      // all before is forgotten, whatever it was
#pragma unroll
                for (int r = 0; r < R; ++r) S[r] = make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int r4 = 0; r4 < R; r4 += 4) {
                float kk[4], qq[4];
                load4(&ks[i][row0 + r4], kk);
                load4(&qs[i][row0 + r4], qq);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float4& st = S[r4 + j];
                    st.x = fmaf(st.x, f, kk[j] * x.x);
                    st.y = fmaf(st.y, f, kk[j] * x.y);
                    st.z = fmaf(st.z, f, kk[j] * x.z);
                    st.w = fmaf(st.w, f, kk[j] * x.w);
                    y[0] = fmaf(qq[j], st.x, y[0]);
                    y[1] = fmaf(qq[j], st.y, y[1]);
                    y[2] = fmaf(qq[j], st.z, y[2]);
                    y[3] = fmaf(qq[j], st.w, y[3]);
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] += __shfl_xor_sync(0xffffffffu, y[j], 16);
            if ((t & 31) < 16) store4(&part[i][t >> 5][c4], y);
        }
        __syncthreads();
        for (int i = t; i < m * 64; i += DECAY_STEP_THREADS) {
            const int r = i >> 6, c = i & 63;
            float sum = part[r][0][c];
#pragma unroll
            for (int w = 1; w < 8; ++w) sum += part[r][w][c];
            store1(o + (tok + r) * p.o.token_stride + c, sum * p.scale);
        }
    }
    if (s.slot >= 0) {
#pragma unroll
        for (int i = 0; i < R; ++i) *reinterpret_cast<float4*>(state + (int64_t)(row0 + i) * p.m.value_dim) = S[i];
    }
}

// ------------------------------------------------------------------------------------------------------ many tokens
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void ldsm(uint32_t at, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t at, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
// Two floats as N pairs of BF16 numbers, each what the ones before leave.  (Infinities leave NaN: their products are not finite anyway.)
template <int N>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t (&out)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        out[i] = pack_bf16(x, y);
        x -= __uint_as_float(out[i] << 16);
        y -= __uint_as_float(out[i] & 0xFFFF0000u);
    }
}

// F32 prompts.  Shared memory of a block: rows of BF16 with 16 bytes between them, so that eight rows of a matrix lie in different banks.
constexpr int DECAY_PARTS = 3;             // BF16 numbers of an F32 one
template <int DK, int NW> struct DecayShape {
    static constexpr int DV = 16 * NW, THREADS = 32 * NW;
    static constexpr int QS = DK + 8, VS = DV + 8, PS = DECAY_CHUNK + 8;                     // elements of a row
    static constexpr int Q = DECAY_CHUNK * QS, V = DECAY_CHUNK * VS, P = DECAY_CHUNK * PS;   // elements of a plane
    static constexpr int BYTES = DECAY_PARTS * (2 * Q + V + P) * 2;
};

struct DecayShared {
    float2 g[DECAY_CHUNK];       // sums of log decays, as two floats
    float end[DECAY_CHUNK];      // exp(G_end - G_j)
    float begin[DECAY_CHUNK];    // exp(G_i)
    float last;                  // exp(G_end)
    int steep;
};

// Segments of a sequence of n tokens that is cut; 0: it is not.
__device__ __forceinline__ int decay_segments(const DecayParams& p, int n) { return n > p.seg ? (n - 1) / p.seg + 1 : 0; }

// Item (cut sequence, segment); false: there is none of this number.  All threads; word: 34 ints in shared memory.
__device__ __forceinline__ bool decay_item(const DecayParams& p, int item, int& b, int& seg, int* word) {
    int* scan = word + 2;
    const int t = threadIdx.x, warps = blockDim.x >> 5;
    int before = 0;
    if (t == 0) word[0] = -1;
    for (int base = 0; base < p.bt.batch; base += blockDim.x) {
        int n = 0, first;
        bool bad;
        if (base + t < p.bt.batch) {
            decay_span(p.bt, base + t, first, n, bad);
            n = decay_segments(p, n);
        }
        const int upto = warp_scan(n);
        if ((t & 31) == 31) scan[t >> 5] = upto;
        __syncthreads();
        int mine = before + upto - n, all = before;
        for (int i = 0; i < warps; ++i) {
            if (i < (t >> 5)) mine += scan[i];
            all += scan[i];
        }
        if (item >= mine && item < mine + n) { word[0] = base + t; word[1] = item - mine; }
        __syncthreads();
        before = all;
        if (item < before) break;
    }
    b = word[0];
    seg = word[1];
    __syncthreads();
    return b >= 0;
}

// Passes over the chunks of a block: outputs of a sequence and its state, or of a cut one's segment; a segment's contribution to the state.
enum { DECAY_OUTPUTS, DECAY_STATES };

// A block's tokens, and where its state comes from and goes to.  All threads; word as above.
struct DecayWork {
    int first, n;
    const float* from;           // nullptr: zeros
    float* to;                   // nullptr: it is not kept
    bool last;                   // the state is wanted behind the last chunk
};
template <int MODE>
__device__ __forceinline__ bool decay_work(const DecayParams& p, int h, int dk, DecayWork& w, int* word) {
    const int64_t size = (int64_t)dk * p.m.value_dim, block = blockIdx.x;
    if (MODE == DECAY_STATES || block < p.items) {
        int b, seg;
        bool bad;
        if (!decay_item(p, blockIdx.x, b, seg, word)) return false;
        decay_span(p.bt, b, w.first, w.n, bad);
        w.first += seg * p.seg;
        w.n = min(p.seg, w.n - seg * p.seg);
        float* part = p.part + (block * p.m.heads + h) * size;
        w.last = MODE == DECAY_STATES;
        w.from = w.last ? nullptr : part;
        w.to = w.last ? part : nullptr;
        return true;
    }
    const DecaySeq s = decay_seq(p, (int)block - p.items, blockIdx.y == 0, p.seg);
    if (s.n == 0) return false;
    float* state = s.slot < 0 ? nullptr : p.m.states + ((int64_t)s.slot * p.m.heads + h) * size;
    w = {s.first, s.n, s.zero ? nullptr : state, state, state != nullptr};
    return true;
}

template <int DK, int NW, int MODE>
__global__ void __launch_bounds__(32 * NW, NW == 4 ? 2 : 1) decay_chunk_kernel(const __grid_constant__ DecayParams p) {
    using S = DecayShape<DK, NW>;
    using T = float;
    constexpr int N = DECAY_PARTS, L = DECAY_CHUNK;
    extern __shared__ __align__(16) __nv_bfloat16 decay_smem[];
    __shared__ DecayShared sh;
    __shared__ int word[34];
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31, g = lane >> 2, tc = lane & 3;
    const int slices = p.m.value_dim / S::DV, slice = blockIdx.y % slices, h = blockIdx.y / slices;
    const int dv0 = slice * S::DV;
    DecayWork work;
    if (!decay_work<MODE>(p, h, DK, work, word)) return;
    const int first = work.first, n = work.n;
    const T* kp = (const T*)p.k.data + h / p.group * p.k.head_stride;
    const T* qp = (const T*)p.q.data + h / p.group * p.q.head_stride;
    const T* vp = (const T*)p.v.data + h * p.v.head_stride + dv0;
    T* op = (T*)p.o.data + h * p.o.head_stride + dv0;

    // S^T of this warp: rows dv = 16 warp + g (+ 8), columns dk = 8 j + 2 tc (+ 1)
    float st[DK / 8][4];
    auto state_at = [&](auto* base, int j, int i) { return base + (int64_t)(8 * j + 2 * tc + (i & 1)) * p.m.value_dim + dv0 + 16 * warp + g + (i >> 1) * 8; };
#pragma unroll
    for (int j = 0; j < DK / 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) st[j][i] = MODE != DECAY_STATES && work.from ? *state_at(work.from, j, i) : 0.f;

    uint32_t most = 0;                                 // of keys and values: whether all are finite (this thread's)
    // rows of `dim` elements of tokens tok .. of a chunk of `live` into planes at `to`; what lies behind them is zero
    auto bring = [&](const T* from, int64_t stride, int tok, int live, __nv_bfloat16* to, int pitch, int dim) {
        const int per = dim / 8;
        for (int i = t; i < L * per; i += S::THREADS) {
            const int r = i / per, c = (i - r * per) * 8;
            const T* at = from + (int64_t)(tok + r) * stride + c;
            float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
            if (r < live) { load4(at, x); load4(at + 4, y); }
            uint32_t w[4][N];
            split_pair<N>(x[0], x[1], w[0]);
            split_pair<N>(x[2], x[3], w[1]);
            split_pair<N>(y[0], y[1], w[2]);
            split_pair<N>(y[2], y[3], w[3]);
#pragma unroll
            for (int z = 0; z < N; ++z) *reinterpret_cast<uint4*>(to + z * L * pitch + r * pitch + c) = make_uint4(w[0][z], w[1][z], w[2][z], w[3][z]);
        }
    };
    __nv_bfloat16 *sq_ = decay_smem, *sk = sq_ + N * S::Q, *sv = sk + N * S::Q, *sp = sv + N * S::V;
    auto bring_chunk = [&](int chunk) {
        const int tok = first + chunk * L, live = min(L, n - chunk * L);
        if (MODE != DECAY_STATES) bring(qp, p.q.token_stride, tok, live, sq_, S::QS, DK);
        bring(kp, p.k.token_stride, tok, live, sk, S::QS, DK);
        bring(vp, p.v.token_stride, tok, live, sv, S::VS, S::DV);
    };
    // whether this thread's share of the keys and values is finite
    auto look = [&](const __nv_bfloat16* at, int pitch, int dim) {
        const int per = dim / 8;
        for (int i = t; i < L * per; i += S::THREADS) {
            const int r = i / per, c = (i - r * per) * 8;
            const uint4 w = *reinterpret_cast<const uint4*>(at + r * pitch + c);
            most = __vmaxu2(most, __vmaxu2(__vmaxu2(w.x & 0x7FFF7FFFu, w.y & 0x7FFF7FFFu), __vmaxu2(w.z & 0x7FFF7FFFu, w.w & 0x7FFF7FFFu)));
        }
    };

    const int chunks = (n + L - 1) / L;
    double total = 0.0;                                // log decay of the chunks so far, and whether it is minus infinity (warp 0)
    bool gone = false;
    bring_chunk(0);
    for (int chunk = 0; chunk < chunks; ++chunk) {
        const int tok0 = first + chunk * L, live = min(L, n - chunk * L);
        if (chunk + 1 < chunks) {                          // the next chunk's rows come to L2
            const int ahead = min(L, n - (chunk + 1) * L), kl = DK * (int)sizeof(T) / 128, vl = S::DV * (int)sizeof(T) / 128;
            for (int i = t; i < ahead * (2 * kl + vl); i += S::THREADS) {
                const int r = i / (2 * kl + vl), c = i - r * (2 * kl + vl);
                const int64_t tok = tok0 + L + r;
                const T* at = c < kl ? kp + tok * p.k.token_stride + c * (128 / sizeof(T))
                              : c < 2 * kl ? qp + tok * p.q.token_stride + (c - kl) * (128 / sizeof(T)) : vp + tok * p.v.token_stride + (c - 2 * kl) * (128 / sizeof(T));
                asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
            }
        }
        if (warp == 0) {
            // log decays of tokens 2 lane, 2 lane + 1 and their sums
            double x[2];
            float rise = 0.f;
            bool forget = false;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = 2 * lane + i;
                const float d = r < live ? __ldg(p.decay + (int64_t)(tok0 + r) * p.d_token + h * p.d_head) : 0.f;
                rise += decay_rise(d);
                forget = forget || d < DECAY_GONE;
                x[i] = d < DECAY_GONE ? (double)DECAY_FORGET : (double)d;
            }
            const bool steep = decay_steep(rise);
            gone = __any_sync(0xffffffffu, forget) || gone;
            double s = x[0] + x[1];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double y = __shfl_up_sync(0xffffffffu, s, o);
                if (lane >= o) s += y;
            }
            const double end = __shfl_sync(0xffffffffu, s, 31);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const double at = i ? s : s - x[1];
                const float hi = (float)at;
                sh.g[2 * lane + i] = make_float2(hi, (float)(at - hi));
                sh.begin[2 * lane + i] = expf((float)at);
                sh.end[2 * lane + i] = expf((float)(end - at));
            }
            if (lane == 31) { sh.last = expf((float)end); sh.steep = steep; }
            total += end;
        }
        most = 0;
        __syncthreads();
        look(sk, S::QS, DK);
        look(sv, S::VS, S::DV);
        const bool odd = __syncthreads_or((most & 0xFFFFu) >= 0x7F80u || (most >> 16) >= 0x7F80u || sh.steep);
        const float last = sh.last;
        if (odd) {
            // token by token; a lane's part of q S is summed over the four lanes of its rows
            auto value = [&](const __nv_bfloat16* at, int plane) {
                float x = 0.f;
#pragma unroll
                for (int z = N - 1; z >= 0; --z) {
                    const float y = __bfloat162float(at[z * plane]);
                    x = isnan(y) && z ? x : x + y;                   // (an infinity's remainders are NaN)
                }
                return x;
            };
#pragma unroll 1
            for (int i = 0; i < live; ++i) {
                const float f = expf(__ldg(p.decay + (int64_t)(tok0 + i) * p.d_token + h * p.d_head));
                const float v0 = value(sv + i * S::VS + 16 * warp + g, S::V), v1 = value(sv + i * S::VS + 16 * warp + g + 8, S::V);
                float y0 = 0.f, y1 = 0.f;
#pragma unroll
                for (int j = 0; j < DK / 8; ++j) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int d = 8 * j + 2 * tc + c;
                        const float kk = value(sk + i * S::QS + d, S::Q);
                        st[j][c] = fade_add(st[j][c], f, kk * v0);
                        st[j][2 + c] = fade_add(st[j][2 + c], f, kk * v1);
                        if (MODE != DECAY_STATES) {
                            const float qq = value(sq_ + i * S::QS + d, S::Q);
                            y0 = fmaf(qq, st[j][c], y0);
                            y1 = fmaf(qq, st[j][2 + c], y1);
                        }
                    }
                }
                if (MODE != DECAY_STATES) {
#pragma unroll
                    for (int o = 1; o < 4; o <<= 1) {
                        y0 += __shfl_xor_sync(0xffffffffu, y0, o);
                        y1 += __shfl_xor_sync(0xffffffffu, y1, o);
                    }
                    if (tc == 0) {
                        T* at = op + (int64_t)(tok0 + i) * p.o.token_stride + 16 * warp + g;
                        store1(at, y0 * p.scale);
                        store1(at + 8, y1 * p.scale);
                    }
                }
            }
        } else {
            if constexpr (MODE != DECAY_STATES) {
                // scores of 16 tokens i with 64 (or 32) tokens j, times their decay, as parts
                {
                    constexpr int JT = 256 / (NW * 8) >= 8 ? 8 : 4;          // 8-token tiles of a warp
                    const int i0 = 16 * (warp & 3), j0 = NW == 8 ? 32 * (warp >> 2) : 0;
                    float sc[JT][4];
#pragma unroll
                    for (int j = 0; j < JT; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) sc[j][i] = 0.f;
                    if (j0 <= i0 + 15) {
#pragma unroll
                        for (int o = N - 1; o >= 0; --o)
#pragma unroll
                            for (int a = o; a >= 0; --a)
#pragma unroll
                                for (int kt = 0; kt < DK / 16; ++kt) {
                                    uint32_t af[4];
                                    ldsm(smem_at(sq_ + a * S::Q + (i0 + (lane & 15)) * S::QS + 16 * kt + (lane >> 4) * 8), af);
#pragma unroll
                                    for (int j = 0; j < JT; j += 2) {
                                        if (j0 + 8 * j > i0 + 15) continue;
                                        uint32_t bf[4];
                                        ldsm(smem_at(sk + (o - a) * S::Q + (j0 + 8 * j + (lane & 7) + (lane >> 4) * 8) * S::QS + 16 * kt + (lane >> 3 & 1) * 8), bf);
                                        mma_bf16(sc[j], af, bf[0], bf[1]);
                                        mma_bf16(sc[j + 1], af, bf[2], bf[3]);
                                    }
                                }
                    }
                    const float2 ga = sh.g[i0 + g], gb = sh.g[i0 + g + 8];
#pragma unroll
                    for (int j = 0; j < JT; ++j) {
                        const int c = j0 + 8 * j + 2 * tc;
                        const float2 g0 = sh.g[c], g1 = sh.g[c + 1];
                        float x[4];
                        const auto weigh = [&](float s, const float2& gi, const float2& gj, bool seen) {
                            const float w = seen ? expf((gi.x - gj.x) + (gi.y - gj.y)) : 0.f;
                            return w == 0.f ? 0.f : s * w;
                        };
                        x[0] = weigh(sc[j][0], ga, g0, c <= i0 + g);
                        x[1] = weigh(sc[j][1], ga, g1, c + 1 <= i0 + g);
                        x[2] = weigh(sc[j][2], gb, g0, c <= i0 + g + 8);
                        x[3] = weigh(sc[j][3], gb, g1, c + 1 <= i0 + g + 8);
                        uint32_t a[N], b[N];
                        split_pair<N>(x[0], x[1], a);
                        split_pair<N>(x[2], x[3], b);
#pragma unroll
                        for (int z = 0; z < N; ++z) {
                            *reinterpret_cast<uint32_t*>(sp + z * S::P + (i0 + g) * S::PS + c) = a[z];
                            *reinterpret_cast<uint32_t*>(sp + z * S::P + (i0 + g + 8) * S::PS + c) = b[z];
                        }
                    }
                }
                // q S, for all 64 tokens and the warp's 16 columns
                float out[4][2][4];
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int i = 0; i < 8; ++i) out[m][i >> 2][i & 3] = 0.f;
                // (the remainders' products of all keys first, so that the whole sums are only added to, and cut, eight times)
#pragma unroll
                for (int pass = 0; pass < 2; ++pass)
#pragma unroll
                    for (int kt = 0; kt < DK / 16; ++kt) {
                        uint32_t b[2][2][N];                // [columns g, g + 8][k halves][part]
#pragma unroll
                        for (int c = 0; c < 2; ++c)
#pragma unroll
                            for (int k = 0; k < 2; ++k) split_pair<N>(st[2 * kt + k][2 * c], st[2 * kt + k][2 * c + 1], b[c][k]);
#pragma unroll
                        for (int m = 0; m < 4; ++m) {
                            if (16 * m >= live) break;
#pragma unroll
                            for (int a = N - 1; a >= 0; --a) {
                                if (pass == 1 && a > 0) continue;
                                uint32_t af[4];
                                ldsm(smem_at(sq_ + a * S::Q + (16 * m + (lane & 15)) * S::QS + 16 * kt + (lane >> 4) * 8), af);
#pragma unroll
                                for (int z = N - 1; z >= 0; --z) {
                                    if (a + z >= N || (pass == 1) != (a + z == 0)) continue;
                                    mma_bf16(out[m][0], af, b[0][0][z], b[0][1][z]);
                                    mma_bf16(out[m][1], af, b[1][0][z], b[1][1][z]);
                                }
                            }
                        }
                    }
                __syncthreads();                             // all scores are there
                // ... faded; the scores' part is summed for itself
                float pv[4][2][4];
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const float e0 = sh.begin[16 * m + g], e1 = sh.begin[16 * m + g + 8];
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            out[m][c][i] = fade(out[m][c][i], i < 2 ? e0 : e1);
                            pv[m][c][i] = 0.f;
                        }
                }
#pragma unroll
                for (int o = N - 1; o >= 0; --o)            // part a of the scores, o - a of the values
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int a = o; a >= 0; --a) {
                            uint32_t bf[4];
                            ldsm_t(smem_at(sv + (o - a) * S::V + (16 * kt + (lane & 15)) * S::VS + 16 * warp + (lane >> 4) * 8), bf);
#pragma unroll
                            for (int m = kt; m < 4; ++m) {
                                if (16 * m >= live) break;
                                uint32_t af[4];
                                ldsm(smem_at(sp + a * S::P + (16 * m + (lane & 15)) * S::PS + 16 * kt + (lane >> 4) * 8), af);
#pragma unroll
                                for (int c = 0; c < 2; ++c) mma_bf16(pv[m][c], af, bf[2 * c], bf[2 * c + 1]);
                            }
                        }
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int r = 16 * m + g + 8 * half;
                        if (r >= live) continue;
                        T* at = op + (int64_t)(tok0 + r) * p.o.token_stride + 16 * warp + 2 * tc;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const float x = out[m][c][2 * half] + pv[m][c][2 * half], y = out[m][c][2 * half + 1] + pv[m][c][2 * half + 1];
                            *reinterpret_cast<float2*>(at + 8 * c) = make_float2(p.scale * x, p.scale * y);
                        }
                    }
            }
            if (work.last || chunk + 1 < chunks) {
                // the state: v with its decay to the chunk's end, as parts, times k
                uint32_t va[L / 16][N][4];
#pragma unroll
                for (int kt = 0; kt < L / 16; ++kt) {
                    uint32_t raw[N][4];
#pragma unroll
                    for (int z = 0; z < N; ++z)
                        ldsm_t(smem_at(sv + z * S::V + (16 * kt + (lane & 7) + (lane >> 4) * 8) * S::VS + 16 * warp + (lane >> 3 & 1) * 8), raw[z]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float x = 0.f, y = 0.f;
#pragma unroll
                        for (int z = N - 1; z >= 0; --z) {
                            x += __uint_as_float(raw[z][i] << 16);
                            y += __uint_as_float(raw[z][i] & 0xFFFF0000u);
                        }
                        const float2 e = *reinterpret_cast<const float2*>(&sh.end[16 * kt + 2 * tc + (i >> 1) * 8]);
                        uint32_t w[N];
                        split_pair<N>(x * e.x, y * e.y, w);
#pragma unroll
                        for (int z = 0; z < N; ++z) va[kt][z][i] = w[z];
                    }
                }
                constexpr int JN = 2;                        // tiles of 8 keys' channels at a time
#pragma unroll
                for (int j = 0; j < DK / 8; j += JN) {
                    float d[JN][4];
#pragma unroll
                    for (int i = 0; i < 4 * JN; ++i) d[i >> 2][i & 3] = 0.f;
#pragma unroll
                    for (int a = N - 1; a >= 0; --a) {      // part a of k; the small products first
                        uint32_t bf[L / 16][JN / 2][4];
#pragma unroll
                        for (int kt = 0; kt < L / 16; ++kt)
#pragma unroll
                            for (int c = 0; c < JN / 2; ++c)
                                ldsm_t(smem_at(sk + a * S::Q + (16 * kt + (lane & 15)) * S::QS + 8 * j + 16 * c + (lane >> 4) * 8), bf[kt][c]);
#pragma unroll
                        for (int z = N - 1 - a; z >= 0; --z)
#pragma unroll
                            for (int kt = 0; kt < L / 16; ++kt)
#pragma unroll
                                for (int c = 0; c < JN; ++c) mma_bf16(d[c], va[kt][z], bf[kt][c >> 1][2 * (c & 1)], bf[kt][c >> 1][2 * (c & 1) + 1]);
                    }
#pragma unroll
                    for (int c = 0; c < JN; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) st[j + c][i] = fade_add(st[j + c][i], last, d[c][i]);
                }
            }
        }
        __syncthreads();                                     // this chunk's rows and scores have been used
        if (chunk + 1 < chunks) bring_chunk(chunk + 1);
    }
    if (work.to) {
#pragma unroll
        for (int j = 0; j < DK / 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) *state_at(work.to, j, i) = st[j][i];
        if (MODE == DECAY_STATES && t == 0 && slice == 0) p.fade[(int64_t)blockIdx.x * p.m.heads + h] = gone ? -INFINITY : (float)total;
    }
}

// States that the segments of a sequence start from, in place of their contributions, and the sequence's last state.
// Block (sequence, head, 1024 elements), a thread to four.
constexpr int DECAY_SCAN_THREADS = 256, DECAY_SCAN_AHEAD = 4;
__global__ void __launch_bounds__(DECAY_SCAN_THREADS) decay_scan_kernel(const __grid_constant__ DecayParams p) {
    const int64_t size = (int64_t)p.m.key_dim * p.m.value_dim, per = p.m.heads * size;
    const int b = blockIdx.x, h = blockIdx.z;
    int first, n;
    bool bad;
    decay_span(p.bt, b, first, n, bad);
    if (!decay_segments(p, n)) return;
    const DecaySeq s = decay_seq(p, b, blockIdx.y == 0 && h == 0);
    // items before this sequence's
    long long before = 0;
    for (int j = threadIdx.x; j < b; j += DECAY_SCAN_THREADS) {
        decay_span(p.bt, j, first, n, bad);
        before += decay_segments(p, n);
    }
    __shared__ long long sums[DECAY_SCAN_THREADS / 32];
#pragma unroll
    for (int o = 16; o; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = before;
    __syncthreads();
    before = 0;
    for (int i = 0; i < DECAY_SCAN_THREADS / 32; ++i) before += sums[i];
    const int64_t e = (int64_t)blockIdx.y * (4 * DECAY_SCAN_THREADS) + 4 * threadIdx.x;
    if (e >= size) return;
    // (offsets that name tokens twice can give more items than there is room for)
    const int items = (int)min((long long)decay_segments(p, s.n), max(0ll, p.items - before));
    float* state = p.m.states + ((int64_t)max(s.slot, 0) * p.m.heads + h) * size + e;
    float4 x = s.zero ? make_float4(0.f, 0.f, 0.f, 0.f) : *reinterpret_cast<const float4*>(state);
    float* at = p.part + before * per + h * size + e;
    const float* fades = p.fade + (int64_t)before * p.m.heads + h;
    for (int i = 0; i < items; i += DECAY_SCAN_AHEAD) {
        float4 y[DECAY_SCAN_AHEAD];
        float f[DECAY_SCAN_AHEAD];
#pragma unroll
        for (int j = 0; j < DECAY_SCAN_AHEAD; ++j)
            if (i + j < items) {
                y[j] = *reinterpret_cast<const float4*>(at + (i + j) * per);
                f[j] = fades[(int64_t)(i + j) * p.m.heads];
            }
#pragma unroll
        for (int j = 0; j < DECAY_SCAN_AHEAD; ++j)
            if (i + j < items) {
                *reinterpret_cast<float4*>(at + (i + j) * per) = x;
                x.x = grow_add(x.x, f[j], y[j].x);
                x.y = grow_add(x.y, f[j], y[j].y);
                x.z = grow_add(x.z, f[j], y[j].z);
                x.w = grow_add(x.w, f[j], y[j].w);
            }
    }
    if (s.slot >= 0) *reinterpret_cast<float4*>(state) = x;
}

}  // namespace ccv3d
