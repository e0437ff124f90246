// Append to the paged E4M3 cache, with the position rotation of keys (and queries) on the way.
//
// Bound by HBM where there are many tokens, by the chain of dependent loads (sequence, page, position, table) where there
// are few.  A block owns the keys and values of one (page, head), or a cluster of 2 or 4 blocks does where the page's tokens are
// more than four rounds of a block: it holds the page's new tokens in registers, takes the largest magnitude over all of them
// (over the cluster through its shared memory), settles the page's scale (the smallest power of two under which
// everything fits into +-448, at least the old one where older tokens stay), moves older codes to it where it grew, and
// writes the new codes.  Every input is read once.  (A page of 128 tokens and 128 channels in one block: 1024 threads or 16
// rounds, either way one block to an SM: 39 us for a frame of 3520 tokens and 12 heads; read twice, 42.)
// The blocks behind those rotate the queries, four heads of a token for each group of lanes that spans a head, so that a
// token's cosines and sines are fetched once for them and their loads are on their way together.
#pragma once
#include "ccv3d_tc_ptx.cuh"
#include "ccv3d_tokens_common.cuh"

namespace ccv3d {

struct AppendParams {
    ccv3d_kv_cache c;
    ccv3d_token_batch bt;
    ccv3d_heads k, v, q, qo;
    ccv3d_rotary rot;        // cos_table == NULL: no rotation
    int q_heads;
    unsigned kv_blocks;      // blocks for pages; the rest rotate queries
    uint32_t* status;
};

// `few`: no sequence brings more tokens than one round of 128 threads takes.
template <int D, int P, bool FEW> struct AppendShape {
    static constexpr int LPT = D / 4, THREADS = FEW ? 128 : 256;               // lanes for one token
    static constexpr int TPI = THREADS / LPT;                                   // tokens at a time
    static constexpr int CLUSTER = FEW || P <= 4 * TPI ? 1 : P / (4 * TPI);     // blocks for a page
    static constexpr int SHARE = P / CLUSTER;                                   // a block's tokens of a page
    static constexpr int R = FEW ? 1 : (SHARE + TPI - 1) / TPI;                 // rounds
};
constexpr int MIN_SCALE_EXP = -64;
constexpr int QUERY_HEADS = 4;

// A lane's part in the rotation of the four elements 4 l .. 4 l + 3 of a head: the same for every token and head.
struct Turn {
    bool on, one;            // any of them turns; all by the same axis
    int pair, axis;          // first pair they belong to (four pairs, or two if interleaved), its axis
};
__device__ __forceinline__ int axis_of(const ccv3d_rotary& r, int pair) {
    return pair < r.section[0] ? 0 : (pair < r.section[0] + r.section[1] ? 1 : 2);
}
__device__ __forceinline__ Turn turn_of(const ccv3d_rotary& r, int l) {
    Turn t;
    const int e = 4 * l;
    t.on = r.cos_table && e < 2 * r.pairs;
    t.pair = r.interleaved ? e / 2 : (e < r.pairs ? e : e - r.pairs);
    t.axis = t.on ? axis_of(r, t.pair) : 0;
    t.one = t.on && t.axis == axis_of(r, t.pair + (r.interleaved ? 1 : 3));
    return t;
}
// Row of the table for a token and axis; positions outside the table are cut and reported.
__device__ __forceinline__ int table_row(const ccv3d_rotary& r, int token, int axis, uint32_t* status) {
    const int row = __ldg(r.positions + (int64_t)token * r.axes + axis);
    if ((unsigned)row < (unsigned)r.rows) return row;
    report(status, CCV3D_TOKENS_BAD_POSITION);
    return row < 0 ? 0 : r.rows - 1;
}
// Cosines and sines of the lane's pairs for a token; `row`: table_row of the lane's axis.
__device__ __forceinline__ void angles(const ccv3d_rotary& r, const Turn& t, int token, int row, float (&c)[4], float (&s)[4], uint32_t* status) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { c[i] = 1.f; s[i] = 0.f; }
    if (!t.on) return;
    if (t.one) {
        const int64_t at = (int64_t)row * r.pairs + t.pair;
        if (r.interleaved) {
            const float2 x = __ldg(reinterpret_cast<const float2*>(r.cos_table + at)), y = __ldg(reinterpret_cast<const float2*>(r.sin_table + at));
            c[0] = x.x; c[1] = x.y; s[0] = y.x; s[1] = y.y;
        } else {
            load4(r.cos_table + at, c);
            load4(r.sin_table + at, s);
        }
        return;
    }
    for (int i = 0; i < (r.interleaved ? 2 : 4); ++i) {          // pairs on both sides of a section's border
        const int64_t at = (int64_t)table_row(r, token, axis_of(r, t.pair + i), status) * r.pairs + t.pair + i;
        c[i] = __ldg(r.cos_table + at);
        s[i] = __ldg(r.sin_table + at);
    }
}
// Turns the four elements of a head held by lane l of a group of LPT lanes (all lanes of the warp call it).  Products and
// sums are rounded one by one, as elementwise code in FP32 would.
template <int LPT>
__device__ __forceinline__ void rotate4(const ccv3d_rotary& r, const Turn& t, int l, const float (&c)[4], const float (&s)[4], float (&v)[4]) {
    if (r.interleaved) {
        if (t.on) {
            const float a0 = v[0], b0 = v[1], a1 = v[2], b1 = v[3];
            v[0] = __fsub_rn(__fmul_rn(a0, c[0]), __fmul_rn(b0, s[0]));
            v[1] = __fadd_rn(__fmul_rn(b0, c[0]), __fmul_rn(a0, s[0]));
            v[2] = __fsub_rn(__fmul_rn(a1, c[1]), __fmul_rn(b1, s[1]));
            v[3] = __fadd_rn(__fmul_rn(b1, c[1]), __fmul_rn(a1, s[1]));
        }
        return;
    }
    const bool lower = 4 * l < r.pairs;
    const int other = lower ? l + r.pairs / 4 : l - r.pairs / 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float w = __shfl_sync(0xffffffffu, v[i], other, LPT);
        const float x = __fmul_rn(w, s[i]), u = __fmul_rn(v[i], c[i]);
        if (t.on) v[i] = lower ? __fsub_rn(u, x) : __fadd_rn(u, x);
    }
}

template <typename T, int D, int P, bool FEW>
__global__ void __launch_bounds__(AppendShape<D, P, FEW>::THREADS, FEW ? 8 : 3) kv_append_kernel(const AppendParams p) {
    using S = AppendShape<D, P, FEW>;
    constexpr int LPT = S::LPT, TPI = S::TPI, R = S::R;
    const int tid = threadIdx.x, l = tid % LPT;
    const Turn turn = turn_of(p.rot, l);
    if (blockIdx.x >= p.kv_blocks) {                 // ---- queries: an item is a token and QUERY_HEADS heads
        const int per_token = (p.q_heads + QUERY_HEADS - 1) / QUERY_HEADS;
        const uint32_t item = (blockIdx.x - p.kv_blocks) * TPI + tid / LPT, items = (uint32_t)p.bt.tokens * per_token;     // (fewer than 2^32: checked)
        const bool live = item < items;
        const int token = live ? item / per_token : 0, h0 = live ? item % per_token * QUERY_HEADS : p.q_heads;
        const int row = live && turn.one ? table_row(p.rot, token, turn.axis, p.status) : 0;
        float v[QUERY_HEADS][4];
#pragma unroll
        for (int h = 0; h < QUERY_HEADS; ++h)
            if (h0 + h < p.q_heads) load4((const T*)p.q.data + token * p.q.token_stride + (h0 + h) * p.q.head_stride + 4 * l, v[h]);
        float c[4], s[4];
        if (p.rot.cos_table) {
            angles(p.rot, turn, token, row, c, s, p.status);
#pragma unroll
            for (int h = 0; h < QUERY_HEADS; ++h) rotate4<LPT>(p.rot, turn, l, c, s, v[h]);
        }
#pragma unroll
        for (int h = 0; h < QUERY_HEADS; ++h)
            if (h0 + h < p.q_heads) store4((T*)p.qo.data + token * p.qo.token_stride + (h0 + h) * p.qo.head_stride + 4 * l, v[h]);
        return;
    }
    // ---- keys and values: block -> (page of a sequence, head), rank in the cluster
    __shared__ int unit_seq, unit_page;
    __shared__ Seq unit_at;
    __shared__ float part[2][S::THREADS / 32], block_most[2];
    const int H = p.c.kv_heads;
    const int rank = blockIdx.x % S::CLUSTER, block = blockIdx.x / S::CLUSTER, unit = block / H, head = block % H;
    if (p.bt.max_new <= 1) {                         // a page to each sequence at most: no search
        if (tid == 0) { unit_seq = unit; unit_page = 0; }
    } else if (tid < 32) {
        if (tid == 0) unit_seq = -1;
        __syncwarp();
        int base = 0;
        for (int b0 = 0; b0 < p.bt.batch; b0 += 32) {
            int pages = 0;
            Seq s = {0, 0, 0};
            if (b0 + tid < p.bt.batch) {
                s = load_seq(p.bt, P, b0 + tid, p.status);
                const int n = min(s.n, s.total);     // more new tokens than cached ones: the first have no place
                if (n < s.n) report(p.status, CCV3D_TOKENS_BAD_LENGTH);
                if (n > 0) pages = (s.total - 1) / P - (s.total - n) / P + 1;
            }
            const int upto = base + warp_scan(pages);
            if (pages > 0 && unit >= upto - pages && unit < upto) {
                unit_seq = b0 + tid;
                unit_page = unit - (upto - pages);
                unit_at = s;
            }
            base = __shfl_sync(0xffffffffu, upto, 31);
            if (unit < base) break;
        }
    }
    __syncthreads();
    const int b = unit_seq;
    if (b < 0) return;                               // the grid is a bound
    Seq s = p.bt.max_new <= 1 ? load_seq(p.bt, P, b, p.status) : unit_at;
    const int lost = max(0, s.n - s.total);
    if (p.bt.max_new <= 1 && lost) report(p.status, CCV3D_TOKENS_BAD_LENGTH);
    s.first += lost;
    s.n -= lost;
    if (s.n == 0) return;
    const int old = s.total - s.n;
    const int j = old / P + unit_page;
    // asked for together: the page, the tokens, their positions; looked at in that order
    int page = __ldg(p.bt.page_table + (size_t)b * p.bt.max_pages + j);
    const int t0 = max(0, old - j * P), t1 = min(P, s.total - j * P);        // the page's new tokens
    const int a0 = max(t0, rank * S::SHARE), a1 = min(t1, (rank + 1) * S::SHARE);        // this block's
    const int first = s.first + (j * P + a0) - old + tid / LPT;              // this thread's token of round 0
    const T* k_in = (const T*)p.k.data + head * p.k.head_stride + 4 * l;
    const T* v_in = (const T*)p.v.data + head * p.v.head_stride + 4 * l;
    float v[2][R][4];
    int row[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        row[r] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[0][r][i] = v[1][r][i] = 0.f;
        if (a0 + r * TPI + tid / LPT < a1) {
            load4(k_in + (int64_t)(first + r * TPI) * p.k.token_stride, v[0][r]);
            load4(v_in + (int64_t)(first + r * TPI) * p.v.token_stride, v[1][r]);
            if (turn.one) row[r] = table_row(p.rot, first + r * TPI, turn.axis, p.status);
        }
    }
    const bool there = (unsigned)page < (unsigned)p.c.pages;
    if (!there) {
        report(p.status, CCV3D_TOKENS_BAD_PAGE);
        page = 0;
    }
    float* at = p.c.scales + (int64_t)page * 2 * H + head;                   // of the keys; of the values H further
    float was[2] = {0.f, 0.f};
    if (t0 > 0) { was[0] = at[0]; was[1] = at[H]; }
    float most[2] = {0.f, 0.f};
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (p.rot.cos_table && a0 + r * TPI < a1) {              // (the same for the whole block)
            float c[4], s[4];
            angles(p.rot, turn, first + min(r * TPI, a1 - 1 - a0 - tid / LPT), row[r], c, s, p.status);
            rotate4<LPT>(p.rot, turn, l, c, s, v[0][r]);
        }
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = fabsf(v[w][r][i]);
                if (a0 + r * TPI + tid / LPT < a1 && a <= 3.402823466e38f) most[w] = fmaxf(most[w], a);      // infinities and NaN stay out
            }
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        most[w] = warp_max(most[w]);
        if ((tid & 31) == 0) part[w][tid >> 5] = most[w];
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int i = 0; i < S::THREADS / 32; ++i) most[w] = fmaxf(most[w], part[w][i]);
    if constexpr (S::CLUSTER > 1) {
        if (tid == 0) { block_most[0] = most[0]; block_most[1] = most[1]; }
        cluster_sync_all();
#pragma unroll
        for (int k = 0; k < S::CLUSTER; ++k)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                uint32_t at_k;
                float other;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at_k) : "r"(smem_u32(&block_most[w])), "r"(k));
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(other) : "r"(at_k) : "memory");
                most[w] = fmaxf(most[w], other);
            }
        cluster_sync_all();                                      // (no block leaves while another still reads its maxima)
    }
    if (!there) return;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        // smallest e with most <= 448 * 2^e = 1.75 * 2^(8 + e)
        const uint32_t bits = __float_as_uint(most[w]);
        int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
        e = max(e, MIN_SCALE_EXP);
        float scale = __uint_as_float((uint32_t)(e + 127) << 23);
        uint32_t* codes = reinterpret_cast<uint32_t*>((uint8_t*)p.c.codes + (((int64_t)page * 2 + w) * H + head) * (P * D));
        if (t0 > 0) {
            scale = fmaxf(was[w], scale);
            if (scale != was[w]) {
                const float f = was[w] / scale;
                for (int i = rank * S::THREADS + tid; i < t0 * (D / 4); i += S::CLUSTER * S::THREADS) {
                    float c[4];
                    e4m3x4_to_float(codes[i], c);
#pragma unroll
                    for (int k = 0; k < 4; ++k) c[k] *= f;
                    codes[i] = to_e4m3x4(c);
                }
            }
        }
        // (every thread of the cluster read the old scale before the barriers above)
        if (tid == 0 && rank == 0) at[w * H] = scale;
        const float inv = 1.f / scale;               // a power of two: exact
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int t = a0 + r * TPI + tid / LPT;
            if (t < a1) {
                float c[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) c[i] = v[w][r][i] * inv;
                codes[t * (D / 4) + l] = to_e4m3x4(c);
            }
        }
    }
}

}  // namespace ccv3d
