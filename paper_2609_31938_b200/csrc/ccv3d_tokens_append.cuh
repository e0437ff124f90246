// Append to the paged E4M3 cache, with the position rotation of keys (and queries) on the way.
//
// A block of 8 warps owns one (page, keys or values, head): it holds the page's new tokens in registers, takes the
// largest magnitude over all of them, settles the page's scale (the smallest power of two under which everything fits
// into +-448, at least the old one where older tokens stay), moves older codes to it where it grew, and writes the new
// codes.  Every input is read once.  The blocks behind those rotate the queries.
#pragma once
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

constexpr int APPEND_THREADS = 256;
constexpr int MIN_SCALE_EXP = -64;

// Rotates the four elements 4l .. 4l+3 of a row held by lane l of a group of LPT lanes (all lanes of the warp call it).
// Products and sums are rounded one by one, as elementwise code in FP32 would.
template <int LPT>
__device__ __forceinline__ void rotate4(const ccv3d_rotary& r, int token, int l, float (&v)[4], uint32_t* status) {
    const int e = 4 * l, pairs = r.pairs;
    const bool on = e < 2 * pairs;
    // the pairs this lane's elements belong to: one each (split halves) or two in all (interleaved)
    const int j = r.interleaved ? e / 2 : (e < pairs ? e : e - pairs);
    float c[4] = {1.f, 1.f, 1.f, 1.f}, s[4] = {0.f, 0.f, 0.f, 0.f};
    if (on) {
        const int n = r.interleaved ? 2 : 4;
        int row_of[3];
#pragma unroll
        for (int a = 0; a < 3; ++a) {
            int row = a < r.axes ? __ldg(r.positions + (int64_t)token * r.axes + a) : 0;
            if ((unsigned)row >= (unsigned)r.rows) {
                report(status, CCV3D_TOKENS_BAD_POSITION);
                row = row < 0 ? 0 : r.rows - 1;
            }
            row_of[a] = row;
        }
        const int s0 = r.section[0], s1 = s0 + r.section[1];
        auto row_at = [&](int i) { return i < s0 ? row_of[0] : (i < s1 ? row_of[1] : row_of[2]); };
        const int first = row_at(j);
        if (!r.interleaved && first == row_at(j + 3)) {
            load4(r.cos_table + (int64_t)first * pairs + j, c);
            load4(r.sin_table + (int64_t)first * pairs + j, s);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < n) {
                    const int64_t at = (int64_t)row_at(j + i) * pairs + j + i;
                    c[i] = __ldg(r.cos_table + at);
                    s[i] = __ldg(r.sin_table + at);
                }
        }
    }
    if (r.interleaved) {
        if (on) {
            const float a0 = v[0], b0 = v[1], a1 = v[2], b1 = v[3];
            v[0] = __fsub_rn(__fmul_rn(a0, c[0]), __fmul_rn(b0, s[0]));
            v[1] = __fadd_rn(__fmul_rn(b0, c[0]), __fmul_rn(a0, s[0]));
            v[2] = __fsub_rn(__fmul_rn(a1, c[1]), __fmul_rn(b1, s[1]));
            v[3] = __fadd_rn(__fmul_rn(b1, c[1]), __fmul_rn(a1, s[1]));
        }
    } else {
        const bool lower = e < pairs;
        const int other = lower ? l + pairs / 4 : l - pairs / 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float w = __shfl_sync(0xffffffffu, v[i], other, LPT);
            if (on) {
                const float t = __fmul_rn(w, s[i]), u = __fmul_rn(v[i], c[i]);
                v[i] = lower ? __fsub_rn(u, t) : __fadd_rn(u, t);
            }
        }
    }
}

template <typename T, int D, int P>
__global__ void __launch_bounds__(APPEND_THREADS) kv_append_kernel(const AppendParams p) {
    constexpr int LPT = D / 4;                       // lanes for one token
    constexpr int TPI = APPEND_THREADS / LPT;        // tokens the block takes at a time
    constexpr int R = (P + TPI - 1) / TPI;           // rounds for a whole page
    const int tid = threadIdx.x, l = tid % LPT;
    if (blockIdx.x >= p.kv_blocks) {                 // ---- queries
        const int64_t rows = (int64_t)p.bt.tokens * p.q_heads;
        const int64_t row = (int64_t)(blockIdx.x - p.kv_blocks) * TPI + tid / LPT;
        const bool live = row < rows;
        const int token = live ? (int)(row / p.q_heads) : 0, head = live ? (int)(row % p.q_heads) : 0;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (live) load4((const T*)p.q.data + token * p.q.token_stride + head * p.q.head_stride + 4 * l, v);
        if (p.rot.cos_table) rotate4<LPT>(p.rot, token, l, v, p.status);
        if (live) store4((T*)p.qo.data + token * p.qo.token_stride + head * p.qo.head_stride + 4 * l, v);
        return;
    }
    // ---- keys and values: block -> (page of a sequence, keys or values, head)
    __shared__ int unit_seq, unit_page;
    __shared__ float part[APPEND_THREADS / 32];
    const int H = p.c.kv_heads;
    const int unit = blockIdx.x / (2 * H), kvh = blockIdx.x % (2 * H), is_v = kvh >= H, head = is_v ? kvh - H : kvh;
    if (tid < 32) {
        if (tid == 0) unit_seq = -1;
        __syncwarp();
        int base = 0;
        for (int b0 = 0; b0 < p.bt.batch; b0 += 32) {
            int pages = 0;
            if (b0 + tid < p.bt.batch) {
                const Seq s = load_seq(p.bt, P, b0 + tid, p.status);
                const int n = min(s.n, s.total);     // more new tokens than cached ones: the first have no place
                if (n < s.n) report(p.status, CCV3D_TOKENS_BAD_LENGTH);
                if (n > 0) pages = (s.total - 1) / P - (s.total - n) / P + 1;
            }
            const int upto = base + warp_scan(pages);
            if (pages > 0 && unit >= upto - pages && unit < upto) {
                unit_seq = b0 + tid;
                unit_page = unit - (upto - pages);
            }
            base = __shfl_sync(0xffffffffu, upto, 31);
            if (unit < base) break;
        }
    }
    __syncthreads();
    const int b = unit_seq;
    if (b < 0) return;                               // the grid is a bound
    Seq s = load_seq(p.bt, P, b, nullptr);
    const int lost = max(0, s.n - s.total);
    s.first += lost;
    s.n -= lost;
    const int old = s.total - s.n;
    const int j = old / P + unit_page;
    const int page = load_page(p.bt, p.c, b, j, p.status);
    if (page < 0) return;
    const int t0 = max(0, old - j * P), t1 = min(P, s.total - j * P);        // the page's new tokens
    const int row0 = s.first + (j * P + t0) - old;
    const ccv3d_heads& src = is_v ? p.v : p.k;
    const T* in = (const T*)src.data + head * src.head_stride + 4 * l;
    float v[R][4];
    float most = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int t = t0 + r * TPI + tid / LPT;
        v[r][0] = v[r][1] = v[r][2] = v[r][3] = 0.f;
        if (t < t1) load4(in + (int64_t)(row0 + t - t0) * src.token_stride, v[r]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int t = t0 + r * TPI + tid / LPT;
        if (!is_v && p.rot.cos_table && t0 + r * TPI < t1)       // (the same for the whole block)
            rotate4<LPT>(p.rot, row0 + min(t, t1 - 1) - t0, l, v[r], p.status);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = fabsf(v[r][i]);
            if (t < t1 && a <= 3.402823466e38f) most = fmaxf(most, a);   // infinities and NaN stay out
        }
    }
    most = warp_max(most);
    if ((tid & 31) == 0) part[tid >> 5] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < APPEND_THREADS / 32; ++i) most = fmaxf(most, part[i]);
    // smallest e with most <= 448 * 2^e = 1.75 * 2^(8 + e)
    const uint32_t bits = __float_as_uint(most);
    int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    e = max(e, MIN_SCALE_EXP);
    float scale = __uint_as_float((uint32_t)(e + 127) << 23);
    float* at = p.c.scales + ((int64_t)page * 2 + is_v) * H + head;
    uint8_t* codes = (uint8_t*)p.c.codes + (((int64_t)page * 2 + is_v) * H + head) * (P * D);
    if (t0 > 0) {
        const float was = *at;
        scale = fmaxf(was, scale);
        if (scale != was) {
            const float f = was / scale;
            for (int i = tid; i < t0 * (D / 4); i += APPEND_THREADS) {
                float c[4];
                e4m3x4_to_float(reinterpret_cast<uint32_t*>(codes)[i], c);
#pragma unroll
                for (int k = 0; k < 4; ++k) c[k] *= f;
                reinterpret_cast<uint32_t*>(codes)[i] = to_e4m3x4(c);
            }
        }
        __syncthreads();                             // all have read the old scale
    }
    if (tid == 0) *at = scale;
    const float inv = 1.f / scale;                   // a power of two: exact
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int t = t0 + r * TPI + tid / LPT;
        if (t < t1) {
            float c[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = v[r][i] * inv;
            reinterpret_cast<uint32_t*>(codes)[t * (D / 4) + l] = to_e4m3x4(c);
        }
    }
}

}  // namespace ccv3d
