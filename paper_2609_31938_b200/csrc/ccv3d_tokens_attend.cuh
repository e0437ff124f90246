// Attention over the paged E4M3 cache: what its kernels share, and the sum over the parts of a split softmax.
//
// The work of a call is a list of items (a sequence, a block of its query rows, a kv head), each a run of units (a
// stretch of cached tokens); block i of G takes units [i U / G, (i + 1) U / G) of the whole list, so every block has
// the same to read whatever the sequences' lengths, and nothing about them has to be known on the host.  An item that
// lies in one block is finished there; one that crosses blocks leaves a part (unnormalised sums, their base
// and weight) in each, and attend_join_kernel adds the parts in block order.
//
// Softmax in powers of two: with t = score * log2(e) and e_v = log2 of the value scale of the token's page, the weight
// of a value code is 2^(t + e_v - base), base the running one of t + e_v, so page scales of any size stay out of the range
// of the 16-bit weights; the softmax's own sum takes that times 1 / value scale.
// Weights are rounded to one half for BF16 (11 bits; the sum of weights takes them unrounded): a second one for the remainder, as
// F32 has, would double the output products for bits that outputs of 8 bits drop but where they decide a rounding, and the
// tile kernel has no TMEM columns for it next to two row blocks.
#pragma once
#include <cuda.h>

#include "ccv3d_tc_ptx.cuh"
#include "ccv3d_tokens_common.cuh"
#include "ccv3d_tokens_softmax.cuh"

namespace ccv3d {

// The item whose first part block i wrote in slot 2 i + 1, to be joined with the slots 2 (i + 1), 2 (i + 2), ...
struct Join { int parts, row0, rows, head0; };   // rows row0 .. row0 + rows - 1 of the (token, head of the kv group) order

struct AttendParams {
    ccv3d_kv_cache c;
    ccv3d_token_batch bt;
    ccv3d_heads q, o;
    float* lse;
    int q_heads, group;      // group = q_heads / kv_heads
    float scale;
    int frame, window;
    uint32_t* status;
    long long wait_clk;      // bound of every wait, in SM clocks
    // scratch: slots 2 i (an item that began before block i) and 2 i + 1 (one that ends behind it)
    float* part;             // [slot][slot_rows][dim] sums
    float2* part_ml;         // [slot][slot_rows] base and weight
    Join* join;              // [block]; parts = 0: nothing to join
    int slot_rows;
};

// Most units of a call.  The host bounds them by the rows of the packed tensors and the page tables' room; offsets that fall can
// name rows again and again, and a list that so grows past the bound is not walked at all.
constexpr int MAX_UNITS = 2000000000;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// log2 and reciprocal of a page's value scale; scales are positive (0, never written by an append, counts as tiny)
__device__ __forceinline__ void scale_terms(float vs, float& e, float& inv) {
    vs = fmaxf(vs, 1e-36f);
    e = __log2f(vs);
    inv = 1.f / vs;
}

// Tokens [lo, hi) that the token at position pos of a sequence of `total` tokens sees.
__device__ __forceinline__ void visible(const AttendParams& p, int pos, int total, int& lo, int& hi) {
    const int start = p.frame > 0 ? pos - pos % p.frame : pos;
    hi = p.frame > 0 ? (int)min((int64_t)total, (int64_t)start + p.frame) : total;
    lo = p.window < 0 ? 0 : max(0, start - p.window);
    if (pos < 0) lo = hi = 0;
}

// Row r of a kv head's query rows: token r / group (packed), head r % group of the kv head's group.
template <typename T>
__device__ __forceinline__ void store_out(const AttendParams& p, int token, int head, int d, const float (&v)[4]) {
    store4((T*)p.o.data + token * p.o.token_stride + head * p.o.head_stride + d, v);
}
__device__ __forceinline__ float lse_of(float base, float l) {
    return l != 0.f ? (base + log2f(l)) * LN2 : -INFINITY;     // (a row that saw NaN has l = NaN)
}

// Adds the parts of the item that starts in block blockIdx.x of the attention kernel, rows blockIdx.y, + gridDim.y, ...
// Few parts (a tile of rows that two blocks share): D / 4 threads to a row, part after part.  But an item can have as many
// parts as there were blocks (one stream behind a long cache): then a row's parts are spread over all threads, their bases
// and weights a part to a thread, their sums D / 4 threads to a part.
constexpr int JOIN_THREADS = 128, JOIN_PARTS = 1024, JOIN_FEW = 8;
template <typename T, int D>
__global__ void __launch_bounds__(JOIN_THREADS) attend_join_kernel(const AttendParams p) {
    constexpr int L = D / 4, SLICES = JOIN_THREADS / L;
    __shared__ float weight[JOIN_PARTS], red[2][JOIN_THREADS / 32];
    __shared__ float4 sums[JOIN_THREADS];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const Join j = p.join[blockIdx.x];
    if (j.parts == 0) return;
    const int tid = threadIdx.x, slice = tid / L, d = tid % L * 4;
    const int64_t slot0 = 2 * (int64_t)blockIdx.x;                  // part i > 0 lies in slot0 + 2 i, part 0 in slot0 + 1
    auto finish = [&](int r, float m, float l, float (&acc)[4]) {
        const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = l != 0.f ? acc[i] * inv : 0.f;
        const int token = (j.row0 + r) / p.group, head = j.head0 + (j.row0 + r) % p.group;
        store_out<T>(p, token, head, d, acc);
        if (d == 0 && p.lse) p.lse[(int64_t)token * p.q_heads + head] = lse_of(m, l);
    };
    if (j.parts <= JOIN_FEW) {
        for (int r = blockIdx.y * SLICES + slice; r < j.rows; r += gridDim.y * SLICES) {
            float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
            float2 ml[JOIN_FEW];
#pragma unroll
            for (int i = 0; i < JOIN_FEW; ++i)
                if (i < j.parts) {
                    ml[i] = p.part_ml[(slot0 + (i ? 2 * i : 1)) * p.slot_rows + r];
                    m = fmaxf(m, ml[i].x);
                }
#pragma unroll
            for (int i = 0; i < JOIN_FEW; ++i)
                if (i < j.parts) {
                    const float4 v = *reinterpret_cast<const float4*>(p.part + ((slot0 + (i ? 2 * i : 1)) * p.slot_rows + r) * D + d);
                    const float w = ml[i].x == -INFINITY ? 0.f : exp2_fast(ml[i].x - m);
                    l = fmaf(w, ml[i].y, l);
                    acc[0] = fmaf(w, v.x, acc[0]); acc[1] = fmaf(w, v.y, acc[1]);
                    acc[2] = fmaf(w, v.z, acc[2]); acc[3] = fmaf(w, v.w, acc[3]);
                }
            finish(r, m, l, acc);
        }
        return;
    }
    for (int r = blockIdx.y; r < j.rows; r += gridDim.y) {
        auto at = [&](int i) { return (slot0 + (i ? 2 * i : 1)) * p.slot_rows + r; };
        float m = -INFINITY;
        for (int i = tid; i < j.parts; i += JOIN_THREADS) m = fmaxf(m, p.part_ml[at(i)].x);
        m = warp_max(m);
        if ((tid & 31) == 0) red[0][tid >> 5] = m;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < JOIN_THREADS / 32; ++k) m = fmaxf(m, red[0][k]);
        float l = 0.f;
        for (int i = tid; i < j.parts; i += JOIN_THREADS) {
            const float2 ml = p.part_ml[at(i)];
            const float w = ml.x == -INFINITY ? 0.f : exp2_fast(ml.x - m);
            weight[i] = w;
            l = fmaf(w, ml.y, l);
        }
        l = warp_sum(l);
        if ((tid & 31) == 0) red[1][tid >> 5] = l;
        __syncthreads();
        l = 0.f;
#pragma unroll
        for (int k = 0; k < JOIN_THREADS / 32; ++k) l += red[1][k];
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int i = slice; i < j.parts; i += SLICES) {
            const float4 v = *reinterpret_cast<const float4*>(p.part + at(i) * D + d);
            const float w = weight[i];
            acc[0] = fmaf(w, v.x, acc[0]); acc[1] = fmaf(w, v.y, acc[1]);
            acc[2] = fmaf(w, v.z, acc[2]); acc[3] = fmaf(w, v.w, acc[3]);
        }
        sums[tid] = make_float4(acc[0], acc[1], acc[2], acc[3]);
        __syncthreads();
        if (slice == 0) {
#pragma unroll
            for (int k = 1; k < SLICES; ++k) {
                const float4 v = sums[k * L + tid];
                acc[0] += v.x; acc[1] += v.y; acc[2] += v.z; acc[3] += v.w;
            }
            finish(r, m, l, acc);
        }
    }
}

}  // namespace ccv3d
