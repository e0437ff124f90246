// Attention of many query rows over the paged E4M3 cache: one block for each row.
#pragma once
#include "ccv3d_tokens_attend.cuh"

namespace ccv3d {

// One block of 128 threads for each (token, head): a running softmax over the cache 128 tokens at a time.
template <typename T, int D>
__global__ void __launch_bounds__(128) kv_attend_row_kernel(const AttendParams p) {
    __shared__ float qs[D], ps[128], part[4];
    const int64_t row = blockIdx.x;
    const int token = (int)(row / p.q_heads), head = (int)(row % p.q_heads), tid = threadIdx.x, P = p.c.page_tokens;
    int b = 0;
    for (int lo = 0, hi = p.bt.batch; lo < hi;) {          // last sequence that starts at or before the token
        const int mid = (lo + hi) / 2;
        if (__ldg(p.bt.new_start + mid) <= token) { b = mid; lo = mid + 1; } else hi = mid;
    }
    const Seq s = load_seq(p.bt, P, b, p.status);
    if (token < s.first || token >= s.first + s.n) return;
    int lo, hi;
    visible(p, s.total - s.n + token - s.first, s.total, lo, hi);
    if (tid < D) qs[tid] = load1((const T*)p.q.data + token * p.q.token_stride + head * p.q.head_stride + tid);
    __syncthreads();
    const int kvh = head / p.group, H = p.c.kv_heads;
    float m = -INFINITY, l = 0.f, acc = 0.f;
    for (int t0 = lo; t0 < hi; t0 += 128) {
        const int t = t0 + tid;
        float x = -INFINITY, vs = 0.f;
        int page = -1;
        if (t < hi) page = load_page(p.bt, p.c, b, t / P, p.status);
        if (page >= 0) {
            const uint8_t* k = (const uint8_t*)p.c.codes + (((int64_t)page * 2 * H + kvh) * P + t % P) * D;
            float sum = 0.f;
            for (int i = 0; i < D; i += 4) {
                float c[4];
                e4m3x4_to_float(*reinterpret_cast<const uint32_t*>(k + i), c);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum = fmaf(c[j], qs[i + j], sum);
            }
            x = sum * p.c.scales[(int64_t)page * 2 * H + kvh] * p.scale;
            vs = p.c.scales[((int64_t)page * 2 + 1) * H + kvh];
        }
        float mm = warp_max(x);
        if ((tid & 31) == 0) part[tid >> 5] = mm;
        __syncthreads();
        mm = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
        const float now = fmaxf(m, mm);
        const float f = m == -INFINITY ? 0.f : __expf(m - now), e = x == -INFINITY ? 0.f : __expf(x - now);
        const float tot = warp_sum(e);
        __syncthreads();
        ps[tid] = e * vs;
        if ((tid & 31) == 0) part[tid >> 5] = tot;
        __syncthreads();
        l = l * f + part[0] + part[1] + part[2] + part[3];
        m = now;
        acc *= f;
        if (tid < D)
            for (int i = 0; i < 128 && t0 + i < hi; ++i) {
                const int pg = load_page(p.bt, p.c, b, (t0 + i) / P, nullptr);
                if (pg < 0) continue;
                const uint8_t* v = (const uint8_t*)p.c.codes + ((((int64_t)pg * 2 + 1) * H + kvh) * P + (t0 + i) % P) * D;
                float c[4];
                e4m3x4_to_float(v[tid], c);
                acc = fmaf(ps[i], c[0], acc);
            }
        __syncthreads();
    }
    if (tid < D)
        store1((T*)p.o.data + token * p.o.token_stride + head * p.o.head_stride + tid, l > 0.f || l != l ? acc / l : 0.f);
    if (tid == 0 && p.lse) p.lse[(int64_t)token * p.q_heads + head] = l != 0.f ? m + logf(l) : -INFINITY;
}

}  // namespace ccv3d
