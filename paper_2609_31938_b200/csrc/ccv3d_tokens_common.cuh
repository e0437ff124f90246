// Shared pieces of the token operators: device views of the C structs, element access, E4M3 conversion, reductions.
#pragma once
#include "../../include/ccv3d.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace ccv3d {

// CCV3D_TOKENS_* reports: bits are only ever set, so a plain atomic OR in any order is enough.
__device__ __forceinline__ void report(uint32_t* status, uint32_t bits) { if (status) atomicOr(status, bits); }

// Four neighbouring elements as floats; p is aligned to 4 elements.
__device__ __forceinline__ void load4(const float* p, float (&v)[4]) {
    const float4 t = *reinterpret_cast<const float4*>(p);
    v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, float (&v)[4]) {
    const uint2 t = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(t.x << 16); v[1] = __uint_as_float(t.x & 0xFFFF0000u);
    v[2] = __uint_as_float(t.y << 16); v[3] = __uint_as_float(t.y & 0xFFFF0000u);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float (&v)[4]) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// Two floats to two E4M3 codes (nearest even, magnitudes beyond 448 and infinities to 448, NaN to NaN); lo in the low byte.
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
    unsigned short r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t to_e4m3x4(const float (&v)[4]) {
    return to_e4m3x2(v[0], v[1]) | (to_e4m3x2(v[2], v[3]) << 16);
}
// Two E4M3 codes to two halves (exact: 3 mantissa bits, magnitudes 2^-9 .. 448).
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t codes16) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)codes16));
    return r;
}
__device__ __forceinline__ void e4m3x4_to_float(uint32_t codes, float (&v)[4]) {
    const uint32_t a = e4m3x2_to_half2(codes & 0xFFFFu), b = e4m3x2_to_half2(codes >> 16);
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&a)), y = __half22float2(*reinterpret_cast<const __half2*>(&b));
    v[0] = x.x; v[1] = x.y; v[2] = y.x; v[3] = y.y;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ int warp_scan(int v) {   // inclusive
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}

// One sequence of a batch after its arrays were checked: new tokens first .. first + n - 1 of the packed rows at
// positions total - n .. total - 1.  Offsets outside 0 .. tokens and lengths past the page table are cut and reported.
struct Seq { int first, n, total; };
__device__ __forceinline__ Seq load_seq(const ccv3d_token_batch& bt, int page_tokens, int b, uint32_t* status) {
    int s = __ldg(bt.new_start + b), e = __ldg(bt.new_start + b + 1), t = __ldg(bt.total + b);
    const long long room = (long long)bt.max_pages * page_tokens;
    if (s < 0 || e < s || e > bt.tokens || t < 0 || t > room || e - s > bt.max_new) {
        report(status, CCV3D_TOKENS_BAD_LENGTH);
        s = min(max(s, 0), bt.tokens);
        e = min(max(e, s), s + min(bt.tokens - s, bt.max_new));
        t = (int)min((long long)max(t, 0), room);
    }
    return {s, e - s, t};
}
// Sum over the warp of numbers below 2^31, which itself may lie beyond.
__device__ __forceinline__ long long warp_sum_wide(int v) {
    return ((long long)__reduce_add_sync(0xffffffffu, (unsigned)v >> 16) << 16) + __reduce_add_sync(0xffffffffu, (unsigned)v & 0xFFFFu);
}
// Page of a sequence's j-th block of tokens, or -1 (reported) where the table names none of the pool's.
__device__ __forceinline__ int load_page(const ccv3d_token_batch& bt, const ccv3d_kv_cache& c, int b, int j, uint32_t* status) {
    const int page = __ldg(bt.page_table + (size_t)b * bt.max_pages + j);
    if ((unsigned)page < (unsigned)c.pages) return page;
    report(status, CCV3D_TOKENS_BAD_PAGE);
    return -1;
}

}  // namespace ccv3d
