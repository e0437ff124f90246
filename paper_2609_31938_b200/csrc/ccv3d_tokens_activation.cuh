// Activations of the products' and group norms' epilogues.
#pragma once
#include "../../include/ccv3d.h"

#include <cuda_runtime.h>

#include <type_traits>

namespace ccv3d {

// x / (1 + exp(-u)).  EXACT: to the last bits; else by the machine's approximations of 2^x and 1 / x, good to 2^-21 beside a rounding to BF16.
template <bool EXACT>
__device__ __forceinline__ float sigmoid_times(float x, float u) {
    if constexpr (EXACT) return x / (1.f + expf(-u));
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(u * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return x * r;
}
template <bool EXACT>
__device__ __forceinline__ float activate(float x, int kind) {
    if (kind == CCV3D_ACT_SILU) return sigmoid_times<EXACT>(x, x);
    if (kind == CCV3D_ACT_GELU) return 0.5f * x * (1.f + erff(x * 0.70710678118654752f));
    if (kind == CCV3D_ACT_GELU_TANH) return sigmoid_times<EXACT>(x, x * fmaf(0.07135481627260025f, x * x, 1.5957691216057308f));
    return x;
}

// The same for N neighbouring values.  Without EXACT, quotients of two values share one reciprocal, 1 / a = b / (a b): the unit that makes 2^x
// and 1 / x takes a sixteenth of a multiprocessor's lanes, and bounds epilogues that do little else.  2^x is cut at 2^60, so that a b stays finite;
// 2^-59 is taken off the quotient, below zero nothing is left, so that a value whose exponent was cut is multiplied by zero (minus infinity becomes
// NaN, as in the formula).  That costs no instruction, and |x| 2^-59 with |x| < 42 where it is more than the value's rounding: less than 2^-53.
template <bool EXACT, int KIND, int N>
__device__ __forceinline__ void activate_all(float (&v)[N]) {
    if constexpr (EXACT || N % 2 || (KIND != CCV3D_ACT_SILU && KIND != CCV3D_ACT_GELU_TANH)) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = activate<EXACT>(v[i], KIND);
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            float d[2], r;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float x = v[i + j];
                const float u = KIND == CCV3D_ACT_SILU ? x * -1.4426950408889634f : x * fmaf(-0.10294324f, x * x, -2.3022082f);
                asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d[j]) : "f"(fminf(u, 60.f)));
                d[j] += 1.f;
            }
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d[0] * d[1]));
            v[i] *= __saturatef(fmaf(r, d[1], -0x1p-59f));
            v[i + 1] *= __saturatef(fmaf(r, d[0], -0x1p-59f));
        }
    }
}

// f with the kind as a constant: loops over many values choose once.
template <typename F>
__device__ __forceinline__ void with_activation(int kind, F&& f) {
    if (kind == CCV3D_ACT_SILU) f(std::integral_constant<int, CCV3D_ACT_SILU>());
    else if (kind == CCV3D_ACT_GELU) f(std::integral_constant<int, CCV3D_ACT_GELU>());
    else if (kind == CCV3D_ACT_GELU_TANH) f(std::integral_constant<int, CCV3D_ACT_GELU_TANH>());
    else f(std::integral_constant<int, CCV3D_ACT_NONE>());
}

}  // namespace ccv3d
