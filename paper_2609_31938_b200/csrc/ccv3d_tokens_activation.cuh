// Activations of the products' and group norms' epilogues.
#pragma once
#include "../../include/ccv3d.h"

#include <cuda_runtime.h>

namespace ccv3d {

// exp and the division by approximations good to some 2^-21 where the result is rounded to BF16 anyway (EXACT: to the last bits)
template <bool EXACT>
__device__ __forceinline__ float sigmoid_times(float x, float u) {    // x / (1 + exp(-u))
    if constexpr (EXACT) return x / (1.f + expf(-u));
    else return __fdividef(x, 1.f + fminf(__expf(-u), 1e38f));       // (the fast division gives 0 for divisors past 2^126)
}
template <bool EXACT>
__device__ __forceinline__ float activate(float x, int kind) {
    if (kind == CCV3D_ACT_SILU) return sigmoid_times<EXACT>(x, x);
    if (kind == CCV3D_ACT_GELU) return 0.5f * x * (1.f + erff(x * 0.70710678118654752f));
    if (kind == CCV3D_ACT_GELU_TANH) return sigmoid_times<EXACT>(x, 1.5957691216057308f * fmaf(0.044715f * x * x, x, x));
    return x;
}

}  // namespace ccv3d
