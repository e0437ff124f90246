// The running base of a softmax in powers of two: a score v (in units of log2) weighs 2^(v - base), as a half.
//
// Plain C++, so that the arithmetic is tested on the host as well.  The base is a whole number 2^8 under the largest score when it was
// taken and only moves when a weight would pass 2^15, so most tiles of a row need one pass.  From 2^22 on the base is the
// largest score itself, and nothing may lie above it: neighbouring floats are a unit and later more apart there, base +- a
// small number rounds to either side, and a weight could end above the largest half.
#pragma once
#include <math.h>

#ifdef __CUDACC__
#define CCV3D_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define CCV3D_HOST_DEVICE inline
#endif

namespace ccv3d {

constexpr float WEIGHT_SHIFT = 8.f, WEIGHT_TOP = 15.f;   // weights start at 2^8 for the largest score and may reach 2^15
constexpr float SCORE_EXACT = 4194304.f;                 // whole numbers to here, and a shift more, add without rounding

// Base for a largest score `most` (-infinity: none yet).
CCV3D_HOST_DEVICE float base_for(float most) {
    const float c = ceilf(most);
    return fabsf(c) <= SCORE_EXACT ? c - WEIGHT_SHIFT : c;
}
// Largest score that a base bears: 2^(v - base) is at most 2^15 for v up to it.
CCV3D_HOST_DEVICE float base_limit(float base) { return fabsf(base) < 2.f * SCORE_EXACT ? base + WEIGHT_TOP : base; }
// What is taken off a score: the base, or any finite number while there is none.
CCV3D_HOST_DEVICE float base_or_start(float base) { return base == -INFINITY ? -WEIGHT_SHIFT : base; }

}  // namespace ccv3d
