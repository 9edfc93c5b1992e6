// The arithmetic of the 4-bit codec, shared by the kernels that pack (format: store_int4.hip).
#pragma once
#include <hip/hip_runtime.h>

namespace kvpr {

// The correctly rounded a / b for |b| of at most 11 significant bits, r = 1 / b to an ulp or two, nothing under- or
// overflowing.  a - q b is exact, so the sum before its rounding is off by about 2^-22 units in the last place, while a
// quotient by 11 bits that is no midpoint between two floats is at least 2^-12 away from one; none is a midpoint.
__device__ __forceinline__ float quotient(float a, float b, float r) {
    const float q = a * r;
    return fmaf(fmaf(-q, b, a), r, q);
}

// float16((max - min) / 15)
__device__ __forceinline__ _Float16 int4_scale(float mn, float mx) {
    const float range = mx - mn;
    return (_Float16)(fabsf(range) < INFINITY ? quotient(range, 15.f, 1.f / 15.f) : range);
}

// code of x as a float (r = rcp(scale)).  A NaN (a NaN value, or an infinite scale) gives code 0: fmed3 returns the smallest of
// its numbers then.
__device__ __forceinline__ float int4_code(float x, float scale, float mn, float r) {
    return rintf(__builtin_amdgcn_fmed3f(quotient(x - mn, scale, r), 0.f, 15.f));
}

}  // namespace kvpr
