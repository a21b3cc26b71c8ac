// cos and sin of an angle of at most an eighth of a turn. Plain C++, so that a host compiler can check it over all angles (where a product is
// not to be joined with the sum behind it, there without contraction).
#pragma once

#include <math.h>
#include <stdint.h>

#ifndef GKV_HOST_DEVICE
#ifdef __CUDACC__
#define GKV_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define GKV_HOST_DEVICE inline
#endif
#endif

namespace gkv {

// Of `rest` times 2^-32 turns, |rest| <= 2^29: their Taylor series, sin to x^9 and cos to x^10. What follows is below 1.8e-9 and 1.2e-10; with all
// roundings, and where the angle was cut to a multiple of 2^-32 turns, cos is off by at most 1.73 and sin by 1.53 times 2^-24 (all 2^30 of them
// gone through). (With sincospif on the same angle an append of one row took 0.7 us longer.)
GKV_HOST_DEVICE void small_cos_sin(int32_t rest, float* cos_x, float* sin_x) {
    const float x = (float)rest * 1.46291807926715968e-9f;      // 2 pi / 2^32
    const float z = x * x;
    float s = fmaf(1.f / 362880.f, z, -1.f / 5040.f), c = fmaf(-1.f / 3628800.f, z, 1.f / 40320.f);
    s = fmaf(s, z, 1.f / 120.f);
    c = fmaf(c, z, -1.f / 720.f);
    s = fmaf(s, z, -1.f / 6.f);
    c = fmaf(c, z, 1.f / 24.f);
#ifdef __CUDA_ARCH__
    s = fmaf(__fmul_rn(s, z), x, x);
#else
    s = fmaf(s * z, x, x);
#endif
    c = fmaf(c, z, -0.5f);
    *cos_x = fmaf(c, z, 1.f);
    *sin_x = s;
}

}  // namespace gkv
