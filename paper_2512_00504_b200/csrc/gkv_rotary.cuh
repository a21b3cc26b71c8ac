// Rotary positions on the device: the angle of a pair at a position, and the turn itself. Every kernel that rotates does it through
// these two, so that a key has the same bits whichever of them it went through.
#pragma once

#include "gkv_common.cuh"
#include "gkv_internal.h"

namespace gkv {

// cos and sin (times the factor) of pos * turns * 2^-64 turns; sign: -1 turns the other way. The 64-bit product wraps at whole turns, so
// nothing is lost at any position. Its upper word is taken relative to the nearest quarter turn, which leaves an angle x of at most pi/4
// (to 2^-32 turns, 1.5e-9), and cos and sin of that are their Taylor series, sin to x^9 and cos to x^10: what follows is below 2e-9 and 6e-11,
// all in all cos and sin are off by less than 1.6 times 2^-24. (With sincospif on the same angle an append of one row took 0.7 us longer.)
__device__ __forceinline__ float2 rotary_cos_sin(uint64_t turns, int32_t pos, float factor, float sign) {
    const uint32_t phase = (uint32_t)((turns * (uint64_t)(int64_t)pos) >> 32);
    const uint32_t quarter = (phase + (1u << 29)) >> 30;
    const float x = (float)(int32_t)(phase - (quarter << 30)) * 1.46291807926715968e-9f;      // 2 pi / 2^32
    const float z = x * x;
    float s = __fmaf_rn(1.f / 362880.f, z, -1.f / 5040.f), c = __fmaf_rn(-1.f / 3628800.f, z, 1.f / 40320.f);
    s = __fmaf_rn(s, z, 1.f / 120.f);
    c = __fmaf_rn(c, z, -1.f / 720.f);
    s = __fmaf_rn(s, z, -1.f / 6.f);
    c = __fmaf_rn(c, z, 1.f / 24.f);
    s = __fmaf_rn(__fmul_rn(s, z), x, x);
    c = __fmaf_rn(c, z, -0.5f);
    c = __fmaf_rn(c, z, 1.f);
    const float cs = quarter & 1 ? s : c, sn = quarter & 1 ? c : s;
    const uint32_t minus_c = ((quarter + 1) & 2) << 30, minus_s = (quarter & 2) << 30;
    return make_float2(__uint_as_float(__float_as_uint(cs) ^ minus_c) * factor, __uint_as_float(__float_as_uint(sn) ^ minus_s) * (factor * sign));
}
// (a, b) turned by it, in 32 bits.
__device__ __forceinline__ float2 rotary_turn(float a, float b, float c, float s) {
    return make_float2(__fmaf_rn(a, c, -__fmul_rn(b, s)), __fmaf_rn(b, c, __fmul_rn(a, s)));
}

}  // namespace gkv
