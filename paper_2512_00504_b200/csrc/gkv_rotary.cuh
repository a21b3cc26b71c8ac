// Rotary positions on the device: the angle of a pair at a position, and the turn itself. Every kernel that rotates does it through
// these two, so that a key has the same bits whichever of them it went through.
#pragma once

#include "gkv_common.cuh"
#include "gkv_internal.h"

namespace gkv {

// cos and sin (times the factor) of pos * turns * 2^-64 turns. The 64-bit product wraps at whole turns, so nothing is lost at any
// position; the angle is taken relative to the nearest quarter turn, which leaves at most an eighth and keeps all 24 bits of
// its fp32 value, and cos and sin of that are CUDA's (about 1e-7 relative). sign: -1 turns the other way.
__device__ __forceinline__ float2 rotary_cos_sin(uint64_t turns, int32_t pos, float factor, float sign) {
    const uint64_t phase = turns * (uint64_t)(int64_t)pos;
    const uint32_t quarter = (uint32_t)((phase + (1ull << 61)) >> 62);
    const int64_t rest = (int64_t)(phase - ((uint64_t)quarter << 62));
    float s, c;
    sincospif(__ll2float_rn(rest) * 0x1p-63f, &s, &c);
    const float x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;     // |cos|, |sin| up to the signs below
    const float cs = quarter == 1 || quarter == 2 ? -x : x, sn = quarter >= 2 ? -y : y;
    return make_float2(cs * factor, sn * factor * sign);
}
// (a, b) turned by it, in 32 bits.
__device__ __forceinline__ float2 rotary_turn(float a, float b, float c, float s) {
    return make_float2(__fmaf_rn(a, c, -__fmul_rn(b, s)), __fmaf_rn(b, c, __fmul_rn(a, s)));
}

}  // namespace gkv
