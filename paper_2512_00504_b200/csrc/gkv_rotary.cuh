// Rotary positions on the device: the angle of a pair at a position, and the turn itself. Every kernel that rotates does it through
// these two, so that a key has the same bits whichever of them it went through.
#pragma once

#include "gkv_common.cuh"
#include "gkv_internal.h"
#include "gkv_rotary_series.h"

namespace gkv {

// cos and sin (times the factor) of pos * turns * 2^-64 turns; sign: -1 turns the other way. The 64-bit product wraps at whole turns, so
// nothing is lost at any position. Its upper word is taken relative to the nearest quarter turn, which leaves an angle of at most pi/4
// (cut to 2^-32 turns, 1.5e-9): cos and sin are off by at most 1.73 times 2^-24 (gkv_rotary_series.h), where 64 bits rounded once would be by
// 0.5, and a factor's product is rounded once more. Elements of 16 bits do not show it (their own rounding is 2^-8 or 2^-11); with fp32 ones it
// is the larger part of a rotation's error.
__device__ __forceinline__ float2 rotary_cos_sin(uint64_t turns, int32_t pos, float factor, float sign) {
    const uint32_t phase = (uint32_t)((turns * (uint64_t)(int64_t)pos) >> 32);
    const uint32_t quarter = (phase + (1u << 29)) >> 30;
    float c, s;
    small_cos_sin((int32_t)(phase - (quarter << 30)), &c, &s);
    const float cs = quarter & 1 ? s : c, sn = quarter & 1 ? c : s;
    const uint32_t minus_c = ((quarter + 1) & 2) << 30, minus_s = (quarter & 2) << 30;
    return make_float2(__uint_as_float(__float_as_uint(cs) ^ minus_c) * factor, __uint_as_float(__float_as_uint(sn) ^ minus_s) * (factor * sign));
}
// (a, b) turned by it, in 32 bits.
__device__ __forceinline__ float2 rotary_turn(float a, float b, float c, float s) {
    return make_float2(__fmaf_rn(a, c, -__fmul_rn(b, s)), __fmaf_rn(b, c, __fmul_rn(a, s)));
}


// How a warp turns rows of 128 elements in an attention kernel: word by word (two bf16 elements), lane l two words of every row. Halves: words
// word_a and word_b have the two sides of two pairs; the words behind the pairs go, two by two, to the lanes that have none. Neighbours: each of
// words l and l + 32 is a pair. Pairs an odd number of elements apart: single elements, pairs l and l + 32 (or what lies behind them).
// Without a rotation (no turns) every word is copied.
struct HeadTurn {
    struct Words { uint32_t a, b; };
    struct Angles { float2 a, b; };                        // cos and sin of the lane's two pairs
    int lane, half, word_a, word_b;
    bool interleaved, single, sides;
    uint64_t turns_a, turns_b;
    float factor;

    __device__ __forceinline__ HeadTurn(const RotaryView& v, int lane_) : lane(lane_), half(v.half), interleaved(v.interleaved != 0), factor(v.factor) {
        single = !interleaved && half % 2 != 0;
        sides = !interleaved && 2 * lane < half;
        word_a = interleaved || sides ? lane : 2 * lane;
        word_b = interleaved ? lane + 32 : sides ? lane + half / 2 : 2 * lane + 1;
        const bool own = interleaved || single;            // pairs l and l + 32; else, of words of first sides, 2l and 2l + 1
        const int pair_a = own ? lane : 2 * lane, pair_b = own ? lane + 32 : 2 * lane + 1;
        turns_a = pair_a < half ? v.turns[pair_a] : 0;
        turns_b = pair_b < half ? v.turns[pair_b] : 0;
    }
    __device__ __forceinline__ Angles angles(int32_t pos) const {
        return Angles{rotary_cos_sin(turns_a, pos, factor, 1.f), rotary_cos_sin(turns_b, pos, factor, 1.f)};
    }
    __device__ __forceinline__ int first_of(int i) const { return i < half ? i : 2 * i; }
    __device__ __forceinline__ int second_of(int i) const { return i < half ? i + half : 2 * i + 1; }
    __device__ __forceinline__ Words load(const __nv_bfloat16* x) const {
        if (!single) return Words{reinterpret_cast<const uint32_t*>(x)[word_a], reinterpret_cast<const uint32_t*>(x)[word_b]};
        const uint16_t* e = reinterpret_cast<const uint16_t*>(x);
        return Words{(uint32_t)e[first_of(lane)] | (uint32_t)e[second_of(lane)] << 16,
                     (uint32_t)e[first_of(lane + 32)] | (uint32_t)e[second_of(lane + 32)] << 16};
    }
    static __device__ __forceinline__ float lo(uint32_t x) { return __uint_as_float(x << 16); }
    static __device__ __forceinline__ float hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
    static __device__ __forceinline__ uint32_t pair(uint32_t w, float2 cs, bool turns) {
        const float2 r = rotary_turn(lo(w), hi(w), cs.x, cs.y);
        return turns ? pack_bf16x2(r.x, r.y) : w;
    }
    // The lane's words of a row, turned and rounded, into y (16-byte aligned).
    __device__ __forceinline__ void put(__nv_bfloat16* y, Words x, const Angles& g) const {
        if (!interleaved && !single) {
            const float2 r = rotary_turn(lo(x.a), lo(x.b), g.a.x, g.a.y), t = rotary_turn(hi(x.a), hi(x.b), g.b.x, g.b.y);
            reinterpret_cast<uint32_t*>(y)[word_a] = sides ? pack_bf16x2(r.x, t.x) : x.a;
            reinterpret_cast<uint32_t*>(y)[word_b] = sides ? pack_bf16x2(r.y, t.y) : x.b;
            return;
        }
        const uint32_t a = pair(x.a, g.a, lane < half), b = pair(x.b, g.b, lane + 32 < half);
        if (!single) {
            reinterpret_cast<uint32_t*>(y)[word_a] = a;
            reinterpret_cast<uint32_t*>(y)[word_b] = b;
        } else {
            uint16_t* e = reinterpret_cast<uint16_t*>(y);
            e[first_of(lane)] = (uint16_t)a;
            e[second_of(lane)] = (uint16_t)(a >> 16);
            e[first_of(lane + 32)] = (uint16_t)b;
            e[second_of(lane + 32)] = (uint16_t)(b >> 16);
        }
    }
};

}  // namespace gkv
