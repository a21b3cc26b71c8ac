// Row formats of the key/value stores: how half a warp quantises and reads back one 128-element row.
//
// Lane l of 16 owns 8 elements of a row in every format, so that one lane's codes are one aligned store and the 16 lanes'
// stores cover the row without gaps:
//   bf16, 8-bit formats   elements 8l .. 8l + 7
//   int4                  l = 2q' + p with q' = l >> 1 = q, p = l & 1: elements 64p + 4q .. + 3 (group 2p) and
//                         64p + 32 + 4q .. + 3 (group 2p + 1), the 16-bit words 4q + 2p and 4q + 2p + 1 of the row
#pragma once

#include <cuda_fp16.h>

#include "gkv_common.cuh"
#include "gkv_internal.h"

namespace gkv {

template <int F> struct StoreFormat;
template <> struct StoreFormat<GKV_STORE_BF16> { static constexpr int kRow = 256, kScales = 0; };
template <> struct StoreFormat<GKV_STORE_E4M3> { static constexpr int kRow = 128, kScales = 1; };
template <> struct StoreFormat<GKV_STORE_INT8> { static constexpr int kRow = 128, kScales = 1; };
template <> struct StoreFormat<GKV_STORE_INT4> { static constexpr int kRow = 64, kScales = 4; };

__device__ __forceinline__ float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
__device__ __forceinline__ float bf16_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// The 8 bf16 elements lane l owns of a contiguous row (16-byte aligned).
template <int F>
__device__ __forceinline__ uint4 store_load_source(const __nv_bfloat16* row, int l) {
    if (F == GKV_STORE_INT4) {
        const __nv_bfloat16* x = row + 64 * (l & 1) + 4 * (l >> 1);
        const uint2 a = *reinterpret_cast<const uint2*>(x), b = *reinterpret_cast<const uint2*>(x + 32);
        return make_uint4(a.x, a.y, b.x, b.y);
    }
    return *reinterpret_cast<const uint4*>(row + 8 * l);
}
template <int F>
__device__ __forceinline__ void store_put_target(__nv_bfloat16* row, int l, uint4 v) {
    if (F == GKV_STORE_INT4) {
        __nv_bfloat16* x = row + 64 * (l & 1) + 4 * (l >> 1);
        *reinterpret_cast<uint2*>(x) = make_uint2(v.x, v.y);
        *reinterpret_cast<uint2*>(x + 32) = make_uint2(v.z, v.w);
    } else {
        *reinterpret_cast<uint4*>(row + 8 * l) = v;
    }
}

// Largest magnitude among the elements of two packed bf16 words, as bits: the order of magnitudes is that of their bits, with
// infinity above every number and NaN above infinity, so one integer maximum also carries "not finite".
__device__ __forceinline__ uint32_t bf16_absmax(uint32_t a, uint32_t b) {
    const uint32_t x = __vmaxu2(a & 0x7fff7fffu, b & 0x7fff7fffu);
    return max(x & 0xffffu, x >> 16);
}

// bf16 bits of the scale of a group whose largest magnitude has the bf16 bits `a`, and what elements are multiplied by.
__device__ __forceinline__ uint16_t e4m3_scale(uint32_t a, float* inv) {
    if (a >= 0x7f80u) { *inv = 0.f; return 0x7fc0u; }
    // a = m 2^E, 1 <= m < 2, against 448 = 1.75 * 2^8: e = E - 8, one more above 1.75 (mantissa bits 1.1100000b = 0x60)
    int e = (int)(a >> 7) - 127 - 8 + ((a & 0x7fu) > 0x60u ? 1 : 0);
    e = max(e, -126);
    *inv = __uint_as_float((uint32_t)(127 - e) << 23);        // exact: e is in -126 .. 120
    return (uint16_t)((e + 127) << 7);
}
__device__ __forceinline__ uint16_t int_scale(uint32_t a, float levels, float* inv) {
    if (a >= 0x7f80u) { *inv = 0.f; return 0x7fc0u; }
    const float s = fmaxf(__bfloat162float(__float2bfloat16_rn(__fdiv_rn(__uint_as_float(a << 16), levels))), 0x1p-126f);
    *inv = __frcp_rn(s);
    return (uint16_t)(__float_as_uint(s) >> 16);
}
// x / s rounded to a whole number, ties to even, as exact arithmetic gives it. x has 8 significant bits and s has 8, so a
// quotient below 128 that is not half-way between whole numbers is at least 2^-10 away from half-way, and x * (1 / s) is within
// 2^-16 of the quotient: rounding it to a multiple of 2^-13 first (adding and taking off 1.5 * 2^10) puts the half-way cases
// exactly on half-way and moves none of the others across.
__device__ __forceinline__ float round_quotient(float x, float inv) {
    const float y = __fadd_rn(__fadd_rn(__fmul_rn(x, inv), 1536.f), -1536.f);
    return rintf(y);
}

__device__ __forceinline__ uint32_t e4m3_pack4(float a, float b, float c, float d) {
    uint16_t lo, hi;   // {second operand low}
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | ((uint32_t)hi << 16);
}
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint16_t x) {
    uint32_t d;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(d) : "h"(x));
    return d;
}

template <int L>   // over the 16 lanes of a half warp (L = 16) or over those with the same lowest bit (L = 8)
__device__ __forceinline__ uint32_t half_warp_max(uint32_t a) {
#pragma unroll
    for (int o = 8; o >= (L == 16 ? 1 : 2); o >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
    return a;
}

// Lane l of a half warp quantises its 8 elements of a row into `data` (the row's codes) and the row's scales. All 32 lanes
// call it (both half warps, each with its own row); `write` = 0 computes without storing.
template <int F>
__device__ __forceinline__ void store_put_row(uint8_t* data, __nv_bfloat16* scale, int l, uint4 x, bool write) {
    if (F == GKV_STORE_BF16) {
        if (write) *reinterpret_cast<uint4*>(data + 16 * l) = x;
        return;
    }
    float v[8] = {bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y), bf16_lo(x.z), bf16_hi(x.z), bf16_lo(x.w), bf16_hi(x.w)};
    uint16_t* sc = reinterpret_cast<uint16_t*>(scale);
    float inv;
    if (F == GKV_STORE_INT4) {
        const uint32_t a0 = half_warp_max<8>(bf16_absmax(x.x, x.y)), a1 = half_warp_max<8>(bf16_absmax(x.z, x.w));
        float inv1;
        const uint16_t s0 = int_scale(a0, 7.f, &inv), s1 = int_scale(a1, 7.f, &inv1);
        uint32_t c = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float f = i < 4 ? inv : inv1;
            const float q = f == 0.f ? 0.f : round_quotient(v[i], f);
            c |= (uint32_t)((int)q + 8) << (4 * i);
        }
        if (write) {
            *reinterpret_cast<uint32_t*>(data + 4 * l) = c;
            if (l < 2) *reinterpret_cast<uint32_t*>(sc + 2 * l) = (uint32_t)s0 | ((uint32_t)s1 << 16);
        }
        return;
    }
    const uint32_t a = half_warp_max<16>(max(bf16_absmax(x.x, x.y), bf16_absmax(x.z, x.w)));
    const uint16_t s = F == GKV_STORE_E4M3 ? e4m3_scale(a, &inv) : int_scale(a, 127.f, &inv);
    uint2 c;
    if (F == GKV_STORE_E4M3) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = inv == 0.f ? 0.f : v[i] * inv;
        c.x = e4m3_pack4(v[0], v[1], v[2], v[3]);
        c.y = e4m3_pack4(v[4], v[5], v[6], v[7]);
    } else {
        uint32_t b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = (uint32_t)(int)(inv == 0.f ? 0.f : round_quotient(v[i], inv));
        c.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
        c.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
    }
    if (write) {
        *reinterpret_cast<uint2*>(data + 8 * l) = c;
        if (l == 0) sc[0] = s;
    }
}

// The raw codes and scales lane l needs of a row, and the 8 bf16 elements they stand for.
template <int F> struct StoreRaw { uint4 c; uint32_t s; };
template <int F>
__device__ __forceinline__ StoreRaw<F> store_get_raw(const uint8_t* data, const __nv_bfloat16* scale, int l) {
    StoreRaw<F> r;
    r.s = 0;
    if (F == GKV_STORE_BF16) r.c = *reinterpret_cast<const uint4*>(data + 16 * l);
    else if (F == GKV_STORE_INT4) {
        r.c.x = *reinterpret_cast<const uint32_t*>(data + 4 * l);
        r.s = *reinterpret_cast<const uint32_t*>(scale + 2 * (l & 1));
    } else {
        const uint2 c = *reinterpret_cast<const uint2*>(data + 8 * l);
        r.c.x = c.x; r.c.y = c.y;
        r.s = *reinterpret_cast<const uint16_t*>(scale);
    }
    return r;
}
template <int F>
__device__ __forceinline__ uint4 store_decode_raw(const StoreRaw<F>& r) {
    if (F == GKV_STORE_BF16) return r.c;
    float v[8];
    if (F == GKV_STORE_INT4) {
        const float s0 = bf16_lo(r.s), s1 = bf16_hi(r.s);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)((int)((r.c.x >> (4 * i)) & 15u) - 8) * (i < 4 ? s0 : s1);
    } else {
        const float s = bf16_lo(r.s);
        if (F == GKV_STORE_E4M3) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t w = i < 2 ? r.c.x : r.c.y;
                const uint32_t h = e4m3x2_to_f16x2((uint16_t)(w >> (16 * (i & 1))));
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
                v[2 * i] = f.x * s; v[2 * i + 1] = f.y * s;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)((i < 4 ? r.c.x : r.c.y) >> (8 * (i & 3))) * s;
        }
    }
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}

}  // namespace gkv
