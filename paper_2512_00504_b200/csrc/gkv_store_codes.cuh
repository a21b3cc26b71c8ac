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
#include "gkv_store_rows.h"

namespace gkv {

template <int F> struct StoreFormat;
template <> struct StoreFormat<GKV_STORE_BF16> { static constexpr int kRow = 256, kScales = 0; };
template <> struct StoreFormat<GKV_STORE_E4M3> { static constexpr int kRow = 128, kScales = 1; };
template <> struct StoreFormat<GKV_STORE_INT8> { static constexpr int kRow = 128, kScales = 1; };
template <> struct StoreFormat<GKV_STORE_INT4> { static constexpr int kRow = 64, kScales = 4; };

__device__ __forceinline__ float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

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

// bf16 bits of the scale of a group whose largest magnitude has the bf16 bits `a`, and what elements are multiplied by (0 where
// the group is not finite: its codes do not matter, its scale is NaN).
__device__ __forceinline__ uint32_t e4m3_scale(uint32_t a, float* inv) {
    // a = m 2^E, 1 <= m < 2, against 448 = 1.75 * 2^8: e = E - 8, one more above 1.75 (mantissa bits 1.1100000b = 0x60)
    const int e = max((int)(a >> 7) - 127 - 8 + ((a & 0x7fu) > 0x60u ? 1 : 0), -126);
    const bool fine = a < 0x7f80u;
    *inv = fine ? __uint_as_float((uint32_t)(127 - e) << 23) : 0.f;        // exact: e is in -126 .. 120
    return fine ? (uint32_t)(e + 127) << 7 : 0x7fc0u;
}
// a / levels rounded to bf16, by a multiplication: with 8 significant bits in a and 3 or 7 in `levels` the quotient is at least
// 2^-16 of itself away from where the rounding changes, and the product is within 2^-23.
__device__ __forceinline__ uint32_t int_scale(uint32_t a, float one_over_levels, float* inv) {
    const float s = fmaxf(__bfloat162float(__float2bfloat16_rn(__uint_as_float(a << 16) * one_over_levels)), 0x1p-126f);
    const bool fine = a < 0x7f80u;
    *inv = fine ? __frcp_rn(s) : 0.f;
    return fine ? __float_as_uint(s) >> 16 : 0x7fc0u;
}
// x / s rounded to a whole number, ties to even, as exact arithmetic gives it, in the low bits of the result (two's complement,
// plus `add`). x has 8 significant bits and s has 8, so a quotient below 128 that is not half-way between whole numbers is at
// least 2^-10 away from half-way, and x * (1 / s) is within 2^-16 of the quotient. Adding 1.5 * 2^10 rounds it to a multiple of
// 2^-13, which puts the half-way cases exactly on half-way and moves none of the others across; going on to 1.5 * 2^23 rounds
// that to a whole number.
__device__ __forceinline__ uint2 round_quotients(float2 x, float inv, float add) {
    const float up = 12582912.f - 1536.f + add;
    const float2 r = add2(fma2(x, make_float2(inv, inv), make_float2(1536.f, 1536.f)), make_float2(up, up));
    return make_uint2(__float_as_uint(r.x), __float_as_uint(r.y));
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

// Of two pairs of bf16 numbers the larger magnitudes, with some sign; NaN if one of them is.
__device__ __forceinline__ uint32_t bf16_larger(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// The largest magnitudes among a lane's 8 elements, two 16-bit numbers still to be reduced: in 4 bits those of groups 2p (low)
// and 2p + 1 over the lanes of the same p, else two of the row over all lanes.
template <int F>
__device__ __forceinline__ uint32_t store_lane_max(uint4 x) {
    const uint32_t m = 0x7fff7fffu, a = bf16_larger(x.x, x.y), b = bf16_larger(x.z, x.w);
    if (F == GKV_STORE_INT4)   // low: groups 2p of both halves, high: 2p + 1
        return bf16_larger(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632)) & m;
    return bf16_larger(a, b) & m;
}
// bf16 bits of the scale(s) for reduced maxima (both groups' in 4 bits), and the factors of the lane's first and last 4 elements.
template <int F>
__device__ __forceinline__ uint32_t store_scale(uint32_t a, float* inv0, float* inv1) {
    if (F == GKV_STORE_INT4) {
        const uint32_t s0 = int_scale(a & 0xffffu, 1.f / 7.f, inv0), s1 = int_scale(a >> 16, 1.f / 7.f, inv1);
        return s0 | (s1 << 16);
    }
    a = max(a & 0xffffu, a >> 16);
    const uint32_t s = F == GKV_STORE_E4M3 ? e4m3_scale(a, inv0) : int_scale(a, 1.f / 127.f, inv0);
    *inv1 = *inv0;
    return s;
}
// Codes of a lane's 8 elements (for bf16 the elements themselves, else in .x and, in 8 bits, .y).
template <int F>
__device__ __forceinline__ uint4 store_codes(uint4 x, float inv0, float inv1) {
    if constexpr (F == GKV_STORE_BF16) return x;
    const float2 v[4] = {{bf16_lo(x.x), bf16_hi(x.x)}, {bf16_lo(x.y), bf16_hi(x.y)}, {bf16_lo(x.z), bf16_hi(x.z)}, {bf16_lo(x.w), bf16_hi(x.w)}};
    uint4 c = make_uint4(0u, 0u, 0u, 0u);
    if constexpr (F == GKV_STORE_E4M3) {
        float2 y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = mul2(v[i], make_float2(inv0, inv0));
        c.x = e4m3_pack4(y[0].x, y[0].y, y[1].x, y[1].y);
        c.y = e4m3_pack4(y[2].x, y[2].y, y[3].x, y[3].y);
    } else {
        uint32_t b[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint2 r = round_quotients(v[i], i < 2 ? inv0 : inv1, F == GKV_STORE_INT4 ? 8.f : 0.f);
            b[2 * i] = r.x;
            b[2 * i + 1] = r.y;
        }
        if constexpr (F == GKV_STORE_INT4) {   // the low 20 bits of the numbers are the codes alone
#pragma unroll
            for (int i = 0; i < 4; ++i) b[i] = b[2 * i] + (b[2 * i + 1] << 4);
        } else {
            c.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
        }
        c.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    }
    return c;
}
template <int F>
__device__ __forceinline__ void store_put_codes(uint8_t* row, int l, uint4 c) {
    if (F == GKV_STORE_BF16) *reinterpret_cast<uint4*>(row + 16 * l) = c;
    else if (F == GKV_STORE_INT4) *reinterpret_cast<uint32_t*>(row + 4 * l) = c.x;
    else *reinterpret_cast<uint2*>(row + 8 * l) = make_uint2(c.x, c.y);
}
// Quantise and store one row (the copy kernel does several at once). All 32 lanes, both half warps with a row of their own.
template <int F>
__device__ __forceinline__ void store_put_row(uint8_t* row, __nv_bfloat16* scale, int l, uint4 x) {
    float inv0 = 1.f, inv1 = 1.f;
    if (F != GKV_STORE_BF16) {
        uint32_t a = store_lane_max<F>(x);
#pragma unroll
        for (int o = 8; o >= (F == GKV_STORE_INT4 ? 2 : 1); o >>= 1) a = __vmaxu2(a, __shfl_xor_sync(0xffffffffu, a, o));
        const uint32_t s = store_scale<F>(a, &inv0, &inv1);
        if (F == GKV_STORE_INT4) { if (l < 2) reinterpret_cast<uint32_t*>(scale)[l] = s; }
        else if (l == 0) *reinterpret_cast<uint16_t*>(scale) = (uint16_t)s;
    }
    store_put_codes<F>(row, l, store_codes<F>(x, inv0, inv1));
}

// Scales of a run of R rows (1, 2, 4 or 8; half a warp, lane l of 16 with 8 elements of each): what store_scale gives for row l / (16 / R), in
// 4 bits for groups 2j and 2j + 1 with j = l & 1.
template <int F, int R>
__device__ __forceinline__ uint32_t store_run_scales(const uint4 (&v)[R], int l, float* inv0, float* inv1) {
    // Maxima of the rows, reduced and handed out at once: a lane gives away half of what it holds at every step
    // (7 exchanges for 8 rows instead of 3 or 4 for each), until it has the row of its scale.
    uint32_t a[R];
#pragma unroll
    for (int i = 0; i < R; ++i) a[i] = store_lane_max<F>(v[i]);
#pragma unroll
    for (int o = 8, n = R / 2; o >= 2; o >>= 1, n >>= 1) {
        const bool upper = (l & o) != 0;
        if (n == 0) a[0] = __vmaxu2(a[0], __shfl_xor_sync(0xffffffffu, a[0], o));
#pragma unroll
        for (int i = 0; i < R / 2; ++i)
            if (i < n) {
                const uint32_t keep = upper ? a[i + n] : a[i], give = upper ? a[i] : a[i + n];
                a[i] = __vmaxu2(keep, __shfl_xor_sync(0xffffffffu, give, o));
            }
    }
    if (F != GKV_STORE_INT4) a[0] = __vmaxu2(a[0], __shfl_xor_sync(0xffffffffu, a[0], 1));
    return store_scale<F>(a[0], inv0, inv1);
}

template <int F>
__device__ __forceinline__ uint4 store_get_codes(const uint8_t* row, int l) {
    if (F == GKV_STORE_BF16) return *reinterpret_cast<const uint4*>(row + 16 * l);
    uint4 c = make_uint4(0u, 0u, 0u, 0u);
    if (F == GKV_STORE_INT4) c.x = *reinterpret_cast<const uint32_t*>(row + 4 * l);
    else { const uint2 d = *reinterpret_cast<const uint2*>(row + 8 * l); c.x = d.x; c.y = d.y; }
    return c;
}
// The 8 bf16 elements that a lane's codes and scale(s) stand for.
template <int F>
__device__ __forceinline__ uint4 store_decode(uint4 c, uint32_t sc) {
    if (F == GKV_STORE_BF16) return c;
    if constexpr (F == GKV_STORE_INT4) {
        // 128 + u of two codes u = c + 8 in bf16, minus 136, times the scale: exact but for the product, which is rounded once.
        uint32_t y[4];
        const uint32_t next = c.x >> 4, s0 = __byte_perm(sc, 0u, 0x1010), s1 = __byte_perm(sc, 0u, 0x3232);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = (__byte_perm(c.x, next, i | (4 + i) << 8) & 0x000f000fu) | 0x43004300u;
            asm("{ .reg .b32 t; sub.rn.bf16x2 t, %1, %2; mul.rn.bf16x2 %0, t, %3; }" : "=r"(y[i]) : "r"(x), "r"(0x43084308u), "r"(i < 2 ? s0 : s1));
        }
        return make_uint4(y[0], y[1], y[2], y[3]);
    }
    float v[8];
    const float s = bf16_lo(sc);
    if (F == GKV_STORE_E4M3) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = i < 2 ? c.x : c.y;
            const uint32_t h = e4m3x2_to_f16x2((uint16_t)(w >> (16 * (i & 1))));
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
            v[2 * i] = f.x * s; v[2 * i + 1] = f.y * s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)((i < 4 ? c.x : c.y) >> (8 * (i & 3))) * s;
    }
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}

}  // namespace gkv
