// What the attention kernels over own rows share: the registers and products of a tile, a warp's running softmax, dealing out pieces
// by lengths, and the end of a CTA, where its warps' results and then its unit's pieces are joined.
#pragma once

#include "gkv_store_codes.cuh"

namespace gkv {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kTile = 16;            // keys of a tile
// How far weights (relative to the running maximum, summed over a warp's lane and step) may go before the maximum is raised: the
// range of fp16 allows no more for scaled rows, and with bf16 ones a larger limit (2^60) would gain nothing and let the sums of
// values near the end of the range overflow.
constexpr float kLagLimit = 256.f;
// state word of a unit's first partial result
constexpr float kPieceOk = 0.f, kPieceNoFit = 1.f, kPieceLeftOut = 2.f;
constexpr float kLift = 6.f;         // the weights of scaled rows are lifted by 2^6: at most 2^14, subnormal below 2^-20
constexpr float kLiftFactor = 64.f;
constexpr float kScaleSpan = 112.f;

// ---- loads of codes. The store may have been written earlier in the same kernel (the new row): no read-only path.
__device__ __forceinline__ uint4 ld16(const void* a) {
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(a) : "memory");
    return r;
}
__device__ __forceinline__ uint2 ld8(const void* a) {
    uint2 r;
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(a) : "memory");
    return r;
}
__device__ __forceinline__ uint32_t ld2(const void* a) {
    uint16_t r;
    asm volatile("ld.global.u16 %0, [%1];" : "=h"(r) : "l"(a) : "memory");
    return r;
}

__device__ __forceinline__ void mma_f16_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The same with zeros for C, which takes no registers and no moves.
template <int F>
__device__ __forceinline__ void mma_row_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (F == GKV_STORE_BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                     : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                     : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
template <int F>
__device__ __forceinline__ void mma_row(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (F == GKV_STORE_BF16) mma_bf16_16816(d, a, b0, b1);
    else mma_f16_16816(d, a, b0, b1);
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
// The weights of the second product are rounded to the type that its rows have, which is what the product takes: bf16 with bf16 rows (8 bits: outputs
// are off by 1.9e-3 to 2.3e-3, against 1.65e-3 with weights of 32 bits, which is the outputs' own rounding to bf16), fp16 with scaled ones, times V's
// scale (11 bits: 1.68e-3). The sums that they are divided by are of the weights before that, in 32 bits.
template <int F>
__device__ __forceinline__ uint32_t pack_weights(float lo, float hi) { return F == GKV_STORE_BF16 ? pack_bf16x2(lo, hi) : pack_f16x2(lo, hi); }

__device__ __forceinline__ uint32_t hsub2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ float fast_log2(float x) {   // absolute error 2^-22; only places a reference
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Four 8-bit codes -> two fp16 pairs (codes 0, 1 and 2, 3).
template <int F>
__device__ __forceinline__ void unpack8(uint32_t w, uint32_t& lo, uint32_t& hi) {
    if (F == GKV_STORE_E4M3) {
        lo = e4m3x2_to_f16x2((uint16_t)w);
        hi = e4m3x2_to_f16x2((uint16_t)(w >> 16));
    } else {   // c + 128 in the low bits of an fp16 1024 + ..., minus 1152
        w ^= 0x80808080u;
        lo = hsub2(__byte_perm(w, 0x64646464u, 0x4140), 0x64806480u);
        hi = hsub2(__byte_perm(w, 0x64646464u, 0x4342), 0x64806480u);
    }
}
// Two bytes of nibbles under the exponent of 1024, x = 1024 + u0 + 16 u1 in both halves (u = c + 8) -> the fp16 pairs c0 and c1,
// exactly. (Integers put into a mantissa under a fixed exponent instead of being converted: for 4-bit weights in fp16 published by
// Kim et al. 2022, arXiv 2211.10017.) Without its low nibble x is y = 1024 + 16 u1, so c1 = y / 16 - 72; without the high one it is 1024 + u0. Two
// instructions for the logic unit and two for the fp32 and half-precision pipe, which are about equally busy then (c0 as
// (x - 16 c1) - 1160 puts three on the latter: 131071 keys take 80 us instead of 78). (Leaving the offset 8 in and taking it
// off the sums would save the latter, but costs precision: as 1024 + u in the fp32 sums, as subnormals u 2^-24 where the
// products are aligned.)
__device__ __forceinline__ void unpack4(uint32_t x, uint32_t& c0, uint32_t& c1) {
    c1 = hfma2(x & 0xfff0fff0u, 0x2c002c00u, 0xd480d480u);
    c0 = hsub2(x & 0xff0fff0fu, 0x64086408u);
}

// Registers of one 16-key tile. K: this lane's pieces of rows r = lane / 4 and r + 8. V: its pieces of keys 2j, 2j + 1, 2j + 8,
// 2j + 9, j = lane & 3.
template <int F> struct TileK;
template <> struct TileK<GKV_STORE_BF16> { uint4 d[2][4]; };
template <> struct TileK<GKV_STORE_E4M3> { uint4 d[2][2]; uint32_t s[2]; };
template <> struct TileK<GKV_STORE_INT8> { uint4 d[2][2]; uint32_t s[2]; };
template <> struct TileK<GKV_STORE_INT4> { uint4 d[2][1]; uint2 s[2]; };
template <int F> struct TileV;
template <> struct TileV<GKV_STORE_BF16> { uint4 d[4][2]; };
template <> struct TileV<GKV_STORE_E4M3> { uint4 d[4]; uint32_t s[2]; };
template <> struct TileV<GKV_STORE_INT8> { uint4 d[4]; uint32_t s[2]; };
template <> struct TileV<GKV_STORE_INT4> { uint2 d[4]; uint2 s[2]; };

// Where a lane's pieces of a tile begin: offsets from the unit's rows (below 2^32: a unit has at most 2^24 rows of 256 bytes);
// everything of a tile is at constant distances.
template <int F>
struct TilePtrs {
    using Fm = StoreFormat<F>;
    const uint8_t *kb, *vb;
    const uint8_t *ksb, *vsb;
    uint32_t k, v, s;
    __device__ __forceinline__ void set(int key0, int lane) {
        const int q = lane >> 2, j = lane & 3;
        k = (uint32_t)(key0 + q) * Fm::kRow + j * 16;
        v = (uint32_t)(key0 + 2 * j) * Fm::kRow + q * (F == GKV_STORE_INT4 ? 8 : 16);
        s = (uint32_t)(key0 + q) * (2 * Fm::kScales);
    }
    __device__ __forceinline__ void advance(int keys) { k += keys * Fm::kRow; v += keys * Fm::kRow; s += keys * (2 * Fm::kScales); }
};
// Rows from `left` on (counted from the tile's first) are not loaded: zeros stand for them, so that whatever lies there cannot
// reach the sums. WHOLE: all 16 exist.
template <int F, bool WHOLE>
__device__ __forceinline__ void load_k(TileK<F>& t, const TilePtrs<F>& p, int left, int lane) {
    constexpr int kPieces = F == GKV_STORE_BF16 ? 4 : F == GKV_STORE_INT4 ? 1 : 2;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
        const bool in = WHOLE || (lane >> 2) + 8 * hf < left;
        const uint8_t* row = p.kb + p.k + 8 * hf * StoreFormat<F>::kRow;
        const uint8_t* sc = p.ksb + p.s + 8 * hf * (2 * StoreFormat<F>::kScales);
#pragma unroll
        for (int c = 0; c < kPieces; ++c) t.d[hf][c] = in ? ld16(row + c * 64) : make_uint4(0u, 0u, 0u, 0u);
        if constexpr (F == GKV_STORE_INT4) t.s[hf] = in ? ld8(sc) : make_uint2(0u, 0u);
        else if constexpr (F != GKV_STORE_BF16) t.s[hf] = in ? ld2(sc) : 0u;
    }
}
template <int F, bool WHOLE>
__device__ __forceinline__ void load_v(TileV<F>& t, const TilePtrs<F>& p, int left, int lane) {
    const int j = lane & 3;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int key = (i & 1) + 8 * (i >> 1);
        const bool in = WHOLE || 2 * j + key < left;
        const uint8_t* row = p.vb + p.v + key * StoreFormat<F>::kRow;
        if constexpr (F == GKV_STORE_BF16) {
            t.d[i][0] = in ? ld16(row) : make_uint4(0u, 0u, 0u, 0u);
            t.d[i][1] = in ? ld16(row + 128) : make_uint4(0u, 0u, 0u, 0u);
        } else if constexpr (F == GKV_STORE_INT4) {
            t.d[i] = in ? ld8(row) : make_uint2(0u, 0u);
        } else {
            t.d[i] = in ? ld16(row) : make_uint4(0u, 0u, 0u, 0u);
        }
    }
    // scales by key as the logits are held: rows r, r + 8
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
        const bool in = WHOLE || (lane >> 2) + 8 * hf < left;
        const uint8_t* sc = p.vsb + p.s + 8 * hf * (2 * StoreFormat<F>::kScales);
        if constexpr (F == GKV_STORE_INT4) t.s[hf] = in ? ld8(sc) : make_uint2(0u, 0u);
        else if constexpr (F != GKV_STORE_BF16) t.s[hf] = in ? ld2(sc) : 0u;
    }
}
// `left` of a tile's keys exist (the same number for the whole warp; none or fewer: no loads).
template <int F>
__device__ __forceinline__ void load_tile_k(TileK<F>& t, const TilePtrs<F>& p, int left, int lane) {
    if (left >= kTile) load_k<F, true>(t, p, 0, lane);
    else load_k<F, false>(t, p, left, lane);
}
template <int F>
__device__ __forceinline__ void load_tile_v(TileV<F>& t, const TilePtrs<F>& p, int left, int lane) {
    if (left >= kTile) load_v<F, true>(t, p, 0, lane);
    else load_v<F, false>(t, p, left, lane);
}

// Logits of a tile in log2 units: z[0], z[1] = key r and heads h0, h0 + 1; z[2], z[3] = key r + 8. f0, f1: factors of the heads.
template <int F>
__device__ __forceinline__ void tile_logits(const TileK<F>& t, const uint32_t (&qf)[8][2], float f0, float f1, float (&z)[4]) {
    if constexpr (F == GKV_STORE_INT4) {
        float2 y0, y1;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float acc[4];
#pragma unroll
            for (int k = 0; k < 2; ++k) {       // the 16-bit words 2j and 2j + 1 of the group: elements 0, 2 and 1, 3 of each
                uint32_t a[4];
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const uint4 d = t.d[hf][0];
                    const uint32_t w = k == 0 ? (g < 2 ? d.x : d.y) : (g < 2 ? d.z : d.w);
                    unpack4(__byte_perm(w, 0x64646464u, (g & 1) ? 0x4342 : 0x4140), a[hf], a[hf + 2]);
                }
                if (k == 0) mma_row_first<F>(acc, a, qf[2 * g + k][0], qf[2 * g + k][1]);
                else mma_row<F>(acc, a, qf[2 * g + k][0], qf[2 * g + k][1]);
            }
            const uint32_t w0 = g < 2 ? t.s[0].x : t.s[0].y, w1 = g < 2 ? t.s[1].x : t.s[1].y;
            const float s0 = (g & 1) ? bf16_hi(w0) : bf16_lo(w0), s1 = (g & 1) ? bf16_hi(w1) : bf16_lo(w1);
            const float2 a0 = make_float2(acc[0], acc[1]), a1 = make_float2(acc[2], acc[3]), s00 = make_float2(s0, s0), s11 = make_float2(s1, s1);
            y0 = g == 0 ? mul2(a0, s00) : fma2(a0, s00, y0);
            y1 = g == 0 ? mul2(a1, s11) : fma2(a1, s11, y1);
        }
        y0 = mul2(y0, make_float2(f0, f1));
        y1 = mul2(y1, make_float2(f0, f1));
        z[0] = y0.x; z[1] = y0.y; z[2] = y1.x; z[3] = y1.y;
    } else {
        float sa[4], sb[4];   // two accumulators: half the dependent chain
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            uint32_t a[4];
            if constexpr (F == GKV_STORE_BF16) {
                const uint4 u = t.d[0][ks >> 1], w = t.d[1][ks >> 1];
                a[0] = (ks & 1) ? u.z : u.x; a[1] = (ks & 1) ? w.z : w.x;
                a[2] = (ks & 1) ? u.w : u.y; a[3] = (ks & 1) ? w.w : w.y;
            } else {
                const uint4 u = t.d[0][ks >> 2], w = t.d[1][ks >> 2];
                const int i = ks & 3;
                unpack8<F>(i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w, a[0], a[2]);
                unpack8<F>(i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w, a[1], a[3]);
            }
            if (ks < 2) mma_row_first<F>((ks & 1) ? sb : sa, a, qf[ks][0], qf[ks][1]);
            else mma_row<F>((ks & 1) ? sb : sa, a, qf[ks][0], qf[ks][1]);
        }
        float e0 = f0, e1 = f1, e2 = f0, e3 = f1;
        if constexpr (F != GKV_STORE_BF16) {
            const float s0 = bf16_lo(t.s[0]), s1 = bf16_lo(t.s[1]);
            e0 *= s0; e1 *= s0; e2 *= s1; e3 *= s1;
        }
        z[0] = (sa[0] + sb[0]) * e0; z[1] = (sa[1] + sb[1]) * e1;
        z[2] = (sa[2] + sb[2]) * e2; z[3] = (sa[3] + sb[3]) * e3;
    }
}

// acc += V^T W for a tile; b0, b1: the weights as the B operand (one pair, or one for each group of head dimensions).
template <int F, int NG>
__device__ __forceinline__ void tile_values(const TileV<F>& t, const uint32_t (&b)[NG][2], float (&acc)[8][4]) {
    if constexpr (F == GKV_STORE_BF16) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                auto word = [&](int key) { const uint4 u = t.d[key][c]; return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w; };
                const uint32_t a[4] = {__byte_perm(word(0), word(1), 0x5410), __byte_perm(word(0), word(1), 0x7632),
                                       __byte_perm(word(2), word(3), 0x5410), __byte_perm(word(2), word(3), 0x7632)};
                mma_row<F>(acc[4 * c + i], a, b[0][0], b[0][1]);
            }
    } else if constexpr (F == GKV_STORE_INT4) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            auto word = [&](int key) { return g < 2 ? t.d[key].x : t.d[key].y; };
            const uint32_t x = __byte_perm(word(0), word(1), (g & 1) ? 0x7632 : 0x5410), y = __byte_perm(word(2), word(3), (g & 1) ? 0x7632 : 0x5410);
#pragma unroll
            for (int k = 0; k < 2; ++k) {       // the group's bytes: dimensions 2k (rows q) and 2k + 1 (rows q + 8)
                uint32_t a[4];
                unpack4(__byte_perm(x, 0x64646464u, k == 0 ? 0x4240 : 0x4341), a[0], a[1]);
                unpack4(__byte_perm(y, 0x64646464u, k == 0 ? 0x4240 : 0x4341), a[2], a[3]);
                mma_row<F>(acc[2 * g + k], a, b[g][0], b[g][1]);
            }
        }
    } else {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            auto word = [&](int key) { const uint4 u = t.d[key]; return w == 0 ? u.x : w == 1 ? u.y : w == 2 ? u.z : u.w; };
            uint32_t a0[4], a1[4];   // bytes 0, 1 and 2, 3 of the four keys
            unpack8<F>(__byte_perm(word(0), word(1), 0x5140), a0[0], a0[1]);
            unpack8<F>(__byte_perm(word(2), word(3), 0x5140), a0[2], a0[3]);
            unpack8<F>(__byte_perm(word(0), word(1), 0x7362), a1[0], a1[1]);
            unpack8<F>(__byte_perm(word(2), word(3), 0x7362), a1[2], a1[3]);
            mma_row<F>(acc[2 * w], a0, b[0][0], b[0][1]);
            mma_row<F>(acc[2 * w + 1], a1, b[0][0], b[0][1]);
        }
    }
}

// Head dimension of accumulator row (m-tile i, lane group q); row 8 + q holds the next one.
template <int F>
__device__ __forceinline__ int out_dim(int i, int q) {
    if (F == GKV_STORE_BF16) return 64 * (i >> 2) + 8 * q + 2 * (i & 3);
    if (F == GKV_STORE_INT4) return 32 * (i >> 1) + 4 * q + 2 * (i & 1);
    return 16 * q + 2 * i;
}
// The two pairs of elements of q that lane j has at step ks.
template <int F>
__device__ __forceinline__ void load_query(const __nv_bfloat16* row, int ks, int j, uint32_t& b0, uint32_t& b1) {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(row);
    if (F == GKV_STORE_BF16) {
        const uint2 x = *reinterpret_cast<const uint2*>(q + 32 * (ks >> 1) + 8 * j + 4 * (ks & 1));
        b0 = x.x; b1 = x.y;
    } else if (F == GKV_STORE_INT4) {
        const uint2 x = *reinterpret_cast<const uint2*>(q + 32 * (ks >> 1) + 8 * j + 4 * (ks & 1));
        b0 = __byte_perm(x.x, x.y, 0x5410); b1 = __byte_perm(x.x, x.y, 0x7632);
    } else {
        const uint2 x = *reinterpret_cast<const uint2*>(q + 64 * (ks >> 2) + 16 * j + 4 * (ks & 3));
        b0 = x.x; b1 = x.y;
    }
}
__device__ __forceinline__ uint32_t bf16x2_to_f16x2(uint32_t x, float f) { return pack_f16x2(bf16_lo(x) * f, bf16_hi(x) * f); }

// Heads as the B operand of the first product, lane (head lane / 4, j = lane & 3), as they were loaded: with 8- and 4-bit rows they
// become fp16 relative to a power of two, which goes into the factors f0, f1 of heads 2j, 2j + 1.
template <int F>
__device__ __forceinline__ void scale_queries(int lane, uint32_t (&qf)[8][2], float& f0, float& f1) {
    if constexpr (F != GKV_STORE_BF16) {
        const int j = lane & 3;
        uint32_t a = 0;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) a = max(a, bf16_absmax(qf[ks][0], qf[ks][1]));
        a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
        a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
        const int e = min(max((int)(a >> 7) - 127, -126), 126);        // exponent of the row's largest element
        const float down = __uint_as_float((uint32_t)(127 - e) << 23), up = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            qf[ks][0] = bf16x2_to_f16x2(qf[ks][0], down);
            qf[ks][1] = bf16x2_to_f16x2(qf[ks][1], down);
        }
        f0 *= __shfl_sync(0xffffffffu, up, 8 * j);
        f1 *= __shfl_sync(0xffffffffu, up, 8 * j + 4);
    }
}
// The same from the rows of a unit's heads (this lane's).
template <int F>
__device__ __forceinline__ void load_queries(const __nv_bfloat16* row, int lane, uint32_t (&qf)[8][2], float& f0, float& f1) {
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) load_query<F>(row, ks, lane & 3, qf[ks][0], qf[ks][1]);
    scale_queries<F>(lane, qf, f0, f1);
}

__device__ __forceinline__ float finite_ref(float m) { return m == -INFINITY ? 0.f : m; }
// Output and log-sum-exp from sums relative to 2^v (values) and 2^m (weights); m = -infinity and no weight: nothing to attend to.
__device__ __forceinline__ float final_value(float o, float m, float l, float v, bool fits) {
    return !fits ? NAN : m == -INFINITY && l == 0.f ? 0.f : o * (fast_exp2(v - m) / l);
}
__device__ __forceinline__ float final_lse(float m, float l, bool fits) {
    return !fits ? NAN : m == -INFINITY && l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

// Groups of head dimensions whose V rows have a scale of their own.
__host__ __device__ constexpr int value_groups(int format) { return format == GKV_STORE_INT4 ? 4 : 1; }

// A warp's running softmax and accumulators over its tiles, for heads h0 = 2 (lane & 3) and h0 + 1.
template <int F>
struct RunningRows {
    static constexpr int NG = value_groups(F);
    static constexpr bool kScaled = F != GKV_STORE_BF16;
    float m0, m1, l0, l1;           // running maxima (they may lag) and sums
    // The same maxima of z + log2(scale of V): with one scale a row in registers, with several, by group, in the warp's part of
    // s_v (they are looked at when maxima are raised, and registers are what limits the CTAs of an SM).
    float v0, v1;
    float n0, n1;                   // what logits are taken relative to: m, once that is finite
    float c0[NG], c1[NG];           // 2^(m - v + kLift), with finite m and v
    float acc[8][4];

    __device__ __forceinline__ void start(float (&s_v)[NG][8], int lane) {
        m0 = m1 = -INFINITY;
        l0 = l1 = 0.f;
        v0 = v1 = -INFINITY;
        if constexpr (NG > 1) {
            const int h0 = 2 * (lane & 3);
            if ((lane >> 2) == 0)
#pragma unroll
                for (int g = 0; g < NG; ++g) s_v[g][h0] = s_v[g][h0 + 1] = -INFINITY;
            __syncwarp();
        }
        n0 = n1 = -INFINITY;
#pragma unroll
        for (int g = 0; g < NG; ++g) c0[g] = c1[g] = 1.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
    }

    // The tile whose logits are z (log2 units; z[0], z[1]: key lane / 4, z[2], z[3]: 8 keys on): its weights as the B operand of the
    // second product. Sums follow, and where they have to be raised maxima and accumulators.
    __device__ __forceinline__ void weigh_tile(const float (&z)[4], const TileV<F>& tv, float (&s_v)[NG][8], int lane, uint32_t (&b)[NG][2]) {
        const int hq = lane >> 2, h0 = 2 * (lane & 3);
        // V scales of this lane's two keys (0 behind the end)
        float sc[2][NG];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            if constexpr (F == GKV_STORE_INT4) {
                const uint2 s = tv.s[hf];
                sc[hf][0] = bf16_lo(s.x); sc[hf][1] = bf16_hi(s.x);
                sc[hf][2] = bf16_lo(s.y); sc[hf][3] = bf16_hi(s.y);
            } else if constexpr (kScaled) {
                sc[hf][0] = bf16_lo(tv.s[hf]);
            } else {
                sc[hf][0] = 1.f;
            }
        }
        float e[4];                     // exp2(z - m)
        // A z that is far above m, or a z + log2(scale) far above v, shows in the results: they are sums of non-negative numbers
        // (at most the limit then), infinite or NaN, also at the first step, where m is -infinity.
        float total = 0.f;
        auto weigh = [&]() {
            if constexpr (NG == 1) {    // (in pairs: 128 x 8 heads of 2200 keys in 8 bits 96.5 us instead of 96.2, with shared documents 145.7 and 144.4)
                e[0] = fast_exp2(z[0] - n0); e[1] = fast_exp2(z[1] - n1);
                e[2] = fast_exp2(z[2] - n0); e[3] = fast_exp2(z[3] - n1);
            } else {
                const float2 n = make_float2(-n0, -n1), d0 = add2(make_float2(z[0], z[1]), n), d1 = add2(make_float2(z[2], z[3]), n);
                e[0] = fast_exp2(d0.x); e[1] = fast_exp2(d0.y);
                e[2] = fast_exp2(d1.x); e[3] = fast_exp2(d1.y);
            }
            total += (e[0] + e[2]) + (e[1] + e[3]);
            if constexpr (NG > 1) {
                float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {      // (e c is finite, c s need not be)
                        const float2 x = mul2(mul2(make_float2(e[2 * hf], e[2 * hf + 1]), make_float2(c0[g], c1[g])), make_float2(sc[hf][g], sc[hf][g]));
                        sum = add2(sum, x);
                        b[g][hf] = pack_weights<F>(x.x, x.y);
                    }
                total += (sum.x + sum.y) * (1.f / kLiftFactor);
            } else if constexpr (kScaled) {
                total += ((e[0] * c0[0] + e[1] * c1[0]) * sc[0][0] + (e[2] * c0[0] + e[3] * c1[0]) * sc[1][0]) * (1.f / kLiftFactor);
            }
        };
        weigh();
        const bool over = !(total <= kLagLimit);
        if (__any_sync(0xffffffffu, over)) {
            float a0 = m0, a1 = m1, b0[NG], b1[NG];
            a0 = fmaxf(a0, fmaxf(z[0], z[2]));
            a1 = fmaxf(a1, fmaxf(z[1], z[3]));
            if constexpr (kScaled) {
#pragma unroll
                for (int g = 0; g < NG; ++g) {          // fmaxf leaves out a NaN
                    const float x0 = fast_log2(sc[0][g]), x1 = fast_log2(sc[1][g]);
                    b0[g] = fmaxf(NG > 1 ? s_v[g][h0] : v0, fmaxf(z[0] + x0, z[2] + x1));
                    b1[g] = fmaxf(NG > 1 ? s_v[g][h0 + 1] : v1, fmaxf(z[1] + x0, z[3] + x1));
                }
            }
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                a0 = fmaxf(a0, __shfl_xor_sync(0xffffffffu, a0, o));
                a1 = fmaxf(a1, __shfl_xor_sync(0xffffffffu, a1, o));
                if constexpr (kScaled) {
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        b0[g] = fmaxf(b0[g], __shfl_xor_sync(0xffffffffu, b0[g], o));
                        b1[g] = fmaxf(b1[g], __shfl_xor_sync(0xffffffffu, b1[g], o));
                    }
                }
            }
            float r0 = fast_exp2(m0 - finite_ref(a0)), r1 = fast_exp2(m1 - finite_ref(a1));
            l0 *= r0;
            l1 *= r1;
            m0 = a0; m1 = a1;
            n0 = finite_ref(m0); n1 = finite_ref(m1);
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                if constexpr (kScaled) {
                    b0[g] = fmaxf(b0[g], a0 - kScaleSpan);
                    b1[g] = fmaxf(b1[g], a1 - kScaleSpan);
                    r0 = fast_exp2((NG > 1 ? s_v[g][h0] : v0) - finite_ref(b0[g]));
                    r1 = fast_exp2((NG > 1 ? s_v[g][h0 + 1] : v1) - finite_ref(b1[g]));
                    c0[g] = fast_exp2(n0 - finite_ref(b0[g]) + kLift);
                    c1[g] = fast_exp2(n1 - finite_ref(b1[g]) + kLift);
                }
#pragma unroll
                for (int i = g * (8 / NG); i < (g + 1) * (8 / NG); ++i) { acc[i][0] *= r0; acc[i][1] *= r1; acc[i][2] *= r0; acc[i][3] *= r1; }
            }
            if constexpr (NG > 1) {
                __syncwarp();           // all lanes have read them
                if (hq == 0)
#pragma unroll
                    for (int g = 0; g < NG; ++g) { s_v[g][h0] = b0[g]; s_v[g][h0 + 1] = b1[g]; }
                __syncwarp();
            } else if constexpr (kScaled) {
                v0 = b0[0]; v1 = b1[0];
            }
            weigh();
            n0 = m0; n1 = m1;           // as long as every logit was -infinity, the next step comes here again
        }
        l0 += e[0] + e[2];
        l1 += e[1] + e[3];
        if constexpr (!kScaled) {
            b[0][0] = pack_weights<F>(e[0], e[1]);
            b[0][1] = pack_weights<F>(e[2], e[3]);
        } else if constexpr (NG == 1) {
            b[0][0] = pack_weights<F>(e[0] * c0[0] * sc[0][0], e[1] * c1[0] * sc[0][0]);
            b[0][1] = pack_weights<F>(e[2] * c0[0] * sc[1][0], e[3] * c1[0] * sc[1][0]);
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) { b[g][0] = movmatrix_trans(b[g][0]); b[g][1] = movmatrix_trans(b[g][1]); }
    }
};

// What becomes of a CTA's result: it is the unit's; it goes to the workspace (kDealt: pieces go by the lengths); it is joined with
// those of the cluster's other CTAs.
enum { kWhole = 0, kPart = 1, kCluster = 2, kDealt = 3 };

// ---- pieces by length: the batch * splits places of a head go to the sequences one after the other, as many to each
// as its tiles need. Every warp works it out for itself; the merge does so again.
template <class P>
__device__ __forceinline__ int own_tiles_of(const P& p, int seq) {
    if (seq >= p.batch) return 0;
    const int len = p.len[seq], n = p.k_new ? 1 : 0;
    return len < 0 || len > p.capacity - n ? 0 : (len + n + kTile - 1) / kTile;
}
__device__ __forceinline__ int pieces_of(int tiles, int per) { return (int)(((unsigned)tiles + (unsigned)per - 1) / (unsigned)per); }
// Pieces of sequences 0 .. seqs - 1, `per` tiles each. t0: tiles of sequence `lane`.
template <class P>
__device__ __forceinline__ int pieces_before(const P& p, int seqs, int per, int lane, int t0) {
    int c = lane < seqs ? pieces_of(t0, per) : 0;
    for (int b = lane + 32; b < seqs; b += 32) c += pieces_of(own_tiles_of(p, b), per);
    return (int)__reduce_add_sync(0xffffffffu, (unsigned)c);
}
// Tiles of a piece: 8 (two turns of the four warps) or more, no unit in more than kMaxPieces pieces, and all pieces in their
// places: the mean, or a little more until roundings fit (with (splits - 1) / splits of the places they always do).
template <class P>
__device__ __forceinline__ int store_piece_tiles(const P& p, int lane, int t0) {
    int sum = t0, most = t0;
    for (int b = lane + 32; b < p.batch; b += 32) {
        const int t = own_tiles_of(p, b);
        sum += t;
        most = max(most, t);
    }
    sum = (int)__reduce_add_sync(0xffffffffu, (unsigned)sum);
    most = (int)__reduce_max_sync(0xffffffffu, (unsigned)most);
    const int places = p.batch * p.splits;
    int per = max(max(8, pieces_of(sum, places)), pieces_of(most, kMaxPieces));
    for (int k = 0; pieces_before(p, p.batch, per, lane, t0) > places; ++k)
        per = k < 4 ? per + per / 32 + 1 : max(per, pieces_of(sum, places - p.batch));
    return per;
}

// The place of a CTA: head slowest, then the sequences' pieces one after the other. False: nobody needs it.
template <class P>
__device__ __forceinline__ bool dealt_place(const P& p, int lane, int* seq, int* head, int* split, int* splits, int* split_tiles) {
    const int places = p.batch * p.splits, t0 = own_tiles_of(p, lane);
    int b = -1, at = blockIdx.x % places;
    *head = blockIdx.x / places;
    *split_tiles = store_piece_tiles(p, lane, t0);
    while (b < p.batch) {                                // 32 sequences at a time
        const int c = pieces_of(b < 0 ? t0 : own_tiles_of(p, b + 1 + lane), *split_tiles);
        int upto = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        const unsigned past = __ballot_sync(0xffffffffu, upto > at);
        if (past) {
            const int k = __ffs(past) - 1;
            *seq = b + 1 + k;
            *split = at - __shfl_sync(0xffffffffu, upto - c, k);
            *splits = __shfl_sync(0xffffffffu, c, k);
            return true;
        }
        at -= __shfl_sync(0xffffffffu, upto, 31);
        b += 32;
    }
    return false;
}

// What a CTA's warps leave for one another, beside their accumulators.
template <int F>
struct RowsShared {
    static constexpr int NG = value_groups(F);
    float m[kWarps][8], l[kWarps][8], v[kWarps][NG][8], wgt[kWarps][NG][8], fin[2 + NG][8];
    float cl[kMaxCluster][NG][8], norm[2 + NG][8];
};

// Joins the warps' results and, as MODE says, writes the unit's outputs or its partial result, or joins the cluster's. s_o: room
// for the accumulators (nothing else is read from it any more by any warp when it comes here). `unit`: seq and head; `fits`: false
// where the length does not fit, which shows as NaN.
template <int F, int MODE, class P>
__device__ __forceinline__ void finish_rows(const P& p, RunningRows<F>& r, RowsShared<F>& sh, float (*s_o)[kHeadDim * 8], int seq,
                                            int head, int split, bool fits, int warp, int lane) {
    constexpr int NG = value_groups(F);
    constexpr bool kScaled = F != GKV_STORE_BF16;
    const int hq = lane >> 2, h0 = 2 * (lane & 3);
    // ---- the warps' results: statistics, then the accumulators weighted to a common maximum
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
        r.l0 += __shfl_xor_sync(0xffffffffu, r.l0, o);
        r.l1 += __shfl_xor_sync(0xffffffffu, r.l1, o);
    }
    if (hq == 0) {
        sh.m[warp][h0] = r.m0; sh.m[warp][h0 + 1] = r.m1;
        sh.l[warp][h0] = r.l0; sh.l[warp][h0 + 1] = r.l1;
        if constexpr (NG > 1) {
#pragma unroll
            for (int g = 0; g < NG; ++g) { sh.v[warp][g][h0] -= kLift; sh.v[warp][g][h0 + 1] -= kLift; }
        } else {
            sh.v[warp][0][h0] = kScaled ? r.v0 - kLift : r.m0; sh.v[warp][0][h0 + 1] = kScaled ? r.v1 - kLift : r.m1;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int d = out_dim<F>(i, hq);
        *reinterpret_cast<float2*>(&s_o[warp][d * 8 + h0]) = make_float2(r.acc[i][0], r.acc[i][1]);
        *reinterpret_cast<float2*>(&s_o[warp][(d + 1) * 8 + h0]) = make_float2(r.acc[i][2], r.acc[i][3]);
    }
    __syncthreads();
    if (threadIdx.x < 8 * NG) {                          // (every group works out the sums, the first leaves them)
        const int h = threadIdx.x & 7, g = threadIdx.x >> 3;
        float m = -INFINITY, v = -INFINITY, l = 0.f;
        for (int w = 0; w < kWarps; ++w) { m = fmaxf(m, sh.m[w][h]); v = fmaxf(v, sh.v[w][g][h]); }
        for (int w = 0; w < kWarps; ++w) {
            l += sh.l[w][h] * fast_exp2(sh.m[w][h] - finite_ref(m));
            sh.wgt[w][g][h] = fast_exp2(sh.v[w][g][h] - finite_ref(v));
        }
        if (g == 0) { sh.fin[0][h] = m; sh.fin[1][h] = l; }
        sh.fin[2 + g][h] = v;
    }
    __syncthreads();
    const int d = threadIdx.x, dg = NG > 1 ? d / (kHeadDim / NG) : 0;
    float o[8];
#pragma unroll
    for (int h = 0; h < 8; ++h) o[h] = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        const float4 a = *reinterpret_cast<const float4*>(&s_o[w][d * 8]), b = *reinterpret_cast<const float4*>(&s_o[w][d * 8 + 4]);
        const float* f = sh.wgt[w][dg];
        o[0] = fmaf(a.x, f[0], o[0]); o[1] = fmaf(a.y, f[1], o[1]); o[2] = fmaf(a.z, f[2], o[2]); o[3] = fmaf(a.w, f[3], o[3]);
        o[4] = fmaf(b.x, f[4], o[4]); o[5] = fmaf(b.y, f[5], o[5]); o[6] = fmaf(b.z, f[6], o[6]); o[7] = fmaf(b.w, f[7], o[7]);
    }
    if (MODE == kPart || MODE == kDealt) {
        float* rec = p.own_part + (size_t)blockIdx.x * kOwnRecFloats;
        if (d < 16 + 8 * NG) rec[d] = sh.fin[d >> 3][d & 7];
        // [dim / 4][head][4], by way of shared memory
        __syncthreads();                              // the warps' accumulators have been read
        float* mine = &s_o[0][0];
#pragma unroll
        for (int h = 0; h < 8; ++h) mine[((d >> 2) * 8 + h) * 4 + (d & 3)] = o[h];
        __syncthreads();
        float4* ro = reinterpret_cast<float4*>(rec + kOwnRecHead);
#pragma unroll
        for (int i = 0; i < 2; ++i) ro[i * kThreads + d] = *reinterpret_cast<const float4*>(mine + (i * kThreads + d) * 4);
        // The merge waits for this kernel only, so this kernel may not end before the prefixes' does.
        if constexpr (MODE == kPart) {
            if (p.prefix_part && blockIdx.x == 0) grid_wait_previous();
        }
        return;
    }
    if (MODE == kCluster) {
        // The CTAs leave their results [head][dim] in their own shared memory, and each then puts together a share of the
        // outputs from all of them. Nobody leaves before everybody has read.
        __syncthreads();                              // the warps' accumulators have been read
        float* mine = &s_o[0][0];
#pragma unroll
        for (int h = 0; h < 8; ++h) mine[h * kHeadDim + d] = o[h];
        cluster_sync_all();
        if (d < 8 * NG) {
            const int h = d & 7, g = d >> 3;
            float m = -INFINITY, v = -INFINITY, l = 0.f;
            float pm[kMaxCluster], pl[kMaxCluster], pv[kMaxCluster];
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c) {
                const bool in = c < p.splits;
                const uint32_t at = cluster_map_shared(smem_u32(&sh.fin[0][h]), in ? c : 0);
                pm[c] = in ? ld_cluster_f32(at) : -INFINITY;
                pl[c] = in ? ld_cluster_f32(at + 32) : 0.f;
                pv[c] = in ? ld_cluster_f32(at + 64 + 32 * g) : -INFINITY;
                m = fmaxf(m, pm[c]);
                v = fmaxf(v, pv[c]);
            }
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c) {
                l += pl[c] * fast_exp2(pm[c] - finite_ref(m));
                sh.cl[c][g][h] = fast_exp2(pv[c] - finite_ref(v));
            }
            if (g == 0) { sh.norm[0][h] = m; sh.norm[1][h] = l; }
            sh.norm[2 + g][h] = v;
        }
        __syncthreads();
        for (int i = split * kThreads + d; i < p.g * kHeadDim; i += p.splits * kThreads) {
            const int h = i / kHeadDim, g = NG > 1 ? i % kHeadDim / (kHeadDim / NG) : 0;
            float part[kMaxCluster];                  // all under way at once
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c)
                if (c < p.splits) part[c] = ld_cluster_f32(cluster_map_shared(smem_u32(&mine[i]), c));
            float x = 0.f;
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c)
                if (c < p.splits) x = fmaf(part[c], sh.cl[c][g][h], x);
            p.out[((size_t)seq * p.h_q + (size_t)head * p.g) * kHeadDim + i] =
                __float2bfloat16_rn(final_value(x, sh.norm[0][h], sh.norm[1][h], sh.norm[2 + g][h], fits));
        }
        if (p.lse && split == 0 && d < p.g)
            p.lse[(size_t)seq * p.h_q + (size_t)head * p.g + d] = final_lse(sh.norm[0][d], sh.norm[1][d], fits);
        cluster_sync_all();
        return;
    }
    __nv_bfloat16* orow = p.out + ((size_t)seq * p.h_q + (size_t)head * p.g) * kHeadDim + d;
#pragma unroll
    for (int h = 0; h < 8; ++h)
        if (h < p.g) orow[(size_t)h * kHeadDim] = __float2bfloat16_rn(final_value(o[h], sh.fin[0][h], sh.fin[1][h], sh.fin[2 + dg][h], fits));
    if (p.lse && d < p.g) p.lse[(size_t)seq * p.h_q + (size_t)head * p.g + d] = final_lse(sh.fin[0][d], sh.fin[1][d], fits);
}

}  // namespace gkv
