// Decode attention over a key/value store (one query token per sequence), and the merge of partial results.
//
// A unit is (sequence, KV head). Its rows are cut into pieces (one CTA each, when there are too few units to fill the device)
// of 16-key tiles, and the tiles of a piece go round the CTA's four warps. A warp works on its own: it loads a tile's codes
// straight into the registers of the matrix instructions' operands -- no shared memory, no barrier -- and keeps its own running
// softmax. Both products are mma.sync m16n8k16 with the keys (then the head dimensions) on M and the g <= 8 query heads on N,
// as in the bf16 decode kernel: 4 to 8 operations a byte, far from where tensor memory would pay. What makes loads without a
// transpose possible is that the order in which a product runs over its inner index is free: the lane that owns a quarter of a
// key's row takes whole 16-byte pieces of it and pairs them with the same elements of q, and on the way out lane group q owns
// the head dimensions of the pieces it read of V. The order of the nibbles of a 4-bit row is chosen for this.
//
// 8- and 4-bit codes become fp16 exactly (their scales stay outside the products), q becomes fp16 after division by a power
// of two (an element is exact down to 2^-17 of its row's largest; below, the error is at most 2^-25 of the largest), weights
// are rounded to fp16 (11 bits: outputs are off by 1.68e-3 instead of the 1.65e-3 that the output's own rounding to bf16 makes;
// it is what the product takes, and codes times fp16 weights are exact in its sums). The scale of a K row multiplies its logit.
// The scale s of a V row goes into the weight: w = p s c with p = exp2(z - m) as it enters the sum of the softmax, and
// c = exp2(m - v) with a running maximum v over z + log2 s, so that the largest of the weights handed to the product lie high in
// fp16's range whatever the scales are (those 2^-20 below lose bits, and 2^-31 below they are 0). A 4-bit row has a scale for
// each 32 head dimensions, and every group of dimensions has its own v and c: groups of very different size do not share a range.
// (v is kept at least at m - 112: c stays finite, and where all of a group's V is below 2^-112 its outputs are numbers of that
// size.) Sums and accumulators are fp32.
//
// The running maxima are allowed to lag: a step raises them (which costs a reduction over the warp and a rescaling of the
// accumulators) only when its weights have grown large.
//
// The pieces of a unit are joined by the CTAs of a cluster reading one another's shared memory (up to 8 pieces, no prefix), or
// leave partial results in the workspace for the merge kernel. Long rows are dealt out by the lengths that the sequences have, so
// that one long sequence among short ones gets the places that they do not need.
//
// Bound by HBM for 8-bit rows in a large batch (128 sequences x 8 heads of about 2200 keys, 585 MB: 97 us, 6.0 TB/s). 4-bit rows
// bring twice the elements per byte to unpack: 2 x 8 heads of about 120000 keys, 274 MB in 77 us, 3.6 TB/s, with the schedulers
// issuing 6 cycles out of 10, the logic and fp32 pipes 4 to 5 (without the products and what feeds them the same loads take 55
// us; with one reference for all groups of a head, which is not precise enough, 75.7). bf16 rows: 128 sequences x 8 heads of 2200
// keys, 1153 MB in 197 us, 5.9 TB/s. A single sequence of 640 keys takes 7.0 us: the launch, four trips to memory (length, q, rows,
// the others' results) one after the other, 3 tiles per warp.
#include "gkv_store_codes.cuh"

namespace gkv {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kTile = 16;            // keys of a tile
constexpr int kMergeHops = 4;
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
            z[0] = g == 0 ? acc[0] * s0 : fmaf(acc[0], s0, z[0]); z[1] = g == 0 ? acc[1] * s0 : fmaf(acc[1], s0, z[1]);
            z[2] = g == 0 ? acc[2] * s1 : fmaf(acc[2], s1, z[2]); z[3] = g == 0 ? acc[3] * s1 : fmaf(acc[3], s1, z[3]);
        }
        z[0] *= f0; z[1] *= f1; z[2] *= f0; z[3] *= f1;
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

__device__ __forceinline__ float finite_ref(float m) { return m == -INFINITY ? 0.f : m; }
// Output and log-sum-exp from sums relative to 2^v (values) and 2^m (weights); m = -infinity and no weight: nothing to attend to.
__device__ __forceinline__ float final_value(float o, float m, float l, float v, bool fits) {
    return !fits ? NAN : m == -INFINITY && l == 0.f ? 0.f : o * (fast_exp2(v - m) / l);
}
__device__ __forceinline__ float final_lse(float m, float l, bool fits) {
    return !fits ? NAN : m == -INFINITY && l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

// Resident CTAs per SM. 8- and 4-bit rows: 128 registers, 16 warps (128 sequences x 8 heads of about 2200 keys in 8 bits: 97 us;
// two tiles per step, 168 registers and 12 warps: 110 us. 2 x 8 heads of up to 131071 keys in 4 bits, with one reference a head: 76
// us; 12 warps: 78, with two tiles per step 85). bf16 rows need twice the registers for a tile.
__host__ __device__ constexpr int store_ctas(int format) { return format == GKV_STORE_BF16 ? 3 : 4; }
int store_attn_ctas_per_sm(int format) { return store_ctas(format); }

// Groups of head dimensions whose V rows have a scale of their own.
__host__ __device__ constexpr int value_groups(int format) { return format == GKV_STORE_INT4 ? 4 : 1; }

// What becomes of a CTA's result: it is the unit's; it goes to the workspace (kDealt: pieces go by the lengths); it is joined with
// those of the cluster's other CTAs.
enum { kWhole = 0, kPart = 1, kCluster = 2, kDealt = 3 };

// ---- pieces by length: the batch * splits places of a head go to the sequences one after the other, as many to each
// as its tiles need. Every warp works it out for itself; the merge does so again.
__device__ __forceinline__ int own_tiles_of(const StoreAttnLaunch& p, int seq) {
    if (seq >= p.batch) return 0;
    const int len = p.len[seq], n = p.k_new ? 1 : 0;
    return len < 0 || len > p.capacity - n ? 0 : (len + n + kTile - 1) / kTile;
}
__device__ __forceinline__ int pieces_of(int tiles, int per) { return (int)(((unsigned)tiles + (unsigned)per - 1) / (unsigned)per); }
// Pieces of sequences 0 .. seqs - 1, `per` tiles each. t0: tiles of sequence `lane`.
__device__ __forceinline__ int pieces_before(const StoreAttnLaunch& p, int seqs, int per, int lane, int t0) {
    int c = lane < seqs ? pieces_of(t0, per) : 0;
    for (int b = lane + 32; b < seqs; b += 32) c += pieces_of(own_tiles_of(p, b), per);
    return (int)__reduce_add_sync(0xffffffffu, (unsigned)c);
}
// Tiles of a piece: 8 (two turns of the four warps) or more, no unit in more than kMaxPieces pieces, and all pieces in their
// places: the mean, or a little more until roundings fit (with (splits - 1) / splits of the places they always do).
__device__ __forceinline__ int store_piece_tiles(const StoreAttnLaunch& p, int lane, int t0) {
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

// Own rows of the units. Grid: units x splits, split fastest; dealt out: a head's places, head slowest.
template <int F, int MODE>
__global__ void __launch_bounds__(kThreads, store_ctas(F)) gkv_store_attn_kernel(const StoreAttnLaunch p) {
    constexpr int NG = value_groups(F);
    constexpr bool kScaled = F != GKV_STORE_BF16;
    __shared__ float s_m[kWarps][8], s_l[kWarps][8], s_v[kWarps][NG][8], s_wgt[kWarps][NG][8], s_fin[2 + NG][8];
    __shared__ float s_cl[kMaxCluster][NG][8], s_norm[2 + NG][8];
    __shared__ __align__(16) float s_o[kWarps][kHeadDim * 8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int unit = blockIdx.x / p.splits, split = blockIdx.x - unit * p.splits, splits = p.splits, split_tiles = p.split_tiles;
    int seq = unit / p.h_kv, head = unit - seq * p.h_kv;
    if (MODE == kPart || MODE == kDealt) grid_launch_dependents();
    if (MODE == kDealt) {
        const int places = p.batch * p.splits;
        head = blockIdx.x / places;
        split = blockIdx.x - head * places;
        const int t0 = own_tiles_of(p, lane);
        split_tiles = store_piece_tiles(p, lane, t0);
        for (seq = -1; seq < p.batch;) {                 // the sequence whose places these are: 32 at a time
            const int c = pieces_of(seq < 0 ? t0 : own_tiles_of(p, seq + 1 + lane), split_tiles);
            int upto = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += x;
            }
            const unsigned past = __ballot_sync(0xffffffffu, upto > split);
            if (past) {
                const int at = __ffs(past) - 1;
                seq += 1 + at;
                split -= __shfl_sync(0xffffffffu, upto - c, at);
                splits = __shfl_sync(0xffffffffu, c, at);
                break;
            }
            split -= __shfl_sync(0xffffffffu, upto, 31);
            seq += 32;
        }
        if (seq >= p.batch) return;                      // a place that nobody needs
        unit = seq * p.h_kv + head;
    }
    const int len = p.len[seq];
    const bool append = p.k_new != nullptr;
    uint4 new_row = make_uint4(0u, 0u, 0u, 0u);           // on its way while the length is (lanes 0-15: K, 16-31: V)
    if (append) new_row = store_load_source<F>((lane < 16 ? p.k_new : p.v_new) + (size_t)unit * kHeadDim, lane & 15);
    const bool fits = append ? len < p.capacity : len <= p.capacity;
    // The merge goes by this word and not by the length, which it may count up itself.
    if (MODE == kPart && split == 0 && threadIdx.x == 0)
        p.own_part[(size_t)blockIdx.x * kOwnRecFloats + kOwnRecState] = len < 0 ? kPieceLeftOut : fits ? kPieceOk : kPieceNoFit;
    if (len < 0) {
        if (MODE == kPart && p.prefix_part && blockIdx.x == 0) grid_wait_previous();   // see the end of the partial form
        return;
    }
    const int n = fits ? len + (append ? 1 : 0) : 0;
    const int tiles = (n + kTile - 1) / kTile;
    const int t_begin = min(split * split_tiles, tiles);
    const int t_end = split == splits - 1 ? tiles : min(t_begin + split_tiles, tiles);

    uint8_t* kb = p.k + (size_t)unit * p.capacity * StoreFormat<F>::kRow;
    uint8_t* vb = p.v + (size_t)unit * p.capacity * StoreFormat<F>::kRow;
    __nv_bfloat16* ksb = p.k_scale + (size_t)unit * p.capacity * StoreFormat<F>::kScales;
    __nv_bfloat16* vsb = p.v_scale + (size_t)unit * p.capacity * StoreFormat<F>::kScales;

    // The warp that comes to the new row's tile puts the row into the store, before it loads anything of that tile (its own
    // writes are ordered before its later reads; no other warp reads the row).
    const int own_tiles = t_end - t_begin;               // tile i of the piece is warp i % kWarps'
    if (append && fits && own_tiles > 0 && t_end == tiles && warp == (own_tiles - 1) % kWarps) {
        store_put_row<F>((lane < 16 ? kb : vb) + (size_t)len * StoreFormat<F>::kRow,
                         (lane < 16 ? ksb : vsb) + (size_t)len * StoreFormat<F>::kScales, lane & 15, new_row);
        __threadfence_block();
        __syncwarp();
    }

    // q as the B operand: lane (head lane / 4, j = lane & 3)
    const int j = lane & 3, hq = lane >> 2, h0 = 2 * j;
    uint32_t qf[8][2];
    float f0 = p.scale_log2, f1 = p.scale_log2;
    {
        const __nv_bfloat16* qrow = p.q + ((size_t)seq * p.h_q + (size_t)head * p.g + min(hq, p.g - 1)) * kHeadDim;
        uint32_t a = 0;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            load_query<F>(qrow, ks, j, qf[ks][0], qf[ks][1]);
            if (kScaled) a = max(a, bf16_absmax(qf[ks][0], qf[ks][1]));
        }
        if (kScaled) {
            a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
            a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
            const int e = min(max((int)(a >> 7) - 127, -126), 126);        // exponent of the row's largest element
            const float down = __uint_as_float((uint32_t)(127 - e) << 23), up = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
                qf[ks][0] = bf16x2_to_f16x2(qf[ks][0], down);
                qf[ks][1] = bf16x2_to_f16x2(qf[ks][1], down);
            }
            f0 *= __shfl_sync(0xffffffffu, up, h0 * 4);
            f1 *= __shfl_sync(0xffffffffu, up, h0 * 4 + 4);
        }
    }

    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;       // running maxima (they may lag) and sums, heads h0, h0 + 1
    // The same maxima of z + log2(scale of V): with one scale a row in registers, with several, by group, in the warp's part of
    // s_v (they are looked at when maxima are raised, and registers are what limits the CTAs of an SM).
    float v0 = -INFINITY, v1 = -INFINITY;
    if constexpr (NG > 1) {
        if (hq == 0)
#pragma unroll
            for (int g = 0; g < NG; ++g) s_v[warp][g][h0] = s_v[warp][g][h0 + 1] = -INFINITY;
        __syncwarp();
    }
    float n0 = -INFINITY, n1 = -INFINITY;                           // what logits are taken relative to: m, once that is finite
    float c0[NG], c1[NG];                                           // 2^(m - v + kLift), with finite m and v
#pragma unroll
    for (int g = 0; g < NG; ++g) c0[g] = c1[g] = 1.f;
    float acc[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;

    TileK<F> tk;
    TileV<F> tv;
    const int end = min(t_end * kTile, n);
    const int key0 = (t_begin + warp) * kTile;
    int left = warp < own_tiles ? end - key0 : 0;        // keys from this tile's first on
    TilePtrs<F> at;
    at.kb = kb; at.vb = vb;
    at.ksb = reinterpret_cast<const uint8_t*>(ksb); at.vsb = reinterpret_cast<const uint8_t*>(vsb);
    at.set(key0, lane);
    load_tile_k<F>(tk, at, left, lane);
    load_tile_v<F>(tv, at, left, lane);
    while (left > 0) {
        at.advance(kWarps * kTile);
        const int left_next = left - kWarps * kTile;
        float z[4];
        tile_logits<F>(tk, qf, f0, f1, z);
        load_tile_k<F>(tk, at, left_next, lane);
        if (left < kTile) {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
                if (hq + 8 * hf >= left) z[2 * hf] = z[2 * hf + 1] = -INFINITY;
        }
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
        uint32_t b[NG][2];              // the weights, of several scales as soon as they are known
        // A z that is far above m, or a z + log2(scale) far above v, shows in the results: they are sums of non-negative numbers
        // (at most the limit then), infinite or NaN, also at the first step, where m is -infinity.
        float total = 0.f;
        auto weigh = [&]() {
            e[0] = fast_exp2(z[0] - n0); e[1] = fast_exp2(z[1] - n1);
            e[2] = fast_exp2(z[2] - n0); e[3] = fast_exp2(z[3] - n1);
            total += (e[0] + e[2]) + (e[1] + e[3]);
            if constexpr (NG > 1) {
                float sum = 0.f;
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {      // (e c is finite, c s need not be)
                        const float x = e[2 * hf] * c0[g] * sc[hf][g], y = e[2 * hf + 1] * c1[g] * sc[hf][g];
                        sum += x + y;
                        b[g][hf] = pack_weights<F>(x, y);
                    }
                total += sum * (1.f / kLiftFactor);
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
                    b0[g] = fmaxf(NG > 1 ? s_v[warp][g][h0] : v0, fmaxf(z[0] + x0, z[2] + x1));
                    b1[g] = fmaxf(NG > 1 ? s_v[warp][g][h0 + 1] : v1, fmaxf(z[1] + x0, z[3] + x1));
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
                    r0 = fast_exp2((NG > 1 ? s_v[warp][g][h0] : v0) - finite_ref(b0[g]));
                    r1 = fast_exp2((NG > 1 ? s_v[warp][g][h0 + 1] : v1) - finite_ref(b1[g]));
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
                    for (int g = 0; g < NG; ++g) { s_v[warp][g][h0] = b0[g]; s_v[warp][g][h0 + 1] = b1[g]; }
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
        tile_values<F, NG>(tv, b, acc);
        load_tile_v<F>(tv, at, left_next, lane);
        left = left_next;
    }

    // ---- the warps' results: statistics, then the accumulators weighted to a common maximum
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
        l0 += __shfl_xor_sync(0xffffffffu, l0, o);
        l1 += __shfl_xor_sync(0xffffffffu, l1, o);
    }
    if (hq == 0) {
        s_m[warp][h0] = m0; s_m[warp][h0 + 1] = m1;
        s_l[warp][h0] = l0; s_l[warp][h0 + 1] = l1;
        if constexpr (NG > 1) {
#pragma unroll
            for (int g = 0; g < NG; ++g) { s_v[warp][g][h0] -= kLift; s_v[warp][g][h0 + 1] -= kLift; }
        } else {
            s_v[warp][0][h0] = kScaled ? v0 - kLift : m0; s_v[warp][0][h0 + 1] = kScaled ? v1 - kLift : m1;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int d = out_dim<F>(i, hq);
        *reinterpret_cast<float2*>(&s_o[warp][d * 8 + h0]) = make_float2(acc[i][0], acc[i][1]);
        *reinterpret_cast<float2*>(&s_o[warp][(d + 1) * 8 + h0]) = make_float2(acc[i][2], acc[i][3]);
    }
    __syncthreads();
    if (threadIdx.x < 8 * NG) {                          // (every group works out the sums, the first leaves them)
        const int h = threadIdx.x & 7, g = threadIdx.x >> 3;
        float m = -INFINITY, v = -INFINITY, l = 0.f;
        for (int w = 0; w < kWarps; ++w) { m = fmaxf(m, s_m[w][h]); v = fmaxf(v, s_v[w][g][h]); }
        for (int w = 0; w < kWarps; ++w) {
            l += s_l[w][h] * fast_exp2(s_m[w][h] - finite_ref(m));
            s_wgt[w][g][h] = fast_exp2(s_v[w][g][h] - finite_ref(v));
        }
        if (g == 0) { s_fin[0][h] = m; s_fin[1][h] = l; }
        s_fin[2 + g][h] = v;
    }
    __syncthreads();
    const int d = threadIdx.x, dg = NG > 1 ? d / (kHeadDim / NG) : 0;
    float o[8];
#pragma unroll
    for (int h = 0; h < 8; ++h) o[h] = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        const float4 a = *reinterpret_cast<const float4*>(&s_o[w][d * 8]), b = *reinterpret_cast<const float4*>(&s_o[w][d * 8 + 4]);
        const float* f = s_wgt[w][dg];
        o[0] = fmaf(a.x, f[0], o[0]); o[1] = fmaf(a.y, f[1], o[1]); o[2] = fmaf(a.z, f[2], o[2]); o[3] = fmaf(a.w, f[3], o[3]);
        o[4] = fmaf(b.x, f[4], o[4]); o[5] = fmaf(b.y, f[5], o[5]); o[6] = fmaf(b.z, f[6], o[6]); o[7] = fmaf(b.w, f[7], o[7]);
    }
    if (MODE == kPart || MODE == kDealt) {
        float* rec = p.own_part + (size_t)blockIdx.x * kOwnRecFloats;
        if (d < 16 + 8 * NG) rec[d] = s_fin[d >> 3][d & 7];
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
        if (MODE == kPart && p.prefix_part && blockIdx.x == 0) grid_wait_previous();
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
            for (int r = 0; r < kMaxCluster; ++r) {
                const bool in = r < p.splits;
                const uint32_t at = cluster_map_shared(smem_u32(&s_fin[0][h]), in ? r : 0);
                pm[r] = in ? ld_cluster_f32(at) : -INFINITY;
                pl[r] = in ? ld_cluster_f32(at + 32) : 0.f;
                pv[r] = in ? ld_cluster_f32(at + 64 + 32 * g) : -INFINITY;
                m = fmaxf(m, pm[r]);
                v = fmaxf(v, pv[r]);
            }
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r) {
                l += pl[r] * fast_exp2(pm[r] - finite_ref(m));
                s_cl[r][g][h] = fast_exp2(pv[r] - finite_ref(v));
            }
            if (g == 0) { s_norm[0][h] = m; s_norm[1][h] = l; }
            s_norm[2 + g][h] = v;
        }
        __syncthreads();
        for (int i = split * kThreads + d; i < p.g * kHeadDim; i += p.splits * kThreads) {
            const int h = i / kHeadDim, g = NG > 1 ? i % kHeadDim / (kHeadDim / NG) : 0;
            float x = 0.f;
            for (int r = 0; r < p.splits; ++r)
                x = fmaf(ld_cluster_f32(cluster_map_shared(smem_u32(&mine[i]), r)), s_cl[r][g][h], x);
            p.out[((size_t)seq * p.h_q + (size_t)head * p.g) * kHeadDim + i] =
                __float2bfloat16_rn(final_value(x, s_norm[0][h], s_norm[1][h], s_norm[2 + g][h], fits));
        }
        if (p.lse && split == 0 && d < p.g)
            p.lse[(size_t)seq * p.h_q + (size_t)head * p.g + d] = final_lse(s_norm[0][d], s_norm[1][d], fits);
        cluster_sync_all();
        return;
    }
    __nv_bfloat16* orow = p.out + ((size_t)seq * p.h_q + (size_t)head * p.g) * kHeadDim + d;
#pragma unroll
    for (int h = 0; h < 8; ++h)
        if (h < p.g) orow[(size_t)h * kHeadDim] = __float2bfloat16_rn(final_value(o[h], s_fin[0][h], s_fin[1][h], s_fin[2 + dg][h], fits));
    if (p.lse && d < p.g) p.lse[(size_t)seq * p.h_q + (size_t)head * p.g + d] = final_lse(s_fin[0][d], s_fin[1][d], fits);
}

// Joins the partial results of a unit: those of its own pieces and, with a prefix, those of the prefix items that hold its
// query rows. 2^ds CTAs per unit, each with a share of the dimensions; thread t holds head t & 7 of four dimensions over every
// (slices)th of the parts, so that 8 lanes read 128 contiguous bytes of a record. The statistics of all parts are loaded at once,
// the values of 8 parts at a time: the kernel is a few trips to L2. NG groups of dimensions have maxima v of their own.
template <bool DEALT, int NG>
__global__ void __launch_bounds__(1024) gkv_store_merge_kernel(const StoreAttnLaunch p, const int ds) {
    // factors: own parts [part][group][8], then those of the prefix (with several groups: their maxima, a factor is worked out
    // where it is used) [part][8]
    extern __shared__ float s_part[];
    __shared__ __align__(16) float s_red[4 * 1024];
    __shared__ float s_fin[2 + NG][8];
    const int unit = blockIdx.x >> ds, share = blockIdx.x & ((1 << ds) - 1), seq = unit / p.h_kv, head = unit - seq * p.h_kv;
    const int t = threadIdx.x, slices = blockDim.x >> (8 - ds), slice = t >> (8 - ds), h = t & 7;
    const int d4 = ((t >> 3) & ((32 >> ds) - 1)) + share * (32 >> ds);
    const int hc = min(h, p.g - 1), warps = blockDim.x >> 5;

    // records: own ones, then those of the prefix items (two results each where the item's streams share the rows)
    int items = 0;
    int row0 = 0;
    size_t step = 0;
    const float *own = p.own_part + (size_t)unit * p.splits * kOwnRecFloats, *pre_rec = nullptr;
    int n_own = p.splits;
    if (DEALT) {
        const int t0 = own_tiles_of(p, t & 31), per = store_piece_tiles(p, t & 31, t0);
        own = p.own_part + ((size_t)head * p.batch * p.splits + pieces_before(p, seq, per, t & 31, t0)) * kOwnRecFloats;
        n_own = pieces_of(own_tiles_of(p, seq), per);
    }
    if (p.prefix_part) {
        const int pre = seq / p.seqs_per_prefix, sl = seq - pre * p.seqs_per_prefix, blk = sl / p.seqs_per_block;
        int base = head * p.n_blocks + blk;
        for (int i = 0; i < pre; ++i) base += ((p.prefix_len[i] + 127) / 128 + p.chunk - 1) / p.chunk * p.h_kv * p.n_blocks;
        items = ((p.prefix_len[pre] + 127) / 128 + p.chunk - 1) / p.chunk;
        step = (size_t)p.h_kv * p.n_blocks * kPrefixRecFloats;
        pre_rec = p.prefix_part + (size_t)base * kPrefixRecFloats;
        row0 = (sl - blk * p.seqs_per_block) * p.g;
    }
    const int twice = p.two_tiles ? 0 : 1, parts = n_own + (items << twice);
    // statistics and values of prefix part j at the unit's first row
    auto pre_stats = [&](int j) { return pre_rec + (size_t)(j >> twice) * step + row0 + (j & twice) * 128; };
    auto pre_values = [&](int j) {
        return reinterpret_cast<const float4*>(pre_rec + (size_t)(j >> twice) * step + 2 * kPrefixRows) + row0 + (j & twice) * 128;
    };
    grid_wait_previous();
    bool fits;
    if (DEALT) {                                     // (a sequence without keys has no piece)
        const int len = p.len[seq];
        if (len < 0) return;
        fits = p.k_new ? len < p.capacity : len <= p.capacity;
    } else {
        const float state = own[kOwnRecState];
        if (state == kPieceLeftOut) return;
        fits = state == kPieceOk;
    }

    // ---- statistics: factors of all parts. Thread t has head t & 7 of parts t / 8, t / 8 + blockDim / 8, ...
    const int hops = (parts * 8 + (int)blockDim.x - 1) / (int)blockDim.x;
    float m = -INFINITY, v[NG], l = 0.f, x[kMergeHops], y[kMergeHops][NG], z[kMergeHops];
#pragma unroll
    for (int g = 0; g < NG; ++g) v[g] = -INFINITY;
#pragma unroll
    for (int k = 0; k < kMergeHops; ++k) {
        x[k] = -INFINITY;
        z[k] = 0.f;
#pragma unroll
        for (int g = 0; g < NG; ++g) y[k][g] = -INFINITY;
        const int part = (t + k * (int)blockDim.x) >> 3;
        if (k < hops && part < parts) {
            if (part < n_own) {
                const float* r = own + (size_t)part * kOwnRecFloats + hc;
                x[k] = r[0]; z[k] = r[8];
#pragma unroll
                for (int g = 0; g < NG; ++g) y[k][g] = r[16 + 8 * g];
            } else {
                const float* r = pre_stats(part - n_own) + hc;
                x[k] = r[0]; z[k] = r[kPrefixRows];
#pragma unroll
                for (int g = 0; g < NG; ++g) y[k][g] = x[k];
            }
        }
        m = fmaxf(m, x[k]);
#pragma unroll
        for (int g = 0; g < NG; ++g) v[g] = fmaxf(v[g], y[k][g]);
    }
    constexpr int kStats = 8 * (1 + NG);             // a warp's maxima
#pragma unroll
    for (int o = 8; o < 32; o <<= 1) {
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll
        for (int g = 0; g < NG; ++g) v[g] = fmaxf(v[g], __shfl_xor_sync(0xffffffffu, v[g], o));
    }
    if ((t & 31) < 8) {
        s_red[(t >> 5) * kStats + h] = m;
#pragma unroll
        for (int g = 0; g < NG; ++g) s_red[(t >> 5) * kStats + 8 + 8 * g + h] = v[g];
    }
    __syncthreads();
    if constexpr (NG == 1) {
        for (int i = 0; i < warps; ++i) { m = fmaxf(m, s_red[i * kStats + h]); v[0] = fmaxf(v[0], s_red[i * kStats + 8 + h]); }
    } else {                                         // one thread a number
        if (t < kStats) {
            float a = -INFINITY;
            for (int i = 0; i < warps; ++i) a = fmaxf(a, s_red[i * kStats + t]);
            s_fin[t < 8 ? 0 : 1 + (t >> 3)][h] = a;
        }
        __syncthreads();
        m = s_fin[0][h];
#pragma unroll
        for (int g = 0; g < NG; ++g) v[g] = s_fin[2 + g][h];
    }
    const float mr = finite_ref(m);
    constexpr int kSums = 2048;                      // (the maxima take up to 32 kStats)
    static_assert(32 * kStats <= kSums && kSums + 32 * 8 <= 4 * 1024, "scratch");
#pragma unroll
    for (int k = 0; k < kMergeHops; ++k) {
        const int i = t + k * (int)blockDim.x, part = i >> 3;
        l += z[k] * fast_exp2(x[k] - mr);            // (a NaN sum comes with a maximum of -infinity)
        if (k < hops && part < parts) {              // 0: no key, values may be missing
            if (NG == 1 || part < n_own) {
#pragma unroll
                for (int g = 0; g < NG; ++g) s_part[(part * NG + g) * 8 + h] = x[k] == -INFINITY ? 0.f : fast_exp2(y[k][g] - finite_ref(v[g]));
            } else {
                s_part[(n_own * (NG - 1) + part) * 8 + h] = x[k];
            }
        }
    }
#pragma unroll
    for (int o = 8; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if ((t & 31) < 8) s_red[kSums + (t >> 5) * 8 + h] = l;
    __syncthreads();
    if (t < 8) {
        float sum = 0.f;
        for (int i = 0; i < warps; ++i) sum += s_red[kSums + i * 8 + h];
        s_fin[1][h] = sum;
        if (NG == 1) { s_fin[0][h] = m; s_fin[2][h] = v[0]; }
    }

    // ---- values
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float w, const float4& a) {
        if (w != 0.f) { o.x = fmaf(a.x, w, o.x); o.y = fmaf(a.y, w, o.y); o.z = fmaf(a.z, w, o.z); o.w = fmaf(a.w, w, o.w); }
    };
    const int dg = NG > 1 ? d4 / (kHeadDim / 4 / NG) : 0;
    const float vr = finite_ref(NG > 1 ? s_fin[2 + dg][h] : v[0]);
    const float4* ov = reinterpret_cast<const float4*>(own + kOwnRecHead) + d4 * 8 + h;
#pragma unroll 4
    for (int i = slice; i < n_own; i += slices) {
        const float4 a = ov[(size_t)i * (kOwnRecFloats / 4)];
        add(s_part[(i * NG + dg) * 8 + h], a);
    }
    const int n_pre = items << twice;
    for (int i0 = slice; i0 < n_pre; i0 += 8 * slices) {
        float4 a[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) a[k] = pre_values(min(i0 + k * slices, n_pre - 1))[d4 * kPrefixRows + hc];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i0 + k * slices < n_pre) {
                const float f = s_part[(n_own * NG + i0 + k * slices) * 8 + h];
                add(NG == 1 ? f : f == -INFINITY ? 0.f : fast_exp2(f - vr), a[k]);
            }
    }
    if (slices > 1) {
        __syncthreads();
        reinterpret_cast<float4*>(s_red)[t] = o;
        __syncthreads();
        if (slice == 0)
            for (int i = 1; i < slices; ++i) {
                const float4 a = reinterpret_cast<const float4*>(s_red)[(i << (8 - ds)) + t];
                o.x += a.x; o.y += a.y; o.z += a.z; o.w += a.w;
            }
    } else {
        __syncthreads();
    }
    if (slice == 0 && h < p.g) {
        const float fm = s_fin[0][h], fl = s_fin[1][h], fv = s_fin[2 + dg][h];
        *reinterpret_cast<uint2*>(p.out + ((size_t)seq * p.h_q + (size_t)head * p.g + h) * kHeadDim + 4 * d4) =
            make_uint2(pack_bf16x2(final_value(o.x, fm, fl, fv, fits), final_value(o.y, fm, fl, fv, fits)),
                       pack_bf16x2(final_value(o.z, fm, fl, fv, fits), final_value(o.w, fm, fl, fv, fits)));
    }
    if (share == 0 && t < p.g) {
        if (p.lse) p.lse[(size_t)seq * p.h_q + (size_t)head * p.g + t] = final_lse(s_fin[0][t], s_fin[1][t], fits);
        if (p.len_out && head == 0 && t == 0 && fits) p.len_out[seq] += 1;
    }
}

// cluster > 1: clusters of that many CTAs; dependent: the kernel may start while the one before it drains.
template <typename... A>
static cudaError_t launch_ex(void (*kernel)(A...), unsigned grid, unsigned threads, size_t smem, int cluster, bool dependent, cudaStream_t s,
                             const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)cluster;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (dependent) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = (unsigned)n;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
template <int F>
static cudaError_t launch_own(const StoreAttnLaunch& p, cudaStream_t s) {
    const unsigned grid = (unsigned)(p.batch * p.h_kv * p.splits);
    if (p.dealt) return launch_ex(gkv_store_attn_kernel<F, kDealt>, grid, kThreads, 0, 1, false, s, p);
    if (store_needs_merge(p)) return launch_ex(gkv_store_attn_kernel<F, kPart>, grid, kThreads, 0, 1, p.prefix_part != nullptr, s, p);
    if (p.splits > 1) return launch_ex(gkv_store_attn_kernel<F, kCluster>, grid, kThreads, 0, p.splits, false, s, p);
    gkv_store_attn_kernel<F, kWhole><<<grid, kThreads, 0, s>>>(p);
    return cudaGetLastError();
}
bool store_needs_merge(const StoreAttnLaunch& p) { return p.dealt || p.splits > kMaxCluster || p.prefix_part != nullptr || p.len_out != nullptr; }
cudaError_t launch_store_attn(const StoreAttnLaunch& p, cudaStream_t s) {
    switch (p.format) {
        case GKV_STORE_BF16: return launch_own<GKV_STORE_BF16>(p, s);
        case GKV_STORE_E4M3: return launch_own<GKV_STORE_E4M3>(p, s);
        case GKV_STORE_INT8: return launch_own<GKV_STORE_INT8>(p, s);
        default:             return launch_own<GKV_STORE_INT4>(p, s);
    }
}
// The fewer units, the more CTAs per unit. 256 threads for up to 8 parts, 512 for up to 16, else 1024. (The plan bounds the parts
// of a unit: kMaxPieces + 2 kMaxRuns = 448, 8 numbers each are 3.5 per thread.) Dealt out, units have few parts or up to
// kMaxPieces, which the host does not know: threads by the number of units (256 units of 2 parts each with 1024, 512, 256 threads,
// attention included: 102, 96, 96 us; one of them with most of the rows: 63, 61, 65; 1024 units: -, 378, 370 and -, 167, 153).
cudaError_t launch_store_merge(const StoreAttnLaunch& p, cudaStream_t s) {
    int longest = 0;
    for (int i = 0; i < p.n_prefix; ++i) longest = p.prefix_len[i] > longest ? p.prefix_len[i] : longest;
    const int items = p.prefix_part ? ((longest + 127) / 128 + p.chunk - 1) / p.chunk * (p.two_tiles ? 1 : 2) : 0;
    const int own = p.dealt ? min(p.batch * p.splits, kMaxPieces) : p.splits, parts = own + items, units = p.batch * p.h_kv;
    const int ds = units <= 40 ? 2 : units <= 80 ? 1 : 0, ng = value_groups(p.format);
    const unsigned threads = p.dealt ? (units <= 148 ? 1024u : units <= 296 ? 512u : 256u) : parts <= 8 ? 256u : parts <= 16 ? 512u : 1024u;
    const auto kernel = ng == 1 ? (p.dealt ? gkv_store_merge_kernel<true, 1> : gkv_store_merge_kernel<false, 1>)
                                : (p.dealt ? gkv_store_merge_kernel<true, 4> : gkv_store_merge_kernel<false, 4>);
    return launch_ex(kernel, (unsigned)units << ds, threads, (size_t)(own * ng + items) * 8 * sizeof(float), 1, true, s, p, ds);
}

}  // namespace gkv
