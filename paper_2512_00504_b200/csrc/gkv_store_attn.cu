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
// are rounded to fp16 (11 bits). The scale of a K row multiplies its logit. The scale s of a V row goes into the weight by way
// of the exponent, w = exp2(z + log2 s - m'), with a running maximum m' of its own over z + log2 s: the weights handed to the
// product then lie in fp16's range whatever the scales are. Sums and accumulators are fp32.
//
// The running maxima are allowed to lag: a tile raises them (which costs a reduction over the warp and a rescaling of the
// accumulators) only when some logit is more than 2^kLag above them.
#include "gkv_store_codes.cuh"

namespace gkv {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kTile = 16;            // keys of a tile
constexpr float kLag = 8.f;
// state word of a unit's first partial result
constexpr float kPieceOk = 0.f, kPieceNoFit = 1.f, kPieceLeftOut = 2.f;
constexpr float kLift = 6.f;         // the weights of scaled rows are lifted by 2^6: at most 2^14, subnormal below 2^-20

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
// Two 16-bit words of nibbles (one in each half of w) -> four fp16 pairs (nibble e of both words): 1024 + u - 1032 for the
// nibbles in the low places, (1024 + 16 u) / 16 - 72 for those in the high ones, u = c + 8.
__device__ __forceinline__ void unpack4(uint32_t w, uint32_t (&e)[4]) {
    const uint32_t w8 = w >> 8;
    e[0] = hsub2((w & 0x000f000fu) | 0x64006400u, 0x64086408u);
    e[1] = hfma2((w & 0x00f000f0u) | 0x64006400u, 0x2c002c00u, 0xd480d480u);
    e[2] = hsub2((w8 & 0x000f000fu) | 0x64006400u, 0x64086408u);
    e[3] = hfma2((w8 & 0x00f000f0u) | 0x64006400u, 0x2c002c00u, 0xd480d480u);
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

// Rows from `end` on are not loaded: zeros stand for them, so that whatever lies there cannot reach the sums.
template <int F>
__device__ __forceinline__ void load_k(TileK<F>& t, const uint8_t* k, const __nv_bfloat16* sc, int key0, int end, int lane) {
    constexpr int kPieces = F == GKV_STORE_BF16 ? 4 : F == GKV_STORE_INT4 ? 1 : 2;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
        const int key = key0 + (lane >> 2) + 8 * hf;
        const uint8_t* row = k + (size_t)key * StoreFormat<F>::kRow + (lane & 3) * 16;
#pragma unroll
        for (int c = 0; c < kPieces; ++c) t.d[hf][c] = key < end ? ld16(row + c * 64) : make_uint4(0u, 0u, 0u, 0u);
        if constexpr (F == GKV_STORE_INT4) t.s[hf] = key < end ? ld8(sc + (size_t)key * 4) : make_uint2(0u, 0u);
        else if constexpr (F != GKV_STORE_BF16) t.s[hf] = key < end ? ld2(sc + key) : 0u;
    }
}
template <int F>
__device__ __forceinline__ void load_v(TileV<F>& t, const uint8_t* v, const __nv_bfloat16* sc, int key0, int end, int lane) {
    const int q = lane >> 2, j = lane & 3;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int key = key0 + 2 * j + (i & 1) + 8 * (i >> 1);
        const uint8_t* row = v + (size_t)key * StoreFormat<F>::kRow;
        const bool in = key < end;
        if constexpr (F == GKV_STORE_BF16) {
            t.d[i][0] = in ? ld16(row + q * 16) : make_uint4(0u, 0u, 0u, 0u);
            t.d[i][1] = in ? ld16(row + 128 + q * 16) : make_uint4(0u, 0u, 0u, 0u);
        } else if constexpr (F == GKV_STORE_INT4) {
            t.d[i] = in ? ld8(row + q * 8) : make_uint2(0u, 0u);
        } else {
            t.d[i] = in ? ld16(row + q * 16) : make_uint4(0u, 0u, 0u, 0u);
        }
    }
    // scales by key as the logits are held: rows r, r + 8
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
        const int key = key0 + (lane >> 2) + 8 * hf;
        if constexpr (F == GKV_STORE_INT4) t.s[hf] = key < end ? ld8(sc + (size_t)key * 4) : make_uint2(0u, 0u);
        else if constexpr (F != GKV_STORE_BF16) t.s[hf] = key < end ? ld2(sc + key) : 0u;
    }
}

// Logits of a tile in log2 units: z[0], z[1] = key r and heads h0, h0 + 1; z[2], z[3] = key r + 8. f0, f1: factors of the heads.
template <int F>
__device__ __forceinline__ void tile_logits(const TileK<F>& t, const uint32_t (&qf)[8][2], float f0, float f1, float (&z)[4]) {
    if constexpr (F == GKV_STORE_INT4) {
        z[0] = z[1] = z[2] = z[3] = 0.f;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            uint32_t a[2][4];   // [row r / r + 8][element pair]
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const uint4 d = t.d[hf][0];
                unpack4(__byte_perm(g < 2 ? d.x : d.y, g < 2 ? d.z : d.w, (g & 1) ? 0x7632 : 0x5410), a[hf]);
            }
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
            const uint32_t a0[4] = {a[0][0], a[1][0], a[0][1], a[1][1]}, a1[4] = {a[0][2], a[1][2], a[0][3], a[1][3]};
            mma_row<F>(acc, a0, qf[2 * g][0], qf[2 * g][1]);
            mma_row<F>(acc, a1, qf[2 * g + 1][0], qf[2 * g + 1][1]);
            const uint32_t w0 = g < 2 ? t.s[0].x : t.s[0].y, w1 = g < 2 ? t.s[1].x : t.s[1].y;
            const float s0 = (g & 1) ? bf16_hi(w0) : bf16_lo(w0), s1 = (g & 1) ? bf16_hi(w1) : bf16_lo(w1);
            z[0] = fmaf(acc[0], s0, z[0]); z[1] = fmaf(acc[1], s0, z[1]);
            z[2] = fmaf(acc[2], s1, z[2]); z[3] = fmaf(acc[3], s1, z[3]);
        }
        z[0] *= f0; z[1] *= f1; z[2] *= f0; z[3] *= f1;
    } else {
        float sa[4] = {0.f, 0.f, 0.f, 0.f}, sb[4] = {0.f, 0.f, 0.f, 0.f};   // two accumulators: half the dependent chain
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
            mma_row<F>((ks & 1) ? sb : sa, a, qf[ks][0], qf[ks][1]);
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
            uint32_t x[4], y[4];
            unpack4(__byte_perm(word(0), word(1), (g & 1) ? 0x7632 : 0x5410), x);
            unpack4(__byte_perm(word(2), word(3), (g & 1) ? 0x7632 : 0x5410), y);
            const uint32_t a0[4] = {x[0], x[1], y[0], y[1]}, a1[4] = {x[2], x[3], y[2], y[3]};
            mma_row<F>(acc[2 * g], a0, b[g][0], b[g][1]);
            mma_row<F>(acc[2 * g + 1], a1, b[g][0], b[g][1]);
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
// First of the two element pairs of q that lane j multiplies at step ks; the second pair is at +step2, the pair's second
// element at +next.
template <int F>
__device__ __forceinline__ void load_query(const __nv_bfloat16* row, int ks, int j, uint32_t& b0, uint32_t& b1) {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(row);
    if (F == GKV_STORE_BF16) {
        const uint2 x = *reinterpret_cast<const uint2*>(q + 32 * (ks >> 1) + 8 * j + 4 * (ks & 1));
        b0 = x.x; b1 = x.y;
    } else if (F == GKV_STORE_INT4) {
        const uint16_t* x = q + 32 * (ks >> 1) + 8 * j + 2 * (ks & 1);
        const uint32_t a = *reinterpret_cast<const uint32_t*>(x), b = *reinterpret_cast<const uint32_t*>(x + 4);
        b0 = __byte_perm(a, b, 0x5410); b1 = __byte_perm(a, b, 0x7632);
    } else {
        const uint2 x = *reinterpret_cast<const uint2*>(q + 64 * (ks >> 2) + 16 * j + 4 * (ks & 3));
        b0 = x.x; b1 = x.y;
    }
}
__device__ __forceinline__ uint32_t bf16x2_to_f16x2(uint32_t x, float f) { return pack_f16x2(bf16_lo(x) * f, bf16_hi(x) * f); }

__device__ __forceinline__ float finite_ref(float m) { return m == -INFINITY ? 0.f : m; }

// Own rows of the units. Grid: units x splits, split fastest. PART: write a partial result instead of the output.
template <int F, int U, bool PART>
__global__ void __launch_bounds__(kThreads, F == GKV_STORE_BF16 ? 3 : 3) gkv_store_attn_kernel(const StoreAttnLaunch p) {
    constexpr int NG = F == GKV_STORE_INT4 ? 4 : 1;
    constexpr bool kScaled = F != GKV_STORE_BF16;
    __shared__ float s_m[kWarps][8], s_l[kWarps][8], s_v[kWarps][8], s_wgt[kWarps][8], s_fin[3][8];
    __shared__ __align__(16) float s_o[kWarps][kHeadDim * 8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int unit = blockIdx.x / p.splits, split = blockIdx.x - unit * p.splits;
    const int seq = unit / p.h_kv, head = unit - seq * p.h_kv;
    const int len = p.len[seq];
    const bool append = p.k_new != nullptr;
    const bool fits = append ? len < p.capacity : len <= p.capacity;
    // The merge goes by this word and not by the length, which it may count up itself.
    if (PART && split == 0 && threadIdx.x == 0)
        p.own_part[(size_t)blockIdx.x * kOwnRecFloats + 24] = len < 0 ? kPieceLeftOut : fits ? kPieceOk : kPieceNoFit;
    if (len < 0) return;
    const int n = fits ? len + (append ? 1 : 0) : 0;
    const int tiles = (n + kTile - 1) / kTile;
    const int t_begin = min(split * p.split_tiles, tiles);
    const int t_end = split == p.splits - 1 ? tiles : min(t_begin + p.split_tiles, tiles);

    uint8_t* kb = p.k + (size_t)unit * p.capacity * StoreFormat<F>::kRow;
    uint8_t* vb = p.v + (size_t)unit * p.capacity * StoreFormat<F>::kRow;
    __nv_bfloat16* ksb = p.k_scale + (size_t)unit * p.capacity * StoreFormat<F>::kScales;
    __nv_bfloat16* vsb = p.v_scale + (size_t)unit * p.capacity * StoreFormat<F>::kScales;

    // Steps of U tiles go round the warps.
    const int steps = (t_end - t_begin + U - 1) / U;
    // The warp that comes to the new row's tile puts the row into the store, before it loads anything of that tile (its own
    // writes are ordered before its later reads; no other warp reads the row).
    if (append && fits && steps > 0 && t_end == tiles && warp == (steps - 1) % kWarps) {
        const int l = lane & 15;
        const __nv_bfloat16* src = (lane < 16 ? p.k_new : p.v_new) + (size_t)unit * kHeadDim;
        const uint4 x = store_load_source<F>(src, l);
        store_put_row<F>((lane < 16 ? kb : vb) + (size_t)len * StoreFormat<F>::kRow,
                         (lane < 16 ? ksb : vsb) + (size_t)len * StoreFormat<F>::kScales, l, x);
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
    float v0 = -INFINITY, v1 = -INFINITY;                           // the same maxima of z + log2(scale of V)
    float acc[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;

    TileK<F> tk[U];
    TileV<F> tv[U];
    int step = warp;
    int key0 = (t_begin + step * U) * kTile;
    const int end = min(t_end * kTile, n);
#pragma unroll
    for (int u = 0; u < U; ++u) load_k<F>(tk[u], kb, ksb, key0 + u * kTile, step < steps ? end : 0, lane);
#pragma unroll
    for (int u = 0; u < U; ++u) load_v<F>(tv[u], vb, vsb, key0 + u * kTile, step < steps ? end : 0, lane);
    for (; step < steps; step += kWarps) {
        const int next0 = key0 + kWarps * U * kTile;
        const int next_end = step + kWarps < steps ? end : 0;
        float z[U][4];
#pragma unroll
        for (int u = 0; u < U; ++u) tile_logits<F>(tk[u], qf, f0, f1, z[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) load_k<F>(tk[u], kb, ksb, next0 + u * kTile, next_end, lane);
        // log2 of the V scales of this lane's two keys, and their largest (the groups of a 4-bit row)
        float lv[U][2][NG], lmax[U][2];
        bool raise = false;
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                lmax[u][hf] = 0.f;
                if constexpr (F == GKV_STORE_INT4) {
                    const uint2 s = tv[u].s[hf];
                    lv[u][hf][0] = __log2f(bf16_lo(s.x)); lv[u][hf][1] = __log2f(bf16_hi(s.x));
                    lv[u][hf][2] = __log2f(bf16_lo(s.y)); lv[u][hf][3] = __log2f(bf16_hi(s.y));
                    lmax[u][hf] = fmaxf(fmaxf(lv[u][hf][0], lv[u][hf][1]), fmaxf(lv[u][hf][2], lv[u][hf][3]));
                } else if constexpr (kScaled) {
                    lmax[u][hf] = lv[u][hf][0] = __log2f(bf16_lo(tv[u].s[hf]));
                }
                const int key = key0 + u * kTile + hq + 8 * hf;
                if (key >= end) { z[u][2 * hf] = z[u][2 * hf + 1] = -INFINITY; if (kScaled) lmax[u][hf] = 0.f; }
                raise |= z[u][2 * hf] > m0 + kLag || z[u][2 * hf + 1] > m1 + kLag;
                if (kScaled) raise |= z[u][2 * hf] + lmax[u][hf] > v0 + kLag || z[u][2 * hf + 1] + lmax[u][hf] > v1 + kLag;
            }
        }
        if (__any_sync(0xffffffffu, raise)) {
            float a0 = m0, a1 = m1, c0 = v0, c1 = v1;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                a0 = fmaxf(a0, fmaxf(z[u][0], z[u][2]));
                a1 = fmaxf(a1, fmaxf(z[u][1], z[u][3]));
                if (kScaled) {
                    c0 = fmaxf(c0, fmaxf(z[u][0] + lmax[u][0], z[u][2] + lmax[u][1]));
                    c1 = fmaxf(c1, fmaxf(z[u][1] + lmax[u][0], z[u][3] + lmax[u][1]));
                }
            }
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                a0 = fmaxf(a0, __shfl_xor_sync(0xffffffffu, a0, o));
                a1 = fmaxf(a1, __shfl_xor_sync(0xffffffffu, a1, o));
                if (kScaled) {
                    c0 = fmaxf(c0, __shfl_xor_sync(0xffffffffu, c0, o));
                    c1 = fmaxf(c1, __shfl_xor_sync(0xffffffffu, c1, o));
                }
            }
            l0 *= fast_exp2(m0 - finite_ref(a0));
            l1 *= fast_exp2(m1 - finite_ref(a1));
            float r0, r1;
            if (kScaled) { r0 = fast_exp2(v0 - finite_ref(c0)); r1 = fast_exp2(v1 - finite_ref(c1)); }
            else { r0 = fast_exp2(m0 - finite_ref(a0)); r1 = fast_exp2(m1 - finite_ref(a1)); }
            m0 = a0; m1 = a1; v0 = c0; v1 = c1;
#pragma unroll
            for (int i = 0; i < 8; ++i) { acc[i][0] *= r0; acc[i][1] *= r1; acc[i][2] *= r0; acc[i][3] *= r1; }
        }
        const float n0 = finite_ref(m0), n1 = finite_ref(m1);
        const float w0 = finite_ref(v0) - kLift, w1 = finite_ref(v1) - kLift;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float p0 = fast_exp2(z[u][0] - n0), p1 = fast_exp2(z[u][1] - n1);
            const float p2 = fast_exp2(z[u][2] - n0), p3 = fast_exp2(z[u][3] - n1);
            l0 += p0 + p2;
            l1 += p1 + p3;
            uint32_t b[NG][2];
            if constexpr (!kScaled) {
                b[0][0] = movmatrix_trans(pack_weights<F>(p0, p1));
                b[0][1] = movmatrix_trans(pack_weights<F>(p2, p3));
            } else {
                const bool in0 = key0 + u * kTile + hq < end, in1 = key0 + u * kTile + hq + 8 < end;
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const float e0 = in0 ? lv[u][0][g] : 0.f, e1 = in1 ? lv[u][1][g] : 0.f;   // z = -inf there: no weight
                    b[g][0] = movmatrix_trans(pack_weights<F>(fast_exp2(z[u][0] + e0 - w0), fast_exp2(z[u][1] + e0 - w1)));
                    b[g][1] = movmatrix_trans(pack_weights<F>(fast_exp2(z[u][2] + e1 - w0), fast_exp2(z[u][3] + e1 - w1)));
                }
            }
            tile_values<F, NG>(tv[u], b, acc);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) load_v<F>(tv[u], vb, vsb, next0 + u * kTile, next_end, lane);
        key0 = next0;
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
        s_v[warp][h0] = kScaled ? v0 - kLift : m0; s_v[warp][h0 + 1] = kScaled ? v1 - kLift : m1;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int d = out_dim<F>(i, hq);
        *reinterpret_cast<float2*>(&s_o[warp][d * 8 + h0]) = make_float2(acc[i][0], acc[i][1]);
        *reinterpret_cast<float2*>(&s_o[warp][(d + 1) * 8 + h0]) = make_float2(acc[i][2], acc[i][3]);
    }
    __syncthreads();
    if (threadIdx.x < 8) {
        const int h = threadIdx.x;
        float m = -INFINITY, v = -INFINITY, l = 0.f;
        for (int w = 0; w < kWarps; ++w) { m = fmaxf(m, s_m[w][h]); v = fmaxf(v, s_v[w][h]); }
        for (int w = 0; w < kWarps; ++w) {
            l += s_l[w][h] * fast_exp2(s_m[w][h] - finite_ref(m));
            s_wgt[w][h] = fast_exp2(s_v[w][h] - finite_ref(v));
        }
        s_fin[0][h] = m; s_fin[1][h] = l; s_fin[2][h] = v;
    }
    __syncthreads();
    const int d = threadIdx.x;
    float o[8];
#pragma unroll
    for (int h = 0; h < 8; ++h) o[h] = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        const float4 a = *reinterpret_cast<const float4*>(&s_o[w][d * 8]), b = *reinterpret_cast<const float4*>(&s_o[w][d * 8 + 4]);
        o[0] = fmaf(a.x, s_wgt[w][0], o[0]); o[1] = fmaf(a.y, s_wgt[w][1], o[1]); o[2] = fmaf(a.z, s_wgt[w][2], o[2]); o[3] = fmaf(a.w, s_wgt[w][3], o[3]);
        o[4] = fmaf(b.x, s_wgt[w][4], o[4]); o[5] = fmaf(b.y, s_wgt[w][5], o[5]); o[6] = fmaf(b.z, s_wgt[w][6], o[6]); o[7] = fmaf(b.w, s_wgt[w][7], o[7]);
    }
    if (PART) {
        float* rec = p.own_part + (size_t)blockIdx.x * kOwnRecFloats;
        if (d < 8) { rec[d] = s_fin[0][d]; rec[8 + d] = s_fin[1][d]; rec[16 + d] = s_fin[2][d]; }
        float4* ro = reinterpret_cast<float4*>(rec + 32 + d * 8);
        ro[0] = make_float4(o[0], o[1], o[2], o[3]);
        ro[1] = make_float4(o[4], o[5], o[6], o[7]);
    } else {
        __nv_bfloat16* orow = p.out + ((size_t)seq * p.h_q + (size_t)head * p.g) * kHeadDim + d;
#pragma unroll
        for (int h = 0; h < 8; ++h) {
            if (h >= p.g) break;
            // (values) * 2^(v - m) / l; nothing to attend to: 0
            const float f = fast_exp2(s_fin[2][h] - s_fin[0][h]) / s_fin[1][h];
            const bool none = s_fin[0][h] == -INFINITY && s_fin[1][h] == 0.f;
            const float x = !fits ? NAN : none ? 0.f : o[h] * f;
            orow[(size_t)h * kHeadDim] = __float2bfloat16_rn(x);
        }
        if (p.lse && d < p.g) {
            const bool none = s_fin[0][d] == -INFINITY && s_fin[1][d] == 0.f;
            const float x = !fits ? NAN : none ? -INFINITY : (s_fin[0][d] + log2f(s_fin[1][d])) * 0.6931471805599453f;
            p.lse[(size_t)seq * p.h_q + (size_t)head * p.g + d] = x;
        }
    }
}

// Joins the partial results of a unit: those of its own pieces and, with a prefix, those of the prefix items that hold its
// query rows. One CTA per unit; thread t holds head t & 7 of dimensions t / 8 + 32 k, so that 8 lanes read 32 contiguous bytes
// of a record.
__global__ void __launch_bounds__(256) gkv_store_merge_kernel(const StoreAttnLaunch p) {
    __shared__ __align__(16) __nv_bfloat16 s_out[8 * kHeadDim];
    const int unit = blockIdx.x, seq = unit / p.h_kv, head = unit - seq * p.h_kv;
    const float* own = p.own_part + (size_t)unit * p.splits * kOwnRecFloats;
    const float state = own[24];
    if (state == kPieceLeftOut) return;
    const bool fits = state == kPieceOk;
    const int h = threadIdx.x & 7, d0 = threadIdx.x >> 3;

    // prefix records of this unit
    int items = 0, base = 0, step = 0, slot = 0;
    const int sub = p.two_tiles ? 1 : 2;             // results per record that belong to the unit
    if (p.prefix_part) {
        const int pre = seq / p.seqs_per_prefix, sl = seq - pre * p.seqs_per_prefix;
        for (int i = 0; i < pre; ++i) base += ((p.prefix_len[i] + 127) / 128 + p.chunk - 1) / p.chunk * p.h_kv * p.n_blocks;
        items = ((p.prefix_len[pre] + 127) / 128 + p.chunk - 1) / p.chunk;
        const int blk = sl / p.seqs_per_block;
        base += head * p.n_blocks + blk;
        step = p.h_kv * p.n_blocks;
        slot = (sl - blk * p.seqs_per_block) * p.g + min(h, p.g - 1);
    }
    float m = -INFINITY, v = -INFINITY;
    for (int i = 0; i < p.splits; ++i) {
        m = fmaxf(m, own[(size_t)i * kOwnRecFloats + h]);
        v = fmaxf(v, own[(size_t)i * kOwnRecFloats + 16 + h]);
    }
    for (int i = 0; i < items * sub; ++i) {
        const float* rec = p.prefix_part + (size_t)(base + (i / sub) * step) * kPrefixRecFloats;
        const float x = rec[slot + (i % sub) * 128];
        m = fmaxf(m, x);
        v = fmaxf(v, x);
    }
    const float mr = finite_ref(m), vr = finite_ref(v);
    float l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < p.splits; ++i) {
        const float* rec = own + (size_t)i * kOwnRecFloats;
        l += rec[8 + h] * fast_exp2(rec[h] - mr);
        const float w = fast_exp2(rec[16 + h] - vr);
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = fmaf(rec[32 + (d0 + 32 * k) * 8 + h], w, o[k]);
    }
    for (int i = 0; i < items * sub; ++i) {
        const float* rec = p.prefix_part + (size_t)(base + (i / sub) * step) * kPrefixRecFloats;
        const int sl = slot + (i % sub) * 128;
        const float x = rec[sl];
        if (x == -INFINITY) continue;   // no key: its values were not written
        l += rec[kPrefixRows + sl] * fast_exp2(x - mr);
        const float w = fast_exp2(x - vr);
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = fmaf(rec[2 * kPrefixRows + (d0 + 32 * k) * kPrefixRows + sl], w, o[k]);
    }
    const bool none = m == -INFINITY && l == 0.f;    // nothing to attend to
    const float f = none ? 0.f : fast_exp2(v - m) / l;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        s_out[h * kHeadDim + d0 + 32 * k] = __float2bfloat16_rn(!fits ? NAN : none ? 0.f : o[k] * f);
    __syncthreads();
    if (threadIdx.x < p.g * 16) {
        uint4* orow = reinterpret_cast<uint4*>(p.out + ((size_t)seq * p.h_q + (size_t)head * p.g) * kHeadDim);
        orow[threadIdx.x] = reinterpret_cast<const uint4*>(s_out)[threadIdx.x];
    }
    if (p.lse && d0 == 0 && h < p.g)
        p.lse[(size_t)seq * p.h_q + (size_t)head * p.g + h] = !fits ? NAN : none ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
    if (p.len_out && head == 0 && threadIdx.x == 0 && fits) p.len_out[seq] += 1;
}

template <int F, int U>
static void launch_own(const StoreAttnLaunch& p, bool part, cudaStream_t s) {
    const unsigned grid = (unsigned)(p.batch * p.h_kv * p.splits);
    if (part) gkv_store_attn_kernel<F, U, true><<<grid, kThreads, 0, s>>>(p);
    else gkv_store_attn_kernel<F, U, false><<<grid, kThreads, 0, s>>>(p);
}
cudaError_t launch_store_attn(const StoreAttnLaunch& p, cudaStream_t s) {
    const bool part = p.splits > 1 || p.prefix_part != nullptr || p.len_out != nullptr;
    switch (p.format) {
        case GKV_STORE_BF16: launch_own<GKV_STORE_BF16, 1>(p, part, s); break;
        case GKV_STORE_E4M3: launch_own<GKV_STORE_E4M3, 2>(p, part, s); break;
        case GKV_STORE_INT8: launch_own<GKV_STORE_INT8, 2>(p, part, s); break;
        default:             launch_own<GKV_STORE_INT4, 2>(p, part, s); break;
    }
    return cudaGetLastError();
}
cudaError_t launch_store_merge(const StoreAttnLaunch& p, cudaStream_t s) {
    gkv_store_merge_kernel<<<(unsigned)(p.batch * p.h_kv), 256, 0, s>>>(p);
    return cudaGetLastError();
}

}  // namespace gkv
