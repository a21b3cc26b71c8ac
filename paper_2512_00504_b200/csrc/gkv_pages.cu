// Appending rows to a cache in pages, with keys rotated on the way, and reading them back.
//
// Two things more than in the copies of a store: a token's row is found through the table, and keys are rotated. cos and sin depend on
// the token and the pair alone, and cost more than all else that is done to a pair. So a half warp that appends has the heads of one token (up to
// kRun rows, all of whose loads start first) and holds the cos and sin of its lanes' elements in registers; the CTA works them out once for its
// tokens, through shared memory. (With kRun tokens of one head instead, as the store's copies go, every row reads its own cos and sin from
// shared memory: 4 x 32768 tokens x 8 heads in bf16 302 us.) K and V take turns in the grid, so that K's arithmetic runs while V moves. A lane has
// 8 neighbouring elements, those on the other side of their pairs come from another lane (4 bits: of the order that lets its codes be one
// store, where the pairs allow it; turned in the plain order and exchanged afterwards, the same rows in 4 bits took 180 us instead of 158). What
// is rotated is rounded to bf16 and goes on from there as if it had been read, so that a fused append leaves the bits that rotating first would.
// Scales of one head's rows lie next to one another in a page while a half warp has different heads: the CTA gathers them in shared memory and
// writes those of its tokens together.
//
// What bounds it: bf16 rows HBM; quantised ones that are rotated the issue of instructions. So fp32 operations go in pairs, the number of heads is
// known at compile time where it can be, pairs half a head apart have a way of their own, and registers are held to eight CTAs an SM (8 bits: 174 us
// without all of it, 155 with the first two, 148 with three, 132 with all).
//
// Reading back takes kRun tokens of a head, so that scales come with one access.
//
// Measured: 4 x 32768 tokens x 8 heads, rotated: in bf16 160 us (1.07 GB, 6.7 TB/s), in 8 bits 132 to 140, in 4 bits 141 to 150; without the rotation 164,
// 120 and 102 to 105; back in 162, 127 and 109. 8 prompts of 129 to 4097 tokens x 4 heads 17 to 18 us (without the rotation 16, 13.3, 12.5), back in 16.1,
// 13.6 and 12.1. One token of 32 sequences x 4 heads: 2.3 us in bf16, 2.8 to 3.1 in the others (1.7 and 2.4 without the rotation), back in 2.
#include "gkv_pages.cuh"
#include "gkv_rotary.cuh"
#include "gkv_store_rows.h"

namespace gkv {

constexpr int kPageCopyThreads = 128;
constexpr int kPageCopyItems = kPageCopyThreads / 16;

// The 8 elements of a row that lane l has, neighbours or those of format F. These loads stay where they are written: all of them ahead of
// what they are to overlap with. (Left to the compiler, they were put off to the rows' turn where registers were short: an append of
// ragged prompts in 8 bits took 31 us instead of 21.)
template <int F>
__device__ __forceinline__ uint4 load_row(const __nv_bfloat16* row, int l, bool neighbours) {
    uint4 r;
    if (F != GKV_STORE_INT4 || neighbours) {
        asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(row + 8 * l) : "memory");
    } else {
        const __nv_bfloat16* x = row + 64 * (l & 1) + 4 * (l >> 1);
        asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(x) : "memory");
        asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(r.z), "=r"(r.w) : "l"(x + 32) : "memory");
    }
    return r;
}

// How keys are turned: not at all; pairs that are neighbours, rot_dim a multiple of a lane's 8 elements; pairs half a head apart; pairs another
// multiple of 8 elements apart; any others.
enum { kStraight = 0, kNeighbours = 1, kWhole = 2, kLanes = 3, kAny = 4 };
// Where a row's lanes hold its elements in the order of 4-bit codes from the start: elements 4i .. 4i + 3 with i = l / 2 + 16 (l % 2), and
// 32 further on. The other sides of pairs half a head apart are then lane l ^ 1's, those of neighbours its own.
template <int F, int OP> constexpr bool kCodeOrder = F == GKV_STORE_INT4 && OP <= kWhole;

// cos and sin of what a lane has of a token: of the pairs of its 8 elements, sin negated where it has the first sides, or (neighbours) of its 4
// pairs.
template <int F, int OP>
struct LaneTurn {
    static constexpr int N = OP == kNeighbours ? 1 : 2;
    float4 c[N], s[N];
    __device__ __forceinline__ void load(int l, int half, const float* cos, const float* sin) {
        if constexpr (OP == kNeighbours && kCodeOrder<F, OP>) {
            const int at = 2 * (l >> 1) + 32 * (l & 1);
            float2 x[2] = {}, y[2] = {};
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (at + 16 * i < half) {
                    x[i] = *reinterpret_cast<const float2*>(cos + at + 16 * i);
                    y[i] = *reinterpret_cast<const float2*>(sin + at + 16 * i);
                }
            c[0] = make_float4(x[0].x, x[0].y, x[1].x, x[1].y);
            s[0] = make_float4(y[0].x, y[0].y, y[1].x, y[1].y);
        } else {
            const int first = OP == kWhole && kCodeOrder<F, OP> ? 4 * (l >> 1) : 8 * l, next = OP == kWhole && kCodeOrder<F, OP> ? 32 : 4;
            const bool negate = OP == kWhole && kCodeOrder<F, OP> ? (l & 1) == 0 : OP != kNeighbours && 8 * l < half;
            const int at = OP == kNeighbours ? 4 * l : first < half ? first : first - half;      // (lanes behind the pairs: not used)
            if (OP == kWhole || (OP == kNeighbours ? at < half : 8 * l < 2 * half))
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    c[i] = *reinterpret_cast<const float4*>(cos + at + next * i);
                    const float4 x = *reinterpret_cast<const float4*>(sin + at + next * i);
                    s[i] = negate ? make_float4(-x.x, -x.y, -x.z, -x.w) : x;
                }
        }
    }
};
// A lane's 8 elements of a row, turned: x c + y s with y the other sides of their pairs, the products in the order of rotary_turn.
template <int F, int OP>
__device__ __forceinline__ uint4 turn_lane(const LaneTurn<F, OP>& r, uint4 v, int l, int half) {
    const uint32_t x[4] = {v.x, v.y, v.z, v.w};
    const int from = OP == kWhole ? (kCodeOrder<F, OP> ? l ^ 1 : l ^ 8) : 8 * l < half ? l + half / 8 : l - half / 8;
    uint32_t y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 a = make_float2(bf16_lo(x[i]), bf16_hi(x[i]));
        float2 t;
        if constexpr (OP == kNeighbours) {
            const float c = i == 0 ? r.c[0].x : i == 1 ? r.c[0].y : i == 2 ? r.c[0].z : r.c[0].w;
            const float s = i == 0 ? r.s[0].x : i == 1 ? r.s[0].y : i == 2 ? r.s[0].z : r.s[0].w;
            t = fma2(a, make_float2(c, c), mul2(make_float2(-a.y, a.x), make_float2(s, s)));
        } else {
            const uint32_t o = __shfl_sync(0xffffffffu, x[i], from, 16);
            const float4 c4 = r.c[i >> 1], s4 = r.s[i >> 1];
            const float2 c = i & 1 ? make_float2(c4.z, c4.w) : make_float2(c4.x, c4.y), s = i & 1 ? make_float2(s4.z, s4.w) : make_float2(s4.x, s4.y);
            t = fma2(a, c, mul2(make_float2(bf16_lo(o), bf16_hi(o)), s));
        }
        y[i] = pack_bf16x2(t.x, t.y);
    }
    if (OP == kWhole || half == 64) return make_uint4(y[0], y[1], y[2], y[3]);
    if constexpr (kCodeOrder<F, OP>) {
        const int at = 4 * (l >> 1) + 64 * (l & 1);
        const bool p = at < 2 * half, q = at + 32 < 2 * half;
        return make_uint4(p ? y[0] : v.x, p ? y[1] : v.y, q ? y[2] : v.z, q ? y[3] : v.w);
    }
    return 8 * l < 2 * half ? make_uint4(y[0], y[1], y[2], y[3]) : v;
}
// The same element by element, for any rot_dim and either order of pairs, with cos and sin from shared memory.
__device__ __forceinline__ uint4 turn_any(uint4 v, int l, const RotaryView& r, const __nv_bfloat16* row, const float* cos, const float* sin) {
    uint32_t x[4] = {v.x, v.y, v.z, v.w};
    const uint16_t* e = reinterpret_cast<const uint16_t*>(row);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int d = 8 * l + i;
        if (row && d < 2 * r.half) {
            const bool first = r.interleaved ? i % 2 == 0 : d < r.half;
            const int pair = r.interleaved ? d >> 1 : first ? d : d - r.half;
            const int o = r.interleaved ? d ^ 1 : first ? d + r.half : d - r.half;
            const float a = i & 1 ? bf16_hi(x[i >> 1]) : bf16_lo(x[i >> 1]), b = __uint_as_float((uint32_t)e[o] << 16);
            const float y = __fmaf_rn(a, cos[pair], __fmul_rn(first ? -b : b, sin[pair]));
            const uint32_t w = pack_bf16x2(y, y);
            x[i >> 1] = i & 1 ? __byte_perm(x[i >> 1], w, 0x5410) : __byte_perm(x[i >> 1], w, 0x3254);
        }
    }
    return make_uint4(x[0], x[1], x[2], x[3]);
}
// A row whose lanes have 8 neighbouring elements each -> the elements that lane l has in format F.
template <int F>
__device__ __forceinline__ uint4 as_format(uint4 v, int l) {
    if constexpr (F != GKV_STORE_INT4) return v;
    const int q = l >> 1, from = 8 * (l & 1) + (q >> 1);
    uint32_t w[2][4];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        w[k][0] = __shfl_sync(0xffffffffu, v.x, from + 4 * k, 16);
        w[k][1] = __shfl_sync(0xffffffffu, v.y, from + 4 * k, 16);
        w[k][2] = __shfl_sync(0xffffffffu, v.z, from + 4 * k, 16);
        w[k][3] = __shfl_sync(0xffffffffu, v.w, from + 4 * k, 16);
    }
    return q & 1 ? make_uint4(w[0][2], w[0][3], w[1][2], w[1][3]) : make_uint4(w[0][0], w[0][1], w[1][0], w[1][1]);
}

// CTA: K or V, heads_per_cta heads, 8 * tokens_per_half tokens of sequence blockIdx.y. Half warp w: tokens_per_half tokens from w *
// tokens_per_half on, all those heads of each (at most R rows).
// CTAs an SM that a kernel's registers are held to (0: as the compiler would have it). Rows that are rotated and quantised do better with eight,
// which hides their arithmetic, although a few registers are spilled (in 8 bits 132 us instead of 147 with six; nine 140); the others wait for memory, and
// do better with all loads under way (bf16 160 us, with eight 173; in 8 bits without a rotation 120 and 148).
__host__ __device__ constexpr int append_ctas(int format, int op, int rows) {
    return rows != kRun || op == kStraight || op == kAny ? 0 : format == GKV_STORE_BF16 ? 1 : 8;
}
template <int F, int OP, int R, int H>
__global__ void __launch_bounds__(kPageCopyThreads, append_ctas(F, OP, R)) gkv_pages_append_kernel(const PagesCopyLaunch p) {
    using Fm = StoreFormat<F>;
    constexpr int kLanesOfRow = 16 / R;                  // that have its scales
    extern __shared__ __align__(16) float s_table[];     // cos and sin of the CTA's tokens: [token][half] each
    __shared__ uint32_t s_row[kPageCopyItems * R];    // [token]: number of head 0's row
    __shared__ uint2 s_scale[kPageCopyItems * R];     // [head][token]
    const int heads_per_cta = H ? H : p.heads_per_cta, tokens_per_half = H ? R / H : p.tokens_per_half;
    const int b = blockIdx.y, l = threadIdx.x & 15, w = threadIdx.x >> 4;
    const bool is_v = blockIdx.x & 1;
    const int block = blockIdx.x >> 1, head_block = block % p.head_blocks;
    const int tokens = kPageCopyItems * tokens_per_half, t0 = block / p.head_blocks * tokens;
    const int head0 = head_block * heads_per_cta, heads = H ? H : min(heads_per_cta, p.h_kv - head0);
    const int half = p.rotary.half;
    const bool turns = OP != kStraight && !is_v;
    // This thread's pairs are those of its number and, blockDim by blockDim, on through the tokens: where a token's pairs divide the threads
    // (the usual case) always the same one, whose frequency is on its way while the count is.
    int token = 0, pair = 0;
    uint64_t frequency = 0;
    if (turns) {
        token = threadIdx.x / half;
        pair = threadIdx.x - token * half;
        frequency = p.rotary.turns[pair];
    }
    const int32_t first = p.first ? p.first[b] : 0, count = p.count ? p.count[b] : p.n_tokens;
    const int n = min(count, p.n_tokens);
    if (t0 >= n) return;
    const int t_half = t0 + w * tokens_per_half;       // the half warp's first token

    // lane l's token of the half warp, as far as there is one, and what the table has for its row
    const int mine = t_half + l;
    const RunRows one = run_rows(first, n, p.n_tokens, p.capacity, mine);
    const bool there = l < tokens_per_half && mine < n && one.lo == 0 && one.hi > 0;
    const int32_t entry = there ? page_entry(p.pages, p.pages.table + b * p.pages.table_stride, first + mine) : 0;
    // Row k is head k % heads_per_cta of token k / heads_per_cta.
    const int rows = tokens_per_half * heads_per_cta;
    const __nv_bfloat16* const x = (is_v ? p.x[1] : p.x[0]) + ((int64_t)b * p.seq_stride + (int64_t)t_half * p.token_stride + (int64_t)head0 * p.head_stride);
    const int64_t next_token = p.token_stride - (heads_per_cta - 1) * p.head_stride;
    uint4 v[R];
    {
        const __nv_bfloat16* src = x;
        int t = t_half, h = 0;
#pragma unroll
        for (int k = 0; k < R; ++k) {
            v[k] = make_uint4(0u, 0u, 0u, 0u);
            if (k < rows && h < heads && t < n) v[k] = load_row<F>(src, l, turns && !kCodeOrder<F, OP>);
            if (++h == heads_per_cta) { h = 0; ++t; src += next_token; }
            else src += p.head_stride;
        }
    }
    const uint32_t row = there ? page_row(p.pages, entry, (uint32_t)head0 * p.pages.head_rows, first + mine) : kNoRow;
    if (OP != kStraight && turns) {
        float* s_sin = s_table + tokens * half;
        const int dk = kPageCopyThreads / half, dp = kPageCopyThreads - dk * half, end = min(n - t0, tokens) * half;
        for (int i = threadIdx.x; i < end; i += kPageCopyThreads) {
            const int t = t0 + token;
            const int32_t pos = p.pos ? p.pos[(int64_t)b * p.pos_seq_stride + (int64_t)t * p.pos_token_stride]
                                      : (int32_t)((uint32_t)first + (uint32_t)t);
            const float2 cs = rotary_cos_sin(frequency, pos, p.rotary.factor, 1.f);
            s_table[i] = cs.x;
            s_sin[i] = cs.y;
            token += dk;
            if (dp) {
                pair += dp;
                if (pair >= half) { pair -= half; ++token; }
                frequency = p.rotary.turns[pair];
            }
        }
        __syncthreads();
        int k0 = w * tokens_per_half, h = 0;           // token within the CTA, head
        if constexpr (OP == kAny) {
            const __nv_bfloat16* src = x;
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (k < rows)
                    v[k] = as_format<F>(turn_any(v[k], l, p.rotary, h < heads && t0 + k0 < n ? src : nullptr, s_table + k0 * half, s_sin + k0 * half), l);
                if (++h == heads_per_cta) { h = 0; ++k0; src += next_token; }
                else src += p.head_stride;
            }
        } else {
            LaneTurn<F, OP> r;
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (k < rows) {
                    if (h == 0) r.load(l, half, s_table + k0 * half, s_sin + k0 * half);
                    v[k] = turn_lane<F, OP>(r, v[k], l, half);
                    if constexpr (!kCodeOrder<F, OP>) v[k] = as_format<F>(v[k], l);
                }
                if (++h == heads_per_cta) { h = 0; ++k0; }
            }
        }
    }

    uint8_t* data = is_v ? p.pages.data[1] : p.pages.data[0];
    if (Fm::kScales != 0 && l < tokens_per_half) s_row[w * tokens_per_half + l] = row;
    float inv0 = 1.f, inv1 = 1.f;
    if (Fm::kScales != 0) {
        const uint32_t sc = store_run_scales<F>(v, l, &inv0, &inv1);
        const int k = l / kLanesOfRow, i = k / heads_per_cta, h = k - i * heads_per_cta;
        if (k < rows && l % kLanesOfRow < (F == GKV_STORE_INT4 ? 2 : 1))
            reinterpret_cast<uint32_t*>(s_scale + h * tokens + w * tokens_per_half + i)[F == GKV_STORE_INT4 ? l & 1 : 0] = sc;
    }
    {
        const size_t head_bytes = (size_t)p.pages.head_rows * Fm::kRow;
        uint32_t at = __shfl_sync(0xffffffffu, row, 0, 16);
        uint8_t* dst = data + (size_t)at * Fm::kRow;
        int i = 0, h = 0;
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int from = k * kLanesOfRow + (F == GKV_STORE_INT4 ? l & 1 : 0);
            float f0 = 1.f, f1 = 1.f;
            if (Fm::kScales != 0) f0 = f1 = __shfl_sync(0xffffffffu, inv0, from, 16);
            if (F == GKV_STORE_INT4) f1 = __shfl_sync(0xffffffffu, inv1, from, 16);
            if (k < rows && h < heads && at < kNoPage) store_put_codes<F>(dst, l, store_codes<F>(v[k], f0, f1));
            dst += head_bytes;
            if (++h == heads_per_cta) {
                h = 0;
                at = __shfl_sync(0xffffffffu, row, ++i, 16);
                dst = data + (size_t)at * Fm::kRow;
            }
        }
    }
    if (Fm::kScales != 0) {
        __syncthreads();
        __nv_bfloat16* scale = is_v ? p.pages.scale[1] : p.pages.scale[0];
        const int h = threadIdx.x / tokens, t = threadIdx.x - h * tokens;
        if (h < heads) {
            const uint32_t at = s_row[t];
            if (at < kNoPage) {
                __nv_bfloat16* dst = scale + (size_t)(at + h * p.pages.head_rows) * Fm::kScales;
                if (F == GKV_STORE_INT4) *reinterpret_cast<uint2*>(dst) = s_scale[threadIdx.x];
                else *reinterpret_cast<uint16_t*>(dst) = (uint16_t)s_scale[threadIdx.x].x;
            }
        }
    }
}

// Work item i of sequence blockIdx.y: head i % h_kv, tokens kRun * (i / h_kv) and on; blockIdx.z = K or V.
template <int F>
__global__ void __launch_bounds__(kPageCopyThreads) gkv_pages_read_kernel(const PagesCopyLaunch p) {
    using Fm = StoreFormat<F>;
    const int b = blockIdx.y, l = threadIdx.x & 15;
    const bool is_v = blockIdx.z != 0;
    const int item = blockIdx.x * kPageCopyItems + (threadIdx.x >> 4);
    const int h = item % p.h_kv, t0 = item / p.h_kv * kRun;
    const int32_t first = p.first ? p.first[b] : 0;
    // the whole warp stays for the shuffles, whatever the run has
    const RunRows rows = run_rows(first, p.count ? p.count[b] : p.n_tokens, p.n_tokens, p.capacity, t0);
    __nv_bfloat16* x = (is_v ? p.x[1] : p.x[0]) + (int64_t)b * p.seq_stride + (int64_t)t0 * p.token_stride + (int64_t)h * p.head_stride;
    const uint8_t* data = is_v ? p.pages.data[1] : p.pages.data[0];
    const __nv_bfloat16* scale = is_v ? p.pages.scale[1] : p.pages.scale[0];
    // lane l's row: that of token l & 7 of the run
    const int mine = l & (kRun - 1);
    uint32_t row = kNoRow;
    if (mine >= rows.lo && mine < rows.hi) {
        const int r = first + t0 + mine;               // (within 0 .. capacity - 1)
        row = page_row(p.pages, page_entry(p.pages, p.pages.table + b * p.pages.table_stride, r), (uint32_t)h * p.pages.head_rows, r);
    }
    uint4 v[kRun];
    uint32_t at[kRun];
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        at[i] = __shfl_sync(0xffffffffu, row, i, 16);
        v[i] = at[i] < kNoPage ? store_get_codes<F>(data + (size_t)at[i] * Fm::kRow, l) : make_uint4(0u, 0u, 0u, 0u);
    }
    // Scales are held by lane 2i + j: in 4 bits those of groups 2j, 2j + 1 of token i, in 8 bits that of token i.
    const uint32_t scale_row = __shfl_sync(0xffffffffu, row, l >> 1, 16);
    uint32_t sc = 0u;
    if (Fm::kScales != 0 && scale_row < kNoPage)
        sc = F == GKV_STORE_INT4 ? *(reinterpret_cast<const uint32_t*>(scale) + (size_t)scale_row * 2 + (l & 1))
                                 : *(reinterpret_cast<const uint16_t*>(scale) + scale_row);
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        const uint32_t s = __shfl_sync(0xffffffffu, sc, 2 * i + (F == GKV_STORE_INT4 ? l & 1 : 0), 16);
        if (at[i] < kNoPage) store_put_target<F>(x + (int64_t)i * p.token_stride, l, store_decode<F>(v[i], s));
    }
}

template <int OP, int R, int H>
static cudaError_t launch_append_rows(const PagesCopyLaunch& p, cudaStream_t s) {
    const int tokens = kPageCopyItems * p.tokens_per_half;
    const dim3 grid((unsigned)((p.n_tokens + tokens - 1) / tokens) * p.head_blocks * 2, (unsigned)p.batch);
    const size_t smem = OP != kStraight ? (size_t)tokens * p.rotary.half * 2 * sizeof(float) : 0;
    switch (p.format) {
        case GKV_STORE_BF16: gkv_pages_append_kernel<GKV_STORE_BF16, OP, R, H><<<grid, kPageCopyThreads, smem, s>>>(p); break;
        case GKV_STORE_E4M3: gkv_pages_append_kernel<GKV_STORE_E4M3, OP, R, H><<<grid, kPageCopyThreads, smem, s>>>(p); break;
        case GKV_STORE_INT8: gkv_pages_append_kernel<GKV_STORE_INT8, OP, R, H><<<grid, kPageCopyThreads, smem, s>>>(p); break;
        default:             gkv_pages_append_kernel<GKV_STORE_INT4, OP, R, H><<<grid, kPageCopyThreads, smem, s>>>(p); break;
    }
    return cudaGetLastError();
}
template <int OP>
static cudaError_t launch_append(PagesCopyLaunch p, cudaStream_t s) {
    // Two rows a half warp, whose chain is shorter, as long as that leaves no more than three CTAs an SM (one token of 32 sequences x 4 heads in 8
    // bits, 128 CTAs, 2.8 us with two, 4.4 with eight; 1024 tokens of one, 512 CTAs, 3.85 and 3.67; 128 x 8 heads, 1024 CTAs, 4.3 and 3.6).
    auto shape = [&](int rows) {
        p.head_blocks = (p.h_kv + rows - 1) / rows;
        p.heads_per_cta = (p.h_kv + p.head_blocks - 1) / p.head_blocks;
        p.tokens_per_half = rows / p.heads_per_cta;
        const int tokens = kPageCopyItems * p.tokens_per_half;
        return (int64_t)((p.n_tokens + tokens - 1) / tokens) * p.head_blocks * 2 * p.batch;
    };
    if (shape(2) <= 3 * device_sm_count()) return launch_append_rows<OP, 2, 0>(p, s);
    shape(kRun);
    if constexpr (OP <= kWhole) {
        const bool even = p.heads_per_cta * p.head_blocks == p.h_kv;
        if (even && p.heads_per_cta == 8) return launch_append_rows<OP, kRun, 8>(p, s);
        if (even && p.heads_per_cta == 4) return launch_append_rows<OP, kRun, 4>(p, s);
    }
    return launch_append_rows<OP, kRun, 0>(p, s);
}
cudaError_t launch_pages_append(const PagesCopyLaunch& p, cudaStream_t s) {
    if (!p.rotary.turns) return launch_append<kStraight>(p, s);
    if (!p.rotary.interleaved && p.rotary.half == 64) return launch_append<kWhole>(p, s);
    if (p.rotary.interleaved) return p.rotary.half % 4 == 0 ? launch_append<kNeighbours>(p, s) : launch_append<kAny>(p, s);
    return p.rotary.half % 8 == 0 ? launch_append<kLanes>(p, s) : launch_append<kAny>(p, s);
}
cudaError_t launch_pages_read(const PagesCopyLaunch& p, cudaStream_t s) {
    const int items = (p.n_tokens + kRun - 1) / kRun * p.h_kv;
    const dim3 grid((unsigned)((items + kPageCopyItems - 1) / kPageCopyItems), (unsigned)p.batch, 2);
    switch (p.format) {
        case GKV_STORE_BF16: gkv_pages_read_kernel<GKV_STORE_BF16><<<grid, kPageCopyThreads, 0, s>>>(p); break;
        case GKV_STORE_E4M3: gkv_pages_read_kernel<GKV_STORE_E4M3><<<grid, kPageCopyThreads, 0, s>>>(p); break;
        case GKV_STORE_INT8: gkv_pages_read_kernel<GKV_STORE_INT8><<<grid, kPageCopyThreads, 0, s>>>(p); break;
        default:             gkv_pages_read_kernel<GKV_STORE_INT4><<<grid, kPageCopyThreads, 0, s>>>(p); break;
    }
    return cudaGetLastError();
}

}  // namespace gkv
