// Appending rows to a cache in pages, with keys rotated on the way, and reading them back.
//
// As the copies of a store (half a warp takes kRun tokens of a head, all loads first), bound by HBM, with two things more. A token's row
// is found through the table: eight lanes look up the eight tokens of the run while its loads are on their way, and hand the rows
// round. And keys are rotated: cos and sin depend on the token and the pair alone, so a CTA works them out once for the tokens
// of its runs, in shared memory, for all heads that it has of them. Pairs (i, i + rot_dim / 2) lie in two lanes; the partner's elements are
// loaded a second time, which the L1 answers, and each lane turns its own side. What is rotated is rounded to bf16 and goes on from
// there as if it had been read, so that a fused append leaves the bits that rotating first would.
#include "gkv_pages.cuh"
#include "gkv_rotary.cuh"
#include "gkv_store_rows.h"

namespace gkv {

constexpr int kPageCopyThreads = 128;
constexpr int kPageCopyItems = kPageCopyThreads / 16;

// What a copy does to K: moves it out, in as it is, or in with the rotation of pairs that are neighbours, that lie half of rot_dim apart (a
// multiple of 4 elements), or the same by single elements.
enum { kRead = 0, kWrite = 1, kWriteNeighbours = 2, kWriteHalves = 3, kWriteAny = 4 };

// First element of a lane's first and last four.
template <int F> __device__ __forceinline__ int lane_dim(int l, int which) {
    return F == GKV_STORE_INT4 ? 64 * (l & 1) + 4 * (l >> 1) + 32 * which : 8 * l + 4 * which;
}

// Four elements of a row (elements e .. e + 3, two packed words) turned. partner: the other sides of their pairs, where those are not
// among them; c, s: cos and sin of the token's pairs.
template <int OP>
__device__ __forceinline__ uint2 rotate_four(uint2 x, uint2 partner, int e, int half, const float* c, const float* s) {
    float v[4] = {bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y)};
    if (OP == kWriteNeighbours) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int pair = (e >> 1) + i;
            if (pair < half) {
                const float2 r = rotary_turn(v[2 * i], v[2 * i + 1], c[pair], s[pair]);
                v[2 * i] = r.x; v[2 * i + 1] = r.y;
            }
        }
    } else {
        const float w[4] = {bf16_lo(partner.x), bf16_hi(partner.x), bf16_lo(partner.y), bf16_hi(partner.y)};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = e + i;                       // (halves a multiple of 4 apart: all four are on the same side)
            if (d < half) v[i] = rotary_turn(v[i], w[i], c[d], s[d]).x;
            else if (d < 2 * half) v[i] = rotary_turn(w[i], v[i], c[d - half], s[d - half]).y;
        }
    }
    return make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}
// The partners of elements e .. e + 3 of a row.
template <int OP>
__device__ __forceinline__ uint2 load_partner(const __nv_bfloat16* row, int e, int half) {
    if constexpr (OP == kWriteHalves) {
        if (e >= 2 * half) return make_uint2(0u, 0u);
        return *reinterpret_cast<const uint2*>(row + (e < half ? e + half : e - half));
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = e + i;
            w[i] = d < 2 * half ? reinterpret_cast<const uint16_t*>(row)[d < half ? d + half : d - half] : 0u;
        }
        return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    }
}

// Work item i of sequence blockIdx.y: head i % h_kv, tokens kRun * (i / h_kv) and on; blockIdx.z = K or V.
template <int F, int OP>
__global__ void __launch_bounds__(kPageCopyThreads) gkv_pages_copy_kernel(const PagesCopyLaunch p) {
    using Fm = StoreFormat<F>;
    extern __shared__ __align__(16) float s_table[];   // cos and sin of the CTA's tokens: [token][half] each
    const int b = blockIdx.y, l = threadIdx.x & 15;
    const bool is_v = blockIdx.z != 0;
    const int item0 = blockIdx.x * kPageCopyItems, item = item0 + (threadIdx.x >> 4);
    const int h = item % p.h_kv, t0 = item / p.h_kv * kRun;
    const int32_t first = p.first ? p.first[b] : 0, count = p.count ? p.count[b] : p.n_tokens;
    // the whole warp stays for the shuffles, whatever the run has
    const RunRows rows = run_rows(first, count, p.n_tokens, p.capacity, t0);
    const int lo = rows.lo, hi = rows.hi;
    const int half = p.rotary.half;
    const bool rotates = OP >= kWriteNeighbours && !is_v;
    __nv_bfloat16* x = (is_v ? p.x[1] : p.x[0]) + (int64_t)b * p.seq_stride + (int64_t)t0 * p.token_stride + (int64_t)h * p.head_stride;

    // lane l's row: that of token l & 7 of the run
    const int mine = l & (kRun - 1);
    uint32_t row = kNoRow;
    if (mine >= lo && mine < hi) {
        const int r = first + t0 + mine;               // (within 0 .. capacity - 1)
        row = page_row(p.pages, page_entry(p.pages, p.pages.table + b * p.pages.table_stride, r), (uint32_t)h * p.pages.head_rows, r);
    }
    uint4 v[kRun];
    uint2 w[kRun][2];                                  // partners
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        v[i] = make_uint4(0u, 0u, 0u, 0u);
        if (OP != kRead && i >= lo && i < hi) {
            const __nv_bfloat16* src = x + (int64_t)i * p.token_stride;
            v[i] = store_load_source<F>(src, l);
            if (OP >= kWriteHalves && rotates)
#pragma unroll
                for (int k = 0; k < 2; ++k) w[i][k] = load_partner<OP>(src, lane_dim<F>(l, k), half);
        }
    }
    const int run0 = item0 / p.h_kv;                   // of the CTA's first item
    if (OP >= kWriteNeighbours && rotates) {
        const int last = min((item0 + kPageCopyItems - 1) / p.h_kv, (p.n_tokens - 1) / kRun);
        const int tokens = (last - run0 + 1) * kRun;
        const int n = count < p.n_tokens ? count : p.n_tokens;
        float* s_sin = s_table + tokens * half;
        for (int i = threadIdx.x; i < tokens * half; i += kPageCopyThreads) {
            const int k = i / half, pair = i - k * half, t = run0 * kRun + k;
            if (t < n) {
                const int32_t pos = p.pos ? p.pos[(int64_t)b * p.pos_seq_stride + (int64_t)t * p.pos_token_stride]
                                          : (int32_t)((uint32_t)first + (uint32_t)t);
                const float2 cs = rotary_cos_sin(p.rotary.turns[pair], pos, p.rotary.factor, 1.f);
                s_table[i] = cs.x;
                s_sin[i] = cs.y;
            }
        }
        __syncthreads();
        const float* c = s_table + (t0 - run0 * kRun) * half;
        const float* s = s_sin + (t0 - run0 * kRun) * half;
#pragma unroll
        for (int i = 0; i < kRun; ++i)
            if (i >= lo && i < hi) {
                const uint2 a = rotate_four<OP>(make_uint2(v[i].x, v[i].y), w[i][0], lane_dim<F>(l, 0), half, c + i * half, s + i * half);
                const uint2 z = rotate_four<OP>(make_uint2(v[i].z, v[i].w), w[i][1], lane_dim<F>(l, 1), half, c + i * half, s + i * half);
                v[i] = make_uint4(a.x, a.y, z.x, z.y);
            }
    }

    uint8_t* data = is_v ? p.pages.data[1] : p.pages.data[0];
    __nv_bfloat16* scale = is_v ? p.pages.scale[1] : p.pages.scale[0];
    // Scales are held and moved by lane 2i + j: in 4 bits those of groups 2j, 2j + 1 of token i, in 8 bits that of token i (the
    // odd lane has a copy).
    const uint32_t scale_row = __shfl_sync(0xffffffffu, row, l >> 1, 16);
    const bool has_scale = Fm::kScales != 0 && scale_row < kNoPage && (F == GKV_STORE_INT4 || (l & 1) == 0);
    uint32_t* scale4 = reinterpret_cast<uint32_t*>(scale) + (size_t)scale_row * 2 + (l & 1);
    uint16_t* scale2 = reinterpret_cast<uint16_t*>(scale) + scale_row;
    if (OP == kRead) {
        uint32_t at[kRun];
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            at[i] = __shfl_sync(0xffffffffu, row, i, 16);
            if (at[i] < kNoPage) v[i] = store_get_codes<F>(data + (size_t)at[i] * Fm::kRow, l);
        }
        uint32_t sc = 0u;
        if (has_scale) sc = F == GKV_STORE_INT4 ? *scale4 : *scale2;
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            const uint32_t s = __shfl_sync(0xffffffffu, sc, 2 * i + (F == GKV_STORE_INT4 ? l & 1 : 0), 16);
            if (at[i] < kNoPage) store_put_target<F>(x + (int64_t)i * p.token_stride, l, store_decode<F>(v[i], s));
        }
        return;
    }
    float inv0 = 1.f, inv1 = 1.f;
    if (Fm::kScales != 0) {
        const uint32_t sc = store_run_scales<F>(v, l, &inv0, &inv1);
        if (has_scale) {
            if (F == GKV_STORE_INT4) *scale4 = sc;
            else *scale2 = (uint16_t)sc;
        }
    }
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        const int from = 2 * i + (F == GKV_STORE_INT4 ? l & 1 : 0);
        float f0 = 1.f, f1 = 1.f;
        if (Fm::kScales != 0) f0 = f1 = __shfl_sync(0xffffffffu, inv0, from, 16);
        if (F == GKV_STORE_INT4) f1 = __shfl_sync(0xffffffffu, inv1, from, 16);
        const uint32_t at = __shfl_sync(0xffffffffu, row, i, 16);
        if (at < kNoPage) store_put_codes<F>(data + (size_t)at * Fm::kRow, l, store_codes<F>(v[i], f0, f1));
    }
}

template <int OP>
static cudaError_t launch_copy(const PagesCopyLaunch& p, cudaStream_t s) {
    const int items = (p.n_tokens + kRun - 1) / kRun * p.h_kv;
    const dim3 grid((unsigned)((items + kPageCopyItems - 1) / kPageCopyItems), (unsigned)p.batch, 2);
    // runs that a CTA's items touch: h_kv items each, and the first may start inside one
    const int runs = kPageCopyItems % p.h_kv == 0 ? kPageCopyItems / p.h_kv : (kPageCopyItems - 2) / p.h_kv + 2;
    const size_t smem = OP >= kWriteNeighbours ? (size_t)runs * kRun * p.rotary.half * 2 * sizeof(float) : 0;
    switch (p.format) {
        case GKV_STORE_BF16: gkv_pages_copy_kernel<GKV_STORE_BF16, OP><<<grid, kPageCopyThreads, smem, s>>>(p); break;
        case GKV_STORE_E4M3: gkv_pages_copy_kernel<GKV_STORE_E4M3, OP><<<grid, kPageCopyThreads, smem, s>>>(p); break;
        case GKV_STORE_INT8: gkv_pages_copy_kernel<GKV_STORE_INT8, OP><<<grid, kPageCopyThreads, smem, s>>>(p); break;
        default:             gkv_pages_copy_kernel<GKV_STORE_INT4, OP><<<grid, kPageCopyThreads, smem, s>>>(p); break;
    }
    return cudaGetLastError();
}
cudaError_t launch_pages_append(const PagesCopyLaunch& p, cudaStream_t s) {
    if (!p.rotary.turns) return launch_copy<kWrite>(p, s);
    if (p.rotary.interleaved) return launch_copy<kWriteNeighbours>(p, s);
    return p.rotary.half % 4 == 0 ? launch_copy<kWriteHalves>(p, s) : launch_copy<kWriteAny>(p, s);
}
cudaError_t launch_pages_read(const PagesCopyLaunch& p, cudaStream_t s) { return launch_copy<kRead>(p, s); }

}  // namespace gkv
