// Key/value stores: quantising rows as they are written and reading them back.
//
// Both directions only move rows: 256 bytes of bf16 on one side, 130 (8 bits) or 72 (4 bits) of codes and scales on the other,
// against a few dozen instructions for every 8 elements, so the kernels are bound by HBM and what matters is that enough rows
// are in flight and that they go in whole sectors. Half a warp takes kRun consecutive tokens of one head: all of their loads
// start before the first is worked on, the codes are one contiguous stretch of the store, and so are the scales, which are
// gathered in the lanes and go with one access (2 bytes at a time they cost a 32-byte sector each). Neighbouring half warps
// have the neighbouring heads of the same tokens, which lie next to each other on the bf16 side.
//
// Measured (bytes of both sides): 4 x 32768 tokens x 8 heads into 4 bits, 688 MB in 111 us: 6.2 TB/s, and back in 106; into 8 bits,
// 809 MB in 143 to 147 us: 5.6 TB/s, and back in 123; bf16, 1074 MB in 160 us either way: 6.7 TB/s; 64 x about 1900 tokens x 8 heads
// back from e4m3, 738 MB in 113 us: 6.5 TB/s; one token of 32 sequences x 4 heads: 2 us, which is a launch.
#include "gkv_store_codes.cuh"
#include "gkv_store_rows.h"

namespace gkv {

// Small blocks: a run of a few sequences is one round of them, and 128 threads end with a shorter tail than 256 (2048 tokens x 8
// heads with ragged counts, write and read back: 26.4 us against 28.2; one sequence: 2.5 against 2.7; 64 threads: 26.8, 2.5).
constexpr int kCopyThreads = 128;

// Work item i of sequence blockIdx.y: head i % h_kv, tokens kRun * (i / h_kv) and on; blockIdx.z = K or V.
template <int F, bool READ>
__global__ void __launch_bounds__(kCopyThreads) gkv_store_copy_kernel(const StoreCopyLaunch p) {
    using Fm = StoreFormat<F>;
    const int b = blockIdx.y;
    const bool is_v = blockIdx.z != 0;
    const int l = threadIdx.x & 15;
    const int item = blockIdx.x * (kCopyThreads / 16) + (threadIdx.x >> 4);
    const int h = item % p.h_kv, t0 = item / p.h_kv * kRun;
    const int32_t first = p.first ? p.first[b] : 0;
    // the whole warp stays for the shuffles, whatever the run has
    const RunRows rows = run_rows(first, p.count ? p.count[b] : p.n_tokens, p.n_tokens, p.capacity, t0);
    const int lo = rows.lo, hi = rows.hi;
    const int64_t row0 = ((int64_t)b * p.h_kv + h) * p.capacity + first + t0;
    uint8_t* data = (is_v ? p.data[1] : p.data[0]) + row0 * Fm::kRow;
    __nv_bfloat16* scale = (is_v ? p.scale[1] : p.scale[0]) + row0 * Fm::kScales;
    __nv_bfloat16* x = (is_v ? p.x[1] : p.x[0]) + (int64_t)b * p.seq_stride + (int64_t)t0 * p.token_stride + (int64_t)h * p.head_stride;

    // Scales are held and moved by lane 2i + j: in 4 bits those of groups 2j, 2j + 1 of token i, in 8 bits that of token i (the
    // odd lane has a copy).
    const int st = l >> 1;
    const bool has_scale = Fm::kScales != 0 && st >= lo && st < hi && (F == GKV_STORE_INT4 || (l & 1) == 0);
    uint32_t* scale4 = reinterpret_cast<uint32_t*>(scale) + l;
    uint16_t* scale2 = reinterpret_cast<uint16_t*>(scale) + st;
    uint4 v[kRun];
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        v[i] = make_uint4(0u, 0u, 0u, 0u);
        if (i >= lo && i < hi) {
            if (READ) v[i] = store_get_codes<F>(data + (int64_t)i * Fm::kRow, l);
            else v[i] = store_load_source<F>(x + (int64_t)i * p.token_stride, l);
        }
    }
    if (READ) {
        uint32_t sc = 0u;
        if (has_scale) sc = F == GKV_STORE_INT4 ? *scale4 : *scale2;
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            const uint32_t s = __shfl_sync(0xffffffffu, sc, 2 * i + (F == GKV_STORE_INT4 ? l & 1 : 0), 16);
            if (i >= lo && i < hi) store_put_target<F>(x + (int64_t)i * p.token_stride, l, store_decode<F>(v[i], s));
        }
    } else {
        float inv0 = 1.f, inv1 = 1.f;
        if (Fm::kScales != 0) {
            // Maxima of the 8 tokens, reduced and handed out at once: a lane gives away half of what it holds at every step
            // (7 exchanges for 8 tokens instead of 3 or 4 for each), until it has the token of its scale.
            uint32_t a[kRun];
#pragma unroll
            for (int i = 0; i < kRun; ++i) a[i] = store_lane_max<F>(v[i]);
#pragma unroll
            for (int o = 8, n = kRun / 2; o >= 2; o >>= 1, n >>= 1) {
                const bool upper = (l & o) != 0;
#pragma unroll
                for (int i = 0; i < kRun / 2; ++i)
                    if (i < n) {
                        const uint32_t keep = upper ? a[i + n] : a[i], give = upper ? a[i] : a[i + n];
                        a[i] = __vmaxu2(keep, __shfl_xor_sync(0xffffffffu, give, o));
                    }
            }
            if (F != GKV_STORE_INT4) a[0] = __vmaxu2(a[0], __shfl_xor_sync(0xffffffffu, a[0], 1));
            const uint32_t sc = store_scale<F>(a[0], &inv0, &inv1);
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
            if (i >= lo && i < hi) store_put_codes<F>(data + (int64_t)i * Fm::kRow, l, store_codes<F>(v[i], f0, f1));
        }
    }
}

template <bool READ>
static cudaError_t launch_copy(const StoreCopyLaunch& p, cudaStream_t s) {
    const int items = (p.n_tokens + kRun - 1) / kRun * p.h_kv;
    const dim3 grid((unsigned)((items + kCopyThreads / 16 - 1) / (kCopyThreads / 16)), (unsigned)p.batch, 2);
    switch (p.format) {
        case GKV_STORE_BF16: gkv_store_copy_kernel<GKV_STORE_BF16, READ><<<grid, kCopyThreads, 0, s>>>(p); break;
        case GKV_STORE_E4M3: gkv_store_copy_kernel<GKV_STORE_E4M3, READ><<<grid, kCopyThreads, 0, s>>>(p); break;
        case GKV_STORE_INT8: gkv_store_copy_kernel<GKV_STORE_INT8, READ><<<grid, kCopyThreads, 0, s>>>(p); break;
        default:             gkv_store_copy_kernel<GKV_STORE_INT4, READ><<<grid, kCopyThreads, 0, s>>>(p); break;
    }
    return cudaGetLastError();
}
cudaError_t launch_store_write(const StoreCopyLaunch& p, cudaStream_t s) { return launch_copy<false>(p, s); }
cudaError_t launch_store_read(const StoreCopyLaunch& p, cudaStream_t s) { return launch_copy<true>(p, s); }

}  // namespace gkv
