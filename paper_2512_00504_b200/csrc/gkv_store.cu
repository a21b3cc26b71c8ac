// Key/value stores: quantising rows as they are written and reading them back.
//
// Both directions only move rows: 256 bytes of bf16 on one side, 130 (8 bits) or 72 (4 bits) of codes and scales on the other,
// against a few dozen instructions for every 8 elements, so the kernels are bound by HBM and what matters is that enough rows
// are in flight: half a warp handles a row (16 lanes x 16 bytes), takes kRowsPerLane rows at once and loads all of them before
// it works on the first.
#include "gkv_store_codes.cuh"

namespace gkv {

constexpr int kCopyThreads = 256;
constexpr int kRowsPerLane = 4;
constexpr int kRowsPerBlock = kCopyThreads / 16 * kRowsPerLane;

// Row j = t * h_kv + h of sequence blockIdx.y; blockIdx.z = K or V. Rows of consecutive j lie next to each other in a
// contiguous source, and a block's rows of one head next to each other in the store.
template <int F, bool READ>
__global__ void __launch_bounds__(kCopyThreads) gkv_store_copy_kernel(const StoreCopyLaunch p) {
    using Fm = StoreFormat<F>;
    const int b = blockIdx.y, which = blockIdx.z;
    const int l = threadIdx.x & 15, hw = threadIdx.x >> 4;
    const int count = p.count ? min(max(p.count[b], 0), p.n_tokens) : p.n_tokens;
    const int first = p.first ? p.first[b] : 0;
    const int total = count * p.h_kv;
    const int j0 = blockIdx.x * kRowsPerBlock + hw;
    if (blockIdx.x * kRowsPerBlock >= total) return;

    uint8_t* data = p.data[which];
    __nv_bfloat16* scale = p.scale[which];
    __nv_bfloat16* xs = p.x[which] + (int64_t)b * p.seq_stride;
    __nv_bfloat16* x[kRowsPerLane];
    int64_t row[kRowsPerLane];      // row of the store, or -1: nothing to do
    uint4 v[kRowsPerLane];
    StoreRaw<F> raw[kRowsPerLane];
#pragma unroll
    for (int i = 0; i < kRowsPerLane; ++i) {
        const int j = j0 + i * (kCopyThreads / 16);
        const int t = j / p.h_kv, h = j - t * p.h_kv;
        const int64_t r = (int64_t)first + t;
        row[i] = (j < total && r >= 0 && r < p.capacity) ? ((int64_t)b * p.h_kv + h) * p.capacity + r : -1;
        x[i] = xs + (int64_t)t * p.token_stride + (int64_t)h * p.head_stride;
        v[i] = make_uint4(0u, 0u, 0u, 0u);
        raw[i].c = v[i];
        raw[i].s = 0u;
        if (row[i] >= 0) {
            if (READ) raw[i] = store_get_raw<F>(data + row[i] * Fm::kRow, scale + row[i] * Fm::kScales, l);
            else v[i] = store_load_source<F>(x[i], l);
        }
    }
#pragma unroll
    for (int i = 0; i < kRowsPerLane; ++i) {
        if (READ) {
            if (row[i] >= 0) store_put_target<F>(x[i], l, store_decode_raw<F>(raw[i]));
        } else {
            const int64_t r = max(row[i], (int64_t)0);
            store_put_row<F>(data + r * Fm::kRow, scale + r * Fm::kScales, l, v[i], row[i] >= 0);
        }
    }
}

template <bool READ>
static cudaError_t launch_copy(const StoreCopyLaunch& p, cudaStream_t s) {
    const int64_t rows = (int64_t)p.n_tokens * p.h_kv;
    const dim3 grid((unsigned)((rows + kRowsPerBlock - 1) / kRowsPerBlock), (unsigned)p.batch, 2);
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
