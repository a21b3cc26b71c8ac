// Rotary positions of q and k: two reads of a pair's elements, two writes, six operations, so the kernel is bound by HBM, or for the
// few rows of a decode step by its launch.
//
// cos and sin depend on the token and the pair alone and cost more than everything else that is done to a pair. A CTA takes all
// heads of a few tokens: it works them out once, in shared memory (cos and sin in arrays of their own, so that a thread's run of
// them is whole 16-byte pieces), and its threads then go over the heads. A thread has up to 16 bytes of each half of a run of pairs,
// the same run in every row that it comes to.
#include "gkv_rotary.cuh"

#include <cuda_fp16.h>

namespace gkv {

constexpr int kRotThreads = 256;
constexpr int kRotRows = 4;        // rows of a thread whose loads are in flight together

template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32(float x) { return x; }
template <> __device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32(float x) { return x; }
template <> __device__ __forceinline__ __half from_f32(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16_rn(x); }

template <typename T, int VEC> struct __align__(sizeof(T) * VEC) Run { T e[VEC]; };

// VEC pairs a thread and row: elements [run VEC, ..) of both halves, or 2 VEC neighbours. Runs behind the pairs are copied.
template <typename T, int VEC, bool INTERLEAVED>
__global__ void __launch_bounds__(kRotThreads) gkv_rotary_kernel(const RotaryLaunch p) {
    extern __shared__ __align__(16) float s_table[];
    const int b = blockIdx.y, t0 = blockIdx.x * p.tokens_per_cta, half = p.rotary.half;
    int n = p.count ? min(p.count[b], p.n_tokens) : p.n_tokens;
    n = min(n - t0, p.tokens_per_cta);
    if (n <= 0) return;
    float *s_cos = s_table, *s_sin = s_table + p.tokens_per_cta * half;
    for (int i = threadIdx.x; i < n * half; i += kRotThreads) {
        const int t = i / half, pair = i - t * half;
        const int32_t pos = p.pos[(int64_t)b * p.pos_seq_stride + (int64_t)(t0 + t) * p.pos_token_stride];
        const float2 cs = rotary_cos_sin(p.rotary.turns[pair], pos, p.rotary.factor, p.sign);
        s_cos[i] = cs.x;
        s_sin[i] = cs.y;
    }
    __syncthreads();
    const int per = kRotThreads / p.runs;          // rows at a time
    const int run = threadIdx.x % p.runs, first = threadIdx.x / p.runs;
    if (first >= per) return;
    const bool turns = run < p.pair_runs;
    const int at0 = turns ? (INTERLEAVED ? 2 : 1) * run * VEC : 2 * half + (run - p.pair_runs) * 2 * VEC;
    const int at1 = turns && !INTERLEAVED ? at0 + half : at0 + VEC;
    int t = first / p.heads, h = first - t * p.heads;
    const int dt = per / p.heads, dh = per - dt * p.heads;     // from one of this thread's rows to the next
    while (t < n) {
        Run<T, VEC> x0[kRotRows], x1[kRotRows];
        T* y[kRotRows];
        int tok[kRotRows];
        int rows = 0;
#pragma unroll
        for (int k = 0; k < kRotRows; ++k) {
            tok[k] = t;
            if (t < n) {
                const RotaryRows& r = p.rows[h >= p.heads0];
                const int64_t hh = h >= p.heads0 ? h - p.heads0 : h, tt = t0 + t;
                const T* x = static_cast<const T*>(r.x) + (b * r.xs[0] + tt * r.xs[1] + hh * r.xs[2]);
                y[k] = static_cast<T*>(r.y) + (b * r.ys[0] + tt * r.ys[1] + hh * r.ys[2]);
                x0[k] = *reinterpret_cast<const Run<T, VEC>*>(x + at0);
                x1[k] = *reinterpret_cast<const Run<T, VEC>*>(x + at1);
                rows = k + 1;
            }
            t += dt;
            h += dh;
            if (h >= p.heads) { h -= p.heads; ++t; }
        }
#pragma unroll
        for (int k = 0; k < kRotRows; ++k) {
            if (k >= rows) break;
            if (turns) {
                float e[2 * VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) { e[i] = to_f32(x0[k].e[i]); e[VEC + i] = to_f32(x1[k].e[i]); }
                const Run<float, VEC < 4 ? VEC : 4>* c4 = reinterpret_cast<const Run<float, VEC < 4 ? VEC : 4>*>(s_cos + tok[k] * half + run * VEC);
                const Run<float, VEC < 4 ? VEC : 4>* s4 = reinterpret_cast<const Run<float, VEC < 4 ? VEC : 4>*>(s_sin + tok[k] * half + run * VEC);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    constexpr int W = VEC < 4 ? VEC : 4;
                    const int a = INTERLEAVED ? 2 * i : i, c = INTERLEAVED ? 2 * i + 1 : VEC + i;
                    const float2 r = rotary_turn(e[a], e[c], c4[i / W].e[i % W], s4[i / W].e[i % W]);
                    e[a] = r.x;
                    e[c] = r.y;
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) { x0[k].e[i] = from_f32<T>(e[i]); x1[k].e[i] = from_f32<T>(e[VEC + i]); }
            }
            *reinterpret_cast<Run<T, VEC>*>(y[k] + at0) = x0[k];
            *reinterpret_cast<Run<T, VEC>*>(y[k] + at1) = x1[k];
        }
    }
}

template <typename T, int VEC>
static cudaError_t launch_typed(const RotaryLaunch& p, cudaStream_t s) {
    const dim3 grid((unsigned)((p.n_tokens + p.tokens_per_cta - 1) / p.tokens_per_cta), (unsigned)p.batch);
    const size_t smem = (size_t)p.tokens_per_cta * p.rotary.half * 2 * sizeof(float);
    if (p.rotary.interleaved) gkv_rotary_kernel<T, VEC, true><<<grid, kRotThreads, smem, s>>>(p);
    else gkv_rotary_kernel<T, VEC, false><<<grid, kRotThreads, smem, s>>>(p);
    return cudaGetLastError();
}
template <typename T>
static cudaError_t launch_type(const RotaryLaunch& p, int vec, cudaStream_t s) {
    switch (vec) {
        case 8: if constexpr (sizeof(T) == 2) return launch_typed<T, 8>(p, s);
        case 4: return launch_typed<T, 4>(p, s);
        case 2: return launch_typed<T, 2>(p, s);
        default: return launch_typed<T, 1>(p, s);
    }
}

// Tokens of a CTA: as many as still leave eight CTAs an SM, at most kRotTable pairs (their cos and sin are 16 KB then).
constexpr int kRotTable = 2048;

cudaError_t launch_rotary(RotaryLaunch& p, int type, int head_dim, int sm_count, cudaStream_t s) {
    const int half = p.rotary.half, size = type == GKV_TYPE_FP32 ? 4 : 2;
    bool in_place = true;
    for (int i = 0; i < (p.heads > p.heads0 ? 2 : 1); ++i) in_place = in_place && p.rows[i].x == p.rows[i].y;
    const int rest = in_place ? 0 : head_dim - 2 * half;      // elements to be copied
    // the widest run that divides both parts and that every row's address allows
    int vec = 16 / size;
    auto fits = [&](int v) {
        if (half % v != 0 || rest % (2 * v) != 0) return false;
        const int64_t bytes = (int64_t)v * size;
        for (int i = 0; i < (p.heads > p.heads0 ? 2 : 1); ++i) {
            uintptr_t bits = reinterpret_cast<uintptr_t>(p.rows[i].x) | reinterpret_cast<uintptr_t>(p.rows[i].y);
            for (int k = 0; k < 3; ++k) bits |= (uintptr_t)(p.rows[i].xs[k] * size) | (uintptr_t)(p.rows[i].ys[k] * size);
            if ((bits & (uintptr_t)(bytes - 1)) != 0) return false;
        }
        return true;
    };
    // a row has at most kRotThreads runs (half <= 512: 2 pairs a thread do)
    while (vec > 1 && !fits(vec)) vec >>= 1;
    p.pair_runs = half / vec;
    p.runs = p.pair_runs + rest / (2 * vec);
    int most = kRotTable / half;
    if (most < 1) most = 1;
    int per = 1;
    while (2 * per <= most && (int64_t)((p.n_tokens + 2 * per - 1) / (2 * per)) * p.batch >= 8ll * sm_count) per *= 2;
    p.tokens_per_cta = per;
    switch (type) {
        case GKV_TYPE_BF16: return launch_type<__nv_bfloat16>(p, vec, s);
        case GKV_TYPE_FP16: return launch_type<__half>(p, vec, s);
        default: return launch_type<float>(p, vec, s);
    }
}

}  // namespace gkv
