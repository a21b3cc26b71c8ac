// Rotary positions of q and k: two reads of a pair's elements, two writes, six operations, so the kernel is bound by HBM, or for the
// few rows of a decode step by its launch.
//
// cos and sin depend on the token and the pair alone. A CTA takes all heads of a few tokens and works them out once, through shared memory;
// a thread then has one run of pairs of one token (up to 16 bytes of each side), holds their cos and sin in registers, and goes over its share of
// the heads, with the loads of several rows in flight. (Reading them from shared memory for every row instead: 8 x 8192 tokens x 32 heads
// in bf16 264 us. With loads that the compiler may put off, and elements of 16 bits converted one by one: 180.)
//
// Measured (bytes read and written): 8 x 8192 tokens x 32 heads in bf16, 1.07 GB in 166 us, 6.5 TB/s; 4 x 4096 x 40 in fp32, half of each head
// turned, 0.67 GB in 105 us, 6.4 TB/s; 4097 tokens x 72 heads, 151 MB in 27 us; 32 tokens x 32 heads 2.5 us, which is a launch.
#include "gkv_rotary.cuh"
#include "gkv_store_rows.h"

#include <cuda_fp16.h>
#include <string.h>

namespace gkv {

constexpr int kRotThreads = 128;     // of a block, twice that where a row has more runs

// Elements of a type in 32-bit words: two of 16 bits, or one.
template <typename T> struct Words;
template <> struct Words<float> {
    static constexpr int kPer = 1;
    static __device__ __forceinline__ float2 open(uint32_t w) { return make_float2(__uint_as_float(w), 0.f); }
    static __device__ __forceinline__ uint32_t close(float a, float) { return __float_as_uint(a); }
};
template <> struct Words<__nv_bfloat16> {
    static constexpr int kPer = 2;
    static __device__ __forceinline__ float2 open(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
    static __device__ __forceinline__ uint32_t close(float a, float b) { return pack_bf16x2(a, b); }
};
template <> struct Words<__half> {
    static constexpr int kPer = 2;
    static __device__ __forceinline__ float2 open(uint32_t w) {
        __half2 h;
        memcpy(&h, &w, 4);
        return __half22float2(h);
    }
    static __device__ __forceinline__ uint32_t close(float a, float b) {
        const __half2 h = __floats2half2_rn(a, b);
        uint32_t w;
        memcpy(&w, &h, 4);
        return w;
    }
};
// N words (0: half of one, in the low bits) at an address, in one access. Loads stay where they are written: those of all rows in flight
// ahead of the first row's work.
template <int N> struct Piece { uint32_t w[N > 0 ? N : 1]; };
template <int N>
__device__ __forceinline__ Piece<N> load_piece(const void* a) {
    Piece<N> r;
    if constexpr (N == 4) asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "l"(a) : "memory");
    else if constexpr (N == 2) asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(r.w[0]), "=r"(r.w[1]) : "l"(a) : "memory");
    else if constexpr (N == 1) asm volatile("ld.global.u32 %0, [%1];" : "=r"(r.w[0]) : "l"(a) : "memory");
    else {
        uint16_t h;
        asm volatile("ld.global.u16 %0, [%1];" : "=h"(h) : "l"(a) : "memory");
        r.w[0] = h;
    }
    return r;
}
template <int N>
__device__ __forceinline__ void store_piece(void* a, const Piece<N>& r) {
    if constexpr (N == 4) *static_cast<uint4*>(a) = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
    else if constexpr (N == 2) *static_cast<uint2*>(a) = make_uint2(r.w[0], r.w[1]);
    else if constexpr (N == 1) *static_cast<uint32_t*>(a) = r.w[0];
    else *static_cast<uint16_t*>(a) = (uint16_t)r.w[0];
}
// A run of VEC pairs turned: x0 and x1 are the pairs' first and second sides, or (neighbours) the first and last VEC elements.
template <typename T, int VEC, bool INTERLEAVED, int N>
__device__ __forceinline__ void turn_run(Piece<N>& x0, Piece<N>& x1, const float (&c)[VEC], const float (&s)[VEC]) {
    using W = Words<T>;
    if constexpr (VEC == 1 || (W::kPer == 1 && !INTERLEAVED)) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float2 r = rotary_turn(W::open(x0.w[i]).x, W::open(x1.w[i]).x, c[i], s[i]);
            x0.w[i] = W::close(r.x, 0.f);
            x1.w[i] = W::close(r.y, 0.f);
        }
    } else if constexpr (W::kPer == 1) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            Piece<N>& x = i < VEC / 2 ? x0 : x1;
            const int k = 2 * (i % (VEC / 2));
            const float2 r = rotary_turn(__uint_as_float(x.w[k]), __uint_as_float(x.w[k + 1]), c[i], s[i]);
            x.w[k] = __float_as_uint(r.x);
            x.w[k + 1] = __float_as_uint(r.y);
        }
    } else if constexpr (INTERLEAVED) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            Piece<N>& x = i < VEC / 2 ? x0 : x1;
            const int k = i % (VEC / 2);
            const float2 e = W::open(x.w[k]), r = rotary_turn(e.x, e.y, c[i], s[i]);
            x.w[k] = W::close(r.x, r.y);
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            const float2 a = W::open(x0.w[i]), b = W::open(x1.w[i]);
            const float2 r = rotary_turn(a.x, b.x, c[2 * i], s[2 * i]), t = rotary_turn(a.y, b.y, c[2 * i + 1], s[2 * i + 1]);
            x0.w[i] = W::close(r.x, t.x);
            x1.w[i] = W::close(r.y, t.y);
        }
    }
}

// VEC pairs a thread and row: elements [run VEC, ..) of both halves, or 2 VEC neighbours. Runs behind the pairs are copied.
template <typename T, int VEC, bool INTERLEAVED>
__global__ void __launch_bounds__(2 * kRotThreads, VEC == 8 ? 4 : 2) gkv_rotary_kernel(const RotaryLaunch p) {
    extern __shared__ __align__(16) float s_table[];
    const int b = blockIdx.y, t0 = blockIdx.x * p.tokens_per_cta, half = p.rotary.half;
    const int n = tokens_here(p.count ? p.count[b] : p.n_tokens, p.n_tokens, t0, p.tokens_per_cta);
    if (n == 0) return;
    float *s_cos = s_table, *s_sin = s_table + p.tokens_per_cta * half;
    for (int i = threadIdx.x; i < n * half; i += blockDim.x) {
        const int t = i / half, pair = i - t * half;
        const int32_t pos = p.pos[(int64_t)b * p.pos_seq_stride + (int64_t)(t0 + t) * p.pos_token_stride];
        const float2 cs = rotary_cos_sin(p.rotary.turns[pair], pos, p.rotary.factor, p.sign);
        s_cos[i] = cs.x;
        s_sin[i] = cs.y;
    }
    __syncthreads();
    const int slot = threadIdx.x / p.runs, run = threadIdx.x - slot * p.runs;       // thread: run of a row, token, share of the heads
    const int local = slot / p.tokens_per_cta, t = slot - local * p.tokens_per_cta, locals = (int)blockDim.x / p.runs / p.tokens_per_cta;
    const int share = blockIdx.z * locals + local, shares = (int)gridDim.z * locals;
    if (local >= locals || t >= n) return;
    const bool turns = run < p.pair_runs;
    const int at0 = turns ? (INTERLEAVED ? 2 : 1) * run * VEC : 2 * half + (run - p.pair_runs) * 2 * VEC;
    const int at1 = turns && !INTERLEAVED ? at0 + half : at0 + VEC;
    // Rows of a thread whose loads are in flight together: two with 8 pairs each, which leaves registers for 8 CTAs of 128 threads on an
    // SM (3 rows: 179 us, 4: 172 and, held to those registers, 231), else four (fp32, 2 rows: 114 us).
    constexpr int kRotRows = VEC == 8 ? 2 : 4, N = VEC * (int)sizeof(T) / 4;
    float c[VEC], s[VEC];
    if (turns)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            c[i] = s_cos[t * half + run * VEC + i];
            s[i] = s_sin[t * half + run * VEC + i];
        }
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        const RotaryRows& r = p.rows[which];
        const int heads = which ? p.heads - p.heads0 : p.heads0;
        const T* x = static_cast<const T*>(r.x) + (b * r.xs[0] + (t0 + t) * r.xs[1] + share * r.xs[2]);
        T* y = static_cast<T*>(r.y) + (b * r.ys[0] + (t0 + t) * r.ys[1] + share * r.ys[2]);
        const int64_t dx = shares * r.xs[2], dy = shares * r.ys[2];
        for (int h = share; h < heads; h += kRotRows * shares) {
            Piece<N> x0[kRotRows], x1[kRotRows];
#pragma unroll
            for (int k = 0; k < kRotRows; ++k)
                if (h + k * shares < heads) {
                    x0[k] = load_piece<N>(x + k * dx + at0);
                    x1[k] = load_piece<N>(x + k * dx + at1);
                }
#pragma unroll
            for (int k = 0; k < kRotRows; ++k)
                if (h + k * shares < heads) {
                    if (turns) turn_run<T, VEC, INTERLEAVED>(x0[k], x1[k], c, s);
                    store_piece<N>(y + k * dy + at0, x0[k]);
                    store_piece<N>(y + k * dy + at1, x1[k]);
                }
            x += kRotRows * dx;
            y += kRotRows * dy;
        }
    }
}

template <typename T, int VEC>
static cudaError_t launch_typed(const RotaryLaunch& p, cudaStream_t s) {
    const dim3 grid((unsigned)((p.n_tokens + p.tokens_per_cta - 1) / p.tokens_per_cta), (unsigned)p.batch, (unsigned)p.parts);
    const int threads = p.runs <= kRotThreads ? kRotThreads : 2 * kRotThreads;      // (at most 256 runs: a head of 512 by single pairs)
    const size_t smem = (size_t)p.tokens_per_cta * p.rotary.half * 2 * sizeof(float);
    if (p.rotary.interleaved) gkv_rotary_kernel<T, VEC, true><<<grid, threads, smem, s>>>(p);
    else gkv_rotary_kernel<T, VEC, false><<<grid, threads, smem, s>>>(p);
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
    while (vec > 1 && !fits(vec)) vec >>= 1;
    p.pair_runs = half / vec;
    p.runs = p.pair_runs + rest / (2 * vec);
    // Tokens of a CTA: as many as leave two threads to share a token's heads, as long as there are twenty CTAs an SM.
    int per = 1;
    while (4 * per * p.runs <= kRotThreads && (int64_t)((p.n_tokens + 2 * per - 1) / (2 * per)) * p.batch >= 20ll * sm_count) per *= 2;
    p.tokens_per_cta = per;
    // Few tokens: up to four CTAs share one's heads, as long as that makes no more than two an SM (1 token x 72 heads 2.7 us instead of 3.2, 128 tokens
    // 3.1 instead of 3.4; with many tokens cos and sin worked out twice cost more: 1000 x 32 heads 5.8 instead of 4.5).
    const int64_t ctas = (int64_t)((p.n_tokens + per - 1) / per) * p.batch;
    p.parts = 1;
    while (p.parts < 4 && 2 * p.parts * ctas <= 2ll * sm_count) p.parts *= 2;
    switch (type) {
        case GKV_TYPE_BF16: return launch_type<__nv_bfloat16>(p, vec, s);
        case GKV_TYPE_FP16: return launch_type<__half>(p, vec, s);
        default: return launch_type<float>(p, vec, s);
    }
}

}  // namespace gkv
