// Attention of a batch's query rows over prefixes that its sequences share: the prefix's rows are read once for all of them.
//
// The query rows of a (prefix, KV head) are the g heads of every sequence of the prefix: 8 to 2000 rows that see the same keys,
// so this is a dense product and belongs on tcgen05. A work item is up to 256 query rows and a run of 128-key tiles; its result
// (running maximum, sum, unscaled output of every row) goes to the workspace and is joined with the other runs' and with the
// sequences' own rows by the merge kernel.
//
// One CTA (one per SM: 226 KB of shared memory, all 512 TMEM columns) holds two streams, A and B, each a softmax warpgroup with
// 128 query rows: with more than 128 rows in the item A and B have a row tile each and both see every key tile; with fewer they
// have the same rows and take the even and the odd key tiles. Per stream and key tile
//     S = Q K^T          128 x 128 x 128, operands in shared memory, S in 128 TMEM columns
//     softmax            thread = TMEM lane = query row, so that maximum and sum are loops in one thread; P as bf16 goes back
//                        over the first 64 of S's columns
//     O += P V           P is read from TMEM as the A operand, V from shared memory with the head dimension contiguous (as it
//                        lies in memory: no transpose), O in 128 TMEM columns
// While one stream is in its softmax the tensor cores work for the other. The running maximum may lag by 2^8 before O is
// rescaled, which makes rescaling (a trip of 128 columns through registers) rare. K and V tiles come by TMA through a ring of
// five 32 KB slots in the order in which the products want them.
//
// Bound: for 256 rows a key tile costs 64 KB of HBM traffic (1.5 us of an SM's share), 2048 cycles of the tensor core and 2048
// cycles of the exponential unit: all three are level.
#include "gkv_tcgen05.cuh"
#include "gkv_internal.h"

namespace gkv {

constexpr int kPxThreads = 320;              // warps 0-3: stream A, 4-7: stream B, 8: TMA, 9: MMA
constexpr int kPxKeys = 128;                 // keys of a tile
constexpr int kPxHalf = 128 * 128;           // bytes of 128 rows x 64 elements
constexpr int kPxSlotBytes = 2 * kPxHalf;    // one K or V tile, or one row tile of q
constexpr int kPxSlots = 5;
constexpr float kPxLag = 8.f;

struct __align__(16) PrefixTail {
    uint64_t q_full;
    uint64_t full[kPxSlots], empty[kPxSlots];
    uint64_t s_full[2], p_ready[2];
    uint64_t o_full;
    uint32_t tmem_base;
    int abort_flag;
    int issued;        // ring slots filled so far
};
constexpr size_t kPxSmem = 1024 + 2 * kPxSlotBytes + kPxSlots * kPxSlotBytes + sizeof(PrefixTail);

// A operand in tensor memory (lane = row, one 32-bit column = two bf16 of the inner index), B in shared memory.
__device__ __forceinline__ void umma_bf16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Operand descriptor (low word) of a tile whose 64-element halves lie kPxHalf apart and whose contiguous direction is the
// outer index of the product: rows of the inner index are 128 bytes, groups of 8 of them 1024 bytes apart (the stride in the
// high word), the next 64 outer elements kPxHalf further on.
__device__ __forceinline__ uint32_t umma_desc_lo_outer(uint32_t smem_addr) { return ((smem_addr & 0x3FFFFu) >> 4) | ((uint32_t)(kPxHalf >> 4) << 16); }

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
          "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
          "r"(r[30]), "r"(r[31])
        : "memory");
}

__global__ void __launch_bounds__(kPxThreads, 1)
gkv_prefix_attn_kernel(const StoreAttnLaunch p, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* q_smem = smem;                              // two row tiles
    uint8_t* ring = smem + 2 * kPxSlotBytes;
    PrefixTail* tail = reinterpret_cast<PrefixTail*>(ring + kPxSlots * kPxSlotBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // ---- the work item
    int item = blockIdx.x, pre = 0, runs = 0;
    for (;; ++pre) {
        runs = ((p.prefix_len[pre] + kPxKeys - 1) / kPxKeys + p.chunk - 1) / p.chunk;
        const int items = runs * p.h_kv * p.n_blocks;
        if (item < items || pre == p.n_prefix - 1) break;
        item -= items;
    }
    const int run = item / (p.h_kv * p.n_blocks), hb = item - run * (p.h_kv * p.n_blocks);
    const int head = hb / p.n_blocks, blk = hb - head * p.n_blocks;
    const int n_keys = p.prefix_len[pre];
    const int t0 = run * p.chunk, n_tiles = min(p.chunk, (n_keys + kPxKeys - 1) / kPxKeys - t0);
    const int seq0 = pre * p.seqs_per_prefix + blk * p.seqs_per_block;
    const int rows = min(p.seqs_per_block, p.seqs_per_prefix - blk * p.seqs_per_block) * p.g;
    const bool two = p.two_tiles != 0;
    const int ahead = two ? 1 : 2;                       // key tiles whose S is asked for before their turn

    if (tid == 0) {
        mbar_init(smem_u32(&tail->q_full), 256);
        for (int s = 0; s < kPxSlots; ++s) { mbar_init(smem_u32(&tail->full[s]), 1); mbar_init(smem_u32(&tail->empty[s]), 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&tail->s_full[s]), 1); mbar_init(smem_u32(&tail->p_ready[s]), 128); }
        mbar_init(smem_u32(&tail->o_full), 1);
        tail->abort_flag = 0;
        tail->issued = 0;
        fence_mbar_init();
    }
    if (warp == 9) {   // one CTA per SM holds all columns: this never waits
        tmem_alloc(smem_u32(&tail->tmem_base), 512);
        tmem_relinquish_alloc_permit();
        tmem_fence_before_sync();
    }
    __syncthreads();
    tmem_fence_after_sync();
    const uint32_t tmem = *(volatile uint32_t*)&tail->tmem_base;
    const int* abort_flag = &tail->abort_flag;
    // ring position of key tile t's V tile and K tile: K_0 [K_1] then V_t, K_(t + ahead) in turn, while there are such tiles
    auto v_pos = [&](int t) { return min(ahead, n_tiles) + t + min(t, max(n_tiles - ahead, 0)); };
    auto k_pos = [&](int t) { return t < ahead ? t : v_pos(t - ahead) + 1; };
    auto wait_full = [&](int pos) { return tc_wait(smem_u32(&tail->full[pos % kPxSlots]), (pos / kPxSlots) & 1, abort_flag); };

    bool ok = true;
    if (warp == 8) {
        // ------------------------------------------------------------------ TMA
        if (lane == 0) {
            prefetch_tensormap(&tm_k);
            prefetch_tensormap(&tm_v);
            const int row0 = (pre * p.h_kv + head) * p.prefix_rows;
            const int total = 2 * n_tiles;
            int kt = 0, vt = 0;
            for (int pos = 0; pos < total && ok; ++pos) {
                const bool is_k = kt < n_tiles && k_pos(kt) == pos;
                const int t = is_k ? kt++ : vt++;
                const int s = pos % kPxSlots;
                if (pos >= kPxSlots) ok = tc_wait(smem_u32(&tail->empty[s]), (pos / kPxSlots - 1) & 1, abort_flag);
                if (!ok) { tail->abort_flag = 1; break; }
                const uint32_t bar = smem_u32(&tail->full[s]), dst = smem_u32(ring + s * kPxSlotBytes);
                const CUtensorMap* m = is_k ? &tm_k : &tm_v;
                const int y = row0 + (t0 + t) * kPxKeys;
                mbar_arrive_expect_tx(bar, kPxSlotBytes);
                tma_load_2d(dst, m, 0, y, bar);
                tma_load_2d(dst + kPxHalf, m, 64, y, bar);
                *(volatile int*)&tail->issued = pos + 1;
            }
        }
    } else if (warp == 9) {
        // ------------------------------------------------------------------ MMA
        if (lane == 0) {
            const uint32_t idesc_s = umma_idesc_bf16_m128(128);
            const uint32_t idesc_o = idesc_s | (1u << 16);           // B's contiguous direction is its outer index
            const uint32_t qa[2] = {umma_desc_lo(smem_u32(q_smem)), umma_desc_lo(smem_u32(q_smem + (two ? kPxSlotBytes : 0)))};
            auto scores = [&](int x, int t) {                        // S_x = Q_x K_t^T
                const int pos = k_pos(t);
                if (!wait_full(pos)) return false;
                tmem_fence_after_sync();
                const uint32_t kb = umma_desc_lo(smem_u32(ring + (pos % kPxSlots) * kPxSlotBytes));
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    umma_bf16(tmem + 128 * x, umma_desc(qa[x] + umma_kstep(ks, kPxHalf)), umma_desc(kb + umma_kstep(ks, kPxHalf)), idesc_s, ks > 0);
                umma_commit(smem_u32(&tail->s_full[x]));
                return true;
            };
            auto values = [&](int x, int t, int nth) {               // O_x += P_x V_t, the nth of the stream
                if (!tc_wait(smem_u32(&tail->p_ready[x]), nth & 1, abort_flag)) return false;
                const int pos = v_pos(t);
                if (!wait_full(pos)) return false;
                tmem_fence_after_sync();
                const uint32_t vb = umma_desc_lo_outer(smem_u32(ring + (pos % kPxSlots) * kPxSlotBytes));
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)                       // 16 keys: 2048 bytes of V, 8 columns of P
                    umma_bf16_ta(tmem + 256 + 128 * x, tmem + 128 * x + 8 * ks, umma_desc(vb + ks * 128), idesc_o, nth > 0 || ks > 0);
                return true;
            };
            ok = tc_wait(smem_u32(&tail->q_full), 0, abort_flag);
            if (two) {
                for (int x = 0; x < 2 && ok; ++x) ok = scores(x, 0);
                if (ok) umma_commit(smem_u32(&tail->empty[k_pos(0) % kPxSlots]));
                for (int t = 0; t < n_tiles && ok; ++t) {
                    for (int x = 0; x < 2 && ok; ++x) {
                        ok = values(x, t, t);
                        if (ok && x == 1) umma_commit(smem_u32(&tail->empty[v_pos(t) % kPxSlots]));
                        if (ok && t + 1 < n_tiles) ok = scores(x, t + 1);
                    }
                    if (ok && t + 1 < n_tiles) umma_commit(smem_u32(&tail->empty[k_pos(t + 1) % kPxSlots]));
                }
            } else {
                for (int t = 0; t < min(2, n_tiles) && ok; ++t) {
                    ok = scores(t, t);
                    if (ok) umma_commit(smem_u32(&tail->empty[k_pos(t) % kPxSlots]));
                }
                for (int t = 0; t < n_tiles && ok; ++t) {
                    ok = values(t & 1, t, t >> 1);
                    if (ok) umma_commit(smem_u32(&tail->empty[v_pos(t) % kPxSlots]));
                    if (ok && t + 2 < n_tiles) {
                        ok = scores(t & 1, t + 2);
                        if (ok) umma_commit(smem_u32(&tail->empty[k_pos(t + 2) % kPxSlots]));
                    }
                }
            }
            if (!ok) tail->abort_flag = 1;
            umma_commit(smem_u32(&tail->o_full));    // also after a wait that expired: what was issued has to end
        }
    } else {
        // ------------------------------------------------------------------ softmax
        const int x = warp >> 2;                        // stream
        const int row = tid & 127;                      // TMEM lane = query row of the stream's tile
        const uint32_t t_lane = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_addr = tmem + t_lane + 128 * x, o_addr = tmem + t_lane + 256 + 128 * x;
        {   // query rows into shared memory in the layout TMA would give them; rows that do not exist are zeros
            const int tiles = two ? 2 : 1;
            for (int i = tid; i < tiles * 128 * 16; i += 256) {
                const int r = i >> 4, c = i & 15;
                uint4 v = make_uint4(0u, 0u, 0u, 0u);
                if (r < rows) {
                    const int s = r / p.g;
                    v = *reinterpret_cast<const uint4*>(p.q + ((size_t)(seq0 + s) * p.h_q + (size_t)head * p.g + (r - s * p.g)) * kHeadDim + c * 8);
                }
                uint8_t* dst = q_smem + (r >> 7) * kPxSlotBytes + (c >> 3) * kPxHalf + (r & 127) * 128 + (((c & 7) ^ (r & 7)) << 4);
                *reinterpret_cast<uint4*>(dst) = v;
            }
            fence_proxy_async_smem();
            mbar_arrive(smem_u32(&tail->q_full));
        }
        float m = -INFINITY, l = 0.f;                   // in log2 units
        const int mine = two ? n_tiles : (n_tiles - x + 1) / 2;
        for (int i = 0; i < mine; ++i) {
            const int t = two ? i : 2 * i + x;
            // a warp gives up as a whole
            if (!__all_sync(0xffffffffu, tc_wait(smem_u32(&tail->s_full[x]), i & 1, abort_flag))) { ok = false; break; }
            tmem_fence_after_sync();
            float z[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld<32>(s_addr + 32 * c, z[c]);
            const int valid = n_keys - (t0 + t) * kPxKeys;      // keys of this tile that exist
            if (valid < kPxKeys) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int k = 0; k < 32; ++k) if (c * 32 + k >= valid) z[c][k] = -INFINITY;
                // V rows behind the prefix's end hold whatever the caller has there (0 * NaN): zeros instead. In the
                // two-tile form stream B's product comes after stream A's, which waits for this.
                if (x == 0 || !two) {
                    const int pos = v_pos(t);
                    if (!__all_sync(0xffffffffu, wait_full(pos))) { ok = false; break; }
                    uint8_t* v = ring + (pos % kPxSlots) * kPxSlotBytes;
                    for (int e = row; e < (kPxKeys - valid) * 16; e += 128)
                        *reinterpret_cast<uint4*>(v + (e & 8 ? kPxHalf : 0) + (valid + (e >> 4)) * 128 + (e & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                    fence_proxy_async_smem();
                }
            }
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int k = 0; k < 32; ++k)
#pragma unroll
                for (int c = 0; c < 4; ++c) mx[c] = fmaxf(mx[c], z[c][k]);
            const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2;
            const bool raise = top > m + kPxLag;
            if (__any_sync(0xffffffffu, raise)) {
                const float m_new = raise ? top : m;
                const float f = m_new == -INFINITY ? 1.f : fast_exp2(m - m_new);
                m = m_new;
                l *= f;
                if (i > 0) {                            // O of the tiles before is complete: S was issued after it
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float o[32];
                        tmem_ld<32>(o_addr + 32 * c, o);
                        uint32_t r[32];
#pragma unroll
                        for (int k = 0; k < 32; ++k) r[k] = __float_as_uint(o[k] * f);
                        tmem_st32(o_addr + 32 * c, r);
                    }
                }
            }
            const float ref = m == -INFINITY ? 0.f : m;
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t r[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                    const int e = 2 * (k & 15), cc = 2 * c + (k >> 4);
                    const float a = fast_exp2(fmaf(z[cc][e], p.scale_log2, -ref)), b = fast_exp2(fmaf(z[cc][e + 1], p.scale_log2, -ref));
                    sum[k & 3] += a + b;
                    r[k] = pack_bf16x2(a, b);
                }
                tmem_st32(s_addr + 32 * c, r);
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            tmem_wait_st();
            tmem_fence_before_sync();
            mbar_arrive(smem_u32(&tail->p_ready[x]));
        }
        if (!ok) tail->abort_flag = 1;
        if (!tc_wait(smem_u32(&tail->o_full), 0, abort_flag)) ok = false;
        ok = __all_sync(0xffffffffu, ok && *(volatile int*)abort_flag == 0);
        // ---- the row's partial result; a wait that expired shows as NaN in the output
        float* rec = p.prefix_part + (size_t)blockIdx.x * kPrefixRecFloats;
        const int slot = 128 * x + row;
        rec[slot] = ok ? m : 0.f;
        rec[kPrefixRows + slot] = ok ? l : NAN;
        tmem_fence_after_sync();
        if (mine > 0 && ok) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float o[32];
                tmem_ld<32>(o_addr + 32 * c, o);
#pragma unroll
                for (int k = 0; k < 32; ++k) rec[2 * kPrefixRows + (32 * c + k) * kPrefixRows + slot] = o[k];
            }
        }
        tmem_fence_before_sync();
    }
    __syncthreads();
    if (*(volatile int*)&tail->abort_flag && tid == 0) {
        // copies and products that are still in flight get a bounded time to end before the CTA does
        const int issued = *(volatile int*)&tail->issued;
        for (int pos = max(0, issued - kPxSlots); pos < issued; ++pos)
            mbar_wait_bounded(smem_u32(&tail->full[pos % kPxSlots]), (pos / kPxSlots) & 1);
        mbar_wait_bounded(smem_u32(&tail->o_full), 0);
    }
    __syncthreads();
    if (warp == 9) {
        tmem_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

cudaError_t launch_prefix_attn(const StoreAttnLaunch& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v, cudaStream_t s) {
    // a property of the function on the current device; setting it again costs less than finding out whether it is set
    const cudaError_t e = cudaFuncSetAttribute(gkv_prefix_attn_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kPxSmem);
    if (e != cudaSuccess) return e;
    gkv_prefix_attn_kernel<<<(unsigned)p.prefix_items, kPxThreads, kPxSmem, s>>>(p, tm_k, tm_v);
    return cudaGetLastError();
}

}  // namespace gkv
