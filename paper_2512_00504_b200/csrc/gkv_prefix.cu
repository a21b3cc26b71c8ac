// Attention of a batch's query rows over prefixes that its sequences share: the prefix's rows are read once for all of them.
//
// The query rows of a (prefix, KV head) are the g heads of every sequence of the prefix: 8 to 2000 rows that see the same keys,
// so this is a dense product and belongs on tcgen05. A work item is up to 256 query rows and a run of 128-key tiles; its result
// (running maximum, sum, unscaled output of every row) goes to the workspace and is joined with the other runs' and with the
// sequences' own rows by the merge kernel.
//
// One CTA (one per SM: 226 KB of shared memory, all 512 TMEM columns) holds two streams, A and B, each with 128 query rows: with more than 128 rows in the item A and B have a row tile each and both see every key tile; with fewer they
// have the same rows and take the even and the odd key tiles. Per stream and key tile
//     S = Q K^T          128 x 128 x 128, operands in shared memory, S in 128 TMEM columns
//     softmax            eight warps: TMEM lane = query row, two threads per row with 64 keys each, whose maximum and sum are
//                        loops in the thread; P as bf16 goes back over the first 64 of S's columns
//     O += P V           P is read from TMEM as the A operand, V from shared memory with the head dimension contiguous (as it
//                        lies in memory: no transpose), O in 128 TMEM columns
// While one stream is in its softmax the tensor cores work for the other. A stream's steps follow one another (S, softmax, P V,
// the next S), so what counts is how long each takes: with one thread per row and 128 exponentials in a row the chain was 6200
// cycles a tile. The running maximum is the first tile's and is raised
// only when the weights of a tile sum up to more than 2^60: bf16 and fp32 have the range for it and the relative precision of
// all sums is the same, so there is no pass for the maximum and no rescaling of O (a trip of 128 columns through registers)
// but in the first tile and in extreme ones. K and V tiles come by TMA through a ring of five 32 KB slots in the order in which
// the products want them.
//
// Bound: for 256 rows a key tile costs 64 KB of HBM traffic (1.5 us of an SM's share), 2048 cycles of the tensor core and 2048
// cycles of the exponential unit: all three are level.
#include "gkv_tcgen05.cuh"
#include "gkv_internal.h"

namespace gkv {

constexpr int kPxSoftmax = 512;              // warps 0-7: stream A, 8-15: stream B (warp / 4 & 1: keys 0-63 or 64-127 of a tile)
constexpr int kPxThreads = kPxSoftmax + 64;  // warp 16: TMA, 17: MMA
constexpr int kPxTmaWarp = kPxSoftmax / 32, kPxMmaWarp = kPxTmaWarp + 1;
constexpr int kPxKeys = 128;                 // keys of a tile
constexpr int kPxHalf = 128 * 128;           // bytes of 128 rows x 64 elements
constexpr int kPxSlotBytes = 2 * kPxHalf;    // one K or V tile, or one row tile of q
constexpr int kPxSlots = 5;
constexpr float kPxLimit = 0x1p60f;          // a row's weights of one tile may sum up to this before the maximum is raised

struct __align__(16) PrefixTail {
    uint64_t q_full;
    uint64_t full[kPxSlots], empty[kPxSlots];
    uint64_t s_full[2], p_ready[2];
    uint64_t o_full;
    float row[2][128];   // [stream][row]: what the two threads of a row tell each other (a maximum, at the end a sum)
    uint32_t tmem_base;
    int abort_flag;
    int issued;        // ring slots filled so far
};
constexpr size_t kPxSmem = 1024 + 2 * kPxSlotBytes + kPxSlots * kPxSlotBytes + sizeof(PrefixTail);
static_assert(kPxSmem <= 227 * 1024, "shared memory of a CTA");

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

// 32 columns of this lane's TMEM row, without waiting; the wait names the registers, so that no use of them comes before it.
__device__ __forceinline__ void tmem_ld32_start(uint32_t taddr, float (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
          "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]),
          "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]),
          "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_ld_wait(float (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]), "+f"(r[8]),
          "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]), "+f"(r[16]), "+f"(r[17]),
          "+f"(r[18]), "+f"(r[19]), "+f"(r[20]), "+f"(r[21]), "+f"(r[22]), "+f"(r[23]), "+f"(r[24]), "+f"(r[25]), "+f"(r[26]),
          "+f"(r[27]), "+f"(r[28]), "+f"(r[29]), "+f"(r[30]), "+f"(r[31])
        :: "memory");
}
// The two warps that share 32 query rows: wait for each other; and whether a predicate holds anywhere among them.
__device__ __forceinline__ void pair_sync(int id) {
    __syncwarp();
    asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory");
}
__device__ __forceinline__ bool pair_any(int id, bool x) {
    uint32_t r;
    __syncwarp();
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\tbar.red.or.pred q, %1, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"(id), "r"((uint32_t)x) : "memory");
    return r != 0;
}
// Keys from `valid` on (32 c is the block's first) do not exist.
__device__ __forceinline__ void mask_block(float (&z)[32], int c, int valid) {
    if (32 * c + 32 > valid) {
#pragma unroll
        for (int k = 0; k < 32; ++k) if (32 * c + k >= valid) z[k] = -INFINITY;
    }
}

__global__ void __launch_bounds__(kPxThreads, 1)
gkv_prefix_attn_kernel(const StoreAttnLaunch p, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
    grid_launch_dependents();   // the attention over own rows takes the SMs as they fall free
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
        mbar_init(smem_u32(&tail->q_full), kPxSoftmax);
        for (int s = 0; s < kPxSlots; ++s) { mbar_init(smem_u32(&tail->full[s]), 1); mbar_init(smem_u32(&tail->empty[s]), 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&tail->s_full[s]), 1); mbar_init(smem_u32(&tail->p_ready[s]), kPxSoftmax / 2); }
        mbar_init(smem_u32(&tail->o_full), 1);
        tail->abort_flag = 0;
        tail->issued = 0;
        fence_mbar_init();
    }
    if (warp == kPxMmaWarp) {   // one CTA per SM holds all columns: this never waits
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
    if (warp == kPxTmaWarp) {
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
    } else if (warp == kPxMmaWarp) {
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
        const int x = warp >> 3, half = (warp >> 2) & 1;    // stream, half of a tile's keys
        const int row = tid & 127;                          // TMEM lane = query row of the stream's tile
        const int pair = 1 + (x << 2) + (warp & 3);         // named barrier of the two warps of these rows
        const uint32_t t_lane = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_addr = tmem + t_lane + 128 * x, o_addr = tmem + t_lane + 256 + 128 * x + 64 * half;
        {   // query rows into shared memory in the layout TMA would give them; rows that do not exist are zeros
            uint4 v[8];                                  // all loads first; two ? 8 : 4 of them count
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int i = tid + k * kPxSoftmax, r = i >> 4, c = i & 15;
                v[k] = make_uint4(0u, 0u, 0u, 0u);
                if (r < rows) {
                    const int s = r / p.g;
                    v[k] = *reinterpret_cast<const uint4*>(p.q + ((size_t)(seq0 + s) * p.h_q + (size_t)head * p.g + (r - s * p.g)) * kHeadDim + c * 8);
                }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int i = tid + k * kPxSoftmax, r = i >> 4, c = i & 15;
                if (k < 4 || two)
                    *reinterpret_cast<uint4*>(q_smem + (r >> 7) * kPxSlotBytes + (c >> 3) * kPxHalf + (r & 127) * 128 + (((c & 7) ^ (r & 7)) << 4)) = v[k];
            }
            fence_proxy_async_smem();
            mbar_arrive(smem_u32(&tail->q_full));
        }
        float m = -INFINITY, l = 0.f;                   // in log2 units; l: this thread's half of the keys
        const int mine = two ? n_tiles : (n_tiles - x + 1) / 2;
        for (int i = 0; i < mine; ++i) {
            const int t = two ? i : 2 * i + x;
            const int valid = n_keys - (t0 + t) * kPxKeys;      // keys of this tile that exist (128 or more: all)
            bool come = tc_wait(smem_u32(&tail->s_full[x]), i & 1, abort_flag);
            if (valid < kPxKeys && (x == 0 || !two)) {
                // V rows behind the prefix's end hold whatever the caller has there (0 * NaN): zeros instead. In the
                // two-tile form stream B's product comes after stream A's, which waits for this.
                const int pos = v_pos(t);
                come = come && wait_full(pos);
                uint8_t* v = ring + (pos % kPxSlots) * kPxSlotBytes;
                if (come)
                    for (int e = (half << 7) + row; e < (kPxKeys - valid) * 16; e += 256)
                        *reinterpret_cast<uint4*>(v + (e & 8 ? kPxHalf : 0) + (valid + (e >> 4)) * 128 + (e & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                fence_proxy_async_smem();
            }
            // the two warps go on or give up together
            if (pair_any(pair, !come)) { ok = false; break; }
            tmem_fence_after_sync();
            uint32_t w[32];                                     // this thread's weights of the tile, bf16 pairs
            float total;
            bool fresh = i == 0;                                // no maximum yet
            for (;;) {
                if (fresh) {
                    float top = -INFINITY;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float z[32];
                        tmem_ld32_start(s_addr + 64 * half + 32 * c, z);
                        tmem_ld_wait(z);
                        mask_block(z, 2 * half + c, valid);
#pragma unroll
                        for (int k = 0; k < 32; ++k) top = fmaxf(top, z[k]);
                    }
                    if (half == 0) tail->row[x][row] = top;
                    pair_sync(pair);
                    if (half == 1) tail->row[x][row] = top = fmaxf(top, tail->row[x][row]);
                    pair_sync(pair);
                    top = tail->row[x][row];
                    const float m_new = fmaxf(m, top * p.scale_log2);
                    const float f = m_new == -INFINITY ? 1.f : fast_exp2(m - m_new);
                    m = m_new;
                    l *= f;
                    if (i > 0) {                        // O of the tiles before is complete: S was issued after it
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float o[32];
                            tmem_ld32_start(o_addr + 32 * c, o);
                            tmem_ld_wait(o);
#pragma unroll
                            for (int k = 0; k < 32; ++k) w[k] = __float_as_uint(o[k] * f);
                            tmem_st32(o_addr + 32 * c, w);
                        }
                    }
                }
                const float ref = m == -INFINITY ? 0.f : -m;
                const float2 scale2 = make_float2(p.scale_log2, p.scale_log2), ref2 = make_float2(ref, ref);
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float z[32];
                    tmem_ld32_start(s_addr + 64 * half + 32 * c, z);
                    tmem_ld_wait(z);
                    mask_block(z, 2 * half + c, valid);
#pragma unroll
                    for (int k = 0; k < 32; k += 2) {
                        const float2 y = fma_f32x2(make_float2(z[k], z[k + 1]), scale2, ref2);
                        const float2 e = make_float2(fast_exp2(y.x), fast_exp2(y.y));
                        sum[(k >> 1) & 1] = add_f32x2(sum[(k >> 1) & 1], e);
                        w[16 * c + (k >> 1)] = pack_bf16x2(e.x, e.y);
                    }
                }
                total = (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                // Both warps have read S when they get past this; weights of a fresh maximum are at most 1.
                const bool over = pair_any(pair, !fresh && !(total <= kPxLimit));
                if (!over) break;
                fresh = true;
            }
            l += total;
            tmem_st32(s_addr + 32 * half, w);
            tmem_wait_st();
            tmem_fence_before_sync();
            mbar_arrive(smem_u32(&tail->p_ready[x]));
        }
        if (!ok) tail->abort_flag = 1;
        if (!tc_wait(smem_u32(&tail->o_full), 0, abort_flag)) ok = false;
        if (half == 1) tail->row[x][row] = l;
        ok = !pair_any(pair, !ok || *(volatile int*)abort_flag != 0);
        // ---- the row's partial result; a wait that expired shows as NaN in the output
        float* rec = p.prefix_part + (size_t)blockIdx.x * kPrefixRecFloats;
        const int slot = 128 * x + row;
        const bool real = (two ? slot : row) < rows;
        if (real && half == 0) {
            rec[slot] = ok ? m : 0.f;
            rec[kPrefixRows + slot] = ok ? l + tail->row[x][row] : NAN;
        }
        tmem_fence_after_sync();
        if (mine > 0 && ok && __any_sync(0xffffffffu, real)) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float o[32];
                __syncwarp();
                tmem_ld32_start(o_addr + 32 * c, o);
                tmem_ld_wait(o);
                float4* dst = reinterpret_cast<float4*>(rec + 2 * kPrefixRows) + (16 * half + 8 * c) * kPrefixRows + slot;
                if (real)
#pragma unroll
                    for (int k = 0; k < 8; ++k) dst[k * kPrefixRows] = make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
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
    if (warp == kPxMmaWarp) {
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
