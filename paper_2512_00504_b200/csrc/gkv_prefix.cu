// Attention of a batch's query rows over prefixes that its sequences share: the prefix's rows are read once for all of them.
//
// The query rows of a (prefix, KV head) are the g heads of every sequence of the prefix: 8 to 2000 rows that see the same keys,
// so this is a dense product and belongs on tcgen05. A work item is up to 256 query rows and a run of 128-key tiles; its result
// (running maximum, sum, unscaled output of every row) goes to the workspace and is joined with the other runs' and with the
// sequences' own rows by the merge kernel.
//
// One CTA (one per SM: all 512 TMEM columns) holds two streams, A and B, each with 128 query rows: with
// more than 128 rows in the item A and B have a row tile each and both see every key tile; with fewer they have the same rows
// and take the even and the odd key tiles. Per stream and key tile
//     S = Q K^T          128 x 128 x 128, operands in shared memory, S in 128 TMEM columns
//     softmax            four warps, thread = TMEM lane = query row, so that the sum over the keys is a loop in one thread; P as
//                        bf16 goes back over S columns that have been read, one half of the keys after the other
//     O += P V           P is read from TMEM as the A operand, V from shared memory with the head dimension contiguous (as it
//                        lies in memory: no transpose), O in 128 TMEM columns; the first half of the keys while the softmax is
//                        at the second
// The steps of a stream follow one another (S, softmax, P V, the next S); while one stream is in its softmax the tensor cores
// work for the other. One warp issues the products of both in turn, which keeps them out of step (with an issuer each they fall
// into step, both in the softmax and then both waiting for products: 5300 cycles a tile of 256 rows).
//
// Weights are relative to the maximum of the row's first tile, and stay so: bf16 and fp32 have the range for weights of 2^60 and
// the relative precision of all sums is the same. There is no pass for the maximum and no rescaling of O. If half a tile's
// weights do sum up to more than 2^60 in some row, or large weights make a sum of values overflow, or the first tile has no
// maximum (every logit -infinity), the item is done again, once to find the rows' maxima and once with them. P has bf16's 8 bits, the
// type that V and with it the product has: outputs are off by 1.9e-3 to 2.3e-3 where their own rounding to bf16 makes 1.65e-3.
//
// K and V tiles come by TMA through a ring of three 32 KB slots in the order in which the products want them.
//
// The kernel is a chain of waits that leaves HBM and most issue slots idle, and the attention over the sequences' own rows, which
// runs next to it, is bound by HBM: 80 registers a thread and 162 KB of shared memory leave room for two CTAs of that kernel on
// the same SM (128 registers, 8- and 4-bit rows) or one (168, bf16 rows).
//
// Bound: for 256 rows a key tile costs 64 KB of HBM traffic (1.5 us of an SM's share), 2048 cycles of the tensor core and 2048
// cycles of the exponential unit: all three are level. Measured: 3900 cycles a tile of 256 rows (2.1 us), tensor cores and
// exponentials half busy, the rest being the hand-overs between the two streams' steps; 4 prefixes of up to 16384 keys x 8 heads
// with 256 query rows each 80 us alone, 145 us with the own rows of 128 sequences (450 MB of e4m3, which alone take 75).
#include "gkv_tcgen05.cuh"
#include "gkv_internal.h"

namespace gkv {

constexpr int kPxSoftmax = 256;              // warps 0-3: stream A, 4-7: stream B
constexpr int kPxThreads = kPxSoftmax + 64;  // warp 8: TMA, 9: MMA
constexpr int kPxTmaWarp = kPxSoftmax / 32, kPxMmaWarp = kPxTmaWarp + 1;
constexpr int kPxKeys = 128;                 // keys of a tile
constexpr int kPxHalf = 128 * 128;           // bytes of 128 rows x 64 elements
constexpr int kPxSlotBytes = 2 * kPxHalf;    // one K or V tile, or one row tile of q
constexpr int kPxSlots = 3;
constexpr float kPxLimit = 0x1p60f;          // a row's weights of half a tile may sum up to this
constexpr float kPxCheck = 0x1p16f;          // from here on (in all) the row's values are looked at
constexpr float kPxSum = 0x1p115f;           // and may be this large: the merge adds up to 320 of them

struct __align__(16) PrefixTail {
    uint64_t q_full;
    uint64_t full[kPxSlots], empty[kPxSlots];
    uint64_t s_full[2], p_ready[2][2];       // per stream (and half of the keys)
    uint64_t o_full;
    uint32_t tmem_base;
    int abort_flag;
    int overflow;      // weights left their range: once more
    int issued;        // ring slots filled so far
};
constexpr size_t kPxSmem = 1024 + 2 * kPxSlotBytes + kPxSlots * kPxSlotBytes + sizeof(PrefixTail);
static_assert(kPxSmem <= 227 * 1024, "shared memory of a CTA");

// One lane of the warp, chosen by the hardware: the branch that it takes leaves the rest of the code uniform for the warp, which
// keeps descriptors in uniform registers. (The same products issued under `lane == 0` took 1580 cycles for a P V and a Q K^T of
// half a tile, more than the tensor cores need.)
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
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
// Keys from `valid` on (`key0` is the block's first) do not exist.
__device__ __forceinline__ void mask_block(float (&z)[32], int key0, int valid) {
    if (key0 + 32 > valid) {
#pragma unroll
        for (int k = 0; k < 32; ++k) if (key0 + k >= valid) z[k] = -INFINITY;
    }
}

__global__ void __maxnreg__(80)
gkv_prefix_attn_kernel(const StoreAttnLaunch p, const PrefixWatch watch, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
    grid_launch_dependents();   // the attention over own rows takes the SMs as they fall free
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* q_smem = smem;                              // two row tiles
    uint8_t* ring = smem + 2 * kPxSlotBytes;
    PrefixTail* tail = reinterpret_cast<PrefixTail*>(ring + kPxSlots * kPxSlotBytes);
    // (numbers that are the same for a warp by a shuffle, which lets the compiler keep what hangs on them in uniform registers)
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);

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

    if (warp < kPxTmaWarp) {
        // Query rows into shared memory, in the layout TMA would give them and before anything else, since they take longest to
        // come; rows that do not exist are zeros. (r / g by a multiplication: exact for r < 256, g <= 8.)
        const int inv_g = (65536 + p.g - 1) / p.g;
        const __nv_bfloat16* q0 = p.q + ((size_t)seq0 * p.h_q + (size_t)head * p.g) * kHeadDim + (tid & 15) * 8;
        for (int k = 0; k < (two ? 16 : 8); ++k) {
            const int r = (tid >> 4) + k * (kPxSoftmax / 16), c = tid & 15, rr = min(r, rows - 1), sq = rr * inv_g >> 16;
            cp_async_16_or_zeros(smem_u32(q_smem + (r >> 7) * kPxSlotBytes + (c >> 3) * kPxHalf + (r & 127) * 128 + (((c & 7) ^ (r & 7)) << 4)),
                                 q0 + ((size_t)sq * p.h_q + (rr - sq * p.g)) * kHeadDim, r < rows);
        }
        cp_async_commit();
    } else if (warp == kPxTmaWarp && elect_one()) {
        prefetch_tensormap(&tm_k);
        prefetch_tensormap(&tm_v);
    }
    if (tid == 0) {
        mbar_init(smem_u32(&tail->q_full), kPxSoftmax);
        for (int s = 0; s < kPxSlots; ++s) { mbar_init(smem_u32(&tail->full[s]), 1); mbar_init(smem_u32(&tail->empty[s]), 1); }
        for (int s = 0; s < 2; ++s) mbar_init(smem_u32(&tail->s_full[s]), 1);
        for (int s = 0; s < 4; ++s) mbar_init(smem_u32(&tail->p_ready[s >> 1][s & 1]), kPxSoftmax / 2);
        mbar_init(smem_u32(&tail->o_full), 1);
        tail->abort_flag = watch.give_up;
        tail->overflow = 0;
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
    const uint32_t tmem = __shfl_sync(0xffffffffu, *(volatile uint32_t*)&tail->tmem_base, 0);
    const int* abort_flag = &tail->abort_flag;
    // ring position of key tile t's V tile and K tile: K_0 [K_1] then V_t, K_(t + ahead) in turn, while there are such tiles
    auto v_pos = [&](int t) { return min(ahead, n_tiles) + t + min(t, max(n_tiles - ahead, 0)); };
    auto k_pos = [&](int t) { return t < ahead ? t : v_pos(t - ahead) + 1; };
    auto wait_full = [&](int pos) { return tc_wait(smem_u32(&tail->full[pos % kPxSlots]), (pos / kPxSlots) & 1, abort_flag); };

    // A stream's key tiles: first(x), first(x) + stride, ...
    const int stride = two ? 1 : 2;
    auto first = [&](int x) { return two ? 0 : x; };
    auto count = [&](int x) { return two ? n_tiles : (n_tiles - x + 1) / 2; };
    bool ok = true;
    float m = -INFINITY, l = 0.f;                        // softmax: in log2 units
    const int x = warp >> 2;                             // softmax: stream
    const int row = tid & 127;                           // TMEM lane = query row of the stream's tile
    const uint32_t t_lane = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + t_lane + 128 * x, o_addr = tmem + t_lane + 256 + 128 * x;

    // One pass over the item, or three: weights relative to the first tile's maxima; the maxima; weights relative to them. (In
    // the second pass the products run as in the others, on whatever is in P's place; the third starts O anew.)
    int pass = 0;
    for (;; ++pass) {
        const int pos0 = pass * 2 * n_tiles;             // ring positions used so far
        if (warp == kPxTmaWarp) {
            // -------------------------------------------------------------- TMA
            if (elect_one()) {
                const int row0 = (pre * p.h_kv + head) * p.prefix_rows;
                int kt = 0, vt = 0;
                for (int pos = 0; pos < 2 * n_tiles && ok; ++pos) {
                    const bool is_k = kt < n_tiles && k_pos(kt) == pos;
                    const int t = is_k ? kt++ : vt++;
                    const int at = pos0 + pos, s = at % kPxSlots;
                    if (at >= kPxSlots) ok = tc_wait(smem_u32(&tail->empty[s]), (at / kPxSlots - 1) & 1, abort_flag);
                    if (!ok) { tail->abort_flag = 1; break; }
                    const uint32_t bar = smem_u32(&tail->full[s]), dst = smem_u32(ring + s * kPxSlotBytes);
                    const CUtensorMap* mp = is_k ? &tm_k : &tm_v;
                    const int y = row0 + (t0 + t) * kPxKeys;
                    mbar_arrive_expect_tx(bar, kPxSlotBytes);
                    tma_load_2d(dst, mp, 0, y, bar);
                    tma_load_2d(dst + kPxHalf, mp, 64, y, bar);
                    *(volatile int*)&tail->issued = at + 1;
                }
            }
        } else if (warp == kPxMmaWarp) {
            // -------------------------------------------------------------- MMA (the whole warp; one lane issues)
            // What stands between two products costs the tensor cores time (they hold few products in advance): slots and
            // parities are worked out once per tile.
            const uint32_t idesc_s = umma_idesc_bf16_m128(128);
            const uint32_t idesc_o = idesc_s | (1u << 16);               // B's contiguous direction is its outer index
            const uint32_t qd0 = umma_desc_lo(smem_u32(q_smem)), qd1 = two ? umma_desc_lo(smem_u32(q_smem + kPxSlotBytes)) : qd0;
            struct Tile { uint32_t addr, full, empty, parity; };
            auto tile_at = [&](int pos) {
                const uint32_t at = (uint32_t)(pos0 + pos), s = at % kPxSlots;
                return Tile{smem_u32(ring) + s * kPxSlotBytes, smem_u32(&tail->full[s]), smem_u32(&tail->empty[s]), (at / kPxSlots) & 1};
            };
            auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, tc_wait(bar, parity, abort_flag)); };
            // S = Q K^T; O += P V. Commits arrive once all that has been issued is done; `last`: nobody reads the tile after this.
            auto scores = [&](int st, const Tile& k, bool last) {
                if (elect_one()) {
                    const uint32_t kb = umma_desc_lo(k.addr), qd = st ? qd1 : qd0;
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        umma_bf16(tmem + 128 * st, umma_desc(qd + umma_kstep(ks, kPxHalf)), umma_desc(kb + umma_kstep(ks, kPxHalf)), idesc_s, ks > 0);
                    umma_commit(smem_u32(&tail->s_full[st]));
                    if (last) umma_commit(k.empty);
                }
                __syncwarp();
            };
            auto values = [&](int st, int hf, const Tile& v, uint32_t more, bool last) {    // for half of the keys
                if (elect_one()) {
                    const uint32_t vb = umma_desc_lo_outer(v.addr);
#pragma unroll
                    for (int ks = 4 * hf; ks < 4 * hf + 4; ++ks)         // 16 keys: 2048 bytes of V, 8 columns of P
                        umma_bf16_ta(tmem + 256 + 128 * st, tmem + 128 * st + 64 * hf + 8 * (ks & 3), umma_desc(vb + ks * 128), idesc_o,
                                     ks > 0 ? 1u : more);
                    if (last) umma_commit(v.empty);
                }
                __syncwarp();
            };
            if (pass == 0) ok = wait(smem_u32(&tail->q_full), 0);
            for (int st = 0; st < 2 && ok; ++st)
                if (count(st) > 0) {
                    const Tile k = tile_at(k_pos(first(st)));
                    ok = wait(k.full, k.parity);
                    tmem_fence_after_sync();
                    if (ok) scores(st, k, !two || st == 1);
                }
            for (int nth = 0; nth < count(0) && ok; ++nth) {
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    const int n = count(st), t = first(st) + nth * stride;
                    if (nth >= n) break;
                    const bool more = nth + 1 < n, last = !two || st == 1;
                    const Tile v = tile_at(v_pos(t)), k = tile_at(more ? k_pos(t + stride) : 0);
                    ok = wait(v.full, v.parity);
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        ok = ok && wait(smem_u32(&tail->p_ready[st][hf]), (pass * n + nth) & 1);
                        if (!ok) break;
                        tmem_fence_after_sync();
                        values(st, hf, v, nth > 0, hf == 1 && last);
                    }
                    if (!ok) break;
                    if (more) {
                        ok = wait(k.full, k.parity);
                        if (!ok) break;
                        tmem_fence_after_sync();
                        scores(st, k, last);
                    }
                }
            }
            if (!ok) tail->abort_flag = 1;
            if (elect_one()) umma_commit(smem_u32(&tail->o_full));    // also after a wait that expired: what was issued has to end
            __syncwarp();
        } else {
            // -------------------------------------------------------------- softmax
            if (pass == 0) {
                cp_async_wait_all();                     // this thread's share of the query rows
                fence_proxy_async_smem();
                mbar_arrive(smem_u32(&tail->q_full));
            }
            const int mine = count(x);
            float top = -INFINITY;                       // second pass
            l = 0.f;
            for (int i = 0; i < mine; ++i) {
                const int t = first(x) + i * stride;
                const int valid = n_keys - (t0 + t) * kPxKeys;      // keys of this tile that exist (128 or more: all)
                ok = tc_wait(smem_u32(&tail->s_full[x]), (pass * mine + i) & 1, abort_flag);
                if (valid < kPxKeys) {
                    // V rows behind the prefix's end hold whatever the caller has there (0 * NaN): zeros instead
                    const int pos = pos0 + v_pos(t);
                    ok = ok && wait_full(pos);
                    uint8_t* v = ring + (pos % kPxSlots) * kPxSlotBytes;
                    if (ok)
                        for (int e = row; e < (kPxKeys - valid) * 16; e += 128)
                            *reinterpret_cast<uint4*>(v + (e & 8 ? kPxHalf : 0) + (valid + (e >> 4)) * 128 + (e & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                    fence_proxy_async_smem();
                }
                ok = __all_sync(0xffffffffu, ok);                   // a warp gives up as a whole
                if (!ok) break;
                tmem_fence_after_sync();
                if (pass == 1 || (pass == 0 && i == 0)) {
                    for (int c = 0; c < 4; ++c) {
                        float z[32];
                        tmem_ld32_start(s_addr + 32 * c, z);
                        tmem_ld_wait(z);
                        mask_block(z, 32 * c, valid);
#pragma unroll
                        for (int k = 0; k < 32; ++k) top = fmaxf(top, z[k]);
                    }
                    if (pass == 0) m = top * p.scale_log2;
                    if (pass == 0 && top == -INFINITY && mine > 1) *(volatile int*)&tail->overflow = 1;   // nothing to be relative to
                }
                const float ref = m == -INFINITY ? 0.f : -m;
                const float2 scale2 = make_float2(p.scale_log2, p.scale_log2), ref2 = make_float2(ref, ref);
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    if (pass != 1) {
                        float2 sum = make_float2(0.f, 0.f);
                        uint32_t w[32];                             // the weights of 64 keys, bf16 pairs
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float z[32];
                            tmem_ld32_start(s_addr + 64 * half + 32 * c, z);
                            tmem_ld_wait(z);
                            mask_block(z, 64 * half + 32 * c, valid);
#pragma unroll
                            for (int k = 0; k < 32; k += 2) {
                                const float2 y = fma_f32x2(make_float2(z[k], z[k + 1]), scale2, ref2);
                                const float2 e = make_float2(fast_exp2(y.x), fast_exp2(y.y));
                                sum = add_f32x2(sum, e);
                                w[16 * c + (k >> 1)] = pack_bf16x2(e.x, e.y);
                            }
                        }
                        const float total = sum.x + sum.y;
                        if (pass == 0 && !(total <= kPxLimit)) *(volatile int*)&tail->overflow = 1;  // (NaN too: it comes out again)
                        l += total;
                        tmem_st32(s_addr + 64 * half, w);
                        tmem_wait_st();
                    }
                    tmem_fence_before_sync();
                    mbar_arrive(smem_u32(&tail->p_ready[x][half]));
                }
            }
            if (!ok) tail->abort_flag = 1;
            if (pass == 1) m = top * p.scale_log2;
            if (!tc_wait(smem_u32(&tail->o_full), pass & 1, abort_flag)) ok = false;
            if (pass == 0 && __any_sync(0xffffffffu, l > kPxCheck)) {
                // large weights of a row may have carried its values out of fp32's range, or so near its end that the runs' sum leaves it
                tmem_fence_after_sync();
                bool bad = false;
                for (int c = 0; c < 4; ++c) {
                    float o[32];
                    tmem_ld32_start(o_addr + 32 * c, o);
                    tmem_ld_wait(o);
#pragma unroll
                    for (int k = 0; k < 32; ++k) bad |= !(fabsf(o[k]) <= kPxSum);
                }
                if (bad) *(volatile int*)&tail->overflow = 1;
                tmem_fence_before_sync();
            }
        }
        __syncthreads();
        if (pass == 2 || *(volatile int*)&tail->overflow == 0) break;    // (written in the first pass only)
    }
    if (warp < kPxTmaWarp) {
        // ---- the row's partial result; a wait that expired shows as NaN in the output
        ok = *(volatile int*)abort_flag == 0;
        float* rec = p.prefix_part + (size_t)blockIdx.x * kPrefixRecFloats;
        const int slot = 128 * x + row;
        const bool real = (two ? slot : row) < rows;
        if (real) {
            rec[slot] = ok ? m : 0.f;
            rec[kPrefixRows + slot] = ok ? l : NAN;
        }
        tmem_fence_after_sync();
        if (count(x) > 0 && ok && __any_sync(0xffffffffu, real)) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float o[32];
                __syncwarp();
                tmem_ld32_start(o_addr + 32 * c, o);
                tmem_ld_wait(o);
                float4* dst = reinterpret_cast<float4*>(rec + 2 * kPrefixRows) + 8 * c * kPrefixRows + slot;
                if (real)
#pragma unroll
                    for (int k = 0; k < 8; ++k) dst[k * kPrefixRows] = make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
            }
        }
        tmem_fence_before_sync();
    }
    __syncthreads();
    if (*(volatile int*)&tail->abort_flag && tid == 0) {
        if (watch.status && atomicCAS(watch.status, 0, kStatusTimeout) == 0) {
            watch.status[1] = 50;
            watch.status[2] = blockIdx.x;
        }
        // copies and products that are still in flight get a bounded time to end before the CTA does
        const int issued = *(volatile int*)&tail->issued;
        for (int pos = max(0, issued - kPxSlots); pos < issued; ++pos)
            mbar_wait_bounded(smem_u32(&tail->full[pos % kPxSlots]), (pos / kPxSlots) & 1);
        mbar_wait_bounded(smem_u32(&tail->o_full), pass & 1);
    }
    __syncthreads();
    if (warp == kPxMmaWarp) {
        tmem_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

cudaError_t launch_prefix_attn(const StoreAttnLaunch& p, const PrefixWatch& watch, const CUtensorMap& tm_k, const CUtensorMap& tm_v, cudaStream_t s) {
    // a property of the function on the current device; setting it again costs less than finding out whether it is set
    // (All of the SM's memory as shared memory, so that CTAs of the next kernel find room beside this one's.)
    cudaError_t e = cudaFuncSetAttribute(gkv_prefix_attn_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kPxSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(gkv_prefix_attn_kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e != cudaSuccess) return e;
    gkv_prefix_attn_kernel<<<(unsigned)p.prefix_items, kPxThreads, kPxSmem, s>>>(p, watch, tm_k, tm_v);
    return cudaGetLastError();
}

}  // namespace gkv
