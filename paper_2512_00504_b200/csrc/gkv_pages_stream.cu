// Decode attention over a cache in pages, for more work than a few clusters: every warp of a grid that fills the device takes an equal
// share of all steps.
//
// The units (sequence, KV head) lie one after the other, each as many steps of 16 or 32 keys long as its sequence, and warp w of W takes steps
// w * per .. (w + 1) * per - 1 of that line, per = ceil(all / W): it may begin and end inside a unit and pass through several. Whatever the lengths are,
// all warps have the same work, none waits for another, and the stream of rows from HBM does not stop at the end of a unit. A warp is a CTA, so
// that an SM's registers and shared memory hold as many as they can. A unit that one warp has to itself is finished by it; of the others (a warp's
// first or last one) it leaves a partial result, and the merge joins them. (Handing out smaller shares as warps become free, to make up for the
// parts of the device that are up to 15% slower: 196 to 214 us instead of 193 in the first case below, since there is more to merge.)
//
// Rows come by bulk copies into a ring of the warp's own, completed on a barrier of its own: with pages whose size is a multiple of the tile and
// that hold a head's rows together, one copy for a tile of K, one for each group of rows of V (four, with 8 bits eight, with 4 bits all), and
// two for their scales, all issued by one lane; with any others, one for each bf16 row, and 16 bytes a lane at a time for shorter ones (a copy
// of its own for each takes 13 cycles: in pages of 5 rows in 8 bits 216 us instead of 156. By cp.async where rows lie together, 16 bytes a lane, a
// tile costs the warp 100 more instructions: in bf16 225 us, 131071 keys in 4 bits 108). Which key is which row of the products is free
// as long as the two agree, and chosen such that lanes that read V at once find their rows at banks of their own (4 bits: of two), groups
// being 32 bytes further apart than the rows.
//
// Products and softmax are those of the attention over a store (gkv_store_rows.cuh). A row that lies on no page makes its unit NaN.
// A wait that runs out (never, but every wait ends) makes the warp's units NaN, too.
//
// Measured (with the merge; the time that the rows' bytes take at 6.46 TB/s): 128 sequences x 8 heads of about 2200 keys in bf16 in pages of 64
// 187 to 190 us (177), of 16 187 to 190, of 5 196 to 199; in 8 bits in pages of 64 109 to 112 (90), of 5 149; in 4 bits 101 (50) and 160. 16 x 4 heads of 300
// to 65535 keys in bf16 216 (206). 2 x 8 heads of up to 131071 in 4 bits 82 to 83 (42). 16-bit rows are bound by HBM. With 4-bit rows the warps
// issue in 60% of all cycles, 420 instructions a tile, of which 170 unpack codes: instructions and what they wait for bound it.
#include "gkv_pages.cuh"
#include "gkv_pages_steps.h"
#include "gkv_rotary.cuh"
#include "gkv_store_rows.cuh"

namespace gkv {

// Warps of an SM, a CTA each: as many as shared memory has room for, three for each scheduler. (bf16 rows that lie together come in copies so
// large that two are enough: 128 sequences x 8 heads of about 2200 keys in pages of 16 191 us, with 12 warps 199. Apart, 16 x 4 heads: 218
// with 12, 296 with 8. 4 bits, 2 x 8 of up to 131071, before later steps: 89, 99; 14 or 16 leave too few registers.)
__host__ __device__ constexpr int stream_warps(int format, bool together) { return format == GKV_STORE_BF16 && together ? 8 : 12; }

// 16-key tiles of a step: what is done once a step (waiting, finding rows, issuing copies) then counts for two of them. bf16 rows are so
// long that one is enough, and two would leave a ring without stages.
__host__ __device__ constexpr int stream_tiles(int format) { return format == GKV_STORE_BF16 ? 1 : 2; }

template <int F>
struct __align__(16) StreamWarp {
    static constexpr int kRow = StoreFormat<F>::kRow, kScales = StoreFormat<F>::kScales;
    static constexpr int kTiles = stream_tiles(F), kKeys = kTiles * kTile;
    static constexpr int kStages = F == GKV_STORE_INT4 ? 3 : 2;
    // Of V, rows of a group, bytes from one group to the next. The shorter the rows, the more a copy for each group costs against what
    // the banks' conflicts do.
    static constexpr int kGroupRows = F == GKV_STORE_INT4 ? kKeys : F == GKV_STORE_BF16 ? 4 : 8;
    static constexpr int kGroup = kGroupRows * kRow + (F == GKV_STORE_INT4 ? 0 : 32);
    static constexpr int kV = kKeys * kRow, kKS = kV + kKeys / kGroupRows * kGroup, kVS = kKS + kKeys * kScales * 2;   // where V and scales begin
    static constexpr int kBytes = kVS + kKeys * kScales * 2;
    uint8_t ring[kStages][kBytes];
    __nv_bfloat16 row[4][kHeadDim];                        // heads as they are turned; the new key (0), and its and its value's codes (2, 3)
    __nv_bfloat16 scale[2][4];
    float v[value_groups(F)][8];
    uint32_t rows[kStages][kKeys];                         // numbers of the rows, where they do not lie together
    uint64_t full[kStages];

    static __device__ __forceinline__ int k_at(int key) { return key * kRow; }
    static __device__ __forceinline__ int v_at(int key) { return kV + key / kGroupRows * kGroup + key % kGroupRows * kRow; }
    // The keys of a tile behind row r = q + 8 hf of the first product, and (i = 0 .. 3) behind the four that lane j has in the second,
    // k = 2j, 2j + 1, 2j + 8, 2j + 9: the two agree.
    static __device__ __forceinline__ int key_of(int q, int hf) {
        return F == GKV_STORE_INT4 ? (q >> 1) + 4 * (q & 1) + 8 * hf : 4 * (q >> 1) + (q & 1) + 2 * hf;
    }
    static __device__ __forceinline__ int key_of_value(int j, int i) { return F == GKV_STORE_INT4 ? j + 4 * i : 4 * j + i; }
};

// A place in the line of steps: every unit has as many as its rows take, KEYS each.
template <int KEYS>
__device__ __forceinline__ int stream_steps(const PagesAttnLaunch& p, int seq) {
    if (seq >= p.batch) return 0;
    const int len = p.len[seq], n = p.k_new ? 1 : 0;
    return len < 0 || len > p.capacity - n ? 0 : (len + n + KEYS - 1) / KEYS;
}
struct StreamPlace {
    int seq, head, tile, tiles, len;                       // tile of so many, KEYS keys each; rows of the sequence in the cache
};
// On to the next one: there is one, as long as nobody changes the lengths meanwhile; if somebody does, this ends all the same.
template <int KEYS>
__device__ __forceinline__ void stream_next(const PagesAttnLaunch& p, StreamPlace& c) {
    if (++c.tile < c.tiles) return;
    c.tile = 0;
    if (++c.head < p.h_kv) return;
    c.head = 0;
    while (c.seq < p.batch - 1) {
        c.tiles = stream_steps<KEYS>(p, ++c.seq);
        if (c.tiles > 0) break;
    }
    c.len = p.len[c.seq];
}
// Steps of all units, and of those of the sequences before `seq`. The first 128 sequences' are kept: lane l's of sequences 32 k + l.
constexpr int kKept = 4;
template <int KEYS>
__device__ __forceinline__ int64_t stream_total(const PagesAttnLaunch& p, int seq, int lane, int (&kept)[kKept], int64_t* before) {
    int64_t all = 0, part = 0;
#pragma unroll
    for (int k = 0; k < kKept; ++k) kept[k] = stream_steps<KEYS>(p, 32 * k + lane);
#pragma unroll
    for (int k = 0; k < kKept; ++k) {
        all += kept[k];
        if (32 * k + lane < seq) part += kept[k];
    }
    for (int b = 32 * kKept + lane; b < p.batch; b += 32) {
        const int t = stream_steps<KEYS>(p, b);
        all += t;
        if (b < seq) part += t;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        all += __shfl_xor_sync(0xffffffffu, all, o);
        part += __shfl_xor_sync(0xffffffffu, part, o);
    }
    *before = part * p.h_kv;
    return all * p.h_kv;
}
// A warp's share of the steps.
__device__ __forceinline__ int64_t stream_share(int64_t all, int warps) {
    const int64_t per = all < 1ll << 30 ? (int64_t)(((uint32_t)all + (uint32_t)warps - 1) / (uint32_t)warps) : (all + warps - 1) / warps;
    return per < kStreamLeast ? kStreamLeast : per;
}
__device__ __forceinline__ int stream_owner(int64_t step, int64_t per) {
    return step < 1ll << 30 && per < 1ll << 30 ? (int)((uint32_t)step / (uint32_t)per) : (int)(step / per);
}

// How rows lie: anyhow; those of a tile, or of a whole step, next to one another in one page.
enum { kApart = 0, kTiles = 1, kSteps = 2 };

// expire: the step of every warp from which on waits are taken for expired (self-test; kNeverExpire otherwise).
template <int F, int LIE>
__global__ void __launch_bounds__(32, stream_warps(F, LIE != kApart)) gkv_pages_stream_kernel(const PagesAttnLaunch p, const int expire) {
    using Warp = StreamWarp<F>;
    constexpr int NG = value_groups(F), S = Warp::kStages, TILES = Warp::kTiles, KEYS = Warp::kKeys, kRow = Warp::kRow, kScales = Warp::kScales;
    constexpr bool kScaled = F != GKV_STORE_BF16, TOGETHER = LIE != kApart;
    extern __shared__ __align__(128) uint8_t s_raw[];
    const int lane = threadIdx.x;
    Warp& sw = *reinterpret_cast<Warp*>(s_raw);
    grid_launch_dependents();

    // ---- this warp's steps
    const int w = blockIdx.x;
    int64_t none;
    int kept[kKept];
    const int64_t all = stream_total<KEYS>(p, 0, lane, kept, &none);
    const int64_t per = stream_share(all, (int)gridDim.x), begin = w * per;
    if (begin >= all) return;
    const int steps = (int)(all - begin < per ? all - begin : per);
    StreamPlace ahead;
    {
        int64_t left = begin;                              // steps between sequence b's first and ours
        bool found = false;
#pragma unroll 1
        for (int b = 0; b < p.batch; b += 32) {
            const int t = b == 0 ? kept[0] : b == 32 ? kept[1] : b == 64 ? kept[2] : b == 96 ? kept[3] : stream_steps<KEYS>(p, b + lane);
            int64_t upto = (int64_t)t * p.h_kv;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t x = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += x;
            }
            const unsigned past = __ballot_sync(0xffffffffu, upto > left);
            if (past) {
                const int at = __ffs(past) - 1;
                ahead.seq = b + at;
                ahead.tiles = __shfl_sync(0xffffffffu, t, at);
                left -= __shfl_sync(0xffffffffu, upto, at) - (int64_t)ahead.tiles * p.h_kv;
                found = true;
                break;
            }
            left -= __shfl_sync(0xffffffffu, upto, 31);
        }
        if (!found) return;                                // (somebody has changed the lengths)
        ahead.head = (int)(left < 1ll << 31 ? (uint32_t)left / (uint32_t)ahead.tiles : left / ahead.tiles);
        ahead.tile = (int)(left - (int64_t)ahead.head * ahead.tiles);
        ahead.len = p.len[ahead.seq];
    }
    StreamPlace at = ahead;
    const int added = p.k_new ? 1 : 0;

    const int q = lane >> 2, j = lane & 3, h0 = 2 * j;
    // A unit's heads: their elements, and the operand made of them.
    uint32_t qf[8][2];
    float f0 = 0.f, f1 = 0.f;
    HeadTurn::Words e[kMaxGroup];
    auto position = [&]() { return p.pos ? p.pos[at.seq] : added ? at.len : at.len - 1; };
    auto load_heads = [&]() {
        const HeadTurn turn(p.rotary, lane);
        const __nv_bfloat16* x = p.q + ((int64_t)at.seq * p.q_stride + (int64_t)at.head * p.g * kHeadDim);
#pragma unroll
        for (int h = 0; h < kMaxGroup; ++h)
            if (h < p.g) e[h] = turn.load(x + h * kHeadDim);
    };
    auto make_heads = [&]() {
        const HeadTurn turn(p.rotary, lane);
        const HeadTurn::Angles g = turn.angles(position());
#pragma unroll
        for (int h4 = 0; h4 < kMaxGroup; h4 += 4)
            if (h4 < p.g) {
#pragma unroll
                for (int h = 0; h < 4; ++h)
                    if (h4 + h < p.g) turn.put(sw.row[h], e[h4 + h], g);
                __syncwarp();
                const int mine = min(q, p.g - 1) - h4;
                if (mine >= 0 && mine < 4)
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) load_query<F>(sw.row[mine], ks, j, qf[ks][0], qf[ks][1]);
                __syncwarp();
            }
        f0 = f1 = p.scale_log2;
        scale_queries<F>(lane, qf, f0, f1);
    };
    load_heads();                                          // the first unit's, ahead of the ring's many bytes

    if (lane == 0) {
#pragma unroll
        for (int s = 0; s < S; ++s) mbar_init(smem_u32(&sw.full[s]), kScaled && !TOGETHER ? 32 : 1);
        fence_mbar_init();
    }
    __syncwarp();

    // ---- rows on their way: the table's entries a step ahead of the copies. A lane looks up its key's, its tile's first one's, or all of them their
    // step's first one's, and that only where a page begins.
    const int mine = LIE == kSteps ? 0 : TOGETHER ? (lane >> 4) * kTile : lane;      // that key within the step
    auto lookup = [&](int& slot, int32_t& entry) {
        if (LIE == kSteps && ahead.tile > 0 && slot + KEYS < p.pages.page_size) {
            slot += KEYS;
            return;
        }
        const int key = ahead.tile * KEYS + mine;
        entry = 0;
        if (LIE != kSteps && (mine >= KEYS || key >= ahead.len + added)) return;      // no such key
        const int page = page_of(p.pages, key);
        slot = key - page * p.pages.page_size;
        entry = p.pages.table[ahead.seq * p.pages.table_stride + page];
    };
    int issued = 0, next_slot = p.pages.page_size;         // (no page has been looked up yet)
    int32_t next;
    lookup(next_slot, next);
    uint32_t lost = 0;                                     // stages with a row on no page
    auto issue = [&](int stage) {
        const int key0 = ahead.tile * KEYS, here = ahead.len - key0;       // rows in the cache from key0 on
        const bool page = (uint32_t)next < (uint32_t)p.pages.n_pages;
        const uint32_t row = (uint32_t)next * p.pages.page_rows + (uint32_t)ahead.head * p.pages.head_rows + (uint32_t)next_slot * p.pages.token_rows;
        const bool fine = LIE == kSteps ? page : __all_sync(0xffffffffu, page || mine >= KEYS || key0 + mine >= ahead.len + added);
        lost = fine ? lost & ~(1u << stage) : lost | 1u << stage;
        const uint32_t bar = smem_u32(&sw.full[stage]), to = smem_u32(sw.ring[stage]);
        const int n = fine ? min(max(here, 0), KEYS) : 0;                  // rows to be copied
        if constexpr (TOGETHER) {
            // One lane issues them all, with numbers that are the same for the warp: a copy takes a few instructions then, and many where every lane
            // has its own.
            constexpr bool joined = LIE == kSteps;
            constexpr int part = joined ? KEYS : kTile;
            const uint32_t first[2] = {__shfl_sync(0xffffffffu, row, 0), joined ? 0u : __shfl_sync(0xffffffffu, row, 16)};
            if (elect_one()) {
                const int scaled = kScaled ? (n + kTile - 1) / kTile * kTile * kScales * 4 : 0;
                mbar_arrive_expect_tx(bar, (uint32_t)(2 * n * kRow + scaled));
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    const int rows = min(n - t * kTile, part), key = t * kTile;
                    if (rows <= 0 || (t > 0 && joined)) break;
                    const uint8_t *ks = p.pages.data[0] + (size_t)first[t] * kRow, *vs = p.pages.data[1] + (size_t)first[t] * kRow;
                    bulk_load(to + Warp::k_at(key), ks, (uint32_t)(rows * kRow), bar);
                    if constexpr (F == GKV_STORE_INT4) {
                        bulk_load(to + Warp::v_at(key), vs, (uint32_t)(rows * kRow), bar);
                    } else {
#pragma unroll
                        for (int g = 0; g < KEYS; g += Warp::kGroupRows)
                            if (rows > g) bulk_load(to + Warp::v_at(key + g), vs + g * kRow, (uint32_t)(min(rows - g, Warp::kGroupRows) * kRow), bar);
                    }
                    if constexpr (kScaled) {               // those of whole tiles: 16 bytes are the least
                        const uint32_t bytes = (uint32_t)((rows + kTile - 1) / kTile * kTile * kScales * 2);
                        bulk_load(to + Warp::kKS + key * kScales * 2, p.pages.scale[0] + (size_t)first[t] * kScales, bytes, bar);
                        bulk_load(to + Warp::kVS + key * kScales * 2, p.pages.scale[1] + (size_t)first[t] * kScales, bytes, bar);
                    }
                }
            }
            __syncwarp();
        } else {
            if (lane < KEYS) sw.rows[stage][lane] = key0 + lane >= ahead.len + added ? kNoRow : page ? row : kNoPage;
            if constexpr (kScaled) {
                constexpr int kPer = kRow / 16;            // pieces of a row
#pragma unroll
                for (int i = 0; i < KEYS * kPer / 32; ++i) {
                    const int key = i * (32 / kPer) + lane / kPer, piece = lane % kPer * 16;
                    const size_t src = (size_t)__shfl_sync(0xffffffffu, row, key) * kRow + piece;
                    if (key < n) {
                        cp_async_16(to + Warp::k_at(key) + piece, p.pages.data[0] + src);
                        cp_async_16(to + Warp::v_at(key) + piece, p.pages.data[1] + src);
                    }
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
            } else {
                if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)(2 * n * kRow));
                if (lane < n) {
                    bulk_load(to + Warp::k_at(lane), p.pages.data[0] + (size_t)row * kRow, kRow, bar);
                    bulk_load(to + Warp::v_at(lane), p.pages.data[1] + (size_t)row * kRow, kRow, bar);
                }
            }
        }
        if (++issued < steps) {
            stream_next<KEYS>(p, ahead);
            lookup(next_slot, next);
            if (ahead.tile == 0) {                         // a unit begins: what it will ask for comes closer
                const __nv_bfloat16* x = p.q + ((int64_t)ahead.seq * p.q_stride + (int64_t)ahead.head * p.g * kHeadDim) + lane * 64;
                if (lane >= 2 * p.g) x = (lane & 2 ? p.v_new : p.k_new) + ((int64_t)ahead.seq * p.kv_stride + (int64_t)ahead.head * kHeadDim) + (lane & 1) * 64;
                if (lane < 2 * p.g || (added && lane < 2 * p.g + 4)) asm volatile("prefetch.global.L2 [%0];" ::"l"(x));
            }
        }
    };
#pragma unroll
    for (int s = 0; s < S; ++s)
        if (issued < steps) issue(s);

    const int key[2] = {Warp::key_of(q, 0), Warp::key_of(q, 1)};       // this lane's keys of a tile, for the logits
    TileK<F> tk;
    TileV<F> tv;
    auto take_scales = [&](auto& t, int which, int stage, int tile) {
        if constexpr (kScaled) {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                if constexpr (TOGETHER) {
                    const uint32_t a = smem_u32(sw.ring[stage]) + (which ? Warp::kVS : Warp::kKS) + (tile * kTile + key[hf]) * 2 * kScales;
                    if constexpr (F == GKV_STORE_INT4) t.s[hf] = lds8(a);
                    else t.s[hf] = lds2(a);
                } else {
                    const uint32_t r = sw.rows[stage][tile * kTile + key[hf]];
                    const __nv_bfloat16* s = p.pages.scale[which] + (size_t)r * kScales;
                    if constexpr (F == GKV_STORE_INT4) t.s[hf] = r < kNoPage ? ld8(s) : make_uint2(0u, 0u);
                    else t.s[hf] = r < kNoPage ? ld2(s) : 0u;
                }
            }
        }
    };
    RunningRows<F> r;
    bool whole = at.tile == 0, ok = true;                  // the unit is ours from its first tile on; no wait has run out
    bool first_unit = true;
    RingPlace<S> place;                                    // of the step that is waited for; stays where a wait has run out
    __syncwarp();
    if (!TOGETHER) {                                       // scales by ordinary loads: a tile ahead
        take_scales(tk, 0, 0, 0);
        take_scales(tv, 1, 0, 0);
    }
    make_heads();
    r.start(sw.v, lane);
    for (int step = 0; step < steps; ++step) {
        // ---- a step
        const int stage = place.stage;
        if (ok && (step >= expire || !__all_sync(0xffffffffu, mbar_wait_bounded(smem_u32(&sw.full[stage]), place.parity)))) {
            ok = false;
            issued -= step;                                // what is under way: this step's copies and those behind it
        }
        const int left = at.len + added - at.tile * KEYS;                        // keys from this step's first on
        const bool last = at.tile == at.tiles - 1, bad = !ok || (lost >> stage & 1u);
        if (last) {
            // What V and its scales have behind the end, whatever it is, becomes zeros.
            constexpr int kPer = kRow / 16;
            for (int i = lane; i < (KEYS - left) * kPer; i += 32) {
                const int gone = left + i / kPer;
                *reinterpret_cast<uint4*>(sw.ring[stage] + Warp::v_at(gone) + i % kPer * 16) = make_uint4(0u, 0u, 0u, 0u);
                if (kScaled && TOGETHER && i % kPer == 0) {
                    uint8_t* z = sw.ring[stage] + Warp::kVS + gone * 2 * kScales;
                    if (F == GKV_STORE_INT4) *reinterpret_cast<uint2*>(z) = make_uint2(0u, 0u);
                    else *reinterpret_cast<uint16_t*>(z) = 0;
                }
            }
            if (added) {
                // The new row, its last key: turned, quantised, into its page and into the tile.
                const int64_t new_row = (int64_t)at.seq * p.kv_stride + (int64_t)at.head * kHeadDim;
                const __nv_bfloat16 *kn = p.k_new + new_row, *vn = p.v_new + new_row;
                const HeadTurn turn(p.rotary, lane);
                const int32_t e = page_entry(p.pages, p.pages.table + at.seq * p.pages.table_stride, at.len);
                turn.put(sw.row[0], turn.load(kn), turn.angles(position()));
                __syncwarp();
                kn = sw.row[0];
                const uint4 x = store_load_source<F>(lane < 16 ? kn : vn, lane & 15);
                const uint32_t to = page_row(p.pages, e, (uint32_t)at.head * p.pages.head_rows, at.len);
                store_put_row<F>(reinterpret_cast<uint8_t*>(sw.row[2 + (lane >> 4)]), sw.scale[lane >> 4], lane & 15, x);
                if (to < kNoPage)
                    store_put_row<F>(p.pages.data[lane >> 4] + (size_t)to * kRow, p.pages.scale[lane >> 4] + (size_t)to * kScales, lane & 15, x);
                __syncwarp();
                uint8_t* dst = sw.ring[stage] + (lane < 16 ? Warp::k_at(left - 1) : Warp::v_at(left - 1));
                if ((lane & 15) < kPer) reinterpret_cast<uint4*>(dst)[lane & 15] = reinterpret_cast<const uint4*>(sw.row[2 + (lane >> 4)])[lane & 15];
                if (kScaled && TOGETHER && lane < 2 * kScales) {       // (the others take them below)
                    constexpr int kDiv = kScales > 0 ? kScales : 1;
                    __nv_bfloat16* z = reinterpret_cast<__nv_bfloat16*>(sw.ring[stage] + (lane < kDiv ? Warp::kKS : Warp::kVS)) + (left - 1) * kScales;
                    z[lane % kDiv] = sw.scale[lane / kDiv][lane % kDiv];
                }
            }
            fence_proxy_async_smem();                      // before the ring's next copies
            __syncwarp();
        }
        const uint32_t base = smem_u32(sw.ring[stage]);
        auto logits = [&](int tile, float (&z)[4]) {
            const int keys = left - tile * kTile;          // of this tile and on
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                for (int c = 0; c < (F == GKV_STORE_BF16 ? 4 : F == GKV_STORE_INT4 ? 1 : 2); ++c)
                    tk.d[hf][c] = lds16(base + Warp::k_at(tile * kTile + key[hf]) + j * 16 + c * 64);
            tile_logits<F>(tk, qf, f0, f1, z);
            if (keys < kTile) {
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
                    if (key[hf] >= keys) z[2 * hf] = z[2 * hf + 1] = -INFINITY;
            }
            if (bad) z[0] = z[1] = z[2] = z[3] = NAN;
        };
        auto values = [&](int tile, const float (&z)[4]) {
            uint32_t b[NG][2];
            r.weigh_tile(z, tv, sw.v, lane, b);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t a = base + Warp::v_at(tile * kTile + Warp::key_of_value(j, i)) + q * (F == GKV_STORE_INT4 ? 8 : 16);
                if constexpr (F == GKV_STORE_INT4) tv.d[i] = lds8(a);
                else if constexpr (F == GKV_STORE_BF16) {
                    tv.d[i][0] = lds16(a);
                    tv.d[i][1] = lds16(a + 128);
                } else tv.d[i] = lds16(a);
            }
            tile_values<F, NG>(tv, b, r.acc);
        };
        if constexpr (TOGETHER && TILES > 1) {
            // The logits of both tiles, then the rest of both: more at a time that does not wait for one another (tile by tile 131071 keys in 4 bits
            // 84 us instead of 83; as a loop that is not unrolled 88). A tile behind the end has no weights, and zeros for V.
            float z[TILES][4];
#pragma unroll
            for (int tile = 0; tile < TILES; ++tile) {
                take_scales(tk, 0, stage, tile);
                logits(tile, z[tile]);
            }
#pragma unroll
            for (int tile = 0; tile < TILES; ++tile) {
                take_scales(tv, 1, stage, tile);
                values(tile, z[tile]);
            }
        } else {
#pragma unroll
            for (int tile = 0; tile < TILES; ++tile) {
                const int keys = left - tile * kTile;
                if (keys <= 0) break;
                if (TOGETHER) {
                    take_scales(tk, 0, stage, tile);
                    take_scales(tv, 1, stage, tile);
                } else if (kScaled && last && added) {     // the new row's
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf)
                        if (key[hf] == keys - 1) {
                            if constexpr (F == GKV_STORE_INT4) {
                                tk.s[hf] = *reinterpret_cast<const uint2*>(sw.scale[0]);
                                tv.s[hf] = *reinterpret_cast<const uint2*>(sw.scale[1]);
                            } else if constexpr (kScaled) {
                                tk.s[hf] = *reinterpret_cast<const uint16_t*>(sw.scale[0]);
                                tv.s[hf] = *reinterpret_cast<const uint16_t*>(sw.scale[1]);
                            }
                        }
                }
                float z[4];
                logits(tile, z);
                values(tile, z);
                if (!TOGETHER && tile + 1 < TILES && keys > kTile) {
                    take_scales(tk, 0, stage, tile + 1);
                    take_scales(tv, 1, stage, tile + 1);
                }
            }
        }
        __syncwarp();                                      // the slot has been read
        if (issued < steps && ok) issue(stage);
        if (ok) place.next();
        if (!TOGETHER && step + 1 < steps) {
            __syncwarp();
            take_scales(tk, 0, place.stage, 0);
            take_scales(tv, 1, place.stage, 0);
        }
        // ---- the end of the unit, or of this warp's part of it
        if (last || step + 1 == steps) {
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                r.l0 += __shfl_xor_sync(0xffffffffu, r.l0, o);
                r.l1 += __shfl_xor_sync(0xffffffffu, r.l1, o);
            }
            auto top = [&](int g, int h) {                 // what the accumulators of a group of dimensions are relative to
                if constexpr (NG > 1) return sw.v[g][h0 + h] - kLift;
                else if constexpr (kScaled) return (h ? r.v1 : r.v0) - kLift;
                else return h ? r.m1 : r.m0;
            };
            if (whole && last) {
                const size_t out = ((size_t)at.seq * p.h_q + (size_t)at.head * p.g + h0) * kHeadDim;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int d = out_dim<F>(i, q), g = i / (8 / NG);
                    if (h0 < p.g)
                        *reinterpret_cast<uint32_t*>(p.out + out + d) = pack_bf16x2(final_value(r.acc[i][0], r.m0, r.l0, top(g, 0), true),
                                                                                    final_value(r.acc[i][2], r.m0, r.l0, top(g, 0), true));
                    if (h0 + 1 < p.g)
                        *reinterpret_cast<uint32_t*>(p.out + out + kHeadDim + d) = pack_bf16x2(final_value(r.acc[i][1], r.m1, r.l1, top(g, 1), true),
                                                                                               final_value(r.acc[i][3], r.m1, r.l1, top(g, 1), true));
                }
                if (p.lse && q == 0) {
                    float* lse = p.lse + (size_t)at.seq * p.h_q + (size_t)at.head * p.g + h0;
                    if (h0 < p.g) lse[0] = final_lse(r.m0, r.l0, true);
                    if (h0 + 1 < p.g) lse[1] = final_lse(r.m1, r.l1, true);
                }
            } else {
                float* rec = p.own_part + (size_t)(2 * w + (first_unit ? 0 : 1)) * kStreamRecFloats;
                if (q == 0) {
                    *reinterpret_cast<float2*>(rec + h0) = make_float2(r.m0, r.m1);
                    *reinterpret_cast<float2*>(rec + 8 + h0) = make_float2(r.l0, r.l1);
#pragma unroll
                    for (int g = 0; g < NG; ++g) *reinterpret_cast<float2*>(rec + 16 + 8 * g + h0) = make_float2(top(g, 0), top(g, 1));
                }
                float4* o = reinterpret_cast<float4*>(rec + kStreamRecHead) + lane;
#pragma unroll
                for (int i = 0; i < 8; ++i) o[32 * i] = make_float4(r.acc[i][0], r.acc[i][1], r.acc[i][2], r.acc[i][3]);
            }
            first_unit = false;
            if (step + 1 == steps) break;
            __syncwarp();
            stream_next<KEYS>(p, at);
            whole = true;
            load_heads();
            make_heads();
            r.start(sw.v, lane);
        } else {
            stream_next<KEYS>(p, at);
        }
    }
    // What is still on its way gets a bounded time to arrive, before this shared memory is another's.
    if (!ok) drain_ring(place, issued, [&](int s, uint32_t parity) { mbar_wait_bounded(smem_u32(&sw.full[s]), parity); });
}

// Joins the partial results of a unit: a running softmax over them, kJoin at a time, all of whose loads are under way before the first is
// looked at. A warp has two dimensions of every lane's (a slice), or kSlices times that; 2^split CTAs a unit, each with its slices, and 2^split shares of
// the parts. It takes 5 to 8 us behind the stream, trips to memory one after the other. Up to two units an SM (296): kJoin = 8, 128 registers, two CTAs of 256
// threads an SM (16 x 4 heads of 300 to 65535 keys, 100 parts of the longest: 2 at a time 219 us, 8 216). More of them: kJoin = 2, CTAs of 128 threads, so
// that those of 1184 units fit the device at once (128 x 8 heads in 8 bits 110 us; with 256 threads, 740 at once, 112).
template <int F, int kJoin, int kSlices>
__global__ void __launch_bounds__(256 / kSlices, kSlices == 2 ? 8 : 2) gkv_pages_stream_merge_kernel(const PagesAttnLaunch p, const int warps, const int split) {
    constexpr int NG = value_groups(F), KEYS = StreamWarp<F>::kKeys;
    const int unit = blockIdx.x >> split, seq = unit / p.h_kv, head = unit - seq * p.h_kv;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int slices = (8 >> split) / kSlices, share = warp / slices;          // warps that share a part; which of the parts
    int64_t before;
    int kept[kKept];
    const int64_t all = stream_total<KEYS>(p, seq, lane, kept, &before);
    const int64_t per = stream_share(all, warps);
    const int len = p.len[seq], tiles = stream_steps<KEYS>(p, seq);
    const int64_t first = before + (int64_t)head * tiles;
    const int w0 = stream_owner(first, per), n = tiles ? stream_owner(first + tiles - 1, per) - w0 + 1 : 0;
    const size_t out = ((size_t)seq * p.h_q + (size_t)head * p.g) * kHeadDim;
    const int slice0 = (blockIdx.x & ((1 << split) - 1)) * slices * kSlices + warp % slices;      // two dimensions each: slice0, slice0 + slices ..
    const int q = lane >> 2, h0 = 2 * (lane & 3);
    grid_wait_previous();                                  // (nobody leaves before: what comes next waits for this kernel alone)
    if (len < 0 || n == 1) return;                         // left out, or finished by the warp that had it
    if (n == 0) {
        const bool fits = p.k_new ? len < p.capacity : len <= p.capacity;
        if (share != 0) return;
        const uint32_t x = fits ? 0u : 0x7fff7fffu;        // bf16 NaN
#pragma unroll
        for (int k = 0; k < kSlices; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (h0 + h < p.g) *reinterpret_cast<uint32_t*>(p.out + out + (h0 + h) * kHeadDim + out_dim<F>(slice0 + k * slices, q)) = x;
        if (p.lse && slice0 == 0 && lane < p.g) p.lse[(size_t)seq * p.h_q + (size_t)head * p.g + lane] = fits ? -INFINITY : NAN;
        return;
    }
    // Part i is warp w0 + i's: the first of its two, but where the unit begins inside a warp's share its last one.
    const bool inside = first != w0 * per;
    struct Values { float2 v; float4 o; };                 // relative to 2^v; dimension d of heads h0 and h0 + 1, then d + 1
    float2 m = make_float2(-INFINITY, -INFINITY), l = make_float2(0.f, 0.f);
    Values r[kSlices];
#pragma unroll
    for (int k = 0; k < kSlices; ++k) r[k] = Values{m, make_float4(0.f, 0.f, 0.f, 0.f)};
    // Takes in another result: weights al relative to 2^am, and by slice its values; am = -infinity: no key, its values may be missing.
    auto raise = [&](float2 am) {
        const float2 nm = make_float2(fmaxf(m.x, am.x), fmaxf(m.y, am.y));
        l.x *= fast_exp2(m.x - finite_ref(nm.x)); l.y *= fast_exp2(m.y - finite_ref(nm.y));
        m = nm;
    };
    auto raise_values = [&](Values& r, float2 av) {
        const float2 nv = make_float2(fmaxf(r.v.x, av.x), fmaxf(r.v.y, av.y));
        const float e0 = fast_exp2(r.v.x - finite_ref(nv.x)), e1 = fast_exp2(r.v.y - finite_ref(nv.y));
        r.o.x *= e0; r.o.z *= e0; r.o.y *= e1; r.o.w *= e1;
        r.v = nv;
    };
    auto add = [&](float2 am, float2 al) {
        l.x += al.x * fast_exp2(am.x - finite_ref(m.x));   // (a NaN sum may come with a maximum of -infinity)
        l.y += al.y * fast_exp2(am.y - finite_ref(m.y));
    };
    auto add_values = [&](Values& r, float2 am, const Values& a) {
        const float e0 = am.x == -INFINITY ? 0.f : fast_exp2(a.v.x - finite_ref(r.v.x)), e1 = am.y == -INFINITY ? 0.f : fast_exp2(a.v.y - finite_ref(r.v.y));
        if (e0 != 0.f) { r.o.x = fmaf(a.o.x, e0, r.o.x); r.o.z = fmaf(a.o.z, e0, r.o.z); }
        if (e1 != 0.f) { r.o.y = fmaf(a.o.y, e1, r.o.y); r.o.w = fmaf(a.o.w, e1, r.o.w); }
    };
    const int step = 1 << split;
    for (int i0 = share; i0 < n; i0 += kJoin * step) {
        float2 am[kJoin], al[kJoin];
        Values x[kJoin][kSlices];
#pragma unroll
        for (int i = 0; i < kJoin; ++i) {
            const int part = i0 + i * step;
            am[i] = make_float2(-INFINITY, -INFINITY);
            al[i] = make_float2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kSlices; ++k) x[i][k] = Values{am[i], make_float4(0.f, 0.f, 0.f, 0.f)};
            if (part < n) {
                const float* a = p.own_part + (size_t)(2 * (w0 + part) + (part == 0 && inside ? 1 : 0)) * kStreamRecFloats;
                am[i] = *reinterpret_cast<const float2*>(a + h0);
                al[i] = *reinterpret_cast<const float2*>(a + 8 + h0);
#pragma unroll
                for (int k = 0; k < kSlices; ++k) {
                    const int slice = slice0 + k * slices;
                    x[i][k].v = *reinterpret_cast<const float2*>(a + 16 + 8 * (slice / (8 / NG)) + h0);
                    x[i][k].o = reinterpret_cast<const float4*>(a + kStreamRecHead)[32 * slice + lane];
                }
            }
        }
        float2 top = am[0];
#pragma unroll
        for (int i = 1; i < kJoin; ++i) { top.x = fmaxf(top.x, am[i].x); top.y = fmaxf(top.y, am[i].y); }
        raise(top);
#pragma unroll
        for (int i = 0; i < kJoin; ++i) add(am[i], al[i]);
#pragma unroll
        for (int k = 0; k < kSlices; ++k) {
            top = x[0][k].v;
#pragma unroll
            for (int i = 1; i < kJoin; ++i) { top.x = fmaxf(top.x, x[i][k].v.x); top.y = fmaxf(top.y, x[i][k].v.y); }
            raise_values(r[k], top);
#pragma unroll
            for (int i = 0; i < kJoin; ++i) add_values(r[k], am[i], x[i][k]);
        }
    }
    if (split > 0) {                                       // the shares of the same dimensions
        __shared__ float4 s_o[kSlices][8 / kSlices][32];
        __shared__ float2 s_m[8 / kSlices][32], s_l[8 / kSlices][32], s_v[kSlices][8 / kSlices][32];
        s_m[warp][lane] = m;
        s_l[warp][lane] = l;
#pragma unroll
        for (int k = 0; k < kSlices; ++k) {
            s_o[k][warp][lane] = r[k].o;
            s_v[k][warp][lane] = r[k].v;
        }
        __syncthreads();
        if (share != 0) return;
        const int shares = min(n, step);
        for (int i = 1; i < shares; ++i) {
            const int other = warp + i * slices;
            const float2 am = s_m[other][lane];
            raise(am);
            add(am, s_l[other][lane]);
#pragma unroll
            for (int k = 0; k < kSlices; ++k) {
                const Values a = {s_v[k][other][lane], s_o[k][other][lane]};
                raise_values(r[k], a.v);
                add_values(r[k], am, a);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kSlices; ++k) {
        const float4 o = r[k].o;
        const float2 v = r[k].v;
        __nv_bfloat16* to = p.out + out + h0 * kHeadDim + out_dim<F>(slice0 + k * slices, q);
        if (h0 < p.g) *reinterpret_cast<uint32_t*>(to) = pack_bf16x2(final_value(o.x, m.x, l.x, v.x, true), final_value(o.z, m.x, l.x, v.x, true));
        if (h0 + 1 < p.g)
            *reinterpret_cast<uint32_t*>(to + kHeadDim) = pack_bf16x2(final_value(o.y, m.y, l.y, v.y, true), final_value(o.w, m.y, l.y, v.y, true));
    }
    if (p.lse && slice0 == 0 && q == 0) {
        float* lse = p.lse + (size_t)seq * p.h_q + (size_t)head * p.g + h0;
        if (h0 < p.g) lse[0] = final_lse(m.x, l.x, true);
        if (h0 + 1 < p.g) lse[1] = final_lse(m.y, l.y, true);
    }
}

template <int F, int LIE>
static cudaError_t launch_stream(const PagesAttnLaunch& p, int ctas, int expire, int sms, cudaStream_t s) {
    constexpr int kSmem = (int)sizeof(StreamWarp<F>);
    static_assert(kSmem + 1024 <= 228 * 1024 / stream_warps(F, LIE != kApart), "room for all warps of an SM");
    const auto kernel = gkv_pages_stream_kernel<F, LIE>;
    // a property of the function on the current device; setting it again costs less than finding out whether it is set
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e != cudaSuccess) return e;
    kernel<<<(unsigned)ctas, 32, kSmem, s>>>(p, expire);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const int units = p.batch * p.h_kv;
    // CTAs a unit, and warps that share its parts: few units have many parts
    const MergeShape shape = merge_shape(units, sms);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)units << shape.split);
    cfg.blockDim = dim3(shape.few ? 256 : 128);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, shape.few ? gkv_pages_stream_merge_kernel<F, 8, 1> : gkv_pages_stream_merge_kernel<F, 2, 2>, p, ctas, shape.split);
}
static bool rows_together(const PagesAttnLaunch& p) { return p.pages.token_rows == 1 && p.pages.page_size % kTile == 0; }
int pages_stream_warps_per_sm(const PagesAttnLaunch& p, int format) { return stream_warps(format, rows_together(p)); }
template <int F>
static cudaError_t launch_format(const PagesAttnLaunch& p, int ctas, int expire, int sms, cudaStream_t s) {
    if (!rows_together(p)) return launch_stream<F, kApart>(p, ctas, expire, sms, s);
    if constexpr (stream_tiles(F) > 1)
        if (p.pages.page_size % StreamWarp<F>::kKeys != 0) return launch_stream<F, kTiles>(p, ctas, expire, sms, s);
    return launch_stream<F, kSteps>(p, ctas, expire, sms, s);
}
cudaError_t launch_pages_stream(const PagesAttnLaunch& p, int format, int ctas, int expire, int sms, cudaStream_t s) {
    switch (format) {
        case GKV_STORE_BF16: return launch_format<GKV_STORE_BF16>(p, ctas, expire, sms, s);
        case GKV_STORE_E4M3: return launch_format<GKV_STORE_E4M3>(p, ctas, expire, sms, s);
        case GKV_STORE_INT8: return launch_format<GKV_STORE_INT8>(p, ctas, expire, sms, s);
        default:             return launch_format<GKV_STORE_INT4>(p, ctas, expire, sms, s);
    }
}

}  // namespace gkv
