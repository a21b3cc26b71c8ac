// Decode attention over a cache in pages, for more work than a few clusters: every warp of a grid that fills the device takes an equal
// share of all tiles.
//
// The units (sequence, KV head) lie one after the other, each as many 16-key tiles long as its sequence, and warp w of W takes tiles
// w * per .. (w + 1) * per - 1 of that line, per = ceil(all / W): it may begin and end inside a unit and pass through several. Whatever the lengths are,
// all warps have the same work, none waits for another, and the stream of rows from HBM does not stop at the end of a unit. A unit that one
// warp has to itself is finished by it; of the others (a warp's first or last one) it leaves a partial result, and the merge joins them.
//
// Rows come by bulk copies into a ring of the warp's own, issued by its lanes and completed on a barrier of the warp's own: with pages whose
// size is a multiple of the tile and that hold a head's rows together, one copy for a tile of K and four for V; with any others, one for
// each row. (By cp.async, 16 bytes a lane, a tile costs the warp 100 more instructions: 128 sequences x 8 heads of about 2200 keys in bf16
// 225 us, 2 x 8 of up to 131071 in 4 bits 108.) V is taken in four groups of four rows, 32 bytes further apart than the rows, and row r of
// the first product (lanes' group q = r % 8) is key 4 (q / 2) + q % 2 + 2 (r / 8): lane j then finds its four keys of V in its own group, at
// banks of its own.
//
// Products and softmax are those of the attention over a store (gkv_store_rows.cuh). A row that lies on no page makes its unit NaN.
// A wait that runs out (never, but every wait ends) makes the warp's units NaN, too.
#include "gkv_pages.cuh"
#include "gkv_rotary.cuh"
#include "gkv_store_rows.cuh"

namespace gkv {

__host__ __device__ constexpr int stream_ctas(int format) { return format == GKV_STORE_E4M3 || format == GKV_STORE_INT8 ? 4 : 3; }
int pages_stream_ctas_per_sm(int format) { return stream_ctas(format); }

template <int F>
struct __align__(16) StreamWarp {
    static constexpr int kRow = StoreFormat<F>::kRow;
    static constexpr int kStages = F == GKV_STORE_BF16 ? 2 : F == GKV_STORE_INT4 ? 6 : 3;
    static constexpr int kGroup = 4 * kRow + 32;           // bytes from one group of V rows to the next
    static constexpr int kK = kTile * kRow, kStage = kK + 4 * kGroup;
    uint8_t ring[kStages][kStage];
    __nv_bfloat16 row[kHeadDim];                           // a head, or the new key, as it is turned
    uint8_t code[2][kRow];                                 // the new row as it stands in the cache
    __nv_bfloat16 scale[2][4];
    float v[value_groups(F)][8];
    uint32_t rows[kStages][kTile];                         // numbers of the tiles' rows
    uint64_t full[kStages];
};

// A place in the line of tiles.
struct StreamPlace {
    int seq, head, tile, tiles, len;
};
// On to the next one: there is one, as long as nobody changes the lengths meanwhile; if somebody does, this ends all the same.
__device__ __forceinline__ void stream_next(const PagesAttnLaunch& p, StreamPlace& c) {
    if (++c.tile < c.tiles) return;
    c.tile = 0;
    if (++c.head < p.h_kv) return;
    c.head = 0;
    while (c.seq < p.batch - 1) {
        c.tiles = own_tiles_of(p, ++c.seq);
        if (c.tiles > 0) break;
    }
    c.len = p.len[c.seq];
}
// Tiles of all units, and of those of the sequences before `seq`.
__device__ __forceinline__ int64_t stream_total(const PagesAttnLaunch& p, int seq, int lane, int64_t* before) {
    int64_t all = 0, part = 0;
    for (int b = lane; b < p.batch; b += 32) {
        const int t = own_tiles_of(p, b);
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
__device__ __forceinline__ int64_t stream_share(int64_t all, int warps) {
    const int64_t per = (all + warps - 1) / warps;
    return per < kStreamLeast ? kStreamLeast : per;
}

template <int F, bool TOGETHER>
__global__ void __launch_bounds__(kThreads, stream_ctas(F)) gkv_pages_stream_kernel(const PagesAttnLaunch p) {
    using Warp = StreamWarp<F>;
    constexpr int NG = value_groups(F), S = Warp::kStages, kRow = Warp::kRow, kScales = StoreFormat<F>::kScales;
    constexpr bool kScaled = F != GKV_STORE_BF16;
    extern __shared__ __align__(128) uint8_t s_raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Warp& sw = reinterpret_cast<Warp*>(s_raw)[warp];
    grid_launch_dependents();

    // ---- this warp's tiles
    const int w = blockIdx.x * kWarps + warp;
    int64_t none;
    const int64_t all = stream_total(p, 0, lane, &none), per = stream_share(all, (int)gridDim.x * kWarps), begin = w * per;
    if (begin >= all) return;
    const int steps = (int)(all - begin < per ? all - begin : per);
    StreamPlace fetch;
    {
        int64_t left = begin;                              // tiles between sequence b's first and ours
        bool found = false;
        for (int b = 0; b < p.batch; b += 32) {
            const int t = own_tiles_of(p, b + lane);
            int64_t upto = (int64_t)t * p.h_kv;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t x = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += x;
            }
            const unsigned past = __ballot_sync(0xffffffffu, upto > left);
            if (past) {
                const int at = __ffs(past) - 1;
                fetch.seq = b + at;
                fetch.tiles = __shfl_sync(0xffffffffu, t, at);
                left -= __shfl_sync(0xffffffffu, upto, at) - (int64_t)fetch.tiles * p.h_kv;
                found = true;
                break;
            }
            left -= __shfl_sync(0xffffffffu, upto, 31);
        }
        if (!found) return;                                // (somebody has changed the lengths)
        fetch.head = (int)(left / fetch.tiles);
        fetch.tile = (int)(left - (int64_t)fetch.head * fetch.tiles);
        fetch.len = p.len[fetch.seq];
    }
    StreamPlace at = fetch;
    const int added = p.k_new ? 1 : 0;

    if (lane == 0) {
#pragma unroll
        for (int s = 0; s < S; ++s) mbar_init(smem_u32(&sw.full[s]), 1);
        fence_mbar_init();
    }
    __syncwarp();

    // ---- tiles on their way: the table's entries one tile ahead of the copies. Lane l & 15 has key l & 15.
    const uint8_t *kb = p.pages.data[0], *vb = p.pages.data[1];
    auto entry = [&]() {
        const int key = fetch.tile * kTile + (TOGETHER ? 0 : lane & 15);
        return key < fetch.len + added ? page_entry(p.pages, p.pages.table + fetch.seq * p.pages.table_stride, key) : 0;
    };
    int issued = 0;
    int32_t next = entry();
    auto issue = [&](int stage) {
        const int key0 = fetch.tile * kTile, key = key0 + (lane & 15), here = fetch.len - key0;      // rows in the cache from key0 on
        const uint32_t first = TOGETHER ? page_row(p.pages, next, (uint32_t)fetch.head * p.pages.head_rows, key0) : 0u;
        uint32_t row = kNoRow;
        if (key < fetch.len + added) {
            if (TOGETHER) row = first == kNoPage ? kNoPage : first + (lane & 15);
            else row = page_row(p.pages, next, (uint32_t)fetch.head * p.pages.head_rows, key);
        }
        const bool fine = __all_sync(0xffffffffu, row != kNoPage);
        if (lane < kTile) sw.rows[stage][lane] = row;
        const uint32_t bar = smem_u32(&sw.full[stage]), k = smem_u32(sw.ring[stage]), v = k + Warp::kK;
        const int n = fine ? min(max(here, 0), kTile) : 0;                                           // rows to be copied
        if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)(2 * n * kRow));
        if (TOGETHER) {
            const size_t src = (size_t)first * kRow;
            if (lane < 4) {
                const int rows = min(n - 4 * lane, 4);
                if (rows > 0) bulk_load(v + lane * Warp::kGroup, vb + src + lane * 4 * kRow, (uint32_t)(rows * kRow), bar);
            } else if (lane == 4 && n > 0) {
                bulk_load(k, kb + src, (uint32_t)(n * kRow), bar);
            }
        } else if ((lane & 15) < n) {
            const size_t src = (size_t)row * kRow;
            const int r = lane & 15;
            if (lane < 16) bulk_load(k + r * kRow, kb + src, kRow, bar);
            else bulk_load(v + (r >> 2) * Warp::kGroup + (r & 3) * kRow, vb + src, kRow, bar);
        }
        if (++issued < steps) {
            stream_next(p, fetch);
            next = entry();
        }
    };
#pragma unroll
    for (int s = 0; s < S; ++s)
        if (issued < steps) issue(s);

    const int q = lane >> 2, j = lane & 3, h0 = 2 * j;
    const int key_a = 4 * (q >> 1) + (q & 1);              // this lane's keys of a tile: key_a and two on
    TileK<F> tk;
    TileV<F> tv;
    auto fetch_scales = [&](auto& t, const __nv_bfloat16* scale, int stage) {
        if constexpr (kScaled) {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const uint32_t r = sw.rows[stage][key_a + 2 * hf];
                const __nv_bfloat16* s = scale + (size_t)r * kScales;
                if constexpr (F == GKV_STORE_INT4) t.s[hf] = r < kNoPage ? ld8(s) : make_uint2(0u, 0u);
                else t.s[hf] = r < kNoPage ? ld2(s) : 0u;
            }
        }
    };
    // Two elements of a head's row that are turned together (or, behind the pairs, copied): those of pair number i.
    const bool rotates = p.rotary.turns != nullptr;
    auto first_of = [&](int i) { return i < p.rotary.half && !p.rotary.interleaved ? i : 2 * i; };
    auto second_of = [&](int i) { return i < p.rotary.half && !p.rotary.interleaved ? i + p.rotary.half : 2 * i + 1; };
    auto cos_sin = [&](int i) {
        if (i >= p.rotary.half) return make_float2(1.f, 0.f);
        return rotary_cos_sin(p.rotary.turns[i], p.pos ? p.pos[at.seq] : added ? at.len : at.len - 1, p.rotary.factor, 1.f);
    };
    auto turn_into = [&](int i, __nv_bfloat16 a, __nv_bfloat16 b, float2 cs) {
        const float2 r = rotary_turn(__bfloat162float(a), __bfloat162float(b), cs.x, cs.y);
        const bool turns = i < p.rotary.half;
        sw.row[first_of(i)] = turns ? __float2bfloat16_rn(r.x) : a;
        sw.row[second_of(i)] = turns ? __float2bfloat16_rn(r.y) : b;
    };

    uint32_t qf[8][2];
    float f0 = 0.f, f1 = 0.f;
    RunningRows<F> r;
    bool begins = true, whole = false, ok = true;          // a unit begins; it is ours from its first tile on; no wait has run out
    int stage = 0;
    bool first_unit = true;
    uint32_t parity = 0;
    __syncwarp();
    fetch_scales(tk, p.pages.scale[0], 0);
    fetch_scales(tv, p.pages.scale[1], 0);
    for (int step = 0; step < steps; ++step) {
        if (begins) {
            // ---- a unit's heads
            const __nv_bfloat16* x = p.q + ((int64_t)at.seq * p.q_stride + (int64_t)at.head * p.g * kHeadDim);
            if (rotates) {
                const float2 cs0 = cos_sin(lane), cs1 = cos_sin(lane + 32);
#pragma unroll 1
                for (int h4 = 0; h4 < p.g; h4 += 4) {                  // four heads' loads at a time
                    __nv_bfloat16 e[4][4];
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        if (h4 + h < p.g)
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                e[h][2 * k] = x[(h4 + h) * kHeadDim + first_of(lane + 32 * k)];
                                e[h][2 * k + 1] = x[(h4 + h) * kHeadDim + second_of(lane + 32 * k)];
                            }
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        if (h4 + h < p.g) {
                            turn_into(lane, e[h][0], e[h][1], cs0);
                            turn_into(lane + 32, e[h][2], e[h][3], cs1);
                            __syncwarp();
                            if (min(q, p.g - 1) == h4 + h)
#pragma unroll
                                for (int ks = 0; ks < 8; ++ks) load_query<F>(sw.row, ks, j, qf[ks][0], qf[ks][1]);
                            __syncwarp();
                        }
                }
            } else {
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) load_query<F>(x + min(q, p.g - 1) * kHeadDim, ks, j, qf[ks][0], qf[ks][1]);
            }
            f0 = f1 = p.scale_log2;
            scale_queries<F>(lane, qf, f0, f1);
            r.start(sw.v, lane);
            whole = at.tile == 0;
            begins = false;
        }
        // ---- a tile
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait_bounded(smem_u32(&sw.full[stage]), parity));
        const uint32_t k = smem_u32(sw.ring[stage]), v = k + Warp::kK;
        const int left = at.len + added - at.tile * kTile;                       // keys from this tile's first on
        const bool last = at.tile == at.tiles - 1;
        const bool bad = !ok || __any_sync(0xffffffffu, sw.rows[stage][lane & 15] == kNoPage);
        if (last) {
            // What V has behind the end, whatever it is, becomes zeros.
            for (int i = lane; i < (kTile - left) * (kRow / 16); i += 32) {
                const int key = left + i / (kRow / 16);
                *reinterpret_cast<uint4*>(sw.ring[stage] + Warp::kK + (key >> 2) * Warp::kGroup + (key & 3) * kRow + i % (kRow / 16) * 16) =
                    make_uint4(0u, 0u, 0u, 0u);
            }
            if (added) {
                // The new row, its last key: turned, quantised, into its page and into the tile.
                const int64_t new_row = (int64_t)at.seq * p.kv_stride + (int64_t)at.head * kHeadDim;
                const __nv_bfloat16 *kn = p.k_new + new_row, *vn = p.v_new + new_row;
                if (rotates) {
                    turn_into(lane, kn[first_of(lane)], kn[second_of(lane)], cos_sin(lane));
                    turn_into(lane + 32, kn[first_of(lane + 32)], kn[second_of(lane + 32)], cos_sin(lane + 32));
                    __syncwarp();
                    kn = sw.row;
                }
                const uint4 x = store_load_source<F>(lane < 16 ? kn : vn, lane & 15);
                const int key = left - 1;
                const uint32_t to = sw.rows[stage][key];
                store_put_row<F>(sw.code[lane >> 4], sw.scale[lane >> 4], lane & 15, x);
                if (to < kNoPage)
                    store_put_row<F>(p.pages.data[lane >> 4] + (size_t)to * kRow, p.pages.scale[lane >> 4] + (size_t)to * kScales, lane & 15, x);
                __syncwarp();
                uint8_t* dst = lane < 16 ? sw.ring[stage] + key * kRow : sw.ring[stage] + Warp::kK + (key >> 2) * Warp::kGroup + (key & 3) * kRow;
                if ((lane & 15) < kRow / 16)
                    reinterpret_cast<uint4*>(dst)[lane & 15] = reinterpret_cast<const uint4*>(sw.code[lane >> 4])[lane & 15];
                if constexpr (kScaled) {
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf)
                        if (key_a + 2 * hf == key) {
                            if constexpr (F == GKV_STORE_INT4) {
                                tk.s[hf] = *reinterpret_cast<const uint2*>(sw.scale[0]);
                                tv.s[hf] = *reinterpret_cast<const uint2*>(sw.scale[1]);
                            } else {
                                tk.s[hf] = *reinterpret_cast<const uint16_t*>(sw.scale[0]);
                                tv.s[hf] = *reinterpret_cast<const uint16_t*>(sw.scale[1]);
                            }
                        }
                }
            }
            fence_proxy_async_smem();                      // before the ring's next copies
            __syncwarp();
        }
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int c = 0; c < (F == GKV_STORE_BF16 ? 4 : F == GKV_STORE_INT4 ? 1 : 2); ++c)
                tk.d[hf][c] = lds16(k + (key_a + 2 * hf) * kRow + j * 16 + c * 64);
        float z[4];
        tile_logits<F>(tk, qf, f0, f1, z);
        if (left < kTile) {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
                if (key_a + 2 * hf >= left) z[2 * hf] = z[2 * hf + 1] = -INFINITY;
        }
        if (bad) z[0] = z[1] = z[2] = z[3] = NAN;
        uint32_t b[NG][2];
        r.weigh_tile(z, tv, sw.v, lane, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t a = v + j * Warp::kGroup + i * kRow + q * (F == GKV_STORE_INT4 ? 8 : 16);
            if constexpr (F == GKV_STORE_INT4) tv.d[i] = lds8(a);
            else if constexpr (F == GKV_STORE_BF16) {
                tv.d[i][0] = lds16(a);
                tv.d[i][1] = lds16(a + 128);
            } else tv.d[i] = lds16(a);
        }
        tile_values<F, NG>(tv, b, r.acc);
        __syncwarp();                                      // the slot has been read
        if (issued < steps && ok) issue(stage);
        if (++stage == S) { stage = 0; parity ^= 1; }
        if (step + 1 < steps) {
            __syncwarp();                                  // (S = 1 aside, the next tile's rows have been there for long)
            fetch_scales(tk, p.pages.scale[0], stage);
            fetch_scales(tv, p.pages.scale[1], stage);
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
            begins = true;
            first_unit = false;
            __syncwarp();
        }
        if (step + 1 < steps) stream_next(p, at);
    }
    if (!ok)                                               // what is still on its way gets a bounded time to arrive
        for (int s = 0; s < S; ++s) mbar_wait_bounded(smem_u32(&sw.full[s]), s < stage ? parity ^ 1 : parity);
}

// Joins the partial results of a unit. `apart`: 8 CTAs a unit, each with two dimensions of every lane's, their threads 32 lanes x 8 shares of
// the records; else one CTA a unit, whose warps have two dimensions each.
template <int F>
__global__ void __launch_bounds__(256) gkv_pages_stream_merge_kernel(const PagesAttnLaunch p, const int warps, const int apart) {
    constexpr int NG = value_groups(F);
    __shared__ float s_max[8][1 + NG][8], s_sum[8][8], s_fin[2 + NG][8];
    __shared__ float4 s_o[8][32];
    const int unit = apart ? blockIdx.x >> 3 : blockIdx.x, seq = unit / p.h_kv, head = unit - seq * p.h_kv;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t before;
    const int64_t all = stream_total(p, seq, lane, &before), per = stream_share(all, warps);
    const int len = p.len[seq], tiles = own_tiles_of(p, seq);
    const int64_t first = before + (int64_t)head * tiles;
    const int w0 = (int)(first / per), n = tiles ? (int)((first + tiles - 1) / per) - w0 + 1 : 0;
    const size_t out = ((size_t)seq * p.h_q + (size_t)head * p.g) * kHeadDim;
    const int slice = apart ? blockIdx.x & 7 : warp;       // the two dimensions
    const int q = lane >> 2, h0 = 2 * (lane & 3), d = out_dim<F>(slice, q), dg = slice / (8 / NG);
    grid_wait_previous();                                  // (nobody leaves before: what comes next waits for this kernel alone)
    if (len < 0 || n == 1) return;                         // left out, or finished by the warp that had it
    if (n == 0) {
        const bool fits = p.k_new ? len < p.capacity : len <= p.capacity;
        if (apart && warp != 0) return;
        const uint32_t x = fits ? 0u : 0x7fff7fffu;        // bf16 NaN
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (h0 + h < p.g) *reinterpret_cast<uint32_t*>(p.out + out + (h0 + h) * kHeadDim + d) = x;
        if (p.lse && slice == 0 && lane < p.g) p.lse[(size_t)seq * p.h_q + (size_t)head * p.g + lane] = fits ? -INFINITY : NAN;
        return;
    }
    // Part i is warp w0 + i's: the first of its two, but where the unit begins inside a warp's share its last one.
    const bool inside = first != w0 * per;
    auto record = [&](int i) { return p.own_part + (size_t)(2 * (w0 + i) + (i == 0 && inside ? 1 : 0)) * kStreamRecFloats; };
    // ---- maxima and the sum of weights: thread t has head t & 7 of every 32nd record
    const int h = threadIdx.x & 7;
    float m = -INFINITY, v[NG], l = 0.f;
#pragma unroll
    for (int g = 0; g < NG; ++g) v[g] = -INFINITY;
    for (int i = threadIdx.x >> 3; i < n; i += 32) {
        const float* a = record(i) + h;
        m = fmaxf(m, a[0]);
#pragma unroll
        for (int g = 0; g < NG; ++g) v[g] = fmaxf(v[g], a[16 + 8 * g]);
    }
#pragma unroll
    for (int o = 8; o < 32; o <<= 1) {
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll
        for (int g = 0; g < NG; ++g) v[g] = fmaxf(v[g], __shfl_xor_sync(0xffffffffu, v[g], o));
    }
    if (lane < 8) {
        s_max[warp][0][h] = m;
#pragma unroll
        for (int g = 0; g < NG; ++g) s_max[warp][1 + g][h] = v[g];
    }
    __syncthreads();
    if (threadIdx.x < 8 * (1 + NG)) {
        float a = -INFINITY;
        for (int i = 0; i < 8; ++i) a = fmaxf(a, s_max[i][threadIdx.x >> 3][h]);
        s_fin[threadIdx.x < 8 ? 0 : 1 + (threadIdx.x >> 3)][h] = a;
    }
    __syncthreads();
    const float mr = finite_ref(s_fin[0][h]);
    for (int i = threadIdx.x >> 3; i < n; i += 32) {
        const float* a = record(i) + h;
        l += a[8] * fast_exp2(a[0] - mr);                  // (a NaN sum may come with a maximum of -infinity)
    }
#pragma unroll
    for (int o = 8; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if (lane < 8) s_sum[warp][h] = l;
    __syncthreads();
    if (threadIdx.x < 8) {
        float a = 0.f;
        for (int i = 0; i < 8; ++i) a += s_sum[i][h];
        s_fin[1][h] = a;
    }
    // ---- values
    const float v0 = finite_ref(s_fin[2 + dg][h0]), v1 = finite_ref(s_fin[2 + dg][h0 + 1]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = apart ? warp : 0; i < n; i += apart ? 8 : 1) {
        const float* a = record(i);
        const float4 x = reinterpret_cast<const float4*>(a + kStreamRecHead)[32 * slice + lane];
        const float2 am = *reinterpret_cast<const float2*>(a + h0), av = *reinterpret_cast<const float2*>(a + 16 + 8 * dg + h0);
        const float e0 = am.x == -INFINITY ? 0.f : fast_exp2(av.x - v0), e1 = am.y == -INFINITY ? 0.f : fast_exp2(av.y - v1);
        if (e0 != 0.f) { o.x = fmaf(x.x, e0, o.x); o.z = fmaf(x.z, e0, o.z); }      // (no key: values may be missing)
        if (e1 != 0.f) { o.y = fmaf(x.y, e1, o.y); o.w = fmaf(x.w, e1, o.w); }
    }
    if (apart) s_o[warp][lane] = o;
    __syncthreads();
    if (apart) {
        if (warp != 0) return;
        for (int i = 1; i < 8; ++i) {
            const float4 x = s_o[i][lane];
            o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
        }
    }
    const float m0 = s_fin[0][h0], m1 = s_fin[0][h0 + 1], l0 = s_fin[1][h0], l1 = s_fin[1][h0 + 1];
    const float t0 = s_fin[2 + dg][h0], t1 = s_fin[2 + dg][h0 + 1];
    if (h0 < p.g) *reinterpret_cast<uint32_t*>(p.out + out + h0 * kHeadDim + d) = pack_bf16x2(final_value(o.x, m0, l0, t0, true), final_value(o.z, m0, l0, t0, true));
    if (h0 + 1 < p.g)
        *reinterpret_cast<uint32_t*>(p.out + out + (h0 + 1) * kHeadDim + d) = pack_bf16x2(final_value(o.y, m1, l1, t1, true), final_value(o.w, m1, l1, t1, true));
    if (p.lse && slice == 0 && lane < p.g) p.lse[(size_t)seq * p.h_q + (size_t)head * p.g + lane] = final_lse(s_fin[0][lane], s_fin[1][lane], true);
}

template <int F, bool TOGETHER>
static cudaError_t launch_stream(const PagesAttnLaunch& p, int ctas, cudaStream_t s) {
    constexpr int kSmem = kWarps * (int)sizeof(StreamWarp<F>);
    const auto kernel = gkv_pages_stream_kernel<F, TOGETHER>;
    // a property of the function on the current device; setting it again costs less than finding out whether it is set
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    kernel<<<(unsigned)ctas, kThreads, kSmem, s>>>(p);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const int units = p.batch * p.h_kv, apart = units <= 128;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)units << (apart ? 3 : 0));
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, gkv_pages_stream_merge_kernel<F>, p, ctas * kWarps, apart);
}
cudaError_t launch_pages_stream(const PagesAttnLaunch& p, int format, int ctas, cudaStream_t s) {
    const bool together = p.pages.token_rows == 1 && p.pages.page_size % kTile == 0;
    switch (format) {
        case GKV_STORE_BF16: return together ? launch_stream<GKV_STORE_BF16, true>(p, ctas, s) : launch_stream<GKV_STORE_BF16, false>(p, ctas, s);
        case GKV_STORE_E4M3: return together ? launch_stream<GKV_STORE_E4M3, true>(p, ctas, s) : launch_stream<GKV_STORE_E4M3, false>(p, ctas, s);
        case GKV_STORE_INT8: return together ? launch_stream<GKV_STORE_INT8, true>(p, ctas, s) : launch_stream<GKV_STORE_INT8, false>(p, ctas, s);
        default:             return together ? launch_stream<GKV_STORE_INT4, true>(p, ctas, s) : launch_stream<GKV_STORE_INT4, false>(p, ctas, s);
    }
}

}  // namespace gkv
