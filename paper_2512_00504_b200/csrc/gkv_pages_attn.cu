// Decode attention over a cache in pages: one query token per sequence, rows found through the sequence's table, q and the new key
// rotated on the way. This form is for short calls: a CTA, or a cluster of up to eight, per unit, all in one launch.
//
// The mathematics and the layout of the products are those of the attention over a store (gkv_store_rows.cuh): a unit is (sequence, KV
// head), a tile 16 keys, the tiles of a piece go round the CTA's four warps, and a warp works on its own. What differs is how rows come.
// A row's address is known only when the table has been read, one trip to memory more, and rows need not lie next to one another. So
// tiles come ahead of time through cp.async into shared memory, kStages tiles of a warp in flight, and the table's entries one tile
// before that. Every lane copies exactly the 16-byte (4-bit V: 8-byte) pieces that it will itself hand to the matrix instructions, into slots
// of its own: any page size and any order of the rows is the same to it, no barrier is needed, no bank conflicts arise, and
// registers hold a tile only while it is worked on. (Scales are loaded into registers a tile ahead.)
//
// The new row is not read back from the cache: its tile's lanes take their pieces of it from shared memory, where the warp that writes
// it to its page leaves a copy. Rotating q and k and quantising them thereby run while the first tiles are on their way.
//
// A piece is an equal share of the tiles that the sequence really has, not of the longest one's: 32 x 4 heads of up to 1151 keys in 8 bits take
// 15.3 us instead of 16.1. The table's entries are guessed for the longest, which is right for calls of equal lengths, and read again otherwise. (So
// places that the sequence has no rows for are read, within the table's width, and left unused.)
//
// Measured: 1 sequence x 4 heads of 639 keys in bf16 7.8 us, whose bytes take 0.2; 32 x 4 heads of up to 1151 keys in 8 bits 15.3 us (3.3). What
// bounds it is a chain of trips to memory (length, table, rows, cluster) of about a microsecond each, rotation and quantising between them.
//
// A place in the table that holds no page stands for rows of NaN, which every join carries into the unit's result.
#include "gkv_pages.cuh"
#include "gkv_rotary.cuh"
#include "gkv_store_rows.cuh"

namespace gkv {

__host__ __device__ constexpr int pages_ctas(int format) { return format == GKV_STORE_BF16 ? 3 : 4; }
int pages_attn_ctas_per_sm(int format) { return pages_ctas(format); }

// A warp's ring: kStages tiles, K pieces [row half][piece][lane][16 bytes], then V pieces [key][piece][lane].
template <int F>
struct PageRing {
    static constexpr int kStages = 2;     // (three or four leave fewer CTAs an SM, and calls are short: no case got faster)
    static constexpr int kPieces = F == GKV_STORE_BF16 ? 4 : F == GKV_STORE_INT4 ? 1 : 2;     // 16-byte pieces of a K row a lane has
    static constexpr int kHalf = kTile * StoreFormat<F>::kRow;                                // bytes of a tile's K or V rows
    static constexpr int kWarp = kStages * 2 * kHalf;
    static constexpr int kCta = kWarps * kWarp;
};

__device__ __forceinline__ void cp_async_8(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void sts16(uint32_t a, uint4 v) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void sts8(uint32_t a, uint2 v) {
    asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(a), "r"(v.x), "r"(v.y) : "memory");
}
constexpr uint32_t kNanPair = 0x7fc07fc0u;    // bf16 NaNs

// The rows of a tile (lane l & 15 has key l & 15's number) into the ring. Rows that do not exist become zeros, those on no page NaN (bf16
// K here, the others by their scales).
template <int F>
__device__ __forceinline__ void fetch_k(uint32_t slot, const uint8_t* kb, uint32_t rows, int lane) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
        const uint32_t r = __shfl_sync(0xffffffffu, rows, (lane >> 2) + 8 * hf);
        const uint8_t* src = kb + (size_t)r * StoreFormat<F>::kRow + (lane & 3) * 16;
        const uint32_t dst = slot + hf * PageRing<F>::kPieces * 512 + lane * 16;
        const uint32_t w = F == GKV_STORE_BF16 && r == kNoPage ? kNanPair : 0u;
#pragma unroll
        for (int c = 0; c < PageRing<F>::kPieces; ++c) {
            if (r < kNoPage) cp_async_16(dst + c * 512, src + c * 64);
            else sts16(dst + c * 512, make_uint4(w, w, w, w));
        }
    }
}
template <int F>
__device__ __forceinline__ void fetch_v(uint32_t slot, const uint8_t* vb, uint32_t rows, int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t r = __shfl_sync(0xffffffffu, rows, 2 * (lane & 3) + (i & 1) + 8 * (i >> 1));
        const uint8_t* src = vb + (size_t)r * StoreFormat<F>::kRow + (lane >> 2) * (F == GKV_STORE_INT4 ? 8 : 16);
        if (F == GKV_STORE_INT4) {
            const uint32_t dst = slot + i * 256 + lane * 8;
            if (r < kNoPage) cp_async_8(dst, src);
            else sts8(dst, make_uint2(0u, 0u));
        } else {
#pragma unroll
            for (int c = 0; c < (F == GKV_STORE_BF16 ? 2 : 1); ++c) {
                const uint32_t dst = slot + (i * (F == GKV_STORE_BF16 ? 2 : 1) + c) * 512 + lane * 16;
                if (r < kNoPage) cp_async_16(dst, src + c * 128);
                else sts16(dst, make_uint4(0u, 0u, 0u, 0u));
            }
        }
    }
}
// Scales of the tile's keys lane / 4 and 8 on.
template <int F, class T>
__device__ __forceinline__ void fetch_scales(T& t, const __nv_bfloat16* scale, uint32_t rows, int lane) {
    if constexpr (F != GKV_STORE_BF16) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const uint32_t r = __shfl_sync(0xffffffffu, rows, (lane >> 2) + 8 * hf);
            const __nv_bfloat16* s = scale + (size_t)r * StoreFormat<F>::kScales;
            const uint32_t other = r == kNoPage ? kNanPair : 0u;
            if constexpr (F == GKV_STORE_INT4) t.s[hf] = r < kNoPage ? ld8(s) : make_uint2(other, other);
            else t.s[hf] = r < kNoPage ? ld2(s) : other & 0xffffu;
        }
    }
}
template <int F>
__device__ __forceinline__ void take_k(TileK<F>& t, uint32_t slot, int lane) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int c = 0; c < PageRing<F>::kPieces; ++c) t.d[hf][c] = lds16(slot + (hf * PageRing<F>::kPieces + c) * 512 + lane * 16);
}
template <int F>
__device__ __forceinline__ void take_v(TileV<F>& t, uint32_t slot, int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (F == GKV_STORE_INT4) t.d[i] = lds8(slot + i * 256 + lane * 8);
        else if constexpr (F == GKV_STORE_BF16) {
            t.d[i][0] = lds16(slot + 2 * i * 512 + lane * 16);
            t.d[i][1] = lds16(slot + (2 * i + 1) * 512 + lane * 16);
        } else t.d[i] = lds16(slot + i * 512 + lane * 16);
    }
}

// The new row as it stands in the cache: codes of K and V, and their scales.
template <int F>
struct __align__(16) NewRow {
    uint8_t code[2][StoreFormat<F>::kRow];
    __nv_bfloat16 scale[2][4];
};
// The pieces of it that this lane has of a tile, of which it is key `at`.
template <int F>
__device__ __forceinline__ void patch_k(TileK<F>& t, const NewRow<F>& n, int at, bool page, int lane) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
        if ((lane >> 2) + 8 * hf != at) continue;
#pragma unroll
        for (int c = 0; c < PageRing<F>::kPieces; ++c) {
            t.d[hf][c] = *reinterpret_cast<const uint4*>(n.code[0] + (lane & 3) * 16 + c * 64);
            if (F == GKV_STORE_BF16 && !page) t.d[hf][c] = make_uint4(kNanPair, kNanPair, kNanPair, kNanPair);
        }
        if constexpr (F == GKV_STORE_INT4) t.s[hf] = page ? *reinterpret_cast<const uint2*>(n.scale[0]) : make_uint2(kNanPair, kNanPair);
        else if constexpr (F != GKV_STORE_BF16) t.s[hf] = page ? *reinterpret_cast<const uint16_t*>(n.scale[0]) : kNanPair & 0xffffu;
    }
}
template <int F>
__device__ __forceinline__ void patch_v_scales(TileV<F>& t, const NewRow<F>& n, int at, int lane) {
    if constexpr (F != GKV_STORE_BF16) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            if ((lane >> 2) + 8 * hf != at) continue;
            if constexpr (F == GKV_STORE_INT4) t.s[hf] = *reinterpret_cast<const uint2*>(n.scale[1]);
            else t.s[hf] = *reinterpret_cast<const uint16_t*>(n.scale[1]);
        }
    }
}
template <int F>
__device__ __forceinline__ void patch_v(TileV<F>& t, const NewRow<F>& n, int at, int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (2 * (lane & 3) + (i & 1) + 8 * (i >> 1) != at) continue;
        const uint8_t* src = n.code[1] + (lane >> 2) * (F == GKV_STORE_INT4 ? 8 : 16);
        if constexpr (F == GKV_STORE_INT4) t.d[i] = *reinterpret_cast<const uint2*>(src);
        else if constexpr (F == GKV_STORE_BF16) {
            t.d[i][0] = *reinterpret_cast<const uint4*>(src);
            t.d[i][1] = *reinterpret_cast<const uint4*>(src + 128);
        } else t.d[i] = *reinterpret_cast<const uint4*>(src);
    }
}

// Grid: units x splits, split fastest.
template <int F, int MODE>
__global__ void __launch_bounds__(kThreads, pages_ctas(F)) gkv_pages_attn_kernel(const PagesAttnLaunch p) {
    using Ring = PageRing<F>;
    constexpr int NG = value_groups(F), S = Ring::kStages;
    __shared__ RowsShared<F> sh;
    __shared__ __align__(16) __nv_bfloat16 s_q[kMaxGroup + 1][kHeadDim];      // rotated: the heads, and the new key
    __shared__ NewRow<F> s_new;
    extern __shared__ __align__(128) uint8_t s_ring[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int unit = blockIdx.x / p.splits, split = blockIdx.x - unit * p.splits, splits = p.splits, split_tiles = p.split_tiles;
    const int seq = unit / p.h_kv, head = unit - seq * p.h_kv;
    // ---- everything that can be loaded before the length is known: the heads (those of this warp), the new row, and what the table has for the
    // first tiles, were they all there
    const bool append = p.k_new != nullptr;
    const HeadTurn turn(p.rotary, lane);
    const __nv_bfloat16* q = p.q + ((int64_t)seq * p.q_stride + (int64_t)head * p.g * kHeadDim);
    const __nv_bfloat16* k_new = append ? p.k_new + ((int64_t)seq * p.kv_stride + (int64_t)head * kHeadDim) : q;
    const __nv_bfloat16* v_new = append ? p.v_new + ((int64_t)seq * p.kv_stride + (int64_t)head * kHeadDim) : q;
    HeadTurn::Words heads[2], key_words;
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (warp + k * kWarps < p.g) heads[k] = turn.load(q + (warp + k * kWarps) * kHeadDim);
    key_words = turn.load(k_new);
    const uint4 value = store_load_source<F>(v_new, lane & 15);
    const int32_t given = p.pos ? p.pos[seq] : 0;
    const int32_t* table = p.pages.table + seq * p.pages.table_stride;
    constexpr int kStep = kWarps * kTile;
    const int guess0 = (split * split_tiles + warp) * kTile + (lane & 15);
    int32_t e[S + 1];
#pragma unroll
    for (int s = 0; s <= S; ++s) e[s] = guess0 + s * kStep < p.capacity ? page_entry(p.pages, table, guess0 + s * kStep) : 0;

    const int len = p.len[seq];
    if (len < 0) return;
    const bool fits = append ? len < p.capacity : len <= p.capacity;
    const int old = fits ? len : 0, n = old + (fits && append ? 1 : 0);      // rows in the pages, rows to attend to
    const int tiles = (n + kTile - 1) / kTile;
    const int cut = (tiles + splits - 1) / splits;       // pieces go by the length that the sequence has
    const int t_begin = min(split * cut, tiles), t_end = min(t_begin + cut, tiles);
    const int own_tiles = t_end - t_begin;               // tile i of the piece is warp i % kWarps'
    const bool writes = append && fits && own_tiles > 0 && t_end == tiles;

    // ---- the first tiles set out. Tile s of this warp begins with key `key0` + s * kWarps * kTile.
    const uint32_t head0 = (uint32_t)head * p.pages.head_rows;
    const int key0 = (t_begin + warp) * kTile;
    const int mine = own_tiles > warp ? (own_tiles - warp + kWarps - 1) / kWarps : 0;
    const int last_old = min(old, t_end * kTile);        // (a piece's tiles are whole but for the unit's last)
    auto entry = [&](int s) {
        const int key = key0 + s * kStep + (lane & 15);
        return key < last_old ? page_entry(p.pages, table, key) : 0;
    };
    if (cut != split_tiles)                              // (the guess went by the longest length)
#pragma unroll
        for (int s = 0; s <= S; ++s) e[s] = entry(s);
    auto row_of = [&](int32_t e, int s) {
        const int key = key0 + s * kStep + (lane & 15);
        return key < last_old ? page_row(p.pages, e, head0, key) : kNoRow;
    };
    const uint8_t *kb = p.pages.data[0], *vb = p.pages.data[1];
    const __nv_bfloat16 *ksb = p.pages.scale[0], *vsb = p.pages.scale[1];
    const uint32_t ring = smem_u32(s_ring) + warp * Ring::kWarp;
    uint32_t rows[S];                                    // of tiles s + 1 .. s + S
    TileK<F> tk;
    TileV<F> tv;
    {
        uint32_t r = row_of(e[0], 0);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (s < mine) fetch_k<F>(ring + s * 2 * Ring::kHalf, kb, r, lane);
            cp_async_commit();
            if (s < mine) fetch_v<F>(ring + s * 2 * Ring::kHalf + Ring::kHalf, vb, r, lane);
            cp_async_commit();
            if (s == 0) {
                fetch_scales<F>(tk, ksb, r, lane);
                fetch_scales<F>(tv, vsb, r, lane);
            }
            r = rows[s] = row_of(e[s + 1], s + 1);
        }
    }
    int32_t next = entry(S + 1);

    // ---- q and the new row
    const int hq = lane >> 2;
    const HeadTurn::Angles angles = turn.angles(p.pos ? given : append ? len : len - 1);
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (warp + k * kWarps < p.g) turn.put(s_q[warp + k * kWarps], heads[k], angles);
    const int new_step = writes && warp == (own_tiles - 1) % kWarps ? mine - 1 : -1;     // the tile that has the new row
    if (new_step >= 0) turn.put(s_q[kMaxGroup], key_words, angles);
    __syncthreads();
    uint32_t qf[8][2];
    float f0 = p.scale_log2, f1 = p.scale_log2;
    load_queries<F>(s_q[min(hq, p.g - 1)], lane, qf, f0, f1);
    bool new_page = true;
    if (new_step >= 0) {
        const uint32_t r = page_row(p.pages, page_entry(p.pages, table, len), head0, len);
        new_page = r < kNoPage;
        const uint4 x = lane < 16 ? store_load_source<F>(s_q[kMaxGroup], lane) : value;
        store_put_row<F>(s_new.code[lane >> 4], s_new.scale[lane >> 4], lane & 15, x);
        if (new_page)
            store_put_row<F>(p.pages.data[lane >> 4] + (size_t)r * StoreFormat<F>::kRow,
                             p.pages.scale[lane >> 4] + (size_t)r * StoreFormat<F>::kScales, lane & 15, x);
        __syncwarp();
    }

    RunningRows<F> r;
    r.start(sh.v[warp], lane);
    int left = last_old + (writes ? 1 : 0) - key0;       // keys from this tile's first on
    uint32_t slot = ring;
    for (int s = 0; s < mine; ++s) {
        cp_async_wait_group<2 * S - 1>();
        take_k<F>(tk, slot, lane);
        if (s == new_step) {
            patch_k<F>(tk, s_new, len - key0 - s * kStep, new_page, lane);
            patch_v_scales<F>(tv, s_new, len - key0 - s * kStep, lane);
        }
        float z[4];
        tile_logits<F>(tk, qf, f0, f1, z);
        fetch_scales<F>(tk, ksb, rows[0], lane);
        if (s + S < mine) fetch_k<F>(slot, kb, rows[S - 1], lane);
        cp_async_commit();
        if (left < kTile) {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
                if (hq + 8 * hf >= left) z[2 * hf] = z[2 * hf + 1] = -INFINITY;
        }
        uint32_t b[NG][2];
        r.weigh_tile(z, tv, sh.v[warp], lane, b);
        cp_async_wait_group<2 * S - 1>();
        take_v<F>(tv, slot + Ring::kHalf, lane);
        if (s == new_step) patch_v<F>(tv, s_new, len - key0 - s * kStep, lane);
        tile_values<F, NG>(tv, b, r.acc);
        fetch_scales<F>(tv, vsb, rows[0], lane);
        if (s + S < mine) fetch_v<F>(slot + Ring::kHalf, vb, rows[S - 1], lane);
        cp_async_commit();
#pragma unroll
        for (int k = 0; k + 1 < S; ++k) rows[k] = rows[k + 1];
        rows[S - 1] = row_of(next, s + 1 + S);
        next = entry(s + 2 + S);
        left -= kStep;
        slot = slot + 2 * Ring::kHalf == ring + Ring::kWarp ? ring : slot + 2 * Ring::kHalf;
    }
    // the accumulators go where the rings were
    cp_async_wait_all();
    __syncthreads();
    static_assert(Ring::kCta >= (int)(kWarps * kHeadDim * 8 * sizeof(float)), "room for the accumulators");
    finish_rows<F, MODE>(p, r, sh, reinterpret_cast<float(*)[kHeadDim * 8]>(s_ring), seq, head, split, fits, warp, lane);
}

template <int F, int MODE>
static cudaError_t launch_mode(const PagesAttnLaunch& p, int cluster, cudaStream_t s) {
    const auto kernel = gkv_pages_attn_kernel<F, MODE>;
    // a property of the function on the current device; setting it again costs less than finding out whether it is set
    cudaError_t e = cudaSuccess;
    if (PageRing<F>::kCta > 32 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PageRing<F>::kCta);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.batch * p.h_kv * p.splits));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = PageRing<F>::kCta;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}
template <int F>
static cudaError_t launch_format(const PagesAttnLaunch& p, cudaStream_t s) {
    return p.splits > 1 ? launch_mode<F, kCluster>(p, p.splits, s) : launch_mode<F, kWhole>(p, 1, s);
}
cudaError_t launch_pages_attn(const PagesAttnLaunch& p, int format, cudaStream_t s) {
    switch (format) {
        case GKV_STORE_BF16: return launch_format<GKV_STORE_BF16>(p, s);
        case GKV_STORE_E4M3: return launch_format<GKV_STORE_E4M3>(p, s);
        case GKV_STORE_INT8: return launch_format<GKV_STORE_INT8>(p, s);
        default:             return launch_format<GKV_STORE_INT4>(p, s);
    }
}

}  // namespace gkv
