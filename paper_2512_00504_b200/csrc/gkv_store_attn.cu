// Decode attention over a key/value store (one query token per sequence), and the merge of partial results.
//
// A unit is (sequence, KV head). Its rows are cut into pieces (one CTA each, when there are too few units to fill the device)
// of 16-key tiles, and the tiles of a piece go round the CTA's four warps. A warp works on its own: it loads a tile's codes
// straight into the registers of the matrix instructions' operands -- no shared memory, no barrier -- and keeps its own running
// softmax. Both products are mma.sync m16n8k16 with the keys (then the head dimensions) on M and the g <= 8 query heads on N,
// as in the bf16 decode kernel: 4 to 8 operations a byte, far from where tensor memory would pay. What makes loads without a
// transpose possible is that the order in which a product runs over its inner index is free: the lane that owns a quarter of a
// key's row takes whole 16-byte pieces of it and pairs them with the same elements of q, and on the way out lane group q owns
// the head dimensions of the pieces it read of V. The order of the nibbles of a 4-bit row is chosen for this.
//
// 8- and 4-bit codes become fp16 exactly (their scales stay outside the products), q becomes fp16 after division by a power
// of two (an element is exact down to 2^-17 of its row's largest; below, the error is at most 2^-25 of the largest), weights
// are rounded to fp16 (11 bits: outputs are off by 1.68e-3 instead of the 1.65e-3 that the output's own rounding to bf16 makes;
// it is what the product takes, and codes times fp16 weights are exact in its sums). The scale of a K row multiplies its logit.
// The scale s of a V row goes into the weight: w = p s c with p = exp2(z - m) as it enters the sum of the softmax, and
// c = exp2(m - v) with a running maximum v over z + log2 s, so that the largest of the weights handed to the product lie high in
// fp16's range whatever the scales are (those 2^-20 below lose bits, and 2^-31 below they are 0). A 4-bit row has a scale for
// each 32 head dimensions, and every group of dimensions has its own v and c: groups of very different size do not share a range.
// (v is kept at least at m - 112: c stays finite, and where all of a group's V is below 2^-112 its outputs are numbers of that
// size.) Sums and accumulators are fp32.
//
// The running maxima are allowed to lag: a step raises them (which costs a reduction over the warp and a rescaling of the
// accumulators) only when its weights have grown large.
//
// The pieces of a unit are joined by the CTAs of a cluster reading one another's shared memory (up to 8 pieces, no prefix), or
// leave partial results in the workspace for the merge kernel. Long rows are dealt out by the lengths that the sequences have, so
// that one long sequence among short ones gets the places that they do not need.
//
// Bound by HBM for 8-bit rows in a large batch (128 sequences x 8 heads of about 2200 keys, 585 MB: 97 us, 6.0 TB/s). 4-bit rows
// bring twice the elements per byte to unpack: 2 x 8 heads of about 120000 keys, 274 MB in 73 us, 3.7 TB/s (before fp32 operations went in pairs 77), with the schedulers
// issuing 6 cycles out of 10, the logic and fp32 pipes 4 to 5 (without the products and what feeds them the same loads take 55
// us; with one reference for all groups of a head, which is not precise enough, 75.7). bf16 rows: 128 sequences x 8 heads of 2200
// keys, 1153 MB in 197 us, 5.9 TB/s. A single sequence of 640 keys takes 6.4 us: the launch, four trips to memory (length, q, rows,
// the others' results) one after the other, 3 tiles per warp.
#include "gkv_store_rows.cuh"

namespace gkv {

constexpr int kMergeHops = 4;

// Resident CTAs per SM. 8- and 4-bit rows: 128 registers, 16 warps (128 sequences x 8 heads of about 2200 keys in 8 bits: 97 us;
// two tiles per step, 168 registers and 12 warps: 110 us. 2 x 8 heads of up to 131071 keys in 4 bits, with one reference a head: 76
// us; 12 warps: 78, with two tiles per step 85). bf16 rows need twice the registers for a tile.
__host__ __device__ constexpr int store_ctas(int format) { return format == GKV_STORE_BF16 ? 3 : 4; }
int store_attn_ctas_per_sm(int format) { return store_ctas(format); }

// Own rows of the units. Grid: units x splits, split fastest; dealt out: a head's places, head slowest.
template <int F, int MODE>
__global__ void __launch_bounds__(kThreads, store_ctas(F)) gkv_store_attn_kernel(const StoreAttnLaunch p) {
    constexpr int NG = value_groups(F);
    __shared__ RowsShared<F> sh;
    __shared__ __align__(16) float s_o[kWarps][kHeadDim * 8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int unit = blockIdx.x / p.splits, split = blockIdx.x - unit * p.splits, splits = p.splits, split_tiles = p.split_tiles;
    int seq = unit / p.h_kv, head = unit - seq * p.h_kv;
    if (MODE == kPart || MODE == kDealt) grid_launch_dependents();
    if (MODE == kDealt) {
        if (!dealt_place(p, lane, &seq, &head, &split, &splits, &split_tiles)) return;   // a place that nobody needs
        unit = seq * p.h_kv + head;
    }
    const int len = p.len[seq];
    const bool append = p.k_new != nullptr;
    uint4 new_row = make_uint4(0u, 0u, 0u, 0u);           // on its way while the length is (lanes 0-15: K, 16-31: V)
    if (append) new_row = store_load_source<F>((lane < 16 ? p.k_new : p.v_new) + (size_t)unit * kHeadDim, lane & 15);
    const bool fits = append ? len < p.capacity : len <= p.capacity;
    // The merge goes by this word and not by the length, which it may count up itself.
    if (MODE == kPart && split == 0 && threadIdx.x == 0)
        p.own_part[(size_t)blockIdx.x * kOwnRecFloats + kOwnRecState] = len < 0 ? kPieceLeftOut : fits ? kPieceOk : kPieceNoFit;
    if (len < 0) {
        if (MODE == kPart && p.prefix_part && blockIdx.x == 0) grid_wait_previous();   // see the end of the partial form
        return;
    }
    const int n = fits ? len + (append ? 1 : 0) : 0;
    const int tiles = (n + kTile - 1) / kTile;
    const int t_begin = min(split * split_tiles, tiles);
    const int t_end = split == splits - 1 ? tiles : min(t_begin + split_tiles, tiles);

    uint8_t* kb = p.k + (size_t)unit * p.capacity * StoreFormat<F>::kRow;
    uint8_t* vb = p.v + (size_t)unit * p.capacity * StoreFormat<F>::kRow;
    __nv_bfloat16* ksb = p.k_scale + (size_t)unit * p.capacity * StoreFormat<F>::kScales;
    __nv_bfloat16* vsb = p.v_scale + (size_t)unit * p.capacity * StoreFormat<F>::kScales;

    // The warp that comes to the new row's tile puts the row into the store, before it loads anything of that tile (its own
    // writes are ordered before its later reads; no other warp reads the row).
    const int own_tiles = t_end - t_begin;               // tile i of the piece is warp i % kWarps'
    if (append && fits && own_tiles > 0 && t_end == tiles && warp == (own_tiles - 1) % kWarps) {
        store_put_row<F>((lane < 16 ? kb : vb) + (size_t)len * StoreFormat<F>::kRow,
                         (lane < 16 ? ksb : vsb) + (size_t)len * StoreFormat<F>::kScales, lane & 15, new_row);
        __threadfence_block();
        __syncwarp();
    }

    // q as the B operand: lane (head lane / 4, j = lane & 3)
    const int hq = lane >> 2;
    uint32_t qf[8][2];
    float f0 = p.scale_log2, f1 = p.scale_log2;
    {
        const __nv_bfloat16* qrow = p.q + ((size_t)seq * p.h_q + (size_t)head * p.g + min(hq, p.g - 1)) * kHeadDim;
        load_queries<F>(qrow, lane, qf, f0, f1);
    }

    RunningRows<F> r;
    r.start(sh.v[warp], lane);

    TileK<F> tk;
    TileV<F> tv;
    const int end = min(t_end * kTile, n);
    const int key0 = (t_begin + warp) * kTile;
    int left = warp < own_tiles ? end - key0 : 0;        // keys from this tile's first on
    TilePtrs<F> at;
    at.kb = kb; at.vb = vb;
    at.ksb = reinterpret_cast<const uint8_t*>(ksb); at.vsb = reinterpret_cast<const uint8_t*>(vsb);
    at.set(key0, lane);
    load_tile_k<F>(tk, at, left, lane);
    load_tile_v<F>(tv, at, left, lane);
    while (left > 0) {
        at.advance(kWarps * kTile);
        const int left_next = left - kWarps * kTile;
        float z[4];
        tile_logits<F>(tk, qf, f0, f1, z);
        load_tile_k<F>(tk, at, left_next, lane);
        if (left < kTile) {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
                if (hq + 8 * hf >= left) z[2 * hf] = z[2 * hf + 1] = -INFINITY;
        }
        uint32_t b[NG][2];
        r.weigh_tile(z, tv, sh.v[warp], lane, b);
        tile_values<F, NG>(tv, b, r.acc);
        load_tile_v<F>(tv, at, left_next, lane);
        left = left_next;
    }

    finish_rows<F, MODE>(p, r, sh, s_o, seq, head, split, fits, warp, lane);
}

// Joins the partial results of a unit: those of its own pieces and, with a prefix, those of the prefix items that hold its
// query rows. 2^ds CTAs per unit, each with a share of the dimensions; thread t holds head t & 7 of four dimensions over every
// (slices)th of the parts, so that 8 lanes read 128 contiguous bytes of a record. The statistics of all parts are loaded at once,
// the values of 8 parts at a time: the kernel is a few trips to L2. NG groups of dimensions have maxima v of their own.
template <bool DEALT, int NG>
__global__ void __launch_bounds__(1024) gkv_store_merge_kernel(const StoreAttnLaunch p, const int ds) {
    // factors: own parts [part][group][8], then those of the prefix (with several groups: their maxima, a factor is worked out
    // where it is used) [part][8]
    extern __shared__ float s_part[];
    __shared__ __align__(16) float s_red[4 * 1024];
    __shared__ float s_fin[2 + NG][8];
    const int unit = blockIdx.x >> ds, share = blockIdx.x & ((1 << ds) - 1), seq = unit / p.h_kv, head = unit - seq * p.h_kv;
    const int t = threadIdx.x, slices = blockDim.x >> (8 - ds), slice = t >> (8 - ds), h = t & 7;
    const int d4 = ((t >> 3) & ((32 >> ds) - 1)) + share * (32 >> ds);
    const int hc = min(h, p.g - 1), warps = blockDim.x >> 5;

    // records: own ones, then those of the prefix items (two results each where the item's streams share the rows)
    int items = 0;
    int row0 = 0;
    size_t step = 0;
    const float *own = p.own_part + (size_t)unit * p.splits * kOwnRecFloats, *pre_rec = nullptr;
    int n_own = p.splits;
    if (DEALT) {
        const int t0 = own_tiles_of(p, t & 31), per = store_piece_tiles(p, t & 31, t0);
        own = p.own_part + ((size_t)head * p.batch * p.splits + pieces_before(p, seq, per, t & 31, t0)) * kOwnRecFloats;
        n_own = pieces_of(own_tiles_of(p, seq), per);
    }
    if (p.prefix_part) {
        const int pre = seq / p.seqs_per_prefix, sl = seq - pre * p.seqs_per_prefix, blk = sl / p.seqs_per_block;
        int base = head * p.n_blocks + blk;
        for (int i = 0; i < pre; ++i) base += ((p.prefix_len[i] + 127) / 128 + p.chunk - 1) / p.chunk * p.h_kv * p.n_blocks;
        items = ((p.prefix_len[pre] + 127) / 128 + p.chunk - 1) / p.chunk;
        step = (size_t)p.h_kv * p.n_blocks * kPrefixRecFloats;
        pre_rec = p.prefix_part + (size_t)base * kPrefixRecFloats;
        row0 = (sl - blk * p.seqs_per_block) * p.g;
    }
    const int twice = p.two_tiles ? 0 : 1, parts = n_own + (items << twice);
    // statistics and values of prefix part j at the unit's first row
    auto pre_stats = [&](int j) { return pre_rec + (size_t)(j >> twice) * step + row0 + (j & twice) * 128; };
    auto pre_values = [&](int j) {
        return reinterpret_cast<const float4*>(pre_rec + (size_t)(j >> twice) * step + 2 * kPrefixRows) + row0 + (j & twice) * 128;
    };
    grid_wait_previous();
    bool fits;
    if (DEALT) {                                     // (a sequence without keys has no piece)
        const int len = p.len[seq];
        if (len < 0) return;
        fits = p.k_new ? len < p.capacity : len <= p.capacity;
    } else {
        const float state = own[kOwnRecState];
        if (state == kPieceLeftOut) return;
        fits = state == kPieceOk;
    }

    // ---- statistics: factors of all parts. Thread t has head t & 7 of parts t / 8, t / 8 + blockDim / 8, ...
    const int hops = (parts * 8 + (int)blockDim.x - 1) / (int)blockDim.x;
    float m = -INFINITY, v[NG], l = 0.f, x[kMergeHops], y[kMergeHops][NG], z[kMergeHops];
#pragma unroll
    for (int g = 0; g < NG; ++g) v[g] = -INFINITY;
#pragma unroll
    for (int k = 0; k < kMergeHops; ++k) {
        x[k] = -INFINITY;
        z[k] = 0.f;
#pragma unroll
        for (int g = 0; g < NG; ++g) y[k][g] = -INFINITY;
        const int part = (t + k * (int)blockDim.x) >> 3;
        if (k < hops && part < parts) {
            if (part < n_own) {
                const float* r = own + (size_t)part * kOwnRecFloats + hc;
                x[k] = r[0]; z[k] = r[8];
#pragma unroll
                for (int g = 0; g < NG; ++g) y[k][g] = r[16 + 8 * g];
            } else {
                const float* r = pre_stats(part - n_own) + hc;
                x[k] = r[0]; z[k] = r[kPrefixRows];
#pragma unroll
                for (int g = 0; g < NG; ++g) y[k][g] = x[k];
            }
        }
        m = fmaxf(m, x[k]);
#pragma unroll
        for (int g = 0; g < NG; ++g) v[g] = fmaxf(v[g], y[k][g]);
    }
    constexpr int kStats = 8 * (1 + NG);             // a warp's maxima
#pragma unroll
    for (int o = 8; o < 32; o <<= 1) {
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll
        for (int g = 0; g < NG; ++g) v[g] = fmaxf(v[g], __shfl_xor_sync(0xffffffffu, v[g], o));
    }
    if ((t & 31) < 8) {
        s_red[(t >> 5) * kStats + h] = m;
#pragma unroll
        for (int g = 0; g < NG; ++g) s_red[(t >> 5) * kStats + 8 + 8 * g + h] = v[g];
    }
    __syncthreads();
    if constexpr (NG == 1) {
        for (int i = 0; i < warps; ++i) { m = fmaxf(m, s_red[i * kStats + h]); v[0] = fmaxf(v[0], s_red[i * kStats + 8 + h]); }
    } else {                                         // one thread a number
        if (t < kStats) {
            float a = -INFINITY;
            for (int i = 0; i < warps; ++i) a = fmaxf(a, s_red[i * kStats + t]);
            s_fin[t < 8 ? 0 : 1 + (t >> 3)][h] = a;
        }
        __syncthreads();
        m = s_fin[0][h];
#pragma unroll
        for (int g = 0; g < NG; ++g) v[g] = s_fin[2 + g][h];
    }
    const float mr = finite_ref(m);
    constexpr int kSums = 2048;                      // (the maxima take up to 32 kStats)
    static_assert(32 * kStats <= kSums && kSums + 32 * 8 <= 4 * 1024, "scratch");
#pragma unroll
    for (int k = 0; k < kMergeHops; ++k) {
        const int i = t + k * (int)blockDim.x, part = i >> 3;
        l += z[k] * fast_exp2(x[k] - mr);            // (a NaN sum comes with a maximum of -infinity)
        if (k < hops && part < parts) {              // 0: no key, values may be missing
            if (NG == 1 || part < n_own) {
#pragma unroll
                for (int g = 0; g < NG; ++g) s_part[(part * NG + g) * 8 + h] = x[k] == -INFINITY ? 0.f : fast_exp2(y[k][g] - finite_ref(v[g]));
            } else {
                s_part[(n_own * (NG - 1) + part) * 8 + h] = x[k];
            }
        }
    }
#pragma unroll
    for (int o = 8; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if ((t & 31) < 8) s_red[kSums + (t >> 5) * 8 + h] = l;
    __syncthreads();
    if (t < 8) {
        float sum = 0.f;
        for (int i = 0; i < warps; ++i) sum += s_red[kSums + i * 8 + h];
        s_fin[1][h] = sum;
        if (NG == 1) { s_fin[0][h] = m; s_fin[2][h] = v[0]; }
    }

    // ---- values
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float w, const float4& a) {
        if (w != 0.f) { o.x = fmaf(a.x, w, o.x); o.y = fmaf(a.y, w, o.y); o.z = fmaf(a.z, w, o.z); o.w = fmaf(a.w, w, o.w); }
    };
    const int dg = NG > 1 ? d4 / (kHeadDim / 4 / NG) : 0;
    const float vr = finite_ref(NG > 1 ? s_fin[2 + dg][h] : v[0]);
    const float4* ov = reinterpret_cast<const float4*>(own + kOwnRecHead) + d4 * 8 + h;
#pragma unroll 4
    for (int i = slice; i < n_own; i += slices) {
        const float4 a = ov[(size_t)i * (kOwnRecFloats / 4)];
        add(s_part[(i * NG + dg) * 8 + h], a);
    }
    const int n_pre = items << twice;
    for (int i0 = slice; i0 < n_pre; i0 += 8 * slices) {
        float4 a[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) a[k] = pre_values(min(i0 + k * slices, n_pre - 1))[d4 * kPrefixRows + hc];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i0 + k * slices < n_pre) {
                const float f = s_part[(n_own * NG + i0 + k * slices) * 8 + h];
                add(NG == 1 ? f : f == -INFINITY ? 0.f : fast_exp2(f - vr), a[k]);
            }
    }
    if (slices > 1) {
        __syncthreads();
        reinterpret_cast<float4*>(s_red)[t] = o;
        __syncthreads();
        if (slice == 0)
            for (int i = 1; i < slices; ++i) {
                const float4 a = reinterpret_cast<const float4*>(s_red)[(i << (8 - ds)) + t];
                o.x += a.x; o.y += a.y; o.z += a.z; o.w += a.w;
            }
    } else {
        __syncthreads();
    }
    if (slice == 0 && h < p.g) {
        const float fm = s_fin[0][h], fl = s_fin[1][h], fv = s_fin[2 + dg][h];
        *reinterpret_cast<uint2*>(p.out + ((size_t)seq * p.h_q + (size_t)head * p.g + h) * kHeadDim + 4 * d4) =
            make_uint2(pack_bf16x2(final_value(o.x, fm, fl, fv, fits), final_value(o.y, fm, fl, fv, fits)),
                       pack_bf16x2(final_value(o.z, fm, fl, fv, fits), final_value(o.w, fm, fl, fv, fits)));
    }
    if (share == 0 && t < p.g) {
        if (p.lse) p.lse[(size_t)seq * p.h_q + (size_t)head * p.g + t] = final_lse(s_fin[0][t], s_fin[1][t], fits);
        if (p.len_out && head == 0 && t == 0 && fits) p.len_out[seq] += 1;
    }
}

// cluster > 1: clusters of that many CTAs; dependent: the kernel may start while the one before it drains.
template <typename... A>
static cudaError_t launch_ex(void (*kernel)(A...), unsigned grid, unsigned threads, size_t smem, int cluster, bool dependent, cudaStream_t s,
                             const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)cluster;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (dependent) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = (unsigned)n;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
template <int F>
static cudaError_t launch_own(const StoreAttnLaunch& p, cudaStream_t s) {
    const unsigned grid = (unsigned)(p.batch * p.h_kv * p.splits);
    if (p.dealt) return launch_ex(gkv_store_attn_kernel<F, kDealt>, grid, kThreads, 0, 1, false, s, p);
    if (store_needs_merge(p)) return launch_ex(gkv_store_attn_kernel<F, kPart>, grid, kThreads, 0, 1, p.prefix_part != nullptr, s, p);
    if (p.splits > 1) return launch_ex(gkv_store_attn_kernel<F, kCluster>, grid, kThreads, 0, p.splits, false, s, p);
    gkv_store_attn_kernel<F, kWhole><<<grid, kThreads, 0, s>>>(p);
    return cudaGetLastError();
}
bool store_needs_merge(const StoreAttnLaunch& p) { return p.dealt || p.splits > kMaxCluster || p.prefix_part != nullptr || p.len_out != nullptr; }
cudaError_t launch_store_attn(const StoreAttnLaunch& p, cudaStream_t s) {
    switch (p.format) {
        case GKV_STORE_BF16: return launch_own<GKV_STORE_BF16>(p, s);
        case GKV_STORE_E4M3: return launch_own<GKV_STORE_E4M3>(p, s);
        case GKV_STORE_INT8: return launch_own<GKV_STORE_INT8>(p, s);
        default:             return launch_own<GKV_STORE_INT4>(p, s);
    }
}
// The fewer units, the more CTAs per unit. 256 threads for up to 8 parts, 512 for up to 16, else 1024. (The plan bounds the parts
// of a unit: kMaxPieces + 2 kMaxRuns = 448, 8 numbers each are 3.5 per thread.) Dealt out, units have few parts or up to
// kMaxPieces, which the host does not know: threads by the number of units (256 units of 2 parts each with 1024, 512, 256 threads,
// attention included: 102, 96, 96 us; one of them with most of the rows: 63, 61, 65; 1024 units: -, 378, 370 and -, 167, 153).
cudaError_t launch_store_merge(const StoreAttnLaunch& p, cudaStream_t s) {
    int longest = 0;
    for (int i = 0; i < p.n_prefix; ++i) longest = p.prefix_len[i] > longest ? p.prefix_len[i] : longest;
    const int items = p.prefix_part ? ((longest + 127) / 128 + p.chunk - 1) / p.chunk * (p.two_tiles ? 1 : 2) : 0;
    const int own = p.dealt ? min(p.batch * p.splits, kMaxPieces) : p.splits, parts = own + items, units = p.batch * p.h_kv;
    const int ds = units <= 40 ? 2 : units <= 80 ? 1 : 0, ng = value_groups(p.format);
    const unsigned threads = p.dealt ? (units <= 148 ? 1024u : units <= 296 ? 512u : 256u) : parts <= 8 ? 256u : parts <= 16 ? 512u : 1024u;
    const auto kernel = ng == 1 ? (p.dealt ? gkv_store_merge_kernel<true, 1> : gkv_store_merge_kernel<false, 1>)
                                : (p.dealt ? gkv_store_merge_kernel<true, 4> : gkv_store_merge_kernel<false, 4>);
    return launch_ex(kernel, (unsigned)units << ds, threads, (size_t)(own * ng + items) * 8 * sizeof(float), 1, true, s, p, ds);
}

}  // namespace gkv
