// C-ABI entry points of the key/value stores and shared prefixes: argument checks, the plan of an attention launch and the
// launches themselves. Nothing here keeps state between calls.
#include <math.h>
#include <stdint.h>

#include "gkv_common.cuh"
#include "gkv_internal.h"

using namespace gkv;

namespace {

constexpr int kMaxStoreCapacity = 1 << 24;
constexpr int kMaxStoreBatch = 65535;      // a grid dimension
constexpr int kTileKeysOwn = 16;           // keys of a tile of the attention over own rows
constexpr int kDealPiece = 128, kDealUnit = 512;   // tiles from which on pieces, and whole units, are dealt out by the lengths
constexpr int64_t kSplitUnits = 2048;      // a launch that cuts units into pieces has at most this many (sizes the workspace)
constexpr int kMaxRuns = 160;              // runs of a prefix
constexpr int kPrefixSplitItems = 296;     // prefix items beyond one per row block are at most this many

uint64_t align_up(uint64_t x) { return (x + 255) / 256 * 256; }
bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
int scales_per_row(int format) { return format == GKV_STORE_BF16 ? 0 : format == GKV_STORE_INT4 ? 4 : 1; }
int row_bytes(int format) { return format == GKV_STORE_BF16 ? 256 : format == GKV_STORE_INT4 ? 64 : 128; }

gkv_status check_shape(const gkv_store* s) {
    if (!s || s->format < GKV_STORE_BF16 || s->format > GKV_STORE_INT4) return GKV_ERR_INVALID_ARG;
    if (s->batch <= 0 || s->n_q_heads <= 0 || s->n_kv_heads <= 0 || s->head_dim <= 0 || s->capacity <= 0) return GKV_ERR_INVALID_ARG;
    if (s->n_q_heads % s->n_kv_heads != 0) return GKV_ERR_INVALID_ARG;
    if (s->head_dim != kHeadDim || s->n_q_heads / s->n_kv_heads > kMaxGroup) return GKV_ERR_UNSUPPORTED;
    if (s->batch > kMaxStoreBatch || s->capacity > kMaxStoreCapacity) return GKV_ERR_UNSUPPORTED;
    if ((int64_t)s->batch * s->n_q_heads >= (1ll << 30)) return GKV_ERR_UNSUPPORTED;
    return GKV_OK;
}
gkv_status check_store(const gkv_store* s) {
    const gkv_status st = check_shape(s);
    if (st != GKV_OK) return st;
    if (!s->k || !s->v || misaligned(s->k, 16) || misaligned(s->v, 16)) return GKV_ERR_INVALID_ARG;
    if (s->format != GKV_STORE_BF16 && (!s->k_scale || !s->v_scale || misaligned(s->k_scale, 8) || misaligned(s->v_scale, 8)))
        return GKV_ERR_INVALID_ARG;
    return GKV_OK;
}

// Row blocks of a (prefix, KV head): up to 256 query rows, whole sequences, about equally many in each.
void row_blocks(int seqs, int g, int* seqs_per_block, int* n_blocks, int* two_tiles) {
    const int most = kPrefixRows / g;
    *n_blocks = (seqs + most - 1) / most;
    *seqs_per_block = (seqs + *n_blocks - 1) / *n_blocks;
    *n_blocks = (seqs + *seqs_per_block - 1) / *seqs_per_block;
    *two_tiles = *seqs_per_block * g > kPrefixRows / 2 ? 1 : 0;
}
int64_t prefix_items(const StoreAttnLaunch& p, int chunk) {
    int64_t items = 0;
    for (int i = 0; i < p.n_prefix; ++i) items += ((p.prefix_len[i] + 127) / 128 + chunk - 1) / chunk;
    return items * p.h_kv * p.n_blocks;
}

// Upper bounds over all lengths, without a device. Partial results of own rows: of every unit when they are merged with
// something else, and of the pieces of cut units.
uint64_t own_part_bytes(const gkv_store* s, bool merged) {
    const uint64_t units = (uint64_t)s->batch * s->n_kv_heads;
    const uint64_t pieces = units * kMaxPieces < (uint64_t)kSplitUnits ? units * kMaxPieces : (uint64_t)kSplitUnits;
    return align_up((pieces > units || !merged ? pieces : units) * kOwnRecFloats * 4);
}
uint64_t prefix_part_bytes(const gkv_store* s, int n_prefix, int rows) {
    if (n_prefix == 0 || rows == 0) return 0;
    int per_block, blocks, two;
    row_blocks(s->batch / n_prefix, s->n_q_heads / s->n_kv_heads, &per_block, &blocks, &two);
    const uint64_t base = (uint64_t)n_prefix * s->n_kv_heads * blocks;
    const uint64_t most = base * (uint64_t)((rows + 127) / 128);
    return align_up((most < base + kPrefixSplitItems ? most : base + kPrefixSplitItems) * kPrefixRecFloats * 4);
}

gkv_status check_prefix(const gkv_prefix* x, int batch, int h_kv) {
    if (x->n_prefix < 1 || x->n_prefix > kMaxPrefixes || batch % x->n_prefix != 0 || x->rows < 0 || !x->len) return GKV_ERR_INVALID_ARG;
    int longest = 0;
    for (int i = 0; i < x->n_prefix; ++i) {
        if (x->len[i] < 0 || x->len[i] > x->rows) return GKV_ERR_INVALID_ARG;
        longest = x->len[i] > longest ? x->len[i] : longest;
    }
    if (longest > 0 && (!x->k || !x->v || misaligned(x->k, 16) || misaligned(x->v, 16))) return GKV_ERR_INVALID_ARG;
    // row coordinates of the tensor maps are signed 32-bit numbers, and a tile may reach past the end
    if ((int64_t)x->n_prefix * h_kv * x->rows >= (1ll << 31) - 256) return GKV_ERR_UNSUPPORTED;
    return GKV_OK;
}

// Everything of an attention launch that is not a pointer, then the launches. `p` has its pointers and shape.
gkv_status run_attn(StoreAttnLaunch& p, const PrefixWatch& watch, const gkv_store* shape, const gkv_prefix* prefix, int max_len, void* workspace,
                    uint64_t workspace_bytes, int sm_count, cudaStream_t s, int* launches) {
    p.prefix_part = nullptr;
    p.n_prefix = 0;
    p.prefix_items = 0;
    int longest = 0;
    if (prefix) {
        p.n_prefix = prefix->n_prefix;
        p.prefix_rows = prefix->rows;
        p.k_prefix = static_cast<const __nv_bfloat16*>(prefix->k);
        p.v_prefix = static_cast<const __nv_bfloat16*>(prefix->v);
        for (int i = 0; i < p.n_prefix; ++i) {
            p.prefix_len[i] = prefix->len[i];
            longest = prefix->len[i] > longest ? prefix->len[i] : longest;
        }
    }
    const uint64_t own = own_part_bytes(shape, longest > 0 || p.len_out);
    const uint64_t need = own + (longest > 0 ? prefix_part_bytes(shape, p.n_prefix, longest) : 0);
    if (!workspace || misaligned(workspace, 16) || workspace_bytes < need) return GKV_ERR_INVALID_ARG;
    p.own_part = static_cast<float*>(workspace);
    if (longest > 0) p.prefix_part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + own);
    store_plan(&p, max_len, sm_count);

    CUtensorMap tm_k, tm_v;
    if (longest > 0) {
        const uint64_t rows = (uint64_t)p.n_prefix * p.h_kv * p.prefix_rows;
        if (encode_map(&tm_k, const_cast<__nv_bfloat16*>(p.k_prefix), rows, 128) != GKV_OK ||
            encode_map(&tm_v, const_cast<__nv_bfloat16*>(p.v_prefix), rows, 128) != GKV_OK)
            return GKV_ERR_CUDA;
        if (launch_prefix_attn(p, watch, tm_k, tm_v, s) != cudaSuccess) { (void)cudaGetLastError(); return GKV_ERR_CUDA; }
        ++*launches;
    }
    if (launch_store_attn(p, s) != cudaSuccess) { (void)cudaGetLastError(); return GKV_ERR_CUDA; }
    ++*launches;
    if (store_needs_merge(p)) {
        if (launch_store_merge(p, s) != cudaSuccess) { (void)cudaGetLastError(); return GKV_ERR_CUDA; }
        ++*launches;
    }
    return GKV_OK;
}

gkv_status copy_args(const gkv_store* store, const void* k, const void* v, int64_t seq_stride, int64_t token_stride, int64_t head_stride,
                     const int32_t* first, const int32_t* count, int32_t n_tokens, bool read, StoreCopyLaunch* p) {
    const gkv_status st = check_store(store);
    if (st != GKV_OK) return st;
    if (n_tokens < 0 || (n_tokens > 0 && (!k || !v)) || misaligned(k, 16) || misaligned(v, 16)) return GKV_ERR_INVALID_ARG;
    if (misaligned(first, 4) || misaligned(count, 4)) return GKV_ERR_INVALID_ARG;
    if (seq_stride < 0 || token_stride < 0 || head_stride < 0 || ((seq_stride | token_stride | head_stride) & 7) != 0) return GKV_ERR_INVALID_ARG;
    if ((int64_t)n_tokens * store->n_kv_heads >= (1ll << 30)) return GKV_ERR_UNSUPPORTED;
    if (read && n_tokens > 0 && k == v) return GKV_ERR_INVALID_ARG;
    if (read && n_tokens > 0 && rows_overlap(kHeadDim, {store->batch, n_tokens, store->n_kv_heads}, {seq_stride, token_stride, head_stride})) return GKV_ERR_INVALID_ARG;
    p->data[0] = static_cast<uint8_t*>(store->k); p->data[1] = static_cast<uint8_t*>(store->v);
    p->scale[0] = static_cast<__nv_bfloat16*>(store->k_scale); p->scale[1] = static_cast<__nv_bfloat16*>(store->v_scale);
    p->x[0] = static_cast<__nv_bfloat16*>(const_cast<void*>(k)); p->x[1] = static_cast<__nv_bfloat16*>(const_cast<void*>(v));
    p->seq_stride = seq_stride; p->token_stride = token_stride; p->head_stride = head_stride;
    p->first = first; p->count = count;
    p->batch = store->batch; p->h_kv = store->n_kv_heads; p->capacity = store->capacity; p->n_tokens = n_tokens; p->format = store->format;
    return GKV_OK;
}

}  // namespace

namespace gkv {

// Whether elements of an array of rows of `width` share an address (or may, with strides that no slice of an array has).
bool rows_overlap(int64_t width, const int64_t (&sizes)[3], const int64_t (&s)[3]) {
    int64_t n[3] = {sizes[0], sizes[1], sizes[2]};
    int64_t least = width;                  // the next larger stride has to step over what the smaller ones span
    for (int k = 0; k < 3; ++k) {
        int next = -1;
        for (int i = 0; i < 3; ++i)
            if (n[i] > 1 && (next < 0 || s[i] < s[next])) next = i;
        if (next < 0) break;
        if (s[next] < least || s[next] > INT64_MAX / n[next]) return true;
        least = s[next] * n[next];
        n[next] = 1;
    }
    return false;
}

int device_sm_count() {
    int dev = 0, sm = 0;
    if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sm, cudaDevAttrMultiProcessorCount, dev);
    return sm > 0 ? sm : 148;
}

// Own rows: as many pieces per unit as fill the places of resident CTAs, none below 8 tiles (two turns of the four warps). (With
// more units than half the places units go whole: cutting 1024 units into thirds, to fill the last round of CTAs better, took 157
// us as clusters and 105 us by way of the workspace where whole units take 110 us.) With long
// rows the pieces are dealt out by the lengths that the sequences really have (store_piece_tiles), by way of the workspace, which
// costs a merge of 4 us when all are equally long and saves more the more they differ (32 sequences x 4 heads of 8192 keys in 8
// bits: 49 us as clusters, 53 dealt out; of 256 to 8192 keys: 43, 36; one of 8192 and 31 of 512: 36, 20. 128 x 8 heads, one of
// 65536 and 127 of 2048 keys: 963 us as whole units, 153; all of 8192 keys: 352, 369). A single sequence, launches with a prefix
// and those of a context are not dealt out: their pieces go by max_len alone, and where that is far above the lengths the last
// pieces have no keys.
// Prefixes: the length of the runs that the prefixes' key tiles are cut into. An item occupies an SM for about 8 us + 1.05 us a
// tile (2.1 with more than 128 query rows); the attention over own rows (at 5.5 TB/s, with sequences three quarters of the
// longest on average) takes the SMs that are left and, in part, the same ones; every run leaves a partial result that is written
// and read again (3.4 TB/s). Short runs end soon, long ones waste less. (32 answers on 8192 shared rows, 64 tiles, by tiles of a
// run: 1: 53 us, 2: 44, 4: 33, 6: 31, 8: 36, 16: 53; 128 answers on 4 documents of up to 128 tiles: 26: 161 us, 43: 145, 64: 177.)
void store_plan(StoreAttnLaunch* p, int max_len, int sm_count) {
    const int64_t units = (int64_t)p->batch * p->h_kv, places = (int64_t)store_attn_ctas_per_sm(p->format) * sm_count;
    const int n = max_len + (p->k_new ? 1 : 0);
    const int tiles = n > 0 ? (n + kTileKeysOwn - 1) / kTileKeysOwn : 1;
    int64_t splits = places / units;
    const int64_t most = (tiles + 7) / 8;
    if (splits > most) splits = most;
    if (splits > kMaxPieces) splits = kMaxPieces;
    if (units * splits > kSplitUnits) splits = kSplitUnits / units;
    if (splits < 1) splits = 1;
    p->dealt = 0;
    if (p->batch > 1 && !p->prefix_part && !p->len_out) {
        if (tiles / splits >= (splits > 1 ? kDealPiece : kDealUnit) && units * 2 <= kSplitUnits) {
            p->dealt = 1;
            if (splits < 2) splits = 2;
        }
        if (splits > kMaxCluster) p->dealt = 1;
    }
    p->split_tiles = (int)((tiles + splits - 1) / splits);
    p->splits = (tiles + p->split_tiles - 1) / p->split_tiles;
    if (!p->prefix_part) return;
    p->seqs_per_prefix = p->batch / p->n_prefix;
    row_blocks(p->seqs_per_prefix, p->g, &p->seqs_per_block, &p->n_blocks, &p->two_tiles);
    int longest = 0;
    for (int i = 0; i < p->n_prefix; ++i) longest = p->prefix_len[i] > longest ? p->prefix_len[i] : longest;
    const int key_tiles = (longest + 127) / 128;
    const int64_t base = prefix_items(*p, key_tiles);
    const double row = row_bytes(p->format) + 2 * scales_per_row(p->format);
    const double own_us = 4 + 0.75 * n * row * 2 * units / 5.5e6, part_us = (double)p->batch * p->h_q * kHeadDim * 8 / 3.4e6;
    double best = -1;
    for (int runs = 1; runs <= key_tiles && runs <= kMaxRuns; ++runs) {
        const int chunk = (key_tiles + runs - 1) / runs;
        const int64_t items = prefix_items(*p, chunk), rounds = (items + sm_count - 1) / sm_count;
        if (runs > 1 && items > base + kPrefixSplitItems) break;
        const double item_us = 8 + (p->two_tiles ? 2.1 : 1.05) * chunk;
        const double alone = rounds * item_us, together = own_us + items * item_us / sm_count;
        const double cost = (alone > together ? alone : together) + part_us * ((key_tiles + chunk - 1) / chunk);
        if (best < 0 || cost < best) { best = cost; p->chunk = chunk; p->prefix_items = (int)items; }
    }
}

}  // namespace gkv

extern "C" {

gkv_status gkv_store_query_sizes(const gkv_store* store, gkv_store_sizes* out) {
    if (!out) return GKV_ERR_INVALID_ARG;
    const gkv_status st = check_shape(store);
    if (st != GKV_OK) return st;
    const uint64_t rows = (uint64_t)store->batch * store->n_kv_heads * store->capacity;
    out->k = out->v = rows * row_bytes(store->format);
    out->k_scale = out->v_scale = rows * scales_per_row(store->format) * 2;
    return GKV_OK;
}

gkv_status gkv_store_write(const gkv_store* store, const void* k, const void* v, int64_t seq_stride, int64_t token_stride,
                           int64_t head_stride, const int32_t* first, const int32_t* count, int32_t n_tokens, void* stream) {
    StoreCopyLaunch p;
    const gkv_status st = copy_args(store, k, v, seq_stride, token_stride, head_stride, first, count, n_tokens, false, &p);
    if (st != GKV_OK || n_tokens == 0) return st;
    if (launch_store_write(p, static_cast<cudaStream_t>(stream)) != cudaSuccess) { (void)cudaGetLastError(); return GKV_ERR_CUDA; }
    return GKV_OK;
}

gkv_status gkv_store_read(const gkv_store* store, void* k, void* v, int64_t seq_stride, int64_t token_stride, int64_t head_stride,
                          const int32_t* first, const int32_t* count, int32_t n_tokens, void* stream) {
    StoreCopyLaunch p;
    const gkv_status st = copy_args(store, k, v, seq_stride, token_stride, head_stride, first, count, n_tokens, true, &p);
    if (st != GKV_OK || n_tokens == 0) return st;
    if (launch_store_read(p, static_cast<cudaStream_t>(stream)) != cudaSuccess) { (void)cudaGetLastError(); return GKV_ERR_CUDA; }
    return GKV_OK;
}

gkv_status gkv_store_attn_workspace(const gkv_store* store, int32_t n_prefix, int32_t prefix_rows, uint64_t* bytes) {
    if (!bytes) return GKV_ERR_INVALID_ARG;
    const gkv_status st = check_shape(store);
    if (st != GKV_OK) return st;
    if (n_prefix < 0 || prefix_rows < 0 || n_prefix > kMaxPrefixes || (n_prefix > 0 && store->batch % n_prefix != 0)) return GKV_ERR_INVALID_ARG;
    uint64_t most = 0;   // fewer prefixes mean larger row blocks: the bound has to hold for each number up to n_prefix
    for (int i = 1; i <= n_prefix; ++i) {
        if (store->batch % i != 0) continue;
        const uint64_t b = prefix_part_bytes(store, i, prefix_rows);
        most = b > most ? b : most;
    }
    *bytes = own_part_bytes(store, n_prefix > 0) + most;
    return GKV_OK;
}

gkv_status gkv_store_attn(const gkv_store* store, const int32_t* len, int32_t max_len, const void* q, const void* k_new, const void* v_new,
                          const gkv_prefix* prefix, void* out, float* lse, void* workspace, uint64_t workspace_bytes, void* stream) {
    gkv_status st = check_store(store);
    if (st != GKV_OK) return st;
    if (!len || !q || !out || misaligned(len, 4) || misaligned(q, 16) || misaligned(out, 16) || misaligned(lse, 4)) return GKV_ERR_INVALID_ARG;
    if ((k_new == nullptr) != (v_new == nullptr) || misaligned(k_new, 16) || misaligned(v_new, 16)) return GKV_ERR_INVALID_ARG;
    if (max_len < 0 || max_len > store->capacity) return GKV_ERR_INVALID_ARG;
    if (prefix) {
        st = check_prefix(prefix, store->batch, store->n_kv_heads);
        if (st != GKV_OK) return st;
    }
    StoreAttnLaunch p = {};
    p.k = static_cast<uint8_t*>(store->k); p.v = static_cast<uint8_t*>(store->v);
    p.k_scale = static_cast<__nv_bfloat16*>(store->k_scale); p.v_scale = static_cast<__nv_bfloat16*>(store->v_scale);
    p.len = len;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k_new = static_cast<const __nv_bfloat16*>(k_new); p.v_new = static_cast<const __nv_bfloat16*>(v_new);
    p.out = static_cast<__nv_bfloat16*>(out);
    p.lse = lse;
    p.format = store->format; p.batch = store->batch; p.h_q = store->n_q_heads; p.h_kv = store->n_kv_heads;
    p.g = store->n_q_heads / store->n_kv_heads; p.capacity = store->capacity;
    p.scale_log2 = (float)(1.4426950408889634 / sqrt((double)kHeadDim));
    int launches = 0;
    return run_attn(p, PrefixWatch{nullptr, 0}, store, prefix, max_len > 0 ? max_len : store->capacity, workspace, workspace_bytes, device_sm_count(),
                    static_cast<cudaStream_t>(stream), &launches);
}

gkv_status gkv_selftest_prefix_wait(gkv_ctx* ctx) {
    if (!ctx) return GKV_ERR_INVALID_ARG;
    ctx->prefix_give_up = 1;
    return GKV_OK;
}

gkv_status gkv_decode_attn_prefix(gkv_ctx* ctx, int32_t layer, const void* q, const void* k_new, const void* v_new,
                                  const gkv_prefix* prefix, void* out, void* workspace, uint64_t workspace_bytes, void* stream) {
    if (!ctx || layer < 0 || layer >= ctx->cfg.n_layers || !q || !k_new || !v_new || !out || !prefix) return GKV_ERR_INVALID_ARG;
    if (misaligned(q, 16) || misaligned(k_new, 16) || misaligned(v_new, 16) || misaligned(out, 16)) return GKV_ERR_INVALID_ARG;
    const gkv_config& c = ctx->cfg;
    const gkv_status st = check_prefix(prefix, c.batch, c.n_kv_heads);
    if (st != GKV_OK) return st;
    if (c.fuse_window_scores) return GKV_ERR_STATE;
    if (ctx->len[layer] >= ctx->C) return GKV_ERR_CAPACITY;
    gkv_store shape = {};
    shape.format = GKV_STORE_BF16; shape.batch = c.batch; shape.n_q_heads = c.n_q_heads; shape.n_kv_heads = c.n_kv_heads;
    shape.head_dim = kHeadDim; shape.capacity = ctx->C;
    StoreAttnLaunch p = {};
    const size_t layer_bytes = (size_t)ctx->units_per_layer * ctx->C * kRowBytes;
    p.k = static_cast<uint8_t*>(ctx->buf.k) + layer * layer_bytes;
    p.v = static_cast<uint8_t*>(ctx->buf.v) + layer * layer_bytes;
    p.len_out = static_cast<int32_t*>(ctx->buf.len) + (size_t)layer * c.batch;
    p.len = p.len_out;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k_new = static_cast<const __nv_bfloat16*>(k_new); p.v_new = static_cast<const __nv_bfloat16*>(v_new);
    p.out = static_cast<__nv_bfloat16*>(out);
    const PrefixWatch watch = {reinterpret_cast<int32_t*>(static_cast<uint8_t*>(ctx->buf.workspace) + ctx->ws.status), ctx->prefix_give_up};
    p.format = GKV_STORE_BF16; p.batch = c.batch; p.h_q = c.n_q_heads; p.h_kv = c.n_kv_heads; p.g = ctx->g; p.capacity = ctx->C;
    p.scale_log2 = (float)(1.4426950408889634 / sqrt((double)kHeadDim));
    int launches = 0;
    const gkv_status r = run_attn(p, watch, &shape, prefix, ctx->len[layer], workspace, workspace_bytes, ctx->sm_count,
                                  static_cast<cudaStream_t>(stream), &launches);
    ctx->launches += launches;
    if (r != GKV_OK) return r;
    ctx->prefix_give_up = 0;
    ctx->len[layer] += 1;
    ctx->since_evict[layer] += 1;
    ctx->stage_next[layer] = 0;
    ctx->cbar_valid[layer] = 0;
    ctx->sacc_valid[layer] = 0;
    return GKV_OK;
}

}  // extern "C"
