// C-ABI entry points of the rotary positions and of the caches in pages: argument checks, the plan of an attention launch and the
// launches themselves. Nothing here keeps state between calls.
#include <math.h>
#include <stdint.h>

#include "gkv_common.cuh"
#include "gkv_internal.h"

using namespace gkv;

namespace {

constexpr int kMaxRotaryHead = 512;
constexpr int kMaxPageSize = 1 << 16;
constexpr int64_t kMaxPagedRows = 1ll << 31;      // over all pages and heads: row numbers are 32 bits
constexpr int64_t kMaxTableRows = 1 << 24;        // of a sequence
constexpr int kMaxPagedBatch = 65535;             // a grid dimension

bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
int scales_per_row(int format) { return format == GKV_STORE_BF16 ? 0 : format == GKV_STORE_INT4 ? 4 : 1; }
int row_bytes(int format) { return format == GKV_STORE_BF16 ? 256 : format == GKV_STORE_INT4 ? 64 : 128; }

gkv_status check_rotary(const gkv_rotary* r) {
    if (!r || r->head_dim < 2 || r->head_dim > kMaxRotaryHead || r->head_dim % 2 != 0) return GKV_ERR_INVALID_ARG;
    if (r->rot_dim < 2 || r->rot_dim > r->head_dim || r->rot_dim % 2 != 0) return GKV_ERR_INVALID_ARG;
    if (!isfinite(r->factor) || !r->turns || misaligned(r->turns, 8)) return GKV_ERR_INVALID_ARG;
    return GKV_OK;
}
RotaryView view(const gkv_rotary* r) {
    if (!r) return RotaryView{nullptr, 0, 0, 1.f};
    return RotaryView{r->turns, r->rot_dim / 2, r->interleaved != 0, r->factor};
}

gkv_status check_shape(const gkv_pages* g) {
    if (!g || g->format < GKV_STORE_BF16 || g->format > GKV_STORE_INT4) return GKV_ERR_INVALID_ARG;
    if (g->n_q_heads <= 0 || g->n_kv_heads <= 0 || g->head_dim <= 0 || g->n_pages <= 0 || g->page_size <= 0) return GKV_ERR_INVALID_ARG;
    if (g->n_q_heads % g->n_kv_heads != 0) return GKV_ERR_INVALID_ARG;
    if (g->head_dim != kHeadDim || g->n_q_heads / g->n_kv_heads > kMaxGroup || g->page_size > kMaxPageSize) return GKV_ERR_UNSUPPORTED;
    if ((int64_t)g->n_pages * g->page_size >= kMaxPagedRows || (int64_t)g->n_pages * g->page_size * g->n_kv_heads >= kMaxPagedRows)
        return GKV_ERR_UNSUPPORTED;
    return GKV_OK;
}
gkv_status check_pages(const gkv_pages* g, const gkv_page_table* t) {
    const gkv_status st = check_shape(g);
    if (st != GKV_OK) return st;
    if (!g->k || !g->v || misaligned(g->k, 16) || misaligned(g->v, 16)) return GKV_ERR_INVALID_ARG;
    if (g->format != GKV_STORE_BF16 && (!g->k_scale || !g->v_scale || misaligned(g->k_scale, 16) || misaligned(g->v_scale, 16)))
        return GKV_ERR_INVALID_ARG;
    if (!t || !t->page || misaligned(t->page, 4) || t->batch <= 0 || t->width <= 0 || t->stride < 0) return GKV_ERR_INVALID_ARG;
    if (t->batch > kMaxPagedBatch || (int64_t)t->batch * g->n_q_heads >= (1ll << 30)) return GKV_ERR_UNSUPPORTED;
    if ((int64_t)t->width * g->page_size > kMaxTableRows) return GKV_ERR_UNSUPPORTED;
    return GKV_OK;
}
PagesView view(const gkv_pages* g, const gkv_page_table* t) {
    PagesView v;
    v.data[0] = static_cast<uint8_t*>(g->k); v.data[1] = static_cast<uint8_t*>(g->v);
    v.scale[0] = static_cast<__nv_bfloat16*>(g->k_scale); v.scale[1] = static_cast<__nv_bfloat16*>(g->v_scale);
    v.table = t->page;
    v.table_stride = t->stride;
    v.inv_page = ((1ull << 40) + (uint64_t)g->page_size - 1) / (uint64_t)g->page_size;
    v.n_pages = g->n_pages; v.page_size = g->page_size;
    v.page_rows = (uint32_t)g->page_size * (uint32_t)g->n_kv_heads;
    v.head_rows = g->token_major ? 1u : (uint32_t)g->page_size;
    v.token_rows = g->token_major ? (uint32_t)g->n_kv_heads : 1u;
    return v;
}
// Room for the partial results of the form that deals out equal shares.
constexpr uint64_t kStreamBytes = (uint64_t)kStreamMaxWarps * 2 * kStreamRecFloats * sizeof(float);
constexpr int kStreamMaxUnits = 16384, kStreamMaxBatch = 2048;      // its merge has a CTA a unit, which adds up all lengths
constexpr int kStreamFrom = 6;

// A cluster of up to kMaxCluster CTAs a unit, if that leaves a warp no more than kStreamFrom tiles (or there are more units than the merge of the
// other form is made for); else equal shares for all warps. Returns the CTAs of the latter, 0 for the former. Both sides, measured: 32 x 4 heads of
// up to 1151 keys in 8 bits, 5 to 6 tiles a warp, 15 us in clusters, 22 in equal shares, which have the merge to pay; 1 x 4 heads of 4096 keys in
// bf16, 8 tiles a warp, 14.3 and 12.8.
int pages_plan(PagesAttnLaunch* p, int format, int max_len, int sm_count) {
    const int64_t units = (int64_t)p->batch * p->h_kv;
    const int tiles = (max_len + (p->k_new ? 1 : 0) + 15) / 16;
    int64_t splits = (int64_t)pages_attn_ctas_per_sm(format) * sm_count / units;
    const int64_t most = (tiles + 7) / 8;                      // two turns of the four warps
    if (splits > most) splits = most;
    if (splits > kMaxCluster) splits = kMaxCluster;
    if (splits < 1) splits = 1;
    p->split_tiles = tiles > 0 ? (int)((tiles + splits - 1) / splits) : 1;
    p->splits = tiles > 0 ? (tiles + p->split_tiles - 1) / p->split_tiles : 1;
    if (p->split_tiles <= 4 * kStreamFrom || units > kStreamMaxUnits || p->batch > kStreamMaxBatch) return 0;
    const int warps = pages_stream_warps_per_sm(*p, format) * sm_count;
    return warps < kStreamMaxWarps ? warps : kStreamMaxWarps;
}

gkv_status copy_args(const gkv_pages* g, const gkv_page_table* t, const void* k, const void* v, int64_t seq_stride, int64_t token_stride,
                     int64_t head_stride, const int32_t* first, const int32_t* count, int32_t n_tokens, const gkv_rotary* rotary,
                     const int32_t* pos, int64_t pos_seq_stride, int64_t pos_token_stride, bool read, PagesCopyLaunch* p) {
    gkv_status st = check_pages(g, t);
    if (st != GKV_OK) return st;
    if (n_tokens < 0 || (n_tokens > 0 && (!k || !v)) || misaligned(k, 16) || misaligned(v, 16)) return GKV_ERR_INVALID_ARG;
    if (misaligned(first, 4) || misaligned(count, 4) || misaligned(pos, 4)) return GKV_ERR_INVALID_ARG;
    if (seq_stride < 0 || token_stride < 0 || head_stride < 0 || ((seq_stride | token_stride | head_stride) & 7) != 0) return GKV_ERR_INVALID_ARG;
    if (pos && (pos_seq_stride < 0 || pos_token_stride < 0)) return GKV_ERR_INVALID_ARG;
    if (rotary) {
        st = check_rotary(rotary);
        if (st != GKV_OK) return st;
        if (rotary->head_dim != kHeadDim) return GKV_ERR_INVALID_ARG;
    }
    if ((int64_t)n_tokens * g->n_kv_heads >= (1ll << 30)) return GKV_ERR_UNSUPPORTED;
    if (read && n_tokens > 0 && k == v) return GKV_ERR_INVALID_ARG;
    if (read && n_tokens > 0 && rows_overlap(kHeadDim, {t->batch, n_tokens, g->n_kv_heads}, {seq_stride, token_stride, head_stride}))
        return GKV_ERR_INVALID_ARG;
    p->pages = view(g, t);
    p->rotary = view(rotary);
    p->pos = pos;
    p->pos_seq_stride = pos_seq_stride; p->pos_token_stride = pos_token_stride;
    p->x[0] = static_cast<__nv_bfloat16*>(const_cast<void*>(k)); p->x[1] = static_cast<__nv_bfloat16*>(const_cast<void*>(v));
    p->seq_stride = seq_stride; p->token_stride = token_stride; p->head_stride = head_stride;
    p->first = first; p->count = count;
    p->batch = t->batch; p->h_kv = g->n_kv_heads; p->capacity = t->width * g->page_size; p->n_tokens = n_tokens; p->format = g->format;
    return GKV_OK;
}

// gkv_pages_attn; expire: the step of every warp from which on its waits are taken for expired.
gkv_status run_attn(const gkv_pages* pages, const gkv_page_table* table, const int32_t* len, int32_t max_len, const void* q,
                    int64_t q_stride, const void* k_new, const void* v_new, int64_t kv_stride, const gkv_rotary* rotary,
                    const int32_t* pos, void* out, float* lse, void* workspace, uint64_t workspace_bytes, int expire, void* stream) {
    gkv_status st = check_pages(pages, table);
    if (st != GKV_OK) return st;
    if (!len || !q || !out || misaligned(len, 4) || misaligned(q, 16) || misaligned(out, 16) || misaligned(lse, 4) || misaligned(pos, 4))
        return GKV_ERR_INVALID_ARG;
    if ((k_new == nullptr) != (v_new == nullptr) || misaligned(k_new, 16) || misaligned(v_new, 16)) return GKV_ERR_INVALID_ARG;
    if (q_stride < 0 || q_stride % 8 != 0 || (k_new && (kv_stride < 0 || kv_stride % 8 != 0))) return GKV_ERR_INVALID_ARG;
    const int capacity = table->width * pages->page_size;
    if (max_len < 0 || max_len > capacity) return GKV_ERR_INVALID_ARG;
    if (rotary) {
        st = check_rotary(rotary);
        if (st != GKV_OK) return st;
        if (rotary->head_dim != kHeadDim) return GKV_ERR_INVALID_ARG;
    }
    if (!workspace || misaligned(workspace, 16) || workspace_bytes < kStreamBytes) return GKV_ERR_INVALID_ARG;

    PagesAttnLaunch p = {};
    p.pages = view(pages, table);
    p.rotary = view(rotary);
    p.pos = pos; p.len = len;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k_new = static_cast<const __nv_bfloat16*>(k_new); p.v_new = static_cast<const __nv_bfloat16*>(v_new);
    p.q_stride = q_stride; p.kv_stride = kv_stride;
    p.out = static_cast<__nv_bfloat16*>(out); p.lse = lse; p.own_part = static_cast<float*>(workspace);
    p.batch = table->batch; p.h_q = pages->n_q_heads; p.h_kv = pages->n_kv_heads; p.g = p.h_q / p.h_kv; p.capacity = capacity;
    p.scale_log2 = (float)(1.4426950408889634 / sqrt((double)kHeadDim));
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int sms = device_sm_count(), stream_ctas = pages_plan(&p, pages->format, max_len > 0 ? max_len : capacity, sms);
    if (expire != kNeverExpire && !stream_ctas) return GKV_ERR_UNSUPPORTED;
    const cudaError_t e = stream_ctas ? launch_pages_stream(p, pages->format, stream_ctas, expire, sms, s) : launch_pages_attn(p, pages->format, s);
    if (e != cudaSuccess) { (void)cudaGetLastError(); return GKV_ERR_CUDA; }
    return GKV_OK;
}

}  // namespace

extern "C" {

gkv_status gkv_rotary_frequencies(double theta, int32_t rot_dim, int32_t scaling, double scale, double original, double low, double high,
                                  double* radians, float* factor) {
    if (!radians || rot_dim < 2 || rot_dim > kMaxRotaryHead || rot_dim % 2 != 0 || !isfinite(theta) || !(theta > 1)) return GKV_ERR_INVALID_ARG;
    if (scaling < GKV_ROTARY_PLAIN || scaling > GKV_ROTARY_YARN) return GKV_ERR_INVALID_ARG;
    if (scaling != GKV_ROTARY_PLAIN && (!isfinite(scale) || !(scale >= 1))) return GKV_ERR_INVALID_ARG;
    if (scaling >= GKV_ROTARY_WAVELENGTH) {
        if (!isfinite(original) || !isfinite(low) || !isfinite(high) || !(original >= 1) || !(low > 0) || !(high > low)) return GKV_ERR_INVALID_ARG;
    }
    const double pi = 3.14159265358979323846;
    const int half = rot_dim / 2;
    const double base = scaling == GKV_ROTARY_NTK && rot_dim > 2 ? theta * pow(scale, (double)rot_dim / (rot_dim - 2)) : theta;
    // pair number at which `turns` turns are made in the original context
    auto pair_of = [&](double turns) { return rot_dim * log(original / (turns * 2 * pi)) / (2 * log(theta)); };
    double a = 0, b = 0;
    if (scaling == GKV_ROTARY_YARN) {
        a = fmax(floor(pair_of(high)), 0.);
        b = fmin(ceil(pair_of(low)), rot_dim - 1.);
    }
    for (int i = 0; i < half; ++i) {
        const double f = pow(base, -2.0 * i / rot_dim);
        double y = f;
        if (scaling == GKV_ROTARY_LINEAR) y = f / scale;
        if (scaling == GKV_ROTARY_WAVELENGTH) {
            const double keep = fmin(fmax((original * f / (2 * pi) - low) / (high - low), 0.), 1.);
            y = keep * f + (1 - keep) * f / scale;
        }
        if (scaling == GKV_ROTARY_YARN) {
            const double s = fmin(fmax((i - a) / fmax(b - a, 0.001), 0.), 1.);
            y = f * (1 - s) + f / scale * s;
        }
        radians[i] = y;
    }
    if (factor) *factor = scaling == GKV_ROTARY_YARN ? (float)(0.1 * log(scale) + 1) : 1.f;
    return GKV_OK;
}

gkv_status gkv_rotary_turns(const double* radians, int32_t n, uint64_t* turns) {
    if (n < 0 || (n > 0 && (!radians || !turns))) return GKV_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i)
        if (!(fabs(radians[i]) <= 0x1p20)) return GKV_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i) {   // 64 bits of mantissa: a frequency keeps all of its own 53
        const long double two_pi = 6.283185307179586476925286766559006L;
        long double t = (long double)radians[i] / two_pi;
        t -= floorl(t);                                        // a fraction of a turn
        const long double scaled = roundl(ldexpl(t, 64));
        turns[i] = scaled >= ldexpl(1.0L, 64) ? 0 : (uint64_t)scaled;
    }
    return GKV_OK;
}

gkv_status gkv_rotary_apply(const gkv_rotary* rotary, int32_t type, int32_t batch, int32_t n_tokens, const int32_t* pos,
                            int64_t pos_seq_stride, int64_t pos_token_stride, const int32_t* count, const gkv_rotary_rows* q,
                            const gkv_rotary_rows* k, int32_t transpose, void* stream) {
    const gkv_status st = check_rotary(rotary);
    if (st != GKV_OK) return st;
    if (type < GKV_TYPE_BF16 || type > GKV_TYPE_FP32 || batch <= 0 || n_tokens < 0 || !q) return GKV_ERR_INVALID_ARG;
    const int size = type == GKV_TYPE_FP32 ? 4 : 2;
    if (pos_seq_stride < 0 || pos_token_stride < 0 || misaligned(pos, 4) || misaligned(count, 4) || (n_tokens > 0 && !pos)) return GKV_ERR_INVALID_ARG;
    int64_t heads = 0;
    RotaryLaunch p = {};
    for (int i = 0; i < (k ? 2 : 1); ++i) {
        const gkv_rotary_rows* r = i ? k : q;
        if (r->n_heads <= 0 || (n_tokens > 0 && (!r->x || !r->y)) || misaligned(r->x, size) || misaligned(r->y, size)) return GKV_ERR_INVALID_ARG;
        const int64_t n[3] = {batch, n_tokens, r->n_heads};
        for (int d = 0; d < 3; ++d) {
            if (r->x_stride[d] < 0 || r->y_stride[d] < 0) return GKV_ERR_INVALID_ARG;
            if (r->x == r->y && n[d] > 1 && r->x_stride[d] != r->y_stride[d]) return GKV_ERR_INVALID_ARG;
            p.rows[i].xs[d] = n[d] > 1 ? r->x_stride[d] : 0;
            p.rows[i].ys[d] = n[d] > 1 ? r->y_stride[d] : 0;
        }
        if (n_tokens > 0 && rows_overlap(rotary->head_dim, n, p.rows[i].ys)) return GKV_ERR_INVALID_ARG;
        p.rows[i].x = r->x;
        p.rows[i].y = r->y;
        heads += r->n_heads;
    }
    if (k && n_tokens > 0 && q->y == k->y) return GKV_ERR_INVALID_ARG;
    if (batch > kMaxPagedBatch || (int64_t)n_tokens * heads >= (1ll << 30) || heads >= (1ll << 30)) return GKV_ERR_UNSUPPORTED;
    if (n_tokens == 0) return GKV_OK;
    p.rotary = view(rotary);
    p.sign = transpose ? -1.f : 1.f;
    p.pos = pos; p.count = count;
    p.pos_seq_stride = pos_seq_stride; p.pos_token_stride = pos_token_stride;
    p.heads0 = q->n_heads; p.heads = (int)heads;
    p.batch = batch; p.n_tokens = n_tokens;
    if (launch_rotary(p, type, rotary->head_dim, device_sm_count(), static_cast<cudaStream_t>(stream)) != cudaSuccess) {
        (void)cudaGetLastError();
        return GKV_ERR_CUDA;
    }
    return GKV_OK;
}

gkv_status gkv_pages_query_sizes(const gkv_pages* pages, gkv_store_sizes* out) {
    if (!out) return GKV_ERR_INVALID_ARG;
    const gkv_status st = check_shape(pages);
    if (st != GKV_OK) return st;
    const uint64_t rows = (uint64_t)pages->n_pages * pages->page_size * pages->n_kv_heads;
    out->k = out->v = rows * row_bytes(pages->format);
    out->k_scale = out->v_scale = rows * scales_per_row(pages->format) * 2;
    return GKV_OK;
}

gkv_status gkv_pages_append(const gkv_pages* pages, const gkv_page_table* table, const void* k, const void* v, int64_t seq_stride,
                            int64_t token_stride, int64_t head_stride, const int32_t* first, const int32_t* count, int32_t n_tokens,
                            const gkv_rotary* rotary, const int32_t* pos, int64_t pos_seq_stride, int64_t pos_token_stride, void* stream) {
    PagesCopyLaunch p;
    const gkv_status st = copy_args(pages, table, k, v, seq_stride, token_stride, head_stride, first, count, n_tokens, rotary, pos,
                                    pos_seq_stride, pos_token_stride, false, &p);
    if (st != GKV_OK || n_tokens == 0) return st;
    if (launch_pages_append(p, static_cast<cudaStream_t>(stream)) != cudaSuccess) { (void)cudaGetLastError(); return GKV_ERR_CUDA; }
    return GKV_OK;
}

gkv_status gkv_pages_read(const gkv_pages* pages, const gkv_page_table* table, void* k, void* v, int64_t seq_stride, int64_t token_stride,
                          int64_t head_stride, const int32_t* first, const int32_t* count, int32_t n_tokens, void* stream) {
    PagesCopyLaunch p;
    const gkv_status st = copy_args(pages, table, k, v, seq_stride, token_stride, head_stride, first, count, n_tokens, nullptr, nullptr, 0, 0, true, &p);
    if (st != GKV_OK || n_tokens == 0) return st;
    if (launch_pages_read(p, static_cast<cudaStream_t>(stream)) != cudaSuccess) { (void)cudaGetLastError(); return GKV_ERR_CUDA; }
    return GKV_OK;
}

gkv_status gkv_pages_attn_workspace(const gkv_pages* pages, int32_t batch, uint64_t* bytes) {
    if (!bytes) return GKV_ERR_INVALID_ARG;
    const gkv_status st = check_shape(pages);
    if (st != GKV_OK) return st;
    if (batch <= 0) return GKV_ERR_INVALID_ARG;
    if (batch > kMaxPagedBatch || (int64_t)batch * pages->n_q_heads >= (1ll << 30)) return GKV_ERR_UNSUPPORTED;
    *bytes = kStreamBytes;
    return GKV_OK;
}

gkv_status gkv_pages_attn(const gkv_pages* pages, const gkv_page_table* table, const int32_t* len, int32_t max_len, const void* q,
                          int64_t q_stride, const void* k_new, const void* v_new, int64_t kv_stride, const gkv_rotary* rotary,
                          const int32_t* pos, void* out, float* lse, void* workspace, uint64_t workspace_bytes, void* stream) {
    return run_attn(pages, table, len, max_len, q, q_stride, k_new, v_new, kv_stride, rotary, pos, out, lse, workspace, workspace_bytes,
                    kNeverExpire, stream);
}

gkv_status gkv_selftest_pages_wait(int32_t step, const gkv_pages* pages, const gkv_page_table* table, const int32_t* len, int32_t max_len,
                                   const void* q, int64_t q_stride, const void* k_new, const void* v_new, int64_t kv_stride,
                                   const gkv_rotary* rotary, const int32_t* pos, void* out, float* lse, void* workspace,
                                   uint64_t workspace_bytes, void* stream) {
    if (step < 0 || step == kNeverExpire) return GKV_ERR_INVALID_ARG;
    return run_attn(pages, table, len, max_len, q, q_stride, k_new, v_new, kv_stride, rotary, pos, out, lse, workspace, workspace_bytes, step,
                    stream);
}

}  // extern "C"
