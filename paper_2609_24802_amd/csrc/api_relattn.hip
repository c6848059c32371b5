// C entry points of attention over rectangular relations: cross attention and the paged cache.
#include <cmath>
#include <new>
#include <vector>

#include "relattn.hpp"
#include "rotary.hpp"

using namespace tiga;

namespace {

bool bad_float(float v) { return !(v > -3.0e38f) || !(v < 3.0e38f); }

// Rows of keys and values lie within 2^23 elements of each other: a tile's offsets are 32-bit.
int check_rows(const char *what, const char *name, const tiga_view *v) {
    if (v->row >= (int64_t(1) << 23)) return fail(TIGA_EUNSUPPORTED, "%s: the row stride of %s must be below 2^23", what, name);
    return TIGA_OK;
}

// A 16-bit tensor whose rows are read and written 16 bytes at a time.
int check_view(const char *what, const char *name, const tiga_view *v, bool output, int64_t batch, int64_t heads,
               int64_t rows) {
    if (!v || !v->data) return fail(TIGA_EINVAL, "%s: %s is required", what, name);
    if (!aligned16(v->data)) return fail(TIGA_EINVAL, "%s: %s must be 16-byte aligned", what, name);
    if ((v->batch | v->head | v->row) & 7) return fail(TIGA_EINVAL, "%s: strides of %s must be multiples of 8", what, name);
    if (v->batch < 0 || v->head < 0 || v->row < 0) return fail(TIGA_EINVAL, "%s: negative stride of %s", what, name);
    if (v->head > 0x7fffffff || v->row > 0x7fffffff)
        return fail(TIGA_EUNSUPPORTED, "%s: the head and row strides of %s must be below 2^31", what, name);
    if (output && ((batch > 1 && v->batch == 0) || (heads > 1 && v->head == 0) || (rows > 1 && v->row == 0)))
        return fail(TIGA_EINVAL, "%s: the rows of %s overlap (a stride is 0)", what, name);
    return TIGA_OK;
}

int check_scale(const char *what, float scale) {
    if (!(scale > 0.0f) || !(scale < 3.0e38f)) return fail(TIGA_EINVAL, "%s: scale must be finite and > 0", what);
    return TIGA_OK;
}

int check_ws(const char *what, const void *ws, size_t have, size_t need) {
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u))
        return fail(TIGA_EINVAL, "%s: the workspace is required and must be 256-byte aligned", what);
    if (have < need) return fail(TIGA_EWORKSPACE, "%s: workspace of %zu bytes, %zu needed", what, have, need);
    return TIGA_OK;
}

int check_heads(const char *what, int32_t heads, int32_t kv_heads, int32_t width, int dtype) {
    if (heads < 0 || kv_heads < 0) return fail(TIGA_EINVAL, "%s: negative number of heads", what);
    if (kv_heads == 0 ? heads != 0 : heads % kv_heads != 0)
        return fail(TIGA_EINVAL, "%s: %d heads are no multiple of %d source heads", what, heads, kv_heads);
    if (dtype != TIGA_DT_F16 && dtype != TIGA_DT_BF16) return fail(TIGA_EINVAL, "%s: unknown dtype %d", what, dtype);
    if (width != 64 && width != 128) return fail(TIGA_EUNSUPPORTED, "%s: width %d (64 or 128 supported)", what, width);
    return TIGA_OK;
}

constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1024;

int check_cross(const tiga_cross *rel) {
    const char *what = "cross attention";
    if (!rel) return fail(TIGA_EINVAL, "%s: the relation is required", what);
    if (rel->num_dst < 0 || rel->num_src < 0 || rel->batch < 0) return fail(TIGA_EINVAL, "%s: negative size", what);
    if (int rc = check_heads(what, rel->heads, rel->kv_heads, rel->width, rel->dtype)) return rc;
    if (reinterpret_cast<uintptr_t>(rel->src_len) & 3u) return fail(TIGA_EINVAL, "%s: src_len misaligned", what);
    if (rel->num_dst >= kMaxRows || rel->num_src >= kMaxRows)
        return fail(TIGA_EUNSUPPORTED, "%s: num_dst and num_src must be < 2^31 - 1024", what);
    if (static_cast<int64_t>(rel->batch) * rel->kv_heads >= (1 << 20))
        return fail(TIGA_EUNSUPPORTED, "%s: batch * kv_heads must be < 2^20", what);
    if (static_cast<double>(rel->batch) * rel->heads * static_cast<double>(rel->num_dst) >= 1099511627776.0)
        return fail(TIGA_EUNSUPPORTED, "%s: batch * heads * num_dst must be < 2^40", what);
    if (rel->kv_heads && rel->num_dst * (rel->heads / rel->kv_heads) >= kMaxRows)
        return fail(TIGA_EUNSUPPORTED, "%s: num_dst * heads / kv_heads must be < 2^31 - 1024", what);
    return TIGA_OK;
}

int check_cache(const char *what, const tiga_cache *c) {
    if (!c) return fail(TIGA_EINVAL, "%s: the cache is required", what);
    if (c->num_pages < 0 || c->batch < 0 || c->table_width < 0) return fail(TIGA_EINVAL, "%s: negative size", what);
    if (int rc = check_heads(what, c->kv_heads, c->kv_heads, c->width, c->dtype)) return rc;
    if (c->page_size < 1 || (c->page_size & (c->page_size - 1)))
        return fail(TIGA_EINVAL, "%s: page_size %d is no power of two", what, c->page_size);
    if (c->page_size > (1 << 15)) return fail(TIGA_EUNSUPPORTED, "%s: page_size %d (at most 32768)", what, c->page_size);
    if (c->batch >= (1 << 16)) return fail(TIGA_EUNSUPPORTED, "%s: batch must be < 2^16", what);
    if (c->num_pages > 0x7fffffff) return fail(TIGA_EUNSUPPORTED, "%s: num_pages must be < 2^31", what);
    if (static_cast<int64_t>(c->table_width) * c->page_size >= kMaxRows)
        return fail(TIGA_EUNSUPPORTED, "%s: table_width * page_size must be < 2^31 - 1024", what);
    return TIGA_OK;
}

// The cache's arrays, for a call with rows to work on.
int check_cache_data(const char *what, const tiga_cache *c, const int32_t *dst_ptr) {
    if (c->num_pages < 1) return fail(TIGA_EINVAL, "%s: the cache has no pages", what);
    if (int rc = check_view(what, "the cache's k", &c->k, true, c->num_pages, c->kv_heads, c->page_size)) return rc;
    if (int rc = check_view(what, "the cache's v", &c->v, true, c->num_pages, c->kv_heads, c->page_size)) return rc;
    if (int rc = check_rows(what, "the cache's k", &c->k)) return rc;
    if (int rc = check_rows(what, "the cache's v", &c->v)) return rc;
    if ((!c->table && c->table_width > 0) || !c->length || !dst_ptr)
        return fail(TIGA_EINVAL, "%s: table, length and dst_ptr are required", what);
    if ((reinterpret_cast<uintptr_t>(c->table) | reinterpret_cast<uintptr_t>(c->length) |
         reinterpret_cast<uintptr_t>(dst_ptr)) & 3u)
        return fail(TIGA_EINVAL, "%s: table, length and dst_ptr must be 4-byte aligned", what);
    return TIGA_OK;
}

int check_packed(const char *what, int64_t num_dst, int32_t heads) {
    if (num_dst < 0) return fail(TIGA_EINVAL, "%s: negative num_dst", what);
    if (num_dst >= kMaxRows || num_dst * heads >= kMaxRows)
        return fail(TIGA_EUNSUPPORTED, "%s: num_dst * heads must be < 2^31 - 1024", what);
    return TIGA_OK;
}

}  // namespace

extern "C" {

size_t tiga_mp_attention_cross_fwd_workspace(const tiga_cross *rel) {
    clear_error();  // no EntryScope: armed kernel events are for the call that follows
    return check_cross(rel) ? 0 : relattn::cross_fwd_ws_bytes(*rel);
}

int tiga_mp_attention_cross_fwd(const tiga_cross *rel, const tiga_view *q, const tiga_view *k, const tiga_view *v,
                                float scale, const tiga_view *y, float *lse, void *ws, size_t ws_bytes, void *stream) {
    EntryScope scope;
    const char *what = "cross attention";
    if (int rc = check_cross(rel)) return rc;
    if (int rc = check_scale(what, scale)) return rc;
    if (rel->batch == 0 || rel->heads == 0 || rel->num_dst == 0) return TIGA_OK;
    if (int rc = check_view(what, "q", q, false, 0, 0, 0)) return rc;
    if (rel->num_src > 0) {
        if (int rc = check_view(what, "k", k, false, 0, 0, 0)) return rc;
        if (int rc = check_view(what, "v", v, false, 0, 0, 0)) return rc;
        if (int rc = check_rows(what, "k", k)) return rc;
        if (int rc = check_rows(what, "v", v)) return rc;
    }
    if (int rc = check_view(what, "y", y, true, rel->batch, rel->heads, rel->num_dst)) return rc;
    if (reinterpret_cast<uintptr_t>(lse) & 3u) return fail(TIGA_EINVAL, "%s: lse misaligned", what);
    if (int rc = check_ws(what, ws, ws_bytes, relattn::cross_fwd_ws_bytes(*rel))) return rc;
    const tiga_view none{};
    return relattn::cross_forward(*rel, *q, rel->num_src ? *k : none, rel->num_src ? *v : none, scale, *y, lse, ws,
                                  static_cast<hipStream_t>(stream));
}

size_t tiga_mp_attention_cross_bwd_workspace(const tiga_cross *rel) {
    clear_error();  // no EntryScope: armed kernel events are for the call that follows
    return check_cross(rel) ? 0 : relattn::cross_bwd_ws_bytes(*rel);
}

int tiga_mp_attention_cross_bwd(const tiga_cross *given, const tiga_view *q, const tiga_view *k, const tiga_view *v,
                                const tiga_view *y, const float *lse, const tiga_view *dy, float scale,
                                const tiga_view *dq, const tiga_view *dk, const tiga_view *dv, void *ws,
                                size_t ws_bytes, void *stream) {
    EntryScope scope;
    const char *what = "cross attention backward";
    if (int rc = check_cross(given)) return rc;
    if (int rc = check_scale(what, scale)) return rc;
    tiga_cross some = *given;
    if (some.heads == 0) {  // source heads that nothing reads: gradients of 0, as without destinations
        some.heads = some.kv_heads;
        some.num_dst = 0;
    }
    const tiga_cross *const rel = &some;
    const bool rows = rel->num_dst > 0, srcs = rel->num_src > 0;
    if (rel->batch == 0 || rel->heads == 0 || (!rows && !srcs)) return TIGA_OK;
    const tiga_view none{};
    if (rows) {
        if (int rc = check_view(what, "q", q, false, 0, 0, 0)) return rc;
        if (int rc = check_view(what, "y", y, false, 0, 0, 0)) return rc;
        if (int rc = check_view(what, "dy", dy, false, 0, 0, 0)) return rc;
        if (!lse || (reinterpret_cast<uintptr_t>(lse) & 3u)) return fail(TIGA_EINVAL, "%s: lse missing or misaligned", what);
        if (dq)
            if (int rc = check_view(what, "dq", dq, true, rel->batch, rel->heads, rel->num_dst)) return rc;
    }
    if (srcs) {
        if (int rc = check_view(what, "k", k, false, 0, 0, 0)) return rc;
        if (int rc = check_view(what, "v", v, false, 0, 0, 0)) return rc;
        if (int rc = check_rows(what, "k", k)) return rc;
        if (int rc = check_rows(what, "v", v)) return rc;
        if (dk)
            if (int rc = check_view(what, "dk", dk, true, rel->batch, rel->kv_heads, rel->num_src)) return rc;
        if (dv)
            if (int rc = check_view(what, "dv", dv, true, rel->batch, rel->kv_heads, rel->num_src)) return rc;
    }
    if (int rc = check_ws(what, ws, ws_bytes, relattn::cross_bwd_ws_bytes(*rel))) return rc;
    return relattn::cross_backward(*rel, rows ? *q : none, srcs ? *k : none, srcs ? *v : none, rows ? *y : none, lse,
                                   rows ? *dy : none, scale, rows && dq ? *dq : none, srcs && dk ? *dk : none,
                                   srcs && dv ? *dv : none, ws, static_cast<hipStream_t>(stream));
}

int tiga_cache_validate(const tiga_cache *cache, int64_t num_dst, const int32_t *dst_ptr, void *stream) {
    EntryScope scope;
    const char *what = "cache validation";
    if (int rc = check_cache(what, cache)) return rc;
    if (int rc = check_packed(what, num_dst, 1)) return rc;
    if (cache->batch == 0 || cache->kv_heads == 0) return TIGA_OK;  // as the calls, which read nothing then
    if (int rc = check_cache_data(what, cache, dst_ptr)) return rc;
    const size_t nb = cache->batch, cells = nb * cache->table_width;
    std::vector<int32_t> ptr, len, table;
    try {
        ptr.resize(nb + 1);
        len.resize(nb);
        table.resize(cells);
    } catch (const std::bad_alloc &) {
        return fail(TIGA_EDEVICE, "%s: no host memory for %zu table entries", what, cells);
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    int rc = check_hip(hipMemcpyAsync(ptr.data(), dst_ptr, 4 * (nb + 1), hipMemcpyDeviceToHost, s), what);
    if (!rc && nb) rc = check_hip(hipMemcpyAsync(len.data(), cache->length, 4 * nb, hipMemcpyDeviceToHost, s), what);
    if (!rc && cells) rc = check_hip(hipMemcpyAsync(table.data(), cache->table, 4 * cells, hipMemcpyDeviceToHost, s), what);
    // also after a failed copy: the ones before it write into the vectors
    const int rs = check_hip(hipStreamSynchronize(s), what);
    if (rc || rs) return rc ? rc : rs;
    if (ptr[0] < 0) return fail(TIGA_EGRAPH, "dst_ptr[0] = %d is negative", ptr[0]);
    for (size_t b = 0; b < nb; ++b) {
        if (ptr[b + 1] < ptr[b]) return fail(TIGA_EGRAPH, "dst_ptr decreases at sequence %zu", b);
        if (ptr[b + 1] > num_dst)
            return fail(TIGA_EGRAPH, "dst_ptr[%zu] = %d passes num_dst = %lld", b + 1, ptr[b + 1], (long long)num_dst);
        if (len[b] < ptr[b + 1] - ptr[b])
            return fail(TIGA_EGRAPH, "sequence %zu of length %d has %d new tokens", b, len[b], ptr[b + 1] - ptr[b]);
        const int64_t need = ceil_div(len[b], cache->page_size);
        if (need > cache->table_width)
            return fail(TIGA_EGRAPH, "sequence %zu of length %d needs %lld pages, the table holds %d", b, len[b],
                        (long long)need, cache->table_width);
        for (int64_t e = 0; e < need; ++e) {
            const int32_t id = table[b * cache->table_width + e];
            if (id < 0 || id >= cache->num_pages)
                return fail(TIGA_EGRAPH, "page %lld of sequence %zu is %d, outside [0, %lld)", (long long)e, b, id,
                            (long long)cache->num_pages);
        }
    }
    return TIGA_OK;
}

size_t tiga_mp_attention_paged_fwd_workspace(const tiga_cache *cache, int64_t num_dst, int32_t heads) {
    clear_error();  // no EntryScope: armed kernel events are for the call that follows
    const char *what = "paged attention";
    if (check_cache(what, cache) || check_heads(what, heads, cache->kv_heads, cache->width, cache->dtype) ||
        check_packed(what, num_dst, heads))
        return 0;
    return relattn::paged_fwd_ws_bytes(*cache, num_dst, heads);
}

int tiga_mp_attention_paged_fwd(const tiga_cache *cache, int64_t num_dst, const int32_t *dst_ptr, int32_t heads,
                                const tiga_view *q, float scale, const tiga_view *y, float *lse, void *ws,
                                size_t ws_bytes, void *stream) {
    EntryScope scope;
    const char *what = "paged attention";
    if (int rc = check_cache(what, cache)) return rc;
    if (int rc = check_heads(what, heads, cache->kv_heads, cache->width, cache->dtype)) return rc;
    if (int rc = check_packed(what, num_dst, heads)) return rc;
    if (int rc = check_scale(what, scale)) return rc;
    if (cache->batch == 0 || heads == 0 || num_dst == 0) return TIGA_OK;
    if (int rc = check_cache_data(what, cache, dst_ptr)) return rc;
    if (int rc = check_view(what, "q", q, false, 0, 0, 0)) return rc;
    if (int rc = check_view(what, "y", y, true, 1, heads, num_dst)) return rc;
    if (q->data == y->data && ((heads > 1 && q->head != y->head) || (num_dst > 1 && q->row != y->row)))
        return fail(TIGA_EINVAL, "%s: y in the place of q needs its strides", what);
    if (reinterpret_cast<uintptr_t>(lse) & 3u) return fail(TIGA_EINVAL, "%s: lse misaligned", what);
    if (int rc = check_ws(what, ws, ws_bytes, relattn::paged_fwd_ws_bytes(*cache, num_dst, heads))) return rc;
    return relattn::paged_forward(*cache, num_dst, dst_ptr, heads, *q, scale, *y, lse, ws,
                                  static_cast<hipStream_t>(stream));
}

}  // extern "C"

// ------------------------------------------------------------------- rotary positions, cache append

namespace {

int check_rotary(const char *what, const tiga_rotary *rot, int32_t width) {
    if (!rot) return fail(TIGA_EINVAL, "%s: the rotation is required", what);
    if (!rot->freq || (reinterpret_cast<uintptr_t>(rot->freq) & 7u))
        return fail(TIGA_EINVAL, "%s: freq missing or misaligned", what);
    if (rot->rot < 2 || rot->rot % 2 || rot->rot > width)
        return fail(TIGA_EINVAL, "%s: rot = %d must be even, positive and at most the width %d", what, rot->rot, width);
    if (rot->pairs != TIGA_PAIRS_HALF && rot->pairs != TIGA_PAIRS_ADJACENT)
        return fail(TIGA_EINVAL, "%s: unknown pairs %d", what, rot->pairs);
    if (bad_float(rot->amplitude)) return fail(TIGA_EINVAL, "%s: the amplitude must be finite", what);
    return TIGA_OK;
}

int rotary_call(const char *what, const char *in, const char *out, int32_t batch, int32_t heads, int64_t rows,
                int32_t width, int dtype, const tiga_view *x, const int32_t *pos, int64_t pos_batch,
                const tiga_rotary *rot, const tiga_view *y, bool back, void *stream) {
    if (batch < 0 || heads < 0 || rows < 0 || width < 1) return fail(TIGA_EINVAL, "%s: bad size", what);
    if (dtype != TIGA_DT_F16 && dtype != TIGA_DT_BF16 && dtype != TIGA_DT_F32)
        return fail(TIGA_EINVAL, "%s: unknown dtype %d", what, dtype);
    if (width >= (1 << 16)) return fail(TIGA_EUNSUPPORTED, "%s: width %d (below 65536 supported)", what, width);
    if (static_cast<double>(batch) * heads * static_cast<double>(rows) >= 1099511627776.0)
        return fail(TIGA_EUNSUPPORTED, "%s: batch * heads * rows must be < 2^40", what);
    if (int rc = check_rotary(what, rot, width)) return rc;
    if (batch == 0 || heads == 0 || rows == 0) return TIGA_OK;
    const uintptr_t mask = dtype == TIGA_DT_F32 ? 3u : 1u;
    if (!x || !x->data || !y || !y->data) return fail(TIGA_EINVAL, "%s: %s and %s are required", what, in, out);
    if ((reinterpret_cast<uintptr_t>(x->data) | reinterpret_cast<uintptr_t>(y->data)) & mask)
        return fail(TIGA_EINVAL, "%s: %s or %s misaligned", what, in, out);
    if (x->batch < 0 || x->head < 0 || x->row < 0 || y->batch < 0 || y->head < 0 || y->row < 0 || pos_batch < 0)
        return fail(TIGA_EINVAL, "%s: negative stride", what);
    if ((batch > 1 && y->batch == 0) || (heads > 1 && y->head == 0) || (rows > 1 && y->row == 0))
        return fail(TIGA_EINVAL, "%s: the rows of %s overlap (a stride is 0)", what, out);
    if (x->data == y->data && ((batch > 1 && x->batch != y->batch) || (heads > 1 && x->head != y->head) ||
                               (rows > 1 && x->row != y->row)))
        return fail(TIGA_EINVAL, "%s: %s in the place of %s needs its strides", what, out, in);
    if (reinterpret_cast<uintptr_t>(pos) & 3u) return fail(TIGA_EINVAL, "%s: pos misaligned", what);
    return rotary::rotate(batch, heads, rows, width, dtype, *x, pos, pos_batch, *rot, back, *y,
                          static_cast<hipStream_t>(stream));
}

}  // namespace

extern "C" {

int tiga_rotary_frequencies(int32_t rot, double base, int scaling, double factor, double trained, double low,
                            double high, double *freq) {
    EntryScope scope;
    const char *what = "rotary frequencies";
    if (rot < 2 || rot % 2 || rot >= (1 << 16)) return fail(TIGA_EINVAL, "%s: rot = %d must be even, in [2, 65536)", what, rot);
    if (!freq) return fail(TIGA_EINVAL, "%s: freq is required", what);
    if (!(base > 0.0) || !std::isfinite(base)) return fail(TIGA_EINVAL, "%s: base must be finite and > 0", what);
    if (scaling < TIGA_ROTARY_PLAIN || scaling > TIGA_ROTARY_BANDS)
        return fail(TIGA_EINVAL, "%s: unknown scaling %d", what, scaling);
    if (scaling != TIGA_ROTARY_PLAIN && (!(factor > 0.0) || !std::isfinite(factor)))
        return fail(TIGA_EINVAL, "%s: factor must be finite and > 0", what);
    if (scaling == TIGA_ROTARY_BASE && rot < 4) return fail(TIGA_EINVAL, "%s: a stretched base needs rot >= 4", what);
    if (scaling == TIGA_ROTARY_BANDS && (!(trained > 0.0) || !std::isfinite(trained) || !(low < high) ||
                                         !std::isfinite(low) || !std::isfinite(high)))
        return fail(TIGA_EINVAL, "%s: bands need a trained length > 0 and low < high", what);
    if (scaling == TIGA_ROTARY_BASE) base *= std::pow(factor, static_cast<double>(rot) / (rot - 2));
    for (int i = 0; i < rot / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rot);
        if (scaling == TIGA_ROTARY_LINEAR) f /= factor;
        if (scaling == TIGA_ROTARY_BANDS) {
            double keep = (trained * f / 6.283185307179586477 - low) / (high - low);
            keep = keep < 0.0 ? 0.0 : (keep > 1.0 ? 1.0 : keep);
            f *= keep + (1.0 - keep) / factor;
        }
        freq[i] = f;
    }
    return TIGA_OK;
}

int tiga_mp_rotary_fwd(int32_t batch, int32_t heads, int64_t rows, int32_t width, int dtype, const tiga_view *x,
                       const int32_t *pos, int64_t pos_batch, const tiga_rotary *rot, const tiga_view *y, void *stream) {
    EntryScope scope;
    return rotary_call("rotary", "x", "y", batch, heads, rows, width, dtype, x, pos, pos_batch, rot, y, false, stream);
}

int tiga_mp_rotary_bwd(int32_t batch, int32_t heads, int64_t rows, int32_t width, int dtype, const tiga_view *dy,
                       const int32_t *pos, int64_t pos_batch, const tiga_rotary *rot, const tiga_view *dx, void *stream) {
    EntryScope scope;
    return rotary_call("rotary backward", "dy", "dx", batch, heads, rows, width, dtype, dy, pos, pos_batch, rot, dx, true,
                       stream);
}

int tiga_mp_cache_append(const tiga_cache *cache, int64_t num_dst, const int32_t *dst_ptr, const tiga_view *k,
                         const tiga_view *v, const tiga_rotary *rot, int32_t heads, const tiga_view *q,
                         const tiga_view *q_out, void *stream) {
    EntryScope scope;
    const char *what = "cache append";
    const bool with_q = q && q->data;
    if (int rc = check_cache(what, cache)) return rc;
    if (heads < 0) return fail(TIGA_EINVAL, "%s: negative number of heads", what);
    if (int rc = check_packed(what, num_dst, with_q && heads > cache->kv_heads ? heads : cache->kv_heads)) return rc;
    if (rot)
        if (int rc = check_rotary(what, rot, cache->width)) return rc;
    if (with_q && !rot) return fail(TIGA_EINVAL, "%s: q is only taken to be rotated", what);
    if (with_q && heads > 0 && cache->kv_heads == 0) return fail(TIGA_EINVAL, "%s: q for a cache without heads", what);
    if (cache->batch == 0 || cache->kv_heads == 0 || num_dst == 0) return TIGA_OK;
    if (int rc = check_cache_data(what, cache, dst_ptr)) return rc;
    if (int rc = check_view(what, "k", k, false, 0, 0, 0)) return rc;
    if (int rc = check_view(what, "v", v, false, 0, 0, 0)) return rc;
    const tiga_view none{};
    if (with_q) {
        if (int rc = check_view(what, "q", q, false, 0, 0, 0)) return rc;
        if (int rc = check_view(what, "q_out", q_out, true, 1, heads, num_dst)) return rc;
        if (q->data == q_out->data && ((heads > 1 && q->head != q_out->head) || (num_dst > 1 && q->row != q_out->row)))
            return fail(TIGA_EINVAL, "%s: q_out in the place of q needs its strides", what);
    }
    return rotary::append(*cache, num_dst, dst_ptr, *k, *v, rot ? *rot : tiga_rotary{}, heads, with_q ? *q : none,
                          with_q ? *q_out : none, static_cast<hipStream_t>(stream));
}

}  // extern "C"
