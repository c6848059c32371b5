// Cross attention over strided sources and causal attention of new tokens over a paged cache, forward: plans and launches.
#include "relattn_fwd.hpp"

namespace tiga {
namespace relattn {

namespace {

bool cross_thin(const tiga_cross &rel) { return rel.num_dst * (rel.heads / rel.kv_heads) <= kThinRows; }
template <class G>
Plan cross_plan(const tiga_cross &rel) {
    const int64_t rows = rel.num_dst * (rel.heads / rel.kv_heads);
    const int64_t items = ceil_div(rows, G::BM) * rel.batch * rel.kv_heads;
    return plan_for<G>(items, items, rel.num_src, rel.src_len == nullptr);
}

// sequences with new tokens, at most
int64_t some_sequences(const tiga_cache &c, int64_t num_dst) { return num_dst < c.batch ? num_dst : c.batch; }
bool paged_thin(const tiga_cache &c, int64_t num_dst, int32_t heads) {
    if (c.page_size < 8) return true;  // the wide tiles load 8 rows of a page at a time
    return num_dst * (heads / c.kv_heads) <= kThinRows * some_sequences(c, num_dst);
}
template <class G>
Plan paged_plan(const tiga_cache &c, int64_t num_dst, int32_t heads) {
    const int64_t rows = num_dst * (heads / c.kv_heads);
    return plan_for<G>((rows / G::BM + some_sequences(c, num_dst)) * c.kv_heads, rows / G::BM * c.kv_heads,
                       static_cast<int64_t>(c.table_width) * c.page_size, false);
}

}  // namespace

size_t cross_fwd_ws_bytes(const tiga_cross &rel) {
    if (rel.kv_heads == 0) return 256;
    return ws_bytes(rel.dtype, rel.width, rel.num_dst * rel.heads, rel.num_src,
                    [&](auto g) { return cross_plan<decltype(g)>(rel).slots; });
}
size_t paged_fwd_ws_bytes(const tiga_cache &c, int64_t num_dst, int32_t heads) {
    if (c.kv_heads == 0 || num_dst == 0) return 256;
    return ws_bytes(c.dtype, c.width, num_dst * heads, static_cast<int64_t>(c.table_width) * c.page_size,
                    [&](auto g) { return paged_plan<decltype(g)>(c, num_dst, heads).slots; });
}

int cross_forward(const tiga_cross &rel, const tiga_view &q, const tiga_view &k, const tiga_view &v, float scale,
                  const tiga_view &y, float *lse, void *ws, hipStream_t stream) {
    Args<kStrided> a{};
    a.q = rows_of(q);
    a.y = rows_of(y);
    a.lse = lse;
    a.lse_head = rel.num_dst;
    a.lse_batch = rel.num_dst * rel.heads;
    a.c = scale * kLog2e;
    a.kv_heads = rel.kv_heads;
    a.group = divider(rel.heads / rel.kv_heads);
    a.src = Strided{rows_of(k), rows_of(v), rel.src_len, static_cast<int32_t>(rel.num_dst),
                    static_cast<int32_t>(rel.num_src), rel.batch};
    return by_type(rel.dtype, rel.width, cross_thin(rel), [&](auto t, auto g) {
        return run<decltype(t), decltype(g), kStrided>(cross_plan<decltype(g)>(rel), a, ws, stream);
    });
}

int paged_forward(const tiga_cache &cache, int64_t num_dst, const int32_t *dst_ptr, int32_t heads, const tiga_view &q,
                  float scale, const tiga_view &y, float *lse, void *ws, hipStream_t stream) {
    Args<kPaged> a{};
    a.q = rows_of(q);
    a.y = rows_of(y);
    a.q.batch = a.y.batch = 0;  // one packed axis
    a.lse = lse;
    a.lse_head = num_dst;
    a.c = scale * kLog2e;
    a.kv_heads = cache.kv_heads;
    a.group = divider(heads / cache.kv_heads);
    a.src = pages_of(cache, num_dst, dst_ptr);
    return by_type(cache.dtype, cache.width, paged_thin(cache, num_dst, heads), [&](auto t, auto g) {
        return run<decltype(t), decltype(g), kPaged>(paged_plan<decltype(g)>(cache, num_dst, heads), a, ws, stream);
    });
}

}  // namespace relattn
}  // namespace tiga
