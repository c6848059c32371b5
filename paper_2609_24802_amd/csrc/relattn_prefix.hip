// Causal attention of new tokens over a paged cache of which groups of sequences share their first positions, in two passes of
// the forward kernels: the rows of all of a group's sequences over the shared positions, whose keys and values are read once
// and whose products have full tiles, and each sequence's rows over the positions behind, starting from what the first pass
// left of them (normalized accumulators and lse in fp32, heads * rows * (width + 1) * 4 bytes written and read).
#include "relattn_fwd.hpp"

namespace tiga {
namespace relattn {

namespace {

int64_t some_sequences(const tiga_cache &c, int64_t num_dst) { return num_dst < c.batch ? num_dst : c.batch; }
// The tile shape of a pass, by the mean number of rows of a group or a sequence.
bool thin_for(const tiga_cache &c, int64_t num_dst, int32_t heads, int64_t sequences) {
    if (c.page_size < 8) return true;  // the wide tiles load 8 rows of a page at a time
    return num_dst * (heads / c.kv_heads) <= kThinRows * sequences;
}
template <class G>
Plan pass_plan(const tiga_cache &c, int64_t num_dst, int32_t heads, int64_t sequences) {
    const int64_t rows = num_dst * (heads / c.kv_heads);
    return plan_for<G>((rows / G::BM + sequences) * c.kv_heads, rows / G::BM * c.kv_heads,
                       static_cast<int64_t>(c.table_width) * c.page_size, false);
}
int64_t some_groups(const tiga_prefix &p, int64_t num_dst) { return num_dst < p.groups ? num_dst : p.groups; }

struct Layout {
    int32_t *skip;
    float *state, *lse2;
    char *parts;
    size_t bytes;
};
Layout layout(const tiga_cache &c, int64_t num_dst, int32_t heads, size_t parts, void *ws) {
    Layout l;
    Carve w(ws);
    l.skip = w.take<int32_t>(c.batch);
    l.state = w.take<float>(static_cast<size_t>(num_dst) * heads * c.width);
    l.lse2 = w.take<float>(static_cast<size_t>(num_dst) * heads);
    l.parts = w.take<char>(parts);
    l.bytes = w.bytes();
    return l;
}

}  // namespace

size_t prefix_fwd_ws_bytes(const tiga_cache &c, const tiga_prefix &p, int64_t num_dst, int32_t heads) {
    if (c.kv_heads == 0 || num_dst == 0) return 256;
    const int64_t positions = static_cast<int64_t>(c.table_width) * c.page_size;
    auto parts = [&](int64_t sequences) {
        return ws_bytes(c.dtype, c.width, num_dst * heads, positions,
                        [&](auto g) { return pass_plan<decltype(g)>(c, num_dst, heads, sequences).slots; });
    };
    const size_t shared = parts(some_groups(p, num_dst)), behind = parts(some_sequences(c, num_dst));
    return layout(c, num_dst, heads, shared > behind ? shared : behind, nullptr).bytes;
}

int prefix_forward(const tiga_cache &c, const tiga_prefix &p, int64_t num_dst, const int32_t *dst_ptr, int32_t heads,
                   const tiga_view &q, float scale, const tiga_view &y, float *lse, void *ws, hipStream_t stream) {
    if (p.groups == 0) return paged_forward(c, num_dst, dst_ptr, heads, q, scale, y, lse, ws, stream);
    const Layout l = layout(c, num_dst, heads, 0, ws);
    const Pages pages = pages_of(c, num_dst, dst_ptr);
    Args<kShared> a{};
    a.q = rows_of(q);
    a.q.batch = 0;  // one packed axis
    a.lse_head = num_dst;
    a.c = scale * kLog2e;
    a.kv_heads = c.kv_heads;
    a.group = divider(heads / c.kv_heads);
    static_cast<Pages &>(a.src) = pages;
    a.src.batch = p.groups;
    a.src.group_ptr = p.ptr;
    a.src.group_len = p.len;
    a.src.sequences = c.batch;
    a.src.whole = pages.shift < 7 ? 7 : pages.shift;
    a.src.skip = l.skip;
    a.src.state = l.state;
    a.src.lse2 = l.lse2;
    const int64_t groups = some_groups(p, num_dst), sequences = some_sequences(c, num_dst);
    int rc = by_type(c.dtype, c.width, thin_for(c, num_dst, heads, groups), [&](auto t, auto g) {
        return run<decltype(t), decltype(g), kShared>(pass_plan<decltype(g)>(c, num_dst, heads, groups), a, l.parts, stream);
    });
    if (rc) return rc;
    Args<kBehind> b{};
    b.q = a.q;
    b.y = rows_of(y);
    b.y.batch = 0;
    b.lse = lse;
    b.lse_head = a.lse_head;
    b.c = a.c;
    b.kv_heads = a.kv_heads;
    b.group = a.group;
    static_cast<Pages &>(b.src) = pages;
    b.src.skip = l.skip;
    b.src.state = l.state;
    b.src.lse2 = l.lse2;
    return by_type(c.dtype, c.width, thin_for(c, num_dst, heads, sequences), [&](auto t, auto g) {
        return run<decltype(t), decltype(g), kBehind>(pass_plan<decltype(g)>(c, num_dst, heads, sequences), b, l.parts, stream);
    });
}

}  // namespace relattn
}  // namespace tiga
