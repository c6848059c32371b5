// Causal attention within packed sequences, forward: plan and launch.
#include "relattn_fwd.hpp"

namespace tiga {
namespace relattn {

namespace {

int64_t some_sequences(const tiga_packed &rel) { return rel.num_rows < rel.batch ? rel.num_rows : rel.batch; }
bool packed_thin(const tiga_packed &rel) {
    return rel.num_rows * (rel.heads / rel.kv_heads) <= kThinRows * some_sequences(rel);
}
template <class G>
Plan packed_plan(const tiga_packed &rel) {
    const int64_t rows = rel.num_rows * (rel.heads / rel.kv_heads);
    Plan p = plan_for<G>((rows / G::BM + some_sequences(rel)) * rel.kv_heads, rows / G::BM * rel.kv_heads, rel.num_rows, false);
    if (p.blocks < 1) p.blocks = kXcds;  // no sequences: all rows are cleared
    return p;
}

}  // namespace

size_t packed_fwd_ws_bytes(const tiga_packed &rel) {
    if (rel.kv_heads == 0 || rel.num_rows == 0) return 256;
    return ws_bytes(rel.dtype, rel.width, rel.num_rows * rel.heads, rel.num_rows,
                    [&](auto g) { return packed_plan<decltype(g)>(rel).slots; });
}

int packed_forward(const tiga_packed &rel, const tiga_view &q, const tiga_view &k, const tiga_view &v, float scale,
                   const tiga_view &y, float *lse, void *ws, hipStream_t stream) {
    Args<kPacked> a{};
    a.q = rows_of(q);
    a.y = rows_of(y);
    a.q.batch = a.y.batch = 0;  // one packed axis
    a.lse = lse;
    a.lse_head = rel.num_rows;
    a.c = scale * kLog2e;
    a.kv_heads = rel.kv_heads;
    a.group = divider(rel.heads / rel.kv_heads);
    a.src = Packed{rows_of(k), rows_of(v), rel.ptr, rel.batch, static_cast<int32_t>(rel.num_rows)};
    return by_type(rel.dtype, rel.width, packed_thin(rel), [&](auto t, auto g) {
        return run<decltype(t), decltype(g), kPacked>(packed_plan<decltype(g)>(rel), a, ws, stream);
    });
}

}  // namespace relattn
}  // namespace tiga
