// Causal attention within packed sequences, forward: plan and launch.
//
// The weights enter the product with the values in the input type, as in the other forward calls: against 64 bits y is 1.1 to 1.45
// times as far off as one that is formed in fp32 and rounded once.
//
// Measured (MI355X): 17 ragged prompts of 16,384 tokens in all, 32 heads over 8 of width 128, bf16: 295 to 302 us, 0.85 to 0.87
// PFLOP/s (matrix cores busy 38 % of the time, in long sequences 56: some 4,200 pieces that each start from nothing, and 4.2
// vector instructions a matrix one, there 3.5); 16,384 tokens in three sequences, 16 heads over 4 of width 128, bf16: 715 us, 1.16 (a large library product 1.24);
// 61 sequences of 8001 tokens in all, 16 heads of width 64, f16: 43 us; three of 37, 8.6, latency.
#include "relattn_fwd.hpp"

namespace tiga {
namespace relattn {

namespace {

// Narrow tiles by the mean length, all that the host knows.  A long sequence among very many short ones goes narrow with them
// and has its keys read again for every 16 rows: one of 14,000 tokens and a thousand of one token, 16 heads over 4 of 128, take
// 853 us, the long one by itself 746.
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

// Sequences of 512 tokens or more on average are worked on in a planned order, longest items first and cut where they are long,
// as long as the order matters: causal items take from nothing to twice the mean, and with few rounds of them on the device the
// last round is left to the long ones.  The launch that plans takes 5 us and the join 5 to 15.  us dealt (as other relations are)
// and planned, width 128: 16 heads over 2 source heads, 4000 tokens 118 and 103; 8 over 8, 8000 tokens 190 and 163; 16, 8 x
// 2000 tokens 175 and 154; 32 over 8, 17 prompts of 16,384 in all 307 and 298; width 64, 8 over 2, 2000 tokens 47 and 32.  Many
// tiles of one sequence fill the device however they come (32 over 4, 4000 tokens 134 and 140; 16 over 4, 16,000 899 and 911), and
// so do very many at width 64; items of shorter sequences are too alike for an order to pay (64 x 256 tokens, 16 heads 64 and 72).
constexpr int64_t kPlannedMean = 512, kPlannedTiles = 8;  // key tiles of a part, at least
constexpr int64_t kPlannedOne = 3;                        // tiles to a CU: of one sequence, and of more
template <int D>
constexpr int64_t kPlannedMost = D == 64 ? 8 : 32;
bool planned(const tiga_packed &rel) {
    const int64_t most = rel.batch < 2 ? kPlannedOne : rel.width == 64 ? kPlannedMost<64> : kPlannedMost<128>;
    return rel.batch > 0 && rel.batch <= kWave && rel.num_rows >= kPlannedMean * rel.batch &&
           rel.num_rows * rel.heads <= most * device_cus() * kTileRows;
}
struct Planning {
    Pieces by_rows;
    float *part;
    int64_t cut;  // pieces of cut items, at most
    size_t bytes;
};
template <int D>
Planning planning(const tiga_packed &rel, void *ws) {
    const int64_t group = rel.kv_heads ? rel.heads / rel.kv_heads : 1;
    Planning p;
    const int resident = 2 * device_cus();
    p.cut = 2 * static_cast<int64_t>(resident);
    p.by_rows.resident = resident;
    p.by_rows.quarters = 5;
    p.by_rows.mult = static_cast<int32_t>(group < 1 ? 1 : group);
    p.by_rows.least = static_cast<int32_t>(ceil_div(kPlannedTiles * Geo<D>::BN * group, kTileRows));
    p.by_rows.places = static_cast<int32_t>(most_items(rel, group) / rel.kv_heads + ceil_div(p.cut, rel.kv_heads));
    Carve c(ws);
    // for any number of source heads, and whether this call is planned or not: a workspace holds every smaller call
    const size_t some = rel.num_rows >= kPlannedMean ? 1 : 0;
    const size_t rows = static_cast<size_t>(rel.num_rows) * rel.heads, most = static_cast<size_t>(kPlannedMost<D>) * device_cus() * kTileRows;
    p.by_rows.table = c.take<int4>(some * 2 * ((rows < most ? rows : most) / kTileRows + kWave + p.cut + 1));
    p.part = c.take<float>(some * (p.cut + rel.heads) * slot_floats<kTileRows, D>());
    p.bytes = c.bytes();
    return p;
}

template <class T, int D>
int run_planned(const tiga_packed &rel, const Args<kPacked> &given, void *ws, hipStream_t stream) {
    const Planning p = planning<D>(rel, ws);
    if (int rc = plan_pieces(rel, p.by_rows, p.by_rows, 1, stream)) return rc;
    Args<kPlanned> a{};
    static_cast<Packed &>(a.src) = given.src;
    a.src.table = p.by_rows.table;
    a.q = given.q;
    a.y = given.y;
    a.lse = given.lse;
    a.lse_head = given.lse_head;
    a.c = given.c;
    a.kv_heads = given.kv_heads;
    a.group = given.group;
    a.part = p.part;
    prof_before(stream);
    hipLaunchKernelGGL((wide_kernel<T, D, kPlanned>), dim3(static_cast<unsigned>(p.by_rows.places * rel.kv_heads)), dim3(kThreads), 0, stream, a);
    prof_after(stream);
    if (int rc = check_launch("packed attention")) return rc;
    const int64_t cut = ceil_div(p.cut, rel.kv_heads) * rel.kv_heads;  // whole places, so that parts of every head are seen
    hipLaunchKernelGGL((planned_merge_kernel<T, Geo<D>>), dim3(static_cast<unsigned>(cut), 4), dim3(kThreads), 0,
                       stream, a);
    return check_launch("packed attention merge");
}

}  // namespace

size_t packed_fwd_ws_bytes(const tiga_packed &rel) {
    if (rel.kv_heads == 0 || rel.num_rows == 0 || rel.heads == 0) return 256;
    const size_t dealt = ws_bytes(rel.dtype, rel.width, rel.num_rows * rel.heads, rel.num_rows,
                                  [&](auto g) { return packed_plan<decltype(g)>(rel).slots; });
    const size_t in_order = rel.width == 64 ? planning<64>(rel, nullptr).bytes : planning<128>(rel, nullptr).bytes;
    return dealt > in_order ? dealt : in_order;
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
    const bool thin = packed_thin(rel);
    return by_type(rel.dtype, rel.width, thin, [&](auto t, auto g) {
        typedef decltype(t) T;
        typedef decltype(g) G;
        if constexpr (!kNarrow<G>)
            if (planned(rel)) return run_planned<T, G::CPR * 8>(rel, a, ws, stream);
        return run<T, G, kPacked>(packed_plan<G>(rel), a, ws, stream);
    });
}

}  // namespace relattn
}  // namespace tiga
