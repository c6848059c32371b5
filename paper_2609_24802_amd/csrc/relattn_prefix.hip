// Causal attention of new tokens over a paged cache of which groups of sequences share their first positions, in two parts of
// the forward kernels' work: the rows of all of a group's sequences over the shared positions, whose keys and values are read
// once and whose products have full tiles, and each sequence's rows over the positions behind.  They do not depend on each
// other, so one launch does both, the second part's blocks behind the first's, which are seldom as many as run at once: that
// part is short of parallel work and waits for its operands, the other is bound by reading keys.  Both leave normalized fp32
// states and lse, which a last launch joins,
//   y = (2^(l1 - m) y1 + 2^(l2 - m) y2) / (2^(l1 - m) + 2^(l2 - m)),  m = max(l1, l2),
// 8 (width + 1) bytes a row and head written and read.
//
// Measured (MI355X), kernel + merge + join in us: 64 single tokens behind 8192 shared positions and up to 1000 of their own, 32
// heads over 8 of width 128, bf16: 45 + 11.2 + 5.1, where reading what there is (121 MB) takes 25; each of the two parts by itself
// takes 26 to 27, of which 10 to start, find its pieces and end.  (Half of the blocks for either part, so that both run side by
// side from the start: 49 + 9.)  5 drafted tokens each of 24 sequences over four documents of up to 40,000
// positions, 16 heads over 2 of width 128, f16: 48.9 + 10.4 + 4.6 for 101 MB and 17 GFLOP (21); 4 single tokens behind 500
// positions, 16 heads over 4 of width 64: 8.1 + 4.4 + 2.2, latency.  What is above the floors is the time to fill and drain the
// device three times and, in the merge, dependent loads of the records of the parts (20 to 60 of an item) before their states.
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
// Blocks are multiples of 8, so that both passes' blocks know their XCD.  A narrow pass has two slots for each of them, not for
// each that the lengths leave work: a length past the table, or pointers that overlap, make more work than the host can know of.
template <class G>
Plan pass_plan(const tiga_cache &c, int64_t num_dst, int32_t heads, int64_t sequences) {
    const int64_t rows = num_dst * (heads / c.kv_heads);
    Plan p = plan_for<G>((rows / G::BM + sequences) * c.kv_heads, rows / G::BM * c.kv_heads,
                         static_cast<int64_t>(c.table_width) * c.page_size, false);
    p.blocks = ceil_div(p.blocks, kXcds) * kXcds;
    if (kNarrow<G> && p.slots) p.slots = 2 * p.blocks;
    return p;
}
int64_t some_groups(const tiga_prefix &p, int64_t num_dst) { return num_dst < p.groups ? num_dst : p.groups; }

// The states of both parts.
struct States {
    float *shared, *shared_lse2, *behind, *behind_lse2;  // [heads, num_dst, width], [heads, num_dst]
};

// The renumbering of xcd_block() for a part of a launch.
__device__ __forceinline__ int xcd_block_of(unsigned b, unsigned blocks) {  // multiples of 8
    return static_cast<int>(b % kXcds * (blocks / kXcds) + b / kXcds);
}

template <class T, int D, bool THIN, Relation REL>
__device__ __forceinline__ void pieces(const Args<REL> &a, unsigned block, unsigned blocks, uint8_t *l0, uint8_t *l1, uint8_t *l2,
                                       uint8_t *l3, int (*wild)[kWaves], float (*ml)[kWaves][Thin<D>::BM]) {
    if constexpr (THIN) {
        constexpr int WAVE = kThinWave<D>;
        thin_pieces<T, D, REL>(a, xcd_block_of(block, blocks), static_cast<int>(blocks),
                               [&](int i) { return (i < 2 ? l0 : l1) + i % 2 * WAVE; }, [&](int i) { return (i < 2 ? l2 : l3) + i % 2 * WAVE; }, ml);
    } else {
        wide_pieces<T, D, REL>(a, block, blocks, l0, l1, l2, l3, wild);
    }
}
template <class T, int D, bool SHARED_THIN, bool BEHIND_THIN>
__global__ __launch_bounds__(kThreads, 2) void prefix_kernel(Args<kShared> s, Args<kBehind> b, unsigned shared, unsigned behind) {
    static_assert(Geo<D>::TILE == 2 * kThinWave<D>, "two wavefronts' steps are a tile");
    constexpr int TILE = Geo<D>::TILE;
    __shared__ __attribute__((aligned(1024))) uint8_t l0[TILE], l1[TILE], l2[TILE], l3[TILE];
    __shared__ int wild[2][kWaves];
    __shared__ float ml[2][kWaves][Thin<D>::BM];
    if (blockIdx.x < shared) pieces<T, D, SHARED_THIN, kShared>(s, blockIdx.x, shared, l0, l1, l2, l3, wild, ml);
    else pieces<T, D, BEHIND_THIN, kBehind>(b, blockIdx.x - shared, behind, l0, l1, l2, l3, wild, ml);
}

// Joins the parts of cut items, of shared positions in the first `shared` blocks.  blocks: of the narrow part's pieces.
template <class T, int D, bool SHARED_THIN, bool BEHIND_THIN>
__global__ __launch_bounds__(kThreads) void prefix_merge_kernel(Args<kShared> s, Args<kBehind> b, unsigned shared, unsigned shared_blocks,
                                                                unsigned behind_blocks) {
    __shared__ f4 so[kWaves][kWave];
    __shared__ float sl[kWaves][kWave];
    if (blockIdx.x < shared) {
        if constexpr (SHARED_THIN) {
            thin_merge<T, D, kShared>(s, static_cast<int>(blockIdx.x / kWaves), static_cast<int>(blockIdx.x % kWaves),
                                      static_cast<int>(shared_blocks), so, sl);
        } else {
            constexpr unsigned PER = Geo<D>::BM / kSharedRows<Geo<D>>;
            shared_merge<T, Geo<D>>(s, static_cast<int>(blockIdx.x / PER), static_cast<int>(blockIdx.x % PER), so, sl);
        }
    } else {
        const unsigned id = blockIdx.x - shared;
        if constexpr (BEHIND_THIN) {
            thin_merge<T, D, kBehind>(b, static_cast<int>(id / kWaves), static_cast<int>(id % kWaves), static_cast<int>(behind_blocks), so, sl);
        } else {
            const int slot = nth_item(b, static_cast<int>(id / (Geo<D>::BM / 16)));
            if (slot >= 0) wide_merge<T, Geo<D>, kBehind>(b, slot, static_cast<int>(id % (Geo<D>::BM / 16)));
        }
    }
}

// A row and head by D / 4 lanes.  Rows before dst_ptr[0] and behind dst_ptr[batch] stay as they are.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void prefix_join_kernel(Args<kBehind> a, States st, Rows y, float *lse) {
    constexpr int L = D / 4;
    const Run rows = run_between(a.src.dst_ptr, 0, a.src.batch, a.src.num_dst);
    const int heads = a.kv_heads * static_cast<int>(a.group.d), w = static_cast<int>(threadIdx.x) % L * 4;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * (kThreads / L) + threadIdx.x / L;; i += static_cast<int64_t>(gridDim.x) * (kThreads / L)) {
        const int64_t token = i / heads;
        if (token >= rows.count) return;
        const int head = static_cast<int>(i - token * heads);
        const int64_t row = rows.first + token, at = head * static_cast<int64_t>(a.src.num_dst) + row;
        const float l1 = st.shared_lse2[at], l2 = st.behind_lse2[at];
        f4 o1{0.0f, 0.0f, 0.0f, 0.0f};
        if (l1 != -__builtin_inff()) o1 = *reinterpret_cast<const f4 *>(st.shared + at * D + w);  // there may be none
        const f4 o2 = *reinterpret_cast<const f4 *>(st.behind + at * D + w);
        const float m = fmaxf(l1, l2), ref = m == -__builtin_inff() ? 0.0f : m;
        const float f1 = __builtin_amdgcn_exp2f(l1 - ref), f2 = __builtin_amdgcn_exp2f(l2 - ref), mass = f1 + f2;
        const f4 v = (o1 * f1 + o2 * f2) * (mass == 0.0f ? 0.0f : 1.0f / mass);
        put<T>(const_cast<uint16_t *>(y.p) + head * y.head + row * y.row + w, v);
        if (lse && w == 0) lse[at] = (ref + __log2f(mass)) * kLn2;
    }
}

constexpr int64_t kMostJoins = 1 << 20;  // blocks

struct Layout {
    States states;
    char *shared_parts, *behind_parts;
    size_t bytes;
};
Layout layout(const tiga_cache &c, int64_t num_dst, int32_t heads, size_t shared, size_t behind, void *ws) {
    Layout l;
    Carve w(ws);
    const size_t rows = static_cast<size_t>(num_dst) * heads;
    l.states.shared = w.take<float>(rows * c.width);
    l.states.shared_lse2 = w.take<float>(rows);
    l.states.behind = w.take<float>(rows * c.width);
    l.states.behind_lse2 = w.take<float>(rows);
    l.shared_parts = w.take<char>(shared);
    l.behind_parts = w.take<char>(behind);
    l.bytes = w.bytes();
    return l;
}
size_t part_bytes(const tiga_cache &c, int64_t num_dst, int32_t heads, int64_t sequences) {
    return ws_bytes(c.dtype, c.width, num_dst * heads, static_cast<int64_t>(c.table_width) * c.page_size,
                    [&](auto g) { return pass_plan<decltype(g)>(c, num_dst, heads, sequences).slots; });
}

template <class T, class GS, class GB>
int launch(const Plan &ps, const Plan &pb, Args<kShared> s, Args<kBehind> b, const Layout &l, const tiga_view &y, float *lse,
           hipStream_t stream) {
    constexpr int D = GS::CPR * 8;
    constexpr bool ST = kNarrow<GS>, BT = kNarrow<GB>;
    auto parts = [](auto &a, const Parts &w, int64_t slots) {
        a.part = w.part;
        a.rec = w.rec;
        a.slots = static_cast<int>(slots);
    };
    if (ps.slots) parts(s, carve<GS>(l.shared_parts, ps.slots), ps.slots);
    if (pb.slots) parts(b, carve<GB>(l.behind_parts, pb.slots), pb.slots);
    const unsigned shared = static_cast<unsigned>(ps.blocks), behind = static_cast<unsigned>(pb.blocks);
    prof_before(stream);
    hipLaunchKernelGGL((prefix_kernel<T, D, ST, BT>), dim3(shared + behind), dim3(kThreads), 0, stream, s, b, shared, behind);
    prof_after(stream);
    if (int rc = check_launch("prefix attention")) return rc;
    // cut items: at most as many as blocks (narrow), or items, or slots (wide)
    auto cut = [](const Plan &p) { return static_cast<unsigned>(p.items < p.slots ? p.items : p.slots); };
    const unsigned ms = ps.slots ? (ST ? shared * kWaves : cut(ps) * (Geo<D>::BM / kSharedRows<Geo<D>>)) : 0;
    const unsigned mb = pb.slots ? (BT ? behind * kWaves : cut(pb) * (Geo<D>::BM / 16)) : 0;
    if (ms + mb) {
        hipLaunchKernelGGL((prefix_merge_kernel<T, D, ST, BT>), dim3(ms + mb), dim3(kThreads), 0, stream, s, b, ms, shared, behind);
        if (int rc = check_launch("prefix attention merge")) return rc;
    }
    // a grid counts its threads in 32 bits (and wraps around without an error): more rows than that go in turns
    const int64_t rows = static_cast<int64_t>(b.src.num_dst) * b.kv_heads * b.group.d, joins = ceil_div(rows, kThreads / (D / 4));
    hipLaunchKernelGGL((prefix_join_kernel<T, D>), dim3(static_cast<unsigned>(joins < kMostJoins ? joins : kMostJoins)), dim3(kThreads), 0,
                       stream, b, l.states, rows_of(y), lse);
    return check_launch("prefix attention join");
}

}  // namespace

size_t prefix_fwd_ws_bytes(const tiga_cache &c, const tiga_prefix &p, int64_t num_dst, int32_t heads) {
    if (c.kv_heads == 0 || num_dst == 0) return 256;
    return layout(c, num_dst, heads, part_bytes(c, num_dst, heads, some_groups(p, num_dst)),
                  part_bytes(c, num_dst, heads, some_sequences(c, num_dst)), nullptr).bytes;
}

int prefix_forward(const tiga_cache &c, const tiga_prefix &p, int64_t num_dst, const int32_t *dst_ptr, int32_t heads,
                   const tiga_view &q, float scale, const tiga_view &y, float *lse, void *ws, hipStream_t stream) {
    if (p.groups == 0) return paged_forward(c, num_dst, dst_ptr, heads, q, scale, y, lse, ws, stream);
    const int64_t groups = some_groups(p, num_dst), sequences = some_sequences(c, num_dst);
    const Layout l = layout(c, num_dst, heads, part_bytes(c, num_dst, heads, groups), part_bytes(c, num_dst, heads, sequences), ws);
    const Pages pages = pages_of(c, num_dst, dst_ptr);
    const Groups all{p.ptr, p.len, p.groups, c.batch, pages.shift < 7 ? 7 : pages.shift};
    auto set = [&](auto &a) {
        a.q = rows_of(q);
        a.q.batch = 0;  // one packed axis
        a.lse_head = num_dst;
        a.c = scale * kLog2e;
        a.kv_heads = c.kv_heads;
        a.group = divider(heads / c.kv_heads);
        static_cast<Pages &>(a.src) = pages;
        a.src.groups = all;
    };
    Args<kShared> a{};
    set(a);
    a.src.batch = p.groups;
    a.src.state = l.states.shared;
    a.src.lse2 = l.states.shared_lse2;
    Args<kBehind> b{};
    set(b);
    b.src.state = l.states.behind;
    b.src.lse2 = l.states.behind_lse2;
    b.src.shared_lse2 = l.states.shared_lse2;
    return by_type(c.dtype, c.width, thin_for(c, num_dst, heads, groups), [&](auto t, auto gs) {
        typedef decltype(t) T;
        typedef decltype(gs) GS;
        const Plan ps = pass_plan<GS>(c, num_dst, heads, groups);
        auto with = [&](auto gb) {
            typedef decltype(gb) GB;
            return launch<T, GS, GB>(ps, pass_plan<GB>(c, num_dst, heads, sequences), a, b, l, y, lse, stream);
        };
        constexpr int D = GS::CPR * 8;
        return thin_for(c, num_dst, heads, sequences) ? with(Thin<D>{}) : with(Geo<D>{});
    });
}

}  // namespace relattn
}  // namespace tiga
