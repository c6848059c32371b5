// Online-softmax reducer over rectangular relations, forward: the kernels of cross attention over strided sources, of causal
// attention of new tokens over a paged cache, and of causal attention within packed sequences.  With the reducer state of Section
// 5.2 (running maximum m, mass l, accumulator o; states combine by rescaling into the common maximum):
//   s_ij = scale * <q_i, k_j>,  y_i = sum_j exp(s_ij) v_j / sum_j exp(s_ij),  lse_i = log sum_j exp(s_ij).
//
// Rows.  The heads that share a source head are rows over the same keys, so a sequence's rows for one source head are
// (token, head of the group), `group` heads to a token; a tile holds BM of them.  An item is one (sequence, source
// head, row tile).
//
// Work.  An item's keys come in tiles of BN.  Where the items alone do not fill the device they are cut along the
// keys, the parts' states (o, m, l) go to the workspace in fp32, and a merge kernel joins the parts of an item in order:
//  - narrow tiles (few rows, bound by reading the keys): the key tiles of all items are laid end to end and every
//    block walks an equal run of them (Walk), whatever the sequences' lengths;
//  - wide tiles (many rows, bound by the matrix cores): items are cut into chunks of one number of key tiles, and chunks
//    of the same keys are neighbours (Deal), so that the row tiles of a head read them from one XCD's L2 at one time.
// Both are found from the lengths on the device, so a captured call follows lengths that change between replays.  The
// orders of all sums depend on the sizes, the lengths and the device's compute units alone.
//
// Measured (MI355X; ranges are of several runs): wide, 2 x 16 x 2048 rows over 8192 keys of width 128, bf16: 250 to 266 us,
// 1.03 to 1.10 PFLOP/s (a large library product reaches 1.2 to 1.4); a prompt of 8192 tokens, 16 heads: 292 to 303 us, 0.91
// to 0.94; bound by the matrix cores at the clock the load leaves (2.0 GHz, half their cycles busy) and the dependent chain
// of a tile, which the second wavefront of the SIMD covers.  Narrow, 64 single tokens over up to 8192 keys, 8 heads of 128:
// 142 to 145 us for 740 MB, 5.1 to 5.2 TB/s (a large copy moves 4.8); one token over 4001 keys: 8.2 to 8.8 us, latency
// (finding the run 2.7, two dependent loads 2.6, the join 1).
#pragma once

#include <type_traits>

#include "mfma16.hpp"
#include "packed_plan.hpp"
#include "relation.hpp"
#include "relattn.hpp"

namespace tiga {
namespace relattn {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
// Weights are formed against a reference point 2^kLift below the row's largest, and enter the value product in the input
// type.  binary16 has no normal numbers below 2^-14: a lift of 10 of its 15 bits above 1 keeps weights down to 2^-24 of the
// largest exact to u, which long contexts need beside a token that nearly all weight goes to and whose value says little.
// (Without it, a weight of e^-17 becomes 2^-24, 44% more.  Times are the same.)  kMassCap: the largest tile mass of a lane, and so weight,
// that keeps the point; alike weights at the lift make 32 of it.
template <class T>
constexpr float kLift = std::is_same<T, Half16>::value ? 10.0f : 0.0f;
template <class T>
constexpr float kMassCap = std::is_same<T, Half16>::value ? 49152.0f : 4096.0f;
constexpr int kLeastChunk = 4;       // key tiles of a part of a wide item, at least
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Strided sources, and the pages of a cache.
struct Strided {
    Rows k, v;
    const int32_t *len;
    int32_t num_dst, num_src, batch;
};
// What a call's rows read: a padded batch of other sequences, a cache's pages up to the row's position, their own
// sequence's rows of packed sequences up to themselves; and for sequences of which groups share their first positions, those
// (the rows of all of a group's sequences are one item's) and the pages behind them, whose results are joined afterwards.
// kPlanned: packed, the pieces in the order of a table.
enum Relation { kStrided, kPaged, kPacked, kShared, kBehind, kPlanned };
template <Relation REL>
constexpr bool kOwnRows = REL == kPacked || REL == kPlanned;
template <Relation REL>
constexpr bool kPages = REL == kPaged || REL == kShared || REL == kBehind;
template <Relation REL>
constexpr bool kHalf = REL == kShared || REL == kBehind;  // results are fp32 states
template <Relation REL>
constexpr bool kCausal = REL == kPaged || REL == kBehind || kOwnRows<REL>;
template <Relation REL>
struct SourceArgs {
    typedef Strided type;
};
template <>
struct SourceArgs<kPaged> {
    typedef Pages type;
};
template <>
struct SourceArgs<kPacked> {
    typedef Packed type;
};
template <>
struct SourceArgs<kPlanned> {
    typedef Planned type;
};
template <>
struct SourceArgs<kShared> {
    typedef Shared type;
};
template <>
struct SourceArgs<kBehind> {
    typedef Behind type;
};
template <Relation REL>
struct Args {
    typename SourceArgs<REL>::type src;
    Rows q, y;
    float *lse;
    int64_t lse_batch, lse_head;
    float c;  // scale * log2 e: scores are kept in the log2 domain
    int kv_heads;
    Divider group;  // rows to a token
    // partial states and what they are of; NULL: items are not cut
    float *part;
    int4 *rec;
    int slots;  // wide tiles: partial states there is room for, as many as blocks run at once
};

// What lies in the place of a page that the cache does not have: keys that give NaN to the rows that need them,
// values that give nothing to the others.
__device__ const uint32_t kNanRow[64] = {
    0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu,
    0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu,
    0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu,
    0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu,
    0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu,
    0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu,
    0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu,
    0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu};
__device__ const uint32_t kZeroRow[64] = {0};

// ------------------------------------------------------------------------------------------ work partition

// A sequence: its rows [0, rows) (token first + r / group), and the keys that row r sees.
struct Seq {
    int32_t first, rows;
    int64_t keys0;  // keys that token 0 sees; token t sees keys0 + t of a paged relation, keys0 of a strided one
};
template <Relation REL>
__device__ __forceinline__ Seq seq_of(const Args<REL> &a, int b) {
    if constexpr (REL == kPaged) {
        const Chunk ch = chunk_of(a.src, b);
        return Seq{ch.first, ch.count * static_cast<int32_t>(a.group.d), ch.pos0 + 1};
    } else if constexpr (kOwnRows<REL>) {
        const Run run = run_of(a.src, b);
        return Seq{run.first, run.count * static_cast<int32_t>(a.group.d), 1};
    } else if constexpr (REL == kShared) {
        const Group g = group_of(a.src, a.src.groups, b);
        const Run run = run_between(a.src.dst_ptr, g.first, g.end, a.src.num_dst);
        return Seq{run.first, g.shared > 0 ? run.count * static_cast<int32_t>(a.group.d) : 0, g.shared};
    } else if constexpr (REL == kBehind) {
        const Chunk ch = chunk_of(a.src, b);
        return Seq{ch.first, ch.count * static_cast<int32_t>(a.group.d), ch.pos0 + 1 - skip_of(a.src, b)};
    } else {
        int32_t n = a.src.num_src;
        if (a.src.len) n = a.src.len[b] < 0 ? 0 : (a.src.len[b] > n ? n : a.src.len[b]);
        return Seq{0, a.src.num_dst * static_cast<int32_t>(a.group.d), n};
    }
}
// Sequence `lane` (uniform) of those that the lanes hold.
__device__ __forceinline__ Seq lane_seq(const Seq &s, int lane) {
    return Seq{__builtin_amdgcn_readlane(s.first, lane), __builtin_amdgcn_readlane(s.rows, lane), lane_value(s.keys0, lane)};
}
// Keys that row r of the sequence sees, at least 0.  A row past the table's end sees one position behind it, which is
// no page: it needs no more of them to become NaN.
template <Relation REL>
__device__ __forceinline__ int32_t keys_of(const Args<REL> &a, const Seq &s, int r) {
    if constexpr (kOwnRows<REL>) {
        return 1 + a.group.div(r);
    } else if constexpr (kCausal<REL>) {
        const int64_t n = s.keys0 + a.group.div(r), most = (static_cast<int64_t>(a.src.table_width) << a.src.shift) + 1;
        return static_cast<int32_t>(n < 0 ? 0 : (n > most ? most : n));
    } else {
        return static_cast<int32_t>(s.keys0);
    }
}

// The row tiles of a sequence for one source head, weighted by their key tiles: tile j starts at start(j).  Causal
// tiles see more keys the later they are; between the first and the last tile's count the weights rise
// linearly (the weight only balances the blocks: a part of an item takes its share of the real key tiles).
template <int BM, int BN>
struct Tiles {
    int32_t count;
    int64_t w0;
    double slope;  // (last - first) / (2 count)
    template <Relation REL>
    static __device__ __forceinline__ Tiles of(const Args<REL> &a, const Seq &s, bool split) {
        Tiles t;
        t.count = (s.rows + BM - 1) / BM;
        t.w0 = 1;
        t.slope = 0.0;
        if (split && t.count > 0) {
            const int32_t n0 = keys_of<REL>(a, s, min(BM, s.rows) - 1), n1 = keys_of<REL>(a, s, s.rows - 1);
            const int32_t w1 = max(1, (n1 + BN - 1) / BN);
            t.w0 = max(1, (n0 + BN - 1) / BN);
            if (w1 != static_cast<int32_t>(t.w0)) t.slope = static_cast<double>(w1 - static_cast<int32_t>(t.w0)) / (2.0 * t.count);
        }
        return t;
    }
    __device__ __forceinline__ int64_t start(int64_t j) const {
        if (slope == 0.0) return j * w0;
        return j * w0 + static_cast<int64_t>(slope * static_cast<double>(j) * static_cast<double>(j));
    }
    __device__ __forceinline__ int64_t total() const { return start(count); }
    // the tile that holds weight position u < total()
    __device__ __forceinline__ int32_t find(int64_t u) const {
        int32_t lo = 0, hi = count - 1;
        while (lo < hi) {
            const int32_t mid = lo + (hi - lo + 1) / 2;
            if (start(mid) <= u) lo = mid;
            else hi = mid - 1;
        }
        return lo;
    }
};

// One wavefront walks the run of its block: the wavefronts of a block do it alike.
template <Relation REL, int BM, int BN>
struct Walk {
    typedef Tiles<BM, BN> T;
    int64_t u, end;       // position and end of the run
    int64_t base, whole;  // where sequence b starts, and a head's weight in it
    int32_t b;
    Seq s;
    T t;
    Seq mine;  // the lane's of the first 64 sequences

    static __device__ __forceinline__ Seq fetch(const Args<REL> &a, int e) {
        return e < a.src.batch ? seq_of<REL>(a, e) : Seq{0, 0, 0};
    }
    static __device__ __forceinline__ int64_t weight(const Args<REL> &a, const Seq &q) {
        return T::template of<REL>(a, q, a.part != nullptr).total() * a.kv_heads;
    }
    static __device__ __forceinline__ bool alike(const Args<REL> &a) {  // every sequence weighs the same
        if constexpr (REL != kStrided) return false;
        else return !a.src.len || !a.part;
    }
    __device__ __forceinline__ void begin(const Args<REL> &a, int w, int blocks) {
        const int nb = a.src.batch;
        mine = fetch(a, lane_id());
        const int64_t first = weight(a, mine), prefix = wave_prefix(first);
        int64_t all = lane_value(prefix, kWave - 1);
        if (alike(a)) all = lane_value(first, 0) * nb;
        else
            for (int e = kWave; e < nb; e += kWave) all += lane_value(wave_prefix(weight(a, fetch(a, e + lane_id()))), kWave - 1);
        const int64_t per = quotient(all, blocks), rem = all - per * blocks;
        u = w * per + (w < rem ? w : rem);
        end = u + per + (w < rem ? 1 : 0);
        base = 0;
        b = 0;
        if (u >= end) return;
        if (alike(a)) {
            b = static_cast<int32_t>(quotient(u, lane_value(first, 0)));
            base = b * lane_value(first, 0);
        } else {
            for (int e = 0; e < nb; e += kWave) {
                const int64_t here = e == 0 ? first : weight(a, fetch(a, e + lane_id()));
                const int64_t incl = e == 0 ? prefix : wave_prefix(here);
                const uint64_t past = __ballot(base + incl > u);
                if (past) {
                    const int l = __builtin_ctzll(past);
                    b = e + l;
                    base += lane_value(incl - here, l);
                    break;
                }
                base += lane_value(incl, kWave - 1);
            }
        }
        load(a);
    }
    __device__ __forceinline__ void load(const Args<REL> &a) {
        s = b < kWave ? lane_seq(mine, b) : seq_of<REL>(a, b);
        t = T::template of<REL>(a, s, a.part != nullptr);
        whole = t.total();
    }
    // The next part of an item of the run: row tile j of source head `head`, key tiles [t0, t1) of n.  starts / ends:
    // whether it holds the item's first and last share.
    struct Piece {
        int32_t head, j;
        int32_t t0, t1, n;
        bool starts, ends;
    };
    __device__ __forceinline__ bool next(const Args<REL> &a, Piece &p) {
        if (u >= end) return false;
        while (u >= base + whole * a.kv_heads) {  // the run is not at its end, so a later sequence holds u
            base += whole * a.kv_heads;
            ++b;
            load(a);
        }
        const int64_t in = u - base;
        p.head = static_cast<int32_t>(quotient(in, whole));
        const int64_t r = in - p.head * whole;
        p.j = t.find(r);
        const int64_t at = t.start(p.j), w = t.start(p.j + 1) - at, off = r - at;
        const int64_t take = min(w - off, end - u);
        p.n = (keys_of<REL>(a, s, min((p.j + 1) * BM, s.rows) - 1) + BN - 1) / BN;
        p.t0 = static_cast<int32_t>(w == p.n ? off : quotient(off * p.n, w));
        p.t1 = static_cast<int32_t>(w == p.n ? off + take : quotient((off + take) * p.n, w));
        p.starts = off == 0;
        p.ends = off + take == w;
        u += take;
        return true;
    }
};

// Wide tiles: what a block works on.
//  - Items cut into chunks of `chunk` key tiles: pieces in the order (sequence, source head, chunk of keys, row tile), and
//    an XCD takes an eighth of them that lies together.  The row tiles that reach into a chunk are the last ones of a
//    causal sequence, all of a strided one, and they come last first.
//  - Whole items: (sequence, eight heads, row tile, head), dealt to the XCDs in turn, so that an XCD's L2 holds one head of
//    the eight, the XCDs get alike shares of unequal sequences, and a causal sequence's longest items start first
//    (blocks start in order: a long one late in the order would end late).
template <Relation REL, int BM, int BN>
struct Deal {
    struct Load {
        Seq s;
        int32_t tiles;    // row tiles of a head
        int32_t n0, n1;   // key tiles of the first and the last of them, at least 1
    };
    static constexpr int32_t kWhole = 0x7fffffff;
    int64_t pieces;
    int32_t chunk;

    static __device__ __forceinline__ Load load(const Args<REL> &a, const Seq &s) {
        Load l{s, (s.rows + BM - 1) / BM, 1, 1};
        if (s.rows > 0) {
            l.n0 = max(1, (keys_of<REL>(a, s, min(BM, s.rows) - 1) + BN - 1) / BN);
            l.n1 = max(1, (keys_of<REL>(a, s, s.rows - 1) + BN - 1) / BN);
        }
        return l;
    }
    static __device__ __forceinline__ Load load(const Args<REL> &a, int e) {
        return load(a, e < a.src.batch ? seq_of<REL>(a, e) : Seq{0, 0, 0});
    }
    static __device__ __forceinline__ bool alike(const Args<REL> &a) {
        if constexpr (REL != kStrided) return false;
        else return a.src.len == nullptr;
    }
    // Sum of f(load) over the sequences, times the heads.
    template <class F>
    static __device__ __forceinline__ int64_t total(const Args<REL> &a, const Load &first, F f) {
        if (alike(a)) return lane_value(f(first), 0) * a.src.batch * a.kv_heads;
        int64_t all = lane_value(wave_prefix(f(first)), kWave - 1);
        for (int e = kWave; e < a.src.batch; e += kWave) all += lane_value(wave_prefix(f(load(a, e + lane_id()))), kWave - 1);
        return all * a.kv_heads;
    }
    static __device__ __forceinline__ int32_t parts(int32_t n, int32_t chunk) {  // n >= 1
        return static_cast<int32_t>(static_cast<uint32_t>(n - 1) / static_cast<uint32_t>(chunk)) + 1;
    }
    // Row tiles that see keys of chunk c: token t does if keys0 + t > c * chunk * BN.
    static __device__ __forceinline__ int32_t reach(const Args<REL> &a, const Load &l, int32_t c, int32_t chunk) {
        if constexpr (kCausal<REL>) {
            const int64_t t = static_cast<int64_t>(c) * chunk * BN - l.s.keys0 + 1;
            return c == 0 || t <= 0 ? l.tiles : l.tiles - static_cast<int32_t>(t * a.group.d / BM);
        } else {
            return l.tiles;
        }
    }
    // Pieces of one head.
    static __device__ __forceinline__ int64_t count(const Args<REL> &a, const Load &l, int32_t chunk) {
        const int32_t n = parts(l.n1, chunk);
        if constexpr (!kCausal<REL>) return static_cast<int64_t>(n) * l.tiles;
        // the chunks below the first token's keys are whole
        const int64_t below = l.s.keys0 > 0 ? static_cast<int64_t>(static_cast<uint32_t>((l.s.keys0 - 1) / BN) / static_cast<uint32_t>(chunk)) + 1 : 1;
        int64_t all = min(static_cast<int64_t>(n), below) * l.tiles;
        for (int64_t c = below; c < n; ++c) all += reach(a, l, static_cast<int32_t>(c), chunk);
        return all;
    }

    // Chunks as small as lets all pieces run at once, but not below kLeastChunk tiles, whose work a part's 64 KB of state, written
    // and read again, are worth.  (Pieces up to twice the resident blocks: some XCDs' in two turns, 281 instead of 182 us
    // for 1023 tokens over 16001 keys.)  Returns what the lanes read of the first 64 sequences.
    __device__ __forceinline__ Load begin(const Args<REL> &a) {
        const Load first = load(a, lane_id());
        chunk = kWhole;
        pieces = total(a, first, [](const Load &l) { return static_cast<int64_t>(l.tiles); });
        if (!a.part || pieces > a.slots) return first;
        const int64_t work = total(a, first, [](const Load &l) { return static_cast<int64_t>(l.tiles) * ((l.n0 + l.n1 + 1) / 2); });
        // Shared positions: twice as many tiles, so half the states (64 tokens behind 8192 positions, 8 heads of 128: 26.1 us and
        // 8.7 of the join, with 4 tiles 24.9 and 13.5).
        const int64_t least = REL == kShared ? 2 * kLeastChunk : kLeastChunk;
        int64_t c = max(least, quotient(work + a.slots - 1, a.slots));
        do {
            chunk = static_cast<int32_t>(min(c, static_cast<int64_t>(kWhole)));
            pieces = total(a, first, [&](const Load &l) { return count(a, l, chunk); });
            c += max(int64_t(1), c / 16);
        } while (pieces > a.slots);
        return first;
    }

    struct Piece {
        int32_t b, head, j;
        int32_t t0, t1;        // key tiles
        int32_t part, parts;   // of the item
    };
    __device__ __forceinline__ Piece piece(const Args<REL> &a, const Load &first, int64_t p, Seq &s) const {
        int64_t base = 0;
        int b = 0;
        if (alike(a)) {
            const int64_t per = lane_value(count(a, first, chunk), 0) * a.kv_heads;
            b = static_cast<int>(quotient(p, per));
            base = b * per;
        } else {
            for (int e = 0; e < a.src.batch; e += kWave) {
                const int64_t mine = count(a, e == 0 ? first : load(a, e + lane_id()), chunk) * a.kv_heads;
                const int64_t incl = wave_prefix(mine);
                const uint64_t past = __ballot(base + incl > p);
                if (past) {
                    const int i = __builtin_ctzll(past);
                    b = e + i;
                    base += lane_value(incl - mine, i);
                    break;
                }
                base += lane_value(incl, kWave - 1);
            }
        }
        s = b < kWave ? lane_seq(first.s, b) : seq_of<REL>(a, b);
        const Load l = load(a, s);
        const int64_t per = count(a, l, chunk);
        Piece r;
        r.b = b;
        r.part = 0;
        int64_t rest = p - base;
        if (chunk == kWhole) {
            const int32_t heads = a.kv_heads % static_cast<int>(kXcds) == 0 ? static_cast<int>(kXcds) : a.kv_heads;
            const int64_t band = static_cast<int64_t>(l.tiles) * heads;
            const int32_t at = static_cast<int32_t>(quotient(rest, band));
            rest -= at * band;
            const int32_t k = static_cast<int32_t>(quotient(rest, heads));
            r.j = l.tiles - 1 - k;
            r.head = at * heads + static_cast<int32_t>(rest - static_cast<int64_t>(k) * heads);
        } else {
            r.head = static_cast<int32_t>(quotient(rest, per));
            rest -= r.head * per;
            for (int32_t here; rest >= (here = reach(a, l, r.part, chunk)); ++r.part) rest -= here;
            r.j = l.tiles - 1 - static_cast<int32_t>(rest);
        }
        const int32_t n = (keys_of<REL>(a, s, min((r.j + 1) * BM, s.rows) - 1) + BN - 1) / BN;
        r.parts = parts(max(1, n), chunk);
        r.t0 = static_cast<int32_t>(min(static_cast<int64_t>(r.part) * chunk, static_cast<int64_t>(n)));
        r.t1 = static_cast<int32_t>(min((r.part + int64_t(1)) * chunk, static_cast<int64_t>(n)));
        return r;
    }
};

// ------------------------------------------------------------------------------------------ sources

// Where the keys (or values) of one source head lie.  Tiles start at multiples of BN, so a page of at most BN rows
// starts at one of the tile's rows, and a larger one holds the tile whole.
template <Relation REL>
struct Source {
    const uint16_t *p;
    int64_t row, page_stride;
    int32_t mask;  // rows of a page - 1
    __device__ __forceinline__ void set(const Args<REL> &a, const Rows &t, int b, const Seq &s, int head) {
        p = t.p + head * t.head;
        row = t.row;
        if constexpr (kOwnRows<REL>) {
            p += s.first * row;
        } else if constexpr (kPages<REL>) {
            page_stride = t.batch;
            mask = (1 << a.src.shift) - 1;
        } else {
            p += b * t.batch;
        }
    }
    // start of the tile at k0 within its page
    __device__ __forceinline__ const uint16_t *tile(int32_t k0) const {
        return p + static_cast<int64_t>(kPages<REL> ? k0 & mask : k0) * row;
    }
    // elements from there to row i of the tile: row strides are below 2^23 and tiles have at most 128 rows
    __device__ __forceinline__ int32_t offset(int32_t i) const {
        return (kPages<REL> ? i & mask : i) * static_cast<int32_t>(row);
    }
    // the row of any position (>= 0)
    __device__ __forceinline__ const uint16_t *at(int32_t pos, int32_t page) const {
        if constexpr (kPages<REL>) return p + page * page_stride + static_cast<int64_t>(pos & mask) * row;
        else return p + pos * row;
    }
};

// The table's entry for an item's position.
template <Relation REL>
struct Cells {
    int32_t row;   // of the table
    int32_t skip;  // positions of the sequence before position 0 of the item
    __device__ __forceinline__ Cells(const Args<REL> &a, int b) : row(b), skip(0) {
        if constexpr (REL == kShared) row = group_of(a.src, a.src.groups, b).first;
        if constexpr (REL == kBehind) skip = skip_of(a.src, b);
    }
    __device__ __forceinline__ int32_t entry(const Args<REL> &a, int32_t pos) const {
        if constexpr (REL == kBehind) return entry_at(a.src, row, static_cast<int64_t>(pos) + skip);
        else return entry_at(a.src, row, pos);
    }
};

// Start of row r's width in a [heads, rows, width] tensor of destinations, for source head `head`.
template <Relation REL>
__device__ __forceinline__ int64_t row_at(const Args<REL> &a, const Rows &t, int b, const Seq &s, int head, int r) {
    const int d = static_cast<int>(a.group.d), token = a.group.div(r), g = r - token * d;
    return b * t.batch + static_cast<int64_t>(head * d + g) * t.head + static_cast<int64_t>(s.first + token) * t.row;
}
template <Relation REL>
__device__ __forceinline__ int64_t lse_at(const Args<REL> &a, int b, const Seq &s, int head, int r) {
    const int d = static_cast<int>(a.group.d), token = a.group.div(r), g = r - token * d;
    return b * a.lse_batch + (head * d + g) * a.lse_head + s.first + token;
}

// Where row r's results go, 4 widths at a time: y in the input type, or an fp32 state (normalized) to be joined; and lse, there
// in the log2 domain.
template <int D, Relation REL>
__device__ __forceinline__ auto out_row(const Args<REL> &a, int b, const Seq &s, int head, int r) {
    if constexpr (kHalf<REL>) return a.src.state + lse_at(a, b, s, head, r) * D;
    else return const_cast<uint16_t *>(a.y.p) + row_at(a, a.y, b, s, head, r);
}
template <class T>
__device__ __forceinline__ void put(uint16_t *p, f4 v) { *reinterpret_cast<u2 *>(p) = u2{T::pack(v[0], v[1]), T::pack(v[2], v[3])}; }
template <class T>
__device__ __forceinline__ void put(float *p, f4 v) { *reinterpret_cast<f4 *>(p) = v; }
template <Relation REL>
__device__ __forceinline__ void put_lse(const Args<REL> &a, int b, const Seq &s, int head, int r, float lse2) {
    if constexpr (kHalf<REL>) a.src.lse2[lse_at(a, b, s, head, r)] = lse2;
    else if (a.lse) a.lse[lse_at(a, b, s, head, r)] = lse2 * kLn2;
}

// Row r of an item behind shared positions, once: its share of mass to start with, NaN where the sequence's first new token is
// among the shared positions, of which it would see too many.  A row that shares nothing says so in the place of the state
// that it does not have.
__device__ __forceinline__ float open_row(const Args<kBehind> &a, const Cells<kBehind> &cells, int b, const Seq &s, int head, int r) {
    if (cells.skip == 0) a.src.shared_lse2[lse_at(a, b, s, head, r)] = -__builtin_inff();
    return cells.skip > 0 && s.keys0 <= 0 ? __builtin_nanf("") : 0.0f;
}

// Rows of no sequence of a packed call: before ptr[0] and behind ptr[batch].  They see nothing: y = 0, lse = -inf.
template <int D, Relation REL>
__device__ __forceinline__ void clear_outside(const Args<REL> &a) {
    if constexpr (kOwnRows<REL>) {
        const Run inside = a.src.batch > 0 ? run_between(a.src.ptr, 0, a.src.batch, a.src.num_rows) : Run{0, 0};
        const int32_t outside = a.src.num_rows - inside.count;
        if (outside == 0) return;
        const int64_t heads = static_cast<int64_t>(a.kv_heads) * a.group.d, all = outside * heads * (D / 8);
        for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < all; i += static_cast<int64_t>(gridDim.x) * kThreads) {
            const int c = static_cast<int>(i % (D / 8));
            const int64_t head = i / (D / 8) % heads;
            int64_t row = i / (D / 8) / heads;
            if (row >= inside.first) row += inside.count;
            reinterpret_cast<u4 *>(const_cast<uint16_t *>(a.y.p) + head * a.y.head + row * a.y.row)[c] = u4{0u, 0u, 0u, 0u};
            if (a.lse && c == 0) a.lse[head * a.lse_head + row] = -__builtin_inff();
        }
    }
}

// ------------------------------------------------------------------------------------------ values that are not finite

// A row must not take anything from a value that it does not see, but its weight of 0 times an infinity would be NaN.  A
// tile that some rows of an item see less of than others (the last ones of a causal chunk) is looked through for values
// that are not finite; where there are any, the rows that see them are given them one by one, and the product gets 0 in their
// places.  (8 x 64 new tokens over up to 4000, f16: 37.1 us without, 37.4 with; a prompt of 8192 tokens 292 and 294.  By
// masks and selects: branches on each half held exec masks that spilled, 0.3 us of a single token's 8.2.)

// ------------------------------------------------------------------------------------------ wide tiles

template <int D>
struct Geo {
    static constexpr int BM = 128;                      // rows a tile: 32 a wavefront
    static constexpr int CPR = D / 8;                   // 16-byte chunks per row
    static constexpr int RB = 2 * D;                    // bytes per row
    static constexpr int R = 256 / RB;                  // rows per 256-byte bank window
    static constexpr int CH = D / 32;                   // 32-deep chunks of the score product
    static constexpr int DB = D / 16;                   // 16-wide blocks of the output
    static constexpr int BN = D == 64 ? 128 : 64;       // keys a tile
    static constexpr int KB = BN / 16;                  // 16-key blocks of the score product
    static constexpr int KC = BN / 32;                  // 32-key chunks of the value product
    static constexpr int TILE = BN * RB;                // bytes of a K or V tile: 16 KB
    static constexpr int LPW = TILE / 1024 / kWaves;    // 1-KB direct loads per wavefront, tile and operand
};

// LDS layouts, free of bank conflicts without padding: the 16-byte chunk c of key row k sits at chunk c ^ (k / R % CPR)
// (16 keys of one chunk fall into 16 bank groups); the 32-byte block c / 2 of value row k at block c / 2 ^ (k / R % DB)
// (the transposing read takes 4 keys x 16 widths per 16 lanes).
template <int D>
__device__ __forceinline__ int k_chunk(int k, int pc) { return pc ^ ((k / Geo<D>::R) % Geo<D>::CPR); }
template <int D>
__device__ __forceinline__ int v_chunk(int k, int pc) {
    return (((pc >> 1) ^ ((k / Geo<D>::R) % Geo<D>::DB)) << 1) | (pc & 1);
}

template <class T, int D>
struct State {
    f4 o[Geo<D>::DB][2];
    float m[2], l[2];  // l: this lane's share of the mass
};

// Weights 2^(c s - m) of query block qb and this lane's sum of them.  They enter the value product rounded to the
// input type (the matrix cores' operand); the mass is of the unrounded fp32 weights.
template <class T, int KB>
__device__ __forceinline__ float weights(const f4 (*s)[2], int qb, float c, float m, u4 (*pb)[2]) {
    float sum = 0.0f;
#pragma unroll
    for (int kc = 0; kc < KB / 2; ++kc) {
        float p[2][4];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) p[e][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * kc + e][qb][i], c, -m));
        sum += ((p[0][0] + p[0][1]) + (p[0][2] + p[0][3])) + ((p[1][0] + p[1][1]) + (p[1][2] + p[1][3]));
        pb[kc][qb] = u4{T::pack(p[0][0], p[0][1]), T::pack(p[0][2], p[0][3]), T::pack(p[1][0], p[1][1]),
                        T::pack(p[1][2], p[1][3])};
    }
    return sum;
}

// One key tile.  keys: how many of it the item sees; lim[qb]: how many this lane's row of block qb does.
template <class T, int D>
__device__ __forceinline__ void tile_step(State<T, D> &st, const u4 (&q)[2][Geo<D>::CH], const uint8_t *kt,
                                          const uint8_t *vt, int kr, int vr, float c, bool edge,
                                          const int32_t *seen, int32_t k0, int g) {
    using G = Geo<D>;
    f4 s[G::KB][2];
    // S^T = K Q^T.  The operand reads run kAhead ahead of their products, in this order: the compiler, left to itself,
    // puts a read next to its use and waits for it.
    {
        constexpr int kReads = G::CH * G::KB, kAhead = 4;
        auto read = [&](int i) {
            return *reinterpret_cast<const u4 *>(kt + (kr ^ (64 * (i / G::KB))) + i % G::KB * 16 * G::RB);
        };
        u4 ka[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) ka[i] = read(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            const int ch = i / G::KB, kb = i % G::KB;
#pragma unroll
            for (int qb = 0; qb < 2; ++qb)
                s[kb][qb] = T::mma(ka[i % kAhead], q[qb][ch], ch == 0 ? f4{0.0f, 0.0f, 0.0f, 0.0f} : s[kb][qb]);
            if (i + kAhead < kReads) ka[i % kAhead] = read(i + kAhead);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (edge) {
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            // key kb * 16 + 4 g + i is seen iff kb * 16 + i < seen - k0 - 4 g
            const int rel = seen[qb] - k0 - 4 * g;
#pragma unroll
            for (int kb = 0; kb < G::KB; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[kb][qb][i] = kb * 16 + i < rel ? s[kb][qb][i] : -__builtin_inff();
        }
    }
    u4 pb[G::KC][2];
    float sum[2];
    __builtin_amdgcn_s_setprio(2);
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) sum[qb] = weights<T, G::KB>(s, qb, c, st.m[qb], pb);
    // Against the current reference point every weight is at most the lane's sum; up to the cap they stay inside
    // every 16-bit type's range.  A larger sum, or NaN (the first tile, where m = -inf, always), moves the point.
    if (!__all(sum[0] <= kMassCap<T> && sum[1] <= kMassCap<T>)) {
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            float mt = s[0][qb][0];
#pragma unroll
            for (int kb = 0; kb < G::KB; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) mt = fmaxf(mt, s[kb][qb][i]);
            mt = column_max(mt) * c - kLift<T>;
            if (mt > st.m[qb]) {
                // nothing seen so far: o is 0, or what add_wild put there
                const float alpha = st.m[qb] == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(st.m[qb] - mt);
                st.m[qb] = mt;
                st.l[qb] *= alpha;
#pragma unroll
                for (int db = 0; db < G::DB; ++db) st.o[db][qb] *= alpha;
            }
            // nothing seen so far: any finite point gives weights of 0
            sum[qb] = weights<T, G::KB>(s, qb, c, st.m[qb] == -__builtin_inff() ? 0.0f : st.m[qb], pb);
        }
    }
    st.l[0] += sum[0];
    st.l[1] += sum[1];
    __builtin_amdgcn_s_setprio(0);
    // O^T += V^T P^T, likewise: an operand is two transposing reads
    {
        constexpr int kReads = G::DB * G::KC, kAhead = 3;
        auto read = [&](int i) {
            const uint8_t *const p = vt + (vr ^ (32 * (i / G::KC))) + i % G::KC * 32 * G::RB;
            const u2 lo = lds_transposed16(p), hi = lds_transposed16(p + 16 * G::RB);
            return u4{lo.x, lo.y, hi.x, hi.y};
        };
        u4 va[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) va[i] = read(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            const int db = i / G::KC, kc = i % G::KC;
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) st.o[db][qb] = T::mma(va[i % kAhead], pb[kc][qb], st.o[db][qb]);
            if (i + kAhead < kReads) va[i % kAhead] = read(i + kAhead);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// Partial state of a slot: o [rows of the tile][D], then m, then l [rows].
template <int BM, int D>
constexpr int64_t slot_floats() { return BM * (D + 2); }

// What block `block` of `blocks` (a multiple of 8) works on.  The buffers are separate arrays; wild: of the tiles in v0buf and
// v1buf, by wavefront.
template <class T, int D, Relation REL>
__device__ __forceinline__ void wide_pieces(const Args<REL> &a, unsigned block, unsigned blocks, uint8_t *k0buf, uint8_t *v0buf,
                                            uint8_t *k1buf, uint8_t *v1buf, int (*wild)[kWaves]) {
    using G = Geo<D>;
    const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave);
    const int col = lane & 15, g = lane >> 4;

    // the rows and chunks of a tile that this lane's direct loads fetch, and where it reads its operands: the swizzles
    // only flip bits that chunk (64 ch bytes) and block (32 db bytes) offsets flip too
    int krow[G::LPW], kch[G::LPW], vch[G::LPW];
#pragma unroll
    for (int r = 0; r < G::LPW; ++r) {
        const int byte = (w * G::LPW + r) * 1024 + 16 * lane;
        krow[r] = byte / G::RB;
        kch[r] = k_chunk<D>(krow[r], byte % G::RB / 16);
        vch[r] = v_chunk<D>(krow[r], byte % G::RB / 16);
    }
    const int kr = col * G::RB + 16 * k_chunk<D>(col, g);
    const int vrow = 4 * g + col / 4;
    const int vr = vrow * G::RB + 32 * ((vrow / G::R) % G::DB) + 8 * (col % 4);

    typedef Deal<REL, G::BM, G::BN> Pieces;
    Pieces deal;
    typename Pieces::Load lanes;
    bool whole_items = false;
    int64_t per = 1, first = 0;  // pieces of this block (planned), or of its XCD: block b of the grid (a multiple of 8) runs on XCD b % 8
    if constexpr (REL != kPlanned) {
        lanes = deal.begin(a);
        if (a.part && threadIdx.x == 0 && deal.pieces + block < a.slots) a.rec[2 * (deal.pieces + block)] = int4{0, 0, 0, 0};
        whole_items = deal.chunk == deal.kWhole;
        const int x = block % kXcds;
        per = deal.pieces / kXcds + (x < deal.pieces % kXcds ? 1 : 0);
        first = whole_items ? x : x * (deal.pieces / kXcds) + min(static_cast<int64_t>(x), deal.pieces % kXcds);
    }
    for (int64_t i = REL == kPlanned ? 0 : block / kXcds; i < per; i += REL == kPlanned ? 1 : blocks / kXcds) {
        int64_t id;
        Seq s;
        typename Pieces::Piece pc;
        if constexpr (REL == kPlanned) {
            id = block;
            const Item it = item_of(a.src.table, a.kv_heads, static_cast<int32_t>(a.group.d), static_cast<int32_t>(block));
            if (it.level == 0) break;
            s = Seq{it.run.first, it.run.count * static_cast<int32_t>(a.group.d), 1};
            pc = typename Pieces::Piece{it.b, it.kv, it.level - 1, 0, 0, it.part, it.parts};
            const int32_t n = (keys_of<REL>(a, s, min((pc.j + 1) * G::BM, s.rows) - 1) + G::BN - 1) / G::BN;
            pc.t0 = part_start(n, it.part, it.parts);
            pc.t1 = part_start(n, it.part + 1, it.parts);
        } else {
            id = first + (whole_items ? i * kXcds : i);
            if (i >= blocks / kXcds) lanes = deal.load(a, lane_id());  // not kept over a piece's work
            pc = deal.piece(a, lanes, id, s);
            if (a.part && threadIdx.x == 0 && id < a.slots) {
                a.rec[2 * id] = pc.part == 0 && pc.parts > 1 ? int4{pc.b + 1, pc.head, pc.j, pc.parts} : int4{0, 0, 0, 0};
                a.rec[2 * id + 1] = REL == kShared ? int4{deal.chunk, s.first, s.rows, 0} : int4{deal.chunk, 0, 0, 0};
            }
        }
        const int r0 = pc.j * G::BM + w * 32;
        Source<REL> ks, vs;
        ks.set(a, a.src.k, pc.b, s, pc.head);
        vs.set(a, a.src.v, pc.b, s, pc.head);
        const Cells<REL> cells(a, pc.b);
        const int32_t keys = keys_of<REL>(a, s, min((pc.j + 1) * G::BM, s.rows) - 1);  // of the tile's last row
        u4 q[2][G::CH];
        int32_t seen[2];
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            const int r = min(r0 + qb * 16 + col, s.rows - 1);
            const u4 *p = reinterpret_cast<const u4 *>(a.q.p + row_at(a, a.q, pc.b, s, pc.head, r));
#pragma unroll
            for (int ch = 0; ch < G::CH; ++ch) q[qb][ch] = p[ch * 4 + g];
            seen[qb] = keys_of<REL>(a, s, r);
        }
        const bool any = r0 < s.rows;                                                      // rows of this wavefront
        const int32_t least = keys_of<REL>(a, s, min(r0, s.rows - 1));                   // its first row sees
        const int32_t most = keys_of<REL>(a, s, min(r0 + 31, s.rows - 1));               // its last row sees
        State<T, D> st;
#pragma unroll
        for (int db = 0; db < G::DB; ++db) st.o[db][0] = st.o[db][1] = f4{0.0f, 0.0f, 0.0f, 0.0f};
        st.m[0] = st.m[1] = -__builtin_inff();
        st.l[0] = st.l[1] = 0.0f;
        if constexpr (REL == kBehind) {
            if (pc.part == 0 && g == 0)
#pragma unroll
                for (int qb = 0; qb < 2; ++qb)
                    if (r0 + qb * 16 + col < s.rows) st.l[qb] = open_row(a, cells, pc.b, s, pc.head, r0 + qb * 16 + col);
        }

        // A load's 1 KB are 4 or 8 rows from a multiple of as many, so in pages of 8 rows or more they lie in one page.
        // Lane r looks load r's page up, a tile ahead of the rows; the entry is read and checked when they are loaded.
        // Positions past the item's last key read that key (its scores there are masked, its value there is cleared
        // once it has arrived: a weight of 0 times an infinity would be NaN); a page that the cache does not have is
        // read from the constant rows.
        auto look_up = [&](int kt) -> int32_t {
            if constexpr (kPages<REL>) {
                const int group = (w * G::LPW + lane % G::LPW) * (1024 / G::RB);
                return cells.entry(a, min(kt * G::BN + group, keys - 1));
            } else {
                return 0;
            }
        };
        auto stage = [&](int kt, int32_t entry, uint8_t *kb, uint8_t *vb) {
            const int32_t k0 = kt * G::BN;
            const uint16_t *const kt0 = ks.tile(k0), *const vt0 = vs.tile(k0);
#pragma unroll
            for (int r = 0; r < G::LPW; ++r) {
                const int run = (w * G::LPW + r) * 1024;
                const int32_t i = min(krow[r], keys - 1 - k0);
                const uint16_t *kp = kt0, *vp = vt0;
                int32_t ko = ks.offset(i), vo = vs.offset(i);
                if constexpr (kPages<REL>) {
                    const int32_t page = __builtin_amdgcn_readlane(entry, r);
                    const bool good = is_page(a.src, page);
                    kp = good ? kp + page * ks.page_stride : reinterpret_cast<const uint16_t *>(kNanRow);
                    vp = good ? vp + page * vs.page_stride : reinterpret_cast<const uint16_t *>(kZeroRow);
                    ko = good ? ko : 0;
                    vo = good ? vo : 0;
                }
                load_to_lds16(kp + ko + 8 * kch[r], kb + run);
                load_to_lds16(vp + vo + 8 * vch[r], vb + run);
            }
        };
        // Tiles that not all of the item's rows see whole.  Before the barrier each wavefront clears what lies past the
        // last key of its own rows of the values, and looks the others through; after it, values that are not finite are
        // taken care of.
        const int32_t edge = keys_of<REL>(a, s, pc.j * G::BM) / G::BN;
        auto own_rows = [&](uint8_t *vb, int r) { return reinterpret_cast<u4 *>(vb + (w * G::LPW + r) * 1024 + 16 * lane); };
        auto tidy = [&](int kt, uint8_t *vb, int *found) {
            if (kt < edge) return;
            const int32_t left = keys - kt * G::BN;
            uint32_t bad = 0;
#pragma unroll
            for (int r = 0; r < G::LPW; ++r) {
                if (krow[r] >= left) *own_rows(vb, r) = u4{0u, 0u, 0u, 0u};
                if (kCausal<REL>) bad |= any_wild<T>(*own_rows(vb, r));
            }
            if (kCausal<REL>) {
                const bool here = __any(bad != 0);
                if (lane == 0) found[w] = here;
            }
        };
        auto mend = [&](int kt, uint8_t *vb, const int *found) {
            if (!kCausal<REL> || kt < edge) return;
            if (uniform(found[0] | found[1] | found[2] | found[3]) == 0) return;
            for (int k = 0; k < G::BN; ++k)
#pragma unroll
                for (int db = 0; db < G::DB; ++db) {
                    const u2 x = *reinterpret_cast<const u2 *>(vb + k * G::RB + 16 * v_chunk<D>(k, 2 * db + g / 2) + 8 * (g % 2));
#pragma unroll
                    for (int qb = 0; qb < 2; ++qb)
                        add_wild<T>(st.o[db][qb], x, kt * G::BN + k < seen[qb]);
                }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < G::LPW; ++r) *own_rows(vb, r) = without_wild<T>(*own_rows(vb, r));
            __syncthreads();
        };
        auto step = [&](int kt, const uint8_t *kb, const uint8_t *vb) {
            const int32_t k0 = kt * G::BN;
            if (any && k0 < most) tile_step<T, D>(st, q, kb, vb, kr, vr, a.c, k0 + G::BN > least, seen, k0, g);
        };
        __syncthreads();  // the previous item's tiles are read
        int32_t entry = 0;
        if (pc.t0 < pc.t1) {
            stage(pc.t0, look_up(pc.t0), k0buf, v0buf);
            entry = look_up(min(pc.t0 + 1, pc.t1 - 1));
        }
        for (int kt = pc.t0; kt < pc.t1; kt += 2) {
            loads_arrived();
            tidy(kt, v0buf, wild[0]);
            __syncthreads();
            if (kt + 1 < pc.t1) stage(kt + 1, entry, k1buf, v1buf);
            entry = look_up(min(kt + 2, pc.t1 - 1));
            mend(kt, v0buf, wild[0]);
            step(kt, k0buf, v0buf);
            if (kt + 1 >= pc.t1) break;
            loads_arrived();
            tidy(kt + 1, v1buf, wild[1]);
            __syncthreads();
            if (kt + 2 < pc.t1) stage(kt + 2, entry, k0buf, v0buf);
            entry = look_up(min(kt + 3, pc.t1 - 1));
            mend(kt + 1, v1buf, wild[1]);
            step(kt + 1, k1buf, v1buf);
        }

        const bool whole = pc.parts == 1;
        float *const po = whole ? nullptr : a.part + id * slot_floats<G::BM, D>();
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            const float lt = column_sum(st.l[qb]);
            const int r = r0 + qb * 16 + col;
            if (r >= s.rows) continue;
            if (whole) {
                const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
                auto *const yr = out_row<D, REL>(a, pc.b, s, pc.head, r);
#pragma unroll
                for (int db = 0; db < G::DB; ++db) put<T>(yr + db * 16 + g * 4, st.o[db][qb] * inv);
                if (g == 0) put_lse(a, pc.b, s, pc.head, r, st.m[qb] + __log2f(lt));
            } else {
                const int tr = r - pc.j * G::BM;
#pragma unroll
                for (int db = 0; db < G::DB; ++db) *reinterpret_cast<f4 *>(po + tr * D + db * 16 + g * 4) = st.o[db][qb];
                if (g == 0) {
                    po[G::BM * D + tr] = st.m[qb];
                    po[G::BM * (D + 1) + tr] = lt;
                }
            }
        }
    }
}

template <class T, int D, Relation REL>
__global__ __launch_bounds__(kThreads, 2) void wide_kernel(Args<REL> a) {
    constexpr int TILE = Geo<D>::TILE;
    __shared__ __attribute__((aligned(1024))) uint8_t k0buf[TILE], v0buf[TILE], k1buf[TILE], v1buf[TILE];
    __shared__ int wild[2][kWaves];
    wide_pieces<T, D, REL>(a, blockIdx.x, gridDim.x, k0buf, v0buf, k1buf, v1buf, wild);
    clear_outside<D, REL>(a);
}

// ------------------------------------------------------------------------------------------ narrow tiles

// Few rows (single tokens): 16 rows a tile, so one column block of the matrix product, and the time is that of reading
// the keys and values.  The four wavefronts take turns of KW keys each, with no barrier between them until the item's
// end: a wavefront's keys go to registers in the operand's layout, its values through its own LDS for the
// transposing read, both a step ahead (16 KB in flight a wavefront, 128 KB a compute unit).
template <int D>
struct Thin {
    static constexpr int BM = 16;
    static constexpr int KW = 4096 / D;                 // keys of a wavefront's step: 8 KB of keys, 8 KB of values
    static constexpr int BN = kWaves * KW;
    static constexpr int CPR = D / 8, RB = 2 * D, R = 256 / RB;
    static constexpr int CH = D / 32, DB = D / 16;
    static constexpr int KB = KW / 16, KC = KW / 32;
    static constexpr int RUNS = KW * RB / 1024;         // 1-KB direct loads of values a step
    static constexpr int LOADS = RUNS + KB * CH;        // loads a step
};

template <class T, int D>
struct ThinState {
    f4 o[Thin<D>::DB];
    float m, l;
};

template <class T, int D>
__device__ __forceinline__ void thin_step(ThinState<T, D> &st, const u4 *q, const u4 (&k)[Thin<D>::KB][Thin<D>::CH],
                                          const uint8_t *vt, int vr, float c, bool edge, int32_t left, int g) {
    using G = Thin<D>;
    f4 s[G::KB];
#pragma unroll
    for (int ch = 0; ch < G::CH; ++ch)
#pragma unroll
        for (int kb = 0; kb < G::KB; ++kb) s[kb] = T::mma(k[kb][ch], q[ch], ch == 0 ? f4{0.0f, 0.0f, 0.0f, 0.0f} : s[kb]);
    if (edge) {
        const int rel = left - 4 * g;
#pragma unroll
        for (int kb = 0; kb < G::KB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[kb][i] = kb * 16 + i < rel ? s[kb][i] : -__builtin_inff();
    }
    float mt = s[0][0];
#pragma unroll
    for (int kb = 0; kb < G::KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) mt = fmaxf(mt, s[kb][i]);
    mt = column_max(mt) * c;
    if (__any(mt > st.m)) {
        const float m = fmaxf(mt, st.m);
        const float alpha = st.m == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(st.m - m);
        st.m = m;
        st.l *= alpha;
#pragma unroll
        for (int db = 0; db < G::DB; ++db) st.o[db] *= alpha;
    }
    const float ref = st.m == -__builtin_inff() ? 0.0f : st.m - kLift<T>;  // nothing seen so far: weights of 0
    u4 pb[G::KC];
#pragma unroll
    for (int kc = 0; kc < G::KC; ++kc) {
        float p[2][4];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) p[e][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * kc + e][i], c, -ref));
        st.l += ((p[0][0] + p[0][1]) + (p[0][2] + p[0][3])) + ((p[1][0] + p[1][1]) + (p[1][2] + p[1][3]));
        pb[kc] = u4{T::pack(p[0][0], p[0][1]), T::pack(p[0][2], p[0][3]), T::pack(p[1][0], p[1][1]),
                    T::pack(p[1][2], p[1][3])};
    }
#pragma unroll
    for (int db = 0; db < G::DB; ++db)
#pragma unroll
        for (int kc = 0; kc < G::KC; ++kc) {
            const uint8_t *const p = vt + (vr ^ (32 * db)) + kc * 32 * G::RB;
            const u2 lo = lds_transposed16(p), hi = lds_transposed16(p + 16 * G::RB);
            st.o[db] = T::mma(u4{lo.x, lo.y, hi.x, hi.y}, pb[kc], st.o[db]);
        }
}

// What block `block` of `blocks` works on.  v0of(i), v1of(i): wavefront i's buffers, in separate arrays.
template <int D>
constexpr int kThinWave = Thin<D>::KW *Thin<D>::RB;  // bytes of a wavefront's step of values: 8 KB, also 16 rows of fp32 states or more
template <class T, int D, Relation REL, class Buffer0, class Buffer1>
__device__ __forceinline__ void thin_pieces(const Args<REL> &a, int block, int blocks, Buffer0 v0of, Buffer1 v1of,
                                            float (*ml)[kWaves][Thin<D>::BM]) {
    using G = Thin<D>;
    static_assert(kThinWave<D> >= G::BM * D * 4, "a wavefront's state fits its buffer");
    const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave);
    const int col = lane & 15, g = lane >> 4;
    uint8_t *const v0 = v0of(w), *const v1 = v1of(w);

    const int vrow = 4 * g + col / 4;
    const int vr = vrow * G::RB + 32 * ((vrow / G::R) % G::DB) + 8 * (col % 4);

    Walk<REL, G::BM, G::BN> walk;
    walk.begin(a, block, blocks);
    if (a.part && threadIdx.x == 0) {
        a.rec[2 * block] = int4{0, 0, 0, 0};
        a.rec[2 * block + 1] = int4{0, 0, 0, 0};
    }
    typename Walk<REL, G::BM, G::BN>::Piece pc;
    while (walk.next(a, pc)) {
        const Seq &s = walk.s;
        const int r0 = pc.j * G::BM;
        Source<REL> ks, vs;
        ks.set(a, a.src.k, walk.b, s, pc.head);
        vs.set(a, a.src.v, walk.b, s, pc.head);
        const Cells<REL> cells(a, walk.b);
        const int32_t keys = keys_of<REL>(a, s, min(r0 + G::BM, s.rows) - 1);
        const int32_t least = keys_of<REL>(a, s, r0);
        const int r = min(r0 + col, s.rows - 1);
        const int32_t seen = keys_of<REL>(a, s, r);
        u4 q[G::CH];
        {
            const u4 *p = reinterpret_cast<const u4 *>(a.q.p + row_at(a, a.q, walk.b, s, pc.head, r));
#pragma unroll
            for (int ch = 0; ch < G::CH; ++ch) q[ch] = p[ch * 4 + g];
        }
        ThinState<T, D> st;
#pragma unroll
        for (int db = 0; db < G::DB; ++db) st.o[db] = f4{0.0f, 0.0f, 0.0f, 0.0f};
        st.m = -__builtin_inff();
        st.l = 0.0f;
        if constexpr (REL == kBehind) {
            if (pc.starts && w == 0 && g == 0 && r0 + col < s.rows) st.l = open_row(a, cells, walk.b, s, pc.head, r0 + col);
        }

        // the step's first key; positions past the last key read that key (masked, and its value cleared)
        auto first = [&](int kt) { return (kt * kWaves + w) * G::KW; };
        auto at = [&](int kt, int i) { return min(first(kt) + i, keys - 1); };
        auto look_up = [&](int kt) {
            if constexpr (kPages<REL>) return cells.entry(a, at(min(kt, pc.t1 - 1), lane % G::KW));
            else return int32_t(0);
        };
        auto has = [&](int32_t entry) {
            if constexpr (kPages<REL>) return is_page(a.src, entry);
            else return true;
        };
        auto stage = [&](int kt, int32_t entry, u4 (&k)[G::KB][G::CH], uint8_t *vb) {
            const int32_t pages = kPages<REL> && !has(entry) ? -1 : entry;
#pragma unroll
            for (int e = 0; e < G::RUNS; ++e) {
                const int row = (e * 1024 + 16 * lane) / G::RB, ch = v_chunk<D>(row, (e * 1024 + 16 * lane) % G::RB / 16);
                const int32_t page = kPages<REL> ? __shfl(pages, row, kWave) : 0;
                const uint16_t *p = vs.at(at(kt, row), page);
                if (kPages<REL> && page < 0) p = reinterpret_cast<const uint16_t *>(kZeroRow);
                load_to_lds16(p + 8 * ch, vb + e * 1024);
            }
#pragma unroll
            for (int kb = 0; kb < G::KB; ++kb) {
                const int32_t page = kPages<REL> ? __shfl(pages, kb * 16 + col, kWave) : 0;
                const uint16_t *p = ks.at(at(kt, kb * 16 + col), page);
                if (kPages<REL> && page < 0) p = reinterpret_cast<const uint16_t *>(kNanRow);
#pragma unroll
                for (int ch = 0; ch < G::CH; ++ch) k[kb][ch] = reinterpret_cast<const u4 *>(p)[ch * 4 + g];
            }
        };
        // Loads of the step before the one just issued have arrived.  The issued ones may be in flight; a paged call's look-up
        // was issued before them, so it has arrived too.
        auto arrived = [&](bool more) {
            if (more) __asm__ volatile("s_waitcnt vmcnt(%0)" ::"i"(G::LOADS) : "memory");
            else __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
        };
        auto reads_done = [] { __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
        auto step = [&](int kt, const u4 (&k)[G::KB][G::CH], uint8_t *vb) {
            const int32_t k0 = first(kt);
            if (k0 < keys && k0 + G::KW > keys) {
#pragma unroll
                for (int e = 0; e < G::RUNS; ++e)
                    if ((e * 1024 + 16 * lane) / G::RB >= keys - k0) *reinterpret_cast<u4 *>(vb + e * 1024 + 16 * lane) = u4{0u, 0u, 0u, 0u};
            }
            if constexpr (kCausal<REL>) {
                if (least < keys && k0 < keys && k0 + G::KW > least) {
                    uint32_t bad = 0;
#pragma unroll
                    for (int e = 0; e < G::RUNS; ++e) bad |= any_wild<T>(*reinterpret_cast<const u4 *>(vb + e * 1024 + 16 * lane));
                    if (__any(bad != 0)) {
                        for (int i = 0; i < G::KW; ++i)
#pragma unroll
                            for (int db = 0; db < G::DB; ++db) {
                                const u2 x = *reinterpret_cast<const u2 *>(vb + i * G::RB + 16 * v_chunk<D>(i, 2 * db + g / 2) + 8 * (g % 2));
                                add_wild<T>(st.o[db], x, k0 + i < seen);
                            }
#pragma unroll
                        for (int e = 0; e < G::RUNS; ++e) {
                            u4 *const p = reinterpret_cast<u4 *>(vb + e * 1024 + 16 * lane);
                            *p = without_wild<T>(*p);
                        }
                    }
                }
            }
            if (k0 < keys) thin_step<T, D>(st, q, k, vb, vr, a.c, k0 + G::KW > least, seen - k0, g);
        };
        u4 ka[G::KB][G::CH], kb[G::KB][G::CH];
        if (pc.t0 < pc.t1) {
            int32_t pages = look_up(pc.t0), ahead = look_up(pc.t0 + 1);
            stage(pc.t0, pages, ka, v0);
            for (int kt = pc.t0; kt < pc.t1; kt += 2) {
                const bool more = kt + 1 < pc.t1;
                reads_done();
                pages = ahead;
                ahead = look_up(kt + 2);
                if (more) stage(kt + 1, pages, kb, v1);
                arrived(more);
                step(kt, ka, v0);
                if (!more) break;
                const bool more2 = kt + 2 < pc.t1;
                reads_done();
                pages = ahead;
                ahead = look_up(kt + 3);
                if (more2) stage(kt + 2, pages, ka, v0);
                arrived(more2);
                step(kt + 1, kb, v1);
            }
        }

        // join the four wavefronts' states
        const float lt = column_sum(st.l);
        reads_done();
        __syncthreads();
        float *const mine = reinterpret_cast<float *>(v0);
#pragma unroll
        for (int db = 0; db < G::DB; ++db)  // chunk c of row r at c ^ r (16 rows in one bank cost 0.8 us)
            *reinterpret_cast<f4 *>(mine + col * D + 4 * ((db * 4 + g) ^ col)) = st.o[db];
        if (g == 0) {
            ml[0][w][col] = st.m - kLift<T>;
            ml[1][w][col] = lt;
        }
        __syncthreads();
        const bool whole = pc.starts && pc.ends;
        const int slot = 2 * block + (pc.starts ? 1 : 0);
        if (!whole && threadIdx.x == 0) a.rec[slot] = int4{walk.b + 1, pc.head, pc.j, pc.ends ? 1 : 0};
        constexpr int E = G::BM * D / kThreads;  // widths a thread: 4 or 8
        const int tr = threadIdx.x * E / D, d0 = threadIdx.x * E % D;
        if (r0 + tr < s.rows) {
            float m = ml[0][0][tr], l = 0.0f, o[E];
#pragma unroll
            for (int i = 1; i < kWaves; ++i) m = fmaxf(m, ml[0][i][tr]);
            const float ref = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = 0.0f;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                const float f = __builtin_amdgcn_exp2f(ml[0][i][tr] - ref);
                l += f * ml[1][i][tr];
                const float *const p = reinterpret_cast<const float *>(v0of(i)) + tr * D;
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] += f * p[4 * ((d0 + e) / 4 ^ tr) + e % 4];
            }
            if (whole) {
                const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                auto *const yr = out_row<D, REL>(a, walk.b, s, pc.head, r0 + tr) + d0;
#pragma unroll
                for (int e = 0; e < E; e += 4) put<T>(yr + e, f4{o[e] * inv, o[e + 1] * inv, o[e + 2] * inv, o[e + 3] * inv});
                if (d0 == 0) put_lse(a, walk.b, s, pc.head, r0 + tr, ref + __log2f(l));
            } else {
                float *const po = a.part + slot * slot_floats<G::BM, D>();
#pragma unroll
                for (int e = 0; e < E; e += 4) *reinterpret_cast<f4 *>(po + tr * D + d0 + e) = f4{o[e], o[e + 1], o[e + 2], o[e + 3]};
                if (d0 == 0) {
                    po[G::BM * D + tr] = m;
                    po[G::BM * (D + 1) + tr] = l;
                }
            }
        }
        __syncthreads();  // the states are read before the next item's values arrive
    }
}

template <class T, int D, Relation REL>
__global__ __launch_bounds__(kThreads, 2) void thin_kernel(Args<REL> a) {
    constexpr int WAVE = kThinWave<D>;
    __shared__ __attribute__((aligned(1024))) uint8_t v0buf[kWaves * WAVE], v1buf[kWaves * WAVE];
    __shared__ float ml[2][kWaves][Thin<D>::BM];
    thin_pieces<T, D, REL>(a, static_cast<int>(xcd_block()), static_cast<int>(gridDim.x), [&](int i) { return v0buf + i * WAVE; },
                           [&](int i) { return v1buf + i * WAVE; }, ml);
    clear_outside<D, REL>(a);
}

// Joins the parts of the narrow item that starts in block x and ends in a later one (slot 1 of x, then slot 0 of the blocks
// after it up to the one that holds the end).  Its rows are spread over 4 blocks, a block's rows over its wavefronts (one,
// two or four a row).  The time is that of a few dependent reads of lines that other XCDs wrote, so 16 bytes a
// lane of 4 or (many parts) 16 parts a lane are in flight in every wavefront; the sums are added in a fixed order.
template <class T, int D, Relation REL>
__device__ __forceinline__ void thin_merge(const Args<REL> &a, int x, int y, int blocks, f4 (*so)[kWave], float (*sl)[kWave]) {
    constexpr int BM = Thin<D>::BM, L = D / 4, PP = kWave / L;  // L lanes a part, PP parts a wavefront's read
    const int4 it = a.rec[2 * x + 1];
    if (it.x == 0) return;
    const int b = it.x - 1, head = it.y, j = it.z;
    const Seq s = seq_of<REL>(a, b);
    const int rows = min(s.rows - j * BM, BM), per_block = (rows + kWaves - 1) / kWaves;
    if (y * per_block >= rows) return;
    const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave);
    const int share = per_block == 1 ? 4 : (per_block == 2 ? 2 : 1);  // wavefronts a row
    const int r = y * per_block + w / share, turn = w % share;
    const bool busy = w / share < per_block && r < rows;
    float m = -__builtin_inff(), l = 0.0f, ref = 0.0f;
    f4 o{0.0f, 0.0f, 0.0f, 0.0f};
    if (busy) {
        // 64 records at a time, then (many parts) 256
        auto ends_at = [&](int at) { return at >= blocks - 1 || a.rec[2 * at].w != 0; };
        int n = 0;
        uint64_t ends = __ballot(ends_at(x + 1 + lane));
        if (ends) n = __builtin_ctzll(ends) + 2;
        for (int from = x + 1 + kWave; n == 0; from += 4 * kWave) {
            bool hit[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) hit[i] = ends_at(from + i * kWave + lane);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                ends = __ballot(hit[i]);
                if (n == 0 && ends) n = from + i * kWave + __builtin_ctzll(ends) - x + 1;
            }
        }
        auto state = [&](int i) { return a.part + static_cast<int64_t>(2 * (x + i) + (i == 0 ? 1 : 0)) * slot_floats<BM, D>(); };
        for (int i0 = lane; i0 - lane < n; i0 += 4 * kWave) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = i0 + i * kWave < n ? state(i0 + i * kWave)[BM * D + r] : -__builtin_inff();
            m = fmaxf(fmaxf(m, fmaxf(v[0], v[1])), fmaxf(v[2], v[3]));
        }
        for (int d = 1; d < kWave; d <<= 1) m = fmaxf(m, shfl_xor_f(m, d));
        ref = m == -__builtin_inff() ? 0.0f : m;
        auto add = [&](auto u) {
            constexpr int U = decltype(u)::value;
            for (int i0 = turn * PP + lane / L; i0 - lane / L < n; i0 += U * share * PP) {
                f4 po[U];
                float pm[U], pl[U];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    po[i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
                    pm[i] = -__builtin_inff();
                    pl[i] = 0.0f;
                    const int part = i0 + i * share * PP;
                    if (part < n) {
                        const float *p = state(part);
                        po[i] = *reinterpret_cast<const f4 *>(p + r * D + 4 * (lane % L));
                        pm[i] = p[BM * D + r];
                        pl[i] = p[BM * (D + 1) + r];
                    }
                }
#pragma unroll
                for (int i = 0; i < U; ++i)
                    if (i0 + i * share * PP < n) {
                        const float f = __builtin_amdgcn_exp2f(pm[i] - ref);
                        o += po[i] * f;
                        l += pl[i] * f;
                    }
            }
        };
        if (n <= 4 * share * PP) add(std::integral_constant<int, 4>{});
        else add(std::integral_constant<int, 16>{});
    }
    so[w][lane] = o;
    sl[w][lane] = l;
    __syncthreads();
    if (!busy || turn != 0 || lane >= L) return;
    o = f4{0.0f, 0.0f, 0.0f, 0.0f};
    l = 0.0f;
    for (int i = w; i < w + share; ++i)
#pragma unroll
        for (int k = 0; k < PP; ++k) {
            o += so[i][k * L + lane];
            l += sl[i][k * L + lane];
        }
    o *= l == 0.0f ? 0.0f : 1.0f / l;
    put<T>(out_row<D, REL>(a, b, s, head, j * BM + r) + 4 * lane, o);
    if (lane == 0) put_lse(a, b, s, head, j * BM + r, ref + __log2f(l));
}

template <class T, int D, Relation REL>
__global__ __launch_bounds__(kThreads) void thin_merge_kernel(Args<REL> a, int blocks) {
    __shared__ f4 so[kWaves][kWave];
    __shared__ float sl[kWaves][kWave];
    // items start every few blocks: in every eighth, one XCD would join all
    thin_merge<T, D, REL>(a, static_cast<int>(xcd_block()), static_cast<int>(blockIdx.y), blocks, so, sl);
}

// Joins the parts of the wide item whose first part is in slot x: a wavefront takes 4 rows, 16 bytes a lane, the parts in
// order and 16 reads of accumulators in flight, rescaling into the common maximum as it goes.
template <class T, class G, Relation REL>
__device__ __forceinline__ void wide_merge(const Args<REL> &a, int x, int y) {
    constexpr int D = G::CPR * 8, BM = G::BM, L = D / 4, AT = kWave / L, N = 4 / AT, U = 16 / N;
    typedef Deal<REL, BM, G::BN> Pieces;
    const int4 it = a.rec[2 * x];
    if (it.x == 0) return;
    const int chunk = a.rec[2 * x + 1].x;
    const int b = it.x - 1, head = it.y, j = it.z, n = it.w;
    const Seq s = seq_of<REL>(a, b);
    const typename Pieces::Load load = Pieces::load(a, s);
    const int rows = min(s.rows - j * BM, BM);
    const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave);
    const int r0 = (y * kWaves + w) * 4;
    if (r0 >= rows) return;
    int row[N];  // rows r0 + 0..3: AT of them at a time
    float m[N], l[N];
    f4 o[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        row[k] = min(r0 + k * AT + lane / L, rows - 1);
        m[k] = -__builtin_inff();
        l[k] = 0.0f;
        o[k] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    int64_t slot = x;  // the parts of a row tile lie the chunk's row tiles apart
    for (int c = 0; c < n; c += U) {
        f4 po[U][N];
        float pm[U][N], pl[U][N];
#pragma unroll
        for (int i = 0; i < U; ++i) {  // past the last part: read again, not added
            const float *p = a.part + slot * slot_floats<BM, D>();
            if (c + i < n - 1) slot += Pieces::reach(a, load, c + i, chunk);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                pm[i][k] = p[BM * D + row[k]];
                pl[i][k] = p[BM * (D + 1) + row[k]];
                po[i][k] = *reinterpret_cast<const f4 *>(p + row[k] * D + 4 * (lane % L));
            }
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float top = m[k];
#pragma unroll
            for (int i = 0; i < U; ++i) top = fmaxf(top, pm[i][k]);
            const float ref = top == -__builtin_inff() ? 0.0f : top, alpha = __builtin_amdgcn_exp2f(m[k] - ref);
            m[k] = top;
            l[k] *= alpha;
            o[k] *= alpha;
#pragma unroll
            for (int i = 0; i < U; ++i) {
                if (c + i >= n) break;
                const float f = __builtin_amdgcn_exp2f(pm[i][k] - ref);
                l[k] += f * pl[i][k];
                o[k] += f * po[i][k];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int r = r0 + k * AT + lane / L;
        if (r >= rows) continue;
        const f4 v = o[k] * (l[k] == 0.0f ? 0.0f : 1.0f / l[k]);
        put<T>(out_row<D, REL>(a, b, s, head, j * BM + r) + 4 * (lane % L), v);
        if (lane % L == 0) put_lse(a, b, s, head, j * BM + r, m[k] + __log2f(l[k]));
    }
}

template <class T, class G, Relation REL>
__global__ __launch_bounds__(kThreads) void wide_merge_kernel(Args<REL> a) {
    wide_merge<T, G, REL>(a, static_cast<int>(blockIdx.x), static_cast<int>(blockIdx.y));
}

// Joins the parts of the planned item whose first part is piece x, kv_heads pieces apart: a wavefront takes the rows that it reads
// at once, the parts in order.
template <class T, class G>
__global__ __launch_bounds__(kThreads) void planned_merge_kernel(Args<kPlanned> a) {
    constexpr int D = G::CPR * 8, BM = G::BM, L = D / 4, AT = kWave / L, U = 8;
    const Item it = item_of(a.src.table, a.kv_heads, static_cast<int32_t>(a.group.d), static_cast<int32_t>(blockIdx.x));
    if (it.level == 0 || it.part != 0 || it.parts == 1) return;
    const Seq s{it.run.first, it.run.count * static_cast<int32_t>(a.group.d), 1};
    const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave), j = it.level - 1, rows = min(s.rows - j * BM, BM);
    for (int r0 = static_cast<int>(blockIdx.y) * kWaves + w; r0 * AT < rows; r0 += static_cast<int>(gridDim.y) * kWaves) {
        const int r = r0 * AT + lane / L, row = min(r, rows - 1);
        float m = -__builtin_inff(), l = 0.0f;
        f4 o{0.0f, 0.0f, 0.0f, 0.0f};
        for (int c = 0; c < it.parts; c += U) {
            f4 po[U];
            float pm[U], pl[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                pm[i] = -__builtin_inff();
                pl[i] = 0.0f;
                po[i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
                if (c + i < it.parts) {
                    const float *const p = a.part + (blockIdx.x + static_cast<int64_t>(c + i) * a.kv_heads) * slot_floats<BM, D>();
                    pm[i] = p[BM * D + row];
                    pl[i] = p[BM * (D + 1) + row];
                    po[i] = *reinterpret_cast<const f4 *>(p + row * D + 4 * (lane % L));
                }
            }
            float top = m;
#pragma unroll
            for (int i = 0; i < U; ++i) top = fmaxf(top, pm[i]);
            const float ref = top == -__builtin_inff() ? 0.0f : top, alpha = __builtin_amdgcn_exp2f(m - ref);
            m = top;
            l *= alpha;
            o *= alpha;
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const float f = __builtin_amdgcn_exp2f(pm[i] - ref);
                l += f * pl[i];
                o += f * po[i];
            }
        }
        if (r >= rows) continue;
        put<T>(out_row<D, kPlanned>(a, it.b, s, it.kv, j * BM + row) + 4 * (lane % L), o * (l == 0.0f ? 0.0f : 1.0f / l));
        if (lane % L == 0) put_lse(a, it.b, s, it.kv, j * BM + row, m + __log2f(l));
    }
}

// The slot of the n-th item that has parts, or -1.
template <Relation REL>
__device__ __forceinline__ int nth_item(const Args<REL> &a, int n) {
    constexpr int U = 8;
    for (int e = 0; e < a.slots; e += U * kWave) {
        int mine[U];
#pragma unroll
        for (int i = 0; i < U; ++i) mine[i] = e + i * kWave + lane_id() < a.slots ? a.rec[2 * (e + i * kWave + lane_id())].x : 0;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const uint64_t starts = __ballot(mine[i] != 0);
            const int here = __popcll(starts);
            if (n < here) {
                const int before = __popcll(starts & ((uint64_t(1) << lane_id()) - 1));
                return e + i * kWave + __builtin_ctzll(__ballot(mine[i] != 0 && before == n));
            }
            n -= here;
        }
    }
    return -1;
}

// Joins the parts of the n-th wide item of shared positions: there are few items (the rows of a group are one tile or two a
// head) of many parts, so a block takes twice the rows that a wavefront reads at once, and each wavefront half of the parts of
// one of them; the halves are joined in order.
template <class G>
constexpr int kSharedRows = 2 * kWave / (G::CPR * 2);  // of a block
template <class T, class G>
__device__ __forceinline__ void shared_merge(const Args<kShared> &a, int nth, int y, f4 (*so)[kWave], float (*sl)[kWave]) {
    constexpr int D = G::CPR * 8, BM = G::BM, L = D / 4, AT = kWave / L, U = 8, H = 2;
    static_assert(kSharedRows<G> == AT * (kWaves / H), "a block's rows");
    __shared__ float sm[kWaves][AT];
    __shared__ int slot;
    if (threadIdx.x < kWave) {
        const int mine = nth_item(a, nth);
        if (threadIdx.x == 0) slot = mine;
    }
    __syncthreads();
    const int x = uniform(slot);
    if (x < 0) return;
    const int4 it = a.rec[2 * x], of = a.rec[2 * x + 1];
    const int b = it.x - 1, head = it.y, j = it.z, n = it.w;
    const Seq s{of.y, of.z, 0};
    const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave), half = w % H;
    const int rows = min(s.rows - j * BM, BM), r = (y * (kWaves / H) + w / H) * AT + lane / L;
    const int row = min(r, rows - 1), tiles = (s.rows + BM - 1) / BM;  // the parts of a row tile lie `tiles` apart
    float m = -__builtin_inff(), l = 0.0f;
    f4 o{0.0f, 0.0f, 0.0f, 0.0f};
    const int last = n * (half + 1) / H;
    for (int c = n * half / H; c < last; c += U) {
        f4 po[U];
        float pm[U], pl[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            pm[i] = -__builtin_inff();
            pl[i] = 0.0f;
            po[i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
            if (c + i < last) {
                const float *const p = a.part + (x + static_cast<int64_t>(c + i) * tiles) * slot_floats<BM, D>();
                pm[i] = p[BM * D + row];
                pl[i] = p[BM * (D + 1) + row];
                po[i] = *reinterpret_cast<const f4 *>(p + row * D + 4 * (lane % L));
            }
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < U; ++i) top = fmaxf(top, pm[i]);
        const float ref = top == -__builtin_inff() ? 0.0f : top, alpha = __builtin_amdgcn_exp2f(m - ref);
        m = top;
        l *= alpha;
        o *= alpha;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const float f = __builtin_amdgcn_exp2f(pm[i] - ref);
            l += f * pl[i];
            o += f * po[i];
        }
    }
    so[w][lane] = o;
    if (lane % L == 0) {
        sm[w][lane / L] = m;
        sl[w][lane / L] = l;
    }
    __syncthreads();
    if (half != 0 || r >= rows) return;
    for (int i = 1; i < H; ++i) m = fmaxf(m, sm[w + i][lane / L]);
    const float ref = m == -__builtin_inff() ? 0.0f : m;
    l = 0.0f;
    o = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < H; ++i) {
        const float f = __builtin_amdgcn_exp2f(sm[w + i][lane / L] - ref);
        l += f * sl[w + i][lane / L];
        o += so[w + i][lane] * f;
    }
    put<T>(out_row<D, kShared>(a, b, s, head, j * BM + row) + 4 * (lane % L), o * (l == 0.0f ? 0.0f : 1.0f / l));
    if (lane % L == 0) put_lse(a, b, s, head, j * BM + row, m + __log2f(l));
}

// ------------------------------------------------------------------------------------------ launch

// How a call is laid out, from what the host knows: sizes and upper bounds of the lengths.
struct Plan {
    int64_t blocks;  // of the main kernel and (narrow) of the merge
    int64_t slots;   // partial states, 0: items are not cut
    int64_t items;   // at most
};
template <class G>
int64_t steps_of(int64_t longest) { return ceil_div(longest < 1 ? 1 : longest, G::BN); }
template <class G>
constexpr bool kNarrow = G::BM < 128;

// items: at most, and at least (where the rows are packed the host knows bounds only); alike: all of `longest` keys
template <class G>
Plan plan_for(int64_t most, int64_t least, int64_t longest, bool alike) {
    const int64_t resident = 2 * static_cast<int64_t>(device_cus()), steps = steps_of<G>(longest);
    Plan p{most, 0, most};
    if (kNarrow<G>) {
        // equal runs for the resident blocks, two slots a block; items of one key tile are dealt whole
        p.blocks = most * steps < resident ? most * steps : resident;
        if (steps > 1) p.slots = 2 * p.blocks;
    } else {
        // cut where there are fewer items than blocks, of more than one chunk (alike: where two parts of all fit)
        if (steps > kLeastChunk && least <= resident && !(alike && 2 * most > resident)) p.slots = resident;
        if (p.blocks < p.slots) p.blocks = p.slots;
        if (p.blocks > (1 << 20)) p.blocks = 1 << 20;
        p.blocks = (p.blocks + kXcds - 1) / kXcds * kXcds;
    }
    return p;
}

// The workspace of `slots` partial states.
struct Parts {
    float *part;
    int4 *rec;
    size_t bytes;
};
template <class G>
Parts carve(void *ws, int64_t slots) {
    Carve c(ws);
    Parts p;
    p.part = c.take<float>(slots * slot_floats<G::BM, G::CPR * 8>());
    p.rec = c.take<int4>(2 * slots);
    p.bytes = c.bytes() < 256 ? 256 : c.bytes();
    return p;
}

// The tile shape: narrow where a sequence has at most 16 rows for a source head (on average, where the host does not know
// more).  Narrow against wide in us, width 128, 4 source heads: at 16 rows 35 and 34 (16 x 4096 keys), 91 and 98 (2 x
// 100,000), 15 and 20 (1 x 4001); at 24 rows 42 and 37, 138 and 99, 16 and 20, where a narrow tile reads the keys twice.
// Unequal sequences that fill the device uncut (64 of up to 8192 keys, 8 heads): 156 and 235 at 4 rows; cut ones (63 of up to
// 4096 keys, 4 heads) 71 and 67.  The mean is no good guide where a chunk stands beside single tokens: 63 of them and a chunk
// of 190, 4 rows to a token, up to 4096 keys 110 (narrow, mean 16) and 81, up to 16,384 keys 364 and 247; a chunk of 260,
// which the mean makes wide, 119 and 91.
constexpr int64_t kThinRows = 16;

template <class F>
auto by_type(int dtype, int width, bool thin, F f) {
    auto go = [&](auto t) {
        if (width == 64) return thin ? f(t, Thin<64>{}) : f(t, Geo<64>{});
        return thin ? f(t, Thin<128>{}) : f(t, Geo<128>{});
    };
    return dtype == TIGA_DT_F16 ? go(Half16{}) : go(Brain16{});
}

template <class T, class G, Relation REL>
int run(const Plan &p, Args<REL> a, void *ws, hipStream_t stream) {
    constexpr int D = G::CPR * 8;
    if (p.slots) {
        const Parts w = carve<G>(ws, p.slots);
        a.part = w.part;
        a.rec = w.rec;
        a.slots = static_cast<int>(p.slots);
    }
    prof_before(stream);
    const dim3 grid(static_cast<unsigned>(p.blocks));
    if constexpr (kNarrow<G>) hipLaunchKernelGGL((thin_kernel<T, D, REL>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((wide_kernel<T, D, REL>), grid, dim3(kThreads), 0, stream, a);
    prof_after(stream);
    if (int rc = check_launch("attention forward")) return rc;
    if (!p.slots) return TIGA_OK;
    if constexpr (kNarrow<G>)
        hipLaunchKernelGGL((thin_merge_kernel<T, D, REL>), dim3(static_cast<unsigned>(p.blocks), kWaves), dim3(kThreads), 0,
                           stream, a, static_cast<int>(p.blocks));
    else
        hipLaunchKernelGGL((wide_merge_kernel<T, G, REL>), dim3(static_cast<unsigned>(p.slots), G::BM / 16), dim3(kThreads), 0,
                           stream, a);
    return check_launch("attention merge");
}

// Workspaces hold every smaller problem. Fewer source heads at the same heads turn narrow tiles wide, and so do fewer sequences
// of packed rows: unless all heads' rows together are few, the wide tiles' slots are asked for, whether the items are
// cut or not.
template <class F>
size_t ws_bytes(int dtype, int width, int64_t rows, int64_t longest, F thin_slots) {
    const bool narrow = rows <= kThinRows;  // of one source head if it has all heads
    const size_t wide = by_type(dtype, width, false, [&](auto, auto g) {
        typedef decltype(g) G;
        return carve<G>(nullptr, !narrow && steps_of<G>(longest) > 1 ? 2 * device_cus() : 0).bytes;
    });
    const size_t thin = by_type(dtype, width, true, [&](auto, auto g) {
        typedef decltype(g) G;
        return carve<G>(nullptr, thin_slots(g)).bytes;
    });
    return wide > thin ? wide : thin;
}

}  // namespace

}  // namespace relattn
}  // namespace tiga
