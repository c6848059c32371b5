// The order in which the tiles of packed sequences are worked on.  A causal sequence's tiles of 128 rows (or keys) need work
// that grows linearly along it, so those with most to do start first, of all sequences and heads, and those that are longer
// than a block's share of all work (one long sequence, few heads) are cut into parts of at most that.  A launch of its own
// finds the order from the sequences' bounds on the device and leaves a table of pieces.
#pragma once

#include "relation.hpp"

namespace tiga {
namespace relattn {

namespace {

constexpr int kTileRows = 128, kPlanThreads = 256;

// An owned tile of a sequence: `level` is how many tiles of the sequence it has to go with itself, of `tiles`.
struct Item {
    Run run;
    int32_t b, kv, level, tiles;  // level 0: there is no such item
    int32_t part, parts;
};
// The pieces of one kind of owned tiles, of 128 / mult tokens: every source head has those of the table.
struct Pieces {
    int4 *table;       // [places][2]: first, count, b, level; part, parts
    int32_t places, mult;
    int32_t resident;  // blocks that run at once
    int32_t least;     // levels of a part, at least (kNoCut: nothing is cut)
    int32_t quarters;  // of a block's share of all levels, that a part has
};
constexpr int32_t kNoCut = 1 << 30;
// Items are cut into parts of at most `cut` levels.  How many pieces the items of the first m levels make:
__device__ __forceinline__ int64_t pieces_upto(int32_t m, int32_t cut) {
    if (m <= cut) return m;
    const uint32_t q = static_cast<uint32_t>(m) / static_cast<uint32_t>(cut), r = static_cast<uint32_t>(m) - q * cut;
    return static_cast<int64_t>(q) * (q + 1) / 2 * cut + static_cast<int64_t>(r) * (q + 1);
}
// Writes the tables.  Sequences are taken 64 at a time (blockIdx.x), whose places start at or behind what the sequences before
// them need at most.  Of 64, the tiles with the most levels come first: a piece of level L stands behind the sum of
// pieces_upto(tiles) - pieces_upto(L) of those with more.  Batches of more than 64 are not cut, whose 64 at a time do not know the
// others' work: a long sequence of few heads is slow among them (dq, dk and dv of one of 10,000 tokens, 4 heads over one of 128,
// beside 63 of 50 tokens 458 us, beside 64 of them 1412).  (Every block finding its own piece so took 12 us of each kernel's 49
// to 65 for 100 short sequences of 16 heads.)
__global__ __launch_bounds__(kPlanThreads) void packed_plan_kernel(const int32_t *ptr, int32_t num_rows, int32_t batch, int32_t kv_heads,
                                                               Pieces by_rows, Pieces by_keys) {
    const Pieces p = blockIdx.z == 0 ? by_rows : by_keys;
    const int lane = lane_id(), base = static_cast<int>(blockIdx.x) * kWave;
    __shared__ int32_t tiles_of[kWave], before[kWave + 1], first_of[kWave], count_of[kWave];
    __shared__ int64_t pieces_of[kWave];
    auto start = [&](int chunk) {
        if (chunk == 0) return 0;
        if (chunk * kWave >= batch) return p.places;
        int32_t s = ptr[chunk * kWave];
        s = s < 0 ? 0 : (s > num_rows ? num_rows : s);
        return min(static_cast<int32_t>(static_cast<int64_t>(s) * p.mult / kTileRows) + chunk * kWave, p.places);
    };
    const int32_t s0 = start(static_cast<int>(blockIdx.x)), s1 = start(static_cast<int>(blockIdx.x) + 1);
    const Run mine = base + lane < batch ? run_between(ptr, base + lane, base + lane + 1, num_rows) : Run{0, 0};
    const int32_t tiles = static_cast<int32_t>((static_cast<int64_t>(mine.count) * p.mult + kTileRows - 1) / kTileRows);
    auto all = [&](int64_t x) { return lane_value(wave_prefix(x), kWave - 1); };
    int32_t cut = kNoCut;
    if (p.least < kNoCut && __any(tiles > p.least)) {
        // Parts of half a block's share of all levels, or of as much more as makes at most two pieces a block, up to the whole
        // share, which makes at most twice as many parts as blocks run at once.  (dk and dv of 10,000 tokens, 4 heads over one
        // of 128: 272 us, 387 with whole shares; 1.3 ms uncut.)  The forward, whose parts are joined at more cost, takes 5/4:
        // 4000 tokens, 16 heads over 2, 90 us and 18 to join with halves, 90 + 16 with 5/4, 91 + 12 with 3/2; 8000, 8 over 8, 164 + 18,
        // 162 + 14, 169 + 11; 10,000, 4 over one, 123 + 20, 129 + 13, 141 + 13.
        const int64_t levels = all(static_cast<int64_t>(tiles) * (tiles + 1) / 2) * kv_heads;
        const int64_t share = min(static_cast<int64_t>(kNoCut) - 1, max(static_cast<int64_t>(p.least), quotient(levels + p.resident - 1, p.resident)));
        const int64_t most = share * max(p.quarters, 4) / 4;
        int64_t c = max(static_cast<int64_t>(p.least), (share * p.quarters + 3) / 4);
        while (c < share && all(pieces_upto(tiles, static_cast<int32_t>(c))) * kv_heads > 2 * p.resident) c += c / 16 + 1;
        cut = static_cast<int32_t>(min(c, most));
    }
    const int64_t pieces = pieces_upto(tiles, cut);
    int64_t total = all(pieces);
    if (total > s1 - s0) total = 0;  // pointers that run backwards: nothing is done
    const int64_t incl = wave_prefix(tiles);
    if (threadIdx.x < kWave) {
        tiles_of[lane] = tiles;
        pieces_of[lane] = pieces;
        before[lane + 1] = static_cast<int32_t>(incl);
        if (lane == 0) before[0] = 0;
        first_of[lane] = mine.first;
        count_of[lane] = mine.count;
    }
    __syncthreads();
    const int here = min(batch - base, kWave);
    for (int32_t s = s0 + static_cast<int32_t>(blockIdx.y) * kPlanThreads + threadIdx.x; s < s1; s += static_cast<int32_t>(gridDim.y) * kPlanThreads) {
        const int32_t r = s - s0;
        if (r >= total) {
            p.table[2 * s] = int4{0, 0, 0, 0};
            continue;
        }
        if (r >= before[kWave]) continue;
        int lo = 0, hi = kWave - 1;  // the r-th tile's sequence
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (before[mid] <= r) lo = mid;
            else hi = mid - 1;
        }
        const int32_t level = r - before[lo] + 1, parts = level <= cut ? 1 : (level + cut - 1) / cut;
        const int64_t upto = pieces_upto(level, cut);
        int64_t place = 0;
#pragma unroll 4
        for (int i = 0; i < here; ++i) {
            if (tiles_of[i] > level) place += pieces_of[i] - upto;
            if (i < lo && tiles_of[i] >= level) place += parts;
        }
        for (int32_t e = 0; e < parts; ++e) {
            const int64_t at = s0 + place + e;
            p.table[2 * at] = int4{first_of[lo], count_of[lo], base + lo, level};
            p.table[2 * at + 1] = int4{e, parts, 0, 0};
        }
    }
}
// Piece id: those of a source head are kv_heads apart.  mult: 128 / tokens of a tile, as in the table's Pieces.
__device__ __forceinline__ Item item_of(const int4 *table, int kv_heads, int32_t mult, int32_t id) {
    const int32_t n = id / kv_heads;
    const int4 x = table[2 * n], y = table[2 * n + 1];
    const int32_t tiles = static_cast<int32_t>((static_cast<int64_t>(x.y) * mult + kTileRows - 1) / kTileRows);
    return Item{Run{x.x, x.y}, x.z, id - n * kv_heads, x.w > tiles ? 0 : x.w, tiles, y.x, y.y};
}
// The streamed steps of a part.
__device__ __forceinline__ int32_t part_start(int32_t steps, int32_t part, int32_t parts) {
    return static_cast<int32_t>(static_cast<int64_t>(steps) * part / parts);
}
// Items of tiles of 128 / mult tokens, at most, not cut.
int64_t most_items(const tiga_packed &rel, int64_t mult) {
    const int64_t some = rel.num_rows < rel.batch ? rel.num_rows : rel.batch;
    return (rel.num_rows * mult / kTileRows + (rel.batch > kWave ? rel.batch : some)) * rel.kv_heads;
}
// The tables of one or two kinds of tiles.
int plan_pieces(const tiga_packed &rel, const Pieces &one, const Pieces &two, int kinds, hipStream_t stream) {
    const int64_t chunks = ceil_div(rel.batch, kWave), places = kinds > 1 && two.places > one.places ? two.places : one.places;
    int64_t turns = rel.batch <= kWave ? ceil_div(places, kPlanThreads) : 4;
    if (turns > 256) turns = 256;
    hipLaunchKernelGGL(packed_plan_kernel, dim3(static_cast<unsigned>(chunks < 1 ? 1 : chunks), static_cast<unsigned>(turns < 1 ? 1 : turns), kinds),
                       dim3(kPlanThreads), 0, stream, rel.ptr, static_cast<int32_t>(rel.num_rows), rel.batch, rel.kv_heads, one, two);
    return check_launch("packed attention, plan");
}

}  // namespace

}  // namespace relattn
}  // namespace tiga
