// Eviction from a paged cache: of every sequence and source head the `keep` positions of the largest weights stay, the last
// `recent` ones among them whatever theirs, ties by the lowest position, and move in order into another cache's pages.
//
// Selection: a block for a sequence and head, which holds the weights in registers as integers of the same order, finds the
// least one that stays by its digits of 8 bits from the top (a histogram in LDS, 16 copies of each counter so that equal
// digits of a wavefront's lanes seldom wait for each other), and lists the positions that stay by prefix sums.  A wavefront
// owns a contiguous run of positions, so the list needs one exchange between wavefronts.  Long sequences, over which one
// block would take long, are shared by blocks of 8192 positions, which exchange their digits' counts (of 11 bits) by way of the
// workspace in three launches before the one that lists.
// Move: 16 bytes a lane, keys and values of a listed position to its new place; bound by the memory.
//
// Measured (MI355X), selection + move in us: 512 of 545 positions, 4 heads of width 64: 8.3 + 5.7, latency; 2048 of up to 2500,
// 64 sequences, 8 heads of width 128: 14.7 + 232 for 1048 MB, 4.5 TB/s (a large copy moves 4.8); 16,384 of two times up to
// 131,072 positions, 8 heads: 5 + 7 + 7 + 13 in four launches + 63 for 278 MB.
#include "mfma16.hpp"
#include "relation.hpp"
#include "retention.hpp"

namespace tiga {
namespace retention {

using namespace relattn;

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;

struct Args {
    Pages from;
    const float *weights;  // [num_pages, kv_heads, page_size]
    int kv_heads;
    int32_t keep, recent;
    int32_t *kept;         // [batch, kv_heads, keep]
};

__device__ __forceinline__ int32_t positions(const Pages &c, int b) {
    const int64_t n = c.length[b], most = static_cast<int64_t>(c.table_width) << c.shift;
    return static_cast<int32_t>(n < 0 ? 0 : (n > most ? most : n));
}

// An integer in the order of the weights: NaN above all, -0 as 0.  0 (no number's) is for a position without a page.
__device__ __forceinline__ uint32_t ordered(float w) {
    if (w != w) return 0xffffffffu;
    const uint32_t x = __float_as_uint(w + 0.0f);
    return x & 0x80000000u ? ~x : x | 0x80000000u;
}

// Sum over the wavefront before this lane; all: over the whole.
__device__ __forceinline__ int32_t lanes_before(int32_t v, int32_t &all) {
    const int64_t incl = wave_prefix(v);
    all = static_cast<int32_t>(lane_value(incl, kWave - 1));
    return static_cast<int32_t>(incl) - v;
}

// A sequence's positions and which of them are candidates: the last `last` stay whatever their weights.
struct Span {
    int32_t n, stay, last, first_recent;
    __device__ __forceinline__ Span(const Args &a, int b)
        : n(positions(a.from, b)), stay(min(n, a.keep)), last(min(a.recent, stay)), first_recent(n - last) {}
};

// A wavefront's weights as integers: `per` groups of 256 positions from `start` on, four neighbouring ones a lane.  PER: the
// most that are held in registers; 0: as many as there are, read again in every turn.
template <int PER>
struct Held {
    u4 x[PER > 0 ? PER : 1];
    int32_t start, per, b, head;
    const Span &span;
    __device__ __forceinline__ Held(const Args &a, const Span &s, int32_t b, int32_t head, int32_t start, int32_t per)
        : start(start), per(per), b(b), head(head), span(s) {
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (j < per) x[j] = read(a, j);
    }
    __device__ __forceinline__ int32_t first(int32_t j) const { return start + j * 256 + lane_id() * 4; }
    __device__ __forceinline__ u4 read(const Args &a, int32_t j) const {
        const int32_t at = first(j), mask = (1 << a.from.shift) - 1;
        u4 v{0u, 0u, 0u, 0u};
        auto cell = [&](int32_t page, int32_t at) {
            return ((static_cast<int64_t>(page) * a.kv_heads + head) << a.from.shift) + (at & mask);
        };
        if (at >= span.first_recent) return v;
        if (mask >= 3) {
            const int32_t page = page_at(a.from, b, at);
            if (page < 0) return v;
            const f4 w = *reinterpret_cast<const f4 *>(a.weights + cell(page, at));
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = ordered(w[e]);
            return v;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + e < span.first_recent) {
                const int32_t page = page_at(a.from, b, at + e);
                v[e] = page < 0 ? 0u : ordered(a.weights[cell(page, at + e)]);
            }
        return v;
    }
    // f(four weights, the first one's position)
    template <class F>
    __device__ __forceinline__ void each(const Args &a, F f) const {
        if constexpr (PER > 0) {
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (j < per) f(x[j], first(j));
        } else {
            for (int32_t j = 0; j < per; ++j) f(read(a, j), first(j));
        }
    }
    // Adds up the digits of those candidates that agree with `least` in the bits of `upper`.
    template <int COPIES>
    __device__ __forceinline__ void count(const Args &a, int32_t *counts, int shift, uint32_t digits, uint32_t upper, uint32_t least) const {
        each(a, [&](u4 v, int32_t at) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (at + e < span.first_recent && (v[e] & upper) == least)
                    atomicAdd(&counts[(v[e] >> shift & digits) * COPIES + lane_id() % COPIES], 1);
        });
    }
    // Whether a position stays for its weight or its place (more), or if it is one of the first of those with the least weight.
    __device__ __forceinline__ void sort_out(int32_t at, uint32_t v, uint32_t least, bool &more, bool &equal) const {
        const bool old = at < span.first_recent, some = span.stay > span.last;
        more = at < span.n && (!old || (some && v > least));
        equal = old && some && v == least;
    }
    // Lists the positions that stay, of which `mores` and `equals` lie in blocks before.
    __device__ __forceinline__ void list(const Args &a, uint32_t least, int32_t need, int32_t mores, int32_t equals,
                                         int32_t (*totals)[kWaves], int32_t *kept) const {
        const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave);
        int32_t m = 0, q = 0, all_m, all_q;
        each(a, [&](u4 v, int32_t at) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                bool more, equal;
                sort_out(at + e, v[e], least, more, equal);
                m += more;
                q += equal;
            }
        });
        lanes_before(m, all_m);
        lanes_before(q, all_q);
        if (lane == 0) {
            totals[0][w] = all_m;
            totals[1][w] = all_q;
        }
        __syncthreads();
        for (int i = 0; i < w; ++i) {
            mores += totals[0][i];
            equals += totals[1][i];
        }
        each(a, [&](u4 v, int32_t at) {
            bool more[4], equal[4];
            m = q = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sort_out(at + e, v[e], least, more[e], equal[e]);
                m += more[e];
                q += equal[e];
            }
            int32_t before_m = mores + lanes_before(m, all_m), before_q = equals + lanes_before(q, all_q);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (more[e] || (equal[e] && before_q < need)) kept[before_m + min(before_q, need)] = at + e;
                before_m += more[e];
                before_q += equal[e];
            }
            mores += all_m;
            equals += all_q;
        });
    }
};

// The whole list of a sequence that has no more positions than stay, and what is behind a list: this thread's share of them.
// (In 64 bits: lists may be as long as 32 bits count, and the step past their end is longer.)
__device__ __forceinline__ bool list_all(const Args &a, const Span &s, int32_t *kept, int32_t thread, int32_t threads) {
    for (int64_t i = static_cast<int64_t>(s.stay) + thread; i < a.keep; i += threads) kept[i] = -1;
    if (s.n > a.keep) return false;
    for (int64_t i = thread; i < s.n; i += threads) kept[i] = static_cast<int32_t>(i);
    return true;
}

template <int PER>
__global__ __launch_bounds__(kThreads) void select_kernel(Args a) {
    constexpr int kCopies = 16;
    __shared__ int32_t count[256 * kCopies];
    __shared__ int32_t found[2], totals[2][kWaves];
    const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave);
    const int b = static_cast<int>(blockIdx.x) / a.kv_heads, head = static_cast<int>(blockIdx.x) % a.kv_heads;
    const Span span(a, b);
    int32_t *const kept = a.kept + static_cast<int64_t>(blockIdx.x) * a.keep;
    if (list_all(a, span, kept, static_cast<int32_t>(threadIdx.x), kThreads)) return;
    // at most 2^19, so that positions up to the end of the last group are below 2^31 (n + 4095 need not be)
    const int32_t per = (span.n - 1) / (kWaves * 256) + 1;
    const Held<PER> held(a, span, b, head, w * per * 256, per);

    // the least weight that stays, from its digits, and how many equal ones stay
    uint32_t least = 0;
    int32_t need = span.stay - span.last;  // of those that agree with `least` so far
    if (need > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = threadIdx.x; i < 256 * kCopies; i += kThreads) count[i] = 0;
            __syncthreads();
            held.template count<kCopies>(a, count, shift, 255u, shift == 24 ? 0u : 0xffffffffu << (shift + 8), least);
            __syncthreads();
            if (w == 0) {  // lane l has digits 255 - 4 l and the three below
                int32_t c[4], sum = 0, all;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    c[e] = 0;
#pragma unroll
                    for (int i = 0; i < kCopies; i += 4) {
                        const i32x4 x = *reinterpret_cast<const i32x4 *>(&count[(255 - 4 * lane - e) * kCopies + i]);
                        c[e] += (x[0] + x[1]) + (x[2] + x[3]);
                    }
                    sum += c[e];
                }
                int32_t above = lanes_before(sum, all);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (above < need && above + c[e] >= need) {
                        found[0] = 255 - 4 * lane - e;
                        found[1] = need - above;
                    }
                    above += c[e];
                }
            }
            __syncthreads();
            least |= static_cast<uint32_t>(found[0]) << shift;
            need = found[1];
        }
    }
    held.list(a, least, need, 0, 0, totals, kept);
}

// ------------------------------------------------------------------------------------------ long sequences

constexpr int kPer = 2, kSegment = kWaves * 256 * kPer;  // positions of a block
// Digits of 11, 11 and 10 bits; the counts of a block in order: [2048], [2048], [1024].
constexpr int kLevels = 3, kBins = 2048, kCounts = 2 * kBins + 1024;
__device__ __forceinline__ int shift_of(int level) { return level == 0 ? 21 : level == 1 ? 10 : 0; }
__device__ __forceinline__ int bins_of(int level) { return level == 2 ? 1024 : kBins; }
struct Shared1 {
    uint16_t *counts;  // [sequence and head][segment][kCounts]
    int2 *found;       // [sequence and head][kLevels]: digit, how many with it stay
    int32_t segments;  // of the longest sequence
};

// Level 0, 1, 2: the counts of a digit, after finding the one before; level 3: the list.
template <int LEVEL>
__global__ __launch_bounds__(kThreads) void segment_kernel(Args a, Shared1 sh) {
    constexpr int kCopies = 4;
    __shared__ __attribute__((aligned(16))) int32_t count[kBins * kCopies];
    __shared__ int32_t found[2], sums[kWaves], totals[2][kWaves];
    const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave), t = static_cast<int>(threadIdx.x);
    const int bh = static_cast<int>(blockIdx.y), b = bh / a.kv_heads, head = bh % a.kv_heads, seg = static_cast<int>(blockIdx.x);
    const Span span(a, b);
    int32_t *const kept = a.kept + static_cast<int64_t>(bh) * a.keep;
    if (LEVEL == kLevels) {
        if (list_all(a, span, kept, seg * kThreads + t, sh.segments * kThreads)) return;
    } else if (span.n <= a.keep) {
        return;
    }
    const int32_t segs = (span.n + kSegment - 1) / kSegment;
    if (seg >= segs) return;
    const Held<kPer> held(a, span, b, head, seg * kSegment + w * kPer * 256, kPer);
    uint16_t *const counts = sh.counts + static_cast<int64_t>(bh) * sh.segments * kCounts;
    int32_t need = span.stay - span.last;
    uint32_t least = 0;
    int digit[kLevels] = {0, 0, 0};
    if (need > 0) {
        // the digits that earlier launches found, and the one of the last launch's counts
#pragma unroll
        for (int level = 0; level < LEVEL; ++level) {
            const int bins = bins_of(level);
            if (level < LEVEL - 1) {
                const int2 f = sh.found[bh * kLevels + level];
                digit[level] = f.x;
                need = f.y;
            } else {
                // thread t has digits bins - 1 - 2 t and the one below
                int32_t c[2] = {0, 0};
                if (2 * t < bins) {
                    const uint16_t *const p = counts + level * kBins + bins - 2 - 2 * t;
#pragma unroll 8
                    for (int s = 0; s < segs; ++s) {
                        const uint32_t x = *reinterpret_cast<const uint32_t *>(p + static_cast<int64_t>(s) * kCounts);
                        c[0] += x >> 16;
                        c[1] += x & 0xffffu;
                    }
                }
                int32_t all;
                int32_t above = lanes_before(c[0] + c[1], all);
                if (lane == 0) sums[w] = all;
                __syncthreads();
                for (int i = 0; i < w; ++i) above += sums[i];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    if (above < need && above + c[e] >= need) {
                        found[0] = bins - 1 - 2 * t - e;
                        found[1] = need - above;
                    }
                    above += c[e];
                }
                __syncthreads();
                digit[level] = found[0];
                need = found[1];
                if (seg == 0 && t == 0) sh.found[bh * kLevels + level] = int2{digit[level], need};
            }
            least |= static_cast<uint32_t>(digit[level]) << shift_of(level);
        }
    }
    if constexpr (LEVEL < kLevels) {
        const int bins = bins_of(LEVEL);
        for (int i = t; i < bins * kCopies / 4; i += kThreads) reinterpret_cast<i32x4 *>(count)[i] = i32x4{0, 0, 0, 0};
        __syncthreads();
        held.template count<kCopies>(a, count, shift_of(LEVEL), bins - 1, LEVEL == 0 ? 0u : 0xffffffffu << shift_of(LEVEL - 1), least);
        __syncthreads();
        uint16_t *const mine = counts + static_cast<int64_t>(seg) * kCounts + LEVEL * kBins;
        for (int i = t; i < bins; i += kThreads) {
            const i32x4 x = reinterpret_cast<const i32x4 *>(count)[i];
            mine[i] = static_cast<uint16_t>((x[0] + x[1]) + (x[2] + x[3]));  // at most kSegment
        }
    } else {
        // what the segments before this one keep: larger digits at each level, and the least weight's equals
        int32_t mores = 0, equals = 0;
        if (span.stay > span.last) {
            const u4 *const p = reinterpret_cast<const u4 *>(counts);  // the segments' counts one after the other, 8 a load
#pragma unroll 4
            for (int32_t i = t; i < seg * (kCounts / 8); i += kThreads) {
                const u4 x = p[i];
                const int at = i % (kCounts / 8) * 8, level = at / kBins, bin = at - level * kBins;
                const int own = level == 0 ? digit[0] : level == 1 ? digit[1] : digit[2];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int32_t n = x[e / 2] >> (16 * (e % 2)) & 0xffffu;
                    mores += bin + e > own ? n : 0;
                    equals += level == kLevels - 1 && bin + e == own ? n : 0;
                }
            }
        }
        int32_t all_m, all_q;
        lanes_before(mores, all_m);
        lanes_before(equals, all_q);
        if (lane == 0) {
            totals[0][w] = all_m;
            totals[1][w] = all_q;
        }
        __syncthreads();
        mores = max(0, seg * kSegment - span.first_recent);  // the recent positions of the segments before
        equals = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            mores += totals[0][i];
            equals += totals[1][i];
        }
        __syncthreads();
        held.list(a, least, need, mores, equals, totals, kept);
    }
}

// ------------------------------------------------------------------------------------------ move

struct Move {
    Pages from, to;
    const int32_t *kept;
    const float *weights;
    float *to_weights;
    int32_t *to_length;
    int kv_heads;
    int32_t keep;
    int64_t rows;  // batch * kv_heads * keep
    // staged rows in order: keys and values [rows, 2, D] and weights [rows]
    uint16_t *staged;
    float *staged_weights;
};

// How a row travels: from page to page, from its page to the staged rows, from there to its page.
enum Way { kThrough, kOut, kIn };

template <int D, Way WAY>
__global__ __launch_bounds__(256) void move_kernel(Move m) {
    constexpr int L = D / 8, U = 4;  // lanes a row, rows a lane in flight
    const int c = static_cast<int>(threadIdx.x) % L;
    if (WAY != kOut)
        for (int b = blockIdx.x * 256 + threadIdx.x; b < m.from.batch; b += gridDim.x * 256)
            m.to_length[b] = min(positions(m.from, b), m.keep);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * (256 / L);
    for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * (256 / L) + threadIdx.x / L; i0 < m.rows; i0 += U * stride) {
        u4 k[U], v[U];
        float weight[U];
        int64_t place[U];  // of the new row: -1 if there is none
        int32_t page[U], at[U], head[U];
#pragma unroll
        for (int x = 0; x < U; ++x) {
            const int64_t i = i0 + x * stride;
            place[x] = -1;
            if (i >= m.rows) continue;
            const int32_t src = m.kept[i];
            if (src < 0) continue;
            const int64_t bh = i / m.keep;
            const int32_t b = static_cast<int32_t>(bh / m.kv_heads), to = static_cast<int32_t>(i - bh * m.keep);
            head[x] = static_cast<int32_t>(bh - static_cast<int64_t>(b) * m.kv_heads);
            if (WAY != kIn) {
                page[x] = page_at(m.from, b, src);
                at[x] = src & ((1 << m.from.shift) - 1);
                if (page[x] < 0) continue;
                k[x] = reinterpret_cast<const u4 *>(m.from.k.p + page[x] * m.from.k.batch + head[x] * m.from.k.head + at[x] * m.from.k.row)[c];
                v[x] = reinterpret_cast<const u4 *>(m.from.v.p + page[x] * m.from.v.batch + head[x] * m.from.v.head + at[x] * m.from.v.row)[c];
                if (c == 0 && m.to_weights)
                    weight[x] = m.weights[((static_cast<int64_t>(page[x]) * m.kv_heads + head[x]) << m.from.shift) + at[x]];
            } else {
                if (page_at(m.from, b, src) < 0) continue;
                k[x] = reinterpret_cast<const u4 *>(m.staged + (2 * i) * D)[c];
                v[x] = reinterpret_cast<const u4 *>(m.staged + (2 * i + 1) * D)[c];
                if (c == 0 && m.to_weights) weight[x] = m.staged_weights[i];
            }
            place[x] = i;
            if (WAY != kOut) {
                page[x] = page_at(m.to, b, to);
                at[x] = to & ((1 << m.to.shift) - 1);
                if (page[x] < 0) place[x] = -1;
            }
        }
#pragma unroll
        for (int x = 0; x < U; ++x) {
            if (place[x] < 0) continue;
            if (WAY == kOut) {
                reinterpret_cast<u4 *>(m.staged + (2 * place[x]) * D)[c] = k[x];
                reinterpret_cast<u4 *>(m.staged + (2 * place[x] + 1) * D)[c] = v[x];
                if (c == 0 && m.to_weights) m.staged_weights[place[x]] = weight[x];
            } else {
                reinterpret_cast<u4 *>(const_cast<uint16_t *>(m.to.k.p) + page[x] * m.to.k.batch + head[x] * m.to.k.head + at[x] * m.to.k.row)[c] = k[x];
                reinterpret_cast<u4 *>(const_cast<uint16_t *>(m.to.v.p) + page[x] * m.to.v.batch + head[x] * m.to.v.head + at[x] * m.to.v.row)[c] = v[x];
                if (c == 0 && m.to_weights)
                    m.to_weights[((static_cast<int64_t>(page[x]) * m.kv_heads + head[x]) << m.to.shift) + at[x]] = weight[x];
            }
        }
    }
}

}  // namespace

namespace {

// Sequences of more than 8 groups a wavefront of one block are shared by blocks, where one for each list would not fill the
// device.  (The four launches read the weights once each, a block of its own six times, from its XCD's L2.)  Up to 256
// segments, over whose counts the last launch runs.
constexpr int64_t kMostGroups = 8, kMostSegments = 256;
int64_t longest(const tiga_cache &c) { return static_cast<int64_t>(c.table_width) * c.page_size; }
bool held_by_one(const tiga_cache &c) { return longest(c) <= kMostGroups * kWaves * 256; }
bool segmented(const tiga_cache &c) {
    return !held_by_one(c) && longest(c) <= kMostSegments * kSegment && static_cast<int64_t>(c.batch) * c.kv_heads <= device_cus();
}

struct Layout {
    uint16_t *staged;
    float *staged_weights;
    Shared1 shared;
    size_t bytes;
};
Layout layout(const tiga_cache &cache, int32_t keep, bool staged, void *ws) {
    Layout l;
    Carve c(ws);
    const size_t heads = static_cast<size_t>(cache.batch) * cache.kv_heads, rows = staged ? heads * keep : 0;
    l.staged = c.take<uint16_t>(rows * 2 * cache.width);
    l.staged_weights = c.take<float>(rows);
    const int64_t segments = ceil_div(longest(cache), kSegment);
    l.shared.segments = static_cast<int32_t>(segments);
    // as many as a smaller call may need
    const size_t lists = heads < static_cast<size_t>(device_cus()) ? heads : device_cus();
    const size_t some = held_by_one(cache) ? 0 : segments < kMostSegments ? segments : kMostSegments;
    l.shared.counts = c.take<uint16_t>(lists * some * kCounts);
    l.shared.found = c.take<int2>(some ? lists * kLevels : 0);
    l.bytes = c.bytes() < 256 ? 256 : c.bytes();
    return l;
}

int select(const Args &a, const tiga_cache &cache, const Shared1 &shared, hipStream_t stream) {
    const unsigned heads = static_cast<unsigned>(cache.batch * cache.kv_heads);
    if (!segmented(cache)) {
        const dim3 grid(heads);
        if (longest(cache) <= kWaves * 256) hipLaunchKernelGGL((select_kernel<1>), grid, dim3(kThreads), 0, stream, a);
        else if (held_by_one(cache)) hipLaunchKernelGGL((select_kernel<kMostGroups>), grid, dim3(kThreads), 0, stream, a);
        else hipLaunchKernelGGL((select_kernel<0>), grid, dim3(kThreads), 0, stream, a);
        return check_launch("cache eviction, selection");
    }
    const dim3 grid(static_cast<unsigned>(shared.segments), heads);
    hipLaunchKernelGGL((segment_kernel<0>), grid, dim3(kThreads), 0, stream, a, shared);
    hipLaunchKernelGGL((segment_kernel<1>), grid, dim3(kThreads), 0, stream, a, shared);
    hipLaunchKernelGGL((segment_kernel<2>), grid, dim3(kThreads), 0, stream, a, shared);
    hipLaunchKernelGGL((segment_kernel<3>), grid, dim3(kThreads), 0, stream, a, shared);
    return check_launch("cache eviction, selection of long sequences");
}

}  // namespace

size_t evict_ws_bytes(const tiga_cache &cache, int32_t keep, bool staged) { return layout(cache, keep, staged, nullptr).bytes; }

int evict(const tiga_cache &cache, const float *weights, int32_t keep, int32_t recent, const tiga_cache &to,
          float *to_weights, int32_t *to_length, int32_t *kept, bool staged, void *ws, hipStream_t stream) {
    const Layout l = layout(cache, keep, staged, ws);
    const Args a{pages_of(cache, 0, nullptr), weights, cache.kv_heads, keep, recent, kept};
    if (int rc = select(a, cache, l.shared, stream)) return rc;
    Move m{};
    m.from = a.from;
    m.to = pages_of(to, 0, nullptr);
    m.kept = kept;
    m.weights = weights;
    m.to_weights = to_weights;
    m.to_length = to_length;
    m.kv_heads = cache.kv_heads;
    m.keep = keep;
    m.rows = static_cast<int64_t>(cache.batch) * cache.kv_heads * keep;
    m.staged = l.staged;
    m.staged_weights = l.staged_weights;
    const int64_t per = 4 * 256 / (cache.width / 8), blocks = ceil_div(m.rows, per), most = 16 * static_cast<int64_t>(device_cus());
    const dim3 moves(static_cast<unsigned>(blocks < most ? (blocks < 1 ? 1 : blocks) : most));
    auto go = [&](auto width) {
        constexpr int D = decltype(width)::value;
        if (!staged) {
            prof_before(stream);
            hipLaunchKernelGGL((move_kernel<D, kThrough>), moves, dim3(256), 0, stream, m);
            prof_after(stream);
            return check_launch("cache eviction, move");
        }
        hipLaunchKernelGGL((move_kernel<D, kOut>), moves, dim3(256), 0, stream, m);
        if (int rc = check_launch("cache eviction, move out")) return rc;
        prof_before(stream);
        hipLaunchKernelGGL((move_kernel<D, kIn>), moves, dim3(256), 0, stream, m);
        prof_after(stream);
        return check_launch("cache eviction, move back");
    };
    return cache.width == 64 ? go(std::integral_constant<int, 64>{}) : go(std::integral_constant<int, 128>{});
}

}  // namespace retention
}  // namespace tiga
