// Eviction from a paged cache: of every sequence and source head the `keep` positions of the largest weights stay, the last
// `recent` ones among them whatever theirs, ties by the lowest position, and move in order into another cache's pages.
//
// Selection: a block for a sequence and head, which holds the weights in registers as integers of the same order, finds the
// least one that stays by its digits of 8 bits from the top (a histogram in LDS, 16 copies of each counter so that equal
// digits of a wavefront's lanes seldom wait for each other), and lists the positions that stay by prefix sums.  A wavefront
// owns a contiguous run of positions, so the list needs one exchange between wavefronts.
// Move: 16 bytes a lane, keys and values of a listed position to its new place; bound by the memory.
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

// PER: groups of four neighbouring positions a lane holds; 0: as many as there are, read again in every turn.
template <int PER>
__global__ __launch_bounds__(kThreads) void select_kernel(Args a) {
    constexpr int kCopies = 16;
    __shared__ int32_t count[256 * kCopies];
    __shared__ int32_t found[2], totals[2][kWaves];
    const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave);
    const int b = static_cast<int>(blockIdx.x) / a.kv_heads, head = static_cast<int>(blockIdx.x) % a.kv_heads;
    const int32_t n = positions(a.from, b), mask = (1 << a.from.shift) - 1;
    const int32_t stay = min(n, a.keep), last = min(a.recent, stay), first_recent = n - last;
    int32_t *const kept = a.kept + (static_cast<int64_t>(b) * a.kv_heads + head) * a.keep;
    for (int32_t i = stay + static_cast<int32_t>(threadIdx.x); i < a.keep; i += kThreads) kept[i] = -1;
    if (n <= a.keep) {
        for (int32_t i = static_cast<int32_t>(threadIdx.x); i < n; i += kThreads) kept[i] = i;
        return;
    }
    // this wavefront's positions: `per` groups of 256
    const int32_t per = (n + kWaves * 256 - 1) / (kWaves * 256), start = w * per * 256;
    auto weight_at = [&](int32_t at) -> uint32_t {
        const int32_t page = page_at(a.from, b, at);
        return page < 0 ? 0u : ordered(a.weights[((static_cast<int64_t>(page) * a.kv_heads + head) << a.from.shift) + (at & mask)]);
    };
    auto read = [&](int32_t j) -> u4 {
        const int32_t at = start + j * 256 + lane * 4;
        u4 x{0u, 0u, 0u, 0u};
        if (at >= first_recent) return x;
        if (mask >= 3) {
            const int32_t page = page_at(a.from, b, at);
            if (page < 0) return x;
            const f4 v = *reinterpret_cast<const f4 *>(a.weights + ((static_cast<int64_t>(page) * a.kv_heads + head) << a.from.shift) + (at & mask));
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = ordered(v[e]);
            return x;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + e < first_recent) x[e] = weight_at(at + e);
        return x;
    };
    u4 held[PER > 0 ? PER : 1];
#pragma unroll
    for (int j = 0; j < PER; ++j)
        if (j < per) held[j] = read(j);
    // f(group, its four weights, how many of them are no recent positions)
    auto each = [&](auto f) {
        if constexpr (PER > 0) {
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (j < per) f(j, held[j], first_recent - (start + j * 256 + lane * 4));
        } else {
            for (int32_t j = 0; j < per; ++j) f(j, read(j), first_recent - (start + j * 256 + lane * 4));
        }
    };

    // the least weight that stays, from its digits, and how many equal ones stay
    uint32_t least = 0;
    int32_t need = stay - last;  // of those that agree with `least` so far
    if (need > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = threadIdx.x; i < 256 * kCopies; i += kThreads) count[i] = 0;
            __syncthreads();
            const uint32_t upper = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
            each([&](int, u4 x, int32_t old) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < old && (x[e] & upper) == least) atomicAdd(&count[(x[e] >> shift & 255u) * kCopies + lane % kCopies], 1);
            });
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
    // the list: larger and recent positions, and the first `need` equal ones
    auto sort_out = [&](int32_t at, uint32_t x, bool &more, bool &equal) {
        more = at < n && (at >= first_recent || (stay > last && x > least));
        equal = at < first_recent && stay > last && x == least;
    };
    int32_t mores = 0, equals = 0;
    each([&](int j, u4 x, int32_t) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            bool more, equal;
            sort_out(start + j * 256 + lane * 4 + e, x[e], more, equal);
            mores += more;
            equals += equal;
        }
    });
    int32_t all[2];
    lanes_before(mores, all[0]);
    lanes_before(equals, all[1]);
    if (lane == 0) {
        totals[0][w] = all[0];
        totals[1][w] = all[1];
    }
    __syncthreads();
    mores = equals = 0;
    for (int i = 0; i < w; ++i) {
        mores += totals[0][i];
        equals += totals[1][i];
    }
    each([&](int j, u4 x, int32_t) {
        bool more[4], equal[4];
        int32_t m = 0, q = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sort_out(start + j * 256 + lane * 4 + e, x[e], more[e], equal[e]);
            m += more[e];
            q += equal[e];
        }
        int32_t all_m, all_q;
        int32_t before_m = mores + lanes_before(m, all_m), before_q = equals + lanes_before(q, all_q);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (more[e] || (equal[e] && before_q < need)) kept[before_m + min(before_q, need)] = start + j * 256 + lane * 4 + e;
            before_m += more[e];
            before_q += equal[e];
        }
        mores += all_m;
        equals += all_q;
    });
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

size_t evict_ws_bytes(const tiga_cache &cache, int32_t keep, bool staged) {
    Carve c(nullptr);
    const size_t rows = staged ? static_cast<size_t>(cache.batch) * cache.kv_heads * keep : 0;
    c.take<uint16_t>(rows * 2 * cache.width);
    c.take<float>(rows);
    return c.bytes() < 256 ? 256 : c.bytes();
}

int evict(const tiga_cache &cache, const float *weights, int32_t keep, int32_t recent, const tiga_cache &to,
          float *to_weights, int32_t *to_length, int32_t *kept, bool staged, void *ws, hipStream_t stream) {
    Args a{pages_of(cache, 0, nullptr), weights, cache.kv_heads, keep, recent, kept};
    const int64_t longest = static_cast<int64_t>(cache.table_width) * cache.page_size, groups = ceil_div(longest, kWaves * 256);
    const dim3 grid(static_cast<unsigned>(cache.batch * cache.kv_heads));
    if (groups <= 1) hipLaunchKernelGGL((select_kernel<1>), grid, dim3(kThreads), 0, stream, a);
    else if (groups <= 8) hipLaunchKernelGGL((select_kernel<8>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((select_kernel<0>), grid, dim3(kThreads), 0, stream, a);
    if (int rc = check_launch("cache eviction, selection")) return rc;
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
    Carve c(ws);
    m.staged = c.take<uint16_t>(staged ? m.rows * 2 * cache.width : 0);
    m.staged_weights = c.take<float>(staged ? m.rows : 0);
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
