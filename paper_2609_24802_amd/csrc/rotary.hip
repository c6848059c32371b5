// Rotary positions, and the append of new tokens to a paged cache with the rotation on the way.
//   pair (a, b) at position p -> amplitude (a cos t - b sin t, a sin t + b cos t),  t = p freq
// The angle is formed in fp64 as turns u = p freq / 2 pi and reduced there to an eighth of a turn
// either side of a quarter (|r| <= 1/8, u = k / 4 + r); in fp32 a position of 10^6 alone would cost
// 0.03 radians.  Sine and cosine of r are fp32.
//
// Bound by reading and writing the rows once.  A block takes a few rows: its threads first form each row's angles once,
// into LDS, and then move 16 bytes a thread and step (a slot: the two 16-byte runs whose elements pair up, or one run
// of adjacent pairs, or one run behind the rotated part), four steps' loads in flight.  Where there are few rows their
// heads are spread over more blocks.  Measured (MI355X): 4 x 4096 rows of 40 heads x 128, bf16, 69 us, 4.85 TB/s (a large
// copy moves 4.84); 61 rows of 36 heads 3.6 to 4.2 us; the append of 64 tokens 4.8 to 5.0 us (a chain of four dependent
// loads), of 8189 tokens 26 us, 3.8 TB/s (element by element and a token a block: 51 us).  Rows that are not 16-byte aligned,
// or do not divide into such slots, go element by element (a thread a pair).
#include "mfma16.hpp"
#include "relation.hpp"
#include "rotary.hpp"

namespace tiga {
namespace rotary {

using relattn::Chunk;
using relattn::chunk_of;
using relattn::Divider;
using relattn::divider;
using relattn::quotient;
using relattn::page_at;
using relattn::Pages;
using relattn::pages_of;

namespace {

constexpr int kThreads = 256;
constexpr double kTurnsPerRadian = 0.15915494309189533577;

struct F16 {
    typedef uint16_t raw;
    static __device__ __forceinline__ float get(raw b) { return static_cast<float>(__builtin_bit_cast(_Float16, b)); }
    static __device__ __forceinline__ raw put(float f) { return __builtin_bit_cast(raw, static_cast<_Float16>(f)); }
};
struct BF16 {
    typedef uint16_t raw;
    static __device__ __forceinline__ float get(raw b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
    static __device__ __forceinline__ raw put(float f) { return __builtin_bit_cast(raw, static_cast<__bf16>(f)); }
};
struct F32 {
    typedef float raw;
    static __device__ __forceinline__ float get(raw b) { return b; }
    static __device__ __forceinline__ raw put(float f) { return f; }
};

struct Angle {
    float c, s;
};
__device__ __forceinline__ Angle angle_of(int64_t pos, double freq, float amp, float sign) {
    const double u = static_cast<double>(pos) * (freq * kTurnsPerRadian);
    const double k = __builtin_rint(4.0 * u);
    const float r = static_cast<float>(u - 0.25 * k);
    float s, c;
    sincospif(2.0f * r, &s, &c);
    const int quarter = static_cast<int>(static_cast<int64_t>(k) & 3);
    const float cc = quarter & 1 ? s : c, ss = quarter & 1 ? c : s;
    Angle a;
    a.c = amp * (quarter == 1 || quarter == 2 ? -cc : cc);
    a.s = amp * sign * (quarter >= 2 ? -ss : ss);
    return a;
}

template <class T>
__device__ __forceinline__ void turn_pair(const typename T::raw *x, typename T::raw *y, int i, int rot, int pairs, Angle a) {
    const int e0 = pairs == TIGA_PAIRS_HALF ? i : 2 * i, e1 = pairs == TIGA_PAIRS_HALF ? i + rot / 2 : 2 * i + 1;
    const float u = T::get(x[e0]), v = T::get(x[e1]);
    y[e0] = T::put(u * a.c - v * a.s);
    y[e1] = T::put(u * a.s + v * a.c);
}

// ------------------------------------------------------------------------------------------ 16-byte slots

// The elements of 16 bytes and back.
template <class T>
struct Run;
template <>
struct Run<F16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void get(u4 v, float *f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f2 x = Half16::unpack(v[i]);
            f[2 * i] = x.x;
            f[2 * i + 1] = x.y;
        }
    }
    static __device__ __forceinline__ u4 put(const float *f) {
        return u4{Half16::pack(f[0], f[1]), Half16::pack(f[2], f[3]), Half16::pack(f[4], f[5]), Half16::pack(f[6], f[7])};
    }
};
template <>
struct Run<BF16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void get(u4 v, float *f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f2 x = Brain16::unpack(v[i]);
            f[2 * i] = x.x;
            f[2 * i + 1] = x.y;
        }
    }
    static __device__ __forceinline__ u4 put(const float *f) {
        return u4{Brain16::pack(f[0], f[1]), Brain16::pack(f[2], f[3]), Brain16::pack(f[4], f[5]), Brain16::pack(f[6], f[7])};
    }
};
template <>
struct Run<F32> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void get(u4 v, float *f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
    }
    static __device__ __forceinline__ u4 put(const float *f) {
        return u4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
};

constexpr int kMaxPairs = 1024;  // of the rows of a block together, for the angles in LDS
constexpr int kSteps = 4;        // slots whose loads a thread has in flight

// The slots of a head: `turned` of them rotate, the rest copy.
struct Slots {
    int turned, all;
    Divider div;  // by all
};
Slots slots_of(const tiga_rotary &rot, int width, int n) {
    const int turned = rot.rot / n / (rot.pairs == TIGA_PAIRS_HALF ? 2 : 1), all = turned + (width - rot.rot) / n;
    return Slots{turned, all, divider(all)};
}

// One slot in flight: where it goes, and its runs.
template <class T>
struct Move {
    typename T::raw *y;
    u4 a, b;
    int slot;  // -1: nothing
};
// Element at which the slot's first run starts; the second of a half-split slot lies rot / 2 further.
__device__ __forceinline__ int start_of(const tiga_rotary &rot, const Slots &s, int slot, int n) {
    return slot < s.turned ? slot * n : rot.rot + (slot - s.turned) * n;
}
template <class T>
__device__ __forceinline__ void fetch(Move<T> &m, const typename T::raw *x, typename T::raw *y, const tiga_rotary &rot,
                                      const Slots &s, int slot) {
    const int e = start_of(rot, s, slot, Run<T>::N);
    m.slot = slot;
    m.y = y + e;
    m.a = *reinterpret_cast<const u4 *>(x + e);
    if (slot < s.turned && rot.pairs == TIGA_PAIRS_HALF) m.b = *reinterpret_cast<const u4 *>(x + e + rot.rot / 2);
}
// c, s: the row's cosines and sines of pair 0 on; turn false: the row is copied.
template <class T>
__device__ __forceinline__ void settle(const Move<T> &m, const tiga_rotary &rot, const Slots &sl, const float *c,
                                       const float *s, bool turn) {
    constexpr int N = Run<T>::N;
    const bool half = rot.pairs == TIGA_PAIRS_HALF;
    u4 a = m.a, b = m.b;
    if (m.slot < sl.turned && turn) {
        float u[N];
        Run<T>::get(a, u);
        if (half) {
            float v[N], p[N], q[N];
            Run<T>::get(b, v);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float ci = c[m.slot * N + i], si = s[m.slot * N + i];
                p[i] = u[i] * ci - v[i] * si;
                q[i] = u[i] * si + v[i] * ci;
            }
            a = Run<T>::put(p);
            b = Run<T>::put(q);
        } else {
            float p[N];
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const float ci = c[m.slot * (N / 2) + i], si = s[m.slot * (N / 2) + i];
                p[2 * i] = u[2 * i] * ci - u[2 * i + 1] * si;
                p[2 * i + 1] = u[2 * i] * si + u[2 * i + 1] * ci;
            }
            a = Run<T>::put(p);
        }
    }
    *reinterpret_cast<u4 *>(m.y) = a;
    if (m.slot < sl.turned && half) *reinterpret_cast<u4 *>(m.y + rot.rot / 2) = b;
}

// Block (x, y): rows [(block0 + x) * per_block, ...) of batch * rows, heads [y * group, ...).
template <class T>
__global__ __launch_bounds__(kThreads) void rotate_rows_kernel(tiga_view x, tiga_view y, const int32_t *__restrict__ pos,
                                                               int64_t pos_batch, int64_t rows, int64_t total,
                                                               int per_block, int heads, int group, tiga_rotary rot,
                                                               Slots sl, Divider heads_div, float sign, int64_t block0) {
    typedef typename T::raw raw;
    __shared__ float c[kMaxPairs], s[kMaxPairs];
    const int64_t row0 = (block0 + blockIdx.x) * per_block;
    const int here = static_cast<int>(min(static_cast<int64_t>(per_block), total - row0));
    const int h0 = blockIdx.y * group, nh = min(group, heads - h0), pairs = rot.rot / 2;
    for (int i = threadIdx.x; i < here * pairs; i += kThreads) {
        const int r = i / pairs, k = i - r * pairs;
        const int64_t b = quotient(row0 + r, rows), at = row0 + r - b * rows;
        const Angle a = angle_of(pos ? pos[b * pos_batch + at] : at, rot.freq[k], rot.amplitude, sign);
        c[i] = a.c;
        s[i] = a.s;
    }
    const int items = here * nh * sl.all;
    auto item = [&](int i, int &r, int &slot, int64_t &xo, int64_t &yo) {
        const int q = sl.div.div(i);
        slot = i - q * sl.all;
        r = nh == heads ? heads_div.div(q) : q / nh;
        const int h = h0 + q - r * nh;
        const int64_t b = quotient(row0 + r, rows), at = row0 + r - b * rows;
        xo = b * x.batch + h * x.head + at * x.row;
        yo = b * y.batch + h * y.head + at * y.row;
    };
    const raw *const xp = static_cast<const raw *>(x.data);
    raw *const yp = static_cast<raw *>(y.data);
    bool ready = false;
    for (int i0 = threadIdx.x; i0 - static_cast<int>(threadIdx.x) < items; i0 += kThreads * kSteps) {
        Move<T> m[kSteps];
        int row[kSteps];
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int i = i0 + k * kThreads;
            m[k].slot = -1;
            if (i < items) {
                int slot;
                int64_t xo, yo;
                item(i, row[k], slot, xo, yo);
                fetch<T>(m[k], xp + xo, yp + yo, rot, sl, slot);
            }
        }
        if (!ready) __syncthreads();  // the angles are there
        ready = true;
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
            if (m[k].slot >= 0) settle<T>(m[k], rot, sl, c + row[k] * pairs, s + row[k] * pairs, true);
    }
}

// The sequence of packed row `row`, batch if it is none's: the number of sequences that end at or before it.
__device__ __forceinline__ int sequence_of(const Pages &cache, int row) {
    int b = 0;
    for (int base = 0; base < cache.batch; base += kWave) {
        const int e = base + lane_id();
        const bool before = e < cache.batch && cache.dst_ptr[e + 1] <= row;
        const int n = __popcll(__ballot(before));
        b += n;
        if (n < kWave) break;
    }
    return b;
}

// A block takes per_block (at most 4) new tokens: slots of their keys and queries (turned) and values (copied).  A
// wavefront finds each token's place while the slots' loads are in flight.
template <class T>
__global__ __launch_bounds__(kThreads) void append_kernel(Pages cache, tiga_view k, tiga_view v, tiga_rotary rot, int heads,
                                                          int kv_heads, tiga_view q, tiga_view qo, int per_block, Slots sl,
                                                          Slots whole, Divider per_token, int block0) {
    typedef typename T::raw raw;
    struct Place {
        int64_t pos;
        int32_t page;  // -1: keys and values are not stored
        bool behind;   // the last sequence: nothing is written
    };
    __shared__ float c[kMaxPairs], s[kMaxPairs];
    __shared__ Place places[4];
    const int row0 = (block0 + static_cast<int>(blockIdx.x)) * per_block, here = min(per_block, cache.num_dst - row0);
    const int pairs = rot.rot / 2;
    const int nk = kv_heads * sl.all, nv = kv_heads * whole.all, each = nk + nv + heads * sl.all, items = here * each;
    const tiga_rotary plain{nullptr, 0, TIGA_PAIRS_ADJACENT, 1.0f};
    Move<T> m[kSteps];
    int kind[kSteps], token[kSteps];  // 0 keys, 1 values, 2 queries
    int64_t off[kSteps];
    auto fetch_all = [&](int i0) {
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            m[j].slot = -1;
            if (i0 + j * kThreads >= items) continue;
            token[j] = per_token.div(i0 + j * kThreads);
            const int i = i0 + j * kThreads - token[j] * each;
            const int64_t row = row0 + token[j];
            if (i < nk) {
                const int h = sl.div.div(i);
                kind[j] = 0;
                off[j] = h * cache.k.head;
                fetch<T>(m[j], static_cast<const raw *>(k.data) + row * k.row + h * k.head, nullptr, rot, sl, i - h * sl.all);
            } else if (i < nk + nv) {
                const int h = whole.div.div(i - nk);
                kind[j] = 1;
                off[j] = h * cache.v.head;
                fetch<T>(m[j], static_cast<const raw *>(v.data) + row * v.row + h * v.head, nullptr, plain, whole,
                         i - nk - h * whole.all);
            } else {
                const int h = sl.div.div(i - nk - nv);
                kind[j] = 2;
                off[j] = h * qo.head + row * qo.row;
                fetch<T>(m[j], static_cast<const raw *>(q.data) + row * q.row + h * q.head, nullptr, rot, sl,
                         i - nk - nv - h * sl.all);
            }
        }
    };
    fetch_all(threadIdx.x);
    const int w = static_cast<int>(threadIdx.x) / kWave;
    if (w < here) {
        const int row = row0 + w, b = sequence_of(cache, row);
        Place p{-1, -1, b >= cache.batch};
        if (!p.behind) {
            const Chunk ch = chunk_of(cache, b);
            if (row >= ch.first && row < ch.first + ch.count) p.pos = ch.pos0 + (row - ch.first);
            if (p.pos >= 0) p.page = page_at(cache, b, p.pos);
        }
        if (lane_id() == 0) places[w] = p;
    }
    __syncthreads();
    if (rot.freq)
        for (int i = threadIdx.x; i < here * pairs; i += kThreads) {
            const int t = i / pairs;
            const Angle a = angle_of(places[t].pos, rot.freq[i - t * pairs], rot.amplitude, 1.0f);
            c[i] = a.c;
            s[i] = a.s;
        }
    __syncthreads();
    for (int i0 = threadIdx.x;;) {
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            if (m[j].slot < 0) continue;
            const Place p = places[token[j]];
            if (p.behind || (kind[j] < 2 && p.page < 0)) continue;
            if (kind[j] == 2) {
                m[j].y = static_cast<raw *>(qo.data) + off[j];
            } else {
                const relattn::Rows &to = kind[j] == 0 ? cache.k : cache.v;
                m[j].y = const_cast<raw *>(to.p) + off[j] + p.page * to.batch + (p.pos & ((1 << cache.shift) - 1)) * to.row;
            }
            if (kind[j] == 1) {
                m[j].y += start_of(plain, whole, m[j].slot, Run<T>::N);
                settle<T>(m[j], plain, whole, c, s, false);
            } else {
                m[j].y += start_of(rot, sl, m[j].slot, Run<T>::N);
                settle<T>(m[j], rot, sl, c + token[j] * pairs, s + token[j] * pairs, rot.freq && p.pos >= 0);
            }
        }
        i0 += kThreads * kSteps;
        if (i0 - static_cast<int>(threadIdx.x) >= items) break;
        fetch_all(i0);
    }
}

// ------------------------------------------------------------------------------------------ element by element

// Pair i of the heads of a row (one thread); past rot / 2, elements rot + 2 (i - rot / 2) and the one after are copied.
template <class T>
__device__ __forceinline__ void turn_heads(const typename T::raw *x, int64_t xh, typename T::raw *y, int64_t yh, int heads,
                                           int i, int width, const tiga_rotary &rot, Angle a) {
    for (int h = 0; h < heads; ++h) {
        if (i < rot.rot / 2) {
            turn_pair<T>(x + h * xh, y + h * yh, i, rot.rot, rot.pairs, a);
        } else {
            y[h * yh + 2 * i] = x[h * xh + 2 * i];
            if (2 * i + 1 < width) y[h * yh + 2 * i + 1] = x[h * xh + 2 * i + 1];
        }
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void rotate_pairs_kernel(tiga_view x, tiga_view y, const int32_t *__restrict__ pos,
                                                                int64_t pos_batch, int64_t rows, int64_t total, int heads,
                                                                int group, int width, tiga_rotary rot, float sign,
                                                                int64_t block0) {
    const int units = (width + 1) / 2, h0 = blockIdx.y * group;
    const int64_t t = (block0 + blockIdx.x) * kThreads + threadIdx.x;
    if (t >= total) return;
    const int64_t line = quotient(t, units), b = quotient(line, rows), r = line - b * rows;
    const int i = static_cast<int>(t - line * units);
    Angle a{};
    if (i < rot.rot / 2) a = angle_of(pos ? pos[b * pos_batch + r] : r, rot.freq[i], rot.amplitude, sign);
    turn_heads<T>(static_cast<const typename T::raw *>(x.data) + b * x.batch + r * x.row + h0 * x.head, x.head,
                  static_cast<typename T::raw *>(y.data) + b * y.batch + r * y.row + h0 * y.head, y.head,
                  min(group, heads - h0), i, width, rot, a);
}

// A block a new token.
template <class T>
__global__ __launch_bounds__(kThreads) void append_pairs_kernel(Pages cache, tiga_view k, tiga_view v, tiga_rotary rot, int heads,
                                                          int kv_heads, tiga_view q, tiga_view qo, int width, int block0) {
    typedef typename T::raw raw;
    const int row = block0 + static_cast<int>(blockIdx.x);
    const int b = sequence_of(cache, row);
    if (b >= cache.batch) return;
    const Chunk ch = chunk_of(cache, b);
    const bool own = row >= ch.first && row < ch.first + ch.count;  // a row before the first sequence has no position
    const int64_t pos = own ? ch.pos0 + (row - ch.first) : -1;
    const int32_t page = pos < 0 ? -1 : page_at(cache, b, pos);
    const int64_t slot = pos & ((1 << cache.shift) - 1);
    for (int i = threadIdx.x; i < width / 2; i += kThreads) {
        Angle a{1.0f, 0.0f};
        tiga_rotary rr = rot;
        if (!rot.freq || pos < 0) rr.rot = 0;
        if (i < rr.rot / 2) a = angle_of(pos, rot.freq[i], rot.amplitude, 1.0f);
        if (page >= 0) {
            raw *kp = const_cast<raw *>(cache.k.p) + page * cache.k.batch + slot * cache.k.row;
            turn_heads<T>(static_cast<const raw *>(k.data) + row * k.row, k.head, kp, cache.k.head, kv_heads, i, width, rr, a);
            raw *vp = const_cast<raw *>(cache.v.p) + page * cache.v.batch + slot * cache.v.row;
            rr.rot = 0;
            turn_heads<T>(static_cast<const raw *>(v.data) + row * v.row, v.head, vp, cache.v.head, kv_heads, i, width, rr, a);
            if (rot.freq && pos >= 0) rr.rot = rot.rot;
        }
        if (q.data)
            turn_heads<T>(static_cast<const raw *>(q.data) + row * q.row, q.head, static_cast<raw *>(qo.data) + row * qo.row,
                          qo.head, heads, i, width, rr, a);
    }
}

// launch(first block, blocks) until all are launched: a grid counts its threads in 32 bits, and a larger one would wrap
// around without an error.
constexpr int64_t kMostBlocks = int64_t(1) << 23;
template <class F>
int in_grids(int64_t blocks, const char *what, hipStream_t stream, F launch) {
    prof_before(stream);
    for (int64_t at = 0; at < blocks; at += kMostBlocks) {
        launch(at, static_cast<unsigned>(blocks - at < kMostBlocks ? blocks - at : kMostBlocks));
        if (int rc = check_launch(what)) return rc;
    }
    prof_after(stream);
    return TIGA_OK;
}

// Whether the rows of a view consist of aligned 16-byte runs that the rotation's slots are made of.
bool sliced(const tiga_view &v, int size) {
    return aligned16(v.data) && (v.batch * size) % 16 == 0 && (v.head * size) % 16 == 0 && (v.row * size) % 16 == 0;
}
bool slots_fit(const tiga_rotary &rot, int width, int n) {
    return width % n == 0 && rot.rot % (rot.pairs == TIGA_PAIRS_HALF ? 2 * n : n) == 0 && rot.rot / 2 <= kMaxPairs;
}

}  // namespace

int rotate(int32_t batch, int32_t heads, int64_t rows, int32_t width, int dtype, const tiga_view &x,
           const int32_t *pos, int64_t pos_batch, const tiga_rotary &rot, bool back, const tiga_view &y,
           hipStream_t stream) {
    const int size = dtype == TIGA_DT_F32 ? 4 : 2, n = 16 / size;
    const int64_t lines = rows * batch, wanted = 4 * static_cast<int64_t>(device_cus());  // blocks, where there is work
    const float sign = back ? -1.0f : 1.0f;
    const bool runs = slots_fit(rot, width, n) && sliced(x, size) && sliced(y, size);
    const Slots sl = runs ? slots_of(rot, width, n) : Slots{};
    // rows a block: as many as give its threads kSteps slots each, with their angles in LDS, while the blocks last
    int64_t per_block = 1, total = lines * ((width + 1) / 2);
    if (runs) {
        const int64_t most = kMaxPairs / (rot.rot / 2), fill = ceil_div(kThreads * kSteps, static_cast<int64_t>(heads) * sl.all);
        per_block = lines / wanted;
        per_block = per_block > most ? most : per_block;
        per_block = per_block > fill ? fill : per_block;
        per_block = per_block < 1 ? 1 : per_block;
    }
    const int64_t blocks = runs ? ceil_div(lines, per_block) : ceil_div(total, kThreads);
    // heads a block: all of them, fewer where the rows alone do not fill the device
    int64_t group = blocks >= wanted ? heads : ceil_div(static_cast<int64_t>(heads) * blocks, wanted);
    if (ceil_div(heads, group) > 65535) group = ceil_div(heads, 65535);
    if (runs && group * sl.all * per_block > 0x3fffffff) group = 0x3fffffff / (sl.all * per_block);  // 32-bit slot numbers
    const unsigned parts = static_cast<unsigned>(ceil_div(heads, group));
    auto go = [&](auto by_runs, auto by_pairs) {
        return in_grids(blocks, "rotary", stream, [&](int64_t at, unsigned n) {
            if (runs)
                hipLaunchKernelGGL(by_runs, dim3(n, parts), dim3(kThreads), 0, stream, x, y, pos, pos_batch, rows, lines,
                                   static_cast<int>(per_block), heads, static_cast<int>(group), rot, sl, divider(heads), sign,
                                   at);
            else
                hipLaunchKernelGGL(by_pairs, dim3(n, parts), dim3(kThreads), 0, stream, x, y, pos, pos_batch, rows, total,
                                   heads, static_cast<int>(group), width, rot, sign, at);
        });
    };
    if (dtype == TIGA_DT_F32) return go(rotate_rows_kernel<F32>, rotate_pairs_kernel<F32>);
    return dtype == TIGA_DT_F16 ? go(rotate_rows_kernel<F16>, rotate_pairs_kernel<F16>)
                                : go(rotate_rows_kernel<BF16>, rotate_pairs_kernel<BF16>);
}

int append(const tiga_cache &cache, int64_t num_dst, const int32_t *dst_ptr, const tiga_view &k, const tiga_view &v,
           const tiga_rotary &given, int32_t heads, const tiga_view &q, const tiga_view &q_out, hipStream_t stream) {
    tiga_rotary rot = given;
    if (!rot.freq) rot = tiga_rotary{nullptr, 0, TIGA_PAIRS_ADJACENT, 1.0f};
    const tiga_rotary none{nullptr, 0, TIGA_PAIRS_ADJACENT, 1.0f};
    const Slots sl = slots_of(rot, cache.width, 8), whole = slots_of(none, cache.width, 8);
    const bool runs = slots_fit(rot, cache.width, 8);
    const int32_t q_heads = q.data ? heads : 0;
    // tokens a block: as many as give its threads kSteps slots each, while the blocks last
    const int64_t each = static_cast<int64_t>(cache.kv_heads) * (sl.all + whole.all) + static_cast<int64_t>(q_heads) * sl.all;
    int64_t per_block = runs ? num_dst / (4 * static_cast<int64_t>(device_cus())) : 1;
    if (per_block > kThreads * kSteps / each) per_block = kThreads * kSteps / each;
    if (per_block > 4) per_block = 4;
    if (per_block < 1) per_block = 1;
    if (each * per_block > 0x3fffffff) return fail(TIGA_EUNSUPPORTED, "cache append: too many heads");
    auto go = [&](auto by_runs, auto by_pairs) {
        return in_grids(ceil_div(num_dst, per_block), "cache append", stream, [&](int64_t at, unsigned n) {
            if (runs)
                hipLaunchKernelGGL(by_runs, dim3(n), dim3(kThreads), 0, stream, pages_of(cache, num_dst, dst_ptr), k, v, rot,
                                   q_heads, cache.kv_heads, q, q_out, static_cast<int>(per_block), sl, whole,
                                   divider(static_cast<int32_t>(each)), static_cast<int>(at));
            else
                hipLaunchKernelGGL(by_pairs, dim3(n), dim3(kThreads), 0, stream, pages_of(cache, num_dst, dst_ptr), k, v, rot,
                                   q_heads, cache.kv_heads, q, q_out, cache.width, static_cast<int>(at));
        });
    };
    return cache.dtype == TIGA_DT_F16 ? go(append_kernel<F16>, append_pairs_kernel<F16>)
                                      : go(append_kernel<BF16>, append_pairs_kernel<BF16>);
}

}  // namespace rotary
}  // namespace tiga
