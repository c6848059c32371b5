// What the cached positions are worth: with s_ij = scale <q_i, k_j> and the rows' lse from attention over the same cache,
//   w_j <- decay w_j + sum_{rows i of the sequence and heads of the group that see j} exp(s_ij - lse_i),
// w_j taken as 0 for the new tokens' own positions.  Every position's sum is of one wavefront, in the order of the rows.
//
// Few rows (next tokens): the time is that of reading the keys once, so tiles of keys of all sequences and heads are laid end
// to end and every block walks an equal run of them.  A wavefront takes 32 or 64 keys a step, a step ahead in registers in
// the matrix operand's layout, with the queries as the other operand: a result's column is a key, and the sum over the rows
// is one over four registers and four lanes.
//
// Many rows (chunks of prompts): bound by the vector unit, 4 quarter-rate and 8 full-rate instructions for 256 pairs (96 cycles),
// and the matrix cores, whose products take 64 at width 128 and hardly overlap with them: 256 keys a block, and the weights
// of 16 rows formed under the products of the next, took the same 74 us as 128 keys and three blocks a compute unit, 72.  A
// block owns 128 keys, 32 a wavefront as operands in registers, and streams the rows through LDS.  The row tiles of all items
// (128 keys of a head) are laid end to end and every block takes an equal run of them; the sums of an item's parts (512 bytes)
// go to the workspace and are added in order by a second launch.
//
// Measured (MI355X), width 128: 64 single tokens over up to 8192 positions, 32 heads over 8, bf16: 83 us for 381 MB, 4.6 TB/s (a
// large copy moves 4.8).  Two chunks of 1023 tokens and three single ones over up to 9000 positions, 16 heads over 4, f16: 5.8
// (narrow) + 71 (wide) + 4.6 (sums of parts) for 43 GFLOP of products, 0.6 PFLOP/s.
#include <type_traits>

#include "mfma16.hpp"
#include "relation.hpp"
#include "retention.hpp"

namespace tiga {
namespace retention {

using namespace relattn;

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr float kLog2e = 1.4426950408889634f;

struct Args {
    Pages src;
    Rows q;
    const float *lse;  // [heads, num_dst]
    const float *in;   // [num_pages, kv_heads, page_size]
    float *out;
    float c, decay;    // c = scale * log2 e
    int kv_heads;
    Divider group;
    int32_t few;       // rows of the sequences that the narrow kernel takes, at most; the others are the wide one's
    float *part;       // [2 * blocks][kOwn]: a block's first and last item may be parts
    int4 *rec;         // [2 * blocks]: b + 1, head, tile, whether the item ends here
};

// Positions of a sequence: none past the table.
__device__ __forceinline__ int32_t positions(const Pages &c, int b) {
    const int64_t n = c.length[b], most = static_cast<int64_t>(c.table_width) << c.shift;
    return static_cast<int32_t>(n < 0 ? 0 : (n > most ? most : n));
}

__device__ __forceinline__ int32_t new_rows(const Args &a, int b) { return chunk_of(a.src, b).count * static_cast<int32_t>(a.group.d); }
// Positions of a sequence that the narrow kernel takes.
__device__ __forceinline__ int32_t narrow_positions(const Args &a, int b) { return new_rows(a, b) <= a.few ? positions(a.src, b) : 0; }

// The tiles of BN keys of all sequences and heads end to end, and a block's run of them.
template <int BN>
struct Run1 {
    int64_t u, end;
    int64_t base;   // where sequence b starts
    int32_t b, n;   // n: its positions
    int32_t mine;   // positions of the lane's of the first 64 sequences

    static __device__ __forceinline__ int32_t tiles(int32_t n) { return (n + BN - 1) / BN; }
    __device__ __forceinline__ void begin(const Args &a, int w, int blocks) {
        const int nb = a.src.batch;
        auto fetch = [&](int e) { return e < nb ? narrow_positions(a, e) : 0; };
        mine = fetch(lane_id());
        int64_t all = 0;
        for (int e = 0; e < nb; e += kWave)
            all += lane_value(wave_prefix(tiles(e == 0 ? mine : fetch(e + lane_id()))), kWave - 1);
        all *= a.kv_heads;
        const int64_t per = quotient(all, blocks), rem = all - per * blocks;
        u = w * per + (w < rem ? w : rem);
        end = u + per + (w < rem ? 1 : 0);
        base = 0;
        b = n = 0;
        if (u >= end) return;
        for (int e = 0; e < nb; e += kWave) {
            const int64_t here = static_cast<int64_t>(tiles(e == 0 ? mine : fetch(e + lane_id()))) * a.kv_heads;
            const int64_t incl = wave_prefix(here);
            const uint64_t past = __ballot(base + incl > u);
            if (past) {
                const int l = __builtin_ctzll(past);
                b = e + l;
                base += lane_value(incl - here, l);
                break;
            }
            base += lane_value(incl, kWave - 1);
        }
        n = b < kWave ? __builtin_amdgcn_readlane(mine, b) : narrow_positions(a, b);
    }
    struct Tile {
        int32_t b, head, n, k0;  // k0: its first key
    };
    __device__ __forceinline__ bool next(const Args &a, Tile &t) {
        if (u >= end) return false;
        while (u >= base + static_cast<int64_t>(tiles(n)) * a.kv_heads) {  // a later sequence holds u
            base += static_cast<int64_t>(tiles(n)) * a.kv_heads;
            ++b;
            n = b < kWave ? __builtin_amdgcn_readlane(mine, b) : narrow_positions(a, b);
        }
        const int64_t in = u - base, head = quotient(in, tiles(n));
        t = Tile{b, static_cast<int32_t>(head), n, static_cast<int32_t>(in - head * tiles(n)) * BN};
        ++u;
        return true;
    }
};

// A row that saw nothing gives no weight, whatever its query holds (a score that is not finite less infinity may be NaN).
__device__ __forceinline__ float log2_of(float lse) { return lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2e; }

template <class T, int D>
struct Step {
    static constexpr int KW = 4096 / D;  // keys of a wavefront's step: 8 KB
    static constexpr int BN = kWaves * KW;
    static constexpr int KB = KW / 16, CH = D / 32;
};

template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void weights_kernel(Args a) {
    using G = Step<T, D>;
    typedef Run1<G::BN> Walk;
    typedef typename Walk::Tile Tile;
    const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave);
    const int col = lane & 15, g = lane >> 4;
    const int32_t d = static_cast<int32_t>(a.group.d), mask = (1 << a.src.shift) - 1;
    Walk walk;
    walk.begin(a, static_cast<int>(xcd_block()), static_cast<int>(gridDim.x));

    // the step's keys of this wavefront; positions past the last read that one (and are not stored)
    auto key = [&](const Tile &t, int i) { return min(t.k0 + w * G::KW + i, t.n - 1); };
    auto look_up = [&](const Tile &t) { return entry_at(a.src, t.b, key(t, lane % G::KW)); };
    auto cell = [&](const Tile &t, int32_t page, int32_t at) {
        return ((static_cast<int64_t>(page) * a.kv_heads + t.head) << a.src.shift) + (at & mask);
    };
    auto stage = [&](const Tile &t, int32_t entry, u4 (&k)[G::KB][G::CH], float &old) {
        const bool good = is_page(a.src, entry);
        const int32_t page = good ? entry : 0;  // a key of some page, whose weight is not stored
#pragma unroll
        for (int kb = 0; kb < G::KB; ++kb) {
            const int32_t pg = __shfl(page, kb * 16 + col, kWave);
            const uint16_t *const p = a.src.k.p + pg * a.src.k.batch + t.head * a.src.k.head +
                                      static_cast<int64_t>(key(t, kb * 16 + col) & mask) * a.src.k.row;
#pragma unroll
            for (int ch = 0; ch < G::CH; ++ch) k[kb][ch] = reinterpret_cast<const u4 *>(p)[ch * 4 + g];
        }
        old = a.in[cell(t, page, key(t, lane % G::KW))];
    };
    u4 q[G::CH];
    float lse2[4];
    int32_t held_b = -1, held_head = -1;  // whose queries are held
    auto step = [&](const Tile &t, int32_t entry, const u4 (&k)[G::KB][G::CH], float old) {
        const Chunk chunk = chunk_of(a.src, t.b);
        const int32_t rows = chunk.count * d;
        float sum[G::KB];
#pragma unroll
        for (int kb = 0; kb < G::KB; ++kb) sum[kb] = 0.0f;
        for (int32_t r0 = 0; r0 < rows; r0 += 16) {
            if (rows > 16 || held_b != t.b || held_head != t.head) {
                auto at = [&](int32_t r, int64_t head_stride, int64_t row_stride) {
                    const int32_t token = a.group.div(r);
                    return static_cast<int64_t>(t.head * d + r - token * d) * head_stride + (chunk.first + token) * row_stride;
                };
                const u4 *const p = reinterpret_cast<const u4 *>(a.q.p + at(min(r0 + col, rows - 1), a.q.head, a.q.row));
#pragma unroll
                for (int ch = 0; ch < G::CH; ++ch) q[ch] = p[ch * 4 + g];
#pragma unroll
                for (int i = 0; i < 4; ++i) lse2[i] = log2_of(a.lse[at(min(r0 + 4 * g + i, rows - 1), a.src.num_dst, 1)]);
                held_b = t.b;
                held_head = t.head;
            }
#pragma unroll
            for (int kb = 0; kb < G::KB; ++kb) {
                f4 s{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int ch = 0; ch < G::CH; ++ch) s = T::mma(q[ch], k[kb][ch], s);
                const int32_t at = t.k0 + w * G::KW + kb * 16 + col;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int32_t r = r0 + 4 * g + i;
                    const bool sees = r < rows && at <= chunk.pos0 + a.group.div(r) && lse2[i] != __builtin_inff();
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.c, -lse2[i]));
                    sum[kb] += sees ? p : 0.0f;
                }
            }
        }
        float mine = 0.0f;  // lane (kb, col) has key kb * 16 + col
#pragma unroll
        for (int kb = 0; kb < G::KB; ++kb) {
            const float all = column_sum(sum[kb]);
            if (kb == g) mine = all;
        }
        const int32_t at = t.k0 + w * G::KW + lane;
        if (lane < G::KW && at < t.n && is_page(a.src, entry))
            a.out[cell(t, entry, at)] = mine + (at < chunk.pos0 ? a.decay * old : 0.0f);
    };
    u4 ka[G::KB][G::CH], kb[G::KB][G::CH];
    float oa = 0.0f, ob = 0.0f;
    // A table's entry is asked for two steps ahead and before the keys of the next: loads arrive in order, so that waiting for an
    // entry asked for behind them would leave no keys in flight.  Past the run's end the last tile is read again, so that the
    // loads in flight are as many on every path.  (64 tokens over up to 8192 positions: 92 us with the entry behind the keys, 90
    // without the last tile's second read, 83.)
    Tile t0, t1, t2;
    if (!walk.next(a, t0)) return;
    int32_t e0 = look_up(t0), e1, e2;
    t1 = t0;
    bool more = walk.next(a, t1);
    e1 = look_up(t1);
    stage(t0, e0, ka, oa);
    if (!more) {
        step(t0, e0, ka, oa);
        return;
    }
    for (;;) {
        t2 = t1;
        bool more2 = walk.next(a, t2);
        e2 = look_up(t2);
        stage(t1, e1, kb, ob);
        step(t0, e0, ka, oa);
        if (!more) break;
        t0 = t2;
        more = walk.next(a, t0);
        e0 = look_up(t0);
        stage(t2, e2, ka, oa);
        step(t1, e1, kb, ob);
        if (!more2) break;
        t1 = t0;
        e1 = e0;
        t0 = t2;
        e0 = e2;
    }
}

// ------------------------------------------------------------------------------------------ many rows

constexpr int kOwn = 128;          // keys of a block
constexpr int kLeastSteps = 4;     // row tiles of a block's run, at least

template <int D>
struct Wide {
    static constexpr int RB = 2 * D, CPR = D / 8, R = 256 / RB, CH = D / 32;
    static constexpr int BN = D == 64 ? 128 : 64;     // rows a tile
    static constexpr int TILE = BN * RB;              // 16 KB
    static constexpr int LPW = TILE / 1024 / kWaves;  // 1-KB direct loads per wavefront and tile
};
// 16-byte chunk c of row k lies at chunk c ^ swizzle(k): the 16 rows of a read fall into 16 bank groups.
template <int D>
__device__ __forceinline__ int swizzle(int k) { return (k / Wide<D>::R) % Wide<D>::CPR; }

// A sequence with many rows: `tiles` of its positions, `steps` of its rows.
struct Load {
    int32_t tiles, steps;
    __device__ __forceinline__ int64_t work() const { return static_cast<int64_t>(tiles) * steps; }
};
template <int D>
__device__ __forceinline__ Load load_of(const Args &a, int b) {
    if (b >= a.src.batch) return Load{0, 0};
    const int32_t rows = new_rows(a, b);
    if (rows <= a.few) return Load{0, 0};
    return Load{(positions(a.src, b) + kOwn - 1) / kOwn, (rows + Wide<D>::BN - 1) / Wide<D>::BN};
}
// A block's run of the steps of all items, in the order (sequence, head, tile).
template <int D>
struct Run2 {
    int64_t u, end, base;  // base: where sequence b starts
    int32_t b;
    Load load, mine;       // of sequence b, and of the lane's of the first 64
    __device__ __forceinline__ void begin(const Args &a, int w, int blocks) {
        mine = load_of<D>(a, lane_id());
        auto work_of = [&](int e) { return (e == 0 ? mine : load_of<D>(a, e + lane_id())).work() * a.kv_heads; };
        int64_t all = 0;
        for (int e = 0; e < a.src.batch; e += kWave) all += lane_value(wave_prefix(work_of(e)), kWave - 1);
        const int64_t per = max(static_cast<int64_t>(kLeastSteps), quotient(all + blocks - 1, blocks));
        u = w * per;
        end = min(all, u + per);
        base = 0;
        b = 0;
        if (u >= end) return;
        for (int e = 0; e < a.src.batch; e += kWave) {
            const int64_t here = work_of(e), incl = wave_prefix(here);
            const uint64_t past = __ballot(base + incl > u);
            if (past) {
                const int l = __builtin_ctzll(past);
                b = e + l;
                base += lane_value(incl - here, l);
                break;
            }
            base += lane_value(incl, kWave - 1);
        }
        fetch(a);
    }
    __device__ __forceinline__ void fetch(const Args &a) {
        load = b < kWave ? Load{__builtin_amdgcn_readlane(mine.tiles, b), __builtin_amdgcn_readlane(mine.steps, b)} : load_of<D>(a, b);
    }
    struct Piece {
        int32_t head, tile, t0, t1;  // steps [t0, t1) of the item
        bool starts, ends;
    };
    __device__ __forceinline__ bool next(const Args &a, Piece &p) {
        if (u >= end) return false;
        while (u >= base + load.work() * a.kv_heads) {  // a later sequence holds u
            base += load.work() * a.kv_heads;
            ++b;
            fetch(a);
        }
        const int64_t in = u - base, head = quotient(in, load.work()), rest = in - head * load.work();
        p.head = static_cast<int32_t>(head);
        p.tile = static_cast<int32_t>(quotient(rest, load.steps));
        p.t0 = static_cast<int32_t>(rest - static_cast<int64_t>(p.tile) * load.steps);
        p.t1 = static_cast<int32_t>(min(static_cast<int64_t>(load.steps), p.t0 + end - u));
        p.starts = p.t0 == 0;
        p.ends = p.t1 == load.steps;
        u += p.t1 - p.t0;
        return true;
    }
};
__device__ __forceinline__ int64_t cell_of(const Args &a, int32_t page, int head, int32_t at) {
    return ((static_cast<int64_t>(page) * a.kv_heads + head) << a.src.shift) + (at & ((1 << a.src.shift) - 1));
}
// The weight of a position: what the rows give it, and what is left of the old one.
__device__ __forceinline__ void put_weight(const Args &a, int b, int head, int64_t pos0, int32_t at, float given) {
    const int32_t page = page_at(a.src, b, at);
    if (page < 0) return;
    const int64_t cell = cell_of(a, page, head, at);
    a.out[cell] = given + (at < pos0 ? a.decay * a.in[cell] : 0.0f);
}

template <class T, int D>
__global__ __launch_bounds__(kThreads, 3) void wide_weights_kernel(Args a, int blocks) {
    using G = Wide<D>;
    __shared__ __attribute__((aligned(1024))) uint8_t qa[G::TILE], qb[G::TILE];
    __shared__ __attribute__((aligned(256))) float sta[G::BN], stb[G::BN];
    __shared__ int nonea[kWaves], noneb[kWaves];  // whether a wavefront's rows of the tile hold one that gives no weight
    const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave);
    const int col = lane & 15, g = lane >> 4;
    const int32_t d = static_cast<int32_t>(a.group.d);
    int krow[G::LPW], kch[G::LPW];
#pragma unroll
    for (int r = 0; r < G::LPW; ++r) {
        const int byte = (w * G::LPW + r) * 1024 + 16 * lane;
        krow[r] = byte / G::RB;
        kch[r] = byte % G::RB / 16 ^ swizzle<D>(krow[r]);
    }
    const int dr = col * G::RB + 16 * (g ^ swizzle<D>(col));
    const int block = static_cast<int>(xcd_block());
    Run2<D> run;
    run.begin(a, block, blocks);
    if (threadIdx.x == 0) a.rec[2 * block] = a.rec[2 * block + 1] = int4{0, 0, 0, 0};
    typename Run2<D>::Piece pc;
    while (run.next(a, pc)) {
        const Chunk chunk = chunk_of(a.src, run.b);
        const int32_t n = positions(a.src, run.b), rows = chunk.count * d, k0 = pc.tile * kOwn;
        // the steps of the part that see a key of the tile
        const int64_t from = static_cast<int64_t>(k0) - chunk.pos0 > 0 ? (static_cast<int64_t>(k0) - chunk.pos0) * d / G::BN : 0;
        const int32_t t0 = static_cast<int32_t>(max(from, static_cast<int64_t>(pc.t0))), t1 = pc.t1;
        // head and row strides are below 2^31
        auto at = [&](int32_t r, int32_t head_stride, int32_t row_stride) {
            const int32_t token = a.group.div(r);
            return static_cast<int64_t>(pc.head * d + r - token * d) * head_stride + static_cast<int64_t>(chunk.first + token) * row_stride;
        };
        const int32_t head_stride = static_cast<int32_t>(a.q.head), row_stride = static_cast<int32_t>(a.q.row);
        // Where tiles start at whole tokens a lane's places in a tile are the same in all of them but the last (as products of
        // 64 bits in every step: 87 us for 1023 tokens over 9000 positions).
        const bool regular = G::BN % d == 0;
        int64_t place[G::LPW], lse_place = 0;
        if (regular) {
#pragma unroll
            for (int r = 0; r < G::LPW; ++r) place[r] = at(krow[r], head_stride, row_stride) + 8 * kch[r];
            lse_place = at(static_cast<int32_t>(threadIdx.x) % G::BN, a.src.num_dst, 1);
        }
        float lse = 0.0f;  // of row threadIdx.x of the staged tile
        auto stage = [&](int kt, uint8_t *buf) {
            const int32_t r0 = kt * G::BN;
            if (regular && r0 + G::BN <= rows) {
                const int64_t token = kt * (G::BN / d);
                const uint16_t *const base = a.q.p + token * row_stride;
#pragma unroll
                for (int r = 0; r < G::LPW; ++r) load_to_lds16(base + place[r], buf + (w * G::LPW + r) * 1024);
                if (threadIdx.x < G::BN) lse = a.lse[lse_place + token];
                return;
            }
#pragma unroll
            for (int r = 0; r < G::LPW; ++r)  // past the end: the last row again, without weight
                load_to_lds16(a.q.p + at(min(r0 + krow[r], rows - 1), head_stride, row_stride) + 8 * kch[r], buf + (w * G::LPW + r) * 1024);
            const int32_t r = r0 + static_cast<int32_t>(threadIdx.x);
            if (threadIdx.x < G::BN) lse = r < rows ? a.lse[at(r, a.src.num_dst, 1)] : -__builtin_inff();
        };
        __syncthreads();  // the previous piece's tiles are read
        if (t0 < t1) stage(t0, qa);
        u4 k[2][G::CH];
        int32_t key[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            key[x] = k0 + w * 32 + x * 16 + col;
            const int32_t pos = min(key[x], n - 1), entry = entry_at(a.src, run.b, pos);
            const int32_t page = is_page(a.src, entry) ? entry : 0;  // a key of some page, whose weight is not stored
            const uint16_t *const p = a.src.k.p + page * a.src.k.batch + pc.head * a.src.k.head +
                                      static_cast<int64_t>(pos & ((1 << a.src.shift) - 1)) * a.src.k.row;
#pragma unroll
            for (int ch = 0; ch < G::CH; ++ch) k[x][ch] = reinterpret_cast<const u4 *>(p)[ch * 4 + g];
        }
        f4 sum[2] = {f4{0.0f, 0.0f, 0.0f, 0.0f}, f4{0.0f, 0.0f, 0.0f, 0.0f}};
        const int64_t last = static_cast<int64_t>(min(k0 + kOwn, n)) - 1 - chunk.pos0;  // the first token that sees all keys
        auto step = [&](int kt, const uint8_t *buf, const float *st) {
            const int32_t r0 = kt * G::BN;
            const bool edge = a.group.div(r0) < last;
#pragma unroll
            for (int rb = 0; rb < G::BN / 16; ++rb) {
                f4 s[2];
#pragma unroll
                for (int ch = 0; ch < G::CH; ++ch) {
                    const u4 q = *reinterpret_cast<const u4 *>(buf + (dr ^ (64 * ch)) + rb * 16 * G::RB);
#pragma unroll
                    for (int x = 0; x < 2; ++x) s[x] = T::mma(q, k[x][ch], ch == 0 ? f4{0.0f, 0.0f, 0.0f, 0.0f} : s[x]);
                }
                const f4 lse2 = *reinterpret_cast<const f4 *>(st + rb * 16 + 4 * g);
                if (edge) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int64_t pos = chunk.pos0 + a.group.div(r0 + rb * 16 + 4 * g + i);
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][i], a.c, -lse2[i]));
                            sum[x][i] += key[x] <= pos ? p : 0.0f;
                        }
                    }
                } else {
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < 4; ++i) sum[x][i] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][i], a.c, -lse2[i]));
                }
            }
        };
        // Queries of rows that give no weight are replaced by 0 in LDS (a select for each weight: 73 -> 81 us for 1023 tokens over
        // 9000 positions).
        static_assert(G::BN <= 2 * kWave, "two wavefronts look at a tile's lse");
        auto arrive = [&](uint8_t *buf, float *st, int *none) {
            loads_arrived();
            if (threadIdx.x < G::BN) st[threadIdx.x] = log2_of(lse);
            const bool some = __any(threadIdx.x < G::BN && lse == -__builtin_inff());
            if (lane == 0) none[w] = some;
            __syncthreads();
            if (uniform(none[0] | none[1]) == 0) return;
#pragma unroll 1
            for (int i = static_cast<int>(threadIdx.x); i < G::BN * G::CPR; i += kThreads)
                if (st[i / G::CPR] == __builtin_inff()) reinterpret_cast<u4 *>(buf)[i] = u4{0u, 0u, 0u, 0u};
            __syncthreads();
        };
        for (int kt = t0; kt < t1; kt += 2) {
            arrive(qa, sta, nonea);
            if (kt + 1 < t1) stage(kt + 1, qb);
            step(kt, qa, sta);
            if (kt + 1 >= t1) break;
            arrive(qb, stb, noneb);
            if (kt + 2 < t1) stage(kt + 2, qa);
            step(kt + 1, qb, stb);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const float all = column_sum((sum[x][0] + sum[x][1]) + (sum[x][2] + sum[x][3]));
            if (g != 0 || key[x] >= n) continue;
            if (pc.starts && pc.ends) put_weight(a, run.b, pc.head, chunk.pos0, key[x], all);
            else a.part[(2 * block + (pc.starts ? 1 : 0)) * kOwn + key[x] - k0] = all;
        }
        if (!(pc.starts && pc.ends) && threadIdx.x == 0) a.rec[2 * block + (pc.starts ? 1 : 0)] = int4{run.b + 1, pc.head, pc.tile, pc.ends ? 1 : 0};
    }
}

// The sums of the item that starts in block x and ends in a later one (slot 1 of x, then slot 0 of the blocks after it up to
// the one that holds the end), in order: a key a thread.
__global__ __launch_bounds__(kOwn) void add_weights_kernel(Args a, int blocks) {
    const int x = static_cast<int>(blockIdx.x);
    const int4 it = a.rec[2 * x + 1];
    if (it.x == 0) return;
    const int b = it.x - 1;
    float sum = a.part[(2 * x + 1) * kOwn + threadIdx.x];
    for (int y = x + 1; y < blocks; ++y) {
        sum += a.part[2 * y * kOwn + threadIdx.x];
        if (a.rec[2 * y].w != 0) break;
    }
    const int32_t key = it.z * kOwn + static_cast<int32_t>(threadIdx.x);
    if (key < positions(a.src, b)) put_weight(a, b, it.y, chunk_of(a.src, b).pos0, key, sum);
}

// Narrow for all sequences where they have at most 16 rows on average; otherwise for those that have, and the wide kernel for
// the others.
constexpr int64_t kFewRows = 16;
bool all_narrow(const tiga_cache &c, int64_t num_dst, int32_t heads) {
    const int64_t some = num_dst < c.batch ? num_dst : c.batch;
    return num_dst * (heads / c.kv_heads) <= kFewRows * some;
}
int64_t wide_blocks() { return 3 * static_cast<int64_t>(device_cus()); }

}  // namespace

size_t weights_ws_bytes(const tiga_cache &, int64_t num_dst, int32_t heads) {
    // of any number of source heads and sequences
    return num_dst * heads <= kFewRows ? 256 : 2 * wide_blocks() * (kOwn * sizeof(float) + sizeof(int4));
}

int accumulate(const tiga_cache &cache, int64_t num_dst, const int32_t *dst_ptr, int32_t heads, const tiga_view &q,
               const float *lse, float scale, float decay, const float *weights, float *out, void *ws, hipStream_t stream) {
    Args a{};
    a.src = pages_of(cache, num_dst, dst_ptr);
    a.q = relattn::rows_of(q);
    a.lse = lse;
    a.in = weights;
    a.out = out;
    a.c = scale * kLog2e;
    a.decay = decay;
    a.kv_heads = cache.kv_heads;
    a.group = divider(heads / cache.kv_heads);
    a.part = static_cast<float *>(ws);
    a.rec = reinterpret_cast<int4 *>(a.part + 2 * wide_blocks() * kOwn);
    const bool narrow = all_narrow(cache, num_dst, heads);
    a.few = narrow ? 0x7fffffff : static_cast<int32_t>(kFewRows);
    const int64_t positions = static_cast<int64_t>(cache.table_width) * cache.page_size;
    auto blocks_for = [&](int64_t keys, int64_t most) {
        const int64_t tiles = ceil_div(positions, keys) * cache.batch * cache.kv_heads;
        return dim3(static_cast<unsigned>(tiles < most ? (tiles < 1 ? 1 : tiles) : most));
    };
    const int blocks = static_cast<int>(wide_blocks());
    auto go = [&](auto t, auto width) -> int {
        typedef decltype(t) T;
        constexpr int D = decltype(width)::value;
        if (narrow) prof_before(stream);
        hipLaunchKernelGGL((weights_kernel<T, D>), blocks_for(Step<T, D>::BN, 2 * device_cus()), dim3(kThreads), 0, stream, a);
        if (narrow) prof_after(stream);
        if (int rc = check_launch("cache weights")) return rc;
        if (narrow) return TIGA_OK;
        prof_before(stream);
        hipLaunchKernelGGL((wide_weights_kernel<T, D>), dim3(blocks), dim3(kThreads), 0, stream, a, blocks);
        prof_after(stream);
        if (int rc = check_launch("cache weights of many rows")) return rc;
        hipLaunchKernelGGL(add_weights_kernel, dim3(blocks), dim3(kOwn), 0, stream, a, blocks);
        return check_launch("cache weights, sums");
    };
    auto by_width = [&](auto t) {
        return cache.width == 64 ? go(t, std::integral_constant<int, 64>{}) : go(t, std::integral_constant<int, 128>{});
    };
    return cache.dtype == TIGA_DT_F16 ? by_width(Half16{}) : by_width(Brain16{});
}

}  // namespace retention
}  // namespace tiga
