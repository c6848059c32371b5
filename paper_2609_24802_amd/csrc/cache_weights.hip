// What the cached positions are worth: with s_ij = scale <q_i, k_j> and the rows' lse from attention over the same cache,
//   w_j <- decay w_j + sum_{rows i of the sequence and heads of the group that see j} exp(s_ij - lse_i),
// w_j taken as 0 for the new tokens' own positions.  Every position's sum is of one wavefront, in the order of the rows.
//
// Few rows (next tokens): the time is that of reading the keys once, so tiles of keys of all sequences and heads are laid end
// to end and every block walks an equal run of them.  A wavefront takes 32 or 64 keys a step, a step ahead in registers in
// the matrix operand's layout, with the queries as the other operand: a result's column is a key, and the sum over the rows
// is one over four registers and four lanes.
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
};

// Positions of a sequence: none past the table.
__device__ __forceinline__ int32_t positions(const Pages &c, int b) {
    const int64_t n = c.length[b], most = static_cast<int64_t>(c.table_width) << c.shift;
    return static_cast<int32_t>(n < 0 ? 0 : (n > most ? most : n));
}

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
        auto fetch = [&](int e) { return e < nb ? positions(a.src, e) : 0; };
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
        n = b < kWave ? __builtin_amdgcn_readlane(mine, b) : positions(a.src, b);
    }
    struct Tile {
        int32_t b, head, n, k0;  // k0: its first key
    };
    __device__ __forceinline__ bool next(const Args &a, Tile &t) {
        if (u >= end) return false;
        while (u >= base + static_cast<int64_t>(tiles(n)) * a.kv_heads) {  // a later sequence holds u
            base += static_cast<int64_t>(tiles(n)) * a.kv_heads;
            ++b;
            n = b < kWave ? __builtin_amdgcn_readlane(mine, b) : positions(a.src, b);
        }
        const int64_t in = u - base, head = quotient(in, tiles(n));
        t = Tile{b, static_cast<int32_t>(head), n, static_cast<int32_t>(in - head * tiles(n)) * BN};
        ++u;
        return true;
    }
};

// A row that saw nothing gives no weight.
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
                    const bool sees = r < rows && at <= chunk.pos0 + a.group.div(r);
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
    Tile t0, t1;
    if (!walk.next(a, t0)) return;
    int32_t e0 = look_up(t0), e1 = 0;
    stage(t0, e0, ka, oa);
    for (;;) {
        const bool more = walk.next(a, t1);
        if (more) {
            e1 = look_up(t1);
            stage(t1, e1, kb, ob);
        }
        step(t0, e0, ka, oa);
        if (!more) break;
        const bool more2 = walk.next(a, t0);
        if (more2) {
            e0 = look_up(t0);
            stage(t0, e0, ka, oa);
        }
        step(t1, e1, kb, ob);
        if (!more2) break;
    }
}

}  // namespace

size_t weights_ws_bytes(const tiga_cache &, int64_t, int32_t) { return 256; }

int accumulate(const tiga_cache &cache, int64_t num_dst, const int32_t *dst_ptr, int32_t heads, const tiga_view &q,
               const float *lse, float scale, float decay, const float *weights, float *out, void *, hipStream_t stream) {
    Args a{};
    a.src = pages_of(cache, num_dst, dst_ptr);
    a.q = rows_of(q);
    a.lse = lse;
    a.in = weights;
    a.out = out;
    a.c = scale * kLog2e;
    a.decay = decay;
    a.kv_heads = cache.kv_heads;
    a.group = divider(heads / cache.kv_heads);
    const int64_t tiles = ceil_div(static_cast<int64_t>(cache.table_width) * cache.page_size, 4 * 4096 / cache.width) *
                          cache.batch * cache.kv_heads;
    const int64_t most = 2 * static_cast<int64_t>(device_cus());
    const dim3 grid(static_cast<unsigned>(tiles < most ? (tiles < 1 ? 1 : tiles) : most));
    prof_before(stream);
    auto go = [&](auto t) {
        typedef decltype(t) T;
        if (cache.width == 64) hipLaunchKernelGGL((weights_kernel<T, 64>), grid, dim3(kThreads), 0, stream, a);
        else hipLaunchKernelGGL((weights_kernel<T, 128>), grid, dim3(kThreads), 0, stream, a);
    };
    if (cache.dtype == TIGA_DT_F16) go(Half16{});
    else go(Brain16{});
    prof_after(stream);
    return check_launch("cache weights");
}

}  // namespace retention
}  // namespace tiga
