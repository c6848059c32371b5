// Vector-Jacobian product of causal attention within packed sequences.  With p_ij = exp(s_ij - lse_i) for j <= i, 0 after,
// delta_i = <dy_i, y_i> and ds_ij = p_ij (<dy_i, v_j> - delta_i):
//   dq_i = scale sum_{j <= i} ds_ij k_j,   dk_j = scale sum_{i >= j} ds_ij q_i,   dv_j = sum_{i >= j} p_ij dy_i,
// i over the tokens of every head that shares source head j's.  The products are those of the rectangular relation
// (relattn_bwd.hpp): dq with 128 rows owned and the keys up to the diagonal streamed, then dk, dv with 128 keys owned and
// the rows from the last token back to the diagonal streamed, so that tiles of one source head that run together read the
// same rows.  Only tiles that the diagonal cuts are masked.
//
// An item is one owned tile of a sequence and source head, in the order that packed_plan.hpp lays down.  Parts of items that
// are cut along the streamed axis leave fp32 sums in the workspace, which packed_reduce_kernel adds in order.
//
// Measured (MI355X): 16,384 tokens of ragged sequences, 16 heads over 4 of width 128, bf16: dq 955 to 1032 us (1.16 to 1.25
// PFLOP/s), dk and dv 1617 to 1792 (0.9 to 1.0; a large library product reaches 1.24 in the same minutes), the order 8, the
// parts' sums 8: bound by the matrix cores and, in dk and dv, whose two accumulators leave one wavefront to a SIMD, by LDS
// reads beside them.  Short sequences (61 with 8001 tokens in all, 16 heads of width 64, f16): order 8, peaks 8, dq 39, dk
// and dv 48, sums of no parts 4, where 131 MB take 27: dk and dv form whole squares of 128 x 128, 21 GFLOP where the pairs
// that exist need 9, and P and DS are formed in both launches.
//
// P and DS enter the products in the input type (relattn_bwd.hpp).  Where a gradient is a sum of few ds, their rounding is not
// averaged out: of 7 rows in 4 sequences, bf16, dq and dk were 0.003 off where fp32 rounded once is 0.0018.
#include "packed_plan.hpp"
#include "relattn.hpp"
#include "relattn_bwd.hpp"

namespace tiga {
namespace relattn {

namespace {

struct Args {
    Rows q, k, v, y, dy, dq, dk, dv;  // one packed axis: the batch strides are not used
    const float *lse;
    const int32_t *ptr;
    float *lse2, *delta;  // [heads * num_rows + 1]: the last is what rows past the end have (no weight)
    f2 *peak;             // [kv_heads][slots]: of 128 tokens' values and cotangents (binary16)
    int32_t slots;
    int32_t num_rows, batch, kv_heads;
    Divider group;
    int64_t stats;        // heads * num_rows
    float scale;
    const int4 *rows_table, *keys_table;  // the pieces of dq, and of dk and dv
    float *rows_part, *keys_part;         // sums of parts
};

// Row r of a sequence's source head is token r / group of head r % group of its group.
__device__ __forceinline__ int64_t row_at(const Args &a, const Rows &t, int32_t first, int kv, int32_t r) {
    const int32_t d = static_cast<int32_t>(a.group.d), token = a.group.div(r), g = r - token * d;
    // row and head strides are below 2^31
    return static_cast<int64_t>(kv * d + g) * static_cast<int32_t>(t.head) +
           static_cast<int64_t>(first + token) * static_cast<int32_t>(t.row);
}
__device__ __forceinline__ int64_t stat_at(const Args &a, int32_t first, int kv, int32_t r) {
    const int32_t d = static_cast<int32_t>(a.group.d), token = a.group.div(r), g = r - token * d;
    return static_cast<int64_t>(kv * d + g) * a.num_rows + first + token;
}

// ------------------------------------------------------------------------------------------ items

__device__ __forceinline__ Item item_of(const Args &a, const int4 *table, int32_t mult, int32_t id) {
    return item_of(table, a.kv_heads, mult, id);
}
// Sums [operand][owned][D] of a part: cut items come first, so that a piece's number is its place.
template <int D, int M>
__device__ __forceinline__ float *part_at(const Args &a, int32_t id) {
    return (M == 1 ? a.rows_part : a.keys_part) + static_cast<int64_t>(id) * M * kOwn * D;
}

// Gradients of rows of no sequence: before ptr[0] and behind ptr[batch].
template <int D>
__device__ __forceinline__ void clear_outside(const Args &a, const Rows &t, int64_t heads) {
    if (!t.p) return;
    const Run inside = a.batch > 0 ? run_between(a.ptr, 0, a.batch, a.num_rows) : Run{0, 0};
    const int32_t outside = a.num_rows - inside.count;
    if (outside == 0) return;
    const int64_t all = outside * heads * (D / 8);
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < all; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t head = i / (D / 8) % heads;
        int64_t row = i / (D / 8) / heads;
        if (row >= inside.first) row += inside.count;
        reinterpret_cast<u4 *>(const_cast<uint16_t *>(t.p) + head * t.head + row * t.row)[i % (D / 8)] = u4{0u, 0u, 0u, 0u};
    }
}

// ------------------------------------------------------------------------------------------ range of binary16

// Where the peaks of 128 tokens lie: the runs of tiles of all sequences, each from at or behind the end of the one before.
__device__ __forceinline__ int32_t slot_of(const Item &it, int32_t tile) { return it.run.first / kOwn + it.b + tile; }

// max |v| and max |dy|_1 of 128 tokens of a source head.  What is not finite is passed over: the results that it reaches are
// not finite, and it must not change the scale of the others.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void packed_peak_kernel(Args a) {
    constexpr int L = D / 8, ROWS = kThreads / L;  // 16 bytes a lane
    __shared__ f2 of_wave[kWaves];
    const Item it = item_of(a, a.keys_table, 1, static_cast<int32_t>(blockIdx.x));
    if (it.level == 0 || it.part != 0) return;
    const int32_t t0 = (it.tiles - it.level) * kOwn, t1 = min(t0 + kOwn, it.run.count);
    const int first = static_cast<int>(threadIdx.x) / L, c = static_cast<int>(threadIdx.x) % L;
    auto finite = [](float x) { return x < __builtin_inff() ? x : 0.0f; };  // of an absolute value; NaN too
    f2 top{0.0f, 0.0f};
    const u4 *const v = reinterpret_cast<const u4 *>(a.v.p + it.kv * a.v.head + it.run.first * a.v.row) + c;
    for (int32_t j = t0 + first; j < t1; j += ROWS) {
        const u4 x = v[j * (a.v.row / 8)];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const f2 u = T::unpack(x[e]);
            top.x = fmaxf(top.x, fmaxf(finite(__builtin_fabsf(u.x)), finite(__builtin_fabsf(u.y))));
        }
    }
    const int32_t d = static_cast<int32_t>(a.group.d);
#pragma unroll 4
    for (int32_t r = t0 * d + first; r < t1 * d; r += ROWS) {
        float l1 = sum_abs<T>(reinterpret_cast<const u4 *>(a.dy.p + row_at(a, a.dy, it.run.first, it.kv, r))[c]);
#pragma unroll
        for (int s = 1; s < L; s <<= 1) l1 += shfl_xor_f(l1, s);  // whole rows: the lanes of a row leave together
        top.y = fmaxf(top.y, finite(l1));
    }
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
        top.x = fmaxf(top.x, shfl_xor_f(top.x, s));
        top.y = fmaxf(top.y, shfl_xor_f(top.y, s));
    }
    if (lane_id() == 0) of_wave[threadIdx.x / kWave] = top;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < kWaves; ++w) top = f2{fmaxf(top.x, of_wave[w].x), fmaxf(top.y, of_wave[w].y)};
    a.peak[static_cast<int64_t>(it.kv) * a.slots + slot_of(it, it.tiles - it.level)] = top;
}
// Of the whole sequence and source head.
__device__ __forceinline__ f2 peak_of(const Args &a, const Item &it) {
    const f2 *const p = a.peak + static_cast<int64_t>(it.kv) * a.slots + slot_of(it, 0);
    f2 top{0.0f, 0.0f};
    for (int i = lane_id(); i < (it.run.count + kOwn - 1) / kOwn; i += kWave) top = f2{fmaxf(top.x, p[i].x), fmaxf(top.y, p[i].y)};
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        top.x = fmaxf(top.x, shfl_xor_f(top.x, d));
        top.y = fmaxf(top.y, shfl_xor_f(top.y, d));
    }
    return f2{__uint_as_float(uniform(__float_as_uint(top.x))), __uint_as_float(uniform(__float_as_uint(top.y)))};
}

// ------------------------------------------------------------------------------------------ tiles in LDS

// This lane's places in a streamed tile: rows and chunks of its direct loads, offsets of its operand reads.
template <int D>
struct Places {
    using G = Geo<D>;
    int krow[G::LPW], kch[G::LPW], dr, tr;
    __device__ __forceinline__ Places(int lane, int w) {
        const int col = lane & 15, g = lane >> 4;
#pragma unroll
        for (int r = 0; r < G::LPW; ++r) {
            const int byte = (w * G::LPW + r) * 1024 + 16 * lane;
            krow[r] = byte / G::RB;
            kch[r] = byte % G::RB / 16 ^ swizzle<D>(krow[r]);
        }
        dr = col * G::RB + 16 * (g ^ swizzle<D>(col));
        const int trow = 4 * g + col / 4;
        tr = trow * G::RB + 16 * ((col % 4 / 2) ^ swizzle<D>(trow)) + 8 * (col % 2);
    }
};
// This lane's 16 bytes of its wavefront's load r of a tile.
template <int D>
__device__ __forceinline__ u4 *own_rows(uint8_t *tile, int w, int r) {
    return reinterpret_cast<u4 *>(tile + (w * Geo<D>::LPW + r) * 1024 + 16 * lane_id());
}

// Tiles that the diagonal cuts hold keys that some rows do not see, and a weight of 0 times an infinity would be NaN.  They
// are looked through for values that are not finite before the barrier that makes them readable; where there are any, those
// are replaced by 0 in LDS, and the rows or keys that see them are given NaN, or the value itself, apart.
// Leaves in *found whether this wavefront's rows of the tile (or two of them) hold one.
template <class T, int D>
__device__ __forceinline__ void look_through(uint8_t *t1, uint8_t *t2, int w, int *found) {
    uint32_t bad = 0;
#pragma unroll
    for (int r = 0; r < Geo<D>::LPW; ++r) {
        bad |= any_wild<T>(*own_rows<D>(t1, w, r));
        if (t2) bad |= any_wild<T>(*own_rows<D>(t2, w, r));
    }
    const bool here = __any(bad != 0);
    if (lane_id() == 0) found[w] = here;
}
__device__ __forceinline__ bool any_found(const int *found) { return uniform(found[0] | found[1] | found[2] | found[3]) != 0; }

// ------------------------------------------------------------------------------------------ dq

// P (in the place of the scores) and DP of 32 streamed keys where the diagonal cuts: this lane's rows see the first
// rel[qb] of the keys from its own 4 g on.
template <class T, int D>
__device__ __forceinline__ void weigh_causal(Scores<T, D> &f, float c, const float *lse2, const int32_t *rel) {
#pragma unroll
    for (int qb = 0; qb < 2; ++qb)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(f.s[e][qb][i], c, -lse2[qb]));
                const bool sees = e * 16 + i < rel[qb];
                f.s[e][qb][i] = sees ? p : 0.0f;
                f.dp[e][qb][i] = sees ? f.dp[e][qb][i] : 0.0f;
            }
}

template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void packed_query_kernel(Args a) {
    using G = Geo<D>;
    __shared__ __attribute__((aligned(1024))) uint8_t y1a[G::TILE], y2a[G::TILE], y1b[G::TILE], y2b[G::TILE];
    __shared__ int found[2][kWaves];
    const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave);
    const int col = lane & 15, g = lane >> 4;
    const int32_t d = static_cast<int32_t>(a.group.d);

    if (blockIdx.x == 0 && threadIdx.x == 0) {  // what rows past the end have
        a.lse2[a.stats] = __builtin_inff();
        a.delta[a.stats] = 0.0f;
    }
    clear_outside<D>(a, a.dq, static_cast<int64_t>(a.kv_heads) * d);
    const Item it = item_of(a, a.rows_table, d, static_cast<int32_t>(blockIdx.x));
    if (it.level == 0) return;
    const int32_t rows = it.run.count * d, own0 = (it.level - 1) * kOwn;
    const int32_t keys = a.group.div(min(own0 + kOwn, rows) - 1) + 1;  // that the tile's last row sees
    const int32_t all_steps = (keys + G::BN - 1) / G::BN;
    const int32_t first_step = part_start(all_steps, it.part, it.parts), steps = part_start(all_steps, it.part + 1, it.parts);
    // The rounding of y (of itself and of the weights in it) makes an error of u |dy| |y| of delta, which matters over few
    // sources: where the tile's keys are few, delta is formed as sum_j p_ij <dy_i, v_j> in fp32, by the tiles' products.
    const bool few = keys <= kOwn;

    const Places<D> at(lane, w);
    const uint16_t *const kb = a.k.p + it.kv * a.k.head + it.run.first * a.k.row;
    const uint16_t *const vb = a.v.p + it.kv * a.v.head + it.run.first * a.v.row;
    auto stage = [&](int kt, uint8_t *b1, uint8_t *b2) {
        const int32_t k0 = kt * G::BN;
        const uint8_t *const kt0 = reinterpret_cast<const uint8_t *>(kb + k0 * a.k.row);
        const uint8_t *const vt0 = reinterpret_cast<const uint8_t *>(vb + k0 * a.v.row);
#pragma unroll
        for (int r = 0; r < G::LPW; ++r) {
            const int run = (w * G::LPW + r) * 1024;
            const uint32_t i = min(at.krow[r], keys - 1 - k0);  // past the end: the last key again, without weight
            load_to_lds16(kt0 + (2u * i * static_cast<uint32_t>(a.k.row) + 16u * at.kch[r]), b1 + run);
            load_to_lds16(vt0 + (2u * i * static_cast<uint32_t>(a.v.row) + 16u * at.kch[r]), b2 + run);
        }
    };
    if (few || a.dq.p) stage(first_step, y1a, y2a);  // under way while the owned operands arrive

    // owned operands; columns past the end repeat the last (what they sum is not stored)
    u4 x1[2][G::CH], x2[2][G::CH];
    f2 peak{0.0f, 0.0f};
    if constexpr (kScaled<T>) peak = peak_of(a, it);
    const float h = kScaled<T> ? two_to(up(peak.x * peak.y) - kUp) : 1.0f;
    float own[2], own_delta[2];
    int own_up[2] = {0, 0};  // the exponent of DS
    int32_t sees[2];
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        const int32_t o = min(own0 + w * 32 + qb * 16 + col, rows - 1);
        sees[qb] = a.group.div(o) + 1;
        own[qb] = log2_of(a.lse[stat_at(a, it.run.first, it.kv, o)]);
        own_delta[qb] = 0.0f;
        const uint16_t *const p1 = a.q.p + row_at(a, a.q, it.run.first, it.kv, o);
        const uint16_t *const p2 = a.dy.p + row_at(a, a.dy, it.run.first, it.kv, o);
#pragma unroll
        for (int ch = 0; ch < G::CH; ++ch) {
            x1[qb][ch] = reinterpret_cast<const u4 *>(p1)[ch * 4 + g];
            x2[qb][ch] = reinterpret_cast<const u4 *>(p2)[ch * 4 + g];
        }
        if constexpr (kScaled<T>) {
            float l1 = 0.0f;
#pragma unroll
            for (int ch = 0; ch < G::CH; ++ch) l1 += sum_abs<T>(x2[qb][ch]);
            own_up[qb] = up(column_sum(l1) * peak.x);
            own[qb] -= static_cast<float>(own_up[qb]);
        }
        if (!few) own_delta[qb] = column_sum(row_product<T>(x2[qb], a.y.p + row_at(a, a.y, it.run.first, it.kv, o), g));
    }
    // The owned rows' statistics, for dk and dv: delta is there.
    auto leave_stats = [&] {
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            const int32_t o = own0 + w * 32 + qb * 16 + col;
            if (o < rows && g == 0) {
                const int64_t at = stat_at(a, it.run.first, it.kv, o);
                a.lse2[at] = kScaled<T> ? log2_of(a.lse[at]) - kUp : own[qb];
                a.delta[at] = own_delta[qb] * h;
            }
        }
    };
    if (!few) {
        if (it.part == 0) leave_stats();
        if (!a.dq.p) return;
    }
    Sums<T, D, kQuery> acc;
#pragma unroll
    for (int db = 0; db < G::DB; ++db) acc.a1[db][0] = acc.a1[db][1] = f4{0.0f, 0.0f, 0.0f, 0.0f};

    const float c = a.scale * kLog2e;
    const int32_t least = a.group.div(own0) + 1;                                                  // the tile's first row sees
    const int32_t my_most = own0 + w * 32 < rows ? a.group.div(min(own0 + w * 32 + 31, rows - 1)) + 1 : 0;
    auto cut = [&](int kt) { return (kt + 1) * G::BN > least; };
    // Before and after the barrier that makes a tile readable.
    auto tidy = [&](int kt, uint8_t *b1, int n) {
        if (cut(kt)) look_through<T, D>(b1, nullptr, w, found[n]);
    };
    // A key that is not finite makes the sums of the rows that see it NaN, and counts as 0 without it.
    auto mend = [&](int kt, uint8_t *b1, int n) {
        if (!cut(kt) || !any_found(found[n])) return;
        for (int k = 0; k < G::BN && kt * G::BN + k < keys; ++k) {
            uint32_t bad = 0;
#pragma unroll 1
            for (int i = 0; i < G::CPR; ++i) bad |= any_wild<T>(reinterpret_cast<const u4 *>(b1 + k * G::RB)[i]);
            if (uniform(bad) == 0) continue;
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) {
                const float nan = kt * G::BN + k < sees[qb] ? __builtin_nanf("") : 0.0f;
                own_delta[qb] += nan;
#pragma unroll
                for (int db = 0; db < G::DB; ++db) acc.a1[db][qb] += nan;
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < G::LPW; ++r) *own_rows<D>(b1, w, r) = without_wild<T>(*own_rows<D>(b1, w, r));
        __syncthreads();
    };
    // 32 keys of a tile that the diagonal may cut
    auto form = [&](Scores<T, D> &f, int kt, int kc, const uint8_t *b1, const uint8_t *b2) {
        f.form(x1, x2, b1 + kc * 32 * G::RB, b2 + kc * 32 * G::RB, at.dr, [](int) {});
        const int32_t k0 = kt * G::BN + kc * 32, rel[2] = {sees[0] - k0 - 4 * g, sees[1] - k0 - 4 * g};
        weigh_causal<T, D>(f, c, own, rel);
    };
    auto step = [&](int kt, const uint8_t *b1, const uint8_t *b2) {
#pragma unroll 1
        for (int kc = 0; kc < G::KC; ++kc) {
            if (kt * G::BN + kc * 32 >= my_most) break;
            Scores<T, D> f;
            form(f, kt, kc, b1, b2);
            add_keys<T, D, kQuery>(acc, f, own_delta, b1 + kc * 32 * G::RB, at.tr);
        }
    };
    auto plain = [&](const uint8_t *b1, const uint8_t *b2) {
#pragma unroll
        for (int kc = 0; kc < G::KC; ++kc) {
            Scores<T, D> f;
            f.form(x1, x2, b1 + kc * 32 * G::RB, b2 + kc * 32 * G::RB, at.dr, [](int) {});
            weigh<T, D>(f, c, own, false, 0, g);
            add_keys<T, D, kQuery>(acc, f, own_delta, b1 + kc * 32 * G::RB, at.tr);
        }
    };
    auto deltas = [&](int kt, const uint8_t *b1, const uint8_t *b2) {
#pragma unroll 1
        for (int kc = 0; kc < G::KC; ++kc) {
            if (kt * G::BN + kc * 32 >= my_most) break;
            Scores<T, D> f;
            form(f, kt, kc, b1, b2);
#pragma unroll
            for (int qb = 0; qb < 2; ++qb)
#pragma unroll
                for (int i = 0; i < 8; ++i) own_delta[qb] += f.s[i / 4][qb][i % 4] * f.dp[i / 4][qb][i % 4];
        }
    };
    if (few) {  // at most two tiles, both in LDS (and never cut)
        if (steps > 1) stage(1, y1b, y2b);
        loads_arrived();
        tidy(0, y1a, 0);
        if (steps > 1) tidy(1, y1b, 1);
        __syncthreads();
        mend(0, y1a, 0);
        if (steps > 1) mend(1, y1b, 1);
        deltas(0, y1a, y2a);
        if (steps > 1) deltas(1, y1b, y2b);
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            own_delta[qb] = column_sum(own_delta[qb]);
            if (kScaled<T>) own_delta[qb] *= two_to(-own_up[qb]);
        }
        leave_stats();
        if (!a.dq.p) return;
        step(0, y1a, y2a);
        if (steps > 1) step(1, y1b, y2b);
    } else {
        int kt = first_step;
        // tiles that all rows see whole, in pairs
        const int seen = min(least / G::BN, steps);
        for (const int whole = seen > kt ? kt + (seen - kt & ~1) : kt; kt < whole; kt += 2) {
            loads_arrived();
            __syncthreads();
            stage(kt + 1, y1b, y2b);
            plain(y1a, y2a);
            loads_arrived();
            __syncthreads();
            if (kt + 2 < steps) stage(kt + 2, y1a, y2a);
            plain(y1b, y2b);
        }
        // one exit, after a whole turn of both buffers: with another between them the sums are moved and spill
        for (; kt + 1 < steps; kt += 2) {
            loads_arrived();
            tidy(kt, y1a, 0);
            __syncthreads();
            stage(kt + 1, y1b, y2b);
            mend(kt, y1a, 0);
            step(kt, y1a, y2a);
            loads_arrived();
            tidy(kt + 1, y1b, 1);
            __syncthreads();
            if (kt + 2 < steps) stage(kt + 2, y1a, y2a);
            mend(kt + 1, y1b, 1);
            step(kt + 1, y1b, y2b);
        }
        if (kt < steps) {
            loads_arrived();
            tidy(kt, y1a, 0);
            __syncthreads();
            mend(kt, y1a, 0);
            step(kt, y1a, y2a);
        }
    }
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        const int32_t o = own0 + w * 32 + qb * 16 + col;
        if (o >= rows) continue;
        if (it.parts > 1) {
            float *const p = part_at<D, 1>(a, static_cast<int32_t>(blockIdx.x)) + (o - own0) * D;
            const float f = kScaled<T> ? two_to(-own_up[qb]) : 1.0f;
#pragma unroll
            for (int db = 0; db < G::DB; ++db) *reinterpret_cast<f4 *>(p + db * 16 + g * 4) = acc.a1[db][qb] * f;
            continue;
        }
        const float f = kScaled<T> ? a.scale * two_to(-own_up[qb]) : a.scale;
        uint16_t *const p = const_cast<uint16_t *>(a.dq.p) + row_at(a, a.dq, it.run.first, it.kv, o);
#pragma unroll
        for (int db = 0; db < G::DB; ++db) {
            const f4 v = acc.a1[db][qb] * f;
            *reinterpret_cast<u2 *>(p + db * 16 + g * 4) = u2{T::pack(v[0], v[1]), T::pack(v[2], v[3])};
        }
    }
}

// ------------------------------------------------------------------------------------------ dk, dv

// Which of this lane's 16 pairs of 32 streamed rows from `r0` on exist, as Weights numbers them: key[qb] is at or before the
// row's token.
__device__ __forceinline__ uint32_t pairs_of(const Divider &group, int32_t r0, int g, const int32_t *key) {
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int32_t token = group.div(r0 + i / 4 * 16 + 4 * g + i % 4);
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) bits |= key[qb] <= token ? 1u << (8 * qb + i) : 0u;
    }
    return bits;
}

template <class T, int D>
__global__ __launch_bounds__(kThreads, (kBlocks<D, true>)) void packed_keys_kernel(Args a) {
    using G = Geo<D>;
    __shared__ __attribute__((aligned(1024))) uint8_t y1a[G::TILE], y2a[G::TILE], y1b[G::TILE], y2b[G::TILE];
    __shared__ __attribute__((aligned(256))) float sta[2 * G::BN], stb[2 * G::BN];
    __shared__ int found[2][kWaves];
    const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave);
    const int col = lane & 15, g = lane >> 4;
    const int32_t d = static_cast<int32_t>(a.group.d);

    clear_outside<D>(a, a.dk, a.kv_heads);
    clear_outside<D>(a, a.dv, a.kv_heads);
    const Item it = item_of(a, a.keys_table, 1, static_cast<int32_t>(blockIdx.x));
    if (it.level == 0) return;
    const int32_t own_n = it.run.count, own0 = (it.tiles - it.level) * kOwn, rows = own_n * d;
    // row tiles from the last one back to that of the first owned key (128 tokens are whole tiles)
    const int32_t end = (rows + G::BN - 1) / G::BN, all_steps = end - own0 / G::BN * d;
    const int32_t first_step = part_start(all_steps, it.part, it.parts), steps = part_start(all_steps, it.part + 1, it.parts);

    const Places<D> at(lane, w);
    // Where tiles start at whole tokens a lane's places in a tile are the same in all of them but the sequence's last (dk and dv
    // of 16,384 ragged tokens, 16 heads over 4 of 128: 1733 us without, 1677 with; at width 64 the registers are not there).
    const int64_t reach = static_cast<int64_t>(d - 1) * max(a.q.head, a.dy.head) + static_cast<int64_t>(G::BN / d) * max(a.q.row, a.dy.row);
    const bool regular = D == 128 && G::BN % d == 0 && reach < (int64_t(1) << 30);
    uint32_t q_place[G::LPW], dy_place[G::LPW];  // bytes
#pragma unroll
    for (int r = 0; r < G::LPW; ++r) {
        const uint32_t token = a.group.div(at.krow[r]), head = at.krow[r] - token * d;
        q_place[r] = 2u * (head * static_cast<uint32_t>(a.q.head) + token * static_cast<uint32_t>(a.q.row) + 8u * at.kch[r]);
        dy_place[r] = 2u * (head * static_cast<uint32_t>(a.dy.head) + token * static_cast<uint32_t>(a.dy.row) + 8u * at.kch[r]);
    }
    auto stage = [&](int n, uint8_t *b1, uint8_t *b2, float *stats) {
        const int32_t k0 = (end - 1 - n) * G::BN;
        if (regular && n > 0) {
            const int64_t token = it.run.first + (end - 1 - n) * (G::BN / d), head = static_cast<int64_t>(it.kv) * d;
            const uint8_t *const q0 = reinterpret_cast<const uint8_t *>(a.q.p + head * a.q.head + token * a.q.row);
            const uint8_t *const dy0 = reinterpret_cast<const uint8_t *>(a.dy.p + head * a.dy.head + token * a.dy.row);
#pragma unroll
            for (int r = 0; r < G::LPW; ++r) {
                load_to_lds16(q0 + q_place[r], b1 + (w * G::LPW + r) * 1024);
                load_to_lds16(dy0 + dy_place[r], b2 + (w * G::LPW + r) * 1024);
            }
        } else {
#pragma unroll
            for (int r = 0; r < G::LPW; ++r) {
                const int run = (w * G::LPW + r) * 1024;
                const int32_t i = min(k0 + at.krow[r], rows - 1);  // past the end: the last row again, without weight
                load_to_lds16(a.q.p + row_at(a, a.q, it.run.first, it.kv, i) + 8 * at.kch[r], b1 + run);
                load_to_lds16(a.dy.p + row_at(a, a.dy, it.run.first, it.kv, i) + 8 * at.kch[r], b2 + run);
            }
        }
        // 64 lanes, 4 bytes each: the first half of the needed wavefronts takes lse2, the other delta
        constexpr int kNeed = 2 * G::BN / kWave;
        if (w < kNeed) {
            const int32_t i = k0 + w % (kNeed / 2) * kWave + lane;
            const int64_t s = i < rows ? stat_at(a, it.run.first, it.kv, i) : a.stats;
            __builtin_amdgcn_global_load_lds((w < kNeed / 2 ? a.lse2 : a.delta) + s,
                                             (__attribute__((address_space(3))) void *)(stats + w * kWave), 4, 0, 0);
        }
    };
    stage(first_step, y1a, y2a, sta);  // under way while the owned operands arrive

    // owned operands; columns past the end repeat the last (what they sum is not stored)
    u4 x1[2][G::CH], x2[2][G::CH];
    f2 peak{0.0f, 0.0f};
    if constexpr (kScaled<T>) peak = peak_of(a, it);
    const int keys_up = kScaled<T> ? up(peak.x * peak.y) : 0;               // the exponent of DS
    const float h = kScaled<T> ? two_to(keys_up - kUp) : 1.0f;              // P has kUp of it
    int32_t key[2];
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        key[qb] = own0 + w * 32 + qb * 16 + col;
        const int32_t o = it.run.first + min(key[qb], own_n - 1);
        const uint16_t *const p1 = a.k.p + it.kv * a.k.head + o * a.k.row, *const p2 = a.v.p + it.kv * a.v.head + o * a.v.row;
#pragma unroll
        for (int ch = 0; ch < G::CH; ++ch) {
            x1[qb][ch] = reinterpret_cast<const u4 *>(p1)[ch * 4 + g];
            x2[qb][ch] = reinterpret_cast<const u4 *>(p2)[ch * 4 + g];
        }
    }
    Sums<T, D, kKeys> acc;
#pragma unroll
    for (int db = 0; db < G::DB; ++db)
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) acc.a1[db][qb] = acc.a2[db][qb] = f4{0.0f, 0.0f, 0.0f, 0.0f};

    const float c = a.scale * kLog2e;
    // tiles whose first row does not see the last owned key
    auto cut = [&](int n) { return static_cast<int64_t>(end - 1 - n) * G::BN < static_cast<int64_t>(own0 + kOwn - 1) * d; };
    auto tidy = [&](int n, uint8_t *b1, uint8_t *b2, int which) {
        if (cut(n)) look_through<T, D>(b1, b2, w, found[which]);
    };
    // A row whose query is not finite has NaN for weights, one whose cotangent is not finite for ds: the sums of the keys that
    // see it get those apart, and dv the cotangent itself; without them the row has no weight, or none in ds.
    auto mend = [&](int n, uint8_t *b1, uint8_t *b2, float *stats, int which) {
        if (!cut(n) || !any_found(found[which])) return;
        const int32_t k0 = (end - 1 - n) * G::BN;
        for (int k = 0; k < G::BN && k0 + k < rows; ++k) {
            const int32_t token = a.group.div(k0 + k);
            uint32_t bad1 = 0, bad2 = 0;
#pragma unroll 1
            for (int i = 0; i < G::CPR; ++i) {
                bad1 |= any_wild<T>(reinterpret_cast<const u4 *>(b1 + k * G::RB)[i]);
                bad2 |= any_wild<T>(reinterpret_cast<const u4 *>(b2 + k * G::RB)[i]);
            }
            if (uniform(bad1 | bad2) == 0) continue;
            const float nan = __builtin_nanf(""), in_dv = uniform(bad1) ? nan : 0.0f;
#pragma unroll
            for (int db = 0; db < G::DB; ++db) {
                const u2 x = *reinterpret_cast<const u2 *>(b2 + k * G::RB + 16 * ((2 * db + g / 2) ^ swizzle<D>(k)) + 8 * (g % 2));
#pragma unroll
                for (int qb = 0; qb < 2; ++qb) {
                    add_wild<T>(acc.a2[db][qb], x, key[qb] <= token);
                    acc.a1[db][qb] += key[qb] <= token ? nan : 0.0f;
                    acc.a2[db][qb] += key[qb] <= token ? in_dv : 0.0f;
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < G::LPW; ++r) {
            u4 *const p1 = own_rows<D>(b1, w, r), *const p2 = own_rows<D>(b2, w, r);
            if (any_wild<T>(*p1)) stats[at.krow[r]] = __builtin_inff();
            if (any_wild<T>(*p1) || any_wild<T>(*p2)) stats[G::BN + at.krow[r]] = 0.0f;
            *p1 = without_wild<T>(*p1);
            *p2 = without_wild<T>(*p2);
        }
        __syncthreads();
    };
    auto plain = [&](const uint8_t *b1, const uint8_t *b2, const float *stats) {
#pragma unroll
        for (int kc = 0; kc < G::KC; kc += 2)
            rows_step<T, D>(acc, x1, x2, b1 + kc * 32 * G::RB, b2 + kc * 32 * G::RB, at.dr, at.tr, c, h, stats + kc * 32,
                            stats + G::BN + kc * 32, g);
    };
    auto step = [&](int n, const uint8_t *b1, const uint8_t *b2, const float *stats) {
        const int32_t k0 = (end - 1 - n) * G::BN;
#pragma unroll 1
        for (int kc = 0; kc < G::KC; kc += 2) {
            const uint32_t exists[2] = {pairs_of(a.group, k0 + kc * 32, g, key), pairs_of(a.group, k0 + kc * 32 + 32, g, key)};
            rows_step<T, D, true>(acc, x1, x2, b1 + kc * 32 * G::RB, b2 + kc * 32 * G::RB, at.dr, at.tr, c, h, stats + kc * 32,
                                  stats + G::BN + kc * 32, g, exists);
        }
    };
    int n = first_step;
    // tiles whose rows all see every owned key, in pairs
    const int64_t from = (static_cast<int64_t>(own0 + kOwn - 1) * d + G::BN - 1) / G::BN;
    const int seen = from < end ? min(static_cast<int>(end - from), steps) : 0;
    for (const int whole = seen > n ? n + (seen - n & ~1) : n; n < whole; n += 2) {
        loads_arrived();
        __syncthreads();
        stage(n + 1, y1b, y2b, stb);
        plain(y1a, y2a, sta);
        loads_arrived();
        __syncthreads();
        if (n + 2 < steps) stage(n + 2, y1a, y2a, sta);
        plain(y1b, y2b, stb);
    }
    for (; n + 1 < steps; n += 2) {
        loads_arrived();
        tidy(n, y1a, y2a, 0);
        __syncthreads();
        stage(n + 1, y1b, y2b, stb);
        mend(n, y1a, y2a, sta, 0);
        step(n, y1a, y2a, sta);
        loads_arrived();
        tidy(n + 1, y1b, y2b, 1);
        __syncthreads();
        if (n + 2 < steps) stage(n + 2, y1a, y2a, sta);
        mend(n + 1, y1b, y2b, stb, 1);
        step(n + 1, y1b, y2b, stb);
    }
    if (n < steps) {
        loads_arrived();
        tidy(n, y1a, y2a, 0);
        __syncthreads();
        mend(n, y1a, y2a, sta, 0);
        step(n, y1a, y2a, sta);
    }
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        if (key[qb] >= own_n) continue;
        const int32_t o = it.run.first + key[qb];
        if (it.parts > 1) {
            float *const p = part_at<D, 2>(a, static_cast<int32_t>(blockIdx.x)) + (key[qb] - own0) * D;
            const float f1 = kScaled<T> ? two_to(-keys_up) : 1.0f, f2 = kScaled<T> ? two_to(-kUp) : 1.0f;
#pragma unroll
            for (int db = 0; db < G::DB; ++db) {
                *reinterpret_cast<f4 *>(p + db * 16 + g * 4) = acc.a1[db][qb] * f1;
                *reinterpret_cast<f4 *>(p + kOwn * D + db * 16 + g * 4) = acc.a2[db][qb] * f2;
            }
            continue;
        }
        const float f1 = kScaled<T> ? a.scale * two_to(-keys_up) : a.scale, f2 = kScaled<T> ? two_to(-kUp) : 1.0f;
        uint16_t *const pk = const_cast<uint16_t *>(a.dk.p) + it.kv * a.dk.head + o * a.dk.row;
        uint16_t *const pv = const_cast<uint16_t *>(a.dv.p) + it.kv * a.dv.head + o * a.dv.row;
        auto put = [&](uint16_t *p, f4 v) { *reinterpret_cast<u2 *>(p) = u2{T::pack(v[0], v[1]), T::pack(v[2], v[3])}; };
#pragma unroll
        for (int db = 0; db < G::DB; ++db) {
            if (a.dk.p) put(pk + db * 16 + g * 4, acc.a1[db][qb] * f1);
            if (a.dv.p) put(pv + db * 16 + g * 4, acc.a2[db][qb] * f2);
        }
    }
}

// Adds the parts of the item whose first part is piece `id`, in order: 4 widths a thread.
template <class T, int D, bool KEYS>
__device__ __forceinline__ void add_parts(const Args &a, int32_t id) {
    constexpr int L = D / 4, M = KEYS ? 2 : 1;
    const int32_t d = KEYS ? 1 : static_cast<int32_t>(a.group.d);
    const Item it = item_of(a, KEYS ? a.keys_table : a.rows_table, d, id);
    if (it.level == 0 || it.part != 0 || it.parts == 1) return;
    const int32_t own0 = (KEYS ? it.tiles - it.level : it.level - 1) * kOwn, rows = min(it.run.count * d - own0, kOwn);
    for (int32_t i = static_cast<int32_t>(blockIdx.y) * kThreads + threadIdx.x; i < rows * L; i += static_cast<int32_t>(gridDim.y) * kThreads) {
        const int32_t o = i / L, w = i % L * 4;
        const float *p = part_at<D, M>(a, id) + o * D + w;
        f4 s1{0.0f, 0.0f, 0.0f, 0.0f}, s2 = s1;
#pragma unroll 4
        for (int e = 0; e < it.parts; ++e) {  // the parts of an item are kv_heads pieces apart
            s1 += *reinterpret_cast<const f4 *>(p);
            if (KEYS) s2 += *reinterpret_cast<const f4 *>(p + kOwn * D);
            p += static_cast<int64_t>(a.kv_heads) * M * kOwn * D;
        }
        auto put = [&](const uint16_t *at, f4 v) {
            *reinterpret_cast<u2 *>(const_cast<uint16_t *>(at) + w) = u2{T::pack(v[0], v[1]), T::pack(v[2], v[3])};
        };
        s1 *= a.scale;
        if constexpr (KEYS) {
            const int32_t row = it.run.first + own0 + o;
            if (a.dk.p) put(a.dk.p + it.kv * a.dk.head + row * a.dk.row, s1);
            if (a.dv.p) put(a.dv.p + it.kv * a.dv.head + row * a.dv.row, s2);
        } else {
            put(a.dq.p + row_at(a, a.dq, it.run.first, it.kv, own0 + o), s1);
        }
    }
}
// The parts of dq (pieces below by_rows), then those of dk and dv.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void packed_reduce_kernel(Args a, int32_t by_rows) {
    const int32_t id = static_cast<int32_t>(blockIdx.x);
    if (id < by_rows) add_parts<T, D, false>(a, id);
    else add_parts<T, D, true>(a, id - by_rows);
}

// ------------------------------------------------------------------------------------------ launch

// A grid counts its threads in 32 bits (and wraps around without an error).
constexpr int64_t kMostBlocks = (int64_t(1) << 24) - 1;

// Which items are cut: batches of up to 64 sequences, whose longest might have more than the least levels of a part, of
// kLeastSteps streamed tiles.  A part's sums (64 or 128 KB at width 128) are worth that many.
constexpr int64_t kLeastSteps = 16;
struct Plan {
    int32_t resident, least;  // as in Pieces
    int64_t cut;              // pieces of cut items, at most
    int64_t places;           // of the table: a source head's pieces, at most
};
Plan plan_for(const tiga_packed &rel, bool keys) {
    const int64_t group = rel.heads / rel.kv_heads, bn = rel.width == 64 ? 128 : 64;
    Plan p;
    p.resident = device_cus() * (keys && rel.width == 128 ? 1 : 2);
    const int64_t least = ceil_div(kLeastSteps * bn * (keys ? 1 : group), kOwn * (keys ? group : 1));
    const int64_t most = ceil_div(rel.num_rows * (keys ? 1 : group), kOwn);
    const bool some = rel.batch <= kWave && most > least;
    p.least = some ? static_cast<int32_t>(least) : kNoCut;
    p.cut = some ? 2 * static_cast<int64_t>(p.resident) : 0;
    p.places = most_items(rel, keys ? 1 : group) / rel.kv_heads + ceil_div(p.cut, rel.kv_heads);
    if (p.places < 1) p.places = 1;  // no sequences: all rows are cleared
    return p;
}

struct Layout {
    Plan rows, keys;
    int4 *rows_table, *keys_table;
    float *lse2, *delta, *rows_part, *keys_part;
    f2 *peak;
    int64_t slots;
    size_t bytes;
};
Layout layout(const tiga_packed &rel, void *ws) {
    Layout l;
    l.rows = plan_for(rel, false);
    l.keys = plan_for(rel, true);
    Carve c(ws);
    const size_t stats = static_cast<size_t>(rel.heads) * rel.num_rows + 1;
    l.lse2 = c.take<float>(stats);
    l.delta = c.take<float>(stats);
    l.slots = rel.num_rows / kOwn + rel.batch + 1;
    l.peak = c.take<f2>(l.slots * rel.kv_heads);
    // for any number of heads, and whether this call's items are cut or not: a workspace holds every smaller call
    const size_t cus = device_cus(), some = rel.num_rows > kOwn ? 1 : 0;
    const size_t places = static_cast<size_t>(rel.num_rows) / kOwn + rel.batch + 4 * cus + 1;
    l.rows_table = c.take<int4>(2 * (places + static_cast<size_t>(rel.num_rows) * rel.heads / kOwn));
    l.keys_table = c.take<int4>(2 * places);
    l.rows_part = c.take<float>(some * (4 * cus + rel.heads) * kOwn * rel.width);
    l.keys_part = c.take<float>(some * ((rel.width == 128 ? 2 : 4) * cus + rel.heads) * 2 * kOwn * rel.width);
    l.bytes = c.bytes();
    return l;
}

template <class T, int D>
int launch(const Layout &l, const tiga_packed &rel, const Args &a, hipStream_t stream) {
    const bool keys = a.dk.p || a.dv.p;
    const Pieces by_rows{l.rows_table, static_cast<int32_t>(l.rows.places), static_cast<int32_t>(a.group.d), l.rows.resident, l.rows.least, 2};
    const Pieces by_keys{l.keys_table, static_cast<int32_t>(l.keys.places), 1, l.keys.resident, l.keys.least, 2};
    if (int rc = plan_pieces(rel, by_rows, by_keys, 2, stream)) return rc;
    const dim3 row_blocks(static_cast<unsigned>(l.rows.places * rel.kv_heads)), key_blocks(static_cast<unsigned>(l.keys.places * rel.kv_heads));
    if constexpr (kScaled<T>) {
        hipLaunchKernelGGL((packed_peak_kernel<T, D>), key_blocks, dim3(kThreads), 0, stream, a);
        if (int rc = check_launch("packed attention backward peaks")) return rc;
    }
    if (!keys) prof_before(stream);
    hipLaunchKernelGGL((packed_query_kernel<T, D>), row_blocks, dim3(kThreads), 0, stream, a);
    if (!keys) prof_after(stream);
    if (int rc = check_launch("packed attention backward, dq")) return rc;
    if (keys) {
        prof_before(stream);
        hipLaunchKernelGGL((packed_keys_kernel<T, D>), key_blocks, dim3(kThreads), 0, stream, a);
        prof_after(stream);
        if (int rc = check_launch("packed attention backward, dk and dv")) return rc;
    }
    // whole places, so that parts of every head are seen
    const int64_t row_parts = a.dq.p && l.rows.cut ? ceil_div(l.rows.cut, rel.kv_heads) * rel.kv_heads : 0;
    const int64_t key_parts = keys && l.keys.cut ? ceil_div(l.keys.cut, rel.kv_heads) * rel.kv_heads : 0;
    if (row_parts + key_parts == 0) return TIGA_OK;
    hipLaunchKernelGGL((packed_reduce_kernel<T, D>), dim3(static_cast<unsigned>(row_parts + key_parts), 4), dim3(kThreads), 0, stream, a,
                       static_cast<int32_t>(row_parts));
    return check_launch("packed attention backward sums");
}

}  // namespace

size_t packed_bwd_ws_bytes(const tiga_packed &rel) { return rel.kv_heads == 0 ? 256 : layout(rel, nullptr).bytes; }

int packed_backward(const tiga_packed &rel, const tiga_view &q, const tiga_view &k, const tiga_view &v, const tiga_view &y,
                    const float *lse, const tiga_view &dy, float scale, const tiga_view &dq, const tiga_view &dk,
                    const tiga_view &dv, void *ws, hipStream_t stream) {
    const int32_t group = rel.heads / rel.kv_heads;
    const Layout l = layout(rel, ws);
    if (l.rows.places * rel.kv_heads > kMostBlocks || l.keys.places * rel.kv_heads > kMostBlocks)
        return fail(TIGA_EUNSUPPORTED, "packed attention backward: at most 2^24 - 1 tiles of 128 rows or sources");
    Args a{};
    a.q = rows_of(q);
    a.k = rows_of(k);
    a.v = rows_of(v);
    a.y = rows_of(y);
    a.dy = rows_of(dy);
    a.dq = rows_of(dq);
    a.dk = rows_of(dk);
    a.dv = rows_of(dv);
    a.lse = lse;
    a.ptr = rel.ptr;
    a.lse2 = l.lse2;
    a.delta = l.delta;
    a.peak = l.peak;
    a.rows_table = l.rows_table;
    a.keys_table = l.keys_table;
    a.rows_part = l.rows_part;
    a.keys_part = l.keys_part;
    a.slots = static_cast<int32_t>(l.slots);
    a.num_rows = static_cast<int32_t>(rel.num_rows);
    a.batch = rel.batch;
    a.kv_heads = rel.kv_heads;
    a.group = divider(group);
    a.stats = static_cast<int64_t>(rel.heads) * rel.num_rows;
    a.scale = scale;
    if (rel.dtype == TIGA_DT_F16) return rel.width == 64 ? launch<Half16, 64>(l, rel, a, stream) : launch<Half16, 128>(l, rel, a, stream);
    return rel.width == 64 ? launch<Brain16, 64>(l, rel, a, stream) : launch<Brain16, 128>(l, rel, a, stream);
}

}  // namespace relattn
}  // namespace tiga
