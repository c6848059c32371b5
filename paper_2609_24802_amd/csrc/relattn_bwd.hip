// Vector-Jacobian product of cross attention.  With p_ij = exp(s_ij - lse_i), delta_i = <dy_i, y_i> and
// ds_ij = p_ij (<dy_i, v_j> - delta_i):
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i,   dv_j = sum_i p_ij dy_i,
// i over the destinations of every head that shares source head j's.  Scores and weights are formed again from q, k and
// lse; nothing of the size of the relation is stored.
//
// Two launches of one kernel: dq with the rows owned and the keys streamed, which also leaves the rows' statistics (lse in
// the log2 domain, delta; these alone where dq is not wanted), then dk, dv with the keys owned and the rows streamed.  A
// wavefront owns 32 columns, whose operands X1 (q or k) and X2 (dy or v) stay in registers, and streams tiles of Y1 (k or
// q) and Y2 (v or dy) through LDS.  Per 32 streamed rows
//   S = Y1 X1^T, DP = Y2 X2^T   (streamed x owned, 16x16x32 MFMA, fp32)
//   P = 2^(c S - lse2), DS = P (DP - delta), rounded to the input type as the operands of the next products (binary16:
//   scaled into its range first)
//   acc1 += Y1^T DS (dq or dk),  acc2 += Y2^T P (dv)
// where the accumulator layout of S is the operand layout of P (each lane's rows of two 16-row blocks fill its 8 slots of
// a 32-deep product, and the transposing LDS reads of Y^T take the rows in that order).  dk and dv need S and DP once
// more than a fused pass would, 14 instead of 10 operations a pair and width; the fused pass would have to add dq over
// blocks of keys, by atomics (an order that varies) or through fp32 partial sums of S / 128 times dq's size.
//
// delta is taken from the forward's y, whose rounding (of itself and of the weights in it) makes an error of u |dy| |y|.
// Over many sources that is small against ds; over a few it is not (twice the error of dq and dk at 2 to 5 sources),
// so where a sequence's sources fit one streamed tile, delta is formed as sum_j p_ij <dy_i, v_j> in fp32 instead, by the
// products S and DP of that tile, in one launch with dq, which takes the same products (and comes first then).  That goes
// by the sequence's own sources: its gradients do not depend on what else is in the batch.
//
// Measured (MI355X; ranges are of several runs, the first of calls repeated while hot), 2 x 16 x 2048 rows, 4 source heads of
// 8192 keys, width 128, bf16: dk and dv 487 to 574 us (0.96 to 1.13 PFLOP/s), dq 318 to 356 (1.16 to 1.30), 818 to 930
// together; binary16 884, with 8 for its range; 4 x 16 x 4096 x 4096 x 64 f16: 512 to 527 us (1.04 to 1.07) and 377 to 389
// (1.06 to 1.09), 15 for the range; 4 x 8 x 4096 rows over 77 of 64: delta and dq 21 to 22 us (apart 15 and 19), dk and dv 17
// and their sums 5.  A large library product reaches 1.2 to 1.4.  Bound by the matrix cores at the clock the load leaves and by
// LDS reads: each operand read feeds two products, 128 bytes a cycle and compute unit at full matrix rate, which is all that
// LDS delivers.
//
// Every sum has a fixed order.  Where the owned tiles do not fill the device, the streamed axis is split, and the parts'
// fp32 sums go to the workspace and are added by reduce_kernel.
#include <type_traits>

#include "mfma16.hpp"
#include "relation.hpp"
#include "relattn.hpp"

namespace tiga {
namespace relattn {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kOwn = 128;  // owned rows or keys of a block: 32 a wavefront
constexpr float kLog2e = 1.4426950408889634f;

struct Args {
    Rows q, k, v, y, dy, dq, dk, dv;
    const float *lse;
    const int32_t *len;
    float *lse2, *delta;  // [batch * heads * num_dst + 1]: the last is what rows past the end have (no weight)
    float *part;          // split sums
    f2 *peak;             // [batch * kv_heads][peaks]: of a share of a source head's values and cotangents (binary16)
    int32_t peaks;
    int32_t num_dst, num_src, batch, heads, kv_heads;
    Divider group;
    int64_t stats;        // batch * heads * num_dst
    int32_t rows;         // num_dst * group
    int32_t splits;
    float scale;
};

__device__ __forceinline__ int32_t sources(const Args &a, int b) {
    if (!a.len) return a.num_src;
    const int32_t n = a.len[b];
    return n < 0 ? 0 : (n > a.num_src ? a.num_src : n);
}
// Row r of a source head is token r / group of head r % group of its group.
__device__ __forceinline__ int64_t row_at(const Args &a, const Rows &t, int b, int kv, int32_t r) {
    const int32_t token = a.group.div(r), g = r - token * static_cast<int32_t>(a.group.d);
    // row and head strides are below 2^31
    return b * t.batch + static_cast<int64_t>(kv * static_cast<int32_t>(a.group.d) + g) * static_cast<int32_t>(t.head) +
           static_cast<int64_t>(token) * static_cast<int32_t>(t.row);
}
__device__ __forceinline__ int64_t stat_at(const Args &a, int b, int kv, int32_t r) {
    const int32_t token = a.group.div(r), g = r - token * static_cast<int32_t>(a.group.d);
    return (static_cast<int64_t>(b) * a.heads + kv * static_cast<int32_t>(a.group.d) + g) * a.num_dst + token;
}

// ------------------------------------------------------------------------------------------ statistics

// A row that saw no weight has no gradient: its weights are formed as 0.
__device__ __forceinline__ float log2_of(float lse) { return lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2e; }

// <dy, y> of a row, lane g of its four: 16-byte chunks g, g + 4, ...; the four lanes' sums are added g ^ 1 first, then g ^ 2.
template <class T, int CH>
__device__ __forceinline__ float row_product(const u4 (&dy)[CH], const uint16_t *y, int g) {
    float s = 0.0f;
#pragma unroll
    for (int ch = 0; ch < CH; ++ch) {
        const u4 x = reinterpret_cast<const u4 *>(y)[ch * 4 + g];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const f2 u = T::unpack(x[e]), v = T::unpack(dy[ch][e]);
            s = __builtin_fmaf(u.y, v.y, __builtin_fmaf(u.x, v.x, s));
        }
    }
    return s;
}

// ------------------------------------------------------------------------------------------ range of binary16

// P and DS enter the products in the input type.  P is of order 1 / S and DS of that times the cotangents, and binary16 has
// no normal numbers below 2^-14, so there they are scaled by powers of two, which the fp32 sums are rid of again:
//  - P by 2^kUp: at most 1 (and what lse's rounding adds), so it stays below 2^16;
//  - DS by 2^up(M), M >= |<dy_i, v_j>|, and so |DS| <= 2 M: below 2^15.  M = |dy_i|_1 max |v| of the row for dq, whose sums
//    are the row's own, and of the source head's largest row for dk, whose sums run over its rows.
// What is then rounded to a multiple of 2^-24 is 2^-38 of those bounds.  (Unscaled, over 8192 sources at cotangents of
// 1e-3: dq and dk 1.1e-2 off, at 1e-4 0.1.)  bfloat16 has the range of fp32.
template <class T>
constexpr bool kScaled = std::is_same<T, Half16>::value;
constexpr int kUp = 14;
// M < 2^(its binary exponent).  0, infinities and NaN, where any factor does, have exponent 0.
__device__ __forceinline__ int up(float m) { return kUp - __builtin_amdgcn_frexp_expf(m); }
__device__ __forceinline__ float two_to(int e) { return __builtin_amdgcn_ldexpf(1.0f, e); }

template <class T>
__device__ __forceinline__ float sum_abs(u4 x) {
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const f2 u = T::unpack(x[e]);
        s += __builtin_fabsf(u.x) + __builtin_fabsf(u.y);
    }
    return s;
}

// max |v| and max |dy|_1 of a share of a source head's sources and rows; what is not a number is passed over (its results
// are none either).  Bound by reading v and dy once: 2 x 16 x 2048 rows and 4 x 8192 sources of 128, 34 MB in 8 us, of 884;
// 8 x 449 ragged rows over 1500 of 64, 23 MB in 8 us, of 95.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void peak_kernel(Args a) {
    constexpr int L = D / 8, ROWS = kThreads / L;  // 16 bytes a lane
    __shared__ f2 of_wave[kWaves];
    const int64_t bh = blockIdx.x / a.peaks;
    const int part = static_cast<int>(blockIdx.x - bh * a.peaks);
    const int b = static_cast<int>(bh / a.kv_heads), kv = static_cast<int>(bh % a.kv_heads);
    const int first = static_cast<int>(threadIdx.x) / L, c = static_cast<int>(threadIdx.x) % L;
    auto from = [&](int64_t n, int i) { return static_cast<int32_t>(n * i / a.peaks); };
    f2 top{0.0f, 0.0f};
    const int32_t n = sources(a, b);
    const u4 *const v = reinterpret_cast<const u4 *>(a.v.p + b * a.v.batch + kv * a.v.head) + c;
    const int32_t v1 = from(n, part + 1);
#pragma unroll 4
    for (int32_t j = from(n, part) + first; j < v1; j += ROWS) {
        const u4 x = v[j * (a.v.row / 8)];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const f2 u = T::unpack(x[e]);
            top.x = fmaxf(top.x, fmaxf(__builtin_fabsf(u.x), __builtin_fabsf(u.y)));
        }
    }
    const int32_t r1 = from(a.rows, part + 1);
#pragma unroll 4
    for (int32_t r = from(a.rows, part) + first; r < r1; r += ROWS) {
        float l1 = sum_abs<T>(reinterpret_cast<const u4 *>(a.dy.p + row_at(a, a.dy, b, kv, r))[c]);
#pragma unroll
        for (int d = 1; d < L; d <<= 1) l1 += shfl_xor_f(l1, d);  // whole rows: the lanes of a row leave together
        top.y = fmaxf(top.y, l1);
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        top.x = fmaxf(top.x, shfl_xor_f(top.x, d));
        top.y = fmaxf(top.y, shfl_xor_f(top.y, d));
    }
    if (lane_id() == 0) of_wave[threadIdx.x / kWave] = top;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < kWaves; ++w) top = f2{fmaxf(top.x, of_wave[w].x), fmaxf(top.y, of_wave[w].y)};
    a.peak[blockIdx.x] = top;
}
// Of the whole source head.
__device__ __forceinline__ f2 peak_of(const Args &a, int64_t bh) {
    f2 top{0.0f, 0.0f};
    for (int i = lane_id(); i < a.peaks; i += kWave) {
        const f2 x = a.peak[bh * a.peaks + i];
        top = f2{fmaxf(top.x, x.x), fmaxf(top.y, x.y)};
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        top.x = fmaxf(top.x, shfl_xor_f(top.x, d));
        top.y = fmaxf(top.y, shfl_xor_f(top.y, d));
    }
    return f2{__uint_as_float(uniform(__float_as_uint(top.x))), __uint_as_float(uniform(__float_as_uint(top.y)))};
}

// ------------------------------------------------------------------------------------------ products

template <int D>
struct Geo {
    static constexpr int CPR = D / 8;                 // 16-byte chunks per row
    static constexpr int RB = 2 * D;                  // bytes per row
    static constexpr int R = 256 / RB;                // rows per 256-byte bank window
    static constexpr int CH = D / 32;                 // 32-deep chunks of S and DP
    static constexpr int DB = D / 16;                 // 16-wide blocks of the sums
    static constexpr int BN = D == 64 ? 128 : 64;     // streamed rows a tile
    static constexpr int KC = BN / 32;                // 32-row chunks of a tile
    static constexpr int TILE = BN * RB;              // 16 KB
    static constexpr int LPW = TILE / 1024 / kWaves;  // 1-KB direct loads per wavefront, tile and operand
};

// LDS layout of a streamed tile: 16-byte chunk c of key row k sits at chunk c ^ swizzle(k), for both kinds of reads:
//  - a transposing read takes 8 neighbouring rows at one 32-byte block, so the swizzle's upper bits differ in rows 0..7 and
//    in rows 8..15 of 16;
//  - a direct read takes 16 rows at chunk g of the four lane groups, and serves rows 0..3 and 12..15 of one group together
//    with rows 4..11 of the next (chunk g ^ 1), so rows 4..11 (and the others) hold both values of every pair 2 i, 2 i + 1.
// (Without the second rule, 1.5 cycles of conflict a read.)
template <int D>
__device__ __forceinline__ int swizzle(int k) {
    constexpr int CPR = Geo<D>::CPR, H = CPR / 2;
    const int y = (k / Geo<D>::R) % CPR, upper = y / H;
    return (((y % H) ^ (upper * (H / 2))) << 1) | upper;
}

// Blocks a compute unit: dk and dv at width 128 take 512 registers a lane (128 of sums, 64 of owned operands).
template <int D, bool KEYS>
constexpr int kBlocks = KEYS && D == 128 ? 1 : 2;

// What the products are formed for: dq (rows owned), dk and dv (keys owned), or delta and dq where no sequence has more than
// one tile of keys (as kQuery would, in half the LDS).
enum Mode { kQuery, kKeys, kFew };

template <class T, int D, Mode MODE>
struct Sums {
    f4 a1[Geo<D>::DB][2];
    f4 a2[MODE == kKeys ? Geo<D>::DB : 1][2];
};

// The 32 streamed rows at `y1`, `y2` (their first row's LDS address) against the owned columns: S and DP as
// [16-row block][column block].  dr: this lane's offset of the direct reads, which run kAhead ahead of their products.
// between(i) is what the vector unit does under the products of read i.
template <class T, int D>
struct Scores {
    static constexpr int kReads = 4 * Geo<D>::CH;
    f4 s[2][2], dp[2][2];
    template <class Between>
    __device__ __forceinline__ void form(const u4 (&x1)[2][Geo<D>::CH], const u4 (&x2)[2][Geo<D>::CH], const uint8_t *y1,
                                         const uint8_t *y2, int dr, Between between) {
        constexpr int kAhead = 4;
        auto read = [&](int i) {
            const uint8_t *const p = (i / 2) % 2 ? y2 : y1;
            return *reinterpret_cast<const u4 *>(p + (dr ^ (64 * (i / 4))) + i % 2 * 16 * Geo<D>::RB);
        };
        u4 w[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) w[i] = read(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            const int ch = i / 4, e = i % 2;
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) {
                if ((i / 2) % 2 == 0)
                    s[e][qb] = T::mma(w[i % kAhead], x1[qb][ch], ch == 0 ? f4{0.0f, 0.0f, 0.0f, 0.0f} : s[e][qb]);
                else
                    dp[e][qb] = T::mma(w[i % kAhead], x2[qb][ch], ch == 0 ? f4{0.0f, 0.0f, 0.0f, 0.0f} : dp[e][qb]);
            }
            if (i + kAhead < kReads) w[i % kAhead] = read(i + kAhead);
            between(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// acc1 += Y1^T DS, acc2 += Y2^T P (dk, dv only) of 32 streamed rows.  tr: this lane's offset of the transposing reads.
template <class T, int D, Mode MODE>
constexpr int kSumReads = (MODE == kKeys ? 2 : 1) * Geo<D>::DB;
template <class T, int D, Mode MODE, class Between>
__device__ __forceinline__ void add_products(Sums<T, D, MODE> &acc, const u4 (&pb)[2], const u4 (&db)[2], const uint8_t *y1,
                                             const uint8_t *y2, int tr, Between between) {
    constexpr bool KEYS = MODE == kKeys;
    constexpr int M = KEYS ? 2 : 1, kReads = kSumReads<T, D, MODE>, kAhead = 3;
    auto read = [&](int i) {
        const uint8_t *const p = (KEYS && i % 2 ? y2 : y1) + (tr ^ (32 * (i / M)));
        const u2 lo = lds_transposed16(p), hi = lds_transposed16(p + 16 * Geo<D>::RB);
        return u4{lo.x, lo.y, hi.x, hi.y};
    };
    u4 w[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) w[i] = read(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kReads; ++i) {
        const int d = i / M;
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            if (KEYS && i % 2) acc.a2[KEYS ? d : 0][qb] = T::mma(w[i % kAhead], pb[qb], acc.a2[KEYS ? d : 0][qb]);
            else acc.a1[d][qb] = T::mma(w[i % kAhead], db[qb], acc.a1[d][qb]);
        }
        if (i + kAhead < kReads) w[i % kAhead] = read(i + kAhead);
        between(i);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// P of 32 streamed keys in the place of their scores; `left` keys exist where `edge` is set.
template <class T, int D>
__device__ __forceinline__ void weigh(Scores<T, D> &f, float c, const float *lse2, bool edge, int left, int g) {
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) f.s[e][qb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(f.s[e][qb][i], c, -lse2[qb]));
        if (edge) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float p = e * 16 + 4 * g + i < left ? f.s[e][qb][i] : 0.0f;
                    __asm__ volatile("" : "+v"(p));  // a branch: selects in every tile take a tenth of the time
                    f.s[e][qb][i] = p;
                }
        }
    }
}
// dq += K^T DS of 32 streamed keys with weights f.s.
template <class T, int D, Mode MODE>
__device__ __forceinline__ void add_keys(Sums<T, D, MODE> &acc, const Scores<T, D> &f, const float *delta, const uint8_t *y1,
                                         int tr) {
    u4 db[2];
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        float ds[2][4];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) ds[e][i] = f.s[e][qb][i] * (f.dp[e][qb][i] - delta[qb]);
        db[qb] = u4{T::pack(ds[0][0], ds[0][1]), T::pack(ds[0][2], ds[0][3]), T::pack(ds[1][0], ds[1][1]),
                    T::pack(ds[1][2], ds[1][3])};
    }
    add_products<T, D, MODE>(acc, db, db, y1, y1, tr, [](int) {});
}

// Weights P and DS of 32 streamed rows, whose statistics lie at st, sd in LDS, one of 16 elements a lane at a time.  In
// binary16 the statistics are of scaled ones, and h is the factor from DP to the statistics' delta.
template <class T, int D>
struct Weights {
    f4 lse2[2], delta[2];
    float p[16], ds[16];
    uint32_t pw[8], dw[8];
    __device__ __forceinline__ void load(const float *st, const float *sd, int g) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            lse2[e] = *reinterpret_cast<const f4 *>(st + e * 16 + 4 * g);
            delta[e] = *reinterpret_cast<const f4 *>(sd + e * 16 + 4 * g);
        }
    }
    __device__ __forceinline__ void form(const Scores<T, D> &f, float c, float h, int n) {
        const int qb = n / 8, e = n / 4 % 2, i = n % 4;
        p[n] = __builtin_amdgcn_exp2f(__builtin_fmaf(f.s[e][qb][i], c, -lse2[e][i]));
        ds[n] = p[n] * (kScaled<T> ? __builtin_fmaf(f.dp[e][qb][i], h, -delta[e][i]) : f.dp[e][qb][i] - delta[e][i]);
        if (n % 2) {
            pw[n / 2] = T::pack(p[n - 1], p[n]);
            dw[n / 2] = T::pack(ds[n - 1], ds[n]);
        }
    }
};

// dk and dv, 64 streamed rows as two halves.  The first half's weights are formed under the products for the second's
// scores, the second's under the first half's sums: at width 128 a SIMD has one wavefront, and nothing else fills its
// matrix unit meanwhile (527 us without, 494).  At width 64 two wavefronts share a SIMD: 8 x 449 rows over 1500 ragged 54.8
// and 52.7 us, 4 x 4096 over 77 23.4 and 21.0, 4 x 4096 over 4096 507 and 525.
template <class T, int D>
__device__ __forceinline__ void rows_step(Sums<T, D, kKeys> &acc, const u4 (&x1)[2][Geo<D>::CH],
                                          const u4 (&x2)[2][Geo<D>::CH], const uint8_t *y1, const uint8_t *y2, int dr,
                                          int tr, float c, float h, const float *st, const float *sd, int g) {
    constexpr int kHalf = 32 * Geo<D>::RB, kScore = 16 / Scores<T, D>::kReads, kSum = 16 / kSumReads<T, D, kKeys>;
    Scores<T, D> f0, f1;
    Weights<T, D> w0, w1;
    w0.load(st, sd, g);
    f0.form(x1, x2, y1, y2, dr, [](int) {});
    f1.form(x1, x2, y1 + kHalf, y2 + kHalf, dr, [&](int i) {
#pragma unroll
        for (int n = 0; n < kScore; ++n) w0.form(f0, c, h, i * kScore + n);
    });
    w1.load(st + 32, sd + 32, g);
    auto operand = [](const uint32_t *x, int qb) { return u4{x[4 * qb], x[4 * qb + 1], x[4 * qb + 2], x[4 * qb + 3]}; };
    const u4 p0[2] = {operand(w0.pw, 0), operand(w0.pw, 1)}, d0[2] = {operand(w0.dw, 0), operand(w0.dw, 1)};
    add_products<T, D, kKeys>(acc, p0, d0, y1, y2, tr, [&](int i) {
#pragma unroll
        for (int n = 0; n < kSum; ++n) w1.form(f1, c, h, i * kSum + n);
    });
    const u4 p1[2] = {operand(w1.pw, 0), operand(w1.pw, 1)}, d1[2] = {operand(w1.dw, 0), operand(w1.dw, 1)};
    add_products<T, D, kKeys>(acc, p1, d1, y1 + kHalf, y2 + kHalf, tr, [](int) {});
}

// kKeys: a block owns 128 keys of a source head and streams its rows; otherwise it owns 128 rows and streams the keys.
// A block's pieces: (eight heads, tile, split, head), so that an XCD (every eighth block) keeps to
// one head of the eight and unequal sequences spread over the XCDs.
template <class T, int D, Mode MODE>
__global__ __launch_bounds__(kThreads, (kBlocks<D, MODE == kKeys>)) void products_kernel(Args a, int tiles) {
    using G = Geo<D>;
    constexpr bool KEYS = MODE == kKeys;
    __shared__ __attribute__((aligned(1024))) uint8_t y1a[G::TILE], y2a[G::TILE], y1b[G::TILE], y2b[G::TILE];
    __shared__ __attribute__((aligned(256))) float sta[KEYS ? 2 * G::BN : 2], stb[KEYS ? 2 * G::BN : 2];
    const int lane = lane_id(), w = uniform(static_cast<int>(threadIdx.x) / kWave);
    const int col = lane & 15, g = lane >> 4;

    const int64_t heads = static_cast<int64_t>(a.batch) * a.kv_heads, per = static_cast<int64_t>(tiles) * a.splits;
    const int64_t band = blockIdx.x / (kXcds * per);
    const int64_t in = blockIdx.x - band * kXcds * per;
    const int width = static_cast<int>(min(heads - band * kXcds, static_cast<int64_t>(kXcds)));
    const int64_t bh = band * kXcds + in % width;
    const int ts = static_cast<int>(in / width), tile = ts / a.splits, split = ts % a.splits;
    const int b = static_cast<int>(bh / a.kv_heads), kv = static_cast<int>(bh % a.kv_heads);

    const int32_t n = sources(a, b);
    const int32_t own_n = KEYS ? n : a.rows, str_n = KEYS ? a.rows : n;
    const int32_t own0 = tile * kOwn;
    if (own0 >= own_n && a.splits > 1) return;  // no part of it is read
    const int32_t steps = own0 < own_n ? (str_n + G::BN - 1) / G::BN : 0;
    const int32_t t0 = static_cast<int32_t>(static_cast<int64_t>(steps) * split / a.splits);
    const int32_t t1 = static_cast<int32_t>(static_cast<int64_t>(steps) * (split + 1) / a.splits);

    // the sequence's sources fit one tile: delta comes from the tile's products
    const bool few = MODE == kFew || (MODE == kQuery && n <= G::BN);

    // owned operands; columns past the end repeat the last (what they sum is not stored)
    u4 x1[2][G::CH], x2[2][G::CH];
    f2 peak{0.0f, 0.0f};
    if constexpr (kScaled<T>) peak = peak_of(a, bh);
    const int keys_up = kScaled<T> ? up(peak.x * peak.y) : 0;               // the exponent of DS in dk
    const float h = kScaled<T> ? two_to(keys_up - kUp) : 1.0f;              // P has kUp of it
    float own[2], own_delta[2];
    int own_up[2] = {0, 0};  // the exponent of DS
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        const int32_t o = min(own0 + w * 32 + qb * 16 + col, own_n - 1);
        own[qb] = own_delta[qb] = 0.0f;
        if (own_n > 0 && own0 < own_n) {
            const uint16_t *p1, *p2;
            if constexpr (KEYS) {
                p1 = a.k.p + b * a.k.batch + kv * a.k.head + o * a.k.row;
                p2 = a.v.p + b * a.v.batch + kv * a.v.head + o * a.v.row;
            } else {
                p1 = a.q.p + row_at(a, a.q, b, kv, o);
                p2 = a.dy.p + row_at(a, a.dy, b, kv, o);
                own[qb] = log2_of(a.lse[stat_at(a, b, kv, o)]);
            }
#pragma unroll
            for (int ch = 0; ch < G::CH; ++ch) {
                x1[qb][ch] = reinterpret_cast<const u4 *>(p1)[ch * 4 + g];
                x2[qb][ch] = reinterpret_cast<const u4 *>(p2)[ch * 4 + g];
            }
            if (!KEYS && kScaled<T>) {
                float l1 = 0.0f;
#pragma unroll
                for (int ch = 0; ch < G::CH; ++ch) l1 += sum_abs<T>(x2[qb][ch]);
                own_up[qb] = up(column_sum(l1) * peak.x);
                own[qb] -= static_cast<float>(own_up[qb]);
            }
            if (MODE == kQuery && !few)
                own_delta[qb] = column_sum(row_product<T>(x2[qb], a.y.p + row_at(a, a.y, b, kv, o), g));
        }
    }
    if (!KEYS && blockIdx.x == 0 && threadIdx.x == 0) {  // what rows past the end have
        a.lse2[a.stats] = __builtin_inff();
        a.delta[a.stats] = 0.0f;
    }
    // The owned rows' statistics, for dk and dv: delta is there.
    auto leave_stats = [&] {
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            const int32_t o = own0 + w * 32 + qb * 16 + col;
            if (o < own_n && g == 0) {
                const int64_t at = stat_at(a, b, kv, o);
                a.lse2[at] = kScaled<T> ? log2_of(a.lse[at]) - kUp : own[qb];
                a.delta[at] = own_delta[qb] * h;
            }
        }
    };
    if (MODE == kQuery && !few) {
        if (split == 0) leave_stats();
        if (!a.dq.p) return;
    }
    Sums<T, D, MODE> acc;
#pragma unroll
    for (int d = 0; d < G::DB; ++d)
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            acc.a1[d][qb] = f4{0.0f, 0.0f, 0.0f, 0.0f};
            if (KEYS) acc.a2[KEYS ? d : 0][qb] = f4{0.0f, 0.0f, 0.0f, 0.0f};
        }

    // this lane's places in a tile: rows and chunks of its direct loads, offsets of its operand reads
    int krow[G::LPW], kch[G::LPW];
#pragma unroll
    for (int r = 0; r < G::LPW; ++r) {
        const int byte = (w * G::LPW + r) * 1024 + 16 * lane;
        krow[r] = byte / G::RB;
        kch[r] = byte % G::RB / 16 ^ swizzle<D>(krow[r]);
    }
    const int dr = col * G::RB + 16 * (g ^ swizzle<D>(col));
    const int trow = 4 * g + col / 4;
    const int tr = trow * G::RB + 16 * ((col % 4 / 2) ^ swizzle<D>(trow)) + 8 * (col % 2);

    const uint16_t *const kb = a.k.p + b * a.k.batch + kv * a.k.head, *const vb = a.v.p + b * a.v.batch + kv * a.v.head;
    auto stage = [&](int kt, uint8_t *b1, uint8_t *b2, float *stats) {
        const int32_t k0 = kt * G::BN;
        const uint8_t *const kt0 = reinterpret_cast<const uint8_t *>(kb + k0 * a.k.row);
        const uint8_t *const vt0 = reinterpret_cast<const uint8_t *>(vb + k0 * a.v.row);
#pragma unroll
        for (int r = 0; r < G::LPW; ++r) {
            const int run = (w * G::LPW + r) * 1024;
            const int32_t i = min(k0 + krow[r], str_n - 1);  // past the end: the last row again, without weight
            const uint8_t *p1, *p2;
            if constexpr (KEYS) {
                p1 = reinterpret_cast<const uint8_t *>(a.q.p + row_at(a, a.q, b, kv, i) + 8 * kch[r]);
                p2 = reinterpret_cast<const uint8_t *>(a.dy.p + row_at(a, a.dy, b, kv, i) + 8 * kch[r]);
            } else {
                // a uniform base and 32-bit offsets in bytes (row strides are below 2^23): 64-bit ones a lane spill
                p1 = kt0 + (2u * static_cast<uint32_t>(i - k0) * static_cast<uint32_t>(a.k.row) + 16u * kch[r]);
                p2 = vt0 + (2u * static_cast<uint32_t>(i - k0) * static_cast<uint32_t>(a.v.row) + 16u * kch[r]);
            }
            load_to_lds16(p1, b1 + run);
            load_to_lds16(p2, b2 + run);
        }
        if constexpr (KEYS) {
            // 64 lanes, 4 bytes each: the first half of the needed wavefronts takes lse2, the other delta
            constexpr int kNeed = 2 * G::BN / kWave;
            if (w < kNeed) {
                const int32_t i = k0 + w % (kNeed / 2) * kWave + lane;
                const int64_t at = i < str_n ? stat_at(a, b, kv, i) : a.stats;
                __builtin_amdgcn_global_load_lds((w < kNeed / 2 ? a.lse2 : a.delta) + at,
                                                 (__attribute__((address_space(3))) void *)(stats + w * kWave), 4, 0, 0);
            }
        }
    };
    const float c = a.scale * kLog2e;
    auto step = [&](int kt, const uint8_t *b1, const uint8_t *b2, const float *stats) {
        const bool edge = (kt + 1) * G::BN > str_n;
        if constexpr (KEYS) {
#pragma unroll
            for (int kc = 0; kc < G::KC; kc += 2)
                rows_step<T, D>(acc, x1, x2, b1 + kc * 32 * G::RB, b2 + kc * 32 * G::RB, dr, tr, c, h, stats + kc * 32,
                                stats + G::BN + kc * 32, g);
        } else {
#pragma unroll
            for (int kc = 0; kc < G::KC; ++kc) {
                Scores<T, D> f;
                f.form(x1, x2, b1 + kc * 32 * G::RB, b2 + kc * 32 * G::RB, dr, [](int) {});
                weigh<T, D>(f, c, own, edge, str_n - kt * G::BN - kc * 32, g);
                add_keys<T, D, MODE>(acc, f, own_delta, b1 + kc * 32 * G::RB, tr);
            }
        }
    };
    if (t0 < t1) stage(t0, y1a, y2a, sta);
    if constexpr (!KEYS) {
        if (few) {
            if (t0 < t1) {
                Scores<T, D> f[G::KC];
                loads_arrived();
                __syncthreads();
#pragma unroll
                for (int kc = 0; kc < G::KC; ++kc) {
                    f[kc].form(x1, x2, y1a + kc * 32 * G::RB, y2a + kc * 32 * G::RB, dr, [](int) {});
                    weigh<T, D>(f[kc], c, own, G::BN > str_n, str_n - kc * 32, g);
#pragma unroll
                    for (int qb = 0; qb < 2; ++qb)
#pragma unroll
                        for (int i = 0; i < 8; ++i) own_delta[qb] += f[kc].s[i / 4][qb][i % 4] * f[kc].dp[i / 4][qb][i % 4];
                }
#pragma unroll
                for (int qb = 0; qb < 2; ++qb) {
                    own_delta[qb] = column_sum(own_delta[qb]);
                    if (kScaled<T>) own_delta[qb] *= two_to(-own_up[qb]);
                }
                if (a.dq.p)
#pragma unroll
                    for (int kc = 0; kc < G::KC; ++kc) add_keys<T, D, MODE>(acc, f[kc], own_delta, y1a + kc * 32 * G::RB, tr);
            }
            if (split == a.splits - 1) leave_stats();  // the split that has the tile, if there is one
            if (!a.dq.p) return;
        }
    }
    if constexpr (MODE != kFew) {
        const int32_t end = few ? t0 : t1;
        int kt = t0;
        // one exit, after a whole turn of both buffers: with another between them the sums are moved and spill
        for (; kt + 1 < end; kt += 2) {
            loads_arrived();
            __syncthreads();
            stage(kt + 1, y1b, y2b, stb);
            step(kt, y1a, y2a, sta);
            loads_arrived();
            __syncthreads();
            if (kt + 2 < end) stage(kt + 2, y1a, y2a, sta);
            step(kt + 1, y1b, y2b, stb);
        }
        if (kt < end) {
            loads_arrived();
            __syncthreads();
            step(kt, y1a, y2a, sta);
        }
    }
    const int32_t total = KEYS ? a.num_src : a.rows;
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        const int32_t o = own0 + w * 32 + qb * 16 + col;
        if (o >= total) continue;
        if constexpr (kScaled<T>) {
#pragma unroll
            for (int d = 0; d < G::DB; ++d) {
                acc.a1[d][qb] *= two_to(KEYS ? -keys_up : -own_up[qb]);
                if (KEYS) acc.a2[KEYS ? d : 0][qb] *= two_to(-kUp);
            }
        }
        if (a.splits > 1) {
            float *const p = a.part + ((bh * tiles + tile) * a.splits + split) * (KEYS ? 2 : 1) * kOwn * D + (o - own0) * D;
#pragma unroll
            for (int d = 0; d < G::DB; ++d) {
                *reinterpret_cast<f4 *>(p + d * 16 + g * 4) = acc.a1[d][qb];
                if (KEYS) *reinterpret_cast<f4 *>(p + kOwn * D + d * 16 + g * 4) = acc.a2[KEYS ? d : 0][qb];
            }
            continue;
        }
        const bool seen = o < own_n;  // keys past the sequence's length have gradient 0
        auto put = [&](uint16_t *p, f4 v) {
            *reinterpret_cast<u2 *>(p) = seen ? u2{T::pack(v[0], v[1]), T::pack(v[2], v[3])} : u2{0u, 0u};
        };
        if constexpr (KEYS) {
            uint16_t *const pk = const_cast<uint16_t *>(a.dk.p) + b * a.dk.batch + kv * a.dk.head + o * a.dk.row;
            uint16_t *const pv = const_cast<uint16_t *>(a.dv.p) + b * a.dv.batch + kv * a.dv.head + o * a.dv.row;
#pragma unroll
            for (int d = 0; d < G::DB; ++d) {
                if (a.dk.p) put(pk + d * 16 + g * 4, acc.a1[d][qb] * a.scale);
                if (a.dv.p) put(pv + d * 16 + g * 4, acc.a2[KEYS ? d : 0][qb]);
            }
        } else {
            uint16_t *const pq = const_cast<uint16_t *>(a.dq.p) + row_at(a, a.dq, b, kv, o);
#pragma unroll
            for (int d = 0; d < G::DB; ++d) put(pq + d * 16 + g * 4, acc.a1[d][qb] * a.scale);
        }
    }
}

// Adds the splits' sums in order: 4 widths a thread.
template <class T, int D, bool KEYS>
__global__ __launch_bounds__(kThreads) void reduce_kernel(Args a, int tiles) {
    constexpr int L = D / 4, M = KEYS ? 2 : 1;
    const int32_t total = KEYS ? a.num_src : a.rows;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t item = t / L;
    const int d = static_cast<int>(t % L) * 4;
    const int64_t bh = item / total;
    if (bh >= static_cast<int64_t>(a.batch) * a.kv_heads) return;
    const int32_t o = static_cast<int32_t>(item - bh * total);
    const int b = static_cast<int>(bh / a.kv_heads), kv = static_cast<int>(bh % a.kv_heads);
    const float *const p = a.part + ((bh * tiles + o / kOwn) * a.splits) * M * kOwn * D + o % kOwn * D + d;
    f4 s1{0.0f, 0.0f, 0.0f, 0.0f}, s2 = s1;
    if (!KEYS || o < sources(a, b)) {
#pragma unroll 8
        for (int i = 0; i < a.splits; ++i) {
            s1 += *reinterpret_cast<const f4 *>(p + static_cast<int64_t>(i) * M * kOwn * D);
            if (KEYS) s2 += *reinterpret_cast<const f4 *>(p + (static_cast<int64_t>(i) * M + 1) * kOwn * D);
        }
    }
    auto put = [&](const uint16_t *at, f4 v) {
        *reinterpret_cast<u2 *>(const_cast<uint16_t *>(at) + d) = u2{T::pack(v[0], v[1]), T::pack(v[2], v[3])};
    };
    s1 *= a.scale;
    if constexpr (KEYS) {
        if (a.dk.p) put(a.dk.p + b * a.dk.batch + kv * a.dk.head + o * a.dk.row, s1);
        if (a.dv.p) put(a.dv.p + b * a.dv.batch + kv * a.dv.head + o * a.dv.row, s2);
    } else {
        put(a.dq.p + row_at(a, a.dq, b, kv, o), s1);
    }
}

// ------------------------------------------------------------------------------------------ launch

struct Plan {
    int64_t tiles, splits;
};
// Owned tiles, and how many parts the streamed axis is cut into where they do not fill the device's blocks: as many as run
// at once, so none above half of those blocks.  Uncut against 2 and 3 parts in us (4096 streamed rows; 512 blocks run at once
// of width 64, of width 128 512 of dq and 256 of dk and dv): dk and dv of 64 at 256 items 82, 80, 86, at 300 118, 109, 101, at
// 384 121, 116, 126, at 448 127, 144, 154, at 512 132, 154, 165; of 128 at 128 items 125, 84, 108, at 160 127, 147, 114, at
// 192 127, 148, 155, at 256 131, 154, 171; dq of 64 at 256 items 76, 64, 69, at 300 97, 93, 83, at 384 98, 94, 102, at 448
// 102, 113, 116.
Plan plan_for(const tiga_cross &rel, bool keys) {
    const int64_t heads = static_cast<int64_t>(rel.batch) * rel.kv_heads, rows = rel.num_dst * (rel.heads / rel.kv_heads);
    const int64_t bn = rel.width == 64 ? 128 : 64;
    const int64_t own = keys ? rel.num_src : rows, streamed = ceil_div(keys ? rows : rel.num_src, bn);
    const int64_t resident = static_cast<int64_t>(device_cus()) * (keys && rel.width == 128 ? 1 : 2);
    Plan p{ceil_div(own, kOwn), 1};
    const int64_t items = p.tiles * heads;
    if (items > 0 && items * 2 <= resident) p.splits = resident / items;
    if (p.splits > streamed) p.splits = streamed < 1 ? 1 : streamed;
    return p;
}

// A grid counts its threads in 32 bits (and wraps around without an error).  The grids are of tiles, and of the sums of
// split items, which are at most as many as run at once.
constexpr int64_t kMostBlocks = (int64_t(1) << 24) - 1;

struct Layout {
    Plan q, kv;
    float *lse2, *delta, *part;
    f2 *peak;
    int64_t peaks;
    size_t bytes;
};
// Shares of a source head's peaks: blocks enough to read v and dy at the memory's rate, of 128 rows at least.
constexpr int64_t kPeakBlocks = 1024, kMostPeaks = 256;
Layout layout(const tiga_cross &rel, void *ws) {
    Layout l;
    l.q = plan_for(rel, false);
    l.kv = plan_for(rel, true);
    Carve c(ws);
    const size_t stats = static_cast<size_t>(rel.batch) * rel.heads * rel.num_dst + 1;
    l.lse2 = c.take<float>(stats);
    l.delta = c.take<float>(stats);
    // parts of as many items as run at once, whether this problem is split or not: a workspace holds every smaller one
    const size_t parts = static_cast<size_t>(device_cus()) * kOwn * rel.width * 2;
    l.part = c.take<float>(rel.width == 128 ? parts : 2 * parts);
    const int64_t heads = static_cast<int64_t>(rel.batch) * rel.kv_heads;
    l.peaks = ceil_div(rel.num_dst * (rel.heads / rel.kv_heads) + rel.num_src, 128);
    if (heads > 0 && l.peaks > kPeakBlocks / heads) l.peaks = kPeakBlocks / heads;
    if (l.peaks > kMostPeaks) l.peaks = kMostPeaks;
    if (l.peaks < 1) l.peaks = 1;
    l.peak = c.take<f2>(kPeakBlocks + heads);  // not less for a larger problem
    l.bytes = c.bytes();
    return l;
}

template <class T, int D, Mode MODE>
int products(const Plan &p, Args a, bool timed, hipStream_t stream) {
    constexpr bool KEYS = MODE == kKeys;
    const int64_t heads = static_cast<int64_t>(a.batch) * a.kv_heads, blocks = heads * p.tiles * p.splits;
    if (blocks == 0) return TIGA_OK;
    const int64_t sums = ceil_div(heads * (KEYS ? a.num_src : a.rows) * (D / 4), kThreads);
    a.splits = static_cast<int32_t>(p.splits);
    if (timed) prof_before(stream);
    hipLaunchKernelGGL((products_kernel<T, D, MODE>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, stream, a,
                       static_cast<int>(p.tiles));
    if (timed) prof_after(stream);
    if (int rc = check_launch("cross attention backward")) return rc;
    if (p.splits == 1) return TIGA_OK;
    hipLaunchKernelGGL((reduce_kernel<T, D, KEYS>), dim3(static_cast<unsigned>(sums)), dim3(kThreads), 0, stream, a,
                       static_cast<int>(p.tiles));
    return check_launch("cross attention backward sums");
}

template <class T, int D>
int launch(const Layout &l, const Args &a, hipStream_t stream) {
    const bool keys = a.dk.p || a.dv.p;
    if constexpr (kScaled<T>) {
        const dim3 grid(static_cast<unsigned>(a.batch * a.kv_heads * a.peaks));
        hipLaunchKernelGGL((peak_kernel<T, D>), grid, dim3(kThreads), 0, stream, a);
        if (int rc = check_launch("cross attention backward peaks")) return rc;
    }
    if (a.stats > 0) {
        Plan p = l.q;
        if (!a.dq.p) p.splits = 1;  // the rows' statistics alone
        const int rc = a.num_src <= Geo<D>::BN ? products<T, D, kFew>(p, a, !keys, stream)  // of one tile of keys: not split
                                               : products<T, D, kQuery>(p, a, !keys, stream);
        if (rc) return rc;
    }
    return keys ? products<T, D, kKeys>(l.kv, a, true, stream) : TIGA_OK;
}

}  // namespace

size_t cross_bwd_ws_bytes(const tiga_cross &rel) { return rel.kv_heads == 0 ? 256 : layout(rel, nullptr).bytes; }

int cross_backward(const tiga_cross &rel, const tiga_view &q, const tiga_view &k, const tiga_view &v,
                   const tiga_view &y, const float *lse, const tiga_view &dy, float scale, const tiga_view &dq,
                   const tiga_view &dk, const tiga_view &dv, void *ws, hipStream_t stream) {
    const Layout l = layout(rel, ws);
    const int64_t heads = static_cast<int64_t>(rel.batch) * rel.kv_heads;
    if (heads * l.q.tiles * l.q.splits > kMostBlocks || heads * l.kv.tiles * l.kv.splits > kMostBlocks)
        return fail(TIGA_EUNSUPPORTED, "cross attention backward: at most 2^24 - 1 tiles of 128 rows or sources");
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
    a.len = rel.src_len;
    a.lse2 = l.lse2;
    a.delta = l.delta;
    a.part = l.part;
    a.peak = l.peak;
    a.peaks = static_cast<int32_t>(l.peaks);
    a.num_dst = static_cast<int32_t>(rel.num_dst);
    a.num_src = static_cast<int32_t>(rel.num_src);
    a.batch = rel.batch;
    a.heads = rel.heads;
    a.kv_heads = rel.kv_heads;
    a.group = divider(rel.heads / rel.kv_heads);
    a.stats = static_cast<int64_t>(rel.batch) * rel.heads * rel.num_dst;
    a.rows = static_cast<int32_t>(rel.num_dst * (rel.heads / rel.kv_heads));
    a.scale = scale;
    if (rel.dtype == TIGA_DT_F16) return rel.width == 64 ? launch<Half16, 64>(l, a, stream) : launch<Half16, 128>(l, a, stream);
    return rel.width == 64 ? launch<Brain16, 64>(l, a, stream) : launch<Brain16, 128>(l, a, stream);
}

}  // namespace relattn
}  // namespace tiga
