// Matrix products of the attention gradients: what a wavefront that owns 32 columns (rows of q and dy, or keys and values)
// does with 32 or 64 streamed rows in LDS.
#pragma once

#include <type_traits>

#include "mfma16.hpp"

namespace tiga {
namespace relattn {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kOwn = 128;  // owned rows or keys of a block: 32 a wavefront
constexpr float kLog2e = 1.4426950408889634f;

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
    // bit n of `exists`: whether the pair does.  In bfloat16, whose products may pass fp32's range, a pair that does not has no DS
    // also where its product or the row's statistics are not finite (0 times which would be NaN): both P and DS are cleared, two
    // in a register.  (Each by itself takes 1.5 % of dk and dv of 16,384 tokens, 16 heads over 4 of 128.)
    __device__ __forceinline__ void form_if(const Scores<T, D> &f, float c, float h, int n, uint32_t exists) {
        const uint32_t mask = static_cast<uint32_t>(__builtin_amdgcn_sbfe(exists, n, 1));
        if constexpr (kScaled<T>) {
            const int qb = n / 8, e = n / 4 % 2, i = n % 4;
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(f.s[e][qb][i], c, -lse2[e][i]));
            p[n] = __uint_as_float(__float_as_uint(x) & mask);
            ds[n] = p[n] * __builtin_fmaf(f.dp[e][qb][i], h, -delta[e][i]);
            if (n % 2) {
                pw[n / 2] = T::pack(p[n - 1], p[n]);
                dw[n / 2] = T::pack(ds[n - 1], ds[n]);
            }
        } else {
            form(f, c, h, n);
            if (n % 2) {
                const uint32_t both = __builtin_amdgcn_perm(mask, static_cast<uint32_t>(__builtin_amdgcn_sbfe(exists, n - 1, 1)), 0x07060100u);
                pw[n / 2] &= both;
                dw[n / 2] &= both;
            }
        }
    }
};

// dk and dv, 64 streamed rows as two halves.  The first half's weights are formed under the products for the second's
// scores, the second's under the first half's sums: at width 128 a SIMD has one wavefront, and nothing else fills its
// matrix unit meanwhile (527 us without, 494).  At width 64 two wavefronts share a SIMD: 8 x 449 rows over 1500 ragged 54.8
// and 52.7 us, 4 x 4096 over 77 23.4 and 21.0, 4 x 4096 over 4096 507 and 525.
// CUT: bit n of exists[half] says whether pair n of the half does; otherwise all do.  At width 64 in bfloat16 the halves of a cut
// tile are taken one after the other: side by side the masks spill 21 registers, in all tiles (61 sequences of 131 tokens, 16
// heads: 60 us of dk and dv, so 51).
template <class T, int D, bool CUT = false>
__device__ __forceinline__ void rows_step(Sums<T, D, kKeys> &acc, const u4 (&x1)[2][Geo<D>::CH],
                                          const u4 (&x2)[2][Geo<D>::CH], const uint8_t *y1, const uint8_t *y2, int dr,
                                          int tr, float c, float h, const float *st, const float *sd, int g,
                                          const uint32_t *exists = nullptr) {
    constexpr int kHalf = 32 * Geo<D>::RB, kScore = 16 / Scores<T, D>::kReads, kSum = 16 / kSumReads<T, D, kKeys>;
    auto operand = [](const uint32_t *x, int qb) { return u4{x[4 * qb], x[4 * qb + 1], x[4 * qb + 2], x[4 * qb + 3]}; };
    if constexpr (CUT && D == 64 && !kScaled<T>) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            Scores<T, D> f;
            Weights<T, D> w;
            w.load(st + 32 * half, sd + 32 * half, g);
            f.form(x1, x2, y1 + half * kHalf, y2 + half * kHalf, dr, [](int) {});
#pragma unroll
            for (int n = 0; n < 16; ++n) w.form_if(f, c, h, n, exists[half]);
            const u4 p[2] = {operand(w.pw, 0), operand(w.pw, 1)}, d[2] = {operand(w.dw, 0), operand(w.dw, 1)};
            add_products<T, D, kKeys>(acc, p, d, y1 + half * kHalf, y2 + half * kHalf, tr, [](int) {});
        }
        return;
    }
    Scores<T, D> f0, f1;
    Weights<T, D> w0, w1;
    w0.load(st, sd, g);
    f0.form(x1, x2, y1, y2, dr, [](int) {});
    f1.form(x1, x2, y1 + kHalf, y2 + kHalf, dr, [&](int i) {
#pragma unroll
        for (int n = 0; n < kScore; ++n) {
            if constexpr (CUT) w0.form_if(f0, c, h, i * kScore + n, exists[0]);
            else w0.form(f0, c, h, i * kScore + n);
        }
    });
    w1.load(st + 32, sd + 32, g);
    const u4 p0[2] = {operand(w0.pw, 0), operand(w0.pw, 1)}, d0[2] = {operand(w0.dw, 0), operand(w0.dw, 1)};
    add_products<T, D, kKeys>(acc, p0, d0, y1, y2, tr, [&](int i) {
#pragma unroll
        for (int n = 0; n < kSum; ++n) {
            if constexpr (CUT) w1.form_if(f1, c, h, i * kSum + n, exists[1]);
            else w1.form(f1, c, h, i * kSum + n);
        }
    });
    const u4 p1[2] = {operand(w1.pw, 0), operand(w1.pw, 1)}, d1[2] = {operand(w1.dw, 0), operand(w1.dw, 1)};
    add_products<T, D, kKeys>(acc, p1, d1, y1 + kHalf, y2 + kHalf, tr, [](int) {});
}

}  // namespace

}  // namespace relattn
}  // namespace tiga
