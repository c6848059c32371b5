// Vector-Jacobian product of cross attention: dq over a destination's sources, dk and dv over a source's
// destinations (of every head that shares it).  One wavefront a row; the lanes hold the width.
#include "relation.hpp"
#include "relattn.hpp"

namespace tiga {
namespace relattn {

namespace {

constexpr int kRows = 4;
constexpr float kLog2e = 1.4426950408889634f;

struct F16 {
    static __device__ __forceinline__ float get(uint16_t b) { return static_cast<float>(__builtin_bit_cast(_Float16, b)); }
    static __device__ __forceinline__ uint16_t put(float f) { return __builtin_bit_cast(uint16_t, static_cast<_Float16>(f)); }
};
struct BF16 {
    static __device__ __forceinline__ float get(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
    static __device__ __forceinline__ uint16_t put(float f) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }
};

__device__ __forceinline__ float wave_sum(float v) {
    for (int d = 1; d < kWave; d <<= 1) v += shfl_xor_f(v, d);
    return v;
}

struct Args {
    Rows q, k, v, y, dy, dq, dk, dv;
    const float *lse;
    const int32_t *len;
    int64_t num_dst, num_src;
    int batch, heads, group;
    float scale;
};

template <class T, int D>
__device__ __forceinline__ void load(float *r, const uint16_t *p) {
    for (int e = 0; e < D / 64; ++e) r[e] = T::get(p[e * 64 + lane_id()]);
}
template <class T, int D>
__device__ __forceinline__ void store(const uint16_t *p, const float *r) {
    for (int e = 0; e < D / 64; ++e) const_cast<uint16_t *>(p)[e * 64 + lane_id()] = T::put(r[e]);
}
template <int D>
__device__ __forceinline__ float dot(const float *a, const float *b) {
    float s = 0.0f;
    for (int e = 0; e < D / 64; ++e) s += a[e] * b[e];
    return wave_sum(s);
}
__device__ __forceinline__ int64_t sources(const Args &a, int b) {
    if (!a.len) return a.num_src;
    return a.len[b] < 0 ? 0 : (a.len[b] > a.num_src ? a.num_src : a.len[b]);
}

template <class T, int D>
__global__ __launch_bounds__(kRows * kWave) void dq_kernel(Args a) {
    const int64_t r = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / kWave;
    if (r >= static_cast<int64_t>(a.batch) * a.heads * a.num_dst) return;
    const int64_t i = r % a.num_dst;
    const int h = static_cast<int>(r / a.num_dst % a.heads), b = static_cast<int>(r / a.num_dst / a.heads);
    const int64_t n = sources(a, b);
    float q[2], y[2], dy[2], k[2], v[2], o[2] = {0.0f, 0.0f};
    load<T, D>(q, a.q.p + b * a.q.batch + h * a.q.head + i * a.q.row);
    load<T, D>(y, a.y.p + b * a.y.batch + h * a.y.head + i * a.y.row);
    load<T, D>(dy, a.dy.p + b * a.dy.batch + h * a.dy.head + i * a.dy.row);
    const float delta = dot<D>(y, dy), lse = a.lse[r];
    for (int64_t j = 0; j < n; ++j) {
        load<T, D>(k, a.k.p + b * a.k.batch + h / a.group * a.k.head + j * a.k.row);
        load<T, D>(v, a.v.p + b * a.v.batch + h / a.group * a.v.head + j * a.v.row);
        const float p = __builtin_amdgcn_exp2f((dot<D>(q, k) * a.scale - lse) * kLog2e);
        const float ds = p * (dot<D>(dy, v) - delta) * a.scale;
        for (int e = 0; e < D / 64; ++e) o[e] += ds * k[e];
    }
    store<T, D>(a.dq.p + b * a.dq.batch + h * a.dq.head + i * a.dq.row, o);
}

template <class T, int D>
__global__ __launch_bounds__(kRows * kWave) void dkv_kernel(Args a) {
    const int64_t r = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / kWave;
    const int kvh = a.heads / a.group;
    if (r >= static_cast<int64_t>(a.batch) * kvh * a.num_src) return;
    const int64_t j = r % a.num_src;
    const int g = static_cast<int>(r / a.num_src % kvh), b = static_cast<int>(r / a.num_src / kvh);
    float q[2], y[2], dy[2], k[2], v[2], dk[2] = {0.0f, 0.0f}, dv[2] = {0.0f, 0.0f};
    if (j < sources(a, b)) {
        load<T, D>(k, a.k.p + b * a.k.batch + g * a.k.head + j * a.k.row);
        load<T, D>(v, a.v.p + b * a.v.batch + g * a.v.head + j * a.v.row);
        for (int h = g * a.group; h < (g + 1) * a.group; ++h)
            for (int64_t i = 0; i < a.num_dst; ++i) {
                load<T, D>(q, a.q.p + b * a.q.batch + h * a.q.head + i * a.q.row);
                load<T, D>(y, a.y.p + b * a.y.batch + h * a.y.head + i * a.y.row);
                load<T, D>(dy, a.dy.p + b * a.dy.batch + h * a.dy.head + i * a.dy.row);
                const float lse = a.lse[(static_cast<int64_t>(b) * a.heads + h) * a.num_dst + i];
                const float p = __builtin_amdgcn_exp2f((dot<D>(q, k) * a.scale - lse) * kLog2e);
                const float ds = p * (dot<D>(dy, v) - dot<D>(y, dy)) * a.scale;
                for (int e = 0; e < D / 64; ++e) {
                    dk[e] += ds * q[e];
                    dv[e] += p * dy[e];
                }
            }
    }
    if (a.dk.p) store<T, D>(a.dk.p + b * a.dk.batch + g * a.dk.head + j * a.dk.row, dk);
    if (a.dv.p) store<T, D>(a.dv.p + b * a.dv.batch + g * a.dv.head + j * a.dv.row, dv);
}

template <class T, int D>
int launch(const Args &a, int64_t num_src_rows, hipStream_t stream) {
    const int64_t rows = a.num_dst * a.heads * a.batch;
    prof_before(stream);
    if (a.dq.p && rows)
        hipLaunchKernelGGL((dq_kernel<T, D>), dim3(static_cast<unsigned>(ceil_div(rows, kRows))), dim3(kRows * kWave), 0,
                           stream, a);
    if ((a.dk.p || a.dv.p) && num_src_rows)
        hipLaunchKernelGGL((dkv_kernel<T, D>), dim3(static_cast<unsigned>(ceil_div(num_src_rows, kRows))),
                           dim3(kRows * kWave), 0, stream, a);
    prof_after(stream);
    return check_launch("cross attention backward");
}

}  // namespace

size_t cross_bwd_ws_bytes(const tiga_cross &) { return 256; }

int cross_backward(const tiga_cross &rel, const tiga_view &q, const tiga_view &k, const tiga_view &v,
                   const tiga_view &y, const float *lse, const tiga_view &dy, float scale, const tiga_view &dq,
                   const tiga_view &dk, const tiga_view &dv, void *, hipStream_t stream) {
    const Args a{rows_of(q), rows_of(k), rows_of(v), rows_of(y), rows_of(dy), rows_of(dq), rows_of(dk), rows_of(dv), lse,
                 rel.src_len, rel.num_dst, rel.num_src, rel.batch, rel.heads, rel.heads / rel.kv_heads, scale};
    const int64_t src_rows = rel.num_src * rel.kv_heads * rel.batch;
    if (ceil_div(rel.num_dst * rel.heads * rel.batch, kRows) > 0x7fffffff || ceil_div(src_rows, kRows) > 0x7fffffff)
        return fail(TIGA_EUNSUPPORTED, "cross attention: too many rows");
    if (rel.dtype == TIGA_DT_F16) return rel.width == 64 ? launch<F16, 64>(a, src_rows, stream) : launch<F16, 128>(a, src_rows, stream);
    return rel.width == 64 ? launch<BF16, 64>(a, src_rows, stream) : launch<BF16, 128>(a, src_rows, stream);
}

}  // namespace relattn
}  // namespace tiga
