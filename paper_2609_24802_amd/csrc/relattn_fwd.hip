// Online-softmax reducer over rectangular relations, forward: cross attention and causal attention of
// new tokens over a paged cache.  One wavefront a destination row and head; the lanes hold the width.
#include "relation.hpp"
#include "relattn.hpp"

namespace tiga {
namespace relattn {

namespace {

constexpr int kRows = 4;  // wavefronts (rows) per block
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

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

struct State {
    float m, l, o[2];
};

template <class T, int D>
__device__ __forceinline__ void key_step(State &s, const float *q, const uint16_t *k, const uint16_t *v, float c, bool bad) {
    float dot = 0.0f;
    for (int i = 0; i < D / 64; ++i) dot += q[i] * T::get(k[i * 64 + lane_id()]);
    float t = wave_sum(dot) * c;
    if (bad) t = __builtin_nanf("");
    if (!(t <= s.m)) {
        const float a = s.m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(s.m - t);
        s.m = t;
        s.l *= a;
        for (int i = 0; i < D / 64; ++i) s.o[i] *= a;
    }
    const float p = s.m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(t - s.m);
    s.l += p;
    for (int i = 0; i < D / 64; ++i) s.o[i] += p * T::get(v[i * 64 + lane_id()]);
}

template <class T, int D>
__device__ __forceinline__ void finish(const State &s, uint16_t *y, float *lse) {
    const float inv = s.l == 0.0f ? 0.0f : 1.0f / s.l;
    for (int i = 0; i < D / 64; ++i) y[i * 64 + lane_id()] = T::put(s.o[i] * inv);
    if (lse && lane_id() == 0) *lse = (s.m + __log2f(s.l)) * kLn2;
}

template <class T, int D>
__global__ __launch_bounds__(kRows * kWave) void cross_kernel(Rows q, Rows k, Rows v, Rows y, float *lse,
                                                             const int32_t *len, int64_t num_dst, int64_t num_src,
                                                             int batch, int heads, int group, float c) {
    const int64_t r = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / kWave;
    if (r >= static_cast<int64_t>(batch) * heads * num_dst) return;
    const int64_t i = r % num_dst;
    const int h = static_cast<int>(r / num_dst % heads), b = static_cast<int>(r / num_dst / heads);
    int64_t n = num_src;
    if (len) n = len[b] < 0 ? 0 : (len[b] > num_src ? num_src : len[b]);
    float qr[2];
    for (int e = 0; e < D / 64; ++e) qr[e] = T::get(q.p[b * q.batch + h * q.head + i * q.row + e * 64 + lane_id()]);
    const uint16_t *kp = k.p + b * k.batch + h / group * k.head, *vp = v.p + b * v.batch + h / group * v.head;
    State s{-__builtin_inff(), 0.0f, {0.0f, 0.0f}};
    for (int64_t j = 0; j < n; ++j) key_step<T, D>(s, qr, kp + j * k.row, vp + j * v.row, c, false);
    finish<T, D>(s, const_cast<uint16_t *>(y.p) + b * y.batch + h * y.head + i * y.row, lse ? lse + r : nullptr);
}

template <class T, int D>
__global__ __launch_bounds__(kRows * kWave) void paged_kernel(Pages cache, Rows q, Rows y, float *lse, int heads, int group,
                                                             float c) {
    const int64_t r = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / kWave;
    if (r >= static_cast<int64_t>(cache.num_dst) * heads) return;
    const int i = static_cast<int>(r / heads), h = static_cast<int>(r % heads);
    for (int b = 0; b < cache.batch; ++b) {
        const Chunk ch = chunk_of(cache, b);
        if (i < ch.first || i >= ch.first + ch.count) continue;
        const int64_t last = ch.pos0 + (i - ch.first);
        float qr[2];
        for (int e = 0; e < D / 64; ++e) qr[e] = T::get(q.p[h * q.head + i * q.row + e * 64 + lane_id()]);
        State s{-__builtin_inff(), 0.0f, {0.0f, 0.0f}};
        for (int64_t j = 0; j <= last; ++j) {
            const int32_t page = page_at(cache, b, j);
            const int64_t pg = page < 0 ? 0 : page, row = j & ((1 << cache.shift) - 1);
            key_step<T, D>(s, qr, cache.k.p + pg * cache.k.batch + h / group * cache.k.head + row * cache.k.row,
                           cache.v.p + pg * cache.v.batch + h / group * cache.v.head + row * cache.v.row, c, page < 0);
        }
        finish<T, D>(s, const_cast<uint16_t *>(y.p) + h * y.head + i * y.row,
                     lse ? lse + static_cast<int64_t>(h) * cache.num_dst + i : nullptr);
        return;
    }
}

}  // namespace

size_t cross_fwd_ws_bytes(const tiga_cross &) { return 256; }
size_t paged_fwd_ws_bytes(const tiga_cache &, int64_t, int32_t) { return 256; }

int cross_forward(const tiga_cross &rel, const tiga_view &q, const tiga_view &k, const tiga_view &v, float scale,
                  const tiga_view &y, float *lse, void *, hipStream_t stream) {
    const int64_t blocks = ceil_div(rel.num_dst * rel.heads * rel.batch, kRows);
    if (blocks > 0x7fffffff) return fail(TIGA_EUNSUPPORTED, "cross attention: too many rows");
    auto go = [&](auto kernel) {
        prof_before(stream);
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kRows * kWave), 0, stream, rows_of(q),
                           rows_of(k), rows_of(v), rows_of(y), lse, rel.src_len, rel.num_dst, rel.num_src, rel.batch,
                           rel.heads, rel.heads / rel.kv_heads, scale * kLog2e);
        prof_after(stream);
        return check_launch("cross attention forward");
    };
    if (rel.dtype == TIGA_DT_F16) return rel.width == 64 ? go(cross_kernel<F16, 64>) : go(cross_kernel<F16, 128>);
    return rel.width == 64 ? go(cross_kernel<BF16, 64>) : go(cross_kernel<BF16, 128>);
}

int paged_forward(const tiga_cache &cache, int64_t num_dst, const int32_t *dst_ptr, int32_t heads, const tiga_view &q,
                  float scale, const tiga_view &y, float *lse, void *, hipStream_t stream) {
    const int64_t blocks = ceil_div(num_dst * heads, kRows);
    auto go = [&](auto kernel) {
        prof_before(stream);
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kRows * kWave), 0, stream,
                           pages_of(cache, num_dst, dst_ptr), rows_of(q), rows_of(y), lse, heads,
                           heads / cache.kv_heads, scale * kLog2e);
        prof_after(stream);
        return check_launch("paged attention forward");
    };
    if (cache.dtype == TIGA_DT_F16) return cache.width == 64 ? go(paged_kernel<F16, 64>) : go(paged_kernel<F16, 128>);
    return cache.width == 64 ? go(paged_kernel<BF16, 64>) : go(paged_kernel<BF16, 128>);
}

}  // namespace relattn
}  // namespace tiga
