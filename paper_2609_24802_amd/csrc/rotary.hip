// Rotary positions, and the append of new tokens to a paged cache with the rotation on the way.
//   pair (a, b) at position p -> amplitude (a cos t - b sin t, a sin t + b cos t),  t = p freq
// The angle is formed in fp64 as turns u = p freq / 2 pi and reduced there to an eighth of a turn
// either side of a quarter (|r| <= 1/8, u = k / 4 + r); in fp32 a position of 10^6 alone would cost
// 0.03 radians.  Sine and cosine of r are fp32.
#include "relation.hpp"
#include "rotary.hpp"

namespace tiga {
namespace rotary {

using relattn::Chunk;
using relattn::chunk_of;
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

// Pair i of every head of a row (one thread); past rot / 2, elements 2 i and 2 i + 1 are copied.
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
__global__ __launch_bounds__(kThreads) void rotate_kernel(tiga_view x, tiga_view y, const int32_t *__restrict__ pos,
                                                          int64_t pos_batch, int64_t rows, int64_t total, int heads,
                                                          int width, tiga_rotary rot, float sign) {
    const int units = (width + 1) / 2;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (t >= total) return;
    const int i = static_cast<int>(t % units);
    const int64_t r = t / units % rows, b = t / units / rows;
    Angle a{};
    if (i < rot.rot / 2) a = angle_of(pos ? pos[b * pos_batch + r] : r, rot.freq[i], rot.amplitude, sign);
    turn_heads<T>(static_cast<const typename T::raw *>(x.data) + b * x.batch + r * x.row, x.head,
                  static_cast<typename T::raw *>(y.data) + b * y.batch + r * y.row, y.head, heads, i, width, rot, a);
}

// A block per new token.
template <class T>
__global__ __launch_bounds__(kThreads) void append_kernel(Pages cache, tiga_view k, tiga_view v, tiga_rotary rot, int heads,
                                                          int kv_heads, tiga_view q, tiga_view qo, int width) {
    typedef typename T::raw raw;
    const int row = blockIdx.x;
    int b = 0;
    for (int base = 0; base < cache.batch; base += kWave) {
        const int e = base + lane_id();
        const bool before = e < cache.batch && cache.dst_ptr[e + 1] <= row;
        const int n = __popcll(__ballot(before));
        b += n;
        if (n < kWave) break;
    }
    if (b >= cache.batch) return;
    const Chunk ch = chunk_of(cache, b);
    if (row < ch.first || row >= ch.first + ch.count) return;
    const int64_t pos = ch.pos0 + (row - ch.first);
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

}  // namespace

int rotate(int32_t batch, int32_t heads, int64_t rows, int32_t width, int dtype, const tiga_view &x,
           const int32_t *pos, int64_t pos_batch, const tiga_rotary &rot, bool back, const tiga_view &y,
           hipStream_t stream) {
    const int64_t total = rows * batch * ((width + 1) / 2);
    const int64_t blocks = ceil_div(total, kThreads);
    if (blocks > 0x7fffffff) return fail(TIGA_EUNSUPPORTED, "rotary: too many rows");
    auto go = [&](auto kernel) {
        prof_before(stream);
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, stream, x, y, pos, pos_batch, rows,
                           total, heads, width, rot, back ? -1.0f : 1.0f);
        prof_after(stream);
        return check_launch("rotary");
    };
    if (dtype == TIGA_DT_F32) return go(rotate_kernel<F32>);
    return dtype == TIGA_DT_F16 ? go(rotate_kernel<F16>) : go(rotate_kernel<BF16>);
}

int append(const tiga_cache &cache, int64_t num_dst, const int32_t *dst_ptr, const tiga_view &k, const tiga_view &v,
           const tiga_rotary &rot, int32_t heads, const tiga_view &q, const tiga_view &q_out, hipStream_t stream) {
    auto go = [&](auto kernel) {
        prof_before(stream);
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(num_dst)), dim3(kThreads), 0, stream,
                           pages_of(cache, num_dst, dst_ptr), k, v, rot, heads, cache.kv_heads, q, q_out, cache.width);
        prof_after(stream);
        return check_launch("cache append");
    };
    return cache.dtype == TIGA_DT_F16 ? go(append_kernel<F16>) : go(append_kernel<BF16>);
}

}  // namespace rotary
}  // namespace tiga
