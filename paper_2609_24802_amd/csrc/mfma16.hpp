// Building blocks of the 16-bit matrix kernels (gfx950): types, MFMA, direct loads to LDS, transposing LDS reads.
#pragma once

#include "common.hpp"

namespace tiga {

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));

// A 16-bit type: MFMA 16x16x32 with fp32 accumulation (A: 16 rows x 32, lane l holds row l % 16, elements
// 8 (l / 16) + 0..7; B: 32 x 16, column l % 16 likewise; C: rows 4 (l / 16) + 0..3 of column l % 16), the packed
// fp32 -> 16-bit conversion (round to nearest even) and back, and the exponent's bits, all set where a number is not finite.
struct Half16 {
    static constexpr uint32_t kExponent = 0x7c00u;
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    typedef _Float16 v2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ f4 mma(u4 a, u4 b, f4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{a, b}), v2));
    }
    static __device__ __forceinline__ f2 unpack(uint32_t x) {
        return __builtin_convertvector(__builtin_bit_cast(v2, x), f2);
    }
};
struct Brain16 {
    static constexpr uint32_t kExponent = 0x7f80u;
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    typedef __bf16 v2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ f4 mma(u4 a, u4 b, f4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{a, b}), v2));
    }
    static __device__ __forceinline__ f2 unpack(uint32_t x) {
        return f2{__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)};
    }
};

// Over the four lanes l, l^16, l^32, l^48 (those that share a column of an MFMA result), with the gfx950 lane
// swaps: each swap returns, per lane, its own value and its partner's.
__device__ __forceinline__ float column_max(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float column_sum(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Bit 15 of each half that is not finite: adding 0x8000 less the exponent's bits carries into it.
template <class T>
__device__ __forceinline__ uint32_t wild(uint32_t x) {
    return ((x & 0x7fff7fffu) + (0x8000u - T::kExponent) * 0x10001u) & 0x80008000u;
}
template <class T>
__device__ __forceinline__ uint32_t any_wild(u4 x) {
    return (wild<T>(x[0]) | wild<T>(x[1])) | (wild<T>(x[2]) | wild<T>(x[3]));
}
template <class T>
__device__ __forceinline__ u4 without_wild(u4 x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] &= ~((wild<T>(x[e]) >> 15) * 0xffffu);
    return x;
}
// o += the values (4 widths) that are not finite, for a row that sees them.
template <class T>
__device__ __forceinline__ void add_wild(f4 &o, u2 x, bool sees) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t m = sees ? wild<T>(x[e]) : 0u;
        const f2 v = T::unpack(x[e]);
        o[2 * e] += m & 0x8000u ? v.x : 0.0f;
        o[2 * e + 1] += m >> 16 ? v.y : 0.0f;
    }
}

// 16 bytes per lane from global memory straight into LDS: lane t writes bytes [16 t, 16 t + 16) of the 1-KB
// run at `run` (a wavefront-uniform LDS address).  Buffers that are read while a load into another is in
// flight are separate __shared__ arrays, so that the compiler sees that the read need not wait.
__device__ __forceinline__ void load_to_lds16(const void *src, uint8_t *run) {
    __builtin_amdgcn_global_load_lds(src, (__attribute__((address_space(3))) void *)run, 16, 0, 0);
}
// Every load of this wavefront has arrived (direct loads to LDS among them).
__device__ __forceinline__ void loads_arrived() { __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// gfx950 transposing LDS read of 16-bit data: within each group of 16 lanes, lane i receives, in slot j, element
// i % 4 of the 8 bytes addressed by lane 4 j + i / 4 of its group.
__device__ __forceinline__ u2 lds_transposed16(const uint8_t *p) {
    typedef short s4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)p));
}

}  // namespace tiga
