// Device-side addressing of the rectangular relations: which sources a destination row has and where
// their keys and values lie.
#pragma once

#include "common.hpp"

namespace tiga {
namespace relattn {

// n / d for n < 2^31 by a multiplication (round-up method; m holds the low 32 bits of a 33-bit factor).
struct Divider {
    uint32_t m, s, d;
    __device__ __forceinline__ int32_t div(int32_t n) const {
        return static_cast<int32_t>((__umulhi(m, static_cast<uint32_t>(n)) + static_cast<uint32_t>(n)) >> s);
    }
};
inline Divider divider(int32_t d) {
    uint32_t s = 0;
    const uint64_t n = static_cast<uint64_t>(d);
    while ((uint64_t(1) << s) < n) ++s;
    return Divider{static_cast<uint32_t>(((uint64_t(1) << 32) * ((uint64_t(1) << s) - n)) / n + 1), s, static_cast<uint32_t>(d)};
}

// a / b for a >= 0, b > 0 (uniform): the 64-bit division is a long subroutine, and these values are small.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}

// Inclusive prefix sum over the wavefront by lane shifts within the vector unit (no LDS round trips): shifts by 1, 2, 4
// and 8 within rows of 16 lanes, then row 0 and 2 into the next, then the lower half into the upper.
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t lanes_shifted(int64_t v) {
    const int lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROWS, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(v >> 32), CTRL, ROWS, 0xf, false);
    return static_cast<int64_t>((static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32) | static_cast<uint32_t>(lo));
}
__device__ __forceinline__ int64_t wave_prefix(int64_t v) {
    v += lanes_shifted<0x111, 0xf>(v);
    v += lanes_shifted<0x112, 0xf>(v);
    v += lanes_shifted<0x114, 0xf>(v);
    v += lanes_shifted<0x118, 0xf>(v);
    v += lanes_shifted<0x142, 0xa>(v);
    v += lanes_shifted<0x143, 0xc>(v);
    return v;
}
__device__ __forceinline__ int64_t lane_value(int64_t v, int lane) {  // lane: uniform
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(v), lane);
    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(static_cast<uint64_t>(v) >> 32), lane);
    return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}

// Element strides of a view as the kernels take them.
struct Rows {
    const uint16_t *p;
    int64_t batch, head, row;
};
inline Rows rows_of(const tiga_view &v) { return Rows{static_cast<const uint16_t *>(v.data), v.batch, v.head, v.row}; }

// A paged cache: the page of position p is table[p >> shift], its row p & mask.
struct Pages {
    Rows k, v;
    const int32_t *table;
    const int32_t *length;
    const int32_t *dst_ptr;
    int64_t num_pages;
    int32_t batch, table_width, shift;
    int32_t num_dst;
};
inline Pages pages_of(const tiga_cache &c, int64_t num_dst, const int32_t *dst_ptr) {
    int shift = 0;
    while ((1 << shift) < c.page_size) ++shift;
    return Pages{rows_of(c.k), rows_of(c.v), c.table, c.length, dst_ptr, c.num_pages, c.batch, c.table_width, shift,
                 static_cast<int32_t>(num_dst)};
}

// Rows [first, first + count) of sequence b and their positions pos0 + t.  Pointers that run
// backwards or past num_dst give an empty or a shortened range, never one outside the tensors.
struct Chunk {
    int32_t first, count;
    int64_t pos0;
};
__device__ __forceinline__ Chunk chunk_of(const Pages &c, int b) {
    int32_t s = c.dst_ptr[b], e = c.dst_ptr[b + 1];
    s = s < 0 ? 0 : (s > c.num_dst ? c.num_dst : s);
    e = e < s ? s : (e > c.num_dst ? c.num_dst : e);
    return Chunk{s, e - s, static_cast<int64_t>(c.length[b]) - (e - s)};
}

// The table's entry for position pos (>= 0) of sequence b, -1 where the table does not reach.  Only an entry that
// is_page() accepts names a page; the check is apart so that a look-up ahead of its use need not wait for the load.
__device__ __forceinline__ int32_t entry_at(const Pages &c, int b, int64_t pos) {
    const int64_t e = pos >> c.shift;
    if (e >= c.table_width) return -1;
    return c.table[static_cast<int64_t>(b) * c.table_width + e];
}
__device__ __forceinline__ bool is_page(const Pages &c, int32_t id) {
    return static_cast<uint32_t>(id) < static_cast<uint32_t>(c.num_pages);  // num_pages < 2^31
}
// The page of a position, -1 if there is none.
__device__ __forceinline__ int32_t page_at(const Pages &c, int b, int64_t pos) {
    const int32_t id = entry_at(c, b, pos);
    return is_page(c, id) ? id : -1;
}

}  // namespace relattn
}  // namespace tiga
