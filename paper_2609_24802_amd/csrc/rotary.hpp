// Host interface of the rotary positions and of the append of new tokens to a paged cache.
#pragma once

#include "common.hpp"

namespace tiga {
namespace rotary {

// y = x rotated by its positions, or (back) turned the other way.  Arguments are validated by the caller.
int rotate(int32_t batch, int32_t heads, int64_t rows, int32_t width, int dtype, const tiga_view &x,
           const int32_t *pos, int64_t pos_batch, const tiga_rotary &rot, bool back, const tiga_view &y,
           hipStream_t stream);

// rot.freq NULL: no rotation; q.data NULL: no queries.
int append(const tiga_cache &cache, int64_t num_dst, const int32_t *dst_ptr, const tiga_view &k, const tiga_view &v,
           const tiga_rotary &rot, int32_t heads, const tiga_view &q, const tiga_view &q_out, hipStream_t stream);

}  // namespace rotary
}  // namespace tiga
