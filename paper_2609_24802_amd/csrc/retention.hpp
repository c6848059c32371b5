// Host interface of what decides which positions of a paged cache stay: the weights that they get, and the eviction of those
// with the least.
#pragma once

#include "common.hpp"

namespace tiga {
namespace retention {

// Arguments are validated by the caller (api_relattn.hip).
size_t weights_ws_bytes(const tiga_cache &cache, int64_t num_dst, int32_t heads);
int accumulate(const tiga_cache &cache, int64_t num_dst, const int32_t *dst_ptr, int32_t heads, const tiga_view &q,
               const float *lse, float scale, float decay, const float *weights, float *out, void *ws, hipStream_t stream);

// staged: the rows that stay pass through the workspace, for a cache that is evicted from in place.
size_t evict_ws_bytes(const tiga_cache &cache, int32_t keep, bool staged);
int evict(const tiga_cache &cache, const float *weights, int32_t keep, int32_t recent, const tiga_cache &to,
          float *to_weights, int32_t *to_length, int32_t *kept, bool staged, void *ws, hipStream_t stream);

}  // namespace retention
}  // namespace tiga
