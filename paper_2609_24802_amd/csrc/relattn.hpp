// Host interface of the online-softmax reducer over rectangular relations: cross attention over strided
// sources (forward and vector-Jacobian product) and causal attention of new tokens over a paged cache.
#pragma once

#include "common.hpp"

namespace tiga {
namespace relattn {

// Arguments are validated by the caller (api_relattn.hip).
size_t cross_fwd_ws_bytes(const tiga_cross &rel);
int cross_forward(const tiga_cross &rel, const tiga_view &q, const tiga_view &k, const tiga_view &v, float scale,
                  const tiga_view &y, float *lse, void *ws, hipStream_t stream);

size_t cross_bwd_ws_bytes(const tiga_cross &rel);
// dq, dk, dv: data NULL where the gradient is not wanted.
int cross_backward(const tiga_cross &rel, const tiga_view &q, const tiga_view &k, const tiga_view &v,
                   const tiga_view &y, const float *lse, const tiga_view &dy, float scale, const tiga_view &dq,
                   const tiga_view &dk, const tiga_view &dv, void *ws, hipStream_t stream);

size_t paged_fwd_ws_bytes(const tiga_cache &cache, int64_t num_dst, int32_t heads);
int paged_forward(const tiga_cache &cache, int64_t num_dst, const int32_t *dst_ptr, int32_t heads, const tiga_view &q,
                  float scale, const tiga_view &y, float *lse, void *ws, hipStream_t stream);

}  // namespace relattn
}  // namespace tiga
