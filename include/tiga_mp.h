/*
 * tiga_mp.h -- C ABI of the MI355X (gfx950) fused message-passing library.
 *
 * Fused message passing (Tiga, "Compiling Graph Message Passing at Scale"):
 * for every destination entity the library traverses a relation, forms one
 * message per (source, destination) pair and folds it into the reducer state
 * immediately, so neither the edge list of a generated relation nor any
 * per-edge message array is ever stored (Section 3.1 message/update equation;
 * Section 4.2 on fused row traversal versus materialized E*F messages).
 *
 * Three relations are supported:
 *   - a stored destination-major CSR graph (Sections 3.1 and 4.3),
 *   - a radius relation generated from positions through a cell directory
 *     (Section 4.9),
 *   - the dense all-pairs relation, which needs no edge array (Section 1).
 * Reverse mode (Section 5, vector-Jacobian products) is provided for the CSR
 * and radius relations.
 * The online-softmax reducer (Section 5.2) also runs over the triangular and
 * the dense relation of a sequence with itself, over the rectangular relation
 * to another sequence (cross attention, with its vector-Jacobian product), and
 * over a sequence's pages in a cache; rotary positions and the append to a
 * cache feed it.
 *
 * Conventions shared by every entry point
 *   - Arrays are DEVICE pointers unless a comment says otherwise.  The caller
 *     owns every buffer, including the workspace `ws` of `ws_bytes` bytes
 *     (size it with the matching *_workspace query; it must be 256-byte
 *     aligned).  The library keeps no pointer after the call returns.
 *   - Work is enqueued on `stream` (a hipStream_t passed as void*; NULL is the
 *     null stream).  Calls return before the work completes; a device fault
 *     surfaces at the caller's next synchronization.  Only
 *     tiga_csr_validate(level 2), tiga_radius_neighbors, tiga_cache_validate,
 *     tiga_prefix_validate and tiga_retention_validate synchronize.
 *   - Outputs are overwritten, never accumulated into.
 *   - fp32 features are row-major [rows, feat], of any width.  Rows need only
 *     the alignment of floats; some paths are faster where feat % 4 == 0 and
 *     arrays are 16-byte aligned.
 *   - Arguments are checked on the host before anything is enqueued.  On
 *     error the call returns a negative status, enqueues nothing, and
 *     tiga_last_error() describes the problem.  There is no silent fallback:
 *     unsupported combinations return TIGA_EUNSUPPORTED (the paper requires
 *     explicit diagnosis rather than a substituted route, Sections 4.1 and 4.8).
 *   - The library holds no global mutable state other than the per-thread
 *     error string and the per-thread profiling events; calls are reentrant.
 */
#ifndef TIGA_MP_H
#define TIGA_MP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define TIGA_MP_ABI_VERSION 2

/* Status codes. */
enum tiga_status {
    TIGA_OK = 0,
    TIGA_EINVAL = -1,       /* bad argument (NULL, negative size, misaligned ws) */
    TIGA_EGRAPH = -2,       /* the relation violates CSR invariants (validation) */
    TIGA_EUNSUPPORTED = -3, /* valid request this library does not implement */
    TIGA_EWORKSPACE = -4,   /* ws_bytes smaller than the workspace query */
    TIGA_EDEVICE = -5       /* a HIP call failed */
};

/* Reducers (Section 3.1: identity, lift, combine, finalize).
 *   SUM: identity 0; an empty row finalizes to 0.
 *   MAX: identity -inf; ties keep the lowest edge position; an empty row
 *        finalizes to value 0 with argmax -1. */
enum tiga_reducer { TIGA_REDUCE_SUM = 0, TIGA_REDUCE_MAX = 1 };

/* Messages over a stored CSR relation (edge function of Section 3.1). */
enum tiga_csr_msg {
    TIGA_MSG_SRC = 0,             /* m_e = x[s(e)]          (w_edge must be NULL) */
    TIGA_MSG_EDGE_SCALED_SRC = 1  /* m_e = w[e] * x[s(e)]   (w_edge required)     */
};

/* Destination-major CSR relation (Sections 3.1, 4.3).  Destination row i owns
 * edge positions [row_ptr[i], row_ptr[i+1]); the edge position indexes edge
 * fields and col_idx[e] is the source id.  Duplicates and self edges are
 * ordinary separate edges; num_src may differ from num_dst.
 *   row_ptr: int64 [num_dst + 1], row_ptr[0] == 0, non-decreasing,
 *            row_ptr[num_dst] == num_edges.
 *   col_idx: int32 [num_edges], each in [0, num_src).
 * The struct itself lives in HOST memory; the two arrays on the device. */
typedef struct {
    int64_t num_dst;
    int64_t num_src;
    int64_t num_edges;
    const int64_t *row_ptr;
    const int32_t *col_idx;
} tiga_csr;

/* Reverse incidence of a tiga_csr (the transposed relation; Section 4.6
 * notes that source gradients accumulate over reverse incidence).
 *   src_ptr: int64 [num_src + 1]; source j owns slots [src_ptr[j], src_ptr[j+1]).
 *   edge_id: int32 [num_edges]; the forward edge position of each slot,
 *            ascending within a source (a stable transpose).
 * Built by tiga_csr_transpose; valid only for the unchanged topology (a
 * topology snapshot is fixed for derivatives, Section 3.2).  The struct lives
 * in HOST memory, the two arrays on the device. */
typedef struct {
    const int64_t *src_ptr;
    const int32_t *edge_id;
} tiga_csr_t;

/* ---------------------------------------------------------------- errors */

/* Message describing the last failure on the calling thread ("" if none).
 * Valid until the next library call on that thread.  Host pointer. */
const char *tiga_last_error(void);

/* TIGA_MP_ABI_VERSION of the built library. */
int tiga_mp_abi_version(void);

/* ------------------------------------------------------------ stored CSR */

/* Workspace bytes for tiga_mp_csr_fwd on this relation shape (0 on error). */
size_t tiga_mp_csr_fwd_workspace(const tiga_csr *rel, int32_t feat, int reducer);

/* Forward fused aggregation over a stored CSR relation (Section 3.1 equation,
 * Section 4.3 destination-major traversal, Section 4.4 bounded neighbour tiles
 * with a degree guard and a split of high-degree rows into partial states
 * merged afterwards):
 *   SUM: y[i,f] = sum_{e in row i} m_e[f]
 *   MAX: y[i,f] = max_{e in row i} m_e[f], argmax[i,f] = that e (lowest on ties)
 * with m_e = x_src[col[e], :] or w_edge[e] * x_src[col[e], :] (one fp32
 * multiply, so MAX values are exact products).
 *   x_src:  fp32 [num_src, feat];  w_edge: fp32 [num_edges] or NULL (see msg)
 *   y:      fp32 [num_dst, feat], overwritten
 *   argmax: int32 [num_dst, feat] for MAX (required), NULL for SUM
 * SUM results are deterministic (fixed reduction tree) but not bit-identical
 * to a serial sum; MAX results are exact.  MAX requires num_edges < 2^31.
 * Errors: TIGA_EINVAL, TIGA_EUNSUPPORTED, TIGA_EWORKSPACE, TIGA_EDEVICE. */
int tiga_mp_csr_fwd(const tiga_csr *rel, int32_t feat, const float *x_src, int msg,
                    const float *w_edge, int reducer, float *y, int32_t *argmax,
                    void *ws, size_t ws_bytes, void *stream);

/* Allocation-free tiga_mp_csr_fwd, for callers that cannot allocate device
 * memory (work under stream capture, tight serving loops, harnesses that
 * forbid allocation).  Same arguments, results and errors as tiga_mp_csr_fwd
 * without the workspace: the library keeps a fixed device array of
 * tiga_mp_csr_fwd_noalloc_limit() bytes (64 MiB) per device, taken from its
 * code object when this entry point is first called on that device and held
 * until the process ends.  A relation whose tiga_mp_csr_fwd_workspace exceeds
 * the limit is rejected with TIGA_EUNSUPPORTED before anything is enqueued.
 * The call makes no allocation (no hipMalloc, hipFree or allocating library
 * routine).  Every call on a device uses that device's one array: calls that
 * overlap on one device (other streams, other threads) race and must be
 * serialized by the caller; calls in order on one stream are safe.  The
 * device is the current device, and `stream` must belong to it. */
size_t tiga_mp_csr_fwd_noalloc_limit(void);
int tiga_mp_csr_fwd_noalloc(const tiga_csr *rel, int32_t feat, const float *x_src, int msg,
                            const float *w_edge, int reducer, float *y, int32_t *argmax,
                            void *stream);

/* Workspace bytes for tiga_mp_csr_fwd_paged with pages of at most page_edges
 * edges (0 on error).  Independent of the relation's size. */
size_t tiga_mp_csr_fwd_paged_workspace(int32_t feat, int reducer, int64_t page_edges);

/* tiga_mp_csr_fwd for a relation kept in HOST memory (Section 6, storage and
 * memory: the relation stays in a persistent store, one destination-row page
 * at a time is staged, and the kernel runs with a bounded device working set;
 * the output stays in device memory).
 *   rel_host: row_ptr and col_idx are HOST pointers (pinned memory lets the
 *             copies run asynchronously); w_host likewise (or NULL, see msg).
 *   x_src, y, argmax: DEVICE pointers, as in tiga_mp_csr_fwd.
 * Pages hold whole destination rows and at most page_edges edges; each page's
 * slices are copied on `stream` into the workspace and reduced there, so the
 * device working set is fixed by page_edges.  Results equal tiga_mp_csr_fwd's
 * (argmax holds global edge positions).  The host reads rel_host->row_ptr
 * during the call (to cut pages and to reject a row longer than page_edges
 * with TIGA_EUNSUPPORTED, or a row_ptr that does not run from 0 to num_edges
 * without decreasing with TIGA_EGRAPH); the host arrays must stay valid until
 * the stream has run the copies.
 * Errors: as tiga_mp_csr_fwd, plus TIGA_EGRAPH. */
int tiga_mp_csr_fwd_paged(const tiga_csr *rel_host, int32_t feat, const float *x_src, int msg,
                          const float *w_host, int reducer, float *y, int32_t *argmax, int64_t page_edges,
                          void *ws, size_t ws_bytes, void *stream);

/* Workspace bytes for tiga_mp_csr_bwd (0 on error). */
size_t tiga_mp_csr_bwd_workspace(const tiga_csr *rel, int32_t feat, int reducer);

/* Vector-Jacobian product of tiga_mp_csr_fwd (Section 5 weighted-sum adjoint):
 *   SUM: dx[j,f] = sum_{e: col[e]=j} w[e] dy[d(e),f];  dw[e] = sum_f x[col[e],f] dy[d(e),f]
 *   MAX: the same terms restricted to the selected edge e* = argmax[i,f] of
 *        each (i,f); argmax is the forward's output (required for MAX).
 * (w = 1 under TIGA_MSG_SRC.)  dx: fp32 [num_src, feat]; dw: fp32 [num_edges];
 * either may be NULL (skipped) and each is overwritten.  dw requires
 * TIGA_MSG_EDGE_SCALED_SRC.
 * rev == NULL: dx accumulates with device fp32 atomics: no set-up, summation
 *   order not fixed, and bound by the atomics (at feat = 64 a little over twice
 *   the time of the gather mode).
 * rev != NULL: dx is gathered over the reverse incidence (deterministic); build
 *   it once per topology with tiga_csr_transpose.  The destination row of
 *   each reverse slot is derived during the call from row_ptr and edge_id
 *   (into the workspace).
 * Errors: as tiga_mp_csr_fwd. */
int tiga_mp_csr_bwd(const tiga_csr *rel, const tiga_csr_t *rev, int32_t feat,
                    const float *x_src, int msg, const float *w_edge, int reducer,
                    const int32_t *argmax, const float *dy, float *dx, float *dw,
                    void *ws, size_t ws_bytes, void *stream);

/* Workspace bytes for tiga_csr_transpose (0 on error). */
size_t tiga_csr_transpose_workspace(const tiga_csr *rel);

/* Build the reverse incidence (see tiga_csr_t) with a stable sort by source:
 * within a source, edge ids ascend.  Topology set-up: build once per
 * unchanged topology.  src_ptr int64 [num_src+1] and edge_id int32
 * [num_edges], both overwritten.  Requires num_edges < 2^31. */
int tiga_csr_transpose(const tiga_csr *rel, int64_t *src_ptr, int32_t *edge_id,
                       void *ws, size_t ws_bytes, void *stream);

/* CSR validation (the paper's validate="full" and basic modes, Section 6.3):
 *   level 1: host-only metadata checks (sizes, pointers); enqueues nothing.
 *   level 2: additionally scans the device arrays: row_ptr[0] == 0,
 *            non-decreasing, row_ptr[num_dst] == num_edges, every col_idx in
 *            [0, num_src).  Synchronizes `stream`.
 * Returns TIGA_OK or TIGA_EGRAPH (the first violation is described by
 * tiga_last_error()). */
int tiga_csr_validate(const tiga_csr *rel, int level, void *stream);

/* -------------------------------------------------- generated radius relation */

/* Workspace bytes for tiga_mp_radius_fwd / _bwd / tiga_radius_neighbors on n
 * points with feat features (0 on error). */
size_t tiga_mp_radius_workspace(int64_t n, int32_t feat);

/* Forward over the radius relation generated from positions (Section 4.9:
 * a cell directory restricts candidates, an exact distance predicate accepts,
 * messages are consumed without storing accepted edges):
 *   N(i) = { j != i : d2(i,j) < fl(radius*radius) },
 *   d2   = fl(fl(fl(dx*dx) + fl(dy*dy)) + fl(dz*dz)), dx = fl(p_j.x - p_i.x), ...
 *   y_i  = sum_{j in N(i)} exp(-|p_i - p_j|^2 / sigma^2) x_j
 *   count_i = |N(i)|
 * The cell directory is rebuilt on every call (stateless).
 *   pos: fp32 [n, 3]; x: fp32 [n, feat]; y: fp32 [n, feat] (input order);
 *   count: int32 [n] or NULL.  reducer must be TIGA_REDUCE_SUM.
 *   feat == 0 computes the counts only (x and y may be NULL; count required):
 *   the first phase of tiga_radius_neighbors.
 * Requires n < 2^31, radius finite and > 0, sigma > 0 with 2 / sigma^2 finite
 * in fp32 (sigma >= 7.7e-20; TIGA_EINVAL otherwise).  A point with a non-finite
 * coordinate has no neighbours (every d2 involving it compares false). */
int tiga_mp_radius_fwd(int64_t n, int32_t feat, const float *pos, const float *x,
                       float radius, float sigma, int reducer, float *y, int32_t *count,
                       void *ws, size_t ws_bytes, void *stream);

/* VJP of tiga_mp_radius_fwd with membership held fixed (Section 5: radius
 * cutoff membership is discrete and not differentiated):
 *   dx_i = sum_{j in N(i)} k_ij dy_j
 *   dpos_i = sum_{j in N(i)} (2 k_ij / sigma^2) (p_j - p_i) (<dy_i, x_j> + <dy_j, x_i>)
 * with k_ij = exp(-|p_i - p_j|^2 / sigma^2).  dx: fp32 [n, feat] or NULL;
 * dpos: fp32 [n, 3] or NULL (x is only read when dpos is requested).
 * The same requirements as tiga_mp_radius_fwd. */
int tiga_mp_radius_bwd(int64_t n, int32_t feat, const float *pos, const float *x,
                       float radius, float sigma, const float *dy, float *dx, float *dpos,
                       void *ws, size_t ws_bytes, void *stream);

/* Accepted neighbour lists of the radius relation, ascending per point (the
 * relation a fused call consumes, exported for exact checking; the paper
 * resolves a generated relation to CSR for inspection, Section 4.9).  Two
 * phases: the counts come from tiga_mp_radius_fwd (feat 0 computes only
 * them), the caller forms nbr_ptr int64 [n+1] as their exclusive prefix sum,
 * and this call fills nbr_idx int32 [nbr_ptr[n]].
 *   nbr_ptr: device, read only.  Each point's list is written only inside its
 *            span [nbr_ptr[i], nbr_ptr[i+1]); if a span differs from that
 *            point's count the call returns TIGA_EINVAL (nothing is written
 *            outside the spans, the lists are then incomplete).
 * Synchronizes `stream`.  Not on the fused path: for tests and inspection. */
int tiga_radius_neighbors(int64_t n, const float *pos, float radius, const int64_t *nbr_ptr,
                          int32_t *nbr_idx, void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------- dense all-pairs relation */

/* Workspace bytes for tiga_mp_dense_fwd (0 on error). */
size_t tiga_mp_dense_workspace(int64_t n);

/* Dense all-pairs relation without an edge array (Section 1), softened
 * inverse-square message, sum reducer:
 *   y_i = sum_{j != i} q_j (p_j - p_i) / (|p_j - p_i|^2 + eps^2)^(3/2)
 * pos: fp32 [n, 3]; q: fp32 [n]; y: fp32 [n, 3].  reducer must be SUM.
 * Requires n < 2^31 and eps > 0. */
int tiga_mp_dense_fwd(int64_t n, const float *pos, const float *q, float eps, int reducer,
                      float *y, void *ws, size_t ws_bytes, void *stream);

/* ----------------------------------------------- generated exact kNN relation */

/* Workspace bytes for tiga_mp_knn_fwd on n points (0 on error). */
size_t tiga_mp_knn_workspace(int64_t n);

/* Forward over the exact k-nearest-neighbour relation generated from positions
 * (Section 4.9, generated relations: candidate tiles are scanned for each query
 * with a padded top-k state keyed by squared distance and source index; no
 * adjacency is stored), with the neighbour-sum message of the exact-kNN
 * workload of Section 7:
 *   S_i  = the k sources j != i with the smallest keys (d2_ij, j), compared
 *          lexicographically (a distance tie keeps the lower index); a source
 *          whose d2 is not finite is never selected, so S_i may hold fewer
 *          than k sources;
 *   d2   = fl(fl(fl(dx*dx) + fl(dy*dy)) + fl(dz*dz)), dx = fl(p_j.x - p_i.x), ...
 *   y_i  = sum_{j in S_i} x_j      (fp32; terms in key order, added sequentially
 *          above 7,168 points and by a fixed pairwise tree at or below)
 *   nbr[i][t] = the t-th selected source in key order, -1 past |S_i|.
 * The relation is rebuilt on every call (stateless).
 *   pos: fp32 [n, 3]; x: fp32 [n, feat] (NULL if feat == 0); y: fp32 [n, feat]
 *   (NULL if feat == 0); nbr: int32 [n, k] or NULL.  reducer must be
 *   TIGA_REDUCE_SUM.  Requires 0 <= k <= 32 (TIGA_EUNSUPPORTED above 32) and
 *   n < 2^31 - 64.  Selection is exact: it equals a full scan of all pairs.
 * Errors: TIGA_EINVAL, TIGA_EUNSUPPORTED, TIGA_EWORKSPACE, TIGA_EDEVICE. */
int tiga_mp_knn_fwd(int64_t n, int32_t feat, const float *pos, const float *x, int32_t k, int reducer, float *y,
                    int32_t *nbr, void *ws, size_t ws_bytes, void *stream);

/* -------------------------------- edge-local MLP message on the radius relation */

/* Workspace bytes for tiga_mp_edgenn_fwd / _bwd (0 on error). */
size_t tiga_mp_edgenn_workspace(int64_t n, int32_t feat, int32_t hidden, int32_t out);

/* Edge-local neural-network message summed over the generated radius relation
 * (appendix "A differentiable EdgeNN example"; the relation as in
 * tiga_mp_radius_fwd: j != i and the fp32 squared distance strictly below
 * fl(radius*radius)):
 *   in_ij = [p_j - p_i ; x_j]  (3 + feat values; fp32 differences)
 *   y_i   = sum_{j in N(i)} ( W2 max(W1 in_ij + b1, 0) + b2 )
 * (the final bias is part of every message; an empty row gives 0).  No edge,
 * message or hidden activation is stored.
 *   pos fp32 [n, 3]; x fp32 [n, feat] (NULL if feat == 0);
 *   W1 [hidden, 3 + feat], b1 [hidden], W2 [out, hidden], b2 [out] fp32
 *   row-major; y fp32 [n, out], overwritten.
 * Requires 0 <= feat <= 64, 1 <= hidden <= 64, 1 <= out <= 8
 * (TIGA_EUNSUPPORTED beyond), radius finite and > 0, n < 2^31 - 64.
 * Errors: TIGA_EINVAL, TIGA_EUNSUPPORTED, TIGA_EWORKSPACE, TIGA_EDEVICE. */
int tiga_mp_edgenn_fwd(int64_t n, int32_t feat, int32_t hidden, int32_t out, const float *pos, const float *x,
                       float radius, const float *W1, const float *b1, const float *W2, const float *b2, float *y,
                       void *ws, size_t ws_bytes, void *stream);

/* Vector-Jacobian product of tiga_mp_edgenn_fwd with the relation held fixed
 * (Section 5: radius membership is discrete and not differentiated); hidden
 * activations are recomputed, never stored.  For L = sum_i <dy_i, y_i>:
 *   dx [n, feat], dpos [n, 3], dW1 [hidden, 3 + feat], db1 [hidden],
 *   dW2 [out, hidden], db2 [out]   (fp32; each may be NULL; overwritten).
 * The derivative of max(a, 0) at a = 0 is 0.  Deterministic: fixed
 * summation orders for every output.  Arguments and errors as the forward. */
int tiga_mp_edgenn_bwd(int64_t n, int32_t feat, int32_t hidden, int32_t out, const float *pos, const float *x,
                       float radius, const float *W1, const float *b1, const float *W2, const float *b2,
                       const float *dy, float *dx, float *dpos, float *dW1, float *db1, float *dW2, float *db2,
                       void *ws, size_t ws_bytes, void *stream);

/* ------------------------------- online-softmax reducer (streaming attention) */

/* 16-bit input types of the attention path. */
enum tiga_dtype { TIGA_DT_F16 = 0 /* IEEE binary16 */, TIGA_DT_BF16 = 1 /* bfloat16 */ };

/* fp32, which only the rotary positions take besides. */
#define TIGA_DT_F32 2

/* Implicit relations of the attention path (no edge array). */
enum tiga_relation {
    TIGA_REL_TRIANGULAR = 0, /* N(i) = {0, ..., i}: causal, the diagonal included */
    TIGA_REL_DENSE = 1       /* N(i) = {0, ..., n-1} */
};

/* Online-softmax reducer over an implicit triangular or dense relation: the
 * streaming attention forward (appendix "Causal attention as message
 * passing"; reducer state of Section 5.2: running maximum, mass and
 * accumulator, combined by rescaling into a common maximum).  Per head h and
 * destination i, with the message (score, value) of source j:
 *   s_ij = scale * <q_i, k_j>,
 *   y_i  = sum_{j in N(i)} exp(s_ij) v_j / sum_{j in N(i)} exp(s_ij),
 *   lse_i = log sum_{j in N(i)} exp(s_ij).
 * No score or weight array is stored.
 *   q, k, v: [heads, n, width] head-major, 16-bit (dtype), 16-byte aligned
 *            (a permuted view of a contiguous (heads, n, width) allocation
 *            is the paper's logical (n, heads, width) tensor).
 *   y:       [heads, n, width] of dtype, overwritten (rounded to nearest even).
 *   lse:     fp32 [heads, n] or NULL.
 * Scores, weights and sums are fp32 (products of the 16-bit inputs are exact);
 * the weights enter both the value product and the mass rounded to dtype, so
 * y is an exactly normalized combination of the values and lse carries up to
 * one unit roundoff of dtype (2^-11 binary16, 2^-8 bfloat16) of absolute
 * error from that rounding.  Every row
 * is nonempty under both relations.  Requires width 64 or 128
 * (TIGA_EUNSUPPORTED otherwise), n < 2^31, heads * n < 2^40, scale finite and
 * > 0.  n == 0 or heads == 0 enqueues nothing.  Needs no workspace.
 * Errors: TIGA_EINVAL, TIGA_EUNSUPPORTED, TIGA_EDEVICE. */
int tiga_mp_attention_fwd(int64_t n, int32_t heads, int32_t width, int dtype, const void *q, const void *k,
                          const void *v, float scale, int relation, void *y, float *lse, void *stream);

/* ------------------- online softmax over a rectangular relation (cross attention) */

/* A strided view of a [batch, heads, rows, width] tensor: element (b, h, r, d)
 * is data[b * batch + h * head + r * row + d] (strides in elements, the width
 * contiguous).  The struct lives in HOST memory, the data on the device.  A
 * stride of 0 repeats an input along that axis; outputs must not overlap. */
typedef struct {
    void *data;
    int64_t batch, head, row;
} tiga_view;

/* The dense relation between num_dst destinations (queries) and num_src sources
 * (keys and values: an encoder's states, a document's) of each sequence of a
 * padded batch.  Destination head h reads source head h / (heads / kv_heads).
 *   src_len: device int32 [batch], the sources of each sequence,
 *            N(b, i) = {0, ..., src_len[b] - 1}; NULL: num_src for all.  A value
 *            outside [0, num_src] is taken as the nearer bound.
 * The struct lives in HOST memory. */
typedef struct {
    int64_t num_dst, num_src;
    int32_t batch, heads, kv_heads, width;
    int32_t dtype; /* TIGA_DT_F16 or TIGA_DT_BF16 */
    const int32_t *src_len;
} tiga_cross;

/* Workspace bytes for tiga_mp_attention_cross_fwd (0 on error; at most about
 * 36 MB).  One sized for a relation holds every smaller one. */
size_t tiga_mp_attention_cross_fwd_workspace(const tiga_cross *rel);

/* The online-softmax reducer of tiga_mp_attention_fwd over a rectangular
 * relation: for sequence b, head h and destination i,
 *   s_ij = scale * <q_i, k_j>,  lse_i = log sum_{j in N(b,i)} exp(s_ij),
 *   y_i  = sum_{j in N(b,i)} exp(s_ij - lse_i) v_j.
 * A destination without sources (src_len[b] == 0) finalizes the reducer's
 * identity: y = 0, lse = -inf.  Sources at and past src_len[b] are not read.
 *   q, y: [batch, heads, num_dst, width];  k, v: [batch, kv_heads, num_src, width]
 *         of dtype, 16-byte aligned, strides multiples of 8, head and row strides
 *         below 2^31 (row strides of k and v below 2^23); y is overwritten.
 *   lse:  fp32 [batch, heads, num_dst], contiguous, or NULL.
 * A value that is not finite reaches the rows that see it, as an infinity or NaN.
 * Products of the inputs are exact and summed in fp32; the mass is the fp32 sum
 * of the fp32 weights; the weights enter the value product rounded to dtype.
 * Deterministic.  Requires width 64 or 128 (TIGA_EUNSUPPORTED otherwise), heads
 * a multiple of kv_heads, num_src and num_dst * heads / kv_heads < 2^31 - 1024,
 * batch * heads * num_dst < 2^40, batch * kv_heads < 2^20, scale finite and > 0.
 * Errors: TIGA_EINVAL, TIGA_EUNSUPPORTED, TIGA_EWORKSPACE, TIGA_EDEVICE. */
int tiga_mp_attention_cross_fwd(const tiga_cross *rel, const tiga_view *q, const tiga_view *k, const tiga_view *v,
                                float scale, const tiga_view *y, float *lse, void *ws, size_t ws_bytes, void *stream);

/* Workspace bytes for tiga_mp_attention_cross_bwd (0 on error): about 34 MB and
 * 8 bytes a destination row and head.  One sized for a relation holds every
 * smaller one. */
size_t tiga_mp_attention_cross_bwd_workspace(const tiga_cross *rel);

/* Vector-Jacobian product of tiga_mp_attention_cross_fwd.  With the forward's y
 * and lse, p_ij = exp(s_ij - lse_i) and delta_i = <dy_i, y_i> (formed as
 * sum_j p_ij <dy_i, v_j> where a sequence's sources fit a tile, at most 128 of
 * width 64 or 64 of width 128, over which y's rounding would matter):
 *   ds_ij = p_ij (<dy_i, v_j> - delta_i)
 *   dq_i = scale sum_j ds_ij k_j;  dk_j = scale sum_i ds_ij q_i;  dv_j = sum_i p_ij dy_i
 * where the sums over i also run over the heads that share source head j's.
 * Gradients of sources at and past src_len[b] are 0.
 *   dy: as y; dq as q, dk and dv as k and v, of dtype, overwritten; each may be
 *   NULL (skipped).  p and ds enter the products rounded to dtype (binary16: as
 *   scaled by powers of two that bring the largest ones near its largest number,
 *   which a pass over v and dy finds); sums in fp32.
 * Deterministic (no atomics).  Requirements and errors as the forward; besides, at
 * most 2^24 - 1 tiles of 128 sources, or rows of a source head, over all batch *
 * kv_heads, TIGA_EUNSUPPORTED otherwise. */
int tiga_mp_attention_cross_bwd(const tiga_cross *rel, const tiga_view *q, const tiga_view *k, const tiga_view *v,
                                const tiga_view *y, const float *lse, const tiga_view *dy, float scale,
                                const tiga_view *dq, const tiga_view *dk, const tiga_view *dv, void *ws,
                                size_t ws_bytes, void *stream);

/* --------------------------------------- causal attention of packed sequences */

/* Sequences of different lengths packed along one axis of num_rows rows (tokens):
 * sequence b is rows [ptr[b], ptr[b + 1]), ptr device int32 [batch + 1],
 * non-decreasing, within [0, num_rows] (a value outside is taken as the nearer
 * bound).  Row i reads its sequence's rows up to itself, N(i) = {ptr[b], ..., i};
 * head h of the queries reads head h / (heads / kv_heads) of the keys and values.
 * The struct lives in HOST memory. */
typedef struct {
    int64_t num_rows;
    int32_t batch, heads, kv_heads, width;
    int32_t dtype; /* TIGA_DT_F16 or TIGA_DT_BF16 */
    const int32_t *ptr;
} tiga_packed;

/* Workspace bytes for tiga_mp_attention_packed_fwd (0 on error; at most about
 * 70 MB and 67 KB a head).  One sized for a call holds every smaller one. */
size_t tiga_mp_attention_packed_fwd_workspace(const tiga_packed *rel);

/* The online-softmax reducer over the triangular relation of every packed
 * sequence with itself, otherwise as tiga_mp_attention_cross_fwd.
 *   q, y: [1, heads, num_rows, width];  k, v: [1, kv_heads, num_rows, width] (the
 *         views' batch strides are not used), requirements as there; y is
 *         overwritten and must not overlap the inputs.
 *   lse:  fp32 [heads, num_rows], contiguous, or NULL.
 * Rows of no sequence (before ptr[0], behind ptr[batch]) see nothing: y = 0,
 * lse = -inf; what they hold is not read.  A row takes nothing from rows after it
 * or of other sequences, whatever they hold.  Deterministic.
 * Requires width 64 or 128, heads a multiple of kv_heads, num_rows * heads <
 * 2^31 - 1024, batch < 2^20, scale finite and > 0.
 * Errors: TIGA_EINVAL, TIGA_EUNSUPPORTED, TIGA_EWORKSPACE, TIGA_EDEVICE. */
int tiga_mp_attention_packed_fwd(const tiga_packed *rel, const tiga_view *q, const tiga_view *k, const tiga_view *v,
                                 float scale, const tiga_view *y, float *lse, void *ws, size_t ws_bytes, void *stream);

/* Workspace bytes for tiga_mp_attention_packed_bwd (0 on error): about 8 bytes a
 * row and head, and from some hundred rows on up to about 135 MB and 0.2 MB a head
 * for parts of long sequences.  One sized for a call holds every smaller one. */
size_t tiga_mp_attention_packed_bwd_workspace(const tiga_packed *rel);

/* Vector-Jacobian product of tiga_mp_attention_packed_fwd, from its y and lse;
 * formulas, arguments and roundings as tiga_mp_attention_cross_bwd (delta formed
 * as sum_j p_ij <dy_i, v_j> for the rows of a tile of 128 whose last row sees at
 * most 128 tokens).  Gradients of rows of no sequence are 0.  Nothing reaches other
 * sequences.  A query or cotangent that is not finite reaches its own dq and the dk,
 * dv of the tokens that it sees; a key or value the dq of the rows that see it, and
 * by way of those rows the dk, dv of what they see.
 * P and ds enter the products rounded to the input type: two roundings of half a
 * step, which few tokens do not average out.
 * Deterministic (no atomics).  Requirements and errors as the forward; besides, at
 * most 2^24 - 1 tiles of 128 rows (heads / kv_heads to a token), counted over all
 * source heads, with one more for each sequence and a few for parts. */
int tiga_mp_attention_packed_bwd(const tiga_packed *rel, const tiga_view *q, const tiga_view *k, const tiga_view *v,
                                 const tiga_view *y, const float *lse, const tiga_view *dy, float scale,
                                 const tiga_view *dq, const tiga_view *dk, const tiga_view *dv, void *ws,
                                 size_t ws_bytes, void *stream);

/* ----------------------------------------------------------- rotary positions */

/* How the elements of a row pair up (rot elements from the front take part). */
enum tiga_pairs {
    TIGA_PAIRS_HALF = 0,    /* (i, i + rot / 2) */
    TIGA_PAIRS_ADJACENT = 1 /* (2 i, 2 i + 1) */
};

/* The rotation of a row at position p: pair i = (a, b) becomes
 *   amplitude * (a cos t - b sin t, a sin t + b cos t),  t = p * freq[i].
 * The struct lives in HOST memory. */
typedef struct {
    const double *freq; /* device fp64 [rot / 2], radians a position */
    int32_t rot;        /* even, 0 < rot <= width; elements past it are copied */
    int32_t pairs;      /* tiga_pairs */
    float amplitude;
} tiga_rotary;

/* How tiga_rotary_frequencies stretches the frequencies for contexts `factor`
 * times the trained length. */
enum tiga_rotary_scaling {
    TIGA_ROTARY_PLAIN = 0,  /* f_i = base^(-2 i / rot) */
    TIGA_ROTARY_LINEAR = 1, /* f_i / factor (positions interpolated) */
    TIGA_ROTARY_BASE = 2,   /* f_i of base * factor^(rot / (rot - 2)) */
    TIGA_ROTARY_BANDS = 3   /* by the turns r = trained f_i / 2 pi over the trained length: f_i / factor
                               where r <= low, f_i where r >= high, in between the two weighted linearly */
};

/* Fill the HOST array freq [rot / 2].  trained, low and high only matter for
 * TIGA_ROTARY_BANDS (low < high).  Enqueues nothing. */
int tiga_rotary_frequencies(int32_t rot, double base, int scaling, double factor, double trained, double low,
                            double high, double *freq);

/* Rotate every row of x [batch, heads, rows, width] by its position into y
 * (y == x, same strides, rotates in place; y must not overlap x otherwise).
 *   dtype: TIGA_DT_F16, TIGA_DT_BF16 or TIGA_DT_F32; x, y strides any.
 *   pos:   device int32, the position of row (b, r) at pos[b * pos_batch + r]
 *          (pos_batch 0 shares one row of positions); NULL: r itself.
 * The angle is formed and reduced in fp64, sine and cosine in fp32, the
 * rotation in fp32, rounded once.  Elements past rot are copied unchanged.
 * Requires width < 2^16, batch * heads * rows < 2^40, amplitude finite.
 * Errors: TIGA_EINVAL, TIGA_EUNSUPPORTED, TIGA_EDEVICE. */
int tiga_mp_rotary_fwd(int32_t batch, int32_t heads, int64_t rows, int32_t width, int dtype, const tiga_view *x,
                       const int32_t *pos, int64_t pos_batch, const tiga_rotary *rot, const tiga_view *y,
                       void *stream);

/* Vector-Jacobian product of tiga_mp_rotary_fwd: dy turned back by the same
 * angles into dx, with the same amplitude.  Arguments as the forward. */
int tiga_mp_rotary_bwd(int32_t batch, int32_t heads, int64_t rows, int32_t width, int dtype, const tiga_view *dy,
                       const int32_t *pos, int64_t pos_batch, const tiga_rotary *rot, const tiga_view *dx,
                       void *stream);

/* ------------------------------------------------- attention over a paged cache */

/* Keys and values of a batch of sequences in pages.  Position p of sequence b
 * lies in row p % page_size of page table[b * table_width + p / page_size].
 *   k, v:   views [num_pages, kv_heads, page_size, width] (batch is the page
 *           stride) of dtype, 16-byte aligned, strides multiples of 8, row
 *           strides below 2^23.
 *   table:  device int32 [batch, table_width]; entries past a sequence's length
 *           are not read.
 *   length: device int32 [batch], positions of each sequence, the new ones of a
 *           call included.
 * Sequences may share pages that no call writes.  page_size is a power of two,
 * at most 2^15.  The struct lives in HOST memory. */
typedef struct {
    int64_t num_pages;
    int32_t page_size, kv_heads, width;
    int32_t dtype; /* TIGA_DT_F16 or TIGA_DT_BF16 */
    int32_t batch, table_width;
    tiga_view k, v;
    const int32_t *table;
    const int32_t *length;
} tiga_cache;

/* The new tokens of a call are rows of one packed axis: sequence b owns rows
 * [dst_ptr[b], dst_ptr[b + 1]), dst_ptr device int32 [batch + 1], non-decreasing,
 * dst_ptr[batch] <= num_dst, and row dst_ptr[b] + t, of c = dst_ptr[b + 1] -
 * dst_ptr[b], is at position length[b] - c + t.
 *
 * tiga_cache_validate checks dst_ptr, length and the table entries that the
 * lengths need on the host and describes the first violation (TIGA_EGRAPH).
 * Synchronizes `stream`; not on the serving path. */
int tiga_cache_validate(const tiga_cache *cache, int64_t num_dst, const int32_t *dst_ptr, void *stream);

/* Store the new tokens' keys and values in their pages: k rotated by its position
 * (rot != NULL) and v unchanged.  With q, the queries of the same tokens are
 * rotated by the same positions into q_out in the same launch (rot required;
 * q_out may be q).
 *   k, v: [1, kv_heads, num_dst, width]; q, q_out: [1, heads, num_dst, width] of
 *   the cache's dtype (the views' batch strides are not used).
 * Rows before dst_ptr[0], and rows whose position is negative or past the
 * table, or whose page is not in [0, num_pages), store nothing; their q is
 * rotated by the position where there is one, and copied unrotated where there
 * is none (before dst_ptr[0], negative).  Rows behind dst_ptr[batch] store
 * nothing, and their q_out is left as it was.
 * No two rows of one call may fall on the same place of a page.
 * Errors: TIGA_EINVAL, TIGA_EUNSUPPORTED, TIGA_EDEVICE. */
int tiga_mp_cache_append(const tiga_cache *cache, int64_t num_dst, const int32_t *dst_ptr, const tiga_view *k,
                         const tiga_view *v, const tiga_rotary *rot, int32_t heads, const tiga_view *q,
                         const tiga_view *q_out, void *stream);

/* Workspace bytes for tiga_mp_attention_paged_fwd (0 on error; at most about
 * 36 MB).  One sized for a call holds every smaller one. */
size_t tiga_mp_attention_paged_fwd_workspace(const tiga_cache *cache, int64_t num_dst, int32_t heads);

/* Causal attention of the new tokens over the cache, their own keys and values
 * already in it: the row at position p of sequence b reads positions 0..p,
 * N(b, p) = {0, ..., p}, otherwise as tiga_mp_attention_cross_fwd.  One token a
 * sequence (generation), chunks of prompts, or both mixed.
 *   q, y: [1, heads, num_dst, width] (the views' batch strides are not used);
 *   y may be q (same strides).  lse: fp32 [heads, num_dst] or NULL.
 * A row with a negative position gives y = 0, lse = -inf.  A row that needs a
 * position past the table or a page outside [0, num_pages) gives NaN (nothing
 * is read there).  Rows before dst_ptr[0] and behind dst_ptr[batch] are left as
 * they were.
 * Requires heads a multiple of kv_heads, width 64 or 128, num_dst * heads <
 * 2^31 - 1024, table_width * page_size < 2^31 - 1024,
 * batch < 2^16, scale finite and > 0.
 * Errors: TIGA_EINVAL, TIGA_EUNSUPPORTED, TIGA_EWORKSPACE, TIGA_EDEVICE. */
int tiga_mp_attention_paged_fwd(const tiga_cache *cache, int64_t num_dst, const int32_t *dst_ptr, int32_t heads,
                                const tiga_view *q, float scale, const tiga_view *y, float *lse, void *ws,
                                size_t ws_bytes, void *stream);

/* Groups of neighbouring sequences of a cache whose first positions hold the same
 * keys and values (a system prompt, a document): sequences [ptr[g], ptr[g + 1])
 * share their positions below len[g].
 *   ptr, len: device int32 [groups + 1] (non-decreasing, within [0, batch]; a value
 *   outside is taken as the nearer bound) and [groups].  Sequences of no group
 *   share nothing.
 * Whether the sequences' tables name the same pages or copies does not matter: the
 * shared positions are read from the pages of a group's first sequence, with or
 * without new tokens (as many as it has, rounded down to a multiple of the page size
 * and of 128; the rest, and groups of one sequence, from each sequence's own).  The
 * struct lives in HOST memory. */
typedef struct {
    int32_t groups;
    const int32_t *ptr;
    const int32_t *len;
} tiga_prefix;

/* tiga_cache_validate, and that ptr and len are in range and no sequence with new
 * tokens has its first one below its group's len (TIGA_EGRAPH), also where the call
 * would read no position once or fewer than len (groups of one; rounding), whose
 * results are right.  That the shared positions hold the same is not looked at.
 * Synchronizes `stream`. */
int tiga_prefix_validate(const tiga_cache *cache, const tiga_prefix *prefix, int64_t num_dst, const int32_t *dst_ptr,
                         void *stream);

/* Workspace bytes for tiga_mp_attention_prefix_fwd (0 on error): at most about 72 MB
 * and 8 (width + 1) bytes a row and head.  One sized for a call holds every smaller
 * one. */
size_t tiga_mp_attention_prefix_fwd_workspace(const tiga_cache *cache, const tiga_prefix *prefix, int64_t num_dst,
                                              int32_t heads);

/* tiga_mp_attention_paged_fwd with the shared positions of each group read once for
 * all of its rows.  The results are those of the paged call but for the order of
 * the sums; a sequence whose first new token is among the positions that are read
 * once (as above: rounded down, none of a group of one) gives NaN.  Arguments,
 * requirements and errors as there. */
int tiga_mp_attention_prefix_fwd(const tiga_cache *cache, const tiga_prefix *prefix, int64_t num_dst,
                                 const int32_t *dst_ptr, int32_t heads, const tiga_view *q, float scale,
                                 const tiga_view *y, float *lse, void *ws, size_t ws_bytes, void *stream);

/* --------------------------------------------- which positions of a cache stay */

/* A weight belongs to a cell of a page and rows move from page to page, so here every
 * page is one sequence's, and named once: sequences that begin alike have the shared
 * positions in copies (which tiga_mp_attention_prefix_fwd reads once a group all the
 * same).  With a page that two name, their sums overwrite each other, and an
 * eviction in place moves one's rows over the other's.  The calls do not look; this
 * one does, on the host, at the pages of every sequence's positions (entries that
 * are no page are passed over): TIGA_EGRAPH names a page and two that name it.
 * Synchronizes `stream`. */
int tiga_retention_validate(const tiga_cache *cache, void *stream);

/* Workspace bytes for tiga_mp_cache_weights (0 on error).  One sized for a call
 * holds every smaller one. */
size_t tiga_mp_cache_weights_workspace(const tiga_cache *cache, int64_t num_dst, int32_t heads);

/* Add the attention weights that a call's new tokens give to the positions of the
 * cache, from the queries and the lse of tiga_mp_attention_paged_fwd (or _prefix_
 * _fwd): with s_ij = scale <q_i, k_j>, for every sequence, source head and position
 * j below the sequence's length,
 *   out_j = decay * weights_j + sum_i exp(s_ij - lse_i)
 * over the new tokens i that see j, of every head that shares the source head;
 * weights_j counts as 0 at the new tokens' own positions, whatever lies there.
 *   q:   as for tiga_mp_attention_paged_fwd;  lse: fp32 [heads, num_dst].
 *   weights, out: fp32 [num_pages, kv_heads, page_size], contiguous, the cells of
 *   the cache's pages; out may be weights.  Cells of no position are left as they
 *   were.  No page may be named twice (tiga_retention_validate).
 * A row with lse = -inf gives nothing.  Positions past the table or without a page
 * have no cell.  Sums in fp32 in a fixed order; deterministic.  Requires decay
 * finite and >= 0; otherwise as tiga_mp_attention_paged_fwd.
 * Errors: TIGA_EINVAL, TIGA_EUNSUPPORTED, TIGA_EWORKSPACE, TIGA_EDEVICE. */
int tiga_mp_cache_weights(const tiga_cache *cache, int64_t num_dst, const int32_t *dst_ptr, int32_t heads,
                          const tiga_view *q, const float *lse, float scale, float decay, const float *weights,
                          float *out, void *ws, size_t ws_bytes, void *stream);

/* Workspace bytes for tiga_mp_cache_evict (0 on error): little; for tables of more
 * than 32,768 positions 10 KB to 8192 positions of at most 256 sequences and heads;
 * in place (to is cache) the rows that stay.  One sized for a call holds every
 * smaller one. */
size_t tiga_mp_cache_evict_workspace(const tiga_cache *cache, const tiga_cache *to, int32_t keep);

/* Keep the `keep` positions of each sequence and source head with the largest
 * weights: the last `recent` positions, and of the others those of the largest
 * weights, of equal ones the first.  They move, in order, to the first positions of
 * the same sequence and head of `to`: keys, values, weights, and lengths.
 *   weights:    fp32 [num_pages, kv_heads, page_size] of cache; NaN counts as more
 *               than everything, a position without a page as less.
 *   to:         a cache of the same batch, kv_heads, width and dtype, whose length
 *               array is not read; its pages are none that cache's tables name, or
 *               it is cache itself (the same table and k.data): in place.
 *   to_weights: fp32 [to->num_pages, kv_heads, to->page_size] or NULL; in place it
 *               may be weights.
 *   to_length:  int32 [batch], min(length, keep); may be cache's length array.
 *   kept:       int32 [batch, kv_heads, keep], the positions that stayed, in order,
 *               -1 past them.
 * Keys that were rotated keep the rotation of the position they had.  Positions past
 * cache's table are none; rows whose new position has no page in `to`, or whose old
 * one had none, are not stored.  Nothing else is written.  No page of `to` may be
 * named twice (tiga_retention_validate), in place none of the cache; another cache's
 * may be read by several.  Deterministic.
 * Requires 1 <= keep, 0 <= recent <= keep, batch * kv_heads < 2^20.
 * Errors: TIGA_EINVAL, TIGA_EUNSUPPORTED, TIGA_EWORKSPACE, TIGA_EDEVICE. */
int tiga_mp_cache_evict(const tiga_cache *cache, const float *weights, int32_t keep, int32_t recent,
                        const tiga_cache *to, float *to_weights, int32_t *to_length, int32_t *kept, void *ws,
                        size_t ws_bytes, void *stream);

/* ------------------------------------------------------------- profiling */

/* Profiling aid.  Arms the calling thread so that its next entry-point call
 * records hipEvent `start` on its stream immediately before, and `stop`
 * immediately after, the launch of that call's dominant kernel (the one that
 * streams the edges or pairs).  The events (hipEvent_t passed as void*) stay
 * owned by the caller and must live until that call returns.  The arming is
 * consumed by that one call; a call without a fused kernel (transpose,
 * validation, neighbour lists) records nothing and drops it.  Passing NULL for
 * both disarms.  Returns TIGA_OK. */
int tiga_mp_set_kernel_events(void *start, void *stop);

#ifdef __cplusplus
}
#endif

#endif /* TIGA_MP_H */
