/*
 * ws_experts.h -- C ABI of the routing of tokens to experts and back for AMD
 * MI355X (gfx950).
 *
 * A router gives each of `tokens` tokens k expert ids.  A slot is one such
 * choice, number t * k + j.  Sorting puts the slots of expert 0 first, in slot
 * order, then those of expert 1, and so on; a slot whose id lies outside
 * 0 .. experts - 1 (a masked token: -1) has no place.
 *   offsets[e]  first sorted row of expert e (offsets[experts]: their number)
 *   token[r]    the token of sorted row r; -1 past offsets[experts]
 *   place[t][j] the sorted row of slot (t, j), or -1
 *
 * Calls, pointers and errors as in ws_fp8.h.  Indices read from device memory
 * are checked where they are used: one out of range counts as none.
 */
#ifndef WS_EXPERTS_H
#define WS_EXPERTS_H

#include "ws_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

#define WS_MAX_EXPERTS 1024

/* Bytes of device memory that ws_expert_sort needs (0: none, then workspace may
 * be NULL); -1 for sizes that it refuses. */
int64_t ws_expert_sort_workspace(int64_t tokens, int32_t k, int32_t experts);

/* ids: tokens x k, int32 (id_bytes 4) or int64 (id_bytes 8), dense.  At most
 * 2^30 slots and WS_MAX_EXPERTS experts.  offsets: experts + 1; token and
 * place: tokens * k.  The workspace (4-byte aligned) is written before it is
 * read; calls on other streams need another. */
ws_status ws_expert_sort(int64_t tokens, int32_t k, int32_t experts, const void* ids, int32_t id_bytes,
                         int32_t* offsets, int32_t* token, int32_t* place, void* workspace,
                         int64_t workspace_bytes, hipStream_t stream);

/* out[place[t][j]] = x[t]: the tokens' rows in sorted order; rows past
 * offsets[experts] are zeros, places out of range are left out.  x and out of one
 * type; out does not overlap x.  place as ws_expert_sort leaves it: below
 * offsets[experts], no row twice. */
ws_status ws_expert_gather(const ws_matrix* x, int32_t k, int32_t experts, const int32_t* offsets, const int32_t* place,
                           const ws_matrix* out, hipStream_t stream);

/* out[t] = sum over j of weights[t][j] h[place[t][j]] (weights NULL: 1), in
 * binary32 in the order of j, rounded once; places out of range are left out.
 * The gradient of ws_expert_gather is this without weights.  weights: dense
 * binary32.  h and out of one type. */
ws_status ws_expert_combine(const ws_matrix* h, int32_t k, const int32_t* place, const float* weights,
                            const ws_matrix* out, hipStream_t stream);

/* Gradient of ws_expert_combine: dh[place[t][j]] = weights[t][j] dy[t], rows
 * past offsets[experts] zero, and dweights[t][j] = dot(dy[t], h[place[t][j]])
 * in binary32, 0 for a place out of range.  weights NULL: 1; dweights NULL: not
 * computed (then h may be NULL).  dy, h and dh of one type; dh may not overlap
 * h or dy.  place as ws_expert_sort leaves it. */
ws_status ws_expert_combine_gradient(const ws_matrix* dy, const ws_matrix* h, int32_t k, int32_t experts,
                                     const int32_t* offsets, const int32_t* place, const float* weights,
                                     const ws_matrix* dh, float* dweights, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* WS_EXPERTS_H */
