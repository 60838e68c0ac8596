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
#define WS_MAX_CHOICES 32

/* Bytes of device memory that ws_expert_choose needs (0: none, then workspace may
 * be NULL); -1 for sizes that it refuses. */
int64_t ws_expert_choose_workspace(int64_t tokens, int32_t experts, int32_t k);

/* A router's choice for logits l (tokens x experts), with p its softmax over the
 * experts:
 *   ids[t][j]      the token's k largest logits, the largest first, the lowest
 *                  index first among equals (both zeros are equal, NaN is the
 *                  largest); a logit of -inf is not chosen: -1 where none is left
 *   weights[t][j]  softmax over the token's choices, 0 for a place without one
 *   counts[e]      choices of expert e; counts[experts]: tokens with a choice
 *   loss           experts * sum over e of counts[e] / choices * mean of p[t][e],
 *                  the mean over tokens with a choice; 0 without any: 1 where the
 *                  experts are chosen alike, up to experts where one is
 * A NaN among a token's logits makes its weights, and so the loss, NaN; so does
 * +inf.  k up to experts and WS_MAX_CHOICES, experts up to WS_MAX_EXPERTS, at most
 * 2^30 choices.  weights and ids: tokens * k, dense; counts: experts + 1; all
 * 4-byte aligned.  Exponentials and sums in binary32 or more; results do not depend
 * on anything but logits and sizes.  The workspace (8-byte aligned) is written
 * before it is read; calls on other streams need another. */
ws_status ws_expert_choose(const ws_matrix* logits, int32_t k, float* weights, int32_t* ids, int32_t* counts,
                           float* loss, void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* Its gradient, from those of weights (dense; NULL: zeros, then weights and ids may
 * be NULL) and of loss (one value; NULL: zero), counts taken for constants:
 *   dlogits[t][e] = w[j] (dw[j] - sum over i of w[i] dw[i])  where e is choice j of t
 *     + dloss experts / (choices tokens_with_one) p[t][e] (counts[e] - sum over i of counts[i] p[t][i])
 * rounded once to the type of logits; dlogits may be logits.  weights, ids and counts
 * as ws_expert_choose leaves them; an id out of range counts as none. */
ws_status ws_expert_choose_gradient(const ws_matrix* logits, int32_t k, const float* dweights, const float* dloss,
                                    const float* weights, const int32_t* ids, const int32_t* counts,
                                    const ws_matrix* dlogits, hipStream_t stream);

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
