/*
 * ws_orthogonal.h -- C ABI of orthogonalised updates for AMD MI355X (gfx950).
 *
 * A weight's update whose directions count alike: for a gradient (or momentum) G,
 *   X = G / |G|  (Frobenius; zeros where G is zero), then `steps` times
 *   X <- a X + (b A + c A^2) X with A = X X^T,
 *   (a, b, c) = (3.4445, -4.7750, 2.0315),
 * which takes every singular value s of X to a s + b s^3 + c s^5: five steps bring
 * those above 0.01 to 0.7 .. 1.2, and the result near U V^T of G = U S V^T.
 *
 * Precision: how far the result is from the exact iteration (in norm), before it is
 * rounded to bf16, which costs 1.7e-3. A shorter side up to 64 and up to six steps: below
 * 1e-4 (five) and 4e-4 (six), by way of A in binary64. Longer ones: products are of
 * binary16 values with sums in binary32. What the steps amplify is kept apart from what is
 * rounded: X as the sum of two binary16 values, the diagonals of A and of a + b A + c A^2
 * in binary32. A shorter side up to 384, or more than five steps of any: all operands are
 * such sums, as good as binary32: below 2e-4 after five steps, 5e-4 after six, 2e-3 after
 * more. Shorter sides over 384 up to five steps: operands of one binary16 value; 2e-4 to
 * 9e-4 where directions are alike or fall off evenly, up to 1.5e-3 where one stands out,
 * up to 2.4e-3 (over 512: 1.8e-3) where a quarter to half of them stands out over a rest
 * of 1/1000. The same matrix in another batch may round otherwise. A matrix with an
 * infinity or NaN becomes NaN.
 *
 * Calls, pointers, sizes and errors as in ws_fp8.h.
 */
#ifndef WS_ORTHOGONAL_H
#define WS_ORTHOGONAL_H

#include "ws_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

#define WS_ORTHOGONAL_STEPS 100   /* at the most */
#define WS_ORTHOGONAL_SIDE 65536  /* rows and columns, at the most */

/* Bytes of device memory that ws_orthogonalize needs for a batch of matrices (0: none,
 * then workspace may be NULL); -1 for sizes that it refuses. */
int64_t ws_orthogonal_workspace(int64_t rows, int64_t cols, int32_t batch);

/* out (bf16) <- the orthogonalised G (f32, bf16 or f16), each matrix of the batch for
 * itself; of the same sizes, out may not overlap G.  The workspace (256-byte aligned) is
 * written before it is read; calls on other streams need another.  Results depend on
 * G and the sizes only: no atomics. */
ws_status ws_orthogonalize(const ws_matrix* G, int32_t steps, const ws_matrix* out, void* workspace,
                           int64_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* WS_ORTHOGONAL_H */
