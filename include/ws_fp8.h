/*
 * ws_fp8.h -- C ABI of the 8-bit path for AMD MI355X (gfx950): quantisation by
 * blocks, the block-scaled matrix product, and its forms for groups of rows.
 *
 * Format: codes are OCP e4m3 (1 sign, 4 exponent, 3 fraction bits, largest
 * value 448, no infinity, NaN 0x7f).  A scale is a power of two in 8 bits
 * (E8M0: byte b stands for 2^(b - 127)) and belongs to 128 values along the
 * contraction (a row's columns), of one row or of 128 rows.  Powers of two,
 * because scaling by them rounds nothing and the matrix instruction of gfx950
 * applies them itself.
 *
 * A quantised matrix (ws_fp8_matrix) has rows of codes, `ld` bytes apart, and
 * scales[b * ld_scales + r / block_rows] for columns 128 b .. 128 b + 127 of
 * row r.  Columns are padded to a multiple of 16 with zero codes.
 *
 * Quantisation of a block: amax is the largest finite |x| in it, the scale is
 * the smallest power of two s with amax <= 448 s (1 for amax = 0; at least
 * 2^-127), and a code is x / s rounded to nearest even.  Infinities and NaN
 * become NaN codes and leave their block's other values alone.
 *
 * Every call only enqueues work on `stream` (0: the null stream of the current
 * device), allocates nothing, synchronises nothing and may be captured into a
 * graph.  All pointers are device pointers of the device current at the call,
 * owned by the caller, apart from the descriptors, which are read before the
 * call returns.  Sizes of zero are valid; what an empty operand would hold may
 * be NULL.  Errors are ws_status values as in ws_gemm.h.
 *
 * Sizes: rows, columns and elements between rows up to 2^30, groups up to 2^20.
 * Quantisation with the transpose, and of weights: fewer than 2^24 tiles of 128 x
 * 128, all groups or matrices of a batch together.  Products: rows of A and B at
 * most 2^22 bytes apart, so that contractions have at most 2^22 columns (for
 * ws_fp8_grouped_gradient: padded rows), and at most 2^31 tiles of 64 x 64
 * results.
 */
#ifndef WS_FP8_H
#define WS_FP8_H

#include "ws_gemm.h"

#ifdef __cplusplus
extern "C" {
#endif

#define WS_FP8_BLOCK 128

/* A matrix in 8 bits (see above).  With `batch` above 1, `batch` matrices of
 * the same size, stride_codes and stride_scales bytes apart (weights of
 * experts).  A call on single matrices takes 0 as 1; where a batch is taken, 0 is
 * an empty one. */
typedef struct {
  void* codes;            /* 16-byte aligned */
  uint8_t* scales;
  int64_t rows, cols;
  int64_t ld;             /* bytes between rows: a multiple of 16, at least cols rounded up to 16 */
  int64_t ld_scales;      /* bytes between the scales of neighbouring column blocks:
                             at least ceil(rows / block_rows) */
  int32_t block_rows;     /* rows that share a scale: 1 or 128 */
  int32_t batch;
  int64_t stride_codes;   /* a multiple of 16; matrices do not overlap */
  int64_t stride_scales;
} ws_fp8_matrix;

/* An operand or result in 16 or 32 bits: element type ws_out_dtype, `ld`
 * elements between rows.  Aligned to its elements; any ld of at least the
 * row's length. */
typedef struct {
  void* data;
  int64_t rows, cols, ld;
  int32_t dtype;
  int32_t batch;
  int64_t stride;         /* elements between matrices of a batch, which do not overlap */
} ws_matrix;

/* Scales of 1 x 128.  out has x's columns and out->rows rows: row r is row
 * index[r] of x (a negative or too large index: a row of zeros), or row r for
 * index NULL (then out->rows == x->rows).  Memory bound: one read of x, one
 * write of the codes. */
ws_status ws_fp8_quantize_rows(const ws_matrix* x, const int32_t* index, const ws_fp8_matrix* out,
                               hipStream_t stream);

/* The same, and from the same read the columns: the quantised transpose of the
 * (gathered) matrix, with scales for 1 x 128 along the rows of x.  out_columns
 * has x's columns as rows.
 *
 * groups == 0: out_columns->cols == out_rows->rows.
 * groups > 0: offsets[0 .. groups] (device, not decreasing, within 0 ..
 * out_rows->rows) cut the rows into groups, and every group's columns start at
 * a multiple of 128 in out_columns: those of group g at the sum of the earlier
 * groups' row counts, each rounded up to 128.  out_columns->cols ==
 * 128 * ws_fp8_padded_blocks(rows, groups); codes of no row are zero, their
 * scales 1.  Rows in no group, before the first or after the last, are zeros in
 * out_rows. */
ws_status ws_fp8_quantize_both(const ws_matrix* x, const int32_t* index, int32_t groups,
                               const int32_t* offsets, const ws_fp8_matrix* out_rows,
                               const ws_fp8_matrix* out_columns, hipStream_t stream);

/* Blocks of 128 that hold the padded groups of `rows` rows, whatever the
 * offsets: (rows + 127 min(groups, rows)) / 128, or for groups == 0 ceil(rows / 128). */
int64_t ws_fp8_padded_blocks(int64_t rows, int32_t groups);

/* Scales of 128 x 128, of w and, where out_transposed is not NULL, of its
 * transpose (the same codes and scales). */
ws_status ws_fp8_quantize_weight(const ws_matrix* w, const ws_fp8_matrix* out,
                                 const ws_fp8_matrix* out_transposed, hipStream_t stream);

/* A part of a product: the tile it is computed in and the stages of its ring of
 * blocks of 128 columns in LDS (0: operands go straight to registers), the launch
 * that computes it (0, or 1 for a second one behind it), and the rows of the result. */
typedef struct {
  int32_t tile_m, tile_n, stages, launch;
  int64_t rows;
} ws_fp8_kernel_info;

/* The parts of a product M x N x K with results of out_dtype, by rising rows
 * (2 at the most).  groups > 0: of ws_fp8_grouped_product, or with depth != 0 of
 * ws_fp8_grouped_gradient of K rows.  Host only; kernels are chosen by sizes and
 * type alone, for the current device's compute units (256 without a device). */
ws_status ws_fp8_plan(int64_t M, int64_t N, int64_t K, int32_t out_dtype, int32_t groups, int32_t depth,
                      ws_fp8_kernel_info* out, int32_t* count);

/* C <- alpha A B^T + beta C0: A is M x K (block_rows 1), B is N x K (block_rows
 * 1 or 128), C and C0 are M x N of the same type; rounded once, from the sums
 * below.  C0 may be C itself, and NULL with beta == 0 (then it is not read).  K
 * may be 0.
 *
 * Precision: a result in 32 bits has products and sums in binary32 (operand
 * values below 2^-126 or of 2^128 and more count as 0 and infinity).  For a
 * result in 16 bits the 8-bit matrix instruction of gfx950 is used, at twice the
 * rate, and its sums hold fewer bits: it adds each eight neighbouring products
 * with 13 bits below the largest one's leading bit, cuts what lies below, and
 * adds their sums in binary32.  That is 1.5e-5 of the result (in norm) on normal
 * values, 4.6e-5 where one column in a hundred is 20 times larger, and 2^-10 of
 * the sum of magnitudes at the very most, beside the rounding's own 1.7e-3 to
 * bf16 and 2.1e-4 to f16.  Sums in binary32 for a result in 16 bits: ask for 32
 * bits and round them.
 *
 * The three products of a linear layer Y = X W^T: X (rows) and W (weight);
 * dX = dY W with dY (rows) and the transposed weight; dW = dY^T X with the
 * columns of both.
 *
 * Results do not depend on anything but the operands and sizes: no atomics. */
ws_status ws_fp8_product(const ws_fp8_matrix* A, const ws_fp8_matrix* B, float alpha, float beta,
                         const ws_matrix* C0, const ws_matrix* C, hipStream_t stream);

/* Rows by group: row r of C is row r of A times B_g^T, for the group g whose
 * rows offsets[g] .. offsets[g + 1] - 1 hold r; rows in no group, before the first
 * or after the last, become zeros.
 * B is a batch of `groups` matrices; offsets as above.  C <- alpha A B^T. */
ws_status ws_fp8_grouped_product(const ws_fp8_matrix* A, const ws_fp8_matrix* B, int32_t groups,
                                 const int32_t* offsets, float alpha, const ws_matrix* C,
                                 hipStream_t stream);

/* Their weight gradient: C_g <- alpha A_g B_g^T + beta C0_g, contracted over
 * group g's rows.  A (M x P) and B (N x P) are columns of `rows` rows as
 * ws_fp8_quantize_both lays them out, P = 128 ws_fp8_padded_blocks(rows,
 * groups); C is a batch of `groups` matrices M x N. */
ws_status ws_fp8_grouped_gradient(const ws_fp8_matrix* A, const ws_fp8_matrix* B, int64_t rows,
                                  int32_t groups, const int32_t* offsets, float alpha, float beta,
                                  const ws_matrix* C0, const ws_matrix* C, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* WS_FP8_H */
