/*
 * ws_fp4.h -- C ABI of weights in 4 bits for AMD MI355X (gfx950): rounding by
 * blocks, the way back, and products of a few rows with such weights.
 *
 * Format: codes are OCP e2m1 (1 sign, 2 exponent, 1 fraction bit: 0, 0.5, 1, 1.5,
 * 2, 3, 4, 6 and their negatives).  A scale is a power of two in 8 bits (E8M0: byte
 * b stands for 2^(b - 127), 255 for NaN) and belongs to 32 neighbouring columns of a
 * row.  Powers of two, as in ws_fp8.h: scaling by them rounds nothing, and gfx950
 * widens codes to bf16 with the scale in one instruction, exactly.
 *
 * A matrix in 4 bits (ws_fp4_matrix) lies in tiles of 16 rows by 128 columns, so that
 * a product reads 1 KiB of codes and 64 bytes of scales in one piece each: rows padded to
 * a multiple of 16 and columns to one of 128, with zero codes and scales of 1.  Tile j
 * of 16 rows i has its codes at codes + i * ld + 1024 j: byte 256 g + 16 r + 4 k + b
 * holds columns 32 k + 8 g + 2 b (low half) and 32 k + 8 g + 2 b + 1 (high half) of the
 * tile's row r; g, k and b go from 0 to 3 (a lane's 16 bytes are its operands of four
 * matrix instructions).  Its scales are at scales + i * ld_scales + 64 j: byte 4 r + k
 * for columns 32 k .. 32 k + 31 of row r.
 *
 * Rounding of a block: amax is its largest |x|, the scale is the smallest power of two s
 * with amax <= 6 s (1 for amax = 0; at least 2^-127; at most 2^125, whose multiples
 * binary32 holds), and a code is x / s rounded to nearest, ties to the code with an
 * even last bit, above 6 to 6.  A block with an infinity or NaN
 * gets a NaN scale: its values are gone.
 *
 * Calls, pointers, sizes and errors as in ws_fp8.h.
 */
#ifndef WS_FP4_H
#define WS_FP4_H

#include "ws_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

#define WS_FP4_BLOCK 32

typedef struct {
  void* codes;            /* 16-byte aligned */
  uint8_t* scales;        /* 4-byte aligned */
  int64_t rows, cols;
  int64_t ld;             /* bytes between 16 rows and the next: a multiple of 16, at least 1024 ceil(cols / 128) */
  int64_t ld_scales;      /* the same of scales: a multiple of 4, at least 64 ceil(cols / 128) */
  int32_t batch;          /* matrices of one size (weights of experts); 0 as in ws_fp8_matrix */
  int64_t stride_codes;   /* between them: a multiple of 16; they do not overlap */
  int64_t stride_scales;  /* a multiple of 4 */
} ws_fp4_matrix;

/* out <- w (f32, bf16 or f16; (a batch of) rows x cols, of the same sizes). */
ws_status ws_fp4_quantize(const ws_matrix* w, const ws_fp4_matrix* out, hipStream_t stream);

/* out (f32 or bf16) <- the values of q, exactly (bf16: from 2^-126 up). */
ws_status ws_fp4_dequantize(const ws_fp4_matrix* q, const ws_matrix* out, hipStream_t stream);

/* out[r][j] <- the scale of columns 32 j .. 32 j + 31 of row r: rows x ceil(cols / 32)
 * bytes, `ld` between rows, `stride` between matrices of a batch. */
ws_status ws_fp4_scales(const ws_fp4_matrix* q, uint8_t* out, int64_t ld, int64_t stride, hipStream_t stream);

/* Bytes of device memory that a product of M rows, N columns and K contracted ones needs
 * (0: none, then workspace may be NULL; so for up to 16 rows, of a group on average), in
 * `groups` groups or -1 for ws_fp4_product; -1 for sizes that it refuses. */
int64_t ws_fp4_product_workspace(int64_t M, int64_t N, int64_t K, int32_t groups);

/* C <- A B^T: B is N x K in 4 bits; C (f32, bf16 or f16) is M x N; its row m is row
 * index[m] of A (a negative or too large index: a row of zeros), or row m for index
 * NULL (then A has M rows).  A is bf16 or f16, K columns.  Products and sums in
 * binary32, rounded once (bf16: operand values below 2^-126 count as 0).  Made for
 * the rows of a decoding step: the weights are read once for every 16 to 64 rows.  Results
 * depend on the operands and sizes only: no atomics.  The workspace (16-byte aligned) is
 * written before it is read; calls on other streams need another. */
ws_status ws_fp4_product(const ws_matrix* A, const int32_t* index, const ws_fp4_matrix* B, const ws_matrix* C,
                         void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* The same by group: row r of C is its row of A times B_g^T, for the group g whose
 * rows offsets[g] .. offsets[g + 1] - 1 hold r (int32 on the device, not decreasing);
 * rows in no group, before the first or after the last, become zeros.  B is a batch of
 * `groups` matrices. */
ws_status ws_fp4_grouped_product(const ws_matrix* A, const int32_t* index, const ws_fp4_matrix* B, int32_t groups,
                                 const int32_t* offsets, const ws_matrix* C, void* workspace, int64_t workspace_bytes,
                                 hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* WS_FP4_H */
