/*
 * mg_experts.h  --  C ABI of the 8-bit products and of the routing of mixture-of-experts layers.
 *
 * Same library and conventions as mg_gemm.h: device pointers owned by the caller, nothing allocated, copied to the host or
 * synchronised, every call only enqueues kernels on `stream`, arguments are checked on the host before any GPU work and
 * errors are negative status codes.  Device contents (offsets, indices, scales) are not checked, but an index outside its
 * range is never followed out of the arrays.  Extents of zero return MG_OK without launching anything unless said otherwise.
 * Except for MG_COL_MAJOR in mg_block_gemm, matrices are row-major: element (r, c) at X[r*ld + c].
 *
 * 8-bit matrices.  An element is an e4m3 number (OCP: sign, 4 bits of exponent, 3 of mantissa; largest 448, no infinity,
 * 0x7F = NaN), one byte.  Each block of 128 consecutive elements of a row (MG_BLOCK_ROW) or of 128 x 128 elements
 * (MG_BLOCK_SQUARE) has one FP32 scale; blocks start at row 0 and column 0, the last ones may be shorter.  An element
 * stands for its 8-bit value times its block's scale.  Scales are row-major with a leading dimension of their own:
 * (row blocks) rows x ceil(cols/128), (square blocks) ceil(rows/128) x ceil(cols/128).
 *
 * MG_ERR_DIM also covers what the kernels' 32-bit counts and a launch cannot hold: extents from 2^31 - 1024 on, 2^21 blocks of 128 x 128
 * of a matrix that is quantised and more than 2^20 of a product's C (2^35 and 2^34 elements; blocks that are not full count, so that a
 * single row counts as 128, and one more row of blocks for every expert), and of the rows that are routed more than 2^31 pieces of four
 * elements and 2^24 tokens.
 *
 * A kernel may read an aligned 16-byte piece of memory whole when at least one of its bytes belongs to an operand.
 */
#ifndef MG_EXPERTS_H
#define MG_EXPERTS_H

#include "mg_gemm.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    MG_ERR_TYPE = -20,        /* element type is none of MG_F32, MG_F16, MG_BF16                            */
    MG_ERR_BLOCK = -21,       /* block form or kind of scales unknown                                      */
    MG_ERR_GROUPS = -22,      /* groups or experts outside 1 .. MG_MOST_GROUPS, or fan outside 1 .. MG_MOST_FAN */
    MG_ERR_SCALES = -23       /* leading dimension of scales smaller than the number of blocks of a row    */
};

enum { MG_BF16 = 2 };                                             /* beside MG_F32 and MG_F16: bfloat16 */
typedef enum { MG_BLOCK_ROW = 151, MG_BLOCK_SQUARE = 152 } mg_block;
/* MG_SCALES_POW2: the caller states that every scale of both operands is a normal power of two (as mg_block_quantize
 * makes them): the scales then go into the matrix instructions as exponents, or into the exponents of the elements, whose
 * values have to be finite FP32 numbers then (below 2^-126 they may count as zero).  Other scales given under it may count as
 * the power of two below them, or as they are: that depends on the kernel. */
typedef enum { MG_SCALES_ANY = 161, MG_SCALES_POW2 = 162 } mg_scales;
/* May be added (|) to either: sums as of FP32 products whatever the type of C, as C in FP32 gets them anyway.
 * Without it C in 16 bits is not summed in FP32 throughout, but on the FP8 matrix pipes, twice as fast: they add eight neighbouring products
 * at a time on a grid of 2^-13 of the largest of the eight, towards zero (these sums, and all else, then in FP32).  That is an error of about
 * 1.5e-5 of the result for normal data, 5e-5 with outliers, whatever the length of the sum; where all terms have one sign it is a bias (measured,
 * of the sum of magnitudes: -2.5e-6 for |normal| data, -9.5e-6 for squares of a rectifier's output, -6e-5 where the terms spread over
 * exp(2 normal)).  The whole error of C, its rounding included: bfloat16 1.6612e-3 of the norm where FP32 sums have 1.6604e-3, FP16 2.13e-4 where
 * they have 2.08e-4.  The largest loss there can be is 2^-10 of the sum of magnitudes. */
enum { MG_SUMS_FP32 = 1 << 16 };
#define MG_MOST_GROUPS 1024
#define MG_MOST_FAN 64

/* ---- quantising ------------------------------------------------------------------------------------------------------
 * X (rows x cols of `dtype`: MG_F32, MG_F16 or MG_BF16) -> 8-bit matrix and scales.  Two results, each optional (Q and S
 * NULL together, T and ST NULL together, not both pairs):
 *   Q, S    X itself: rows x cols;
 *   T, ST   its transpose: cols x rows, blocks along ITS rows (MG_BLOCK_ROW: a block is 128 consecutive rows of one column
 *           of X) - the operand of a product that sums over the rows of X.
 * A block's scale is the smallest power of two, 2^-126 at least, with which the block's largest finite magnitude is at
 * most 448 (1 for a block without a finite non-zero element); elements are divided by it, which is exact, and rounded to
 * the nearest e4m3 number, ties to even.  Infinities and NaN become NaN.
 * Errors: MG_ERR_DIM, MG_ERR_LDA (ldx), MG_ERR_LDB (ldq), MG_ERR_LDC (ldt), MG_ERR_NULL, MG_ERR_TYPE, MG_ERR_BLOCK, MG_ERR_SCALES. */
mg_status mg_block_quantize(int dtype, int block, int64_t rows, int64_t cols, const void *X, int64_t ldx,
                            uint8_t *Q, int64_t ldq, float *S, int64_t lds, uint8_t *T, int64_t ldt, float *ST, int64_t ldst,
                            void *stream);
/* The same for `batch` matrices (the weights of all experts), matrix b at X + b*stride_x and so on; strides in elements,
 * >= 0 (MG_ERR_STRIDE), batch >= 0 (MG_ERR_BATCH; at most 65535). */
mg_status mg_block_quantize_batched(int dtype, int block, int64_t batch, int64_t rows, int64_t cols,
                                    const void *X, int64_t ldx, int64_t stride_x,
                                    uint8_t *Q, int64_t ldq, int64_t stride_q, float *S, int64_t lds, int64_t stride_s,
                                    uint8_t *T, int64_t ldt, int64_t stride_t, float *ST, int64_t ldst, int64_t stride_st,
                                    void *stream);
/* Rows that belong to `groups` experts: rows offsets[e] .. offsets[e+1]-1 are expert e's (device array of groups + 1
 * ascending counts from 0 to at most `rows`, as mg_expert_sort writes it).  Row r of the result is row source[r]/fan of X
 * (source: device array of `rows` slots, or NULL: row r of X; X then has `rows` rows).  Row blocks.  Q, S: rows x cols.
 * T, ST: the transpose, cols x mg_grouped_columns(rows, groups): expert e's rows start at column
 * 128*ceil(offsets[e]/128) + 128*e, so that every expert has blocks of its own; the columns between its last row and the
 * end of its last block are written as zeros, other columns are not written.  Rows from offsets[groups] on are not written.
 * Errors: as above and MG_ERR_GROUPS. */
mg_status mg_block_quantize_grouped(int dtype, int groups, const int32_t *offsets, int64_t rows, int64_t cols,
                                    const void *X, int64_t ldx, const int32_t *source, int fan,
                                    uint8_t *Q, int64_t ldq, float *S, int64_t lds, uint8_t *T, int64_t ldt, float *ST, int64_t ldst,
                                    void *stream);
/* 128*ceil(rows/128) + 128*groups: columns of a transposed result of mg_block_quantize_grouped (-1 for invalid arguments) */
int64_t mg_grouped_columns(int64_t rows, int groups);

/* ---- product of two 8-bit matrices -----------------------------------------------------------------------------------
 *     C = alpha * A * B^T + beta * C        C(i,j): sum over blocks b of sa(i,b) * sb(j,b) * sum over l in b of A(i,l) * B(j,l)
 * A m x k, B n x k, both with the summed index contiguous in memory; C m x n of c_type (MG_F32, MG_F16, MG_BF16), stored as
 * `layout` says (column-major: element (i, j) at C[i + j*ldc]).  How it is summed follows from c_type and MG_SUMS_FP32 (above): FP32 throughout for
 * C in FP32 or with the flag, on the FP8 pipes' grid otherwise; one rounding to c_type.  alpha, beta: host scalars;
 * beta == 0: C is not read; alpha == 0 or k == 0: A and B are not read.
 * workspace (256-byte aligned, may be NULL): with mg_block_gemm_workspace_bytes() few outputs with long sums run as slices
 * that a second launch adds; with less, in fewer slices: same result up to summation order.
 * Operands whose rows start on 16 bytes (pointer and leading dimension) take the fastest kernels.
 * Errors: MG_ERR_LAYOUT, MG_ERR_DIM, MG_ERR_LDA, MG_ERR_LDB, MG_ERR_LDC, MG_ERR_NULL, MG_ERR_TYPE, MG_ERR_BLOCK, MG_ERR_SCALES. */
mg_status mg_block_gemm(int layout, int64_t m, int64_t n, int64_t k, float alpha, int scales,
                        int a_block, const uint8_t *A, int64_t lda, const float *SA, int64_t ldsa,
                        int b_block, const uint8_t *B, int64_t ldb, const float *SB, int64_t ldsb,
                        float beta, int c_type, void *C, int64_t ldc, void *workspace, size_t workspace_bytes, void *stream);
size_t mg_block_gemm_workspace_bytes(int64_t m, int64_t n, int64_t k);

/* ---- the experts' products -------------------------------------------------------------------------------------------
 * Row r of C (rows x n, row-major), offsets[e] <= r < offsets[e+1]:
 *     C(r,:) = alpha * A(source[r]/fan, :) * B[e]^T + beta * C(r,:)
 * A with row blocks (source NULL: row r of A itself), B[e] n x k at B + e*stride_b, its scales at SB + e*stride_sb.  Rows of C
 * from offsets[groups] on are not touched.  With B[e] holding an expert's transposed weights this is the gradient of its input.
 * Errors: as mg_block_gemm, MG_ERR_GROUPS, MG_ERR_STRIDE. */
mg_status mg_block_gemm_grouped(int groups, const int32_t *offsets, int64_t rows, int64_t n, int64_t k, float alpha, int scales,
                                const uint8_t *A, int64_t lda, const float *SA, int64_t ldsa, const int32_t *source, int fan,
                                int b_block, const uint8_t *B, int64_t ldb, int64_t stride_b, const float *SB, int64_t ldsb, int64_t stride_sb,
                                float beta, int c_type, void *C, int64_t ldc, void *workspace, size_t workspace_bytes, void *stream);
size_t mg_block_gemm_grouped_workspace_bytes(int groups, int64_t rows, int64_t n, int64_t k);
/* For every expert e, C[e] (m x n at C + e*stride_c):
 *     C[e] = alpha * sum over its rows r of A(:,r) * B(:,r)^T + beta * C[e]
 * A (m x columns) and B (n x columns): transposed results of mg_block_quantize_grouped with their scales (row blocks); an
 * expert without rows gets beta * C[e].  The gradient of the experts' weights.  Errors: as above. */
mg_status mg_block_gemm_grouped_sum(int groups, const int32_t *offsets, int64_t rows, int64_t m, int64_t n, float alpha, int scales,
                                    const uint8_t *A, int64_t lda, const float *SA, int64_t ldsa,
                                    const uint8_t *B, int64_t ldb, const float *SB, int64_t ldsb,
                                    float beta, int c_type, void *C, int64_t ldc, int64_t stride_c,
                                    void *workspace, size_t workspace_bytes, void *stream);
size_t mg_block_gemm_grouped_sum_workspace_bytes(int groups, int64_t rows, int64_t m, int64_t n);

/* ---- routing ---------------------------------------------------------------------------------------------------------
 * Slot t*fan + j is token t's j-th choice of an expert, ids[slot] (device, tokens x fan, dense).  Sorting writes
 *   offsets[experts + 1]   expert e's rows are offsets[e] .. offsets[e+1] - 1;
 *   position[slot]         the slot's row, or -1 where ids[slot] is not in 0 .. experts-1 (a dropped slot);
 *   source[row]            the row's slot, slots of one expert in ascending order; -1 from offsets[experts] on.
 * The workspace is required: mg_expert_sort_workspace_bytes() bytes, 256-byte aligned (MG_ERR_WORKSPACE); 0 for calls that one
 * work-group sorts.  No tokens: offsets are written, nothing else.
 * Errors: MG_ERR_DIM (tokens*fan beyond 2^30), MG_ERR_NULL, MG_ERR_WORKSPACE, MG_ERR_GROUPS. */
mg_status mg_expert_sort(int64_t tokens, int fan, int experts, const int32_t *ids, int32_t *offsets, int32_t *position, int32_t *source,
                         void *workspace, size_t workspace_bytes, void *stream);
size_t mg_expert_sort_workspace_bytes(int64_t tokens, int fan, int experts);
/* Y(r,:) = weights[source[r]] * X(source[r]/fan, :) for all tokens*fan rows; weights: FP32 device array of tokens*fan, or NULL: 1;
 * rows whose source is negative become zeros.  X: tokens x cols, Y: tokens*fan x cols, both of `dtype`. */
mg_status mg_expert_gather(int dtype, int64_t tokens, int fan, int64_t cols, const void *X, int64_t ldx, const int32_t *source,
                           const float *weights, void *Y, int64_t ldy, void *stream);
/* O(t,:) = sum over j of weights[t*fan+j] * Y(position[t*fan+j], :), dropped slots left out (a token without any gets zeros),
 * summed in FP32 in the order of j, rounded once.  weights NULL: 1 - the gradient of an unweighted mg_expert_gather. */
mg_status mg_expert_combine(int dtype, int64_t tokens, int fan, int64_t cols, const void *Y, int64_t ldy, const int32_t *position,
                            const float *weights, void *O, int64_t ldo, void *stream);
/* Gradient of mg_expert_combine:  dY(position[s],:) = weights[s] * dO(t,:),  dweights[s] = sum over c of dO(t,c) * Y(position[s],c)
 * (FP32; 0 for dropped slots).  Rows of dY that no slot has are not written.  dY or dweights may be NULL (Y then, too, if it is
 * dweights).  Errors of these three: MG_ERR_DIM, MG_ERR_LDA/LDB/LDC (of the matrices in their order), MG_ERR_NULL, MG_ERR_TYPE, MG_ERR_GROUPS. */
mg_status mg_expert_combine_grad(int dtype, int64_t tokens, int fan, int64_t cols, const void *dO, int64_t lddo, const void *Y, int64_t ldy,
                                 const int32_t *position, const float *weights, void *dY, int64_t lddy, float *dweights, void *stream);

#ifdef __cplusplus
}
#endif
#endif
