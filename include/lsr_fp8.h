/*
 * lsr_fp8.h - C ABI of the head's dense logits in 8-bit floating point: the same H, W and bias as lsr_head.h, every operand held as e4m3
 * values times a power of two for each block of 128, for serving and for training.
 *
 *   lsr_fp8_quantize   values to e4m3 blocks, by rows, transposed, or both
 *   lsr_fp8_matmul     logits
 *   lsr_fp8_backward   gradients of the hidden states, the matrix and the bias from those of the logits
 *
 * The conventions of lsr_head.h and lsr_distill.h hold for every entry point: device pointers owned by the caller, a caller-owned
 * workspace whose size the library states, work enqueued on `stream` without a synchronisation, every check on the host before
 * anything is enqueued, a status as the return value, no state kept, outputs overwritten.  All calls can be recorded into a HIP
 * graph.  Pointers are 16-byte aligned where nothing else is said.  Arrays are row-major; a leading dimension (ld) counts elements from
 * one row to the next.
 *
 * A block of values x is held as bytes q (e4m3: 4 bits of exponent, 3 of mantissa, largest value 448, no infinities) and one exponent e:
 *   e = the smallest whole number >= -127 with max |x| <= 448 2^e over the block's finite values;   q = x / 2^e rounded to nearest, ties to even
 * Dividing by 2^e is exact and nothing saturates.  An infinity or a NaN is held as the NaN of e4m3, and whatever is multiplied by it shows it.
 * The exponents of a matrix of `rows` rows are bytes e + 127, those of four blocks of a row beside each other:
 *   exps[(b / 4) rows 4 + row 4 + b % 4] belongs to columns 128 b .. 128 b + 127 of the row          (4 rows ceil(cols / 512) bytes in all;
 * bytes of blocks behind the last are not looked at.)  So an exponent can be a row's own, or the same for 128 rows.
 */
#ifndef LSR_FP8_H
#define LSR_FP8_H

#include "lsr_head.h"

#ifdef __cplusplus
extern "C" {
#endif

/* An element type beside LSR_F32 and LSR_BF16: e4m3 values with exponents as above. */
#define LSR_E4M3 3

/*
 * Bytes of a row of `cols` e4m3 values, a multiple of 128; of the exponents of a matrix; and of a matrix laid out by slab (all 0 where out of range):
 * 256 rows of 64 bytes behind each other, then the next 64 columns of the same rows, so that what a tile of a product reads at a time lies in one
 * piece however long the rows are.  Byte c of row r is byte ((r / 256) (lsr_fp8_row_bytes(cols) / 64) + c / 64) 16384 + (r % 256) 64 + c % 64.
 */
int64_t lsr_fp8_row_bytes(int64_t cols);
int64_t lsr_fp8_exp_bytes(int64_t rows, int64_t cols);
int64_t lsr_fp8_slab_bytes(int64_t rows, int64_t cols);

/*
 * X [rows, ldx] x_dtype (LSR_F32 or LSR_BF16), any alignment of its elements, ldx >= cols, to one or both of
 *   Q  [rows, ldq], exps    blocks of 1 x 128 along the rows: operands whose contracted axis is the columns
 *   Qt [cols, ldqt], exps_t X transposed, blocks along the rows of X: operands whose contracted axis is the rows
 * With `square` not 0 a block is 128 x 128 of X, and Qt is Q transposed.  ldq and ldqt are multiples of 16, at least lsr_fp8_row_bytes(cols)
 * and (rows); bytes behind the end of a row are set to zero up to there, and not touched behind that.  ldqt = 0: Qt by slab (rows behind the last of the
 * last 256 are not touched).  Either pair may be NULL.
 * The exponents are laid out as said above (for exps_t with `cols` rows), 4-byte aligned.
 * Limits: 1 <= rows, cols <= 2^22, rows cols < 2^36.
 */
int lsr_fp8_quantize(int64_t rows, int64_t cols, int32_t x_dtype, const void* X, int64_t ldx, int32_t square,
                     uint8_t* Q, int64_t ldq, uint8_t* exps, uint8_t* Qt, int64_t ldqt, uint8_t* exps_t, lsr_stream_t stream);

/*
 * out[n,v] = sum_k A[n,k] W[v,k] + bias[v], of the values that the operands stand for.
 *   a_dtype   LSR_E4M3: A [N, lda] bytes as lsr_fp8_quantize writes Q (zero from K to lsr_fp8_row_bytes(K)), lda a multiple of 16, a_exps its exponents.
 *             LSR_F32 or LSR_BF16: A [N, lda] values, any alignment of its elements, lda >= K, held in blocks of 1 x 128 within the call
 *             exactly as by lsr_fp8_quantize; a_exps must be NULL.
 *   W         [V, ldw] bytes, w_exps as lsr_fp8_quantize writes them (square or not)
 *   bias      [V] f32, or NULL for none
 *   out       [N, ldo] out_dtype (LSR_F32 or LSR_BF16), any alignment of its elements, ldo >= V
 *   workspace lsr_fp8_matmul_workspace_bytes (0 for LSR_E4M3: then it may be NULL; 0 also for an invalid shape)
 * For LSR_F32 results products are exact and sums are float32, in an order that does not depend on N: a row's results have the same bits whatever rows are beside it.
 * For LSR_BF16 results of up to 24 rows (fewer where K is above 1536: N rows of 2 K + 16 bytes, K up to a multiple of 128, are at most 76 KB) the same sums are rounded.
 * From there on the matrix cores add products in small groups, in which what lies more than 13 bits below the largest is cut off: 2e-5 of the norm of the sums on normal
 * values (5e-5 where magnitudes spread over 2^8), under a rounding of 1.7e-3.  So a row's bfloat16 results in a call of few rows and in one of many may be a rounding apart.
 * A value of A or W below 2^-126 may count as zero; one above 1.9375 2^127 rounds to 2^128, which may count as infinite.  Exponents and bias are 4-byte aligned.
 * Limits: 1 <= N, V <= 2^22, N V < 2^36, 1 <= K <= 65536, ldw and the lda of bytes at most 2^23.
 */
size_t lsr_fp8_matmul_workspace_bytes(int64_t N, int64_t V, int64_t K, int32_t a_dtype);

int lsr_fp8_matmul(int64_t N, int64_t V, int64_t K, int32_t a_dtype, int32_t out_dtype,
                   const void* A, int64_t lda, const uint8_t* a_exps,
                   const uint8_t* W, int64_t ldw, const uint8_t* w_exps, const float* bias,
                   void* out, int64_t ldo,
                   void* workspace, size_t workspace_bytes, lsr_stream_t stream);

/*
 * The same logits of a matrix that is a parameter, as a training step forms them: W [V, ldw] and H [N, ldh] of h_dtype (LSR_F32 or LSR_BF16), any alignment of their
 * elements, W held in blocks of 128 x 128 and H in blocks of 1 x 128 within the call.
 *   Wt [D, ldwt], wt_exps: what lsr_fp8_backward takes of the matrix, as lsr_fp8_quantize writes Qt (square; ldwt = 0 by slab), or NULL for no dH
 *   out, bias: as above; the results are the bits of lsr_fp8_quantize and lsr_fp8_matmul.
 * Limits: 1 <= N, V <= 2^22, 1 <= D <= 65536, N V, N D and V D < 2^36.
 */
size_t lsr_fp8_forward_workspace_bytes(int64_t N, int64_t V, int64_t D);

int lsr_fp8_forward(int64_t N, int64_t V, int64_t D, int32_t h_dtype, int32_t out_dtype,
                    const void* H, int64_t ldh, const void* W, int64_t ldw, const float* bias,
                    void* out, int64_t ldo, uint8_t* Wt, int64_t ldwt, uint8_t* wt_exps,
                    void* workspace, size_t workspace_bytes, lsr_stream_t stream);

/*
 * Gradients of sum dY . (q(H) q(W)^T + bias), the rounding of the operands passed over (its derivative taken as one):
 *   dH[n,:] = sum_v q(dY)[n,v] q(W)[v,:]     dY in blocks of 1 x 128 along its rows, W as it was multiplied
 *   dW[v,:] = sum_n qt(dY)[n,v] qt(H)[n,:]   both in blocks of 128 x 1 along their columns (the tokens)
 *   db[v]   = sum_n dY[n,v]                  of the values as given
 *   dY [N, ldy] y_dtype, H [N, ldh] h_dtype (each LSR_F32 or LSR_BF16), any alignment of their elements
 *   Wt [D, ldwt], wt_exps: W transposed as lsr_fp8_quantize leaves Qt and exps_t (square), with ldwt = 0 by slab, which is faster
 *   dH [N, D], dW [V, D] of h_dtype, contiguous; db [V] f32; each may be NULL to skip it.  H is needed for dW alone, Wt for dH alone.
 * Sums are formed as in lsr_fp8_matmul (exact products and float32 sums where h_dtype is LSR_F32), over cuts of the contracted axis where there are
 * few tiles, joined in float32 in a fixed order and rounded once.  Results are the same bits from call to call.  The workspace may be of 0 bytes, and then NULL.
 * Limits: 1 <= N, V <= 2^22, 1 <= D <= 65536, N V, N D and V D < 2^36, ldwt <= 2^23.
 */
size_t lsr_fp8_backward_workspace_bytes(int64_t N, int64_t V, int64_t D, int32_t need_dh, int32_t need_dw, int32_t need_db);

int lsr_fp8_backward(int64_t N, int64_t V, int64_t D, int32_t y_dtype, int32_t h_dtype,
                     const void* dY, int64_t ldy, const void* H, int64_t ldh,
                     const uint8_t* Wt, int64_t ldwt, const uint8_t* wt_exps,
                     void* dH, void* dW, float* db,
                     void* workspace, size_t workspace_bytes, lsr_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* LSR_FP8_H */
