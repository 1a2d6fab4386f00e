/*
 * lsr_distill.h - C ABI of the operators around the dense logits of the head: the same H, W and bias as
 * lsr_head.h, before the maximum over the sequence is taken.
 *
 *   lsr_quantize_rows    rows of values to 8-bit integers, one scale for each row
 *   lsr_int8_matmul      logits of a head whose matrix (and whose hidden states) are held in 8 bits
 *   lsr_top_logits       the largest K logits of each row and the logarithm of the row's normaliser
 *   lsr_distill_forward  loss of a head against a teacher's top logits; the N x V logits are never stored
 *   lsr_distill_backward its gradients
 *
 * The conventions of lsr_head.h hold for every entry point: device pointers owned by the caller, a
 * caller-owned workspace whose size the library states, work enqueued on `stream` without a synchronisation,
 * every check on the host before anything is enqueued, a status as the return value, no state kept, outputs
 * overwritten.  All calls can be recorded into a HIP graph.  Pointers are 16-byte aligned where nothing else
 * is said.  Arrays are row-major; a leading dimension (ld) counts elements from one row to the next.
 */
#ifndef LSR_DISTILL_H
#define LSR_DISTILL_H

#include "lsr_head.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A third element type beside LSR_F32 and LSR_BF16: 8-bit integers with a scale for each row. */
#define LSR_I8 2

/* Bytes of a row of `cols` 8-bit values: cols rounded up to a multiple of 128 (0 for cols out of range). */
int64_t lsr_int8_row_bytes(int64_t cols);

/*
 * Rows to 8 bits, the same for hidden states (one scale per token) and matrices (one per vocabulary entry):
 *   scale[r] = m_r / 127,  m_r = max_c |X[r,c]|;   Q[r,c] = 127 X[r,c] / m_r rounded to nearest, ties to even
 * For LSR_F32 the quotient that is rounded is the float32 one, (127 X) / m with a rounding each: where the exact one is within 2^-16 of half-way, the
 * neighbouring level is possible.  For LSR_BF16 the levels are those of the exact quotient.
 * A row of zeros has scale 0 and zeros.  A row with an infinity or a NaN has scale NaN and zeros, so that whatever
 * is multiplied by it shows it.
 *   X     [rows, cols] x_dtype (LSR_F32 or LSR_BF16), any alignment of its elements, ldx >= cols
 *   Q     [rows, ldq] int8, ldq a multiple of 16 and at least lsr_int8_row_bytes(cols); the bytes behind cols are
 *         set to zero up to lsr_int8_row_bytes(cols), and not touched behind that
 *   scale [rows] f32 (4-byte aligned)
 * Limits: 1 <= rows < 2^26, 1 <= cols <= 65536.
 */
int lsr_quantize_rows(int64_t rows, int64_t cols, int32_t x_dtype, const void* X, int64_t ldx,
                      int8_t* Q, int64_t ldq, float* scale, lsr_stream_t stream);

/*
 * out[n,v] = a_scale[n] w_scale[v] sum_k A[n,k] W[v,k] + bias[v]
 * The sum is exact (32-bit integers); scales and bias are applied in float32, and the result is rounded once.
 *   a_dtype   LSR_I8: A [N, lda] int8 rows as lsr_quantize_rows writes them (bytes from K to lsr_int8_row_bytes(K)
 *             zero), lda a multiple of 16 and at least lsr_int8_row_bytes(K), a_scale [N].
 *             LSR_F32 or LSR_BF16: A [N, lda] values, any alignment of its elements, lda >= K, quantised within the
 *             call exactly as by lsr_quantize_rows; a_scale must be NULL.
 *   W         [V, ldw] int8 rows, w_scale [V] f32, as lsr_quantize_rows writes them
 *   bias      [V] f32, or NULL for none
 *   out       [N, ldo] out_dtype (LSR_F32 or LSR_BF16), any alignment of its elements, ldo >= V
 *   workspace lsr_int8_matmul_workspace_bytes (0 for LSR_I8: then it may be NULL; 0 also for an invalid shape)
 * Scales and bias are 4-byte aligned.  Limits: 1 <= N < 2^26, 1 <= V < 2^31 - 4096, N V < 2^38, 1 <= K <= 65536,
 * ldw and the lda of int8 rows at most 2^23.
 */
size_t lsr_int8_matmul_workspace_bytes(int64_t N, int64_t V, int64_t K, int32_t a_dtype);

int lsr_int8_matmul(int64_t N, int64_t V, int64_t K, int32_t a_dtype, int32_t out_dtype,
                    const void* A, int64_t lda, const float* a_scale,
                    const int8_t* W, int64_t ldw, const float* w_scale, const float* bias,
                    void* out, int64_t ldo,
                    void* workspace, size_t workspace_bytes, lsr_stream_t stream);

/*
 * The K largest logits of every row, in descending order, equal ones by ascending index, and
 * lse[r] = log sum_v exp(X[r,v] / temperature) over the whole row.
 *   X       [rows, ldx] x_dtype (LSR_F32 or LSR_BF16), any alignment of its elements, ldx >= V
 *   values  [rows, K] f32, ids [rows, K] int32, lse [rows] f32 or NULL (all 4-byte aligned)
 * Logits of -inf are ordinary values (they come last, and add nothing to lse; a row of them has lse = -inf).
 * -0 and +0 are equal.  NaN comes before +inf and makes lse NaN.
 * Limits: 1 <= rows < 2^23, 1 <= K <= min(V, 256), V < 2^31 - 4096, temperature finite and at least 5e-39.
 */
size_t lsr_top_logits_workspace_bytes(int64_t rows, int64_t V, int64_t K);

int lsr_top_logits(int64_t rows, int64_t V, int64_t K, int32_t x_dtype, float temperature,
                   const void* X, int64_t ldx, float* values, int32_t* ids, float* lse,
                   void* workspace, size_t workspace_bytes, lsr_stream_t stream);

/*
 * Distillation from a teacher's top logits.  With z[n,v] = (H[n,:] . W[v,:] + bias[v]) / temperature:
 *   lse[n]  = log sum_v exp(z[n,v])
 *   p[n,j]  = exp(teacher_logits[n,j] / temperature - L[n])
 *   loss[n] = sum_j p[n,j] (log p[n,j] - z[n, teacher_ids[n,j]] + lse[n])
 * L[n] is teacher_lse[n] where that array is given (the normaliser over the teacher's whole vocabulary, as
 * lsr_top_logits leaves it, at the same temperature); else the logarithm of sum_j exp(teacher_logits[n,j] / temperature), so
 * that the kept probabilities sum to one.
 * An id outside [0, V) and a teacher logit of -inf are padding: such an entry is left out.  Ids of a row are meant to differ;
 * one that comes twice counts with both probabilities.
 * Rows whose mask byte is 0 are left out: loss 0, lse 0, no gradient.  A row without any entry has loss 0 and no gradient.
 * bias[v] = -inf excludes an entry (a teacher's probability on it makes the loss infinite); everything else is finite.
 * (A row whose logits hold a NaN and no +inf has lse NaN, and loss NaN where it has an entry; other rows do not see it.)
 *
 * N counts tokens (B * S of the head), D is the hidden size, V the vocabulary, K the teacher's entries per token.
 * Limits: 1 <= N <= 2^22; D a multiple of 8, 8 <= D <= 8192; 1 <= V <= 2^21; N V < 2^38; N D < 2^33;
 * 1 <= K <= 256; temperature finite and at least 5e-39 (log2(e) / temperature is a float32).
 *   H [N,D], W [V,D] hw_dtype;  bias [V] f32;  teacher_ids [N,K] int32;  teacher_logits [N,K] f32;
 *   teacher_lse [N] f32 or NULL;  mask [N] uint8 or NULL (no row left out);  loss [N], lse [N] f32.
 * LSR_BF16 multiplies in bfloat16 with float32 sums; LSR_F32 to the precision of float32.
 */
typedef struct {
    int64_t N, D, V, K;
    int32_t hw_dtype;     /* lsr_dtype */
    float temperature;
} lsr_distill_desc;

/* Bytes of workspace of the forward (for_backward = 0) or the backward; 0 for an invalid desc.  Neither holds an array of
 * N * V elements beyond a bounded piece: O(N (D + K + V/32) + V D) and, for the backward, two pieces of at most 2^28 + 256 (N + 256)
 * bfloat16 values (three times that for LSR_F32). */
size_t lsr_distill_workspace_bytes(const lsr_distill_desc* desc, int for_backward);

int lsr_distill_forward(const lsr_distill_desc* desc, const void* H, const void* W, const float* bias,
                        const int32_t* teacher_ids, const float* teacher_logits, const float* teacher_lse,
                        const uint8_t* mask, float* loss, float* lse,
                        void* workspace, size_t workspace_bytes, lsr_stream_t stream);

/*
 * Gradients of sum_n dloss[n] loss[n], from the lse that the forward left:
 *   g[n,v]  = dloss[n] / temperature (exp(z[n,v] - lse[n]) sum_j p[n,j] - sum over j with teacher_ids[n,j] = v of p[n,j])
 *   dH[n,:] = sum_v g[n,v] W[v,:]     dW[v,:] = sum_n g[n,v] H[n,:]     db[v] = sum_n g[n,v]
 * dH [N,D] and dW [V,D] are of hw_dtype, db [V] is f32; each may be NULL to skip it.  Sums are formed in float32 in a fixed
 * order and rounded once when the result is stored; db is summed from the unrounded g.  For LSR_BF16 g is a bfloat16 operand of the
 * matrix cores: rounded to 8 significant bits once (error of dH and dW 0.0024 of their norm, 0.0017 of it their own rounding), or, for
 * up to 64 rows whose hidden states fit LDS (N up to a multiple of 32, times 2 D up to a multiple of 32, and 16, at most 136 KiB), held in
 * two bfloat16 with 16 bits (0.0017).  Results are the same bits from call to call where the ids of a row differ.
 */
int lsr_distill_backward(const lsr_distill_desc* desc, const void* H, const void* W, const float* bias,
                         const int32_t* teacher_ids, const float* teacher_logits, const float* teacher_lse,
                         const uint8_t* mask, const float* lse, const float* dloss,
                         void* dH, void* dW, float* db,
                         void* workspace, size_t workspace_bytes, lsr_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* LSR_DISTILL_H */
