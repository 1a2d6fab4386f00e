/*
 * lsr_beam.h - C ABI of a beam search over the head's dense logits: the selection of the next beams, and the reordering of what they keep.
 *
 * The conventions of lsr_head.h hold for every entry point: device pointers owned by the caller, a caller-owned workspace whose size
 * the library states, work enqueued on `stream` without a synchronisation, every check on the host before anything is enqueued, a status
 * as the return value, no state kept, outputs overwritten.  All calls can be recorded into a HIP graph.
 */
#ifndef LSR_BEAM_H
#define LSR_BEAM_H

#include "lsr_head.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * For each of B sequences the K best continuations of its beams:
 *   s(m, v) = scores[b,m] + X[b beams + m, v] / temperature - lse(b, m),   lse = log sum_v exp(X[b beams + m, v] / temperature)
 * in descending order, equal ones by ascending beam and, of one beam, by descending logit and ascending token.  Scores are compared as
 * formed in 64 bits.  lse is off by about 1e-8 where the largest logits hold most of the sum, and by less than 3e-6 whatever they are (a term below the largest ones, a =
 * log2 of its ratio to them, is formed in float32 to (1.4 |a| + 14) 2^-24 of itself; sums are 64 bits from a batch of a few thousand logits on).  Beams of equal rows have
 * equal lse; continuations of different rows whose scores are closer than that may change places.
 *   X          [B beams, ldx] x_dtype (LSR_F32 or LSR_BF16), any alignment of its elements, ldx >= V
 *   scores     [B, beams] f32; a beam of -inf has no continuation, and its logits are not read
 *   finished   [B, beams] uint8 or NULL: a beam whose byte is not 0 has one continuation, end_id with its own score; its logits are not read
 *   out_scores [B, K] f32, out_beams [B, K] int32, out_tokens [B, K] int32
 * A logit of -inf is no continuation; logits of the type's lowest value are ordinary.  Where there are fewer than K continuations the places behind them have score -inf,
 * beam 0 and token end_id.  A beam whose logits hold a NaN or +inf has continuations of score NaN, which come before all others (its K largest
 * logits that are numbers, then end_id).  beams = 1 gives the K largest log-probabilities of each row.
 * f32 and int32 arrays are 4-byte aligned.  Limits: 1 <= B, 1 <= beams <= 64, B beams < 2^22, 1 <= K <= 128, K <= beams V, 1 <= V < 2^31 - 4096,
 * 0 <= end_id < V, temperature between 5e-39 and 1e38.
 */
size_t lsr_beam_select_workspace_bytes(int64_t B, int64_t beams, int64_t V, int64_t K);

int lsr_beam_select(int64_t B, int64_t beams, int64_t V, int64_t K, int32_t x_dtype, double temperature,
                    const void* X, int64_t ldx, const float* scores, const uint8_t* finished, int64_t end_id,
                    float* out_scores, int32_t* out_beams, int32_t* out_tokens,
                    void* workspace, size_t workspace_bytes, lsr_stream_t stream);

/*
 * One thing that beams keep: for each of B sequences and each beam `pieces` pieces of `piece_bytes` contiguous bytes.  Strides in bytes, not negative: from sequence to
 * sequence, from beam to beam and from piece to piece.
 */
typedef struct {
    const void* src;
    void* dst;
    int64_t src_batch, src_beam, src_piece;
    int64_t dst_batch, dst_beam, dst_piece;
    int64_t pieces, piece_bytes;
} lsr_beam_state;

/*
 * dst[b, k] = src[b, parents[b, k]] for every state, b < B, k < K; zeros where parents[b, k] is outside [0, beams).
 *   parents  [B, K] int32 (4-byte aligned)
 *   states   n of them in HOST memory, read before the call returns
 * Any alignment (the widest access that addresses, strides and pieces allow).  No dst may overlap a src or another dst.
 * Limits: 1 <= B, beams, K; B beams, B K < 2^31; 0 <= n <= 4096; pieces >= 1, piece_bytes >= 1, pieces piece_bytes < 2^31; B K pieces piece_bytes < 2^40 and,
 * in accesses of 16 bytes or of as few as the alignment of an array's addresses, strides and pieces allows, at most 1024 (2^24 - 1) of them (16 GiB of single bytes).
 */
int lsr_beam_reorder(int64_t B, int64_t beams, int64_t K, const int32_t* parents, int64_t n, const lsr_beam_state* states, lsr_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* LSR_BEAM_H */
