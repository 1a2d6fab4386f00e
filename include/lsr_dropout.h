/*
 * lsr_dropout.h - C ABI of dropout whose mask is never stored: it is drawn again from a counter wherever it is needed.
 * The conventions of lsr_head.h hold: device pointers, `stream`, checks on the host, a status, no state.  The call can be recorded into a HIP graph.
 */
#ifndef LSR_DROPOUT_H
#define LSR_DROPOUT_H

#include "lsr_head.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Y[i] = X[i] 65536 / (65536 - t) where r(i) >= t, else 0;   t = 65536 p rounded to a whole number (ties to even)
 * r(i) is 16-bit number i % 8 (the low half of 32-bit word 0, its high half, the low half of word 1, ...) of the Philox4x32-10 block (Salmon,
 * Moraes, Dror, Shaw: Parallel random numbers, as easy as 1, 2, 3; SC 2011) whose counter is (i / 8, offset') and whose key is seed', 64 bits each, low words first.
 *   state   [2] uint64 on the device (8-byte aligned) or NULL: seed' = seed + state[0], offset' = offset + state[1] modulo 2^64, read when
 *           the work runs, so that a replayed graph can draw new numbers; without it seed' = seed, offset' = offset
 * The gradient is the same call on the gradient of Y.  A value that is dropped is +0 whatever it was.  The probability is p to within 2^-17; t = 65536
 * drops everything.
 *   X, Y    n values of dtype (LSR_F32 or LSR_BF16), any alignment of their elements; Y may be X, or must not overlap it.  Products in float32, rounded once.
 * Limits: 1 <= n < 2^40, 0 <= p <= 1.
 */
int lsr_dropout(int64_t n, int32_t dtype, const void* X, void* Y, double p, uint64_t seed, uint64_t offset, const uint64_t* state,
                lsr_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* LSR_DROPOUT_H */
