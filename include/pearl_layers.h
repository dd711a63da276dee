/*
 * pearl_layers.h -- C ABI of the operators of a layer, on the handle of pearl_rows.h.
 *
 * What stands around the router and the rows' way to their experts and back:
 *
 *   layer_norm, layer_norm_grad   the norm before a layer, and its gradient with that of its weight and bias
 *   dropout                       a branch with elements dropped, added to the residual rows; its gradient is the same call
 *   experts                       a whole expert layer for the few rows of a policy's step: the router's product and choice, the
 *                                 chosen experts' two products, their weighted sum
 *
 * Conventions: those of pearl_rows.h (device pointers that the caller owns, the handle's stream, nothing allocated, nothing
 * kept, rows that may lie apart by ld_* elements, one rounding to a narrower type, the same bits whatever the timing).  A call that
 * needs scratch is given it: d_work, 256-byte aligned, of the bytes that the *_work_bytes call names.  Two calls that may run at the same
 * time (two streams, two captured graphs that are replayed side by side) need scratch of their own.
 * What is read beside a row is at most the rest of the 16-byte words that it starts and ends in; that holds for the first and last row of an
 * array, and for the first of the experts' weights, too.
 */
#ifndef PEARL_LAYERS_H_
#define PEARL_LAYERS_H_

#include "pearl_rows.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PEARL_LAYER_MAX_WIDTH 65536u   /* D of the norm */
#define PEARL_LAYER_MAX_FEW 64u        /* T of the expert layer */
#define PEARL_LAYER_MAX_INNER 65536u   /* D and H of the expert layer */

#define PEARL_ACT_SILU_GATED 0u        /* h = silu(gate) * value; an expert's first product has 2H rows: H gates, then H values */
#define PEARL_ACT_RELU 1u              /* h = max(value, 0); an expert's first product has H rows (a NaN stays one) */

/* y[t] = (x[t] - mean_t) * rstd_t * gamma + beta, mean_t the mean of row t's D elements, rstd_t = 1 / sqrt(var_t + eps), var_t the mean of
 * (x - mean_t)^2.  gamma and beta (D elements of param_dtype, which is PEARL_F32 or dtype) may each be NULL: weights of 1, a
 * bias of 0.  d_mean and d_rstd (binary32, T entries, what the gradient wants) may each be NULL.  A row with an element that is not
 * finite has NaN for results; other rows are not touched by it.  Sums and squares are binary32's, too: a row whose sum passes that range has NaN, one whose
 * squared differences do (from some 1e19 on) has a d_rstd of 0 and the bias for results.
 * 1 <= D <= PEARL_LAYER_MAX_WIDTH, eps >= 0 and finite; T < 2^31 may be 0. */
int pearl_layer_norm(pearl_rows_t* rows, uint32_t T, uint32_t D, uint32_t dtype, const void* d_x, uint64_t ld_x, uint32_t param_dtype,
                     const void* d_gamma, const void* d_beta, double eps, void* d_y, uint64_t ld_y, float* d_mean, float* d_rstd);

/* The norm's gradient, given its input and what it returned.  With n = (x - mean_t) * rstd_t and g = dy * gamma:
 *   dx[t] = rstd_t * (g - mean(g) - n * mean(g * n)),  dgamma = sum over t of dy * n,  dbeta = sum over t of dy
 * d_dx, d_dgamma and d_dbeta may be NULL where they are not wanted (not all three); d_gamma NULL stands for weights of 1.  dgamma and dbeta
 * (binary32, D elements) are written, not added to; T of 0 gives zeros.  d_work is read and written only for them and may be NULL
 * without them; its contents do not matter. */
int pearl_layer_norm_grad(pearl_rows_t* rows, uint32_t T, uint32_t D, uint32_t dtype, const void* d_dy, uint64_t ld_dy, const void* d_x,
                          uint64_t ld_x, const float* d_mean, const float* d_rstd, uint32_t param_dtype, const void* d_gamma, void* d_dx,
                          uint64_t ld_dx, float* d_dgamma, float* d_dbeta, void* d_work, uint64_t work_bytes);
/* At least 1; 0 for a width out of range. */
uint64_t pearl_layer_norm_grad_work_bytes(uint32_t T, uint32_t D);

/* y[t][d] = (keep ? x[t][d] * s : 0) + residual[t][d].  The mask is not stored: element (t, d) has 16 bits of Philox4x32-10 with
 * counter (d / 8, t, call_lo, call_hi) and key (seed_lo, seed_hi): of its word (d % 8) / 2 the low half for even d, the high half for
 * odd; it is kept where those, as a number, are not below m = floor(65536 p + 0.5), and s = 65536 / (65536 - m), so that the mean
 * is exact for the probability m / 65536 that is used (m = 65536: nothing is kept).  The same seed and call give the same mask, whatever
 * the types, sizes and distances: the gradient is this call on dy, without a residual.  d_calls, where it is not NULL, is a number in device
 * memory that is added to `call` (modulo 2^64): a captured graph that counts it up draws a new mask in each replay.
 * d_residual NULL: 0.  A dropped element does not matter, whatever it is.  The product and the sum are binary32 operations, rounded once more to the type.
 * y may be x or the residual itself (the same address and distance).
 * 0 <= p <= 1; 1 <= D <= PEARL_ROWS_MAX_ROW_BYTES / the element's size; T < 2^31 may be 0. */
int pearl_layer_dropout(pearl_rows_t* rows, uint32_t T, uint32_t D, uint32_t dtype, const void* d_x, uint64_t ld_x, const void* d_residual,
                        uint64_t ld_residual, double p, uint64_t seed, uint64_t call, const uint64_t* d_calls, void* d_y, uint64_t ld_y);

/* An expert layer for a few rows: y[t] = sum over j of w_j * (down[e_j] h_j), h_j = act(up[e_j] x[t]), over the k experts of row t.
 *   d_router  E x D.  The logits are router . x[t], summed in binary64 and rounded to binary32; the choice and the weights go by them as in
 *             pearl_rows_route (over_chosen; ties to the lower expert; NaN and +infinity bar an expert and raise PEARL_ST_BAD_SCORE) and
 *             are written to d_w and d_ids (T x k).  NULL: d_w and d_ids are given; an id of -1 is a slot without an expert, another one
 *             outside [0, E) counts as -1 and raises PEARL_ST_BAD_INDEX; a row may name an expert more than once.
 *   d_up      E x (2H or H) x D, by `act`;  d_down  E x D x H;  both dense, of the rows' type
 * Sums run in binary32 or wider.  h is held as a binary32, in 16-bit layers as the sum of numbers of the type: three of bfloat16, which are all of it; two
 * of binary16, which are it but for 2^-22 of it or 2^-36, whichever is more (an h beyond 65504 is infinite).  Infinities and NaN go by the formula in
 * 16-bit layers (but a binary16 h below 2^-25 times an infinite weight is NaN).  Products of binary32 are formed from two parts of 11 bits each, all but
 * 2^-21 of them; an infinite factor, or one above 3.4e38, gives NaN there, as a NaN does.  An expert that no row asks for is not read.  A row without
 * experts is zero.
 * d_work must be zero before its first use; every call leaves it fit for the next one, of any sizes it has room for.
 * 1 <= k <= min(E, PEARL_ROWS_MAX_CHOICES), E <= PEARL_ROWS_MAX_EXPERTS, T <= PEARL_LAYER_MAX_FEW (0: nothing to do), D and H within
 * 1 .. PEARL_LAYER_MAX_INNER. */
int pearl_layer_experts(pearl_rows_t* rows, uint32_t T, uint32_t D, uint32_t H, uint32_t E, uint32_t k, uint32_t dtype, uint32_t act,
                        const void* d_x, uint64_t ld_x, const void* d_router, int over_chosen, const void* d_up, const void* d_down,
                        float* d_w, int32_t* d_ids, void* d_y, uint64_t ld_y, void* d_work, uint64_t work_bytes);
/* 0 for sizes out of range.  It does not fall where a size grows. */
uint64_t pearl_layer_experts_work_bytes(uint32_t T, uint32_t D, uint32_t H, uint32_t E, uint32_t k);

#ifdef __cplusplus
}
#endif
#endif /* PEARL_LAYERS_H_ */
