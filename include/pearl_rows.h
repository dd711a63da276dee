/*
 * pearl_rows.h -- C ABI of the row operators beside the replay buffer: choose, weigh and move rows of a batch.
 *
 * pearl_prb_sample chooses transitions by a number each of them has, hands out indices and weights and moves the
 * rows that the indices name.  The calls here do the same for what a learner and a policy put around that batch:
 *
 *   expert layers   a router picks k of E experts for each of T rows (route), the rows are sorted by expert and
 *                   copied there (sort, dispatch), the experts' answers are brought back and weighted (combine);
 *                   with the gradient of each (route_grad, combine, combine_grad);
 *   beam search     one step's choice over the beams and the vocabulary (beam_select) and the move of the beams'
 *                   states to where that choice says (beam_reorder).
 *
 * Conventions (those of pearl_prb.h, whose error codes and status bits are used here)
 *   - Every d_* argument is a DEVICE pointer owned by the caller; nothing is kept after the work is enqueued.  Calls
 *     check their host-visible arguments, enqueue on the handle's stream and return PEARL_OK or a negative
 *     PEARL_ERR_* (then nothing was enqueued).  They allocate nothing, keep no scratch between calls and can be
 *     captured into a CUDA graph; graphs of one handle may be replayed side by side (they share the status word, which
 *     only collects bits).
 *   - Outputs must not overlap inputs or each other, except where a call says so.
 *   - `dtype` names the element type of logits and rows.  Sums, softmax statistics, weights and scores are computed in
 *     binary32 or wider, the router's exponentials within 2 units of the last place; what is handed out in a narrower type is
 *     rounded to it once.
 *   - Rows of a matrix may lie apart (the ld_* arguments, in elements, at least the row's length); the elements of
 *     a row are consecutive.  The bytes between rows are never written; up to 31 of them beside a row may be read.
 *     Pointers must be aligned to their element size, else PEARL_ERR_ALIGN.  Rows whose start and length are multiples of
 *     16 bytes move fastest.
 *   - Results do not depend on timing: the same inputs give the same bits.
 *   - Conditions found on the device never trap; they set PEARL_ST_* bits that pearl_rows_sync() returns and clears.
 *   - One handle is used from one host thread at a time.
 */
#ifndef PEARL_ROWS_H_
#define PEARL_ROWS_H_

#include "pearl_prb.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pearl_rows pearl_rows_t;

#define PEARL_F32 0u               /* IEEE binary32 */
#define PEARL_F16 1u               /* IEEE binary16 */
#define PEARL_BF16 2u              /* bfloat16 */

#define PEARL_ST_BAD_SCORE 64u     /* a logit is NaN or +infinity, or a beam's score is: treated as -infinity */

#define PEARL_ROWS_MAX_EXPERTS 1024u
#define PEARL_ROWS_MAX_ROW_BYTES (1u << 23)
#define PEARL_ROWS_MAX_CHOICES 32u     /* k of the router */
#define PEARL_ROWS_MAX_BEAMS 32u       /* W */
#define PEARL_ROWS_MAX_BEST 64u        /* C */
#define PEARL_ROWS_MAX_VOCAB (1u << 24)

/* Device memory of a handle (its status word). */
uint64_t pearl_rows_slab_bytes(void);

/* Creates a handle on `device` whose calls enqueue on `cuda_stream` (a cudaStream_t; NULL = the legacy default
 * stream).  slab: optional caller-owned device memory of at least pearl_rows_slab_bytes() bytes, 256-byte aligned; NULL
 * lets the library allocate (and free in destroy).  It is zeroed on the stream. */
int pearl_rows_create(pearl_rows_t** out, int device, void* cuda_stream, void* slab, uint64_t slab_bytes);
/* Synchronises the stream, frees what the library owns.  Graphs captured from the handle's calls must not run after this: their kernels
 * raise bits in its status word. */
int pearl_rows_destroy(pearl_rows_t* rows);

/* The router.  Of row t's E logits the k largest are chosen, in falling order, the lower expert first among equal ones:
 * d_ids[t*k + j] and its weight d_w[t*k + j] = exp(l_j) / sum exp(l), the sum over all E experts, or with
 * over_chosen != 0 over the k chosen ones.  A logit of -infinity bars its expert; a row with fewer than k experts left
 * has id -1 and weight 0 in the places that remain.  A logit that is NaN or +infinity raises PEARL_ST_BAD_SCORE and counts as
 * -infinity.  1 <= k <= min(E, PEARL_ROWS_MAX_CHOICES), E <= PEARL_ROWS_MAX_EXPERTS, T*k < 2^31; T may be 0. */
int pearl_rows_route(pearl_rows_t* rows, uint32_t T, uint32_t E, uint32_t k, uint32_t dtype, const void* d_logits,
                     uint64_t ld_logits, int over_chosen, float* d_w, int32_t* d_ids);

/* The router's gradient: from dL/dw (d_dw) to dL/dlogits (d_dlogits, of the logits' type), given what route returned.
 *   over all:     dl_e = p_e (g_e - sum_j w_j dw_j),  p the softmax over all E, g_e = dw_j where e = ids_j, else 0
 *   over chosen:  dl_e = w_j (dw_j - sum_i w_i dw_i) where e = ids_j, else 0
 * Barred experts and places with id -1 have gradient 0.  An id outside [-1, E) raises PEARL_ST_BAD_INDEX and counts as -1.
 * d_logits may be NULL if over_chosen (it is not read). */
int pearl_rows_route_grad(pearl_rows_t* rows, uint32_t T, uint32_t E, uint32_t k, uint32_t dtype, const void* d_logits,
                          uint64_t ld_logits, int over_chosen, const float* d_w, const int32_t* d_ids, const float* d_dw,
                          void* d_dlogits, uint64_t ld_dlogits);

/* Slots sorted by expert.  Slot s = t*k + j asks for expert d_ids[s]; an id of -1 asks for none (any other id outside
 * [0, E) does so too and raises PEARL_ST_BAD_INDEX).  Stable counting sort:
 *   d_offsets[e]   (E + 1 entries) the slots that ask for an expert below e; d_offsets[E] = n, those that ask at all
 *   d_order[r]     the slot in sorted place r, r < n; entries from n on are left as they were (may be NULL)
 *   d_place[s]     the sorted place of slot s, -1 if it asks for none
 * slots = T*k < 2^31, may be 0; 1 <= E <= PEARL_ROWS_MAX_EXPERTS. */
int pearl_rows_sort(pearl_rows_t* rows, uint32_t slots, uint32_t E, const int32_t* d_ids, int32_t* d_offsets,
                    int32_t* d_order, int32_t* d_place);

/* Rows copied to their experts: xs[place[t*k + j]] = x[t], for every slot with a place.  Rows are row_bytes bytes of any
 * kind; x's rows lie ld_x BYTES apart, those of xs are dense.  xs has `sorted_rows` rows; a place outside [-1, sorted_rows)
 * raises PEARL_ST_BAD_INDEX and is skipped.  Rows of xs that no slot names are left as they were.  Every place is to
 * be named once (as sort does); where one is named twice, one of the two rows is there.
 * k >= 1, T*k < 2^31; T may be 0; row_bytes >= 1. */
int pearl_rows_dispatch(pearl_rows_t* rows, uint32_t T, uint32_t k, uint32_t row_bytes, const void* d_x, uint64_t ld_x,
                        const int32_t* d_place, uint32_t sorted_rows, void* d_xs);

/* The experts' answers brought back: y[t] = sum over j of w[t*k + j] * z[place[t*k + j]], slots without a place left out (none
 * left: zeros), in binary32 with j ascending, rounded once.  d_w == NULL stands for weights of 1: with z the gradient of
 * the dispatched rows, y is then the gradient of dispatch.  Rows are D elements; z is dense with `sorted_rows` rows (a place
 * outside: as for dispatch), y's rows lie ld_y elements apart.  k >= 1, T*k < 2^31; T may be 0; D >= 1. */
int pearl_rows_combine(pearl_rows_t* rows, uint32_t T, uint32_t k, uint32_t D, uint32_t dtype, const void* d_z,
                       uint32_t sorted_rows, const int32_t* d_place, const float* d_w, void* d_y, uint64_t ld_y);

/* The gradient of combine: dz[place[t*k + j]] = w[t*k + j] * dy[t] (rows that no slot names are left as they were) and
 * dw[t*k + j] = sum over d of dy[t][d] * z[place[t*k + j]][d], in binary32 (0 for a slot without a place).  d_dz or d_dw may be
 * NULL if it is not wanted (then d_w or d_z is not read); d_w == NULL with d_dz stands for weights of 1.  Other arguments as
 * for combine; dy's rows lie ld_dy elements apart. */
int pearl_rows_combine_grad(pearl_rows_t* rows, uint32_t T, uint32_t k, uint32_t D, uint32_t dtype, const void* d_dy,
                            uint64_t ld_dy, const void* d_z, uint32_t sorted_rows, const int32_t* d_place, const float* d_w,
                            void* d_dz, float* d_dw);

/* One step of a beam search for G groups of W beams over V tokens.  A beam b of group g with score s = d_scores[g*W + b] and
 * logits l (row g*W + b of d_logits, rows ld_logits elements apart) offers every token v with l_v > -infinity at
 * s + (l_v - log sum exp l).  A beam whose flag d_done[g*W + b] is not 0 is finished: it offers end_token alone, at s;
 * d_done may be NULL.  A score of -infinity takes its beam out.  Of a group's offers the C best
 * are handed out, best first: between tokens of a beam the larger logit wins and among equal ones the lower token, between
 * beams the larger sum and among equal ones the lower beam.  d_best_score (the sum, rounded to binary32), d_best_beam,
 * d_best_token: C entries a group; with fewer than C offers the rest is -infinity, -1, -1.
 * A row's sum of exponentials runs in binary64 and in whole numbers over binary32 sums of 8 or 16 terms; equal rows with equal scores have
 * equal sums wherever they lie.  The sums are compared in binary64.  Bytes between rows may be read; the logits of finished beams may be
 * read but do not matter.
 * A logit that is NaN or +infinity (or such a score) raises PEARL_ST_BAD_SCORE and counts as -infinity.
 * 1 <= W <= PEARL_ROWS_MAX_BEAMS, 1 <= C <= PEARL_ROWS_MAX_BEST, 1 <= V <= PEARL_ROWS_MAX_VOCAB; G may be 0. */
int pearl_rows_beam_select(pearl_rows_t* rows, uint32_t G, uint32_t W, uint32_t V, uint32_t C, uint32_t dtype,
                           const void* d_logits, uint64_t ld_logits, const float* d_scores, const uint8_t* d_done,
                           int32_t end_token, float* d_best_score, int32_t* d_best_beam, int32_t* d_best_token);

/* The beams' states moved: state[o, g, i] <- state[o, g, parent[g*W + i]] for every block o, group g and beam i.  A state is
 * `pieces` pieces of piece_bytes bytes, piece_pitch bytes apart (a cache [heads, room, dim] of which a part of the room is
 * in use is `heads` pieces); the state of beam i of group g in block o starts at o*block_pitch + (g*W + i)*state_pitch
 * bytes.  src and dst have pitches of their own.  d_dst == d_src (with the same pitches) moves the states in place, and
 * states that stay where they are are not touched; otherwise the bytes from src's first state to its last must not
 * overlap those of dst (PEARL_ERR_BAD_ARG).  A parent of -1 leaves the
 * state (of dst) as it was; any other parent outside [0, W) does so too and raises PEARL_ST_BAD_INDEX.
 * The pieces of different states must not overlap in dst.  1 <= W <= PEARL_ROWS_MAX_BEAMS; blocks, G, pieces or piece_bytes
 * of 0 is a call with nothing to do; blocks * G < 2^31 (PEARL_ERR_BAD_BATCH). */
typedef struct pearl_states {
    uint64_t block_pitch, state_pitch, piece_pitch;      /* bytes */
} pearl_states_t;
int pearl_rows_beam_reorder(pearl_rows_t* rows, uint32_t blocks, uint32_t G, uint32_t W, uint32_t pieces, uint64_t piece_bytes,
                            const int32_t* d_parent, const void* d_src, const pearl_states_t* src, void* d_dst,
                            const pearl_states_t* dst);

/* Waits for the handle's stream; returns the accumulated PEARL_ST_* bits in *status_bits (may be NULL) and clears them.  A bit that
 * a graph on another stream raises meanwhile is in this answer or in the next one. */
int pearl_rows_sync(pearl_rows_t* rows, uint32_t* status_bits);
/* Number of kernels this handle has launched so far (among them the one that clears the bits, where sync found any). */
uint64_t pearl_rows_kernel_launches(pearl_rows_t* rows);

#ifdef __cplusplus
}
#endif
#endif /* PEARL_ROWS_H_ */
