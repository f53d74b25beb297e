/*
 * nimble_moe.h -- C ABI of the routing operators: from the router's logits of a
 * mixture-of-experts layer to the demand vector the planner reads (nimble_plan.h), and the
 * balance loss that works in training against the skew the planner routes around.
 *
 *   nimble_moe_route           choice of experts per token, their weights, and the counts and
 *                              probability sums that the loss is made of
 *   nimble_moe_balance_loss    the loss of every segment
 *   nimble_moe_route_backward  gradient of the logits from the gradients of weights and loss
 *   nimble_moe_counts          slots per expert and distinct tokens per destination GPU
 *   nimble_moe_traffic         these tokens as bytes per commodity (the monitoring step of
 *                              Sec. IV-A: per-pair byte counts for the planner)
 *
 * Rows are tokens.  Segments are runs of rows -- the tokens of a source GPU, a sequence, a
 * micro-batch -- given by ascending offsets d_seg_ptr [n_segments + 1]: segment s has rows
 * d_seg_ptr[s] .. d_seg_ptr[s+1]-1 (none is fine).  Rows in no segment make no difference and are
 * not written.  Offsets below 0 or beyond the rows are taken as 0 and the number of rows; offsets
 * that do not ascend give unspecified values (never an access out of range).  A NULL d_seg_ptr
 * stands for one segment of all rows and needs n_segments = 1.
 *
 * All pointers are device memory of the current GPU, aligned to their element type (d_scratch
 * to 16 bytes), and outputs overlap neither each other nor inputs.  Offsets into arrays are
 * taken in 64 bits.  Scores, statistics, weights and sums are IEEE binary32 or wider, whatever
 * the type of the logits; sums are made in a fixed order, so results are the same on every run
 * (they do depend, within rounding, on the number of rows).
 *
 * Calls only enqueue work on hip_stream (NULL = default stream); they allocate nothing, never
 * synchronise and keep nothing between calls, so they may be captured into HIP graphs.
 * d_scratch belongs to a call until the work it enqueued is done: calls that may overlap, two
 * captured graphs among them, need scratch memory of their own.  Its contents do not matter.
 * Errors: NIMBLE_ERR_INVALID for bad arguments, NIMBLE_ERR_RANGE for sizes beyond the limits
 * below, NIMBLE_ERR_HIP for a failed launch; the message is in nimble_last_error().
 */
#ifndef NIMBLE_MOE_H
#define NIMBLE_MOE_H

#include <stdint.h>

#include "nimble_plan.h"

#ifdef __cplusplus
extern "C" {
#endif

/* limits (NIMBLE_ERR_RANGE beyond them) */
enum {
    NIMBLE_MOE_MAX_TOKENS = 0x7FFF0000,
    NIMBLE_MOE_MAX_EXPERTS = 2048,
    NIMBLE_MOE_MAX_TOP_K = 16,
    NIMBLE_MOE_MAX_RANKS = 4096,
    NIMBLE_MOE_MAX_SEGMENTS = 1 << 20
};

/* element types of logits and of their gradient */
enum { NIMBLE_F32 = 0, NIMBLE_F16 = 1, NIMBLE_BF16 = 2 };

/* flags of nimble_moe_route and nimble_moe_route_backward */
enum {
    NIMBLE_MOE_SOFTMAX = 0u, /* score s_e = exp(x_e) / sum exp(x)                   (default) */
    NIMBLE_MOE_SIGMOID = 1u, /* score s_e = 1 / (1 + exp(-x_e)) */
    NIMBLE_MOE_RENORM = 2u   /* weights are divided by the sum over the chosen experts */
};

/* flag of nimble_moe_traffic */
enum { NIMBLE_MOE_WAY_BACK = 1u /* the demand of the way back: destination to source */ };

/*
 * Chooses top_k experts per row of logits x and gives their weights.
 *
 *   choice   key_e = x_e + bias_e in binary32 (the bias steers the choice alone: weights,
 *            probabilities and gradients are those of x).  The top_k experts with the largest
 *            keys, largest first, ties to the lower index.  Experts with x = -inf (a mask) or
 *            key = -inf are not chosen; slots they leave empty, and rows they leave
 *            without a choice, have index -1 and weight 0.  A row that holds NaN or +inf has
 *            no choice either: its indices are -1, its weights NaN, and so are the probability
 *            sums of its segment and the row of the gradient.
 *   weight   scale * s_e, or with NIMBLE_MOE_RENORM scale * s_e / (sum of s over the row's
 *            chosen experts)
 *   sums     per segment: counts_e = slots that chose e; routed = rows with a choice;
 *            prob_sum_e = sum over these rows of p_e, where p_e = s_e / sum s (up to 64 rows after
 *            another in binary32, the parts in binary64: adding up costs less than 80 * 2^-24 of
 *            the sum, whatever the number of rows)
 *
 *   tokens, experts   rows and columns of d_logits; tokens may be 0; 1 <= experts <= 2048
 *   top_k        1 <= top_k <= min(experts, 16)
 *   dtype        NIMBLE_F32, NIMBLE_F16 or NIMBLE_BF16
 *   d_logits     [tokens][experts], rows row_stride >= experts elements apart
 *   d_bias       float [experts], or NULL; NaN counts as -inf, +inf as the largest finite number
 *   d_keep       [tokens], 0 for rows to leave out (padding): they have no choice and may hold
 *                anything; or NULL
 *   scale        finite and > 0 (and no denormal number)
 *   d_index      int32 [tokens][top_k] out
 *   d_weight     float [tokens][top_k] out
 *   d_counts     int32 [n_segments][experts] out   \
 *   d_routed     int32 [n_segments] out             > all three, or all NULL
 *   d_prob_sum   float [n_segments][experts] out   /
 *   d_scratch    scratch_bytes >= nimble_moe_route_scratch_bytes(...) bytes; may be NULL when
 *                that is 0 or when no sums are wanted
 */
nimble_status_t nimble_moe_route(int32_t tokens, int32_t experts, int32_t top_k, uint32_t flags,
                                 int32_t dtype, const void *d_logits, int64_t row_stride,
                                 const float *d_bias, const uint8_t *d_keep, float scale,
                                 int32_t n_segments, const int32_t *d_seg_ptr, int32_t *d_index,
                                 float *d_weight, int32_t *d_counts, int32_t *d_routed,
                                 float *d_prob_sum, void *d_scratch, int64_t scratch_bytes,
                                 void *hip_stream);

/*
 * Scratch bytes of nimble_moe_route with sums; -1 for sizes it refuses.  They do not rise with every
 * size: a call with fewer rows may need more, so memory for calls of several sizes is the most of theirs.
 */
int64_t nimble_moe_route_scratch_bytes(int32_t tokens, int32_t experts, int32_t n_segments);

/*
 * loss_s = alpha * experts / top_k * sum_e (counts_e / routed) * (prob_sum_e / routed), which is
 * alpha where choices and probabilities are even, and more the more both favour the same
 * experts; 0 for a segment with routed = 0.
 *
 *   d_counts, d_routed, d_prob_sum   as nimble_moe_route gives them, or added up over GPUs:
 *            the loss is then that of the whole group, and nimble_moe_route_backward with the
 *            same counts gives each GPU its part of the gradient
 *   alpha    finite
 *   d_loss   float [n_segments] out
 */
nimble_status_t nimble_moe_balance_loss(int32_t n_segments, int32_t experts, int32_t top_k,
                                        const int32_t *d_counts, const int32_t *d_routed,
                                        const float *d_prob_sum, float alpha, float *d_loss,
                                        void *hip_stream);

/*
 * Gradient of the logits from g = d/d weight and h = d/d loss.  Counts and the choice are
 * constants.  With c_e = h_s * alpha * experts * counts_e / (top_k * routed^2) and
 * a_j = w_j * (g_j - [renorm] sum_i w_i g_i / scale):
 *   softmax   dx_e = p_e (c_e - sum p c - [not renorm] sum_j w_j g_j) + sum_j [index_j = e] a_j
 *   sigmoid   dx_e = p_e (1 - s_e) (c_e - sum p c) + sum_j [index_j = e] a_j (1 - s_e)
 * Rows left out by d_keep and rows without a choice get zeros.
 *
 *   d_index, d_weight   what nimble_moe_route gave for the same logits, flags, scale, d_keep and
 *                  segments (indices outside 0 .. experts-1 are empty slots; an index that a row holds
 *                  more than once adds up, in the order of the slots)
 *   d_grad_weight  float [tokens][top_k], or NULL for zeros
 *   d_counts, d_routed, d_grad_loss   [n_segments][experts], [n_segments], float [n_segments]:
 *                  all three, or all NULL: no loss
 *   d_grad_logits  [tokens][experts] out, of the logits' type, rows grad_stride elements apart
 */
nimble_status_t nimble_moe_route_backward(int32_t tokens, int32_t experts, int32_t top_k,
                                          uint32_t flags, int32_t dtype, const void *d_logits,
                                          int64_t row_stride, const uint8_t *d_keep, float scale,
                                          int32_t n_segments, const int32_t *d_seg_ptr,
                                          const int32_t *d_index, const float *d_weight,
                                          const float *d_grad_weight, float alpha,
                                          const int32_t *d_counts, const int32_t *d_routed,
                                          const float *d_grad_loss, void *d_grad_logits,
                                          int64_t grad_stride, void *hip_stream);

/*
 * Counts of routed tokens, per segment.
 *
 *   d_index        int32 [tokens][top_k], experts per row; entries outside 0 .. experts-1 are
 *                  empty slots
 *   d_counts       int32 [n_segments][experts] out or NULL: slots per expert
 *   d_expert_rank  int32 [experts]: the GPU an expert lives on; entries outside
 *                  0 .. n_ranks-1 live nowhere
 *   d_rank_tokens  int32 [n_segments][n_ranks] out or NULL: rows with at least one expert on
 *                  that GPU: a token goes to a GPU once, however many of its experts are there.
 *                  (An All-to-Allv that sends every slot carries up to top_k times as much: the sums
 *                  of d_counts over the experts of a GPU, which no call here makes.)
 * At least one of the outputs; n_ranks >= 1 and d_expert_rank with d_rank_tokens.
 */
nimble_status_t nimble_moe_counts(int32_t tokens, int32_t top_k, const int32_t *d_index,
                                  int32_t experts, int32_t n_segments, const int32_t *d_seg_ptr,
                                  const int32_t *d_expert_rank, int32_t n_ranks,
                                  int32_t *d_counts, int32_t *d_rank_tokens, void *d_scratch,
                                  int64_t scratch_bytes, void *hip_stream);

/* Scratch bytes of nimble_moe_counts, as above; -1 for sizes it refuses.  n_ranks 0: no rank tokens. */
int64_t nimble_moe_counts_scratch_bytes(int32_t tokens, int32_t top_k, int32_t experts,
                                        int32_t n_ranks, int32_t n_segments);

/*
 * The demand vectors of `batch` layers or micro-batches, as nimble_plan_solve_batch reads them.
 *
 *   d_rank_tokens    int32 [batch][n_ranks][n_ranks]: tokens that GPU r (row) sends to GPU q, as
 *                    nimble_moe_counts gives them for a segment per source GPU
 *   bytes_per_token  finite and >= 0 (hidden size times bytes per element)
 *   n_comm, d_src, d_dst   the commodities: int32 [n_comm] GPUs, entries outside
 *                    0 .. n_ranks-1 give NaN; both NULL for all ordered pairs of different GPUs
 *                    in row-major order, n_comm = n_ranks * (n_ranks - 1)
 *   flags            NIMBLE_MOE_WAY_BACK: commodity (s, d) carries what s receives in the
 *                    dispatch from d
 *   d_traffic        double [batch][n_comm] out: bytes, tokens * bytes_per_token
 */
nimble_status_t nimble_moe_traffic(int32_t batch, int32_t n_ranks, const int32_t *d_rank_tokens,
                                   double bytes_per_token, int32_t n_comm, const int32_t *d_src,
                                   const int32_t *d_dst, uint32_t flags, double *d_traffic,
                                   void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* NIMBLE_MOE_H */
