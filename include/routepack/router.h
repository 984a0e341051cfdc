/*
 * routepack/router.h -- C-ABI of the router's operators (gfx950).
 *
 * The planner of routepack.h starts from replayed expert demand.  These entry
 * points are a trainer's side of the same routing: the gates of chosen or
 * replayed experts, the demand counted from recorded expert ids, the balance
 * loss over such counts, and the gradient of gates and loss with respect to
 * the router's logits.  They take the sizes L = n_layers, E = n_experts,
 * k = top_k and, for the demand, N = n_samples of a routepack_problem and
 * look at none of its other fields.
 *
 * Conventions, besides those of routepack.h
 * -----------------------------------------
 * - Every call is asynchronous on `stream`, allocates nothing, and may be
 *   captured into a graph.  The current device is the stream's.
 * - T tokens stand in one stream; sample (or group) i is the tokens
 *   [offsets[i], offsets[i + 1]) of it, offsets non-decreasing within [0, T],
 *   int64 in device memory.  An empty sample is allowed.  Rows before the
 *   first offset and behind the last one are padding.  (Offsets that
 *   decrease or leave [0, T] give undefined results, but no access out of
 *   the arrays.)
 * - Logits z[t][l][e] may have any strides over tokens and layers; experts
 *   are adjacent.  An expert is available to a token when its logit is
 *   neither -inf nor NaN; a mask is -inf.  The type's lowest finite value is
 *   an ordinary, very low logit.
 * - Ids outside [0, E) mark a choice that was not made: such a choice counts
 *   nowhere and its gate and gate gradient are 0.
 * - Calls whose logits have 2^59 elements and more (broadcast ones can) give
 *   E_UNSUPPORTED.
 * - Scores, sums and gradients are formed in 32 bits or more and rounded
 *   once, to the output's type.  An exponential e^(z - m) of a chosen expert's
 *   gate, and of fp32 logits' gradient, is good to 4 steps of 32 bits beside
 *   the rounding of z - m; one that enters a row's sum in the forward call, a
 *   share, or the gradient of 16-bit logits is off by up to 1.3 |z - m| + 2
 *   steps of itself.  Results do not depend on the launch: no floating-point
 *   atomics.
 */
#ifndef ROUTEPACK_ROUTER_H
#define ROUTEPACK_ROUTER_H

#include "routepack.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of logits and of ids. */
#define ROUTEPACK_F32  0
#define ROUTEPACK_BF16 1
#define ROUTEPACK_F16  2
#define ROUTEPACK_U8   3
#define ROUTEPACK_I16  4
#define ROUTEPACK_I32  5
#define ROUTEPACK_I64  6

/* Scores of an expert: softmax over the token's experts, or the logistic
 * function of its own logit. */
#define ROUTEPACK_SOFTMAX 0
#define ROUTEPACK_SIGMOID 1

/* Router logits, [n_tokens][L][E] with strides in elements (>= 0). */
typedef struct routepack_logits {
    const void *data;
    int32_t type;  /* ROUTEPACK_F32, _BF16 or _F16 */
    int64_t n_tokens;
    int64_t token_stride, layer_stride;
} routepack_logits;

/* Recorded expert ids, [n_tokens][L][k] with strides in elements (>= 0). */
typedef struct routepack_ids {
    const void *data;
    int32_t type;  /* ROUTEPACK_U8, _I16, _I32 or _I64 */
    int64_t n_tokens;
    int64_t token_stride, layer_stride;
} routepack_ids;

/* The gates of every token's k experts.
 * With replay == NULL the experts are chosen: the k available ones of largest
 * logit, or, given a bias, of largest score + bias (compared in 64 bits; the
 * bias takes no part in the gates, and -inf or NaN there bars its expert; a
 * NaN logit takes no part in the softmax scores that a bias is added to, and
 * experts of +inf share those alone, in equal parts);
 * ties go to the lowest index, largest first, and -1 stands where none is
 * left.  With replay the experts are those of the record (a repeated expert
 * has a gate for each mention).  Gates: scale times the chosen experts'
 * scores, divided by their sum over the token's choices when `normalize`
 * (all 0 when every one of them is unavailable).  A NaN logit makes NaN the
 * gates that its score enters (all of its token's under an unnormalised
 * softmax), and so does +inf under a softmax.
 *   replay   the record, or NULL
 *   bias     float [L][E] or NULL (with replay: NULL)
 *   ids      int32 [T][L][k] out (ignored with replay: may be NULL)
 *   gates    float [T][L][k] out
 * E_INVALID on null pointers, a negative size or stride, k outside [1, E], an
 * unknown type or score, a scale that is not finite, a bias with a replay, or
 * a replay of another number of tokens; E_UNSUPPORTED when E > 2048 or
 * k > 32. */
int routepack_route_tokens(const routepack_problem *prob, const routepack_logits *logits,
                           const routepack_ids *replay, const float *bias, int32_t score,
                           int32_t normalize, float scale, int32_t *ids, float *gates,
                           hipStream_t stream);

/* routepack_route_tokens, choosing among a few groups of experts: n_groups
 * groups of E / n_groups adjacent experts, of which each token keeps the `keep`
 * of largest sum of their group_top largest keys (of the available ones; a
 * group without any is not kept; ties go to the lowest group).  The keys are
 * score + bias, or the scores without a bias, compared in 64 bits; with
 * group_top = 1 and no bias they are compared as logits.  The gates are
 * routepack_route_tokens': an unnormalised softmax is over all experts.
 *   bias     float [L][E] or NULL, as there
 *   ids      int32 [T][L][k] out
 *   gates    float [T][L][k] out
 * Errors as there, and E_INVALID when n_groups < 1 does not divide E, keep is
 * outside [1, n_groups], group_top is neither 1 nor 2, or k exceeds the experts
 * of `keep` groups; E_UNSUPPORTED when E > 1024 or n_groups > 64 (a wave holds a
 * token in lanes of whole groups, with their number rounded up to a power of two:
 * of 2048 experts that may be twice what it has room for). */
int routepack_route_grouped(const routepack_problem *prob, const routepack_logits *logits, const float *bias,
                            int32_t n_groups, int32_t keep, int32_t group_top, int32_t score,
                            int32_t normalize, float scale, int32_t *ids, float *gates,
                            hipStream_t stream);

/* The demand of routepack.h from recorded ids:
 *   demand[i][l][e] = #{(t, j): t in sample i, ids[t][l][j] = e}.
 *   offsets  int64 [N + 1]
 *   demand   int32 [N][L][E] out
 * E_INVALID on null pointers, a negative size or stride, k < 1 or an unknown
 * type; E_UNSUPPORTED when E > 16384, k > 256 or T k >= 2^31 (a count would not
 * fit). */
int routepack_count_demand(const routepack_problem *prob, const routepack_ids *ids,
                           const int64_t *offsets, int32_t *demand, hipStream_t stream);

/* Bytes of workspace that routepack_balance_loss needs for n_tokens tokens
 * in n_groups groups, or ROUTEPACK_E_INVALID (E_UNSUPPORTED where that number
 * does not fit 64 bits). */
int64_t routepack_balance_workspace(const routepack_problem *prob, int64_t n_tokens, int32_t n_groups);

/* The balance loss of every layer, a mean over groups of tokens (the samples
 * of a row, or one group for a whole window):
 *   f[g][l][e]      = E counts[g][l][e] / sum_e' counts[g][l][e'] (0 where the sum is 0)
 *   shares[g][l][e] = mean over the group's tokens of s_e / sum_e' s_e' with
 *                     the scores s of the token (0 for an empty group, and a
 *                     token with no available expert adds 0; a NaN score,
 *                     or +inf under a softmax, makes its group's NaN)
 *   loss[l]         = 1/G sum_g sum_e f[g][l][e] shares[g][l][e].
 * The counts are constants to the loss (they may be summed over ranks).
 *   offsets    int64 [G + 1], G = n_groups
 *   counts     [G][L][E] of counts_type (ROUTEPACK_I32 or _I64), >= 0:
 *              a demand, or an aggregate of routepack_aggregate_demand
 *   loss       float [L] out
 *   shares     float [G][L][E] out
 *   workspace  at least routepack_balance_workspace bytes, 16-byte aligned,
 *              for this call alone until its work has ended
 * E_INVALID on null pointers, a negative size or stride, G < 1, an unknown
 * type or score, or a workspace too small or misaligned; E_UNSUPPORTED when
 * E > 2048. */
int routepack_balance_loss(const routepack_problem *prob, const routepack_logits *logits,
                           int32_t n_groups, const int64_t *offsets, const void *counts,
                           int32_t counts_type, int32_t score, float *loss, float *shares,
                           void *workspace, int64_t workspace_bytes, hipStream_t stream);

/* The gradient of a scalar with respect to the logits, given its gradients
 * with respect to the gates of routepack_route_tokens (ids are constants) and
 * to the losses of routepack_balance_loss (counts are constants); either part
 * may be absent (its ids, or its dloss, NULL), not both.
 *   ids        the chosen or replayed experts, or NULL
 *   dgates     float [T][L][k] (with ids)
 *   normalize, scale   as in the forward call
 *   n_groups, offsets, counts, counts_type   as in the forward call (with dloss)
 *   dloss      float [L] or NULL
 *   dlogits    [T][L][E] out, of the logits' type, not overlapping them; rows
 *              that are padding get the gates' part alone, and unavailable
 *              experts 0 (NaN where a NaN logit, or +inf under a softmax,
 *              enters the sum over the row or over the choices)
 * Errors as routepack_route_tokens and routepack_balance_loss. */
int routepack_route_backward(const routepack_problem *prob, const routepack_logits *logits,
                             const routepack_ids *ids, const float *dgates, int32_t normalize,
                             float scale, int32_t n_groups, const int64_t *offsets,
                             const void *counts, int32_t counts_type, const float *dloss,
                             int32_t score, void *dlogits, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* ROUTEPACK_ROUTER_H */
