/*
 * routepack/experts.h -- C-ABI of the experts' operators (gfx950).
 *
 * What follows the router of router.h: the order that puts each expert's
 * (token, choice) pairs side by side, matrices in microscaled 4-bit floating
 * point, the experts' products on them with their gradients, and the sum of a
 * token's experts under its gates with its gradients.
 *
 * Conventions, besides those of routepack.h and router.h
 * -------------------------------------------------------
 * - Every call is asynchronous on `stream`, allocates nothing, and may be
 *   captured into a graph.  The current device is the stream's.
 * - P = T k pairs; pair p = t k + j is token t's choice j.  An order of them has
 *     rows[r]     the pair that stands in row r, or -1 behind the last pair made
 *     offsets[s]  the first row of slot s (int64, E + 1 of them, offsets[0] = 0)
 *     places[t][j]  the row of the pair, or -1 where no choice was made.
 *   The slots are the experts, or where the planner placed them.  Offsets that
 *   decrease or leave the rows, and rows or places outside their range, give
 *   undefined results but no access out of the arrays; rows outside every slot
 *   are 0 in what is written.
 * - A matrix in 4 bits: columns in blocks of 32, a row padded to a multiple of
 *   128 columns by zero codes (and scale bytes 0).  A code is sign (bit 3), two
 *   bits of exponent and one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6.  codes[r][c / 2]
 *   holds columns c (low half) and c + 1; scales[r][c / 32] = x stands for 2^(x - 127),
 *   255 for a block of NaN.  (These are the element and scale formats of the
 *   OCP microscaling specification, MXFP4.)
 * - Sums are formed in 32 bits or more and rounded once, to the output's type.
 *   No floating-point atomics: results do not depend on the launch.
 * - Sizes whose bytes would leave 2^62 give E_UNSUPPORTED.
 */
#ifndef ROUTEPACK_EXPERTS_H
#define ROUTEPACK_EXPERTS_H

#include "router.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A matrix [n_rows][n_cols] of ROUTEPACK_F32, _BF16 or _F16, columns adjacent,
 * row_stride in elements (>= 0 for inputs; outputs are dense). */
typedef struct routepack_matrix {
    void *data;
    int32_t type;
    int64_t n_rows, n_cols, row_stride;
} routepack_matrix;

/* A matrix in 4 bits, [n_rows][n_cols], dense; codes 16-byte and scales 4-byte
 * aligned (as runs of a larger matrix's rows are). */
typedef struct routepack_mx {
    void *codes;   /* uint8 [n_rows][64 ceil(n_cols / 128)] */
    void *scales;  /* uint8 [n_rows][4 ceil(n_cols / 128)] */
    int64_t n_rows, n_cols;
} routepack_mx;

/* Bytes of workspace that routepack_order_tokens needs for n_tokens tokens (0 for
 * few), or an error of it. */
int64_t routepack_order_workspace(const routepack_problem *prob, int64_t n_tokens);

/* The order of every layer's pairs by slot, and by pair within a slot.
 *   ids        [T][L][k], any strides; an id outside [0, E) is no choice
 *   slots      int32 [L][E], the slot of each expert (as routepack_place_experts
 *              gives them), or NULL: an expert's slot is its index.  A slot
 *              outside [0, E) makes its expert's pairs no choices
 *   rows       int32 [L][T k] out
 *   offsets    int64 [L][E + 1] out
 *   places     int32 [T][L][k] out
 *   workspace  at least routepack_order_workspace bytes, 16-byte aligned, for
 *              this call alone until its work has ended (may be NULL where those are 0)
 * E_INVALID on null pointers, a negative size or stride, E < 1, k < 1, an
 * unknown type, or a workspace too small or misaligned; E_UNSUPPORTED when
 * E > 2048, k > 256, T k >= 2^31, or the layers' pairs, each layer's in chunks of
 * 4096 and seven more, make 2^22 chunks. */
int routepack_order_tokens(const routepack_problem *prob, const routepack_ids *ids, const int32_t *slots,
                           int32_t *rows, int64_t *offsets, int32_t *places, void *workspace,
                           int64_t workspace_bytes, hipStream_t stream);

/* A matrix into 4 bits.  A block's exponent is that of its largest magnitude
 * less 2 (at least -127); its values, divided by that power of two, are rounded
 * to the nearest code, ties to the even one, and end at 6.  A block with NaN or
 * an infinity is NaN (codes 0, scale 255), a block of zeros has scale 0.
 *   rows, places  NULL, or an order: q's row r is the row of x of the token of
 *         pair rows[r], where that pair's place is r, else zeros.  rows int32
 *         [q.n_rows]; places [x.n_rows][1][k] of ROUTEPACK_I32 (the layer stride is
 *         not looked at)
 * E_INVALID on null pointers, a negative size or stride, an unknown type, other
 * columns in q than in x, one of rows and places, places of other tokens than x's
 * rows or k < 1 with them, other rows without them, or q misaligned;
 * E_UNSUPPORTED when n_cols > 2^24, k > 256 or x.n_rows k >= 2^31. */
int routepack_quantize_mx(const routepack_matrix *x, const int32_t *rows, const routepack_ids *places,
                          int32_t top_k, const routepack_mx *q, hipStream_t stream);

/* The values of a matrix in 4 bits, in x's type (exact in fp32 and bf16; in
 * fp16 rounded, and infinite beyond its range).  x's row_stride is n_cols.
 * Errors as routepack_quantize_mx. */
int routepack_dequantize_mx(const routepack_mx *q, const routepack_matrix *x, hipStream_t stream);

/* Each slot's rows times its matrix:
 *   y[r][n] = sum_c x[r][c] w[s][n][c]   for r in [offsets[s], offsets[s + 1]).
 *   x        n_rows x C;  w  (n_slots N) x C;  offsets  int64 [n_slots + 1]
 *   y        n_rows x N out, row_stride N
 * E_INVALID on null pointers, a negative size, n_slots < 1, w rows that are not
 * a multiple of it, other columns or rows, an unknown type, or x or w
 * misaligned; E_UNSUPPORTED when n_slots > 2048, n_cols > 2^24 or N > 2^24. */
int routepack_expert_product(const routepack_mx *x, const routepack_mx *w, int32_t n_slots, const int64_t *offsets,
                             const routepack_matrix *y, hipStream_t stream);

/* The gradients of that product, given its gradient dy (n_rows x N, any
 * row_stride):
 *   dx[r][c]    = sum_n dy[r][n] w[s][n][c]               n_rows x C out, or NULL
 *   dw[s][n][c] = sum over slot s's r of dy[r][n] x[r][c]   (n_slots N) x C out, or NULL
 * both of dy's type, row_stride C; not both NULL.  The products are exact: dy is
 * split into bf16 parts (fp32 values below 2^-110 are cut to multiples of 2^-133,
 * where bf16 ends).  x is read for dw alone (else its pointers may be
 * null), w for dx alone.
 * Errors as routepack_expert_product. */
int routepack_expert_product_backward(const routepack_matrix *dy, const routepack_mx *x, const routepack_mx *w,
                                      int32_t n_slots, const int64_t *offsets, const routepack_matrix *dx,
                                      const routepack_matrix *dw, hipStream_t stream);

/* The sum of a token's rows under its gates, in the order of its choices:
 *   out[t] = sum_j gates[t][j] y[places[t][j]]   over places in [0, y.n_rows).
 *   places  [T][1][k] of ROUTEPACK_I32 (the layer stride is not looked at)
 *   gates   float [T][k] with gate_stride elements between tokens, or NULL: ones
 *   out     T x C, of y's type, row_stride C
 * E_INVALID on null pointers, a negative size or stride, k < 1, an unknown type,
 * or other sizes or types; E_UNSUPPORTED when k > 32, C > 2^24 or T k >= 2^31. */
int routepack_combine_tokens(const routepack_matrix *y, const routepack_ids *places, int32_t top_k,
                             const float *gates, int64_t gate_stride, const routepack_matrix *out,
                             hipStream_t stream);

/* The gradients of that sum, given its gradient dout (T x C):
 *   dy[r]        = gates[t][j] dout[t], t k + j = rows[r], where that pair's place
 *                  is r, else 0                       y.n_rows x C out, row_stride C
 *   dgates[t][j] = sum_c y[places[t][j]][c] dout[t][c], 0 for no choice   float [T][k] out
 * either may be NULL, not both; y is read for dgates alone (else its data may be
 * null), rows (int32 [y.n_rows]) for dy alone.
 * Errors as routepack_combine_tokens. */
int routepack_combine_backward(const routepack_matrix *dout, const routepack_matrix *y, const int32_t *rows,
                               const routepack_ids *places, int32_t top_k, const float *gates, int64_t gate_stride,
                               const routepack_matrix *dy, float *dgates, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* ROUTEPACK_EXPERTS_H */
