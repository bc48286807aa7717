/* Expert layers of large language models: products grouped by expert, products
 * with 4-bit weights, routing and the weighted sum of answers.  Same library,
 * same conventions (device pointers, streams, workspaces, flags, status values)
 * as emu.h. */
#ifndef EMU_EXPERTS_H
#define EMU_EXPERTS_H

#include "emu.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EMU_FLAG_INDEX     0x10u /* a row index or group end lies outside its range (or group ends
                                    decrease); such rows count as zero rows, such ends are clamped */

/* Element types of the expert-layer entry points. */
#define EMU_F32  0
#define EMU_BF16 1
#define EMU_I32  2   /* results of emu_i8_gemm alone */

/* Added to the first argument (type or slices) of emu_grouped_split,
 * emu_grouped_split_rows, emu_grouped_prodsum and emu_grouped_prodsum_wgrad: the
 * call adds its flags to those in the workspace instead of starting anew, so
 * that one word reports a product and the splits of its operands. */
#define EMU_KEEP_FLAGS 0x100

/* ---------------------------------------------------------------------------
 * Expert layers: matrix products grouped by expert, of ragged sizes.
 *
 * `rows` token rows are ordered by group (expert): group g owns the rows
 * ends[g-1] .. ends[g]-1 (ends[-1] = 0; device int32[G], non-decreasing, at
 * most rows).  Groups may be empty; rows from ends[G-1] on belong to no group:
 * they contribute nothing and their result rows are zero.  Group sizes are
 * read on the device, nothing synchronises with the host.  1 <= G <= 1024; rows,
 * K and N (M and N) each below 2^31 - 65536.
 *
 * Operands are plane sets of nslices BF16 planes: 3 for FP32 operands (the
 * split of Eq. (fp32split); products are Eq. (fp32six), FP32 accumulation), 1
 * for BF16 operands (exact products, one rounding to the result's type).  Sums are
 * in FP32: for FP32 results rounded every 256 terms, for BF16 results in one
 * accumulator, to which the tensor cores add with truncation (1.6e-4 of a result
 * over 32768 terms of one sign, before the rounding to BF16's 8 bits).  BF16 token rows and weights whose base is 16-byte aligned
 * and whose row pitch and matrix distance are multiples of 8 elements are such
 * a plane as they stand.
 * ------------------------------------------------------------------------- */

/* Rows of a padded token plane: every group starts at a multiple of 16 rows
 * and is followed by zero rows up to one. */
int64_t emu_grouped_plane_rows(int64_t rows, int64_t G);

/* Planes of G weight matrices X_g (rows x cols, row pitch ldx, stridex
 * elements apart; dtype EMU_F32 or EMU_BF16): comps [S][G*rows][ldcomp],
 * S = 3 (FP32) or 1 (BF16), ldcomp a multiple of 8 and >= cols.  One plane
 * set serves the product (op N or T) and both gradients.  ws: at least
 * emu_split_workspace_bytes(32).  Flags: EMU_FLAG_NONFINITE, EMU_FLAG_SLICE. */
emu_status emu_grouped_split(int dtype, int64_t G, int64_t rows, int64_t cols, const void *X, int64_t ldx,
                             int64_t stridex, uint16_t *comps, int64_t ldcomp, void *ws, size_t ws_bytes,
                             emu_stream_t stream);

/* Planes of token rows in group order at padded positions: plane row of token
 * row r is X[src[r]] (src: device int32[rows], values 0 .. xrows-1), or X[r]
 * with src NULL (xrows >= rows); comps [S][emu_grouped_plane_rows(rows, G)][ldcomp].
 * Flags: as above, and EMU_FLAG_INDEX. */
emu_status emu_grouped_split_rows(int dtype, int64_t rows, int64_t cols, const void *X, int64_t xrows, int64_t ldx,
                                  const int32_t *src, const int32_t *ends, int64_t G, uint16_t *comps,
                                  int64_t ldcomp, void *ws, size_t ws_bytes, emu_stream_t stream);

/* Y[r] = X[r] op(W_g) for every row r of group g: X (rows x K) planes
 * (padded = 1: from emu_grouped_split_rows with the same rows, G and ends, so of
 * emu_grouped_plane_rows(rows, G) rows each; 0: rows in their own order), W_g
 * K x N (EMU_OP_N) or N x K (EMU_OP_T) planes, not overlapping, dense over the
 * groups when nslices = 3.  Y: rows x N of ytype, row pitch ldy, any alignment.  The
 * gradient with respect to X is the same call with dY for X and the other op.
 * K = 0 writes zeros.  ws: at least emu_split_workspace_bytes(32).  Flags:
 * EMU_FLAG_INDEX, EMU_FLAG_TIMEOUT. */
emu_status emu_grouped_prodsum(int nslices, int opW, int64_t G, int64_t rows, int64_t N, int64_t K,
                               const uint16_t *Xcomps, int64_t ldx, int padded, const uint16_t *Wcomps, int64_t ldw,
                               int64_t stridew, const int32_t *ends, void *Y, int ytype, int64_t ldy, void *ws,
                               size_t ws_bytes, emu_stream_t stream);

/* The same on FP32 operands in memory (any alignment), split and multiplied
 * in one call; src as in emu_grouped_split_rows, ws at least
 * emu_grouped_gemm_workspace_bytes. */
size_t emu_grouped_gemm_workspace_bytes(int dtype, int64_t G, int64_t rows, int64_t N, int64_t K);
emu_status emu_grouped_gemm_f32(int opW, int64_t G, int64_t rows, int64_t N, int64_t K, const float *X, int64_t xrows,
                                int64_t ldx, const int32_t *src, const float *W, int64_t ldw, int64_t stridew,
                                const int32_t *ends, float *Y, int64_t ldy, void *ws, size_t ws_bytes,
                                emu_stream_t stream);

/* Weight gradient: D_g = A_g^T B_g over the rows of group g, from planes of A
 * (rows x M) and B (rows x N): apadded / bpadded as in emu_grouped_prodsum, 1
 * for both when nslices = 3.  D: G matrices M x N of dtype, row pitch ldd,
 * strided elements apart; empty groups write zeros.  With A = X, B = dY this is the gradient of W for
 * EMU_OP_N, with A = dY, B = X for EMU_OP_T. */
emu_status emu_grouped_prodsum_wgrad(int nslices, int64_t G, int64_t rows, int64_t M, int64_t N,
                                     const uint16_t *Acomps, int64_t lda, int apadded, const uint16_t *Bcomps,
                                     int64_t ldb, int bpadded, const int32_t *ends, void *D, int dtype, int64_t ldd,
                                     int64_t strided, void *ws, size_t ws_bytes, emu_stream_t stream);

/* Matrix-vector products with 4-bit weights and group scales, for one row or a
 * few rows (of each expert):
 *   Y[r, n] = sum_k X[r, k] (q[g, n, k] - z[g, n, k/group]) s[g, n, k/group]
 * for every row r of group g.  q: unsigned 4-bit codes, uint8 [G][N][K/2], the
 * even k in the low half of a byte; s: stype [G][N][K/group]; z: uint8
 * [G][N][K/group] with values 0 .. 15 (the low half counts), or NULL for 8
 * throughout.  group: a multiple of 32 that divides K.  X: rows x K and Y:
 * rows x N of dtype (EMU_F32: FP32 rows as their three BF16 slices, exact
 * products; EMU_BF16), any alignment; sums in FP32.  ends as above, or NULL
 * with G = 1: one matrix for all rows.  Values in ends outside 0 .. rows or
 * decreasing are clamped.  Rows of no group are zero.  Up to
 * 131070 rows are computed; the weights are read again for every 24 (BF16) or 8
 * (FP32) of an expert.  q 16-byte aligned.  ws: emu_w4_workspace_bytes, 16-byte aligned, for
 * X's slices; for BF16 rows of 16-byte aligned base and pitch
 * emu_split_workspace_bytes(32) are enough (the flags), or NULL, which reports none.
 * An FP32 value of 0x1.FFp+127 or more (in magnitude) has slices that are not
 * finite, and a row with one comes out as NaN.  Flags: EMU_FLAG_INDEX,
 * EMU_FLAG_NONFINITE and EMU_FLAG_SLICE (of all of X, FP32). */
size_t emu_w4_workspace_bytes(int dtype, int64_t rows, int64_t K);
emu_status emu_w4_matvec(int dtype, int64_t G, int64_t rows, int64_t N, int64_t K, int64_t group, const void *X,
                         int64_t ldx, const uint8_t *q, const void *s, int stype, const uint8_t *z,
                         const int32_t *ends, void *Y, int64_t ldy, void *ws, size_t ws_bytes, emu_stream_t stream);

/* Routing of T tokens to the k of E experts with the largest logits (dtype,
 * T x E, row pitch ldl; ties: the lower index; NaN counts as minus infinity):
 *   experts [T][k] by falling logit; weights [T][k] FP32, the softmax over the
 *   chosen (renorm = 1) or over all experts (renorm = 0), 0 where the logit is
 *   minus infinity (all of a token's where all its logits are);
 * and the order of the T k assignments by expert, then token, then rank:
 *   slots [T][k] the place of each in that order, rows [T k] the token at each
 *   place, ends [E] the places' ends by expert, as the grouped calls take them.
 * 1 <= k <= 32, k <= E <= 1024, T k < 2^31 - 65536.  Deterministic.  ws: at least
 * emu_route_workspace_bytes.  Flags: EMU_FLAG_NONFINITE (a logit is NaN or plus
 * infinity), EMU_FLAG_TIMEOUT (slots, rows and ends are then not whole). */
size_t emu_route_workspace_bytes(int64_t T, int64_t E, int64_t k);
emu_status emu_route(int dtype, int64_t T, int64_t E, int64_t k, int renorm, const void *logits, int64_t ldl,
                     float *weights, int32_t *experts, int32_t *slots, int32_t *rows, int32_t *ends, void *ws,
                     size_t ws_bytes, emu_stream_t stream);

/* Watchdog self-test of emu_route (FP32, renorm = 1, more than 32 tokens): its
 * blocks wait, timeout_us microseconds at most (1 .. 10^6), for one more than there
 * are, set EMU_FLAG_TIMEOUT and return; slots, rows and ends are not written. */
emu_status emu_selftest_route_timeout(uint32_t timeout_us, int64_t T, int64_t E, int64_t k, const float *logits,
                                      int64_t ldl, float *weights, int32_t *experts, int32_t *slots, int32_t *rows,
                                      int32_t *ends, void *ws, size_t ws_bytes, emu_stream_t stream);

/* Gradient of the weights' softmax: dlogits (T x E of dtype, row pitch lddl,
 * all entries written) from the weights' gradients dweights [T][k] and the
 * experts that emu_route chose for the same logits and renorm. */
emu_status emu_route_backward(int dtype, int64_t T, int64_t E, int64_t k, int renorm, const void *logits, int64_t ldl,
                              const int32_t *experts, const float *dweights, void *dlogits, int64_t lddl,
                              emu_stream_t stream);

/* Weighted sum of the answers: O[t] = sum_j weights[t, j] Y[slots[t, j]], j
 * ascending in FP32, one rounding to dtype.  Y: yrows x cols, O: T x cols of
 * dtype; weights [T][k] FP32, or NULL for 1 throughout (the gradient of a
 * gather of token rows).  A slot outside 0 .. yrows-1 contributes nothing. */
emu_status emu_rows_combine(int dtype, int64_t T, int64_t k, int64_t cols, const void *Y, int64_t yrows, int64_t ldy,
                            const int32_t *slots, const float *weights, void *O, int64_t ldo, emu_stream_t stream);

/* Its gradients: dY[slots[t, j]] = weights[t, j] dO[t] (dY: yrows x cols; rows
 * that no slot names are not written; no two slots may name the same row) and
 * dweights[t, j] = Y[slots[t, j]] . dO[t] in FP32 (0 for a slot outside), or
 * dweights NULL when they are not wanted (Y is then not read). */
emu_status emu_rows_combine_backward(int dtype, int64_t T, int64_t k, int64_t cols, const void *dO, int64_t lddo,
                                     const void *Y, int64_t yrows, int64_t ldy, const int32_t *slots,
                                     const float *weights, void *dY, int64_t lddy, float *dweights,
                                     emu_stream_t stream);

/* The same, and zeros in the rows of dY that no slot names: all of dY is
 * written.  ws: at least emu_rows_combine_workspace_bytes, 16-byte aligned. */
size_t emu_rows_combine_workspace_bytes(int64_t yrows);
emu_status emu_rows_combine_backward_full(int dtype, int64_t T, int64_t k, int64_t cols, const void *dO, int64_t lddo,
                                          const void *Y, int64_t yrows, int64_t ldy, const int32_t *slots,
                                          const float *weights, void *dY, int64_t lddy, float *dweights, void *ws,
                                          size_t ws_bytes, emu_stream_t stream);

/* Balance loss of a routing: with the n tokens t whose mask[t] is not 0 (mask: device
 * uint8[T]; NULL: all), p_t the softmax of token t's logits over all experts, counts[e]
 * their assignments to expert e (experts [T][k], as emu_route gives them), P_e the mean of p_te:
 *   loss = coef E / (n k) sum_e counts[e] P_e, 0 for n = 0
 * (device float; 1 x coef for a perfectly even routing).  counts: device int32[E],
 * tokens: device int32, n.  NaN counts as a logit of minus infinity; a token whose
 * logits all are has p = 0.  An entry of experts outside 0 .. E-1 is not counted.
 * 1 <= k <= 32, k <= E <= 1024, T k < 2^31 - 65536.  Sums in FP32, in an order that depends
 * on the sizes alone: same inputs, same bits.  ws: at least
 * emu_route_balance_workspace_bytes, 16-byte aligned, not shared by calls in flight at once; where
 * that is 0, emu_split_workspace_bytes(32) for the flags, or NULL, which reports none.
 * Flags: EMU_FLAG_NONFINITE (a counted token's logit is NaN or plus infinity),
 * EMU_FLAG_INDEX. */
size_t emu_route_balance_workspace_bytes(int64_t T, int64_t E);
emu_status emu_route_balance(int dtype, int64_t T, int64_t E, int64_t k, const void *logits, int64_t ldl,
                             const int32_t *experts, const uint8_t *mask, float coef, float *loss, int32_t *counts,
                             int32_t *tokens, void *ws, size_t ws_bytes, emu_stream_t stream);

/* Its gradient, counts being constants:
 *   dlogits[t, e] = add[t, e] + dloss / n p_te (f_e - sum_e' f_e' p_te'), f_e = coef E / (n k) counts[e],
 * without the second term where mask[t] is 0.  counts, tokens: those of emu_route_balance for the same
 * logits and mask.  dloss: device float, NULL for 1.  add: T x E of dtype (a gradient
 * of the same logits; may be dlogits itself, then with the same pitch), or NULL for 0; it
 * may not overlap dlogits otherwise.  One rounding to dtype; all of dlogits is written. */
emu_status emu_route_balance_backward(int dtype, int64_t T, int64_t E, int64_t k, const void *logits, int64_t ldl,
                                      const int32_t *counts, const int32_t *tokens, const uint8_t *mask, float coef,
                                      const float *dloss, const void *add, int64_t lda, void *dlogits, int64_t lddl, emu_stream_t stream);

/* Rows to 8-bit integers: scales[g, r] = max_k |X[g, r, k]| / 127 in FP32 and
 * codes[g, r, k] = X / scale rounded to the nearest integer, ties to even, exactly, clamped to
 * -127 .. 127 (which only subnormal scales need).  A row whose scale is 0 has zero codes; one with a NaN or
 * infinity has zero codes and a NaN for its scale.  X: G matrices of rows x cols of dtype, row
 * pitch ldx, stridex apart, any alignment; codes likewise int8; scales FP32 [G][rows].  Rows of the
 * result may not overlap.  ws: for the flags (emu_split_workspace_bytes(32)), or NULL, which reports none.
 * Flags: EMU_FLAG_NONFINITE. */
emu_status emu_i8_quantize(int dtype, int64_t G, int64_t rows, int64_t cols, const void *X, int64_t ldx, int64_t stridex,
                           int8_t *codes, int64_t ldq, int64_t strideq, float *scales, void *ws, size_t ws_bytes,
                           emu_stream_t stream);

/* Products in 8-bit integers with a scale for each token and each channel, dense or
 * grouped by expert:
 *   Y[r, n] = (sum_k X[src[r], k] W[g, n, k]) wscales[g, n] xscales[src[r]]
 * for the rows r of group g (ends as above; NULL with G = 1: one matrix for all rows;
 * src NULL: row r itself, xrows >= rows).  The sum is exact: codes are -128 .. 127 and
 * K <= 131071.  It is rounded to FP32, multiplied by the channel's and then by the token's
 * scale (NULL: 1) and rounded to ytype (EMU_F32, EMU_BF16); EMU_I32 gives the sums themselves and
 * takes no scales.  X: xrows x K, W: G matrices N x K, stridew apart, int8 of any alignment:
 * read as they stand where base, row pitch and distance are multiples of 16 bytes and W's matrices do
 * not overlap, and copied first otherwise where more than a few rows meet.  xscales [xrows], wscales
 * [G][N] FP32.  Rows of no group, and rows whose src is outside 0 .. xrows-1, are zero whatever the
 * scales are.  aligned: whether both X and W are such (0 is enough for any).  ws: at least emu_i8_gemm_workspace_bytes, 16-byte
 * aligned, not shared by calls in flight at once; where that is 0, emu_split_workspace_bytes(32) for the
 * flags, or NULL, which reports none.  Flags: EMU_FLAG_INDEX, EMU_FLAG_TIMEOUT. */
size_t emu_i8_gemm_workspace_bytes(int64_t G, int64_t rows, int64_t N, int64_t K, int aligned);
emu_status emu_i8_gemm(int64_t G, int64_t rows, int64_t N, int64_t K, const int8_t *X, int64_t xrows, int64_t ldx,
                       const float *xscales, const int32_t *src, const int8_t *W, int64_t ldw, int64_t stridew,
                       const float *wscales, const int32_t *ends, void *Y, int ytype, int64_t ldy, void *ws,
                       size_t ws_bytes, emu_stream_t stream);

/* Watchdog self-test of emu_i8_gemm (with a workspace, at sizes whose products are one launch on single
 * SMs; others are unsupported): nothing is multiplied, a wait runs out after timeout_us microseconds (1 .. 10^6) and sets
 * EMU_FLAG_TIMEOUT beside the call's other flags; rows of groups keep what they hold. */
emu_status emu_selftest_i8_timeout(uint32_t timeout_us, int64_t G, int64_t rows, int64_t N, int64_t K, const int8_t *X,
                                   int64_t xrows, int64_t ldx, const float *xscales, const int32_t *src, const int8_t *W,
                                   int64_t ldw, int64_t stridew, const float *wscales, const int32_t *ends, void *Y,
                                   int ytype, int64_t ldy, void *ws, size_t ws_bytes, emu_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif
