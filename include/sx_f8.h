/* libsx layer body with operands in 8-bit floating point: the row-sparse layer body of include/sx.h
 * (sx_rmsnorm_rows, sx_gemm_rows, sx_silu_mul_rows) with 8-bit products, for a plan's row lists and for
 * the plain rows of a decoding step, and the feed-forward module as a mixture of experts.  One layer:
 *
 *   sx_add_rmsnorm_f8   residual addition and RMSNorm, rounded to 8 bits for the next product (without
 *                       gamma: rounded only, as for the attention's output)
 *   sx_gemm_f8          product with an 8-bit weight of one to four stacked parts, residual added
 *   sx_silu_mul_f8      SwiGLU of a gate|up product, rounded to 8 bits
 *
 * and where the feed-forward module is a mixture of experts, after the router's logits:
 *
 *   sx_moe_route        every row's top experts and their weights; the rows' places grouped by expert
 *   sx_gemm_experts_f8  gate|up product of the grouped rows, each with its expert's weight; sx_silu_mul_f8;
 *                       sx_gemm_experts_f8 again, down
 *   sx_moe_combine      weighted sum of every row's experts, added to the residual stream
 *
 * sx_f8_pack_weight rounds a bfloat16 weight to 8 bits, once.
 *
 * Status, streams, memory ownership and sx_last_error are as in include/sx.h: no call allocates,
 * synchronises the host, aborts or throws; every tensor is caller-owned DEVICE memory on the current
 * device, 16-byte aligned but for rows and n_rows (4 bytes).  Nothing is kept between calls: calls may run at the
 * same time on any streams when their outputs and workspaces differ, and any of them can be captured into
 * a graph.  An output must not overlap another argument of its call (SX_EINVAL) but where this says so.
 * Index arrays in device memory are trusted by the release library, but an entry that is out of range is
 * left out and never followed; the checked library refuses it with SX_EDEVICE, which cannot be done while
 * the stream is captured.
 *
 * The 8-bit format.  128 consecutive elements of a row share a power of two 2^e, the smallest with
 * amax <= 448 * 2^e and -126 <= e <= 120, held as the byte e + 127.  An element is the nearest e4m3 number
 * (OCP e4m3fn: 4 bits of exponent, 3 of mantissa, largest 448), ties to even, times 2^e; it is off by at
 * most 2^-4 of its value, or 2^-10 * 2^e where it is below 2^-6 * 2^e.  A group with a NaN or an infinity
 * gets the byte 255 and codes 0 and stands for NaN in all its 128 elements: a product reads NaN in every
 * column of that row, and in no other row.  Products take any codes and scale bytes, such as weights
 * rounded elsewhere (bytes 0 .. 254: 2^-127 .. 2^127).
 *   rows      codes [..][k], scales [..][ld] bytes with ld = sx_f8_scale_ld(k): group g of a row at [g];
 *             the bytes behind a row's last group are written as 0 and never looked at
 *   weights   codes [n][k] (k contiguous), scales [n / 128][ld]: one byte for 128 x 128 elements
 * k and n are multiples of 128.
 *
 * Rows.  With a plan (bfloat16) rows, n_rows, max_rows and the addressing by slot or by token are those of
 * the layer body in include/sx.h; listed rows beyond their request are left out.  plan == NULL: `rows` must
 * be NULL, the rows are 0 .. max_rows - 1 of every array, or the first min(*n_rows, max_rows) of them where
 * n_rows (DEVICE [1]) is given, as in a padded batch; the by_token arguments say nothing then.  Rows not
 * listed, and rows behind the last one, are neither read nor written.  A call may have no rows at all: its arrays of rows
 * may then be NULL.
 *
 * Results: a call gives the same bits every time, and a row's results do not depend on the other rows of
 * the call, nor on how loose max_rows is: every product sums an element over k in one order, whatever tile
 * the call's size chooses.
 */
#ifndef SX_F8_H
#define SX_F8_H

#include "sx.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes between the scale rows of rows of k elements: k / 128 rounded up to a multiple of four. */
sx_status sx_f8_scale_ld(int32_t k, int32_t* ld);

/* Rounds a bfloat16 weight w [n][k] to 8 bits: codes [n][k], scales [n / 128][ld]. */
sx_status sx_f8_pack_weight(const void* w, int64_t n, int32_t k, void* codes, void* scales, void* stream);

/* For every row, with rows of h elements (h a multiple of 128):
 *   s = x[row] + delta[slot]                       rounded to bfloat16 (delta NULL: s = x)
 *   y = s / sqrt(mean s^2 + eps) * gamma           (gamma NULL: y = s, eps not read)
 *   x_out[row] = s      y16[y row] = y in bfloat16      y8, y_scale [y row] = y in 8 bits
 * x and x_out are addressed by x_by_token, delta by slot, y16, y8 and y_scale by y_by_token.  x_out, y16
 * may be NULL, and so may y8 and y_scale together; x_out may be x itself.  x_out needs delta, y16 needs gamma.
 * The norm is formed in float64 in a fixed order and rounded to float32, and from there to its outputs. */
sx_status sx_add_rmsnorm_f8(const sx_plan* plan, const int32_t* rows, const int32_t* n_rows, int32_t max_rows,
                            const void* x, int32_t x_by_token, const void* delta, const void* gamma, float eps,
                            int32_t h, void* x_out, void* y16, void* y8, void* y_scale, int32_t y_by_token,
                            void* stream);

/* SwiGLU activation, by slot: y[row][j] = silu(g) * u with g = gate_up[row][j], u = gate_up[row][f + j],
 * silu(g) = g / (1 + e^-g), in float32, rounded to 8 bits; gate_up [..][2f] bfloat16 (f a multiple of 128). */
sx_status sx_silu_mul_f8(const sx_plan* plan, const int32_t* n_rows, int32_t max_rows, const void* gate_up,
                         int32_t f, void* y8, void* y_scale, void* stream);

/* y[row] = x[row] . w^T (+ residual[row]) for rows x8, x_scale [..][k] and a weight of n_parts (1 .. 4) stacked
 * parts, w8 [sum part_n][k] and w_scale: columns of part i land in y_parts[i], [..][part_n[i]] bfloat16.  part_n
 * (host array) holds multiples of 128, y_parts is a host array of DEVICE pointers.  residual (nullable, one part
 * only) is bfloat16, addressed like y, and may be y itself.  Matrix cores with the blocks' scales, float32
 * accumulation, one rounding at the end; among eight consecutive elements the matrix cores cut products off 13 bits
 * below the largest one's exponent (2^-14.5 of a result over normal data).  k up to 65536. */
sx_status sx_gemm_f8(const sx_plan* plan, const int32_t* rows, const int32_t* n_rows, int32_t max_rows,
                     const void* x8, const void* x_scale, int32_t x_by_token, const void* w8, const void* w_scale,
                     int32_t k, int32_t n_parts, const int32_t* part_n, const void* residual, void* const* y_parts,
                     int32_t y_by_token, void* stream);

/* Bytes of workspace that sx_moe_route needs for n_requests (1 without a plan) of at most max_rows rows. */
sx_status sx_moe_route_workspace(int32_t n_experts, int32_t top_k, int32_t n_requests, int32_t max_rows,
                                 int64_t* bytes);

/* Routing, by slot, of rows of logits [..][n_experts] (SX_F32 or SX_BF16): the top_k largest of a row, the lower
 * index first among equals, and their softmax over all experts, or over the row's own top_k (renormalise != 0).
 *   ids      [..][top_k] int32, weights [..][top_k] float32
 *   offsets  [n_experts + 1] int32: the places of expert e are offsets[e] .. offsets[e + 1] - 1
 *   order    [slots * top_k] int32 (slots: sum T, or max_rows): place p holds slot * top_k + j of a row's j-th expert;
 *            the places of one expert are in ascending order.  Places from offsets[n_experts] on are left as they were.
 * A NaN logit is one of -inf.  A row of -inf alone takes the experts 0 .. top_k - 1 with weights 0; where a logit is
 * +inf, those that are share the weight.  n_experts <= 1024, top_k <= min(n_experts, 16), slots * top_k
 * below 2^31.  workspace: sx_moe_route_workspace bytes, 16-byte aligned, any content. */
sx_status sx_moe_route(const sx_plan* plan, const int32_t* n_rows, int32_t max_rows, const void* logits,
                       int32_t logits_dtype, int32_t n_experts, int32_t top_k, int32_t renormalise, int32_t* ids,
                       float* weights, int32_t* offsets, int32_t* order, void* workspace, int64_t workspace_bytes,
                       void* stream);

/* Products grouped by expert: for every expert e and every place p of offsets[e] .. offsets[e + 1] - 1,
 *   y[y row] = x[x row] . w[e]^T
 * with w8 [n_experts][n][k], w_scale [n_experts][n / 128][ld], x8, x_scale [x_rows][k], y [n_places][n] bfloat16, rounded
 * once as in sx_gemm_f8: of the down projection that is one rounding of each expert's result before their weighted sum.
 *   gather   0: the x row is p (a place from x_rows on is out of range); else order[p] / gather (the row that place p
 *            stands for, gather = top_k)
 *   scatter  0: the y row is p; else order[p] (the layout that sx_moe_combine reads)
 * order may be NULL when gather and scatter are 0.  offsets [n_experts + 1] and order [n_places] are DEVICE int32, as
 * sx_moe_route writes them; n_places (host) bounds offsets[n_experts].  n_experts <= 65536. */
sx_status sx_gemm_experts_f8(const int32_t* offsets, const int32_t* order, int32_t n_experts, int32_t n_places,
                             const void* x8, const void* x_scale, int32_t x_rows, int32_t gather, const void* w8,
                             const void* w_scale, int32_t k, int32_t n, void* y, int32_t scatter, void* stream);

/* out[row] = residual[row] + sum_j weights[slot][j] * y[slot * top_k + j], in float32 in ascending j, rounded once;
 * y [slots * top_k][h] bfloat16 and weights [slots][top_k] by slot, out and residual (nullable; may be out itself)
 * [..][h] bfloat16 by out_by_token.  h a multiple of 8.  A weight of 0 leaves its y out, whatever y holds. */
sx_status sx_moe_combine(const sx_plan* plan, const int32_t* rows, const int32_t* n_rows, int32_t max_rows,
                         const void* y, const float* weights, int32_t top_k, int32_t h, const void* residual, void* out,
                         int32_t out_by_token, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SX_F8_H */
