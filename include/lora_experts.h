/*
 * liblora_gfx950 -- the frozen layers beside an adapter: products in block-scaled 8-bit floating point, and products grouped by expert.
 *
 * The delta of include/lora.h is added to what a frozen layer gives.  Where that layer is held in 8 bits, or is one of the experts that a
 * router picks for each token, these calls compute it on the same terms (same status codes, lora_last_error, streams, pointers, no
 * allocation, no synchronisation; every argument is checked on the host before the device is touched, and nothing throws or aborts):
 *
 *     lora_rows_quantize         x (bf16) -> q (E4M3) and a scale for every 128 values of a row
 *     lora_linear_scaled         y = x W of one layer in 8 bits
 *     lora_experts_group         a router's picks -> rows in expert order, on the GPU: the host never learns who picked what
 *     lora_experts_linear        y = x W_e, row by row in that order, in bf16
 *     lora_experts_linear_scaled the same in 8 bits
 *     lora_experts_combine       a token's rows, weighted and added up
 *
 * One adapted layer on an 8-bit base is lora_rows_quantize, lora_linear_scaled, then lora_apply on the same y.
 *
 * Shapes: in_features a multiple of 64 and out_features of 128, as everywhere in this library, neither beyond
 * LORA_EXPERTS_MAX_FEATURES; up to LORA_MAX_EXPERTS experts.  x of a product spans up to 64 GiB, its scales up to 16.
 * "blocks" is in_features / 128 rounded up: the last block of 128 may be half there.
 *
 * 8-bit format: OCP E4M3 (largest value 448, no infinities), fp32 scales.  value(q[t][k]) = q[t][k] * x_scales[t][k / 128],
 * value(w[e][o][k]) = w[e][o][k] * w_scales[e][o / 128][k / 128].  The 128 products of a block are added up by the matrix instruction, exact but for
 * what of each lies below 2^-17 of the block's largest (so a block is off by less than 2^-10 of its largest product; without cancellation a few 1e-5 of
 * the sum, measured); the block's sum times both scales is added to the row's in fp32, and y is rounded to bf16 once; the
 * scales' own product may be below or beyond what fp32 holds.
 *
 * Device data that the calls read as indices (expert ids, starts, order, place) is checked where it is used: a place outside the rows, an order
 * entry outside the tokens or starts that do not fit the rows reach no memory outside the buffers; rows that would be meant are not written.
 */
#ifndef LORA_EXPERTS_GFX950_H
#define LORA_EXPERTS_GFX950_H

#include "lora.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LORA_MAX_EXPERTS 512
#define LORA_MAX_PICKS 64
#define LORA_EXPERTS_MAX_FEATURES (1 << 24)

/* Rows of bf16 to 8 bits: for every row t and block b of 128 (what lies behind in_features counts as zero)
 *     d = max(largest |x| of the block, 448 * 2^-126),   scales[t][b] = d / 448,   q[t][k] = nearest E4M3 of x[t][k] * 448 / d
 * where the quotient is rounded once, ties to even (bf16 over bf16 meets ties of E4M3 exactly, and they are kept).  A block that holds an infinity has
 * that for its scale, and 0 for its finite values and NaN for the others; one that holds a NaN has NaN for its scale and all its values.
 * x: device, bf16, [rows][in], row stride ldx elements (ldx >= in, ldx % 8 == 0, 16-byte aligned).
 * q: device, [rows][128 * blocks] bytes, row stride ldq bytes (ldq >= 128 * blocks, ldq % 16 == 0, 16-byte aligned); bytes behind in_features are
 *    written as zero, which the products below rely on.
 * scales: device, fp32, [rows][blocks], row stride ld_scales elements (ld_scales >= blocks). */
lora_status_t lora_rows_quantize(const void *x, int64_t ldx, int64_t rows, int32_t in_features, void *q, int64_t ldq, float *scales,
                                 int64_t ld_scales, void *stream);

/* Weights in the kernels' operand order, made once (set-up, not the per-step path).  bits: 16 (bf16) or 8 (E4M3).
 * w: device, [n_experts][out][in] row-major (the layout of linear layers' weights); for 8 bits rows of 128 * blocks bytes, those behind
 * in_features of no account.  dev_packed: device, 256-byte aligned, lora_experts_packed_bytes() long, owned by the caller.  One dense layer
 * is n_experts = 1.  Scales stay as they are. */
lora_status_t lora_experts_packed_bytes(int32_t n_experts, int32_t in_features, int32_t out_features, int32_t bits, size_t *bytes);
lora_status_t lora_experts_pack_weight(const void *w, int32_t n_experts, int32_t in_features, int32_t out_features, int32_t bits,
                                       void *dev_packed, size_t packed_bytes, void *stream);

/* y[t, :] = bf16(x[t, :] W) for every row, x and W in 8 bits.  q, ldq, scales, ld_scales: as lora_rows_quantize writes them.  w_packed: of
 * lora_experts_pack_weight, n_experts = 1.  w_scales: device, fp32, [out / 128][blocks].  y: device, bf16, [rows][out], row stride ldy
 * elements (ldy >= out, ldy % 8 == 0, 16-byte aligned), need not be initialised. */
lora_status_t lora_linear_scaled(const void *q, int64_t ldq, const float *scales, int64_t ld_scales, int32_t rows, int32_t in_features,
                                 const void *w_packed, const float *w_scales, int32_t out_features, void *y, int64_t ldy, void *stream);

/* The picks of a router, grouped by expert.  ids: device, int32, [tokens][picks], row stride ld_ids elements; an id outside 0 .. n_experts - 1
 * is a pick without an expert (one that another GPU holds).  Pick i = t * picks + j.  Written, all device int32 and tokens * picks long
 * (starts: n_experts + 1):
 *   starts[e]: the first place of expert e's rows, starts[n_experts]: how many places are taken;
 *   order[p]: the pick at place p, the picks of an expert in their own order, -1 from starts[n_experts] on;
 *   place[i]: the place of pick i, or -1.
 * No atomics whose order could show: the same ids give the same bits.  workspace: device, 16-byte aligned, as many bytes as
 * lora_experts_group_workspace_bytes says (0 is possible); its contents are of no account.  What that says for a number of picks and of experts is enough for
 * any smaller ones. */
lora_status_t lora_experts_group_workspace_bytes(int64_t n_picks, int32_t n_experts, size_t *bytes);
lora_status_t lora_experts_group(const int32_t *ids, int64_t ld_ids, int32_t tokens, int32_t picks, int32_t n_experts, int32_t *starts,
                                 int32_t *order, int32_t *place, void *workspace, size_t ws_bytes, void *stream);

/* y[p, :] = bf16(x[order[p] / picks, :] W_e) for the places p of every expert e, starts[e] <= p < starts[e + 1].  starts, order: as
 * lora_experts_group writes them; order NULL: place p reads row p of x (rows that are in expert order already, as the second product of
 * an expert's layer has them; tokens is then n_rows, and picks of no account).  Rows of y from starts[n_experts] on are left as they are.
 * x: device, bf16, [tokens][in], row stride ldx as above.  y: device, bf16, [n_rows][out], row stride ldy as above.  n_rows: places,
 * tokens * picks where order is given.  w_packed: of lora_experts_pack_weight.  x, y and the weights must not overlap. */
lora_status_t lora_experts_linear(const void *x, int64_t ldx, int32_t tokens, const int32_t *starts, const int32_t *order, int32_t picks,
                                  int32_t n_rows, int32_t n_experts, int32_t in_features, const void *w_packed, int32_t out_features,
                                  void *y, int64_t ldy, void *stream);

/* The same in 8 bits: q, ldq, scales, ld_scales, w_scales ([n_experts][out / 128][blocks]) as for lora_linear_scaled. */
lora_status_t lora_experts_linear_scaled(const void *q, int64_t ldq, const float *scales, int64_t ld_scales, int32_t tokens,
                                         const int32_t *starts, const int32_t *order, int32_t picks, int32_t n_rows, int32_t n_experts,
                                         int32_t in_features, const void *w_packed, const float *w_scales, int32_t out_features, void *y,
                                         int64_t ldy, void *stream);

/* z[t, :] = bf16(sum over j of weights[t][j] * y[place[t][j], :]), the products and the sum in fp32, in the order of j; picks whose place is
 * outside 0 .. n_rows - 1 are left out (whatever their weights hold), and a token without any is a row of zeros.  y: device, bf16, [n_rows][out],
 * row stride ldy; place, weights: device, int32 and fp32, [tokens][picks]; z: device, bf16, [tokens][out], row stride ldz as above.
 * z must not overlap y. */
lora_status_t lora_experts_combine(const void *y, int64_t ldy, int32_t n_rows, const int32_t *place, const float *weights, int32_t tokens,
                                   int32_t picks, int32_t out_features, void *z, int64_t ldz, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* LORA_EXPERTS_GFX950_H */
