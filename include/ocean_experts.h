/*
 * Experts in training and in four bits, for AMD MI355X (gfx950), beside the routed products of ocean_routed.h: the losses that keep a
 * router's experts evenly used, with the gradient of the logits, and matrices in microscaled four bits, their making and their products with
 * ragged groups of rows.
 *
 * The conventions of ocean_routed.h hold: every array is a DEVICE pointer on the current HIP device, calls enqueue kernels on `stream`,
 * allocate nothing, read nothing back and may be captured into a HIP graph; sums are in 32 bits or more, results are rounded once to their
 * type, have the same bits each time, and may not overlap inputs.
 */
#ifndef OCEAN_EXPERTS_H
#define OCEAN_EXPERTS_H

#include "ocean_routed.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * What a router is told about its experts' use.  Over the rows of logits (tokens x experts) that have a logit which is not masked (masked: NaN, -inf
 * or the type's lowest value; +inf counts as the largest finite value, as in ocean_route), of which there are `rows`:
 * prob[e] = the mean of softmax(row)[e], counts[e] = the entries of expert e in the routing (n of all), and
 *   loss[0] = experts * sum over e of counts[e] / n * prob[e]   (1 where all are used evenly),
 *   loss[1] = the mean of logsumexp(row)^2.
 * Without such rows, or without entries, what has no value is 0.  Row strides of logits and of their gradient are below 2^23 elements, tokens
 * at most 2^28.
 */
typedef struct ocean_balance {
    float *loss;        /* 2 */
    int64_t *counts;    /* experts */
    float *prob;        /* experts */
    int64_t *rows;      /* 1 */
} ocean_balance;

/* Reads tokens, experts and expert_ptr of the routing.  workspace: ocean_route_balance_workspace bytes, aligned to 256, needed until the
 * kernels have run. */
size_t ocean_route_balance_workspace(int64_t tokens, int64_t experts);
int ocean_route_balance(const ocean_routing *r, const void *logits, int32_t dtype, int64_t ld, const ocean_balance *out, void *workspace,
                        size_t workspace_bytes, ocean_stream_t stream);

/*
 * Gradient of the logits from that of the losses, dloss[2].  counts count as constants; counts and rows of `b` are read (those of all
 * devices, where a program has added them up), its loss and prob are not (they may be NULL).
 * dval: NULL, or tokens * k gradients of the routing's weights: what ocean_route_backward gives for them (normalize as there; reads row_ptr,
 * col_idx and val; the columns of a row differ, as ocean_route makes them) is added before the one rounding to the logits' type.
 * Masked logits get 0.  Without dval, only tokens and experts of the routing are read.
 */
int ocean_route_balance_backward(const ocean_balance *b, const ocean_routing *r, const void *logits, int32_t dtype, int64_t ld, const float *dloss,
                                 const float *dval, int32_t normalize, void *dlogits, int64_t ld_dlogits, ocean_stream_t stream);

/*
 * `count` matrices of rows x inner in microscaled four bits: every 32 numbers of a row (the last ones of a row may be fewer: `inner` is any) are a block of 16
 * bytes of codes, two a byte, the earlier number in the low four bits, and a byte s of scale.  A code is a sign (8), two bits of exponent and one behind
 * the point: 0, 0.5, 1, 1.5, 2, 3, 4, 6; the number is that times 2^(s - 127); s = 255 makes a block of NaN.  (The format called
 * MXFP4: e2m1 with e8m0.)  With blocks = (inner + 31) / 32: row i of matrix e has its codes at codes + e * stride_codes + i * ld_codes
 * (16 * blocks bytes; those behind `inner` are not used, whatever they hold) and its scales at scales + e * stride_scales + i * ld_scales (blocks bytes, and
 * up to the next multiple of 16 there has to be memory, whose content does not count).  Strides are in bytes; codes, scales and all strides are multiples of 16.  Numbers beyond a type's range are infinite in it; single precision and bfloat16 hold all with s <= 252.
 */
typedef struct ocean_mx4 {
    int64_t count, rows, inner;
    uint8_t *codes;
    int64_t ld_codes, stride_codes;
    uint8_t *scales;
    int64_t ld_scales, stride_scales;
} ocean_mx4;

/*
 * x, `count` matrices of rows x inner at stride_x elements, into q.  A block's scale is 2^(floor(log2 of its largest magnitude) - 2), not below
 * 2^-127, or 1 where all are 0; its numbers are rounded to the nearest (ties to the even code) and magnitudes beyond 6 become 6.  A block that holds an
 * infinite number or NaN becomes NaN.  Codes behind `inner` are 0, and so are scales' bytes up to the next multiple of 16.  count * rows < 2^31 - 4096, and
 * count at most OCEAN_GROUPS_MAX.
 */
int ocean_mx4_quantize(const void *x, int32_t dtype, int64_t ld_x, int64_t stride_x, const ocean_mx4 *q, ocean_stream_t stream);

/* And back: out, count matrices of rows x inner, of the same limits. */
int ocean_mx4_dequantize(const ocean_mx4 *q, int32_t dtype, void *out, int64_t ld_out, int64_t stride_out, ocean_stream_t stream);

/*
 * As ocean_grouped_matmul, with matrices in four bits: y[s] = x[row(s)] * W_e^T for the rows of group e (transposed == 0; x: x_rows x w->inner, y: rows x
 * w->rows), or y[s] = x[row(s)] * W_e (transposed != 0; x: x_rows x w->rows, y: rows x w->inner), which is the gradient of x's rows.
 * w->count is the groups' `experts`, and its row strides are below 2^23.  The matrices' numbers are taken as they are, x's too: in the type they have, or, float16
 * where the matrices' numbers are beyond it and single precision, as the exact sum of two and three bfloat16 numbers (what is left of a number below 2^-133 is not kept).
 * Matrix numbers beyond bfloat16 (some of those with s = 253 or 254) count as infinite, times x an infinity or, for a 0, NaN; beside rows in four bits they count as they are.
 * Beside float16 rows, matrices' numbers of scales up to 51 (below 2^-73) may count as 0, also where x is infinite.
 * One launch has fewer than 2^32 threads.  In tiles of 256 x 256 that is 2^23 (16 bits, rows at 16 bytes), of 128 x 128 2^24 (16 bits), of 64 x 64 2^24 (single precision),
 * those that groups' last tiles add among them: what has more is refused.
 */
int ocean_grouped_matmul_mx4(const ocean_groups *g, int32_t dtype, const void *x, int64_t ld_x, const ocean_mx4 *w, int32_t transposed, void *y,
                             int64_t ld_y, ocean_stream_t stream);

/* The same with x in four bits too (one matrix, x->count == 1, x->rows == x_rows, x->inner == w->inner); y has type dtype.  (Tiles as above, of 256 x 256
 * for results of 16 bits.  Where 256 rows of x's codes or scales, or all of them if they are gathered, span 4 GB or more, those of 64 x 64 and 128 x 128.)
 */
int ocean_grouped_matmul_mx4_mx4(const ocean_groups *g, const ocean_mx4 *x, const ocean_mx4 *w, int32_t dtype, void *y, int64_t ld_y,
                                 ocean_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* OCEAN_EXPERTS_H */
