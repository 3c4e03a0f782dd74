/*
 * Products in which every row chooses its matrix, for AMD MI355X (gfx950): the mixture of experts and the adapters of
 * many requests.  A routing matrix R (tokens x experts, at most k entries a row) is a CSR matrix like those of
 * ocean_spgemm.h; here it is made from logits, applied to the dense rows that the experts gave, and differentiated, and the
 * dense products of the ragged groups of rows that it forms are computed.
 *
 * The conventions of ocean_spgemm.h hold: plain C, OCEAN_OK or an error code, ocean_last_error() describes the last
 * failure on the calling thread, no exception and no abort.  Every array is a DEVICE pointer on the current HIP device.
 * All calls are asynchronous: they enqueue kernels on `stream`, allocate nothing, read nothing back and may be captured
 * into a HIP graph.  Dense matrices are row-major with a row stride (ld...) in elements, not less than their width; any
 * alignment of the element type works (multiples of 16 bytes, in base and stride, are fastest).  Sums are in 32 bits, results are rounded
 * once to their type.  Outputs may not overlap inputs.
 *
 * Types of dense matrices: OCEAN_BF16, OCEAN_F16, OCEAN_F32; all those of one call have the same.
 */
#ifndef OCEAN_ROUTED_H
#define OCEAN_ROUTED_H

#include "ocean_spgemm.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { OCEAN_BF16 = 2, OCEAN_F16 = 3 };   /* beside OCEAN_F64 (not taken here) and OCEAN_F32 */

#define OCEAN_ROUTE_MAX_EXPERTS 1024
#define OCEAN_ROUTE_MAX_K 64

/*
 * A routing matrix, in CSR and in the order of its columns.  With n = row_ptr[tokens] <= tokens * k entries: entry p (row by
 * row, columns ascending) belongs to expert col_idx[p], has weight val[p] and the number slot[p] in the experts' order;
 * the entries of expert e are the slots expert_ptr[e] .. expert_ptr[e+1]-1, and token[s] is the row of slot s (ascending within an
 * expert).  row_ptr, col_idx and val are the arrays of an ocean_csr of type OCEAN_F32.  All arrays belong to the caller.
 */
typedef struct ocean_routing {
    int64_t tokens, experts;
    int32_t k, reserved;
    int64_t *row_ptr;    /* tokens + 1 */
    int32_t *col_idx;    /* tokens * k; -1 from entry n on */
    float *val;          /* tokens * k; 0 from entry n on.  NULL where a call allows it: every weight is 1 */
    int64_t *expert_ptr; /* experts + 1 */
    int32_t *token;      /* tokens * k; -1 from slot n on */
    int32_t *slot;       /* tokens * k; -1 from entry n on */
} ocean_routing;

/*
 * R from logits (tokens x experts): each row takes its k largest logits, or as many as there are; of equal ones those of the lowest columns.
 * A logit that is NaN, -inf or the lowest finite value of its type is masked: it is never taken (a row of
 * such logits stays empty).  +inf counts as the largest finite value.  Weights: the softmax of the row's logits, over the
 * entries taken (normalize != 0) or over all that are not masked (0).  1 <= k <= min(experts, OCEAN_ROUTE_MAX_K), experts <=
 * OCEAN_ROUTE_MAX_EXPERTS, tokens * k < 2^31.  workspace: ocean_route_workspace bytes, aligned to 256, needed until the kernels have run (0
 * bytes, and NULL will do, for few tokens).
 */
size_t ocean_route_workspace(int64_t tokens, int64_t experts, int32_t k);
int ocean_route(const void *logits, int32_t dtype, int64_t ld, int32_t normalize, const ocean_routing *out, void *workspace,
                size_t workspace_bytes, ocean_stream_t stream);

/* Gradient of the logits from that of the weights, dval[tokens * k] in the order of val.  Masked logits get 0.  `logits` is read
 * only without normalize (may be NULL with it).  dlogits has the logits' type.  Reads row_ptr, col_idx and val. */
int ocean_route_backward(const ocean_routing *r, const float *dval, const void *logits, int32_t dtype, int64_t ld, int32_t normalize,
                         void *dlogits, int64_t ld_dlogits, ocean_stream_t stream);

/*
 * out[t] = sum over the entries p of row t of val[p] * y[slot[p]]; an empty row gives zeros.  y: tokens * k rows of
 * `width`, in the experts' order; out: tokens rows.  Reads row_ptr, slot, val (NULL: ones).  An entry whose slot
 * is outside 0 .. tokens * k - 1 adds nothing.
 */
int ocean_combine(const ocean_routing *r, const void *y, int32_t dtype, int64_t width, int64_t ld_y, void *out, int64_t ld_out,
                  ocean_stream_t stream);

/* Its gradients: dy[slot[p]] = val[p] * dout[t] (tokens * k rows; those from row_ptr[tokens] on are 0) and dval[p] =
 * <dout[t], y[slot[p]]> (tokens * k values, 0 from entry row_ptr[tokens] on; NULL: not wanted, and y is not read).
 * slot has to number the entries 0 .. n-1 as ocean_route does. */
int ocean_combine_backward(const ocean_routing *r, const void *dout, int64_t ld_dout, const void *y, int64_t ld_y, int32_t dtype,
                           int64_t width, void *dy, int64_t ld_dy, float *dval, ocean_stream_t stream);

/*
 * Sizes: rows and widths below 2^31 - 4096, experts of a grouped product at most OCEAN_GROUPS_MAX (each workgroup finds its group by
 * going through their offsets).  Straight loads to LDS address 4 GB from a matrix's first row that a workgroup
 * needs: gathered rows of an x larger than that go through registers, which is slower and otherwise the same.
 * A result is made in one launch, which takes less than 2^24 tiles of 128 x 128 or, in 16 bits and aligned, 2^23 of 256 x 256: of (rows / 128 + experts that
 * may have rows) by outer / 128, a gradient of matrices of experts by outer / 128 by inner / 128, adapters of rows / 128 by outer / 128, and of (rows / 64 +
 * adapters) by rank / 64.  What is larger is refused.
 */
#define OCEAN_GROUPS_MAX 16384

/*
 * Products of ragged groups of rows with their group's matrix.  Group e has rows group_ptr[e] .. group_ptr[e+1]-1 of `rows`
 * rows (group_ptr: experts + 1 ascending offsets; values outside 0 .. rows are limited to it).  With row_index, row s of the left matrix
 * is row row_index[s] of x; NULL: row s itself, and x_rows = rows.  An index outside 0 .. x_rows-1 stands for a row of zeros: its product is 0 and it
 * adds nothing to a gradient, whatever w and dy[s] hold.
 */
typedef struct ocean_groups {
    int64_t rows, experts;
    const int64_t *group_ptr; /* experts + 1 */
    const int32_t *row_index; /* rows, or NULL */
    int64_t x_rows;
} ocean_groups;

/*
 * y[s] = x[row(s)] * W_e^T for the rows of group e; rows of no group are 0.  x: x_rows x inner, y: rows x outer.
 * W_e begins at w + e * stride_w elements: outer x inner (transposed == 0), or inner x outer (transposed != 0, then y[s] = x[row(s)] * W_e).
 * The gradient of x's rows is this product of dy with the same w and the other value of transposed.
 */
int ocean_grouped_matmul(const ocean_groups *g, int32_t dtype, int64_t inner, int64_t outer, const void *x, int64_t ld_x, const void *w,
                         int64_t ld_w, int64_t stride_w, int32_t transposed, void *y, int64_t ld_y, ocean_stream_t stream);

/*
 * dW_e = sum over the rows s of group e of dy[s]^T x[row(s)] (outer x inner; transposed != 0: its transpose, inner x outer);
 * an empty group's is 0.  dy: rows x outer.  dW_e is written at dw + e * stride_dw elements; each begins behind the one before it (interleaved ones are
 * refused).
 */
int ocean_grouped_weight_grad(const ocean_groups *g, int32_t dtype, int64_t inner, int64_t outer, const void *dy, int64_t ld_dy,
                              const void *x, int64_t ld_x, void *dw, int64_t ld_dw, int64_t stride_dw, int32_t transposed,
                              ocean_stream_t stream);

/*
 * A shared projection with a low-rank adapter for each row beside it: y[m] = x[m] * W^T + scale[a] * (x[m] * A_a^T) * B_a^T with
 * a = ids[m]; an id outside 0 .. adapters-1 stands for no adapter.  x: rows x inner, W: outer x inner, A_a: rank x inner at
 * a + id * stride_a, B_a: outer x rank at b + id * stride_b, y: rows x outer.  ranks (adapters, or NULL): adapter a uses only
 * its first ranks[a] <= rank rows of A_a and columns of B_a; the others are not used, whatever they hold.  scale: NULL means 1.
 * rank <= OCEAN_ADAPTER_MAX_RANK, adapters <= OCEAN_ADAPTER_MAX.  The inner product x * A_a^T is kept to 32 bits (types of
 * 16 bits: to 2 * 16 at least; float16: or to 2^-39 of the row's largest).  workspace: ocean_adapter_workspace bytes, aligned to 256, needed until the
 * kernels have run.
 */
#define OCEAN_ADAPTER_MAX_RANK 256
#define OCEAN_ADAPTER_MAX 8192
typedef struct ocean_adapters {
    int64_t adapters, rank;
    const void *a;
    int64_t ld_a, stride_a;
    const void *b;
    int64_t ld_b, stride_b;
    const int32_t *ranks;
    const float *scale;
} ocean_adapters;
size_t ocean_adapter_workspace(int64_t rows, int64_t inner, int64_t outer, int64_t adapters, int64_t rank, int32_t dtype);
int ocean_adapter_matmul(const ocean_adapters *l, const int32_t *ids, int32_t dtype, int64_t rows, int64_t inner, int64_t outer,
                         const void *x, int64_t ld_x, const void *w, int64_t ld_w, void *y, int64_t ld_y, void *workspace,
                         size_t workspace_bytes, ocean_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* OCEAN_ROUTED_H */
