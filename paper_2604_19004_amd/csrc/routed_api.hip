// C-ABI entry points of the routed products (ocean_routed.h): checks of the arguments, then the launches.
#include "checks.hpp"

using namespace ocean;

static constexpr char HEADER[] = "ocean_routed.h";

extern "C" {

size_t ocean_route_workspace(int64_t tokens, int64_t experts, int32_t k)
{
    if (tokens < 0 || experts < 1 || k < 1 || tokens > (1ll << 28) || experts > OCEAN_ROUTE_MAX_EXPERTS || k > OCEAN_ROUTE_MAX_K) return 0;
    return route_workspace(tokens, experts, k);
}

int ocean_route(const void *logits, int32_t dtype, int64_t ld, int32_t normalize, const ocean_routing *out, void *workspace,
                size_t workspace_bytes, ocean_stream_t stream)
{
    if (!known_type(dtype)) return bad("dtype must be OCEAN_F32, OCEAN_BF16 or OCEAN_F16");
    REFUSE(routing_fault(out, true, true));
    REFUSE(matrix_fault(logits, out->tokens, out->experts, ld, dtype));
    const size_t need = route_workspace(out->tokens, out->experts, out->k);
    if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need))
        return bad("workspace is null, not aligned to 256 bytes or smaller than ocean_route_workspace");
    return launched(launch_route(logits, dtype, ld, normalize != 0, *out, workspace, static_cast<hipStream_t>(stream)), "ocean_route", HEADER);
}

int ocean_route_backward(const ocean_routing *r, const float *dval, const void *logits, int32_t dtype, int64_t ld, int32_t normalize,
                         void *dlogits, int64_t ld_dlogits, ocean_stream_t stream)
{
    if (!known_type(dtype)) return bad("dtype must be OCEAN_F32, OCEAN_BF16 or OCEAN_F16");
    REFUSE(routing_fault(r, true, false));
    if (r->tokens > 0 && (!r->col_idx || !dval)) return bad("col_idx or dval is null");
    if (!normalize) REFUSE(matrix_fault(logits, r->tokens, r->experts, ld, dtype));
    REFUSE(matrix_fault(dlogits, r->tokens, r->experts, ld_dlogits, dtype));
    return launched(launch_route_backward(*r, dval, logits, dtype, ld, normalize != 0, dlogits, ld_dlogits, static_cast<hipStream_t>(stream)),
                    "ocean_route_backward", HEADER);
}

int ocean_combine(const ocean_routing *r, const void *y, int32_t dtype, int64_t width, int64_t ld_y, void *out, int64_t ld_out,
                  ocean_stream_t stream)
{
    if (!known_type(dtype)) return bad("dtype must be OCEAN_F32, OCEAN_BF16 or OCEAN_F16");
    REFUSE(routing_fault(r, false, false));
    if (r->tokens > 0 && !r->slot) return bad("slot is null");
    REFUSE(matrix_fault(y, r->tokens * r->k, width, ld_y, dtype));
    REFUSE(matrix_fault(out, r->tokens, width, ld_out, dtype));
    return launched(launch_combine(*r, y, dtype, width, ld_y, out, ld_out, static_cast<hipStream_t>(stream)), "ocean_combine", HEADER);
}

int ocean_combine_backward(const ocean_routing *r, const void *dout, int64_t ld_dout, const void *y, int64_t ld_y, int32_t dtype,
                           int64_t width, void *dy, int64_t ld_dy, float *dval, ocean_stream_t stream)
{
    if (!known_type(dtype)) return bad("dtype must be OCEAN_F32, OCEAN_BF16 or OCEAN_F16");
    REFUSE(routing_fault(r, false, false));
    if (r->tokens > 0 && !r->slot) return bad("slot is null");
    REFUSE(matrix_fault(dout, r->tokens, width, ld_dout, dtype));
    if (dval) REFUSE(matrix_fault(y, r->tokens * r->k, width, ld_y, dtype));
    REFUSE(matrix_fault(dy, r->tokens * r->k, width, ld_dy, dtype));
    return launched(launch_combine_backward(*r, dout, ld_dout, y, ld_y, dtype, width, dy, ld_dy, dval, static_cast<hipStream_t>(stream)),
                    "ocean_combine_backward", HEADER);
}

int ocean_grouped_matmul(const ocean_groups *g, int32_t dtype, int64_t inner, int64_t outer, const void *x, int64_t ld_x, const void *w,
                         int64_t ld_w, int64_t stride_w, int32_t transposed, void *y, int64_t ld_y, ocean_stream_t stream)
{
    if (!known_type(dtype)) return bad("dtype must be OCEAN_F32, OCEAN_BF16 or OCEAN_F16");
    REFUSE(groups_fault(g));
    REFUSE(matrix_fault(x, g->x_rows, inner, ld_x, dtype));
    REFUSE(matrices_fault(w, g->experts, stride_w, transposed ? inner : outer, transposed ? outer : inner, ld_w, dtype, false));
    REFUSE(matrix_fault(y, g->rows, outer, ld_y, dtype));
    return launched(launch_grouped_matmul(*g, dtype, inner, outer, x, ld_x, w, ld_w, stride_w, transposed != 0, y, ld_y,
                                          static_cast<hipStream_t>(stream)), "ocean_grouped_matmul", HEADER);
}

int ocean_grouped_weight_grad(const ocean_groups *g, int32_t dtype, int64_t inner, int64_t outer, const void *dy, int64_t ld_dy,
                              const void *x, int64_t ld_x, void *dw, int64_t ld_dw, int64_t stride_dw, int32_t transposed,
                              ocean_stream_t stream)
{
    if (!known_type(dtype)) return bad("dtype must be OCEAN_F32, OCEAN_BF16 or OCEAN_F16");
    REFUSE(groups_fault(g));
    REFUSE(matrix_fault(dy, g->rows, outer, ld_dy, dtype));
    REFUSE(matrix_fault(x, g->x_rows, inner, ld_x, dtype));
    REFUSE(matrices_fault(dw, g->experts, stride_dw, transposed ? inner : outer, transposed ? outer : inner, ld_dw, dtype, true));
    return launched(launch_grouped_weight_grad(*g, dtype, inner, outer, dy, ld_dy, x, ld_x, dw, ld_dw, stride_dw, transposed != 0,
                                               static_cast<hipStream_t>(stream)), "ocean_grouped_weight_grad", HEADER);
}

size_t ocean_adapter_workspace(int64_t rows, int64_t inner, int64_t outer, int64_t adapters, int64_t rank, int32_t dtype)
{
    if (rows < 0 || rows >= MAX_DIM || inner < 0 || inner >= MAX_DIM || outer < 0 || outer >= MAX_DIM || adapters < 0 || adapters > OCEAN_ADAPTER_MAX ||
        rank < 0 || rank > OCEAN_ADAPTER_MAX_RANK || !known_type(dtype))
        return 0;
    return adapter_workspace(rows, inner, outer, adapters, rank, dtype);
}

int ocean_adapter_matmul(const ocean_adapters *l, const int32_t *ids, int32_t dtype, int64_t rows, int64_t inner, int64_t outer,
                         const void *x, int64_t ld_x, const void *w, int64_t ld_w, void *y, int64_t ld_y, void *workspace,
                         size_t workspace_bytes, ocean_stream_t stream)
{
    if (!known_type(dtype)) return bad("dtype must be OCEAN_F32, OCEAN_BF16 or OCEAN_F16");
    if (!l) return bad("the adapters are null");
    if (l->adapters < 0 || l->adapters > OCEAN_ADAPTER_MAX || l->rank < 0 || l->rank > OCEAN_ADAPTER_MAX_RANK)
        return bad("adapters or rank out of range (OCEAN_ADAPTER_MAX, OCEAN_ADAPTER_MAX_RANK)");
    REFUSE(matrix_fault(x, rows, inner, ld_x, dtype));
    REFUSE(matrix_fault(w, outer, inner, ld_w, dtype));
    REFUSE(matrix_fault(y, rows, outer, ld_y, dtype));
    REFUSE(matrices_fault(l->a, l->adapters, l->stride_a, l->rank, inner, l->ld_a, dtype, false));
    REFUSE(matrices_fault(l->b, l->adapters, l->stride_b, outer, l->rank, l->ld_b, dtype, false));
    if (rows > 0 && !ids) return bad("ids is null");
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < adapter_workspace(rows, inner, outer, l->adapters, l->rank, dtype))
        return bad("workspace is null, not aligned to 256 bytes or smaller than ocean_adapter_workspace");
    return launched(launch_adapter(*l, ids, dtype, rows, inner, outer, x, ld_x, w, ld_w, y, ld_y, workspace, static_cast<hipStream_t>(stream)),
                    "ocean_adapter_matmul", HEADER);
}

}  // extern "C"
