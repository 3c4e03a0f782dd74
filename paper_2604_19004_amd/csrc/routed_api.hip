// C-ABI entry points of the routed products (ocean_routed.h): checks of the arguments, then the launches.
#include <cstdio>

#include "routed.hpp"

using namespace ocean;

namespace {

int bad(const char *msg) { return set_error(OCEAN_EINVAL, msg); }

int launched(hipError_t e, const char *what)
{
    if (e == hipSuccess) return OCEAN_OK;
    if (e == TOO_MANY_TILES) return bad("the result has more tiles than one launch takes (see the sizes in ocean_routed.h)");
    char msg[256];
    std::snprintf(msg, sizeof msg, "%s: %s", what, hipGetErrorString(e));
    return set_error(OCEAN_EHIP, msg);
}

bool known_type(int32_t dtype) { return dtype == OCEAN_F32 || dtype == OCEAN_BF16 || dtype == OCEAN_F16; }
bool aligned(const void *p, int size) { return reinterpret_cast<uintptr_t>(p) % size == 0; }
constexpr int64_t MAX_DIM = (1ll << 31) - 4096;   // rows and widths are below this: tiles count in 32 bits

// Null where the matrix is fine: base there (if it has elements), aligned to its type, rows apart.
const char *matrix_fault(const void *p, int64_t rows, int64_t width, int64_t ld, int dtype)
{
    if (rows < 0 || rows >= MAX_DIM || width < 0 || width >= MAX_DIM) return "a matrix's size is negative or not below 2^31 - 4096";
    if (ld < width) return "a row stride is less than the row's width";
    if (ld >= (1ll << 40) || (rows > 1 && ld > (1ll << 46) / rows)) return "a matrix spans more than 2^46 elements";
    if (rows > 0 && width > 0 && !p) return "a matrix is null";
    if (!aligned(p, type_size(dtype))) return "a matrix is not aligned to its type";
    return nullptr;
}

const char *routing_fault(const ocean_routing *r, bool need_val, bool need_all)
{
    if (!r) return "the routing is null";
    if (r->tokens < 0 || r->experts < 1 || r->experts > OCEAN_ROUTE_MAX_EXPERTS) return "tokens or experts out of range (experts <= OCEAN_ROUTE_MAX_EXPERTS)";
    if (r->k < 1 || r->k > OCEAN_ROUTE_MAX_K || r->k > r->experts) return "k must be 1 to min(experts, OCEAN_ROUTE_MAX_K)";
    if (r->tokens > (1ll << 28) || r->tokens * r->k >= MAX_DIM) return "tokens * k must be below 2^31 (and tokens at most 2^28)";
    if (!r->row_ptr) return "row_ptr is null";
    if (r->tokens > 0 && need_val && !r->val) return "val is null";
    if (need_all && (!r->expert_ptr || (r->tokens > 0 && (!r->col_idx || !r->token || !r->slot)))) return "an array of the routing is null";
    return nullptr;
}

const char *groups_fault(const ocean_groups *g)
{
    if (!g) return "the groups are null";
    if (g->rows < 0 || g->rows >= MAX_DIM || g->experts < 0 || g->experts > OCEAN_GROUPS_MAX || g->x_rows < 0 || g->x_rows >= MAX_DIM)
        return "rows, experts (OCEAN_GROUPS_MAX) or x_rows out of range";
    if (!g->group_ptr) return "group_ptr is null";
    if (!g->row_index && g->rows > 0 && g->x_rows != g->rows) return "without row_index, x_rows must be rows";
    return nullptr;
}

// Null where the matrices of the groups are fine, each rows x width and `stride` elements from the next.
const char *matrices_fault(const void *p, int64_t count, int64_t stride, int64_t rows, int64_t width, int64_t ld, int dtype, bool written)
{
    if (const char *why = matrix_fault(p, count > 0 ? rows : 0, width, ld, dtype)) return why;
    if (stride < 0 || stride >= (1ll << 44)) return "the stride between matrices is out of range";
    if (written && count > 1 && rows > 0 && stride < (rows - 1) * ld + width) return "matrices that are written overlap";
    return nullptr;
}

#define REFUSE(expr)                                   \
    do {                                               \
        if (const char *why__ = (expr)) return bad(why__); \
    } while (0)

}  // namespace

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
    return launched(launch_route(logits, dtype, ld, normalize != 0, *out, workspace, static_cast<hipStream_t>(stream)), "ocean_route");
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
                    "ocean_route_backward");
}

int ocean_combine(const ocean_routing *r, const void *y, int32_t dtype, int64_t width, int64_t ld_y, void *out, int64_t ld_out,
                  ocean_stream_t stream)
{
    if (!known_type(dtype)) return bad("dtype must be OCEAN_F32, OCEAN_BF16 or OCEAN_F16");
    REFUSE(routing_fault(r, false, false));
    if (r->tokens > 0 && !r->slot) return bad("slot is null");
    REFUSE(matrix_fault(y, r->tokens * r->k, width, ld_y, dtype));
    REFUSE(matrix_fault(out, r->tokens, width, ld_out, dtype));
    return launched(launch_combine(*r, y, dtype, width, ld_y, out, ld_out, static_cast<hipStream_t>(stream)), "ocean_combine");
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
                    "ocean_combine_backward");
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
                                          static_cast<hipStream_t>(stream)), "ocean_grouped_matmul");
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
                                               static_cast<hipStream_t>(stream)), "ocean_grouped_weight_grad");
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
                    "ocean_adapter_matmul");
}

}  // extern "C"
