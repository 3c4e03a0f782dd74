// C-ABI entry points of ocean_experts.h: checks of the arguments, then the launches.
#include "checks.hpp"
#include "experts.hpp"

using namespace ocean;

static constexpr char HEADER[] = "ocean_experts.h";

namespace {

// Null where the matrices are fine (their places, and that rows and matrices that are written lie apart).
const char *mx4_fault(const ocean_mx4 *q, bool written)
{
    if (!q) return "the matrix in four bits is null";
    if (q->count < 0 || q->count > OCEAN_GROUPS_MAX || q->rows < 0 || q->rows >= MAX_DIM || q->inner < 0 || q->inner >= MAX_DIM)
        return "count (OCEAN_GROUPS_MAX), rows or inner of the matrix in four bits out of range";
    const int64_t blocks = mx4_blocks(q->inner), width = blocks * 16, up = (blocks + 15) / 16 * 16;
    if (q->ld_codes % 16 || q->stride_codes % 16 || !aligned(q->codes, 16)) return "codes are not aligned to 16 bytes (base and strides)";
    if (q->ld_scales % 16 || q->stride_scales % 16 || !aligned(q->scales, 16)) return "scales are not aligned to 16 bytes (base and strides)";
    if (q->ld_codes < width || q->ld_scales < up) return "a row stride of codes or scales is less than the row's width";
    if (q->ld_codes >= (1ll << 40) || q->ld_scales >= (1ll << 40) || (q->rows > 1 && (q->ld_codes > (1ll << 46) / q->rows || q->ld_scales > (1ll << 46) / q->rows)))
        return "a matrix in four bits spans more than 2^46 bytes";
    if (q->stride_codes < 0 || q->stride_codes >= (1ll << 44) || q->stride_scales < 0 || q->stride_scales >= (1ll << 44))
        return "the stride between matrices in four bits is out of range";
    if (q->count > 0 && q->rows > 0 && blocks > 0) {
        if (!q->codes || !q->scales) return "codes or scales are null";
        if (written && q->count > 1 && (q->stride_codes < (q->rows - 1) * q->ld_codes + width || q->stride_scales < (q->rows - 1) * q->ld_scales + up))
            return "matrices in four bits that are written overlap";
    }
    return nullptr;
}

// (tiles reach a matrix's lines by 32-bit offsets)
const char *product_fault(const ocean_mx4 *w, const ocean_groups *g)
{
    if (const char *why = mx4_fault(w, false)) return why;
    if (w->count != g->experts) return "the matrices in four bits are not as many as the groups";
    if (w->ld_codes >= (1 << 23) || w->ld_scales >= (1 << 23)) return "row strides of the matrices of a product must be below 2^23 bytes";
    return nullptr;
}

const char *converted_fault(const ocean_mx4 *q, const void *p, int32_t dtype, int64_t ld, int64_t stride, bool to_q)
{
    if (!known_type(dtype)) return "dtype must be OCEAN_F32, OCEAN_BF16 or OCEAN_F16";
    if (const char *why = mx4_fault(q, to_q)) return why;
    if (q->count * q->rows >= MAX_DIM) return "count * rows of the matrix in four bits must be below 2^31 - 4096";
    return matrices_fault(p, q->count, stride, q->rows, q->inner, ld, dtype, !to_q);
}

// (turns of 64 rows are reached by 32-bit offsets)
const char *logits_fault(const void *p, const ocean_routing *r, int64_t ld, int32_t dtype)
{
    if (const char *why = matrix_fault(p, r->tokens, r->experts, ld, dtype)) return why;
    return ld >= (1 << 23) ? "row strides of logits must be below 2^23 elements" : nullptr;
}

}  // namespace

extern "C" {

size_t ocean_route_balance_workspace(int64_t tokens, int64_t experts)
{
    if (tokens < 0 || tokens > (1ll << 28) || experts < 1 || experts > OCEAN_ROUTE_MAX_EXPERTS) return 0;
    return balance_workspace(tokens, experts);
}

int ocean_route_balance(const ocean_routing *r, const void *logits, int32_t dtype, int64_t ld, const ocean_balance *out, void *workspace,
                        size_t workspace_bytes, ocean_stream_t stream)
{
    if (!known_type(dtype)) return bad("dtype must be OCEAN_F32, OCEAN_BF16 or OCEAN_F16");
    REFUSE(routing_size_fault(r));
    if (!r->expert_ptr) return bad("expert_ptr is null");
    REFUSE(logits_fault(logits, r, ld, dtype));
    if (!out || !out->loss || !out->counts || !out->prob || !out->rows) return bad("the balance or an array of it is null");
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < balance_workspace(r->tokens, r->experts))
        return bad("workspace is null, not aligned to 256 bytes or smaller than ocean_route_balance_workspace");
    return launched(launch_balance(*r, logits, dtype, ld, *out, workspace, static_cast<hipStream_t>(stream)), "ocean_route_balance", HEADER);
}

int ocean_route_balance_backward(const ocean_balance *b, const ocean_routing *r, const void *logits, int32_t dtype, int64_t ld, const float *dloss,
                                 const float *dval, int32_t normalize, void *dlogits, int64_t ld_dlogits, ocean_stream_t stream)
{
    if (!known_type(dtype)) return bad("dtype must be OCEAN_F32, OCEAN_BF16 or OCEAN_F16");
    REFUSE(dval ? routing_fault(r, true, false) : routing_size_fault(r));
    if (dval && r->tokens > 0 && !r->col_idx) return bad("col_idx is null");
    if (!b || !b->counts || !b->rows || !dloss) return bad("the balance, its counts or rows, or dloss is null");
    REFUSE(logits_fault(logits, r, ld, dtype));
    REFUSE(logits_fault(dlogits, r, ld_dlogits, dtype));
    return launched(launch_balance_backward(*b, *r, logits, dtype, ld, dloss, dval, normalize != 0, dlogits, ld_dlogits, static_cast<hipStream_t>(stream)),
                    "ocean_route_balance_backward", HEADER);
}

int ocean_mx4_quantize(const void *x, int32_t dtype, int64_t ld_x, int64_t stride_x, const ocean_mx4 *q, ocean_stream_t stream)
{
    REFUSE(converted_fault(q, x, dtype, ld_x, stride_x, true));
    return launched(launch_mx4_quantize(x, dtype, ld_x, stride_x, *q, static_cast<hipStream_t>(stream)), "ocean_mx4_quantize", HEADER);
}

int ocean_mx4_dequantize(const ocean_mx4 *q, int32_t dtype, void *out, int64_t ld_out, int64_t stride_out, ocean_stream_t stream)
{
    REFUSE(converted_fault(q, out, dtype, ld_out, stride_out, false));
    return launched(launch_mx4_dequantize(*q, dtype, out, ld_out, stride_out, static_cast<hipStream_t>(stream)), "ocean_mx4_dequantize", HEADER);
}

int ocean_grouped_matmul_mx4(const ocean_groups *g, int32_t dtype, const void *x, int64_t ld_x, const ocean_mx4 *w, int32_t transposed, void *y,
                             int64_t ld_y, ocean_stream_t stream)
{
    if (!known_type(dtype)) return bad("dtype must be OCEAN_F32, OCEAN_BF16 or OCEAN_F16");
    REFUSE(groups_fault(g));
    REFUSE(product_fault(w, g));
    REFUSE(matrix_fault(x, g->x_rows, transposed ? w->rows : w->inner, ld_x, dtype));
    REFUSE(matrix_fault(y, g->rows, transposed ? w->inner : w->rows, ld_y, dtype));
    return launched(launch_grouped_mx4(*g, dtype, x, ld_x, *w, transposed != 0, y, ld_y, static_cast<hipStream_t>(stream)), "ocean_grouped_matmul_mx4", HEADER);
}

int ocean_grouped_matmul_mx4_mx4(const ocean_groups *g, const ocean_mx4 *x, const ocean_mx4 *w, int32_t dtype, void *y, int64_t ld_y,
                                 ocean_stream_t stream)
{
    if (!known_type(dtype)) return bad("dtype must be OCEAN_F32, OCEAN_BF16 or OCEAN_F16");
    REFUSE(groups_fault(g));
    REFUSE(mx4_fault(x, false));
    REFUSE(product_fault(w, g));
    if (x->count != 1 || x->rows != g->x_rows || x->inner != w->inner) return bad("x must be one matrix of x_rows rows with the matrices' inner");
    REFUSE(matrix_fault(y, g->rows, w->rows, ld_y, dtype));
    return launched(launch_grouped_mx4_mx4(*g, *x, *w, dtype, y, ld_y, static_cast<hipStream_t>(stream)), "ocean_grouped_matmul_mx4_mx4", HEADER);
}

}  // extern "C"
