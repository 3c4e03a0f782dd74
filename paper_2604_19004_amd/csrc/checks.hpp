// Checks of the arguments that the entry points of the routed products share, and what they answer.
#pragma once

#include <cstdio>

#include "routed.hpp"

namespace ocean {

namespace {

inline int bad(const char *msg) { return set_error(OCEAN_EINVAL, msg); }

// (header: where the sizes of the operator stand)
inline int launched(hipError_t e, const char *what, const char *header)
{
    if (e == hipSuccess) return OCEAN_OK;
    char msg[256];
    if (e == TOO_MANY_TILES) {
        std::snprintf(msg, sizeof msg, "the result has more tiles than one launch takes (see the sizes in %s)", header);
        return bad(msg);
    }
    std::snprintf(msg, sizeof msg, "%s: %s", what, hipGetErrorString(e));
    return set_error(OCEAN_EHIP, msg);
}

inline bool known_type(int32_t dtype) { return dtype == OCEAN_F32 || dtype == OCEAN_BF16 || dtype == OCEAN_F16; }
inline bool aligned(const void *p, int size) { return reinterpret_cast<uintptr_t>(p) % size == 0; }
constexpr int64_t MAX_DIM = (1ll << 31) - 4096;   // rows and widths are below this: tiles count in 32 bits

// Null where the matrix is fine: base there (if it has elements), aligned to its type, rows apart.
inline const char *matrix_fault(const void *p, int64_t rows, int64_t width, int64_t ld, int dtype)
{
    if (rows < 0 || rows >= MAX_DIM || width < 0 || width >= MAX_DIM) return "a matrix's size is negative or not below 2^31 - 4096";
    if (ld < width) return "a row stride is less than the row's width";
    if (ld >= (1ll << 40) || (rows > 1 && ld > (1ll << 46) / rows)) return "a matrix spans more than 2^46 elements";
    if (rows > 0 && width > 0 && !p) return "a matrix is null";
    if (!aligned(p, type_size(dtype))) return "a matrix is not aligned to its type";
    return nullptr;
}

// (what has no entries of its own: a routing's rows and columns)
inline const char *routing_size_fault(const ocean_routing *r)
{
    if (!r) return "the routing is null";
    if (r->tokens < 0 || r->tokens > (1ll << 28) || r->experts < 1 || r->experts > OCEAN_ROUTE_MAX_EXPERTS)
        return "tokens (at most 2^28) or experts (1 to OCEAN_ROUTE_MAX_EXPERTS) out of range";
    return nullptr;
}

inline const char *routing_fault(const ocean_routing *r, bool need_val, bool need_all)
{
    if (const char *why = routing_size_fault(r)) return why;
    if (r->k < 1 || r->k > OCEAN_ROUTE_MAX_K || r->k > r->experts) return "k must be 1 to min(experts, OCEAN_ROUTE_MAX_K)";
    if (r->tokens * r->k >= MAX_DIM) return "tokens * k must be below 2^31 - 4096";
    if (!r->row_ptr) return "row_ptr is null";
    if (r->tokens > 0 && need_val && !r->val) return "val is null";
    if (need_all && (!r->expert_ptr || (r->tokens > 0 && (!r->col_idx || !r->token || !r->slot)))) return "an array of the routing is null";
    return nullptr;
}

inline const char *groups_fault(const ocean_groups *g)
{
    if (!g) return "the groups are null";
    if (g->rows < 0 || g->rows >= MAX_DIM || g->experts < 0 || g->experts > OCEAN_GROUPS_MAX || g->x_rows < 0 || g->x_rows >= MAX_DIM)
        return "rows, experts (OCEAN_GROUPS_MAX) or x_rows out of range";
    if (!g->group_ptr) return "group_ptr is null";
    if (!g->row_index && g->rows > 0 && g->x_rows != g->rows) return "without row_index, x_rows must be rows";
    return nullptr;
}

// Null where the matrices of the groups are fine, each rows x width and `stride` elements from the next.
inline const char *matrices_fault(const void *p, int64_t count, int64_t stride, int64_t rows, int64_t width, int64_t ld, int dtype, bool written)
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

}  // namespace ocean
