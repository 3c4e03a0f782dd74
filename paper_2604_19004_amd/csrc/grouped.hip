// Products of ragged groups of rows with their group's matrix, and the gradient of the matrices.
#include "gmm.hpp"

namespace ocean {

namespace {

template <class T, bool LCOL, bool RCOL, GmmMode MODE> hipError_t pick_tile(const GmmArgs &a, bool aligned, hipStream_t s)
{
    if constexpr (sizeof(T) == 2) {
        const int64_t rows = MODE == GM_DEPTH ? a.m : a.rows / std::max<int64_t>(a.groups, 1);
        if (aligned && rows >= 256 && a.n >= 256) return launch_gmm<T, LCOL, RCOL, 256, 256, 2, 4, true, MODE>(a, s);
    }
    if (aligned) return launch_gmm<T, LCOL, RCOL, 128, 128, 2, 2, true, MODE>(a, s);
    return launch_gmm<T, LCOL, RCOL, 128, 128, 2, 2, false, MODE>(a, s);
}

}  // namespace

hipError_t launch_grouped_matmul(const ocean_groups &g, int dtype, int64_t inner, int64_t outer, const void *x, int64_t ldx, const void *w,
                                 int64_t ldw, int64_t stride, bool transposed, void *y, int64_t ldy, hipStream_t s)
{
    if (g.rows == 0 || outer == 0) return hipSuccess;
    const int size = type_size(dtype), e = 16 / size;
    GmmArgs a{};
    a.l = x, a.ldl = ldx;
    a.r = w, a.ldr = ldw, a.stride = stride;
    a.out = y, a.ldo = ldy;
    a.ptr = g.group_ptr, a.groups = g.experts, a.rows = g.rows;
    a.n = outer, a.c = inner;
    a.index = g.row_index, a.index_rows = g.x_rows;
    if (g.x_rows == 0 || inner == 0) a.c = 0, a.index_rows = 0, a.index = nullptr;
    const bool aligned = pieces_aligned(x, ldx, 0, size) && pieces_aligned(w, ldw, stride, size) && inner % e == 0 && (!transposed || outer % e == 0);
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        return transposed ? pick_tile<T, false, true, GM_ROWS>(a, aligned, s) : pick_tile<T, false, false, GM_ROWS>(a, aligned, s);
    });
}

hipError_t launch_grouped_weight_grad(const ocean_groups &g, int dtype, int64_t inner, int64_t outer, const void *dy, int64_t lddy, const void *x,
                                      int64_t ldx, void *dw, int64_t lddw, int64_t stride, bool transposed, hipStream_t s)
{
    if (g.experts == 0 || inner == 0 || outer == 0) return hipSuccess;
    const int size = type_size(dtype), e = 16 / size;
    // the matrix is outer x inner: its rows come from dy, its columns from x; transposed, the other way round
    GmmArgs a{};
    a.l = transposed ? x : dy, a.ldl = transposed ? ldx : lddy;
    a.r = transposed ? dy : x, a.ldr = transposed ? lddy : ldx;
    a.out = dw, a.ldo = lddw, a.stride = stride;
    a.ptr = g.group_ptr, a.groups = g.experts, a.rows = g.rows;
    a.m = transposed ? inner : outer, a.n = transposed ? outer : inner;
    a.index = g.row_index, a.index_rows = g.x_rows, a.index_on_r = transposed ? 0 : 1;
    if (g.x_rows == 0) a.rows = 0;   // (nothing to add up)
    const bool aligned = pieces_aligned(x, ldx, 0, size) && pieces_aligned(dy, lddy, 0, size) && inner % e == 0 && outer % e == 0;
    return with_type(dtype, [&](auto t) { return pick_tile<decltype(t), true, true, GM_DEPTH>(a, aligned, s); });
}

}  // namespace ocean
