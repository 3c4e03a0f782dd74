// Products of ragged groups of rows with their group's matrix, and the gradient of the matrices.
#include "few.hpp"

namespace ocean {

namespace {

// Groups of few rows: workgroup (x, y) has columns 16 TN x .. of the y-th tile of up to 64 (32) rows of a group.  (Tiles, not groups: where all rows meet in
// one of 128 groups, 2560 rows by 64 x 2048, 13 us; one after the other in the same workgroups they took 391.)
constexpr int few_rows(bool col) { return col ? 32 : 64; }   // (more fragments at a time than registers take)
template <class T, bool RCOL, int TN, int WAVES, bool ALIGNED>
__global__ void __launch_bounds__(WAVES * WAVE, 2) k_few(GmmArgs a)
{
    constexpr int FEW_ROWS = few_rows(RCOL), SUMS = WAVES * FEW_ROWS * (TN * 16 + 4) * 4, RINGS = RCOL ? WAVES * FEW_RING * FEW_STAGE : 0;
    __shared__ __align__(16) char s_lds[SUMS > RINGS ? SUMS : RINGS];
    __shared__ int64_t s_row[FEW_ROWS];
    int group, m0, hi, tiles = 0;
    const int64_t n0 = (int64_t)blockIdx.x * TN * 16;
    T *out = static_cast<T *>(a.out);
    auto item_of = [&](int n) { tiles = n; return (int)blockIdx.y; };
    if (!find_tile(a, FEW_ROWS, item_of, group, m0, hi)) {
        clear_outside<T>(a, n0, min((int64_t)TN * 16, a.n - n0), (int)blockIdx.y - tiles, (int)gridDim.y - tiles);
        return;
    }
    const T *x = static_cast<const T *>(a.l), *w = static_cast<const T *>(a.r) + (int64_t)group * a.stride;
    const int rows = min(FEW_ROWS, hi - m0);
    if ((int)threadIdx.x < rows) {
        const int64_t row = a.index ? a.index[m0 + threadIdx.x] : m0 + threadIdx.x;
        s_row[threadIdx.x] = (uint64_t)row < (uint64_t)a.index_rows ? row : -1;
    }
    __syncthreads();
    auto store = [&](int row, int64_t col, float v) { out[(int64_t)(m0 + row) * a.ldo + col] = (T)(s_row[row] < 0 ? 0.0f : v); };
    auto tile = [&](auto tm) {
        constexpr int TM = decltype(tm)::value;
        if constexpr (RCOL) few_tile_col<T, TM, WAVES, ALIGNED>(x, a.ldl, s_row, rows, w, a.ldr, n0, a.n, a.c, s_lds, store);
        else few_tile<T, TM, TN, WAVES, ALIGNED>(x, a.ldl, s_row, rows, w, a.ldr, n0, a.n, a.c, reinterpret_cast<float *>(s_lds),
                                                        [](int, int64_t) { return 0.0f; }, store);
    };
    if (rows <= 16) tile(std::integral_constant<int, 1>{});
    else if (rows <= 32) tile(std::integral_constant<int, 2>{});
    else if constexpr (!RCOL) tile(std::integral_constant<int, 4>{});
}

template <class T, bool RCOL, int TN, int WAVES, bool ALIGNED> hipError_t launch_few(const GmmArgs &a, hipStream_t s)
{
    // (the most tiles that the groups may make, and one that clears the rows of no group)
    const dim3 grid((uint32_t)((a.n + TN * 16 - 1) / (TN * 16)), (uint32_t)(a.rows / few_rows(RCOL) + std::min(a.groups, a.rows)) + 1);
    hipLaunchKernelGGL((k_few<T, RCOL, TN, WAVES, ALIGNED>), grid, dim3(WAVES * WAVE), 0, s, a);
    return hipGetLastError();
}

template <class T, bool LCOL, bool RCOL, GmmMode MODE> hipError_t pick_tile(const GmmArgs &a, bool aligned, hipStream_t s)
{
    const int64_t groups = MODE == GM_DEPTH ? a.groups : std::min(a.groups, a.rows);
    if constexpr (MODE == GM_ROWS) {
        // Where tiles of 64 x 64 would leave compute units without work, c is divided among the waves of a workgroup instead: eight
        // products with 4096 x 1024 weights take 15 us with a row each, 19 with 16, 23 with 24 and in tiles 25 (lines along c); 15 to 22 with
        // up to 32 and in tiles 29 (across c).  By the tiles that there are, 8 rows each: 128 16 and in tiles 25, 192 22 and 25, 248 28 and 26, 320
        // 34 and 31 (along c), 17 and 29, 20 and 29, 22 and 29, 38 and 34 (across c).  All rows in one group take no more than that.
        if (groups > 0 && groups * ((a.n + 63) / 64) < 256 && a.rows <= groups * (RCOL ? 32 : 24)) {
            if constexpr (!RCOL) return aligned ? launch_few<T, false, 1, 8, true>(a, s) : launch_few<T, false, 1, 8, false>(a, s);
            else return aligned ? launch_few<T, true, 4, 8, true>(a, s) : launch_few<T, true, 4, 8, false>(a, s);
        }
    }
    return launch_tiles<T, LCOL, RCOL, MODE>(a, [&](int64_t bm) {
        if (MODE == GM_DEPTH) return groups * ((a.m + bm - 1) / bm);
        return std::max(groups, a.rows / bm + groups / 2);   // (a group's last tile is half full on the average)
    }, aligned, s);
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
    if (!g.row_index) a.index_rows = g.rows;
    if (g.x_rows == 0 || inner == 0) a.c = 0, a.index_rows = 0, a.index = nullptr;
    // (the rows of a tile lie within 256 lines, gathered ones anywhere in x)
    const bool aligned = pieces_aligned(x, ldx, 0, size) && pieces_aligned(w, ldw, stride, size) && inner % e == 0 && (!transposed || outer % e == 0) &&
                         offsets_fit(g.row_index ? std::max<int64_t>(g.x_rows, 256) : 256, ldx, size) && offsets_fit(256, ldw, size);
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
    const bool aligned = pieces_aligned(x, ldx, 0, size) && pieces_aligned(dy, lddy, 0, size) && inner % e == 0 && outer % e == 0 &&
                         offsets_fit(256, ldx, size) && offsets_fit(256, lddy, size);
    return with_type(dtype, [&](auto t) { return pick_tile<decltype(t), true, true, GM_DEPTH>(a, aligned, s); });
}

}  // namespace ocean
