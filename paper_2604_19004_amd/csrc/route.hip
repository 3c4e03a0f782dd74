// The routing matrix: the largest logits of each row as a CSR matrix, its entries in the order of the columns, and the gradient of the logits.
#include <algorithm>
#include <type_traits>

#include "routed.hpp"

namespace ocean {

namespace {

constexpr int BLOCK_ROWS = 64;        // rows of a workgroup: one bit each in a 64-bit mask per expert
constexpr int PLACE_TPB = 256;

// Workspace, per block of 64 rows: for each of its entries the column, the rank among the block's entries of that column and the weight
// (k places a row, filled from the front), and per expert the block's entries, blocks of an expert side by side.
struct RouteSpace {
    uint32_t *pick;     // [tokens * k] column | rank << 16 | 1 << 31
    float *weight;      // [tokens * k]
    uint32_t *count;    // [experts][blocks]; after k_route_scan the entries of earlier blocks
    uint32_t *total;    // [experts]
};
inline int64_t route_blocks(int64_t tokens) { return (tokens + BLOCK_ROWS - 1) / BLOCK_ROWS; }
inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
inline RouteSpace route_space(void *at, int64_t tokens, int64_t experts, int k, size_t *bytes)
{
    char *p = static_cast<char *>(at);
    size_t o = 0;
    RouteSpace w;
    w.pick = reinterpret_cast<uint32_t *>(p + o);
    o += up256((size_t)tokens * k * 4);
    w.weight = reinterpret_cast<float *>(p + o);
    o += up256((size_t)tokens * k * 4);
    w.count = reinterpret_cast<uint32_t *>(p + o);
    o += up256((size_t)experts * route_blocks(tokens) * 4);
    w.total = reinterpret_cast<uint32_t *>(p + o);
    o += up256((size_t)experts * 4);
    *bytes = o;
    return w;
}

// Whole numbers in the order of the values; 0 stands for a masked logit, below every other.  -0 and 0 are the same.
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return (b >> 31) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t key) { return __uint_as_float((key >> 31) ? (key & 0x7fffffffu) : ~key); }

template <class T> __device__ __forceinline__ uint32_t logit_key(T v)
{
    const float x = (float)v;
    if (!(x > TypeTraits<T>::lowest)) return 0;   // (NaN as well)
    return order_key(fminf(x, -TypeTraits<T>::lowest));
}

// Moves among the G lanes that share a row, every lane receiving the result: inside 16 lanes by lane swaps (neighbours, pairs, mirrored halves
// of 8, mirrored rows of 16), over the whole wave by the prefix moves of ocean_internal.hpp.  All lanes must be active.
template <class F> __device__ __forceinline__ uint32_t row16(uint32_t v, F f)
{
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false));    // quad_perm [1,0,3,2]
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false));    // quad_perm [2,3,0,1]
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, false));   // row_half_mirror
    return f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, false));   // row_mirror
}
template <int G> __device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
    if constexpr (G == 16) return row16(v, [](uint32_t x, uint32_t y) { return max(x, y); });
    else return wave_max_u32(v);
}
template <int G> __device__ __forceinline__ float lanes_sum(float v)
{
    if constexpr (G == 16)
        return __uint_as_float(row16(__float_as_uint(v), [](uint32_t x, uint32_t y) { return __float_as_uint(__uint_as_float(x) + __uint_as_float(y)); }));
    else return wave_sum(v);
}

// Takes the largest logits of the block's rows.  G lanes share a row, lane l has columns l, l + G, ...: the largest key, then the lowest
// column that holds it, k times.  Bound by instructions, some thirty a turn whatever G is: four rows in 16 lanes each take a third of the
// time of a row a wave (32768 rows of 100, 8 taken: 18 us instead of 40; at the rate of a large copy the bytes would take 3).  A row's softmax is relative to
// its largest logit.  The bits of s_mask (expert: which of the 64 rows took it) give the entries' rank among the block's of the same
// column without an order of arrival.
template <class T, int G, int NV, class Put>
__device__ __forceinline__ void pick_rows(const T *logits, int64_t ld, int64_t row0, int rows, int experts, int k, int normalize,
                                          unsigned long long *s_mask, Put put)
{
    const int lane = lane_id(), sub = lane % G, group = lane / G, wave = threadIdx.x / WAVE, waves = blockDim.x / WAVE;
    constexpr int PER = WAVE / G;
    for (int r0 = wave * PER; r0 < rows; r0 += waves * PER) {
        const int r = r0 + group;
        const T *row = logits + (row0 + min(r, rows - 1)) * ld;
        uint32_t key[NV], left[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = i * G + sub;
            key[i] = r < rows && e < experts ? logit_key(row[e]) : 0u;
            left[i] = key[i];
        }
        uint32_t first = 0;
        for (int j = 0; j < k; ++j) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < NV; ++i) m = max(m, left[i]);
            m = lanes_max<G>(m);
            if (!__any(m != 0)) break;
            if (j == 0) first = m;
            uint32_t at = 0;   // the complement of the column, so that the lowest is the largest
#pragma unroll
            for (int i = NV - 1; i >= 0; --i) at = left[i] == m && m != 0 ? ~(uint32_t)(i * G + sub) : at;
            at = ~lanes_max<G>(at);
#pragma unroll
            for (int i = 0; i < NV; ++i) left[i] = at == (uint32_t)(i * G + sub) ? 0u : left[i];
        }
        const float top = key_value(first);
        float e[NV], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool taken = left[i] != key[i];
            e[i] = key[i] && (taken || !normalize) ? expf(key_value(key[i]) - top) : 0.0f;
            sum += e[i];
        }
        sum = lanes_sum<G>(sum);
        int at = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool taken = left[i] != key[i];
            const unsigned long long all = __ballot(taken), b = G == WAVE ? all : (all >> (group * G)) & ((1ull << (G % WAVE)) - 1);
            if (taken) {
                put(r * k + at + __popcll(b & ((1ull << sub) - 1)), (uint32_t)(i * G + sub) | 0x80000000u, e[i] / sum);
                atomicOr(&s_mask[i * G + sub], 1ull << r);
            }
            at += __popcll(b);
        }
        if (r < rows)
            for (int j = at + sub; j < k; j += G) put(r * k + j, 0u, 0.0f);
    }
}

template <class T, int G, int NV>
__global__ void __launch_bounds__(1024) k_route_pick(const T *logits, int64_t ld, int tokens, int experts, int k, int normalize,
                                                     RouteSpace w, int64_t blocks)
{
    __shared__ unsigned long long s_mask[NV * G];
    const int64_t row0 = (int64_t)blockIdx.x * BLOCK_ROWS;
    const int rows = (int)min((int64_t)BLOCK_ROWS, tokens - row0);
    for (int e = threadIdx.x; e < NV * G; e += blockDim.x) s_mask[e] = 0;
    __syncthreads();
    pick_rows<T, G, NV>(logits, ld, row0, rows, experts, k, normalize, s_mask, [&](int at, uint32_t pick, float weight) {
        w.pick[row0 * k + at] = pick;
        w.weight[row0 * k + at] = weight;
    });
    __syncthreads();
    for (int e = threadIdx.x; e < experts; e += blockDim.x) w.count[e * blocks + blockIdx.x] = (uint32_t)__popcll(s_mask[e]);
    for (int i = threadIdx.x; i < rows * k; i += blockDim.x) {
        const uint32_t p = w.pick[row0 * k + i];
        if (p >> 31) w.pick[row0 * k + i] = p | (uint32_t)__popcll(s_mask[p & 0xffffu] & ((1ull << (i / k)) - 1)) << 16;
    }
}

// A single block: all in one launch, and no workspace (64 rows of 64 in bfloat16, 4 taken: 5 us, the chain of loads, turns and scans).
template <class T, int G, int NV>
__global__ void __launch_bounds__(1024) k_route_one(const T *logits, int64_t ld, int tokens, int experts, int k, int normalize, ocean_routing r)
{
    __shared__ unsigned long long s_mask[NV * G];
    __shared__ uint32_t s_base[NV * G];
    __shared__ uint32_t s_pick[BLOCK_ROWS * OCEAN_ROUTE_MAX_K], s_row[BLOCK_ROWS], s_wave[1024 / WAVE];
    __shared__ float s_weight[BLOCK_ROWS * OCEAN_ROUTE_MAX_K];
    for (int e = threadIdx.x; e < NV * G; e += 1024) s_mask[e] = 0;
    __syncthreads();
    pick_rows<T, G, NV>(logits, ld, 0, tokens, experts, k, normalize, s_mask, [&](int at, uint32_t pick, float weight) {
        s_pick[at] = pick;
        s_weight[at] = weight;
    });
    __syncthreads();
    const int e = threadIdx.x;   // (at most 1024 experts)
    const uint32_t c = e < experts ? (uint32_t)__popcll(s_mask[e]) : 0u, incl = wave_inclusive_scan_u32(c);
    if (lane_id() == WAVE - 1) s_wave[threadIdx.x / WAVE] = incl;
    __syncthreads();
    uint32_t n = 0, before = incl - c;
    for (int i = 0; i < 1024 / WAVE; ++i) {
        if (i < (int)threadIdx.x / WAVE) before += s_wave[i];
        n += s_wave[i];
    }
    if (e < experts) {
        s_base[e] = before;
        r.expert_ptr[e] = before;
    }
    if (threadIdx.x < WAVE) {
        uint32_t mine = 0;
        if ((int)threadIdx.x < tokens)
            for (int j = 0; j < k; ++j) mine += s_pick[threadIdx.x * k + j] >> 31;
        const uint32_t upto = wave_inclusive_scan_u32(mine);
        s_row[threadIdx.x] = upto - mine;
        if ((int)threadIdx.x < tokens) r.row_ptr[threadIdx.x] = upto - mine;
    }
    if (threadIdx.x == 0) { r.expert_ptr[experts] = n; r.row_ptr[tokens] = n; }
    __syncthreads();
    for (int i = threadIdx.x; i < tokens * k; i += 1024) {
        const uint32_t v = s_pick[i];
        if (v >> 31) {
            const uint32_t col = v & 0xffffu, p = s_row[i / k] + i % k, slot = s_base[col] + (uint32_t)__popcll(s_mask[col] & ((1ull << (i / k)) - 1));
            r.col_idx[p] = (int32_t)col;
            r.val[p] = s_weight[i];
            r.slot[p] = (int32_t)slot;
            r.token[slot] = i / k;
        }
        if (i >= (int)n) {
            r.col_idx[i] = -1;
            r.val[i] = 0.0f;
            r.slot[i] = -1;
            r.token[i] = -1;
        }
    }
}

// Entries of earlier blocks, per expert (one workgroup each), and the expert's entries (512 blocks, 100 experts: 4 us, a launch and one scan).
__global__ void __launch_bounds__(PLACE_TPB) k_route_scan(uint32_t *count, uint32_t *total, int64_t blocks)
{
    __shared__ uint32_t s_wave[PLACE_TPB / WAVE];
    uint32_t *c = count + blockIdx.x * blocks;
    uint32_t before = 0;
    for (int64_t b0 = 0; b0 < blocks; b0 += PLACE_TPB) {
        const int64_t b = b0 + threadIdx.x;
        const uint32_t v = b < blocks ? c[b] : 0u;
        const uint32_t incl = wave_inclusive_scan_u32(v);
        if (lane_id() == WAVE - 1) s_wave[threadIdx.x / WAVE] = incl;
        __syncthreads();
        uint32_t mine = before;
        for (int i = 0; i < PLACE_TPB / WAVE; ++i) {
            if (i < (int)threadIdx.x / WAVE) mine += s_wave[i];
            before += s_wave[i];
        }
        if (b < blocks) c[b] = mine + incl - v;
        __syncthreads();
    }
    if (threadIdx.x == 0) total[blockIdx.x] = before;
}

// Entries go to their places in both orders (32768 rows of 100, 8 taken: 6 us, 5 MB of entries).
__global__ void __launch_bounds__(PLACE_TPB) k_route_place(RouteSpace w, int64_t blocks, int tokens, int experts, int k, ocean_routing r)
{
    __shared__ uint32_t s_base[OCEAN_ROUTE_MAX_EXPERTS];   // slot of the block's first entry of each expert
    __shared__ uint32_t s_row[BLOCK_ROWS + 1];
    __shared__ uint32_t s_wave[PLACE_TPB / WAVE], s_earlier[PLACE_TPB / WAVE];
    const int64_t block = blockIdx.x, row0 = block * BLOCK_ROWS;
    const int rows = (int)min((int64_t)BLOCK_ROWS, tokens - row0);
    uint32_t before = 0, earlier = 0;   // entries of lower experts; entries of earlier blocks
    for (int e0 = 0; e0 < experts; e0 += PLACE_TPB) {
        const int e = e0 + threadIdx.x;
        const uint32_t n = e < experts ? w.total[e] : 0u, c = e < experts ? w.count[e * blocks + block] : 0u;
        const uint32_t incl = wave_inclusive_scan_u32(n), cincl = wave_inclusive_scan_u32(c);
        if (lane_id() == WAVE - 1) { s_wave[threadIdx.x / WAVE] = incl; s_earlier[threadIdx.x / WAVE] = cincl; }
        __syncthreads();
        uint32_t mine = before;
        for (int i = 0; i < PLACE_TPB / WAVE; ++i) {
            if (i < (int)threadIdx.x / WAVE) mine += s_wave[i];
            before += s_wave[i];
            earlier += s_earlier[i];
        }
        if (e < experts) {
            s_base[e] = mine + incl - n + c;
            if (block == 0) r.expert_ptr[e] = mine + incl - n;
        }
        __syncthreads();
    }
    const uint32_t n = before;   // entries of R
    if (threadIdx.x < WAVE) {
        uint32_t c = 0;
        if ((int)threadIdx.x < rows)
            for (int j = 0; j < k; ++j) c += w.pick[(row0 + threadIdx.x) * k + j] >> 31;
        const uint32_t incl = wave_inclusive_scan_u32(c);
        s_row[threadIdx.x] = earlier + incl - c;
        if ((int)threadIdx.x < rows) r.row_ptr[row0 + threadIdx.x] = earlier + incl - c;
    }
    if (block == 0 && threadIdx.x == 0) { r.expert_ptr[experts] = n; r.row_ptr[tokens] = n; }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * k; i += PLACE_TPB) {
        const uint32_t v = w.pick[row0 * k + i];
        if (!(v >> 31)) continue;
        const uint32_t p = s_row[i / k] + i % k, e = v & 0xffffu, slot = s_base[e] + ((v >> 16) & 0x3fu);
        r.col_idx[p] = (int32_t)e;
        r.val[p] = w.weight[row0 * k + i];
        r.slot[p] = (int32_t)slot;
        r.token[slot] = (int32_t)(row0 + i / k);
    }
    for (int64_t p = n + block * PLACE_TPB + threadIdx.x; p < (int64_t)tokens * k; p += blocks * PLACE_TPB) {   // places of masked rows
        r.col_idx[p] = -1;
        r.val[p] = 0.0f;
        r.slot[p] = -1;
        r.token[p] = -1;
    }
}

// Gradient of a row's logits, G lanes a row.  Weights over the entries taken: dl_c = w_c (g_c - m) with m = sum w g;
// over all: p_e ([e taken] g_e - m).  The row's gradient is put together in LDS, where an entry finds its column; in single precision, 32768
// rows of 100, 8 taken, over all: 11 us, where the bytes would take 6 at the rate of a large copy (over the entries taken 7 and 3).
template <class T, int G, int NV>
__global__ void __launch_bounds__(256) k_route_backward(ocean_routing r, const float *dval, const T *logits, int64_t ld, int normalize,
                                                        T *dlogits, int64_t ldd)
{
    constexpr int ROWS = 256 / G;
    __shared__ float s_g[ROWS][NV * G];
    const int sub = lane_id() % G, experts = (int)r.experts, at = threadIdx.x / G;
    const int64_t cap = r.tokens * r.k;
    float *g = s_g[at];
    for (int64_t t0 = (int64_t)blockIdx.x * ROWS; t0 < r.tokens; t0 += (int64_t)gridDim.x * ROWS) {
        const bool there = t0 + at < r.tokens;
        const int64_t t = there ? t0 + at : r.tokens - 1;
#pragma unroll
        for (int i = 0; i < NV; ++i) g[i * G + sub] = 0.0f;
        uint32_t key[NV], first = 0;
        if (!normalize) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int e = i * G + sub;
                key[i] = e < experts ? logit_key(logits[t * ld + e]) : 0u;
            }
        }
        wave_sync();
        const int64_t lo = min(max(r.row_ptr[t], (int64_t)0), cap), hi = min(max(r.row_ptr[t + 1], lo), lo + min(cap - lo, (int64_t)OCEAN_ROUTE_MAX_K));
        float mean = 0.0f;
        constexpr int TURNS = OCEAN_ROUTE_MAX_K / G;
        int col[TURNS];
        float weight[TURNS], grad[TURNS];
#pragma unroll
        for (int j = 0; j < TURNS; ++j) {
            const int64_t p = lo + j * G + sub;
            col[j] = p < hi ? r.col_idx[p] : -1;
            weight[j] = p < hi ? r.val[p] : 0.0f;
            grad[j] = p < hi ? dval[p] : 0.0f;
            mean += weight[j] * grad[j];
        }
        mean = lanes_sum<G>(mean);
#pragma unroll
        for (int j = 0; j < TURNS; ++j)
            if ((unsigned)col[j] < (unsigned)experts) g[col[j]] = normalize ? weight[j] * (grad[j] - mean) : weight[j] * grad[j];
        wave_sync();
        float scale = 0.0f, e[NV];
        if (!normalize) {
#pragma unroll
            for (int i = 0; i < NV; ++i) first = max(first, key[i]);
            const float top = key_value(lanes_max<G>(first));
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                e[i] = key[i] ? expf(key_value(key[i]) - top) : 0.0f;
                sum += e[i];
            }
            sum = lanes_sum<G>(sum);
            scale = sum > 0.0f ? mean / sum : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (there && i * G + sub < experts)   // (a masked logit's is 0 also where the scale is infinite or NaN)
                dlogits[t * ldd + i * G + sub] = (T)(normalize || !key[i] ? g[i * G + sub] : g[i * G + sub] - e[i] * scale);
        wave_sync();
    }
}

// Calls f with the lanes that share a row and the columns of a lane as constants.
template <class F> hipError_t with_columns(int64_t experts, F f)
{
    using std::integral_constant;
    if (experts <= 16) return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    if (experts <= 32) return f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
    if (experts <= 64) return f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
    if (experts <= 128) return f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
    if (experts <= 256) return f(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    if (experts <= 512) return f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    return f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

}  // namespace

size_t route_workspace(int64_t tokens, int64_t experts, int32_t k)
{
    size_t bytes;
    if (route_blocks(tokens) <= 1) return 0;
    route_space(nullptr, tokens, experts, k, &bytes);
    return bytes;
}

hipError_t launch_route(const void *logits, int dtype, int64_t ld, bool normalize, const ocean_routing &r, void *workspace, hipStream_t s)
{
    const int64_t blocks = route_blocks(r.tokens);
    const int tokens = (int)r.tokens, experts = (int)r.experts, k = r.k;
    if (blocks <= 1)
        return with_type(dtype, [&](auto t) {
            using T = decltype(t);
            return with_columns(r.experts, [&](auto g, auto nv) {
                hipLaunchKernelGGL((k_route_one<T, decltype(g)::value, decltype(nv)::value>), dim3(1), dim3(1024), 0, s, static_cast<const T *>(logits), ld,
                                   tokens, experts, k, normalize ? 1 : 0, r);
                return hipGetLastError();
            });
        });
    size_t bytes;
    const RouteSpace w = route_space(workspace, r.tokens, r.experts, r.k, &bytes);
    hipError_t e = with_type(dtype, [&](auto t) {
        using T = decltype(t);
        return with_columns(r.experts, [&](auto g, auto nv) {
            // (16 waves, so that a wave has few rows one after the other, while there are not many blocks)
            hipLaunchKernelGGL((k_route_pick<T, decltype(g)::value, decltype(nv)::value>), dim3((uint32_t)blocks), dim3(blocks < 2048 ? 1024 : 256), 0, s,
                               static_cast<const T *>(logits), ld, tokens, experts, k, normalize ? 1 : 0, w, blocks);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_route_scan, dim3((uint32_t)experts), dim3(PLACE_TPB), 0, s, w.count, w.total, blocks);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_route_place, dim3((uint32_t)blocks), dim3(PLACE_TPB), 0, s, w, blocks, tokens, experts, k, r);
    return hipGetLastError();
}

hipError_t launch_route_backward(const ocean_routing &r, const float *dval, const void *logits, int dtype, int64_t ld, bool normalize,
                                 void *dlogits, int64_t ldd, hipStream_t s)
{
    if (r.tokens == 0) return hipSuccess;
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        return with_columns(r.experts, [&](auto g, auto nv) {
            constexpr int G = decltype(g)::value;
            hipLaunchKernelGGL((k_route_backward<T, G, decltype(nv)::value>), dim3((uint32_t)std::min((r.tokens * G + 255) / 256, (int64_t)1 << 20)), dim3(256), 0, s, r, dval,
                               static_cast<const T *>(logits), ld, normalize ? 1 : 0, static_cast<T *>(dlogits), ldd);
            return hipGetLastError();
        });
    });
}

}  // namespace ocean
