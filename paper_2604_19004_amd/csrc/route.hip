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

// Takes the largest logits of the block's rows, one wave a row.  Lane l has the logits of columns l, l + 64, ...: the
// largest key of the wave, then the lowest column that holds it by ballots.  A row's softmax is relative to its largest logit.
// The bits of s_mask (expert: which of the 64 rows took it) give the entries' rank among the block's of the same column without
// an order of arrival.
template <class T, int NV>
__global__ void __launch_bounds__(1024) k_route_pick(const T *logits, int64_t ld, int tokens, int experts, int k, int normalize,
                                                     RouteSpace w, int64_t blocks)
{
    __shared__ unsigned long long s_mask[NV * WAVE];
    const int lane = lane_id(), wave = threadIdx.x / WAVE, waves = blockDim.x / WAVE;
    const int64_t row0 = (int64_t)blockIdx.x * BLOCK_ROWS;
    const int rows = (int)min((int64_t)BLOCK_ROWS, tokens - row0);
    for (int e = threadIdx.x; e < NV * WAVE; e += blockDim.x) s_mask[e] = 0;
    __syncthreads();
    for (int r = wave; r < rows; r += waves) {
        const T *row = logits + (row0 + r) * ld;
        uint32_t key[NV], left[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = i * WAVE + lane;
            key[i] = e < experts ? logit_key(row[e]) : 0u;
            left[i] = key[i];
        }
        uint32_t first = 0;
        for (int j = 0; j < k; ++j) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < NV; ++i) m = max(m, left[i]);
            m = wave_max_u32(m);
            if (m == 0) break;
            if (j == 0) first = m;
            bool found = false;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const unsigned long long b = __ballot(left[i] == m);
                if (!found && b) {
                    found = true;
                    if (lane == __ffsll(b) - 1) left[i] = 0;
                }
            }
        }
        const float top = key_value(first);
        float e[NV], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool taken = left[i] != key[i];
            e[i] = key[i] ? expf(key_value(key[i]) - top) : 0.0f;
            sum += (taken || !normalize) ? e[i] : 0.0f;
        }
        sum = wave_sum(sum);
        int at = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool taken = left[i] != key[i];
            const unsigned long long b = __ballot(taken);
            if (taken) {
                const int64_t p = (row0 + r) * k + at + __popcll(b & ((1ull << lane) - 1));
                w.pick[p] = (uint32_t)(i * WAVE + lane) | 0x80000000u;
                w.weight[p] = e[i] / sum;
                atomicOr(&s_mask[i * WAVE + lane], 1ull << r);
            }
            at += __popcll(b);
        }
        for (int j = at + lane; j < k; j += WAVE) w.pick[(row0 + r) * k + j] = 0;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < experts; e += blockDim.x) w.count[e * blocks + blockIdx.x] = (uint32_t)__popcll(s_mask[e]);
    for (int i = threadIdx.x; i < rows * k; i += blockDim.x) {
        const uint32_t p = w.pick[row0 * k + i];
        if (p >> 31) w.pick[row0 * k + i] = p | (uint32_t)__popcll(s_mask[p & 0xffffu] & ((1ull << (i / k)) - 1)) << 16;
    }
}

// Entries of earlier blocks, per expert (one workgroup each), and the expert's entries.
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

// Entries go to their places in both orders.
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

// Gradient of a row's logits, one wave a row.  Weights over the entries taken: dl_c = w_c (g_c - m) with m = sum w g;
// over all: p_e ([e taken] g_e - m).
template <class T, int NV>
__global__ void __launch_bounds__(256) k_route_backward(ocean_routing r, const float *dval, const T *logits, int64_t ld, int normalize,
                                                        T *dlogits, int64_t ldd)
{
    __shared__ float s_g[256 / WAVE][NV * WAVE];
    const int lane = lane_id(), experts = (int)r.experts;
    float *g = s_g[threadIdx.x / WAVE];
    for (int64_t t = (int64_t)blockIdx.x * (256 / WAVE) + threadIdx.x / WAVE; t < r.tokens; t += (int64_t)gridDim.x * (256 / WAVE)) {
#pragma unroll
        for (int i = 0; i < NV; ++i) g[i * WAVE + lane] = 0.0f;
        wave_sync();
        const int64_t cap = r.tokens * r.k;
        const int64_t lo = min(max(r.row_ptr[t], (int64_t)0), cap), hi = min(max(r.row_ptr[t + 1], lo), lo + min(cap - lo, (int64_t)WAVE));
        int col = -1;
        float weight = 0.0f, grad = 0.0f;
        if (lo + lane < hi) {
            col = r.col_idx[lo + lane];
            weight = r.val[lo + lane];
            grad = dval[lo + lane];
        }
        const float mean = wave_sum(weight * grad);
        if ((unsigned)col < (unsigned)experts) g[col] = normalize ? weight * (grad - mean) : weight * grad;
        wave_sync();
        if (normalize) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i * WAVE + lane < experts) dlogits[t * ldd + i * WAVE + lane] = (T)g[i * WAVE + lane];
            continue;
        }
        uint32_t key[NV], first = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = i * WAVE + lane;
            key[i] = e < experts ? logit_key(logits[t * ld + e]) : 0u;
            first = max(first, key[i]);
        }
        const float top = key_value(wave_max_u32(first));
        float e[NV], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            e[i] = key[i] ? expf(key_value(key[i]) - top) : 0.0f;
            sum += e[i];
        }
        sum = wave_sum(sum);
        const float scale = sum > 0.0f ? mean / sum : 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * WAVE + lane < experts) dlogits[t * ldd + i * WAVE + lane] = (T)(g[i * WAVE + lane] - e[i] * scale);
    }
}

// Calls f with the number of 64-column registers as a constant.
template <class F> hipError_t with_columns(int64_t experts, F f)
{
    if (experts <= 64) return f(std::integral_constant<int, 1>{});
    if (experts <= 128) return f(std::integral_constant<int, 2>{});
    if (experts <= 256) return f(std::integral_constant<int, 4>{});
    if (experts <= 512) return f(std::integral_constant<int, 8>{});
    return f(std::integral_constant<int, 16>{});
}

}  // namespace

size_t route_workspace(int64_t tokens, int64_t experts, int32_t k)
{
    size_t bytes;
    route_space(nullptr, tokens, experts, k, &bytes);
    return bytes;
}

hipError_t launch_route(const void *logits, int dtype, int64_t ld, bool normalize, const ocean_routing &r, void *workspace, hipStream_t s)
{
    size_t bytes;
    const RouteSpace w = route_space(workspace, r.tokens, r.experts, r.k, &bytes);
    const int64_t blocks = route_blocks(r.tokens);
    const int tokens = (int)r.tokens, experts = (int)r.experts, k = r.k;
    if (blocks > 0) {
        hipError_t e = with_type(dtype, [&](auto t) {
            using T = decltype(t);
            return with_columns(r.experts, [&](auto nv) {
                hipLaunchKernelGGL((k_route_pick<T, decltype(nv)::value>), dim3((uint32_t)blocks), dim3(blocks < 256 ? 1024 : 256), 0, s,
                                   static_cast<const T *>(logits), ld, tokens, experts, k, normalize ? 1 : 0, w, blocks);
                return hipGetLastError();
            });
        });
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(k_route_scan, dim3((uint32_t)experts), dim3(PLACE_TPB), 0, s, w.count, w.total, blocks);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_route_place, dim3((uint32_t)(blocks > 0 ? blocks : 1)), dim3(PLACE_TPB), 0, s, w, blocks, tokens, experts, k, r);
    return hipGetLastError();
}

hipError_t launch_route_backward(const ocean_routing &r, const float *dval, const void *logits, int dtype, int64_t ld, bool normalize,
                                 void *dlogits, int64_t ldd, hipStream_t s)
{
    if (r.tokens == 0) return hipSuccess;
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        return with_columns(r.experts, [&](auto nv) {
            hipLaunchKernelGGL((k_route_backward<T, decltype(nv)::value>), dim3((uint32_t)std::min((r.tokens + 3) / 4, (int64_t)1 << 20)), dim3(256), 0, s, r, dval,
                               static_cast<const T *>(logits), ld, normalize ? 1 : 0, static_cast<T *>(dlogits), ldd);
            return hipGetLastError();
        });
    });
}

}  // namespace ocean
