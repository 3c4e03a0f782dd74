// The losses that keep a router's experts evenly used, and the gradient of the logits.
#include <algorithm>

#include "experts.hpp"
#include "rowlanes.hpp"

namespace ocean {

namespace {

constexpr int TPB = 256, FINISH_TPB = 1024;
constexpr int64_t MAX_BLOCKS = 256;   // workgroups of the first pass, each of which leaves a sum per expert

// Sums of a workgroup's rows, per expert, of logsumexp^2, and its rows that have an open logit.
struct BalanceSpace {
    float *prob;        // [blocks][experts]
    float *z;           // [blocks]
    int64_t *rows;      // [blocks]
};
inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
inline BalanceSpace balance_space(void *at, int64_t experts, size_t *bytes)
{
    char *p = static_cast<char *>(at);
    size_t o = 0;
    BalanceSpace w;
    w.rows = reinterpret_cast<int64_t *>(p + o);
    o += up256(MAX_BLOCKS * 8);
    w.z = reinterpret_cast<float *>(p + o);
    o += up256(MAX_BLOCKS * 4);
    w.prob = reinterpret_cast<float *>(p + o);
    o += up256((size_t)MAX_BLOCKS * experts * 4);
    *bytes = o;
    return w;
}

// A row's softmax relative to its largest logit: e[i] = exp(logit - top) (0: masked), their sum (0: the row has no open logit), and its
// logsumexp = top + log(sum).
template <class T, int G, int NV>
__device__ __forceinline__ float row_softmax(const T *row, int experts, bool there, uint32_t (&key)[NV], float (&e)[NV], float &top)
{
    const int sub = lane_id() % G;
    uint32_t first = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = i * G + sub;
        key[i] = there && c < experts ? logit_key(row[c]) : 0u;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) first = max(first, key[i]);
    first = lanes_max<G>(first);
    top = first ? key_value(first) : 0.0f;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        e[i] = key[i] ? expf(key_value(key[i]) - top) : 0.0f;
        sum += e[i];
    }
    return lanes_sum<G>(sum);
}

// G lanes share a row and keep their columns' sums over all rows that they see; those of a workgroup meet in LDS in a fixed order.
template <class T, int G, int NV>
__global__ void __launch_bounds__(TPB) k_balance(const T *logits, int64_t ld, int64_t tokens, int experts, BalanceSpace w)
{
    constexpr int GROUPS = TPB / G;
    __shared__ float s_prob[GROUPS][NV * G];
    __shared__ float s_z[GROUPS];
    __shared__ int s_rows[GROUPS];
    const int sub = lane_id() % G, group = threadIdx.x / G;
    float prob[NV] = {}, z = 0.0f;
    int rows = 0;
    for (int64_t t0 = (int64_t)blockIdx.x * GROUPS; t0 < tokens; t0 += (int64_t)gridDim.x * GROUPS) {
        const int64_t t = t0 + group;
        uint32_t key[NV];
        float e[NV], top;
        const float sum = row_softmax<T, G, NV>(logits + min(t, tokens - 1) * ld, experts, t < tokens, key, e, top);
        const float scale = sum > 0.0f ? 1.0f / sum : 0.0f, lse = sum > 0.0f ? top + logf(sum) : 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) prob[i] += e[i] * scale;
        z += lse * lse;
        rows += sum > 0.0f;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) s_prob[group][i * G + sub] = prob[i];
    if (sub == 0) {
        s_z[group] = z;
        s_rows[group] = rows;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < experts; c += TPB) {
        float v = 0.0f;
        for (int i = 0; i < GROUPS; ++i) v += s_prob[i][c];
        w.prob[(int64_t)blockIdx.x * experts + c] = v;
    }
    if (threadIdx.x == 0) {
        float v = 0.0f;
        int64_t n = 0;
        for (int i = 0; i < GROUPS; ++i) {
            v += s_z[i];
            n += s_rows[i];
        }
        w.z[blockIdx.x] = v;
        w.rows[blockIdx.x] = n;
    }
}

__device__ __forceinline__ int64_t entries_of(const int64_t *expert_ptr, int e) { return max(expert_ptr[e + 1] - expert_ptr[e], (int64_t)0); }

// The workgroups' sums together, in 64 bits.
__global__ void __launch_bounds__(FINISH_TPB) k_balance_finish(const int64_t *expert_ptr, int experts, int blocks, BalanceSpace w, ocean_balance out)
{
    __shared__ double s_sum[FINISH_TPB];
    __shared__ double s_f[FINISH_TPB / WAVE];
    __shared__ int64_t s_n[FINISH_TPB / WAVE];
    const int tid = threadIdx.x, cols = min(FINISH_TPB, (experts + WAVE - 1) / WAVE * WAVE), parts = FINISH_TPB / cols;
    const int part = tid / cols, c = tid % cols;
    double v = 0.0;
    if (c < experts && part < parts)
        for (int b = part; b < blocks; b += parts) v += (double)w.prob[(int64_t)b * experts + c];
    s_sum[tid] = v;
    int64_t rows = 0;
    double z = 0.0;
    for (int b = tid; b < blocks; b += FINISH_TPB) {
        rows += w.rows[b];
        z += (double)w.z[b];
    }
    auto all = [&](auto x, auto *lds) {   // sum over the workgroup
        for (int d = WAVE / 2; d > 0; d >>= 1) x += __shfl_xor(x, d);
        __syncthreads();
        if (lane_id() == 0) lds[tid / WAVE] = x;
        __syncthreads();
        x = 0;
        for (int i = 0; i < FINISH_TPB / WAVE; ++i) x += lds[i];
        return x;
    };
    rows = all(rows, s_n);
    z = all(z, s_f);
    const int64_t count = tid < experts ? entries_of(expert_ptr, tid) : 0, n = all(count, s_n);
    double prob = 0.0;
    if (tid < experts) {
        for (int p = 0; p < parts; ++p) prob += s_sum[p * cols + tid];
        prob = rows > 0 ? prob / (double)rows : 0.0;
        out.prob[tid] = (float)prob;
        out.counts[tid] = count;
    }
    const double balance = all(n > 0 ? (double)count / (double)n * prob : 0.0, s_f);
    if (tid == 0) {
        out.loss[0] = (float)(balance * experts);
        out.loss[1] = rows > 0 ? (float)(z / (double)rows) : 0.0f;
        out.rows[0] = rows;
    }
}

// dl_c = p_c (a (f_c - sum f p) + b lse) with f the experts' shares of the entries, a = dloss[0] experts / rows and b = 2 dloss[1] / rows; with `dval` what
// k_route_backward gives beside it.
template <class T, int G, int NV, bool WEIGHTS>
__global__ void __launch_bounds__(TPB) k_balance_backward(ocean_balance b, ocean_routing r, const float *dloss, const float *dval, const T *logits,
                                                          int64_t ld, int normalize, T *dlogits, int64_t ldd)
{
    constexpr int ROWS = TPB / G;
    __shared__ float s_g[WEIGHTS ? ROWS : 1][WEIGHTS ? NV * G : 1];
    const int sub = lane_id() % G, experts = (int)r.experts, at = threadIdx.x / G;
    const int64_t cap = r.tokens * r.k, rows = b.rows[0];
    float share[NV], total = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        share[i] = i * G + sub < experts ? (float)max(b.counts[i * G + sub], (int64_t)0) : 0.0f;
        total += share[i];
    }
    total = lanes_sum<G>(total);
    const float per_row = rows > 0 ? 1.0f / (float)rows : 0.0f, even = dloss[0] * per_row * (float)experts, size = 2.0f * dloss[1] * per_row;
#pragma unroll
    for (int i = 0; i < NV; ++i) share[i] = total > 0.0f ? share[i] / total : 0.0f;
    for (int64_t t0 = (int64_t)blockIdx.x * ROWS; t0 < r.tokens; t0 += (int64_t)gridDim.x * ROWS) {
        const bool there = t0 + at < r.tokens;
        const int64_t t = there ? t0 + at : r.tokens - 1;
        uint32_t key[NV];
        float e[NV], top;
        const float sum = row_softmax<T, G, NV>(logits + t * ld, experts, there, key, e, top);
        const float scale = sum > 0.0f ? 1.0f / sum : 0.0f, lse = sum > 0.0f ? top + logf(sum) : 0.0f;
        float met = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            e[i] *= scale;
            met += e[i] * share[i];
        }
        met = lanes_sum<G>(met);
        float mean = 0.0f;
        if constexpr (WEIGHTS) {
            float *g = s_g[at];
#pragma unroll
            for (int i = 0; i < NV; ++i) g[i * G + sub] = 0.0f;
            wave_sync();
            const int64_t lo = min(max(r.row_ptr[t], (int64_t)0), cap), hi = min(max(r.row_ptr[t + 1], lo), lo + min(cap - lo, (int64_t)OCEAN_ROUTE_MAX_K));
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
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = i * G + sub;
            if (!there || c >= experts) continue;
            float v = e[i] > 0.0f ? e[i] * (even * (share[i] - met) + size * lse) : 0.0f;
            if constexpr (WEIGHTS) v += normalize ? s_g[at][c] : s_g[at][c] - e[i] * mean;
            dlogits[t * ldd + c] = (T)(key[i] ? v : 0.0f);   // (masked: also where a loss's gradient is infinite or NaN)
        }
        if constexpr (WEIGHTS) wave_sync();
    }
}

}  // namespace

size_t balance_workspace(int64_t tokens, int64_t experts)
{
    size_t bytes;
    balance_space(nullptr, experts, &bytes);
    return bytes;
}

hipError_t launch_balance(const ocean_routing &r, const void *logits, int dtype, int64_t ld, const ocean_balance &out, void *workspace, hipStream_t s)
{
    size_t bytes;
    const BalanceSpace w = balance_space(workspace, r.experts, &bytes);
    int blocks = 0;
    if (r.tokens > 0) {
        const hipError_t e = with_type(dtype, [&](auto t) {
            using T = decltype(t);
            return with_columns(r.experts, [&](auto g, auto nv) {
                constexpr int G = decltype(g)::value, ROWS = TPB / G;
                blocks = (int)std::min((r.tokens + ROWS - 1) / ROWS, MAX_BLOCKS);
                hipLaunchKernelGGL((k_balance<T, G, decltype(nv)::value>), dim3(blocks), dim3(TPB), 0, s, static_cast<const T *>(logits), ld, r.tokens,
                                   (int)r.experts, w);
                return hipGetLastError();
            });
        });
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(k_balance_finish, dim3(1), dim3(FINISH_TPB), 0, s, r.expert_ptr, (int)r.experts, blocks, w, out);
    return hipGetLastError();
}

hipError_t launch_balance_backward(const ocean_balance &b, const ocean_routing &r, const void *logits, int dtype, int64_t ld, const float *dloss,
                                   const float *dval, bool normalize, void *dlogits, int64_t ldd, hipStream_t s)
{
    if (r.tokens == 0) return hipSuccess;
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        return with_columns(r.experts, [&](auto g, auto nv) {
            constexpr int G = decltype(g)::value, NV = decltype(nv)::value;
            const dim3 grid((uint32_t)std::min((r.tokens * G + TPB - 1) / TPB, (int64_t)1 << 20));
            auto launch = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, grid, dim3(TPB), 0, s, b, r, dloss, dval, static_cast<const T *>(logits), ld, normalize ? 1 : 0,
                                   static_cast<T *>(dlogits), ldd);
                return hipGetLastError();
            };
            return dval ? launch(k_balance_backward<T, G, NV, true>) : launch(k_balance_backward<T, G, NV, false>);
        });
    });
}

}  // namespace ocean
