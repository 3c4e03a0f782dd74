// The losses that keep a router's experts evenly used, and the gradient of the logits.
#include <algorithm>

#include "experts.hpp"
#include "rowlanes.hpp"

namespace ocean {

namespace {

constexpr int TPB = 256, SUM_TPB = 1024, FINISH_TPB = 1024;
constexpr int64_t AT_ONCE = 1536;     // workgroups of the gradient that run together, six a compute unit
constexpr int64_t MAX_BLOCKS = 256;   // workgroups of the first pass, each of which leaves a sum per expert

// Sums of a workgroup's rows, per expert, of logsumexp^2 (in 64 bits: those of a mean that single precision has may be beyond it), and its rows that have an open logit.
struct BalanceSpace {
    float *prob;        // [blocks][experts]
    double *z;          // [blocks]
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
    w.z = reinterpret_cast<double *>(p + o);
    o += up256(MAX_BLOCKS * 8);
    w.prob = reinterpret_cast<float *>(p + o);
    o += up256((size_t)MAX_BLOCKS * experts * 4);
    *bytes = o;
    return w;
}

// The rows of a turn of the workgroup, from row t0 on: what lies behind the last row reads as 0 and is not written.
template <class T> __device__ __forceinline__ Memory rows_from(const T *p, int64_t ld, int64_t t0, int64_t tokens, int experts)
{
    const int64_t bytes = t0 < tokens ? ((tokens - 1 - t0) * ld + experts) * (int64_t)sizeof(T) : 0;
    return memory_at(p + t0 * ld, (uint32_t)min(bytes, (int64_t)MEMORY_BYTES));
}
// Offsets of a lane's columns of row `row` of a turn.
template <class T, int G, int NV> __device__ __forceinline__ void offsets_of(uint32_t (&at)[NV], int row, int64_t ld, int experts)
{
    const int sub = lane_id() % G;
#pragma unroll
    for (int i = 0; i < NV; ++i) at[i] = i * G + sub < experts ? (uint32_t)((row * ld + i * G + sub) * (int64_t)sizeof(T)) : NOWHERE;
}
template <class T> __device__ __forceinline__ T load_one(Memory m, uint32_t at)
{
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(T, (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(m, at, 0, 0));
    else return __builtin_bit_cast(T, (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(m, at, 0, 0));
}
template <class T> __device__ __forceinline__ void store_one(T v, Memory m, uint32_t at)
{
    if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), m, at, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), m, at, 0, 0);
}

// e^d for d <= 0: 2^(d log2 e) with what the product's rounding left, off by two roundings or so; below 2^-126 it is 0.
__device__ __forceinline__ float exp_of(float d)
{
    constexpr float LOG2E = 1.44269504f, REST = (float)(1.4426950408889634074 - (double)LOG2E), LN2 = 0.693147181f;
    const float t = d * LOG2E, left = fmaf(d, REST, fmaf(d, LOG2E, -t)), e = __builtin_amdgcn_exp2f(t);
    return d > -1e30f ? fmaf(e, left * LN2, e) : 0.0f;   // (-inf, where t - t is NaN)
}

template <int G> __device__ __forceinline__ float lanes_top(float v)
{
    if constexpr (G == 16)
        return __uint_as_float(row16(__float_as_uint(v), [](uint32_t x, uint32_t y) { return __float_as_uint(fmaxf(__uint_as_float(x), __uint_as_float(y))); }));
    else return key_value(lanes_max<G>(order_key(v)));
}

// A row's softmax relative to its largest logit: e[i] = exp(x[i] - top), their sum (0: the row has no open logit).  x: the logits, -inf where they are masked or
// not there.
template <class T, int G, int NV>
__device__ __forceinline__ float row_softmax(const T (&row)[NV], const uint32_t (&at)[NV], bool there, float (&x)[NV], float (&e)[NV], float &top)
{
    top = -INFINITY;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const float v = (float)row[i];
        x[i] = v > TypeTraits<T>::lowest && at[i] != NOWHERE ? fminf(v, -TypeTraits<T>::lowest) : -INFINITY;   // (NaN is not)
        top = fmaxf(top, x[i]);
    }
    top = lanes_top<G>(there ? top : -INFINITY);
    if (!(top > -INFINITY)) top = 0.0f;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        e[i] = exp_of(x[i] - top);
        sum += e[i];
    }
    sum = lanes_sum<G>(sum);
    return there ? sum : 0.0f;
}

template <class V> __device__ __forceinline__ V wave_total(V v)
{
#pragma unroll
    for (int d = WAVE / 2; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// G lanes share a row and keep their columns' sums over all rows that they see; those of a workgroup meet in LDS in a fixed order.  65536 rows of 100, f32: 9.5 us for
// 26 MB, of which 870 instructions a wave, four waves to a SIMD, are 6.
template <class T, int G, int NV>
__global__ void __launch_bounds__(SUM_TPB) k_balance(const T *logits, int64_t ld, int64_t tokens, int experts, BalanceSpace w)
{
    constexpr int GROUPS = SUM_TPB / G;
    __shared__ float s_prob[GROUPS][NV * G];
    __shared__ double s_z[GROUPS];
    __shared__ int s_rows[GROUPS];
    const int sub = lane_id() % G, group = threadIdx.x / G;
    float prob[NV] = {};
    double z = 0.0;
    int rows = 0;
    uint32_t at[NV];
    offsets_of<T, G, NV>(at, group, ld, experts);
    T now[NV], next[NV];
    auto load = [&](T (&to)[NV], int64_t t0) {
        const Memory m = rows_from(logits, ld, t0, tokens, experts);
#pragma unroll
        for (int i = 0; i < NV; ++i) to[i] = load_one<T>(m, at[i]);
    };
    load(now, (int64_t)blockIdx.x * GROUPS);
    for (int64_t t0 = (int64_t)blockIdx.x * GROUPS; t0 < tokens; t0 += (int64_t)gridDim.x * GROUPS) {
        load(next, t0 + (int64_t)gridDim.x * GROUPS);   // (the next row is on its way)
        float x[NV], e[NV], top;
        const float sum = row_softmax<T, G, NV>(now, at, t0 + group < tokens, x, e, top);
        const float scale = sum > 0.0f ? 1.0f / sum : 0.0f, lse = sum > 0.0f ? top + logf(sum) : 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) prob[i] += e[i] * scale;
        z = fma((double)lse, (double)lse, z);
        rows += sum > 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) now[i] = next[i];
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) s_prob[group][i * G + sub] = prob[i];
    if (sub == 0) {
        s_z[group] = z;
        s_rows[group] = rows;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < experts; c += SUM_TPB) {
        float v = 0.0f;
#pragma unroll 16
        for (int i = 0; i < GROUPS; ++i) v += s_prob[i][c];
        w.prob[(int64_t)blockIdx.x * experts + c] = v;
    }
    if (threadIdx.x >= SUM_TPB - WAVE) {   // (the last wave, which has no column unless there are many)
        const int lane = lane_id();
        double v = 0.0;
        uint32_t n = 0;
        for (int i = lane; i < GROUPS; i += WAVE) {
            v += s_z[i];
            n += (uint32_t)s_rows[i];   // (a workgroup has fewer than 2^32 rows)
        }
        v = wave_total(v);
        n = wave_sum_u32(n);
        if (lane == 0) {
            w.z[blockIdx.x] = v;
            w.rows[blockIdx.x] = n;
        }
    }
}

__device__ __forceinline__ int64_t entries_of(const int64_t *expert_ptr, int e) { return max(expert_ptr[e + 1] - expert_ptr[e], (int64_t)0); }

// The workgroups' sums together, in 64 bits: 1024 / experts threads an expert, each every so many workgroups.  A chain of two trips to memory and three barriers, 5 to 6 us.
__global__ void __launch_bounds__(FINISH_TPB) k_balance_finish(const int64_t *expert_ptr, int experts, int blocks, BalanceSpace w, ocean_balance out)
{
    constexpr int WAVES = FINISH_TPB / WAVE, DEEP = 32;
    __shared__ double s_sum[FINISH_TPB], s_z, s_f[WAVES];
    __shared__ int64_t s_rows, s_n[WAVES];
    const int tid = threadIdx.x, wave = tid / WAVE, cols = (experts + WAVE - 1) / WAVE * WAVE, parts = FINISH_TPB / cols;
    const int part = tid / cols, c = tid - part * cols;
    const int64_t count = tid < experts ? entries_of(expert_ptr, tid) : 0;
    double v = 0.0;
    if (c < experts && part < parts)
        for (int b0 = part; b0 < blocks; b0 += parts * DEEP) {
            float x[DEEP];
#pragma unroll
            for (int i = 0; i < DEEP; ++i) x[i] = w.prob[(int64_t)min(b0 + i * parts, blocks - 1) * experts + c];   // (no branch: all are under way at once)
#pragma unroll
            for (int i = 0; i < DEEP; ++i) v += (double)(b0 + i * parts < blocks ? x[i] : 0.0f);
        }
    s_sum[tid] = v;
    if (wave == WAVES - 1) {
        int64_t rows = 0;
        double z = 0.0;
#pragma unroll
        for (int i = 0; i < (int)(MAX_BLOCKS / WAVE); ++i) {
            const int b = i * WAVE + lane_id();
            rows += b < blocks ? w.rows[b] : 0;
            z += b < blocks ? w.z[b] : 0.0;
        }
        rows = wave_total(rows);
        z = wave_total(z);
        if (lane_id() == 0) s_rows = rows, s_z = z;
    }
    const int64_t n_wave = wave_total(count);
    if (lane_id() == 0) s_n[wave] = n_wave;
    __syncthreads();
    int64_t n = 0;
    for (int i = 0; i < WAVES; ++i) n += s_n[i];
    const int64_t rows = s_rows;
    double prob = 0.0;
    if (tid < experts) {
        for (int p = 0; p < parts; ++p) prob += s_sum[p * cols + tid];
        prob = rows > 0 ? prob / (double)rows : 0.0;
        out.prob[tid] = (float)prob;
        out.counts[tid] = count;
    }
    const double even = wave_total(n > 0 ? (double)count / (double)n * prob : 0.0);
    if (lane_id() == 0) s_f[wave] = even;
    __syncthreads();
    if (tid == 0) {
        double balance = 0.0;
        for (int i = 0; i < WAVES; ++i) balance += s_f[i];
        out.loss[0] = (float)(balance * experts);
        out.loss[1] = rows > 0 ? (float)(s_z / (double)rows) : 0.0f;
        out.rows[0] = rows;
    }
}

// dl_c = p_c (a (f_c - sum f p) + b lse) with f the experts' shares of the entries, a = dloss[0] experts / rows and b = 2 dloss[1] / rows; with `dval` what
// k_route_backward gives beside it.  65536 rows of 100, k 8, f32: 19 us for 59 MB (12 at the rate of a copy); 1315 instructions a wave are 12 of
// them.  Without dval 14.5 us for 52 MB.
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
    uint32_t from[NV], to[NV];
    offsets_of<T, G, NV>(from, at, ld, experts);
    offsets_of<T, G, NV>(to, at, ldd, experts);
    T now[NV], next[NV];
    auto load = [&](T (&v)[NV], int64_t t0) {
        const Memory m = rows_from(logits, ld, t0, r.tokens, experts);
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = load_one<T>(m, from[i]);
    };
    // A row's entries are loaded before its softmax is worked out, and where they lie a turn ahead.
    constexpr int TURNS = WEIGHTS ? OCEAN_ROUTE_MAX_K / G : 1;
    int64_t lo = 0, hi = 0, lo_next = 0, hi_next = 0;
    auto place = [&](int64_t t0, int64_t &first, int64_t &last) {
        const int64_t t = min(t0 + at, r.tokens - 1);
        first = r.row_ptr[t], last = r.row_ptr[t + 1];
    };
    load(now, (int64_t)blockIdx.x * ROWS);
    if constexpr (WEIGHTS) place((int64_t)blockIdx.x * ROWS, lo, hi);
    for (int64_t t0 = (int64_t)blockIdx.x * ROWS; t0 < r.tokens; t0 += (int64_t)gridDim.x * ROWS) {
        const bool there = t0 + at < r.tokens;
        int col[TURNS];
        float weight[TURNS], grad[TURNS];
        if constexpr (WEIGHTS) {
            lo = min(max(lo, (int64_t)0), cap);
            hi = min(max(hi, lo), lo + min(cap - lo, (int64_t)r.k));   // (a row has at most k)
#pragma unroll
            for (int j = 0; j < TURNS; ++j) {
                if (j > 0 && j * G >= r.k) break;   // (the same for all)
                const int64_t p = lo + j * G + sub;
                col[j] = p < hi ? r.col_idx[p] : -1;
                weight[j] = p < hi ? r.val[p] : 0.0f;
                grad[j] = p < hi ? dval[p] : 0.0f;
            }
            place(t0 + (int64_t)gridDim.x * ROWS, lo_next, hi_next);
        }
        load(next, t0 + (int64_t)gridDim.x * ROWS);
        float x[NV], e[NV], top;
        const float sum = row_softmax<T, G, NV>(now, from, there, x, e, top);
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
#pragma unroll
            for (int j = 0; j < TURNS; ++j) {
                if (j > 0 && j * G >= r.k) break;
                mean += weight[j] * grad[j];
            }
            mean = lanes_sum<G>(mean);
#pragma unroll
            for (int j = 0; j < TURNS; ++j) {
                if (j > 0 && j * G >= r.k) break;
                if ((unsigned)col[j] < (unsigned)experts) g[col[j]] = normalize ? weight[j] * (grad[j] - mean) : weight[j] * grad[j];
            }
            wave_sync();
            lo = lo_next, hi = hi_next;
        }
        const Memory out = rows_from(dlogits, ldd, t0, r.tokens, experts);
        const float all = size * lse - even * met;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float v = e[i] > 0.0f ? e[i] * fmaf(even, share[i], all) : 0.0f;
            if constexpr (WEIGHTS) v += normalize ? s_g[at][i * G + sub] : s_g[at][i * G + sub] - e[i] * mean;
            store_one<T>((T)(x[i] > -INFINITY ? v : 0.0f), out, to[i]);   // (masked: also where a loss's gradient is infinite or NaN)
        }
        if constexpr (WEIGHTS) wave_sync();
#pragma unroll
        for (int i = 0; i < NV; ++i) now[i] = next[i];
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
                constexpr int G = decltype(g)::value, ROWS = SUM_TPB / G;
                blocks = (int)std::min((r.tokens + ROWS - 1) / ROWS, MAX_BLOCKS);
                hipLaunchKernelGGL((k_balance<T, G, decltype(nv)::value>), dim3(blocks), dim3(SUM_TPB), 0, s, static_cast<const T *>(logits), ld, r.tokens,
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
            // (as many turns each: 65536 rows of 100 in 1366 workgroups of three)
            const int64_t turns = (r.tokens * G + TPB - 1) / TPB, each = (turns + AT_ONCE - 1) / AT_ONCE;
            const dim3 grid((uint32_t)((turns + each - 1) / each));
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
