// Declarations shared by the translation units of ocean_experts.h.
#pragma once

#include "ocean_experts.h"
#include "routed.hpp"

namespace ocean {

constexpr int MX4_BLOCK = 32;   // numbers that share a scale
inline int64_t mx4_blocks(int64_t inner) { return (inner + MX4_BLOCK - 1) / MX4_BLOCK; }

#if defined(__HIPCC__)
// `bytes` of memory from `base` on, for accesses by 32-bit offsets: what lies behind them reads as 0 and is not written (the hardware's range check), so does an
// offset of NOWHERE.  Ends of rows and lines take no branch that way.  (With a choice of addresses for loads to LDS, the compiler made a branch of it and, where a
// workgroup's first step was the end of the lines, used a piece's offset from a register that it had written in the other lanes only.)
typedef __amdgpu_buffer_rsrc_t Memory;
constexpr uint32_t MEMORY_BYTES = 0xfffff000u, NOWHERE = 0xfffffff0u;
__device__ __forceinline__ Memory memory_at(const void *base, uint32_t bytes = MEMORY_BYTES)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, bytes, 0x00027000);
}
#endif

// balance.hip
size_t balance_workspace(int64_t tokens, int64_t experts);
hipError_t launch_balance(const ocean_routing &r, const void *logits, int dtype, int64_t ld, const ocean_balance &out, void *workspace, hipStream_t s);
hipError_t launch_balance_backward(const ocean_balance &b, const ocean_routing &r, const void *logits, int dtype, int64_t ld, const float *dloss,
                                   const float *dval, bool normalize, void *dlogits, int64_t ldd, hipStream_t s);

// mx4.hip
hipError_t launch_mx4_quantize(const void *x, int dtype, int64_t ldx, int64_t stride, const ocean_mx4 &q, hipStream_t s);
hipError_t launch_mx4_dequantize(const ocean_mx4 &q, int dtype, void *out, int64_t ldo, int64_t stride, hipStream_t s);

// mx4_grouped.hip, mx4_both.hip
hipError_t launch_grouped_mx4(const ocean_groups &g, int dtype, const void *x, int64_t ldx, const ocean_mx4 &w, bool transposed, void *y, int64_t ldy,
                              hipStream_t s);
hipError_t launch_grouped_mx4_mx4(const ocean_groups &g, const ocean_mx4 &x, const ocean_mx4 &w, int dtype, void *y, int64_t ldy, hipStream_t s);

}  // namespace ocean
