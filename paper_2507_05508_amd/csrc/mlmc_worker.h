// Shared by the kernels of a worker's own step (mlmc_norm.hip, mlmc_linear.hip, mlmc_distill.hip): entries of 32 or 16 bits
// as floats, reductions over a wave and over a workgroup in a fixed order.
#pragma once
#include "mlmc_internal.h"

namespace mlmc {

template <int DT> struct EntryOf { using type = float; };
template <> struct EntryOf<MLMC_BF16> { using type = __bf16; };
template <int DT> using entry_t = typename EntryOf<DT>::type;

__device__ inline float to_f32(float v) { return v; }
__device__ inline float to_f32(__bf16 v) { return (float)v; }
template <int DT> __device__ inline entry_t<DT> from_f32(float v) { return (entry_t<DT>)v; }   // 16 bits: to nearest, ties to even

__device__ inline float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
// the greatest operand that is a number
__device__ inline float wave_max(float v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

// Sum over a workgroup of WAVES waves; every thread gets it, the waves' sums added in wave order.  `part`: LDS, WAVES floats,
// free for reuse after the next barrier.
template <int WAVES> __device__ inline float group_sum(float v, float* part) {
    v = wave_sum(v);
    if (WAVES == 1) return v;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = part[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s += part[w];
    return s;
}
template <int WAVES> __device__ inline float group_max(float v, float* part) {
    v = wave_max(v);
    if (WAVES == 1) return v;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = part[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s = fmaxf(s, part[w]);
    return s;
}

inline bool entry_dtype_ok(int dtype) { return dtype == MLMC_F32 || dtype == MLMC_BF16; }
// pointers of entries have to be aligned to an entry, no more
inline bool entry_ptr_ok(const void* p, int dtype) { return p && (uintptr_t)p % (dtype == MLMC_BF16 ? 2 : 4) == 0; }
inline bool f32_ptr_ok(const void* p) { return (uintptr_t)p % 4 == 0; }

}  // namespace mlmc
