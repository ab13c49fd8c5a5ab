// Shared by the kernels of a worker's own step (mlmc_norm.hip, mlmc_rms.hip, mlmc_linear.hip, mlmc_dropout.hip, mlmc_distill.hip, mlmc_logprobs.hip): entries of 32 or 16 bits
// as floats, reductions over a wave and over a workgroup in a fixed order.
#pragma once
#include "mlmc_internal.h"

namespace mlmc {

template <int DT> struct EntryOf { using type = float; };
template <> struct EntryOf<MLMC_BF16> { using type = __bf16; };
constexpr int DT_E4M3 = 2;   // matrices in 8 bits, whose entries are only looked at by the matrix instructions
template <> struct EntryOf<DT_E4M3> { using type = uint8_t; };
template <int DT> using entry_t = typename EntryOf<DT>::type;
template <int DT> constexpr int ENTRIES = 16 / sizeof(entry_t<DT>);   // of 16 bytes

__device__ inline float to_f32(float v) { return v; }
__device__ inline float to_f32(__bf16 v) { return (float)v; }
template <int DT> __device__ inline entry_t<DT> from_f32(float v) { return (entry_t<DT>)v; }   // 16 bits: to nearest, ties to even

using v4f = float __attribute__((ext_vector_type(4)));
using v8b = __bf16 __attribute__((ext_vector_type(8)));
using chunk_t = int __attribute__((ext_vector_type(4)));                 // 16 bytes of a row
using chunk_u = int __attribute__((ext_vector_type(4), aligned(2)));     // the same at any entry's place
using chunk_b = int __attribute__((ext_vector_type(4), aligned(1)));     // and of 8 bits

// 16 bytes of row `r`, columns c .. c + 16 / size - 1, of a matrix of R rows and C columns; zero outside, once cut_chunk has been over them.  A chunk
// that the row's end cuts is taken from the row's last 16 bytes and shifted down later: no branch and no wait between the loads.  WIDE: rows
// have 16 bytes.
template <int DT, bool WIDE> __device__ inline chunk_t raw_chunk(const void* p, int64_t ld, int64_t r, int64_t R, int64_t c, int64_t C) {
    constexpr int E = ENTRIES<DT>, BITS = 128 / E;
    const entry_t<DT>* q = (const entry_t<DT>*)p + (r < R ? r : R - 1) * ld;
    if (WIDE || C >= E) {
        q += c < C - E ? c : C - E;
        if constexpr (DT == DT_E4M3) return *(const chunk_b*)q;
        else return *(const chunk_u*)q;
    }
    unsigned __int128 v = 0;
#pragma unroll 1
    for (int e = 0; e < C; ++e) v |= (unsigned __int128)(DT == DT_E4M3 ? ((const uint8_t*)q)[e] : DT == MLMC_BF16 ? ((const uint16_t*)q)[e] : ((const uint32_t*)q)[e]) << (BITS * e);
    return __builtin_bit_cast(chunk_t, v);
}
template <int DT, bool WIDE> __device__ inline chunk_t cut_chunk(chunk_t w, int64_t r, int64_t R, int64_t c, int64_t C) {
    constexpr int E = ENTRIES<DT>, BITS = 128 / E;
    const int64_t first = WIDE || C >= E ? C - E : 0, over = c < first ? 0 : c - first;
    const unsigned __int128 v = __builtin_bit_cast(unsigned __int128, w);
    return __builtin_bit_cast(chunk_t, over >= E || r >= R ? (unsigned __int128)0 : v >> (BITS * (int)over));
}

template <int CTRL, int ROWS> __device__ inline float dpp(float v, float outside) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, outside), __builtin_bit_cast(int, v), CTRL, ROWS, 0xF, false));
}
// Sum over a wave, the same in every lane: prefixes within 16 lanes, then across the four sixteens, all lane to lane (a shuffle through LDS takes ten times as long).
__device__ inline float wave_sum(float v) {
    v += dpp<0x111, 0xF>(v, 0.f);   // from 1, 2, 4 and 8 lanes below
    v += dpp<0x112, 0xF>(v, 0.f);
    v += dpp<0x114, 0xF>(v, 0.f);
    v += dpp<0x118, 0xF>(v, 0.f);
    v += dpp<0x142, 0xA>(v, 0.f);   // lane 15 of the sixteen below, into sixteens 1 and 3
    v += dpp<0x143, 0xC>(v, 0.f);   // lane 31, into sixteens 2 and 3
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
// the greatest operand that is a number
__device__ inline float wave_max(float v) {
    v = fmaxf(v, dpp<0x111, 0xF>(v, v));
    v = fmaxf(v, dpp<0x112, 0xF>(v, v));
    v = fmaxf(v, dpp<0x114, 0xF>(v, v));
    v = fmaxf(v, dpp<0x118, 0xF>(v, v));
    v = fmaxf(v, dpp<0x142, 0xA>(v, v));
    v = fmaxf(v, dpp<0x143, 0xC>(v, v));
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
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

// A thread's chunk of 16 bytes of a row as floats; -Inf past the end.
template <int DT> __device__ inline void chunk_floats(float (&f)[DT == MLMC_BF16 ? 8 : 4], chunk_t v) {
    if constexpr (DT == MLMC_BF16) {
        const v8b u = __builtin_bit_cast(v8b, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (float)u[e];
    } else {
        const v4f u = __builtin_bit_cast(v4f, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = u[e];
    }
}
template <int DT> __device__ inline chunk_t load_chunk(const entry_t<DT>* s, int64_t col, int64_t end) {
    constexpr int E = DT == MLMC_BF16 ? 8 : 4;
    if (col + E <= end) return *(const chunk_u*)(s + col);
    entry_t<DT> __attribute__((ext_vector_type(E))) u;
#pragma unroll
    for (int e = 0; e < E; ++e) u[e] = col + e < end ? s[col + e] : (entry_t<DT>)-INFINITY;
    return __builtin_bit_cast(chunk_t, u);
}
template <int DT> __device__ inline void store_chunk(entry_t<DT>* s, int64_t col, int64_t end, const float (&f)[DT == MLMC_BF16 ? 8 : 4]) {
    constexpr int E = DT == MLMC_BF16 ? 8 : 4;
    if (col + E <= end) {
        entry_t<DT> __attribute__((ext_vector_type(E))) u;
#pragma unroll
        for (int e = 0; e < E; ++e) u[e] = (entry_t<DT>)f[e];
        *(chunk_u*)(s + col) = __builtin_bit_cast(chunk_t, u);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (col + e < end) s[col + e] = (entry_t<DT>)f[e];
    }
}

// exp(x / T) with unit = log2(e) / T, x a difference of logits: scaled before it is taken, large logits would lose it
__device__ inline float power(float x, float unit) { return __builtin_amdgcn_exp2f(x * unit); }

// A launch has less than 2^32 threads along an axis: of more, some workgroups never run, and no error is reported.  Kernels that may need more are launched in slices.
constexpr int64_t LAUNCH_THREADS = (int64_t)1 << 31;

inline bool entry_dtype_ok(int dtype) { return dtype == MLMC_F32 || dtype == MLMC_BF16; }
// pointers of entries have to be aligned to an entry, no more
inline bool entry_ptr_ok(const void* p, int dtype) { return p && (uintptr_t)p % (dtype == MLMC_BF16 ? 2 : 4) == 0; }
inline bool f32_ptr_ok(const void* p) { return (uintptr_t)p % 4 == 0; }

}  // namespace mlmc
