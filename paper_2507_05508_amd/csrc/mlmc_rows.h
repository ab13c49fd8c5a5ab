// Rows of a matrix in the registers of the threads that work on them, and the sums over rows that a weight's gradient is: shared by layer norm (mlmc_norm.hip), root-mean-square norm and
// rounding to 8 bits (mlmc_rms.hip).
#pragma once
#include "mlmc_worker.h"

namespace mlmc {

// ---- rows that fit in the registers of T threads, P entries each ------------------------------------------------------

// A thread's N chunks of 16 bytes of a row, T threads side by side; zeros from column d >= 8 on.  A row's base is uniform over a wave, so that an address is one
// register.  A chunk that the row's end cuts is the row's last 16 bytes, shifted down.
template <int DT, int T, int P> struct RowChunks {
    static constexpr int E = DT == MLMC_BF16 ? 8 : 4, N = P / E, BYTES = 16 / E;
    int d, col0;
    __device__ RowChunks(int64_t d_, int t) : d((int)d_), col0(t * E) {}
    __device__ int col(int n) const { return col0 + n * T * E; }
    __device__ void load(chunk_t (&v)[N], const void* row) const {
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = *(const chunk_u*)((const char*)row + (unsigned)(min(col(n), d - E) * BYTES));
    }
    __device__ void to_floats(float (&f)[P], const chunk_t (&v)[N]) const {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            chunk_t c = v[n];
            const int over = col(n) - (d - E);
            if (over > 0) c = over >= E ? chunk_t{0, 0, 0, 0} : __builtin_bit_cast(chunk_t, __builtin_bit_cast(unsigned __int128, c) >> (over * BYTES * 8));
            if constexpr (DT == MLMC_BF16) {
                const v8b u = __builtin_bit_cast(v8b, c);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[n * E + e] = (float)u[e];
            } else {
                const v4f u = __builtin_bit_cast(v4f, c);
#pragma unroll
                for (int e = 0; e < 4; ++e) f[n * E + e] = u[e];
            }
        }
    }
    __device__ void store(void* row, const float (&f)[P]) const {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            char* q = (char*)row + (unsigned)(col(n) * BYTES);
            if (col(n) + E <= d) {
                entry_t<DT> __attribute__((ext_vector_type(E))) u;
#pragma unroll
                for (int e = 0; e < E; ++e) u[e] = (entry_t<DT>)f[n * E + e];
                *(chunk_u*)q = __builtin_bit_cast(chunk_t, u);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (col(n) + e < d) ((entry_t<DT>*)q)[e] = (entry_t<DT>)f[n * E + e];
            }
        }
    }
    // zero from column d on
    __device__ void cut(float (&f)[P]) const {
#pragma unroll
        for (int n = 0; n < N; ++n)
            if (col(n) + E > d) {
#pragma unroll
                for (int e = 0; e < E; ++e) f[n * E + e] = col(n) + e < d ? f[n * E + e] : 0.f;
            }
    }
    // column of entry e of the thread
    __device__ int at(int e) const { return col(e / E) + e % E; }
};

// Sums of two values over the T threads of a row; `part`: LDS that no earlier round may still be reading.
template <int T> __device__ inline void row_sums(float& a, float& b, float2* part) {
    a = wave_sum(a);
    b = wave_sum(b);
    if (T == 64) return;
    const int first = threadIdx.x / T * (T / 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = make_float2(a, b);
    __syncthreads();
    a = b = 0.f;
#pragma unroll 4
    for (int w = 0; w < T / 64; ++w) {
        const float2 v = part[first + w];
        a += v.x;
        b += v.y;
    }
}

// 1 / sqrt v: the instruction where it is exact to an ulp, which leaves out subnormal numbers
__device__ inline float inverse_root(float v) { return v >= 1.2e-38f ? __builtin_amdgcn_rsqf(v) : 1.0f / sqrtf(v); }

// s / d by the reciprocal of d and what that leaves over, which is exact: a row of equal entries has them as its mean at every width.  (A division took 0.3 us of 19; an infinite sum leaves NaN.)
__device__ inline float quotient(float s, float d, float inv_d) {
    const float q = s * inv_d, left = fmaf(-q, d, s);
    return left == left ? fmaf(left, inv_d, q) : q;
}

// The groups' partial sums of `vectors` (1 or 2) columns' vectors, [groups][vectors][d]: a lane has a column, the 16 waves take the groups in turn and their sums are added in the waves' order.
struct JoinArgs {
    const float* part;
    int64_t groups, d;
    int64_t col0;         // first column of a launch
    int vectors;
    void* out[2];         // or NULL
    int grad_dtype;
};
constexpr int JOIN_WAVES = 16;
static __global__ __launch_bounds__(JOIN_WAVES * 64) void k_norm_join(JoinArgs a) {
    __shared__ float sum[JOIN_WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, which = blockIdx.y;
    void* out = a.out[which];
    if (!out) return;
    const int64_t j = a.col0 + (int64_t)blockIdx.x * 64 + lane;
    float v = 0.f;
    if (j < a.d) {
#pragma unroll 8
        for (int64_t g = wave; g < a.groups; g += JOIN_WAVES) v += a.part[(a.vectors * g + which) * a.d + j];
    }
    sum[wave][lane] = v;
    __syncthreads();
    if (wave || j >= a.d) return;
    v = 0.f;
#pragma unroll
    for (int w = 0; w < JOIN_WAVES; ++w) v += sum[w][lane];
    if (a.grad_dtype == MLMC_F32) ((float*)out)[j] = v;
    else ((__bf16*)out)[j] = (__bf16)v;
}
static mlmc_status join_columns(JoinArgs a, hipStream_t st) {
    constexpr int64_t slice = LAUNCH_THREADS / JOIN_WAVES;   // columns of a launch: 64 a workgroup, each by a thread of every wave
    for (; a.col0 < a.d; a.col0 += slice) {
        const int64_t cols = a.d - a.col0 < slice ? a.d - a.col0 : slice;
        MLMC_LAUNCH(K_NORM_JOIN, st, (k_norm_join<<<dim3((unsigned)((cols + 63) / 64), (unsigned)a.vectors), JOIN_WAVES * 64, 0, st>>>(a)));
    }
    return MLMC_OK;
}

constexpr int64_t NORM_ROW_MIN = 8, NORM_ROW_MAX = 16384;   // widths of the rows that are kept in registers
static int row_threads(int64_t d) { return d <= 512 ? 64 : d <= 1024 ? 128 : d <= 2048 ? 256 : d <= 4096 ? 512 : 1024; }   // 8 entries each, 16 from 8192 on

// Workgroups of the backward pass, of 1024 threads, each of which leaves a partial sum of every column: one for every CU (its registers are full then), fewer if there are not the rows.
static int64_t norm_groups(int64_t rows, int64_t d) {
    if (d < NORM_ROW_MIN || d > NORM_ROW_MAX) return rows < 64 ? rows : 64;
    const int64_t at_once = 1024 / row_threads(d), groups = (rows + at_once - 1) / at_once;
    return groups < 256 ? groups : 256;
}

static bool norm_sizes_ok(int64_t rows, int64_t d) { return rows >= 0 && rows < ((int64_t)1 << 31) && d >= 1 && d < ((int64_t)1 << 31); }

}  // namespace mlmc
