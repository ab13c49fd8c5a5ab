// Matrix product with bias, activation and residual in its epilogue, and its two gradients (entry points mlmc_linear,
// mlmc_linear_dgrad, mlmc_linear_wgrad).
//
//   forward:  z = x W^T + b, y = act(z) + r         x [n][k], W [m][k]; contraction over k
//   dgrad:    dx = (dy W) act'(z) + r               dy [n][m];          contraction over m
//   wgrad:    dW = dy^T x, db = sum over rows of dy;                    contraction over n
#include "mlmc_worker.h"

namespace mlmc {

// C[i][j] = sum_c A(i, c) B(j, c), A(i, c) at a[i * a_i + c * a_c], likewise B.
struct LinearArgs {
    const void *a, *b;
    int64_t a_i, a_c, b_j, b_c, I, J, C;
    int act;
    const float* bias;     // forward: of column j
    const void* slope_z;   // dgrad: C is multiplied with act' of this
    int64_t ld_slope;
    const void* residual;
    int64_t ldr;
    void* z;               // forward: receives C + bias
    int64_t ldz;
    void* out;
    int64_t ldo;
    int out_dtype;
    void* row_sum;         // wgrad: sum_c A(i, c), in out_dtype
};

__device__ inline float act_value(float z, int act) {
    if (act == MLMC_ACT_RELU) return z > 0.f || z != z ? z : 0.f;   // a NaN stays one
    if (act == MLMC_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    return z;
}
__device__ inline float act_slope(float z, int act) {
    if (act == MLMC_ACT_RELU) return z > 0.f ? 1.f : 0.f;
    if (act == MLMC_ACT_GELU) return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * 0.39894228040143268f * expf(-0.5f * z * z);
    return 1.f;
}
__device__ inline void store_as(void* p, int64_t at, int dtype, float v) {
    if (dtype == MLMC_F32) ((float*)p)[at] = v;
    else ((__bf16*)p)[at] = (__bf16)v;
}

constexpr int LIN_T = 64, LIN_C = 16;

template <int DT> __global__ __launch_bounds__(256) void k_linear(LinearArgs g) {
    __shared__ float sa[LIN_C][LIN_T + 1], sb[LIN_C][LIN_T + 1];
    const int64_t i0 = (int64_t)blockIdx.y * LIN_T, j0 = (int64_t)blockIdx.x * LIN_T;
    const int ti = (threadIdx.x >> 4) * 4, tj = (threadIdx.x & 15) * 4;
    float acc[4][4] = {};
    float sums = 0.f;
    for (int64_t c0 = 0; c0 < g.C; c0 += LIN_C) {
        for (int e = threadIdx.x; e < LIN_T * LIN_C; e += 256) {
            // neighbouring threads along whichever index is contiguous
            const int ic = g.a_c == 1 ? e % LIN_C : e / LIN_T, ii = g.a_c == 1 ? e / LIN_C : e % LIN_T;
            const int jc = g.b_c == 1 ? e % LIN_C : e / LIN_T, jj = g.b_c == 1 ? e / LIN_C : e % LIN_T;
            sa[ic][ii] = i0 + ii < g.I && c0 + ic < g.C ? to_f32(((const entry_t<DT>*)g.a)[(i0 + ii) * g.a_i + (c0 + ic) * g.a_c]) : 0.f;
            sb[jc][jj] = j0 + jj < g.J && c0 + jc < g.C ? to_f32(((const entry_t<DT>*)g.b)[(j0 + jj) * g.b_j + (c0 + jc) * g.b_c]) : 0.f;
        }
        __syncthreads();
        for (int c = 0; c < LIN_C; ++c)
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[u][v] = fmaf(sa[c][ti + u], sb[c][tj + v], acc[u][v]);
        if (g.row_sum && blockIdx.x == 0 && threadIdx.x < LIN_T)
            for (int c = 0; c < LIN_C; ++c) sums += sa[c][threadIdx.x];
        __syncthreads();
    }
    for (int u = 0; u < 4; ++u)
        for (int v = 0; v < 4; ++v) {
            const int64_t i = i0 + ti + u, j = j0 + tj + v;
            if (i >= g.I || j >= g.J) continue;
            float z = acc[u][v];
            if (g.bias) z += g.bias[j];
            if (g.z) store_as(g.z, i * g.ldz + j, DT, z);
            z = g.slope_z ? z * act_slope(to_f32(((const entry_t<DT>*)g.slope_z)[i * g.ld_slope + j]), g.act) : act_value(z, g.act);
            if (g.residual) z += to_f32(((const entry_t<DT>*)g.residual)[i * g.ldr + j]);
            store_as(g.out, i * g.ldo + j, g.out_dtype, z);
        }
    if (g.row_sum && blockIdx.x == 0 && threadIdx.x < LIN_T && i0 + threadIdx.x < g.I) store_as(g.row_sum, i0 + threadIdx.x, g.out_dtype, sums);
}

static mlmc_status linear_run(const LinearArgs& g, int dtype, hipStream_t st) {
    const dim3 grid((unsigned)((g.J + LIN_T - 1) / LIN_T), (unsigned)((g.I + LIN_T - 1) / LIN_T));
    if (dtype == MLMC_F32) MLMC_LAUNCH(K_LINEAR, st, (k_linear<MLMC_F32><<<grid, 256, 0, st>>>(g)));
    else MLMC_LAUNCH(K_LINEAR, st, (k_linear<MLMC_BF16><<<grid, 256, 0, st>>>(g)));
    return MLMC_OK;
}

constexpr int64_t LINEAR_ROWS_MAX = (int64_t)1 << 21;   // workgroups of 64 rows along the grid's second axis: under 2^16
static bool linear_sizes_ok(int64_t n, int64_t m, int64_t k) {
    return n >= 0 && n <= LINEAR_ROWS_MAX && m >= 1 && m <= LINEAR_ROWS_MAX && k >= 1 && k <= LINEAR_ROWS_MAX;
}
static bool act_ok(int act) { return act == MLMC_ACT_NONE || act == MLMC_ACT_RELU || act == MLMC_ACT_GELU; }

}  // namespace mlmc

using namespace mlmc;

extern "C" {

size_t mlmc_linear_workspace(int64_t rows, int64_t outputs, int64_t inputs) {
    (void)rows; (void)outputs; (void)inputs;
    return 0;
}

mlmc_status mlmc_linear(const void* x, int64_t ldx, const void* weight, int64_t ldw, int64_t rows, int64_t outputs, int64_t inputs, int dtype,
                        const float* bias, int act, const void* residual, int64_t ldr, void* z, int64_t ldz, void* y, int64_t ldy,
                        void* ws, size_t ws_bytes, void* hip_stream) {
    if (!linear_sizes_ok(rows, outputs, inputs) || !entry_dtype_ok(dtype) || !act_ok(act) || ldx < inputs || ldw < inputs || ldy < outputs) return MLMC_EINVAL;
    if ((residual && ldr < outputs) || (z && ldz < outputs)) return MLMC_EINVAL;
    if (rows == 0) return MLMC_OK;
    if (!entry_ptr_ok(x, dtype) || !entry_ptr_ok(weight, dtype) || !entry_ptr_ok(y, dtype) || !f32_ptr_ok(bias)) return MLMC_EINVAL;
    if ((residual && !entry_ptr_ok(residual, dtype)) || (z && !entry_ptr_ok(z, dtype))) return MLMC_EINVAL;
    const size_t need = mlmc_linear_workspace(rows, outputs, inputs);
    if (need && (!ws || (uintptr_t)ws % 256 || ws_bytes < need)) return MLMC_EINVAL;
    LinearArgs g = {};
    g.a = x; g.a_i = ldx; g.a_c = 1; g.b = weight; g.b_j = ldw; g.b_c = 1; g.I = rows; g.J = outputs; g.C = inputs;
    g.act = act; g.bias = bias; g.residual = residual; g.ldr = ldr; g.z = z; g.ldz = ldz; g.out = y; g.ldo = ldy; g.out_dtype = dtype;
    return linear_run(g, dtype, (hipStream_t)hip_stream);
}

mlmc_status mlmc_linear_dgrad(const void* dy, int64_t lddy, const void* weight, int64_t ldw, int64_t rows, int64_t outputs, int64_t inputs,
                              int dtype, int act, const void* z, int64_t ldz, const void* residual, int64_t ldr, void* dx, int64_t lddx,
                              void* ws, size_t ws_bytes, void* hip_stream) {
    if (!linear_sizes_ok(rows, outputs, inputs) || !entry_dtype_ok(dtype) || !act_ok(act) || lddy < outputs || ldw < inputs || lddx < inputs) return MLMC_EINVAL;
    if ((residual && ldr < inputs) || (act != MLMC_ACT_NONE && ldz < inputs)) return MLMC_EINVAL;
    if (rows == 0) return MLMC_OK;
    if (!entry_ptr_ok(dy, dtype) || !entry_ptr_ok(weight, dtype) || !entry_ptr_ok(dx, dtype)) return MLMC_EINVAL;
    if ((residual && !entry_ptr_ok(residual, dtype)) || (act != MLMC_ACT_NONE && !entry_ptr_ok(z, dtype))) return MLMC_EINVAL;
    const size_t need = mlmc_linear_workspace(rows, outputs, inputs);
    if (need && (!ws || (uintptr_t)ws % 256 || ws_bytes < need)) return MLMC_EINVAL;
    LinearArgs g = {};
    g.a = dy; g.a_i = lddy; g.a_c = 1; g.b = weight; g.b_j = 1; g.b_c = ldw; g.I = rows; g.J = inputs; g.C = outputs;
    g.act = act; g.slope_z = act != MLMC_ACT_NONE ? z : nullptr; g.ld_slope = ldz; g.residual = residual; g.ldr = ldr;
    g.out = dx; g.ldo = lddx; g.out_dtype = dtype;
    return linear_run(g, dtype, (hipStream_t)hip_stream);
}

mlmc_status mlmc_linear_wgrad(const void* dy, int64_t lddy, const void* x, int64_t ldx, int64_t rows, int64_t outputs, int64_t inputs, int dtype,
                              void* dweight, int64_t lddw, void* dbias, int grad_dtype, void* ws, size_t ws_bytes, void* hip_stream) {
    if (!linear_sizes_ok(rows, outputs, inputs) || !entry_dtype_ok(dtype) || !entry_dtype_ok(grad_dtype) || lddy < outputs || ldx < inputs || lddw < inputs) return MLMC_EINVAL;
    if (!entry_ptr_ok(dweight, grad_dtype) || (dbias && !entry_ptr_ok(dbias, grad_dtype))) return MLMC_EINVAL;
    if (rows > 0 && (!entry_ptr_ok(dy, dtype) || !entry_ptr_ok(x, dtype))) return MLMC_EINVAL;
    const size_t need = mlmc_linear_workspace(rows, outputs, inputs);
    if (need && (!ws || (uintptr_t)ws % 256 || ws_bytes < need)) return MLMC_EINVAL;
    LinearArgs g = {};
    g.a = dy; g.a_i = 1; g.a_c = lddy; g.b = x; g.b_j = 1; g.b_c = ldx; g.I = outputs; g.J = inputs; g.C = rows;
    g.act = MLMC_ACT_NONE; g.out = dweight; g.ldo = lddw; g.out_dtype = grad_dtype; g.row_sum = dbias;
    return linear_run(g, dtype, (hipStream_t)hip_stream);
}

}  // extern "C"
