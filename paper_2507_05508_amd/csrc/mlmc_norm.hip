// Layer norm of the rows of a matrix, forward and backward (entry points mlmc_layer_norm, mlmc_layer_norm_backward).
//
//   mu = mean_j x_j,  v = mean_j (x_j - mu)^2,  r = 1 / sqrt(v + eps),  h_j = (x_j - mu) r,  y_j = h_j w_j + b_j
//   backward, with c_j = dy_j w_j:  dx_j = r (c_j - mean c - h_j mean(c h)),  dw_j = sum_rows dy_j h_j,  db_j = sum_rows dy_j
//
// The variance is the mean square of the differences from the mean, not E x^2 - mu^2, which loses the variance of rows that lie far
// from zero.  All sums are fp32, in an order that depends on the sizes alone: no atomics.
#include "mlmc_worker.h"

namespace mlmc {

constexpr int NORM_WG = 256;

struct NormArgs {
    const void *x, *dy;
    int64_t ldx, lddy, rows, d;
    const float *weight, *bias, *stats_in;
    float eps;
    void *y, *dx;
    int64_t ldy, lddx;
    float* stats;
    float* part;          // [groups][2][d] sums of a group's rows
    int64_t groups;       // workgroups, each takes rows group, group + groups, ...
    void *dweight, *dbias;
    int grad_dtype;
};

// One workgroup per row, which it reads three times; the second and third read come from the caches.
template <int DT> __global__ __launch_bounds__(NORM_WG) void k_norm_forward(NormArgs a) {
    __shared__ float part[2][NORM_WG / 64];
    const entry_t<DT>* x = (const entry_t<DT>*)a.x + (int64_t)blockIdx.x * a.ldx;
    entry_t<DT>* y = (entry_t<DT>*)a.y + (int64_t)blockIdx.x * a.ldy;
    float s = 0.f;
    for (int64_t j = threadIdx.x; j < a.d; j += NORM_WG) s += to_f32(x[j]);
    const float mean = group_sum<NORM_WG / 64>(s, part[0]) / (float)a.d;
    s = 0.f;
    for (int64_t j = threadIdx.x; j < a.d; j += NORM_WG) {
        const float u = to_f32(x[j]) - mean;
        s = fmaf(u, u, s);
    }
    const float rstd = 1.0f / sqrtf(group_sum<NORM_WG / 64>(s, part[1]) / (float)a.d + a.eps);
    for (int64_t j = threadIdx.x; j < a.d; j += NORM_WG) {
        const float h = (to_f32(x[j]) - mean) * rstd;
        y[j] = from_f32<DT>(fmaf(h, a.weight ? a.weight[j] : 1.0f, a.bias ? a.bias[j] : 0.0f));
    }
    if (a.stats && threadIdx.x == 0) {
        a.stats[2 * (int64_t)blockIdx.x] = mean;
        a.stats[2 * (int64_t)blockIdx.x + 1] = rstd;
    }
}

template <int DT> __global__ __launch_bounds__(NORM_WG) void k_norm_backward(NormArgs a) {
    __shared__ float part[2][NORM_WG / 64];
    const entry_t<DT>* x = (const entry_t<DT>*)a.x + (int64_t)blockIdx.x * a.ldx;
    const entry_t<DT>* dy = (const entry_t<DT>*)a.dy + (int64_t)blockIdx.x * a.lddy;
    entry_t<DT>* dx = (entry_t<DT>*)a.dx + (int64_t)blockIdx.x * a.lddx;
    const float mean = a.stats_in[2 * (int64_t)blockIdx.x], rstd = a.stats_in[2 * (int64_t)blockIdx.x + 1];
    float s = 0.f, t = 0.f;
    for (int64_t j = threadIdx.x; j < a.d; j += NORM_WG) {
        const float c = to_f32(dy[j]) * (a.weight ? a.weight[j] : 1.0f);
        s += c;
        t = fmaf(c, (to_f32(x[j]) - mean) * rstd, t);
    }
    const float cm = group_sum<NORM_WG / 64>(s, part[0]) / (float)a.d;
    const float ch = group_sum<NORM_WG / 64>(t, part[1]) / (float)a.d;
    for (int64_t j = threadIdx.x; j < a.d; j += NORM_WG) {
        const float c = to_f32(dy[j]) * (a.weight ? a.weight[j] : 1.0f);
        const float h = (to_f32(x[j]) - mean) * rstd;
        dx[j] = from_f32<DT>(rstd * (c - cm - h * ch));
    }
}

// A thread sums its column over the rows of the group.  Before k_norm_backward, whose dx may be dy or x themselves.
template <int DT> __global__ __launch_bounds__(NORM_WG) void k_norm_columns(NormArgs a) {
    const int64_t j = (int64_t)blockIdx.x * NORM_WG + threadIdx.x;
    if (j >= a.d) return;
    float dw = 0.f, db = 0.f;
    for (int64_t i = blockIdx.y; i < a.rows; i += a.groups) {
        const float g = to_f32(((const entry_t<DT>*)a.dy)[i * a.lddy + j]);
        const float h = (to_f32(((const entry_t<DT>*)a.x)[i * a.ldx + j]) - a.stats_in[2 * i]) * a.stats_in[2 * i + 1];
        dw = fmaf(g, h, dw);
        db += g;
    }
    a.part[(2 * (int64_t)blockIdx.y) * a.d + j] = dw;
    a.part[(2 * (int64_t)blockIdx.y + 1) * a.d + j] = db;
}

// The groups' sums of a column, in the order of the groups.
__global__ __launch_bounds__(NORM_WG) void k_norm_join(NormArgs a) {
    const int64_t j = (int64_t)blockIdx.x * NORM_WG + threadIdx.x;
    if (j >= a.d) return;
    float dw = 0.f, db = 0.f;
    for (int64_t g = 0; g < a.groups; ++g) {
        dw += a.part[(2 * g) * a.d + j];
        db += a.part[(2 * g + 1) * a.d + j];
    }
    if (a.grad_dtype == MLMC_F32) {
        if (a.dweight) ((float*)a.dweight)[j] = dw;
        if (a.dbias) ((float*)a.dbias)[j] = db;
    } else {
        if (a.dweight) ((__bf16*)a.dweight)[j] = (__bf16)dw;
        if (a.dbias) ((__bf16*)a.dbias)[j] = (__bf16)db;
    }
}

static int64_t norm_groups(int64_t rows, int64_t d) {
    (void)d;
    return rows < 64 ? rows : 64;
}

static bool norm_sizes_ok(int64_t rows, int64_t d) { return rows >= 0 && rows < ((int64_t)1 << 31) && d >= 1 && d < ((int64_t)1 << 31); }

}  // namespace mlmc

using namespace mlmc;

extern "C" {

size_t mlmc_layer_norm_workspace(int64_t rows, int64_t d) {
    return norm_sizes_ok(rows, d) ? (size_t)norm_groups(rows, d) * 2 * (size_t)d * sizeof(float) : 0;
}

mlmc_status mlmc_layer_norm(const void* x, int64_t ldx, int64_t rows, int64_t d, int dtype, const float* weight, const float* bias,
                            float eps, void* y, int64_t ldy, float* stats, void* hip_stream) {
    if (!norm_sizes_ok(rows, d) || !entry_dtype_ok(dtype) || ldx < d || ldy < d || !(eps >= 0.0f) || eps > 3.402823e38f) return MLMC_EINVAL;
    if (rows == 0) return MLMC_OK;
    if (!entry_ptr_ok(x, dtype) || !entry_ptr_ok(y, dtype) || !f32_ptr_ok(weight) || !f32_ptr_ok(bias) || !f32_ptr_ok(stats)) return MLMC_EINVAL;
    hipStream_t st = (hipStream_t)hip_stream;
    NormArgs a = {};
    a.x = x; a.ldx = ldx; a.rows = rows; a.d = d; a.weight = weight; a.bias = bias; a.eps = eps; a.y = y; a.ldy = ldy; a.stats = stats;
    if (dtype == MLMC_F32) MLMC_LAUNCH(K_NORM_FORWARD, st, (k_norm_forward<MLMC_F32><<<(unsigned)rows, NORM_WG, 0, st>>>(a)));
    else MLMC_LAUNCH(K_NORM_FORWARD, st, (k_norm_forward<MLMC_BF16><<<(unsigned)rows, NORM_WG, 0, st>>>(a)));
    return MLMC_OK;
}

mlmc_status mlmc_layer_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, int64_t rows, int64_t d, int dtype,
                                     const float* weight, const float* stats, void* dx, int64_t lddx, void* dweight, void* dbias,
                                     int grad_dtype, void* ws, size_t ws_bytes, void* hip_stream) {
    if (!norm_sizes_ok(rows, d) || !entry_dtype_ok(dtype) || lddy < d || ldx < d || lddx < d) return MLMC_EINVAL;
    const bool sums = dweight || dbias;
    if (sums && (!entry_dtype_ok(grad_dtype) || (dweight && !entry_ptr_ok(dweight, grad_dtype)) || (dbias && !entry_ptr_ok(dbias, grad_dtype)))) return MLMC_EINVAL;
    if (rows > 0 && (!entry_ptr_ok(dy, dtype) || !entry_ptr_ok(x, dtype) || !entry_ptr_ok(dx, dtype) || !stats || !f32_ptr_ok(stats) || !f32_ptr_ok(weight))) return MLMC_EINVAL;
    if (sums && rows > 0 && (!ws || (uintptr_t)ws % 256 || ws_bytes < mlmc_layer_norm_workspace(rows, d))) return MLMC_EINVAL;
    hipStream_t st = (hipStream_t)hip_stream;
    NormArgs a = {};
    a.x = x; a.ldx = ldx; a.dy = dy; a.lddy = lddy; a.rows = rows; a.d = d; a.weight = weight; a.stats_in = stats; a.dx = dx; a.lddx = lddx;
    a.part = (float*)ws; a.groups = norm_groups(rows, d); a.dweight = dweight; a.dbias = dbias; a.grad_dtype = grad_dtype;
    const unsigned cols = (unsigned)((d + NORM_WG - 1) / NORM_WG);
    if (sums && rows > 0) {
        if (dtype == MLMC_F32) MLMC_LAUNCH(K_NORM_COLUMNS, st, (k_norm_columns<MLMC_F32><<<dim3(cols, (unsigned)a.groups), NORM_WG, 0, st>>>(a)));
        else MLMC_LAUNCH(K_NORM_COLUMNS, st, (k_norm_columns<MLMC_BF16><<<dim3(cols, (unsigned)a.groups), NORM_WG, 0, st>>>(a)));
    }
    if (rows > 0) {
        if (dtype == MLMC_F32) MLMC_LAUNCH(K_NORM_BACKWARD, st, (k_norm_backward<MLMC_F32><<<(unsigned)rows, NORM_WG, 0, st>>>(a)));
        else MLMC_LAUNCH(K_NORM_BACKWARD, st, (k_norm_backward<MLMC_BF16><<<(unsigned)rows, NORM_WG, 0, st>>>(a)));
    }
    if (sums) MLMC_LAUNCH(K_NORM_JOIN, st, (k_norm_join<<<cols, NORM_WG, 0, st>>>(a)));
    return MLMC_OK;
}

}  // extern "C"
