// Layer norm of the rows of a matrix, forward and backward (entry points mlmc_layer_norm, mlmc_layer_norm_backward).
//
//   mu = mean_j x_j,  v = mean_j (x_j - mu)^2,  r = 1 / sqrt(v + eps),  h_j = (x_j - mu) r,  y_j = h_j w_j + b_j
//   backward, with c_j = dy_j w_j:  dx_j = r (c_j - mean c - h_j mean(c h)),  dw_j = sum_rows dy_j h_j,  db_j = sum_rows dy_j
//
// The variance is the mean square of the differences from the mean, not E x^2 - mu^2, which loses the variance of rows that lie far
// from zero.  All sums are fp32, in an order that depends on the sizes alone: no atomics.
//
// Bound by memory: forward reads x and writes y, backward reads x and dy and writes dx, once each, where a row fits in the registers of its threads (8 to 16384 entries).
// Kernel times: forward 16384 x 1024 bf16 20 us (67 MB, 3.4 TB/s; the start of a launch and its last rows are a third of it), 8192 x 4096 33 us (4.1),
// 16381 x 8191 fp32 204 us (5.3); backward 16384 x 1024 bf16 23 + 4 us, 16381 x 8191 fp32 312 + 6 us (1.63 GB, 5.2 TB/s), the second figure the join of the partial sums.
// A plain copy of 2 GB runs at 4.8 TB/s here.
#include "mlmc_rows.h"

namespace mlmc {

constexpr int NORM_WG = 256;

struct NormArgs {
    const void *x, *dy;
    int64_t ldx, lddy, rows, d;
    int64_t row0;         // first row of a launch of a workgroup a row
    const float *weight, *bias, *stats_in;
    float eps;
    void *y, *dx;
    int64_t ldy, lddx;
    float* stats;
    float* part;          // [groups][2][d] sums of a group's rows
    int64_t groups;
};

// A workgroup takes WG / T rows at a time, and weight and bias stay in registers from round to round.  The next round's rows are on their way while one is worked on.
template <int DT, int T, int P, int WG> __global__ __launch_bounds__(WG, P <= 8 ? 8 : 4) void k_norm_forward_rows(NormArgs a) {
    using Row = RowChunks<DT, T, P>;
    constexpr int R = WG / T;
    __shared__ float2 part[2][2][WG / 64];
    const Row of(a.d, threadIdx.x % T);
    float w[P], b[P];
#pragma unroll
    for (int e = 0; e < P; ++e) {
        const int j = of.at(e);
        w[e] = a.weight && j < of.d ? a.weight[j] : 1.0f;
        b[e] = a.bias && j < of.d ? a.bias[j] : 0.0f;
    }
    const float inv_d = 1.0f / (float)a.d;
    chunk_t next[Row::N];
    const auto fetch = [&](int64_t row) { of.load(next, (const entry_t<DT>*)a.x + (row < a.rows ? row : a.rows - 1) * a.ldx); };
    int64_t row = (int64_t)blockIdx.x * R + __builtin_amdgcn_readfirstlane(threadIdx.x / T);
    fetch(row);
    int odd = 0;
    for (int64_t base = (int64_t)blockIdx.x * R; base < a.rows; base += (int64_t)gridDim.x * R, row += (int64_t)gridDim.x * R, odd ^= 1) {
        float x[P], s = 0.f, q = 0.f, none = 0.f;
        of.to_floats(x, next);
        fetch(row + (int64_t)gridDim.x * R);
#pragma unroll
        for (int e = 0; e < P; ++e) s += x[e];
        row_sums<T>(s, none, part[odd][0]);
        const float mean = quotient(s, (float)a.d, inv_d);
#pragma unroll
        for (int e = 0; e < P; ++e) x[e] -= mean;
        of.cut(x);
#pragma unroll
        for (int e = 0; e < P; ++e) q = fmaf(x[e], x[e], q);
        row_sums<T>(q, none, part[odd][1]);
        const float rstd = inverse_root(fmaf(q, inv_d, a.eps));
        if (row >= a.rows) continue;
#pragma unroll
        for (int e = 0; e < P; ++e) x[e] = fmaf(x[e] * rstd, w[e], b[e]);
        of.store((entry_t<DT>*)a.y + row * a.ldy, x);
        if (a.stats && threadIdx.x % T == 0) *(float2*)(a.stats + 2 * row) = make_float2(mean, rstd);
    }
}

// The same for the gradient, always in workgroups of 1024 threads, one for every CU: x and dy are read once, a thread's columns of dweight and dbias are added up in its registers over all its rows, then over the workgroup's rows
// in LDS, and a workgroup leaves one partial sum of each for k_norm_join.
template <int DT, int T, int P, int WG> __global__ __launch_bounds__(WG) void k_norm_backward_rows(NormArgs a) {
    constexpr bool AHEAD = P <= 8;   // the next round's rows on their way: with 16 entries a thread there are no registers for them
    using Row = RowChunks<DT, T, P>;
    constexpr int R = WG / T;
    __shared__ float2 part[2][WG / 64];
    __shared__ float add[R > 1 ? 2 * T * P : 1];
    const int t = threadIdx.x % T, sub = __builtin_amdgcn_readfirstlane(threadIdx.x / T);
    const Row of(a.d, t);
    float w[P], dw[P] = {}, db[P] = {};
#pragma unroll
    for (int e = 0; e < P; ++e) {
        const int j = of.at(e);
        w[e] = a.weight && j < of.d ? a.weight[j] : 1.0f;
    }
    const float inv_d = 1.0f / (float)a.d;
    chunk_t nx[Row::N], ny[Row::N];
    float2 ns;
    const auto fetch = [&](int64_t row) {
        row = row < a.rows ? row : a.rows - 1;
        of.load(nx, (const entry_t<DT>*)a.x + row * a.ldx);
        of.load(ny, (const entry_t<DT>*)a.dy + row * a.lddy);
        ns = make_float2(a.stats_in[2 * row], a.stats_in[2 * row + 1]);
    };
    int64_t row = (int64_t)blockIdx.x * R + sub;
    if (AHEAD) fetch(row);
    int odd = 0;
    for (int64_t base = (int64_t)blockIdx.x * R; base < a.rows; base += a.groups * R, row += a.groups * R, odd ^= 1) {
        if (!AHEAD) fetch(row);
        float h[P], c[P], s = 0.f, q = 0.f;
        float mean = ns.x, rstd = ns.y;
        of.to_floats(h, nx);
        of.to_floats(c, ny);
        if (R > 1 && row >= a.rows) {   // the last round's rows that are not there: what was read is the last row, or where dx is x or dy, what another wave has put there, Inf and NaN too
            mean = rstd = 0.f;
#pragma unroll
            for (int e = 0; e < P; ++e) h[e] = c[e] = 0.f;
        }
        if (AHEAD) fetch(row + a.groups * R);
#pragma unroll
        for (int e = 0; e < P; ++e) {
            h[e] = (h[e] - mean) * rstd;
            dw[e] = fmaf(c[e], h[e], dw[e]);   // past column d dy is zero
            db[e] += c[e];
            c[e] *= w[e];
            s += c[e];
            q = fmaf(c[e], h[e], q);
        }
        row_sums<T>(s, q, part[odd]);
        if (row >= a.rows) continue;
        s *= inv_d;
        q *= inv_d;
#pragma unroll
        for (int e = 0; e < P; ++e) c[e] = rstd * (fmaf(-h[e], q, c[e]) - s);
        of.store((entry_t<DT>*)a.dx + row * a.lddx, c);
    }
    if (!a.part) return;
    if constexpr (R > 1) {   // the sub-rows' sums one after the other
        for (int r = 0; r < R; ++r) {
            if (sub == r) {
#pragma unroll
                for (int e = 0; e < P; ++e) {   // thread-major: a wave's lanes side by side
                    float* p = add + 2 * e * T + t;
                    if (r == 0) { p[0] = dw[e]; p[T] = db[e]; }
                    else if (r < R - 1) { p[0] += dw[e]; p[T] += db[e]; }
                    else { dw[e] += p[0]; db[e] += p[T]; }
                }
            }
            __syncthreads();
        }
        if (sub != R - 1) return;
    }
    float* p = a.part + 2 * (int64_t)blockIdx.x * a.d;
#pragma unroll
    for (int e = 0; e < P; ++e) {
        const int j = of.at(e);
        if (j < of.d) {
            p[j] = dw[e];
            p[of.d + j] = db[e];
        }
    }
}

// ---- wider rows, and those of less than 16 bytes ----------------------------------------------------------------------------------------------------

// One workgroup per row, which it reads three times; the second and third read come from the caches (1000 x 20000 fp32: 100 us, 1.6 TB/s of x and y).
template <int DT> __global__ __launch_bounds__(NORM_WG) void k_norm_forward(NormArgs a) {
    __shared__ float part[2][NORM_WG / 64];
    const int64_t row = a.row0 + blockIdx.x;
    const entry_t<DT>* x = (const entry_t<DT>*)a.x + row * a.ldx;
    entry_t<DT>* y = (entry_t<DT>*)a.y + row * a.ldy;
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
        a.stats[2 * row] = mean;
        a.stats[2 * row + 1] = rstd;
    }
}

template <int DT> __global__ __launch_bounds__(NORM_WG) void k_norm_backward(NormArgs a) {
    __shared__ float part[2][NORM_WG / 64];
    const int64_t row = a.row0 + blockIdx.x;
    const entry_t<DT>* x = (const entry_t<DT>*)a.x + row * a.ldx;
    const entry_t<DT>* dy = (const entry_t<DT>*)a.dy + row * a.lddy;
    entry_t<DT>* dx = (entry_t<DT>*)a.dx + row * a.lddx;
    const float mean = a.stats_in[2 * row], rstd = a.stats_in[2 * row + 1];
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

// Half as many workgroups as the chip holds: each has more rounds for its copy of weight and bias and for the loads ahead (bf16, us, as many as it holds / half:
// 16384 x 512 18.7 / 13.0, 16384 x 1024 23.3 / 19.6, 8192 x 4096 36.8 / 32.6; fp32 16381 x 8191 203 / 205).
template <int DT, int T, int P> static mlmc_status forward_rows(const NormArgs& a, hipStream_t st) {
    constexpr int WG = T < 256 ? 256 : T, R = WG / T;
    const int64_t all = (a.rows + R - 1) / R, most = 256 * (1024 / WG);
    MLMC_LAUNCH(K_NORM_FORWARD, st, (k_norm_forward_rows<DT, T, P, WG><<<(unsigned)(all < most ? all : most), WG, 0, st>>>(a)));
    return MLMC_OK;
}
constexpr int64_t NORM_SLICE = LAUNCH_THREADS / NORM_WG;   // rows of a launch of a workgroup a row
static unsigned slice_rows(const NormArgs& a) { return (unsigned)(a.rows - a.row0 < NORM_SLICE ? a.rows - a.row0 : NORM_SLICE); }

template <int DT> static mlmc_status norm_forward(NormArgs a, hipStream_t st) {
    if (a.d < NORM_ROW_MIN || a.d > NORM_ROW_MAX) {
        for (; a.row0 < a.rows; a.row0 += NORM_SLICE) MLMC_LAUNCH(K_NORM_FORWARD, st, (k_norm_forward<DT><<<slice_rows(a), NORM_WG, 0, st>>>(a)));
        return MLMC_OK;
    }
    switch (row_threads(a.d)) {
        case 64: return forward_rows<DT, 64, 8>(a, st);
        case 128: return forward_rows<DT, 128, 8>(a, st);
        case 256: return forward_rows<DT, 256, 8>(a, st);
        case 512: return forward_rows<DT, 512, 8>(a, st);
        default: return a.d <= 8192 ? forward_rows<DT, 1024, 8>(a, st) : forward_rows<DT, 1024, 16>(a, st);
    }
}
template <int DT, int T, int P> static mlmc_status backward_rows(const NormArgs& a, hipStream_t st) {
    MLMC_LAUNCH(K_NORM_BACKWARD, st, (k_norm_backward_rows<DT, T, P, 1024><<<(unsigned)a.groups, 1024, 0, st>>>(a)));
    return MLMC_OK;
}
template <int DT> static mlmc_status norm_backward(NormArgs a, hipStream_t st) {
    if (a.d < NORM_ROW_MIN || a.d > NORM_ROW_MAX) {
        const dim3 grid((unsigned)((a.d + NORM_WG - 1) / NORM_WG), (unsigned)a.groups);
        if (a.part) MLMC_LAUNCH(K_NORM_COLUMNS, st, (k_norm_columns<DT><<<grid, NORM_WG, 0, st>>>(a)));
        for (; a.row0 < a.rows; a.row0 += NORM_SLICE) MLMC_LAUNCH(K_NORM_BACKWARD, st, (k_norm_backward<DT><<<slice_rows(a), NORM_WG, 0, st>>>(a)));
        return MLMC_OK;
    }
    switch (row_threads(a.d)) {
        case 64: return backward_rows<DT, 64, 8>(a, st);
        case 128: return backward_rows<DT, 128, 8>(a, st);
        case 256: return backward_rows<DT, 256, 8>(a, st);
        case 512: return backward_rows<DT, 512, 8>(a, st);
        default: return a.d <= 8192 ? backward_rows<DT, 1024, 8>(a, st) : backward_rows<DT, 1024, 16>(a, st);
    }
}

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
    return dtype == MLMC_F32 ? norm_forward<MLMC_F32>(a, st) : norm_forward<MLMC_BF16>(a, st);
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
    a.part = (float*)ws; a.groups = norm_groups(rows, d);
    if (!sums) a.part = nullptr;
    if (rows > 0) {
        const mlmc_status rc = dtype == MLMC_F32 ? norm_backward<MLMC_F32>(a, st) : norm_backward<MLMC_BF16>(a, st);
        if (rc != MLMC_OK) return rc;
    }
    return sums ? join_columns({a.part, rows > 0 ? a.groups : 0, d, 0, 2, {dweight, dbias}, grad_dtype}, st) : MLMC_OK;
}

}  // extern "C"
