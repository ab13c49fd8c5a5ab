// Root-mean-square norm of rows with the residual's addition, forward and backward, and rows brought into 8 bits (entry points mlmc_rms_norm, mlmc_rms_norm_backward,
// mlmc_quantize).
//
//   s = x + residual,  r = 1 / sqrt(mean_j s_j^2 + eps),  y_j = s_j r w_j;  in 8 bits: scale = max_j |y_j| / 448 (at least 2^-100), q_j = e4m3(448 y_j / max |y|)
//   backward, with h_j = s_j r and c_j = dy_j w_j:  ds_j = r (c_j - h_j mean(c h)) + what reaches s by another way,  dw_j = sum_rows dy_j h_j
//
// 448 is the greatest e4m3 value.  One scale a row, so that a product of two such matrices takes its scales in the epilogue.  The least scale keeps the division within
// normal numbers; entries below 2^-110 become zeros then.  y comes from the fp32 sum, not from the rounded one that is stored: every output is rounded once.
//
// Bound by memory: x and the residual are read once, the sum and the norm written once, where a row fits in the registers of its threads (8 to 16384 entries).
#include "mlmc_rows.h"

namespace mlmc {

constexpr int RMS_WG = 256;

struct RmsArgs {
    const void *x, *residual, *dy;
    int64_t ldx, ldr, lddy, rows, d;
    int64_t row0;         // first row of a launch of a workgroup a row
    const float *weight, *rstd_in;
    float eps;
    void *sum, *y, *dx;
    int64_t lds, ldy, lddx;
    uint8_t* q;
    int64_t ldq;
    float *scale, *rstd;
    float* part;          // [groups][d] sums of a group's rows
    int64_t groups;
    void* dweight;        // written by the only group, if there is no more than one
    int grad_dtype;
};

constexpr float E4M3_MAX = 448.f, LEAST_SCALE = 0x1p-100f;

// What brings a row whose greatest magnitude has these bits into 8 bits: its scale (NaN for infinities and NaN, which have the greatest bits), and the scale's inverse 448 / greatest as a sum of
// two, so that entries are rounded once on their way to e4m3, where they lie next to the middle of two values too.
struct ToEight {
    float scale, hi, lo;
    __device__ ToEight(uint32_t most) {
        const float m = __builtin_bit_cast(float, most);
        scale = fmaxf(m / E4M3_MAX, LEAST_SCALE);
        hi = m < E4M3_MAX * LEAST_SCALE ? 1.0f / LEAST_SCALE : E4M3_MAX / m;
        lo = m < E4M3_MAX * LEAST_SCALE ? 0.f : fmaf(-hi, m, E4M3_MAX) / m;
        if (most >= 0x7f800000u) scale = hi = __builtin_nanf("");
    }
    __device__ float operator()(float y, float rest) const { return fmaf(y, hi, fmaf(y, lo, rest * hi)); }   // of y + rest
};
// s r w, rounded once, and what that leaves over.  c is a number: where w or r is infinite it is an infinity of either sign or NaN, and y is h w (the median takes the least for a NaN).
// The median takes 8192 x 8192 bf16 from 44.4 us to 45.7 and no time with a residual; a branch for rows without infinities took 46.9, and 45.5 for 42.2 with residual and 8 bits (8192 x 4096).
__device__ inline float normed(float s, float r, float w, float& rest) {
    const float h = s * r, c = __builtin_amdgcn_fmed3f(fmaf(s, r, -h) * w, -3.402823466e38f, 3.402823466e38f), y = fmaf(h, w, c);
    rest = fmaf(h, w, -y) + c;
    return y;
}
__device__ inline int four_e4m3(float a, float b, float c, float d) {
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
__device__ inline uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

// Greatest of the T threads of a row, and of a wave.
template <int CTRL, int ROWS> __device__ inline uint32_t dpp_max(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, ROWS, 0xF, false);
    return v > o ? v : o;
}
__device__ inline uint32_t wave_most(uint32_t v) {
    v = dpp_max<0x111, 0xF>(v);
    v = dpp_max<0x112, 0xF>(v);
    v = dpp_max<0x114, 0xF>(v);
    v = dpp_max<0x118, 0xF>(v);
    v = dpp_max<0x142, 0xA>(v);
    v = dpp_max<0x143, 0xC>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
template <int T> __device__ inline uint32_t row_most(uint32_t v, uint32_t* part) {
    v = wave_most(v);
    if (T == 64) return v;
    const int first = threadIdx.x / T * (T / 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll 4
    for (int w = 0; w < T / 64; ++w) v = max(v, part[first + w]);
    return v;
}
template <int T> __device__ inline float row_sum(float v, float* part) {
    v = wave_sum(v);
    if (T == 64) return v;
    const int first = threadIdx.x / T * (T / 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll 4
    for (int w = 0; w < T / 64; ++w) v += part[first + w];
    return v;
}

// A thread's entries of a row of 8 bits: as many bytes as a chunk of the row has entries.
using pair_u = int __attribute__((ext_vector_type(2), aligned(1)));
using word_u = int __attribute__((aligned(1)));
template <int DT, int T, int P> __device__ inline void store_e4m3(const RowChunks<DT, T, P>& of, uint8_t* row, const float (&f)[P]) {
    using Row = RowChunks<DT, T, P>;
    constexpr int E = Row::E;
#pragma unroll
    for (int n = 0; n < Row::N; ++n) {
        uint8_t* p = row + (unsigned)of.col(n);
        int w[E / 4];
#pragma unroll
        for (int k = 0; k < E / 4; ++k) w[k] = four_e4m3(f[n * E + 4 * k], f[n * E + 4 * k + 1], f[n * E + 4 * k + 2], f[n * E + 4 * k + 3]);
        if (of.col(n) + E <= of.d) {
            if constexpr (E == 8) *(pair_u*)p = pair_u{w[0], w[1]};
            else *(word_u*)p = w[0];
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (of.col(n) + e < of.d) p[e] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
        }
    }
}

// A workgroup takes WG / T rows at a time, and the weight stays in registers from round to round.  The next round's rows are on their way while one is worked on.  NORM: else rows are
// only brought into 8 bits.  Every row has its own threads, which read all of it before they write: outputs may lie in the inputs' place.
template <int DT, int T, int P, int WG, bool NORM, bool RES> __global__ __launch_bounds__(WG, !NORM && P <= 8 ? 8 : 4) void k_rms_forward_rows(RmsArgs a) {
    using Row = RowChunks<DT, T, P>;
    constexpr int R = WG / T;
    __shared__ float part[2][WG / 64];
    __shared__ uint32_t most[2][WG / 64];
    const Row of(a.d, threadIdx.x % T);
    float w[P];
#pragma unroll
    for (int e = 0; e < P; ++e) {
        const int j = of.at(e);
        w[e] = NORM && a.weight && j < of.d ? a.weight[j] : 1.0f;
    }
    const float inv_d = 1.0f / (float)a.d;
    chunk_t nx[Row::N], nr[Row::N];
    const auto fetch = [&](int64_t row) {
        row = row < a.rows ? row : a.rows - 1;
        of.load(nx, (const entry_t<DT>*)a.x + row * a.ldx);
        if (RES) of.load(nr, (const entry_t<DT>*)a.residual + row * a.ldr);
    };
    int64_t row = (int64_t)blockIdx.x * R + __builtin_amdgcn_readfirstlane(threadIdx.x / T);
    fetch(row);
    int odd = 0;
    for (int64_t base = (int64_t)blockIdx.x * R; base < a.rows; base += (int64_t)gridDim.x * R, row += (int64_t)gridDim.x * R, odd ^= 1) {
        float x[P];
        of.to_floats(x, nx);
        if (RES) {
            float u[P];
            of.to_floats(u, nr);
#pragma unroll
            for (int e = 0; e < P; ++e) x[e] += u[e];
        }
        fetch(row + (int64_t)gridDim.x * R);
        const bool here = row < a.rows;
        if (NORM) {
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < P; ++e) s = fmaf(x[e], x[e], s);   // past column d there are zeros
            s = row_sum<T>(s, part[odd]);
            const float rstd = inverse_root(fmaf(s, inv_d, a.eps));
            if (here && RES && a.sum) of.store((entry_t<DT>*)a.sum + row * a.lds, x);
            if (here && a.rstd && threadIdx.x % T == 0) a.rstd[row] = rstd;
            float y[P], rest;
            if (!a.q) {
#pragma unroll
                for (int e = 0; e < P; ++e) x[e] = normed(x[e], rstd, w[e], rest);
                if (here) of.store((entry_t<DT>*)a.y + row * a.ldy, x);
                continue;
            }
#pragma unroll
            for (int e = 0; e < P; ++e) y[e] = normed(x[e], rstd, w[e], rest);
            if (here && a.y) of.store((entry_t<DT>*)a.y + row * a.ldy, y);
            of.cut(y);   // zero times an infinite weight or root
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < P; ++e) m = max(m, magnitude(y[e]));
            const ToEight eight(row_most<T>(m, most[odd]));
            if (!here) continue;
#pragma unroll
            for (int e = 0; e < P; ++e) {
                y[e] = normed(x[e], rstd, w[e], rest);
                y[e] = eight(y[e], rest);
            }
            store_e4m3(of, a.q + row * a.ldq, y);
            if (threadIdx.x % T == 0) a.scale[row] = eight.scale;
        } else {
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < P; ++e) m = max(m, magnitude(x[e]));
            const ToEight eight(row_most<T>(m, most[odd]));
            if (!here) continue;
#pragma unroll
            for (int e = 0; e < P; ++e) x[e] = eight(x[e], 0.f);
            store_e4m3(of, a.q + row * a.ldq, x);
            if (threadIdx.x % T == 0) a.scale[row] = eight.scale;
        }
    }
}

__device__ inline void sum_of_group(const RmsArgs& a, int64_t group, int64_t j, float v) {
    if (a.part) a.part[group * a.d + j] = v;
    else if (a.grad_dtype == MLMC_F32) ((float*)a.dweight)[j] = v;
    else ((__bf16*)a.dweight)[j] = (__bf16)v;
}

// The gradient, in workgroups of 1024 threads, one for every CU: dy and s are read once, a thread's columns of dweight are added up in its registers over all its rows, then over the
// workgroup's rows in LDS, and a workgroup leaves one partial sum for k_norm_join.
template <int DT, int T, int P, int WG, bool RES> __global__ __launch_bounds__(WG) void k_rms_backward_rows(RmsArgs a) {
    constexpr bool AHEAD = P <= 8;   // the next round's rows on their way: with 16 entries a thread there are no registers for them
    using Row = RowChunks<DT, T, P>;
    constexpr int R = WG / T;
    __shared__ float part[2][WG / 64];
    __shared__ float add[R > 1 ? T * P : 1];
    const int t = threadIdx.x % T, sub = __builtin_amdgcn_readfirstlane(threadIdx.x / T);
    const Row of(a.d, t);
    float w[P], dw[P] = {};
#pragma unroll
    for (int e = 0; e < P; ++e) {
        const int j = of.at(e);
        w[e] = a.weight && j < of.d ? a.weight[j] : 1.0f;
    }
    const float inv_d = 1.0f / (float)a.d;
    chunk_t nx[Row::N], ny[Row::N], nr[Row::N];
    float nrstd;
    const auto fetch = [&](int64_t row) {
        row = row < a.rows ? row : a.rows - 1;
        of.load(nx, (const entry_t<DT>*)a.x + row * a.ldx);
        of.load(ny, (const entry_t<DT>*)a.dy + row * a.lddy);
        if (RES) of.load(nr, (const entry_t<DT>*)a.residual + row * a.ldr);
        nrstd = a.rstd_in[row];
    };
    int64_t row = (int64_t)blockIdx.x * R + sub;
    if (AHEAD) fetch(row);
    int odd = 0;
    for (int64_t base = (int64_t)blockIdx.x * R; base < a.rows; base += a.groups * R, row += a.groups * R, odd ^= 1) {
        if (!AHEAD) fetch(row);
        float h[P], c[P], u[P], q = 0.f, rstd = nrstd;
        of.to_floats(h, nx);
        of.to_floats(c, ny);
        if (RES) of.to_floats(u, nr);
        if (R > 1 && row >= a.rows) {   // the last round's rows that are not there: what was read is the last row, or where dx lies in an input's place, what another wave has put there, Inf and NaN too
            rstd = 0.f;
#pragma unroll
            for (int e = 0; e < P; ++e) h[e] = c[e] = 0.f;
        }
        if (AHEAD) fetch(row + a.groups * R);
#pragma unroll
        for (int e = 0; e < P; ++e) {
            h[e] *= rstd;
            dw[e] = fmaf(c[e], h[e], dw[e]);   // past column d there are zeros
            c[e] *= w[e];
            q = fmaf(c[e], h[e], q);
        }
        q = row_sum<T>(q, part[odd]) * inv_d;
        if (row >= a.rows) continue;
#pragma unroll
        for (int e = 0; e < P; ++e) {
            c[e] = rstd * fmaf(-h[e], q, c[e]);
            if (RES) c[e] += u[e];
        }
        of.store((entry_t<DT>*)a.dx + row * a.lddx, c);
    }
    if (!a.part && !a.dweight) return;
    if constexpr (R > 1) {   // the sub-rows' sums one after the other
        for (int r = 0; r < R; ++r) {
            if (sub == r) {
#pragma unroll
                for (int e = 0; e < P; ++e) {   // thread-major: a wave's lanes side by side
                    float* p = add + e * T + t;
                    if (r == 0) *p = dw[e];
                    else if (r < R - 1) *p += dw[e];
                    else dw[e] += *p;
                }
            }
            __syncthreads();
        }
        if (sub != R - 1) return;
    }
#pragma unroll
    for (int e = 0; e < P; ++e) {
        const int j = of.at(e);
        if (j < of.d) sum_of_group(a, blockIdx.x, j, dw[e]);
    }
}

// ---- wider rows, and those of less than 16 bytes ----------------------------------------------------------------------------------------------------

// One workgroup per row, which it reads up to three times, the second and third time from the caches; a thread reads an entry for the last time before it writes in its place.
template <int DT, bool NORM> __global__ __launch_bounds__(RMS_WG) void k_rms_forward(RmsArgs a) {
    __shared__ float part[RMS_WG / 64];
    __shared__ uint32_t most[RMS_WG / 64];
    const int64_t row = a.row0 + blockIdx.x;
    const entry_t<DT>* x = (const entry_t<DT>*)a.x + row * a.ldx;
    const entry_t<DT>* u = a.residual ? (const entry_t<DT>*)a.residual + row * a.ldr : nullptr;
    const auto entry = [&](int64_t j) { return u ? to_f32(x[j]) + to_f32(u[j]) : to_f32(x[j]); };
    float rstd = 1.0f;
    if (NORM) {
        float s = 0.f;
        for (int64_t j = threadIdx.x; j < a.d; j += RMS_WG) {
            const float v = entry(j);
            s = fmaf(v, v, s);
        }
        rstd = inverse_root(row_sum<RMS_WG>(s, part) / (float)a.d + a.eps);
    }
    const auto result = [&](float v, int64_t j, float& rest) {
        rest = 0.f;
        return NORM ? normed(v, rstd, a.weight ? a.weight[j] : 1.0f, rest) : v;
    };
    float rest;
    uint32_t m = 0;
    if (a.q) {
        for (int64_t j = threadIdx.x; j < a.d; j += RMS_WG) m = max(m, magnitude(result(entry(j), j, rest)));
        m = row_most<RMS_WG>(m, most);
    }
    const ToEight eight(m);
    for (int64_t j = threadIdx.x; j < a.d; j += RMS_WG) {
        const float v = entry(j), y = result(v, j, rest);
        if (u && a.sum) ((entry_t<DT>*)a.sum)[row * a.lds + j] = from_f32<DT>(v);
        if (a.y) ((entry_t<DT>*)a.y)[row * a.ldy + j] = from_f32<DT>(y);
        if (a.q) a.q[row * a.ldq + j] = (uint8_t)four_e4m3(eight(y, rest), 0.f, 0.f, 0.f);
    }
    if (threadIdx.x == 0) {
        if (NORM && a.rstd) a.rstd[row] = rstd;
        if (a.q) a.scale[row] = eight.scale;
    }
}

template <int DT> __global__ __launch_bounds__(RMS_WG) void k_rms_backward(RmsArgs a) {
    __shared__ float part[RMS_WG / 64];
    const int64_t row = a.row0 + blockIdx.x;
    const entry_t<DT>* x = (const entry_t<DT>*)a.x + row * a.ldx;
    const entry_t<DT>* dy = (const entry_t<DT>*)a.dy + row * a.lddy;
    const entry_t<DT>* u = a.residual ? (const entry_t<DT>*)a.residual + row * a.ldr : nullptr;
    entry_t<DT>* dx = (entry_t<DT>*)a.dx + row * a.lddx;
    const float rstd = a.rstd_in[row];
    float q = 0.f;
    for (int64_t j = threadIdx.x; j < a.d; j += RMS_WG) q = fmaf(to_f32(dy[j]) * (a.weight ? a.weight[j] : 1.0f), to_f32(x[j]) * rstd, q);
    q = row_sum<RMS_WG>(q, part) / (float)a.d;
    for (int64_t j = threadIdx.x; j < a.d; j += RMS_WG) {
        const float c = to_f32(dy[j]) * (a.weight ? a.weight[j] : 1.0f), v = rstd * fmaf(-(to_f32(x[j]) * rstd), q, c);
        dx[j] = from_f32<DT>(u ? v + to_f32(u[j]) : v);
    }
}

// A thread sums its column over the rows of the group.  Before k_rms_backward, whose dx may lie in an input's place.
template <int DT> __global__ __launch_bounds__(RMS_WG) void k_rms_columns(RmsArgs a) {
    const int64_t j = (int64_t)blockIdx.x * RMS_WG + threadIdx.x;
    if (j >= a.d) return;
    float dw = 0.f;
    for (int64_t i = blockIdx.y; i < a.rows; i += a.groups)
        dw = fmaf(to_f32(((const entry_t<DT>*)a.dy)[i * a.lddy + j]), to_f32(((const entry_t<DT>*)a.x)[i * a.ldx + j]) * a.rstd_in[i], dw);
    sum_of_group(a, blockIdx.y, j, dw);
}

// Half as many workgroups as the chip holds, each with more rounds for its copy of the weight and the loads ahead; without a weight, and where a thread has one load a round, all of them (us, as many
// as it holds / half: 8 bits of bf16 8192 x 8192 38 / 48, 20122 x 1880 25 / 28, 4096 x 4096 10.4 / 11.3, of 8000 x 16000 71 / 69.5, of fp32 4096 x 8192 29.7 / 28.9;
// the norm of bf16 8192 x 8192 50.4 / 46.5, 4096 x 4096 17.3 / 14.4, of 8192 x 8192 with residual and 8 bits 98 / 93).
template <int DT, int T, int P, bool NORM> static mlmc_status rms_forward_rows(const RmsArgs& a, hipStream_t st) {
    constexpr int WG = T < 256 ? 256 : T, R = WG / T;
    const int64_t all = (a.rows + R - 1) / R, most = (!NORM && P / ENTRIES<DT> == 1 ? 512 : 256) * (1024 / WG);
    const unsigned grid = (unsigned)(all < most ? all : most);
    if constexpr (!NORM) MLMC_LAUNCH(K_QUANTIZE, st, (k_rms_forward_rows<DT, T, P, WG, false, false><<<grid, WG, 0, st>>>(a)));
    else if (a.residual) MLMC_LAUNCH(K_RMS_FORWARD, st, (k_rms_forward_rows<DT, T, P, WG, true, true><<<grid, WG, 0, st>>>(a)));
    else MLMC_LAUNCH(K_RMS_FORWARD, st, (k_rms_forward_rows<DT, T, P, WG, true, false><<<grid, WG, 0, st>>>(a)));
    return MLMC_OK;
}
constexpr int64_t RMS_SLICE = LAUNCH_THREADS / RMS_WG;   // rows of a launch of a workgroup a row
static unsigned rms_slice(const RmsArgs& a) { return (unsigned)(a.rows - a.row0 < RMS_SLICE ? a.rows - a.row0 : RMS_SLICE); }

template <int DT, bool NORM> static mlmc_status rms_forward(RmsArgs a, hipStream_t st) {
    if (a.d < NORM_ROW_MIN || a.d > NORM_ROW_MAX) {
        for (; a.row0 < a.rows; a.row0 += RMS_SLICE) MLMC_LAUNCH(NORM ? K_RMS_FORWARD : K_QUANTIZE, st, (k_rms_forward<DT, NORM><<<rms_slice(a), RMS_WG, 0, st>>>(a)));
        return MLMC_OK;
    }
    switch (row_threads(a.d)) {
        case 64: return rms_forward_rows<DT, 64, 8, NORM>(a, st);
        case 128: return rms_forward_rows<DT, 128, 8, NORM>(a, st);
        case 256: return rms_forward_rows<DT, 256, 8, NORM>(a, st);
        case 512: return rms_forward_rows<DT, 512, 8, NORM>(a, st);
        default: return a.d <= 8192 ? rms_forward_rows<DT, 1024, 8, NORM>(a, st) : rms_forward_rows<DT, 1024, 16, NORM>(a, st);
    }
}
template <int DT, int T, int P> static mlmc_status rms_backward_rows(const RmsArgs& a, hipStream_t st) {
    if (a.residual) MLMC_LAUNCH(K_RMS_BACKWARD, st, (k_rms_backward_rows<DT, T, P, 1024, true><<<(unsigned)a.groups, 1024, 0, st>>>(a)));
    else MLMC_LAUNCH(K_RMS_BACKWARD, st, (k_rms_backward_rows<DT, T, P, 1024, false><<<(unsigned)a.groups, 1024, 0, st>>>(a)));
    return MLMC_OK;
}
template <int DT> static mlmc_status rms_backward(RmsArgs a, hipStream_t st) {
    if (a.d < NORM_ROW_MIN || a.d > NORM_ROW_MAX) {
        const dim3 grid((unsigned)((a.d + RMS_WG - 1) / RMS_WG), (unsigned)a.groups);
        if (a.part || a.dweight) MLMC_LAUNCH(K_RMS_COLUMNS, st, (k_rms_columns<DT><<<grid, RMS_WG, 0, st>>>(a)));
        for (; a.row0 < a.rows; a.row0 += RMS_SLICE) MLMC_LAUNCH(K_RMS_BACKWARD, st, (k_rms_backward<DT><<<rms_slice(a), RMS_WG, 0, st>>>(a)));
        return MLMC_OK;
    }
    switch (row_threads(a.d)) {
        case 64: return rms_backward_rows<DT, 64, 8>(a, st);
        case 128: return rms_backward_rows<DT, 128, 8>(a, st);
        case 256: return rms_backward_rows<DT, 256, 8>(a, st);
        case 512: return rms_backward_rows<DT, 512, 8>(a, st);
        default: return a.d <= 8192 ? rms_backward_rows<DT, 1024, 8>(a, st) : rms_backward_rows<DT, 1024, 16>(a, st);
    }
}

}  // namespace mlmc

using namespace mlmc;

extern "C" {

size_t mlmc_rms_norm_workspace(int64_t rows, int64_t d) {
    const int64_t groups = norm_sizes_ok(rows, d) ? norm_groups(rows, d) : 0;
    return groups > 1 ? (size_t)groups * (size_t)d * sizeof(float) : 0;
}

mlmc_status mlmc_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, int64_t rows, int64_t d, int dtype, const float* weight, float eps,
                          void* sum, int64_t lds, void* y, int64_t ldy, uint8_t* q, int64_t ldq, float* scale, float* rstd, void* hip_stream) {
    if (!norm_sizes_ok(rows, d) || !entry_dtype_ok(dtype) || ldx < d || (residual && ldr < d) || !(eps >= 0.0f) || eps > 3.402823e38f) return MLMC_EINVAL;
    if ((sum && (!residual || lds < d)) || (y && ldy < d) || (q && ldq < d)) return MLMC_EINVAL;
    if (rows == 0) return MLMC_OK;
    if (!entry_ptr_ok(x, dtype) || (residual && !entry_ptr_ok(residual, dtype)) || (sum && !entry_ptr_ok(sum, dtype)) || (y && !entry_ptr_ok(y, dtype))) return MLMC_EINVAL;
    if ((!y && !q) || (y && y == sum) || (q && !scale) || !f32_ptr_ok(weight) || !f32_ptr_ok(scale) || !f32_ptr_ok(rstd)) return MLMC_EINVAL;
    hipStream_t st = (hipStream_t)hip_stream;
    RmsArgs a = {};
    a.x = x; a.ldx = ldx; a.residual = residual; a.ldr = ldr; a.rows = rows; a.d = d; a.weight = weight; a.eps = eps;
    a.sum = sum; a.lds = lds; a.y = y; a.ldy = ldy; a.q = q; a.ldq = ldq; a.scale = scale; a.rstd = rstd;
    return dtype == MLMC_F32 ? rms_forward<MLMC_F32, true>(a, st) : rms_forward<MLMC_BF16, true>(a, st);
}

mlmc_status mlmc_rms_norm_backward(const void* dy, int64_t lddy, const void* s, int64_t lds, int64_t rows, int64_t d, int dtype, const float* weight, const float* rstd,
                                   const void* residual, int64_t ldr, void* dx, int64_t lddx, void* dweight, int grad_dtype, void* ws, size_t ws_bytes,
                                   void* hip_stream) {
    if (!norm_sizes_ok(rows, d) || !entry_dtype_ok(dtype) || lddy < d || lds < d || lddx < d || (residual && ldr < d)) return MLMC_EINVAL;
    if (dweight && (!entry_dtype_ok(grad_dtype) || !entry_ptr_ok(dweight, grad_dtype))) return MLMC_EINVAL;
    if (rows > 0 && (!entry_ptr_ok(dy, dtype) || !entry_ptr_ok(s, dtype) || !entry_ptr_ok(dx, dtype) || !rstd || !f32_ptr_ok(rstd) || !f32_ptr_ok(weight))) return MLMC_EINVAL;
    if (rows > 0 && residual && !entry_ptr_ok(residual, dtype)) return MLMC_EINVAL;
    const size_t need = dweight ? mlmc_rms_norm_workspace(rows, d) : 0;
    if (need && (!ws || (uintptr_t)ws % 256 || ws_bytes < need)) return MLMC_EINVAL;
    hipStream_t st = (hipStream_t)hip_stream;
    RmsArgs a = {};
    a.dy = dy; a.lddy = lddy; a.x = s; a.ldx = lds; a.rows = rows; a.d = d; a.weight = weight; a.rstd_in = rstd; a.residual = residual; a.ldr = ldr;
    a.dx = dx; a.lddx = lddx; a.part = need ? (float*)ws : nullptr; a.groups = norm_groups(rows, d); a.dweight = dweight; a.grad_dtype = grad_dtype;
    if (rows > 0) {
        const mlmc_status rc = dtype == MLMC_F32 ? rms_backward<MLMC_F32>(a, st) : rms_backward<MLMC_BF16>(a, st);
        if (rc != MLMC_OK) return rc;
    }
    if (!dweight || (rows > 0 && !need)) return MLMC_OK;
    return join_columns({a.part, rows > 0 ? a.groups : 0, d, 0, 1, {dweight, nullptr}, grad_dtype}, st);
}

mlmc_status mlmc_quantize(const void* x, int64_t ldx, int64_t rows, int64_t d, int dtype, uint8_t* q, int64_t ldq, float* scale, void* hip_stream) {
    if (!norm_sizes_ok(rows, d) || !entry_dtype_ok(dtype) || ldx < d || ldq < d) return MLMC_EINVAL;
    if (rows == 0) return MLMC_OK;
    if (!entry_ptr_ok(x, dtype) || !q || !scale || !f32_ptr_ok(scale)) return MLMC_EINVAL;
    hipStream_t st = (hipStream_t)hip_stream;
    RmsArgs a = {};
    a.x = x; a.ldx = ldx; a.rows = rows; a.d = d; a.q = q; a.ldq = ldq; a.scale = scale;
    return dtype == MLMC_F32 ? rms_forward<MLMC_F32, false>(a, st) : rms_forward<MLMC_BF16, false>(a, st);
}

}  // extern "C"
