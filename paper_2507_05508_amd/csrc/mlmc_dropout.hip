// Dropout whose mask is made again instead of stored (entry point mlmc_dropout).
//
//   y_ij = x_ij keep_ij / (1 - p) + residual_ij
//
// keep_ij is one of eight 16-bit halves of a block of Philox4x32-10 (Salmon et al., SC'11): key = seed, counter = (step, stream, first row + i, 1 + j / 8); the half, counted from the low
// half of word 0, is j % 8; the entry is kept if it is at least p 2^16.  So the mask is a function of the place in the matrix alone, not of types, strides or launches, and the backward pass
// is the same call on the gradient.  The last counter word is never zero, which that of the level draws always is: no block serves both.  Sixteen bits an entry: the generator is
// quarter-rate multiplications, and a block for four entries would take longer than memory does for entries of 16 bits; p is one of 65536 values, the scale is that of the p that is taken.
//
// Bound by memory, the generator beside it.
#include "mlmc_device.h"
#include "mlmc_worker.h"

namespace mlmc {

constexpr int DROP_WG = 256;

struct DropoutArgs {
    const void *x, *residual;
    void* y;
    int64_t ldx, ldr, ldy, rows, d;
    uint64_t seed;
    uint32_t step, stream, row0, least;   // least: of a half that keeps its entry
    float scale;
    int along;                            // log2 of a workgroup's threads along a row
};

template <int DT> __device__ inline void load_eight(float (&f)[8], const entry_t<DT>* p) {
    if constexpr (DT == MLMC_BF16) {
        const v8b u = __builtin_bit_cast(v8b, (chunk_t) * (const chunk_u*)p);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (float)u[e];
    } else {
        const v4f u = __builtin_bit_cast(v4f, (chunk_t) * (const chunk_u*)p), v = __builtin_bit_cast(v4f, (chunk_t) * (const chunk_u*)(p + 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) { f[e] = u[e]; f[4 + e] = v[e]; }
    }
}
template <int DT> __device__ inline void store_eight(entry_t<DT>* p, const float (&f)[8]) {
    if constexpr (DT == MLMC_BF16) {
        v8b u;
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = (__bf16)f[e];
        *(chunk_u*)p = __builtin_bit_cast(chunk_t, u);
    } else {
        *(chunk_u*)p = __builtin_bit_cast(chunk_t, v4f{f[0], f[1], f[2], f[3]});
        *(chunk_u*)(p + 4) = __builtin_bit_cast(chunk_t, v4f{f[4], f[5], f[6], f[7]});
    }
}

// A thread has eight neighbouring entries of a row, a workgroup a power of two of such groups and several rows.
template <int DT, bool RES> __global__ __launch_bounds__(DROP_WG) void k_dropout(DropoutArgs a) {
    const int along = 1 << a.along;
    const int64_t group = (int64_t)blockIdx.x * along + (threadIdx.x & (along - 1)), j = group * 8;
    if (j >= a.d) return;
    const bool whole = j + 8 <= a.d;
    const int n = whole ? 8 : (int)(a.d - j);
    const int64_t stride = (int64_t)gridDim.y * (DROP_WG >> a.along);
    for (int64_t row = (int64_t)blockIdx.y * (DROP_WG >> a.along) + (threadIdx.x >> a.along); row < a.rows; row += stride) {
        const entry_t<DT>* x = (const entry_t<DT>*)a.x + row * a.ldx + j;
        const entry_t<DT>* u = (const entry_t<DT>*)a.residual + (RES ? row * a.ldr + j : 0);
        entry_t<DT>* y = (entry_t<DT>*)a.y + row * a.ldy + j;
        float f[8] = {}, g[8] = {};
        if (whole) {
            load_eight<DT>(f, x);
            if (RES) load_eight<DT>(g, u);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n) {
                    f[e] = to_f32(x[e]);
                    if (RES) g[e] = to_f32(u[e]);
                }
        }
        const uint4 w = philox(a.step, a.stream, a.row0 + (uint32_t)row, (uint32_t)group + 1, a.seed);
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t half = e & 1 ? word[e / 2] >> 16 : word[e / 2] & 0xffff;
            const bool keep = half >= a.least;   // a choice, not a product: what is dropped may be infinite
            f[e] = RES ? (keep ? fmaf(f[e], a.scale, g[e]) : g[e]) : keep ? f[e] * a.scale : 0.f;
        }
        if (whole) store_eight<DT>(y, f);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n) y[e] = from_f32<DT>(f[e]);
        }
    }
}

template <int DT> static mlmc_status dropout_run(DropoutArgs a, hipStream_t st) {
    const int64_t groups = (a.d + 7) / 8;
    while (a.along < 8 && (1 << a.along) < groups) ++a.along;
    const int64_t gx = (groups + (1 << a.along) - 1) >> a.along, rows_at_once = DROP_WG >> a.along, gy = (a.rows + rows_at_once - 1) / rows_at_once;
    const int64_t want = 8192 / gx, most = want > 1 ? want : 1;
    const dim3 grid((unsigned)gx, (unsigned)(gy < most ? gy : most));
    if (a.residual) MLMC_LAUNCH(K_DROPOUT, st, (k_dropout<DT, true><<<grid, DROP_WG, 0, st>>>(a)));
    else MLMC_LAUNCH(K_DROPOUT, st, (k_dropout<DT, false><<<grid, DROP_WG, 0, st>>>(a)));
    return MLMC_OK;
}

}  // namespace mlmc

using namespace mlmc;

extern "C" mlmc_status mlmc_dropout(const void* x, int64_t ldx, int64_t rows, int64_t d, int dtype, double p, uint64_t seed, uint64_t step, uint32_t stream, int64_t row0,
                                    const void* residual, int64_t ldr, void* y, int64_t ldy, void* hip_stream) {
    if (rows < 0 || rows >= ((int64_t)1 << 31) || d < 1 || d >= ((int64_t)1 << 31) || !entry_dtype_ok(dtype) || ldx < d || ldy < d || (residual && ldr < d)) return MLMC_EINVAL;
    if (!(p >= 0.0) || !(p * 65536.0 + 0.5 < 65536.0) || step >> 32 || row0 < 0 || row0 > ((int64_t)1 << 32) - rows) return MLMC_EINVAL;
    if (rows == 0) return MLMC_OK;
    if (!entry_ptr_ok(x, dtype) || !entry_ptr_ok(y, dtype) || (residual && !entry_ptr_ok(residual, dtype))) return MLMC_EINVAL;
    DropoutArgs a = {};
    a.x = x; a.ldx = ldx; a.residual = residual; a.ldr = ldr; a.y = y; a.ldy = ldy; a.rows = rows; a.d = d; a.seed = seed; a.step = (uint32_t)step; a.stream = stream;
    a.row0 = (uint32_t)row0;
    a.least = (uint32_t)(p * 65536.0 + 0.5);
    a.scale = (float)(65536.0 / (double)(65536 - a.least));
    return dtype == MLMC_F32 ? dropout_run<MLMC_F32>(a, (hipStream_t)hip_stream) : dropout_run<MLMC_BF16>(a, (hipStream_t)hip_stream);
}
