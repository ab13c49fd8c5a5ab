// Matrix product with bias, activation and residual in its epilogue, and its two gradients (entry points mlmc_linear,
// mlmc_linear_dgrad, mlmc_linear_wgrad).
//
//   forward:  z = x W^T + b, y = act(z) + r         x [n][k], W [m][k]; contraction over k
//   dgrad:    dx = (dy W) act'(z) + r               dy [n][m];          contraction over m
//   wgrad:    dW = dy^T x, db = sum over rows of dy;                    contraction over n
//
// Products of many rows are bound by the matrix units and what feeds them, those of few rows by reading the weight.  Kernel times: 8192 x 4096 x 4096 bf16 with gelu,
// v stored too, 250 us (1.1 PFLOP/s; the matrix units are busy in 55 % of the cycles at the 1.86 GHz that the card runs then; a library product without the epilogue
// takes 177 to 220 us); input gradient 4001 x 4096 x 4096 with gelu 130 us (1.03 PFLOP/s); weight gradient 4096 x 1024 over 8192 rows, fp32 out, 73 + 10 us (the second is the
// join of two parts; library 82 to 88); fp32 1000 x 2049 x 1537 80 us (library 78), 2048 x 2048 x 2048 124 us (139 TFLOP/s); one row of 4096 x 4096 8.6 us (3.9 TB/s).
#include "mlmc_linear.h"

namespace mlmc {

template <bool AA, bool BA> static mlmc_status linear_run(const LinearArgs& g, int dtype, hipStream_t st) {
    return dtype == MLMC_F32 ? linear_layout<MLMC_F32, AA, BA>(g, st) : linear_layout<MLMC_BF16, AA, BA>(g, st);
}

}  // namespace mlmc

using namespace mlmc;


extern "C" {

size_t mlmc_linear_workspace(int64_t rows, int64_t outputs, int64_t inputs, int call, int only) {
    if (!linear_sizes_ok(rows, outputs, inputs) || rows == 0 || call < 0 || call > 3 || (only != -1 && !entry_dtype_ok(only))) return 0;
    const int64_t size[3][3] = {{rows, outputs, inputs}, {rows, inputs, outputs}, {outputs, inputs, rows}};
    size_t most = 0;
    for (int c = 0; c < 3; ++c) {
        if (call && call != c + 1) continue;
        for (int dtype : {MLMC_F32, MLMC_BF16}) {
            if ((only != -1 && dtype != only) || (c == 0 && few_rows(rows, outputs, inputs, dtype))) continue;
            for (int fast = 0; fast < (dtype == MLMC_BF16 ? 2 : 1); ++fast) {   // 32-bit entries have the same tiles either way
                const size_t need = align256(linear_part_bytes(linear_plan(size[c][0], size[c][1], size[c][2], dtype, fast), size[c][0], size[c][1]));
                most = need > most ? need : most;
            }
        }
        if (only == MLMC_F32 || (c == 0 && few_rows(rows, outputs, inputs, MLMC_BF16))) continue;
        for (int way : {WAY_WORDS, WAY_REGISTERS})
            for (int which = 1; which < 4; ++which) {
                const PackPlan k = pack_plan(size[c][0], size[c][1], size[c][2], MLMC_BF16, c < 2, c == 0, way, which & 1, which & 2);
                const size_t need = align256(linear_part_bytes(k.plan, size[c][0], size[c][1])) + align256(k.bytes[0]) + k.bytes[1];
                most = need > most ? need : most;
            }
    }
    return most;
}

mlmc_status mlmc_linear(const void* x, int64_t ldx, const void* weight, int64_t ldw, int64_t rows, int64_t outputs, int64_t inputs, int dtype,
                        const float* bias, int act, const void* residual, int64_t ldr, void* z, int64_t ldz, void* y, int64_t ldy,
                        void* ws, size_t ws_bytes, void* hip_stream) {
    if (!linear_sizes_ok(rows, outputs, inputs) || !entry_dtype_ok(dtype) || !act_ok(act) || ldx < inputs || ldw < inputs || ldy < outputs) return MLMC_EINVAL;
    if ((residual && ldr < outputs) || (z && ldz < outputs)) return MLMC_EINVAL;
    if (rows == 0) return MLMC_OK;
    if (!entry_ptr_ok(x, dtype) || !entry_ptr_ok(weight, dtype) || !entry_ptr_ok(y, dtype) || !f32_ptr_ok(bias)) return MLMC_EINVAL;
    if ((residual && !entry_ptr_ok(residual, dtype)) || (z && !entry_ptr_ok(z, dtype))) return MLMC_EINVAL;
    LinearArgs g = {};
    g.a = x; g.lda = ldx; g.b = weight; g.ldb = ldw; g.I = rows; g.J = outputs; g.C = inputs;
    g.act = act; g.bias = bias; g.residual = residual; g.ldr = ldr; g.z = z; g.ldz = ldz; g.out = y; g.ldo = ldy; g.out_dtype = dtype; g.part = (float*)ws; g.ws_bytes = ws_bytes;
    if (few_rows(rows, outputs, inputs, dtype)) return dtype == MLMC_F32 ? linear_few<MLMC_F32>(g, (hipStream_t)hip_stream) : linear_few<MLMC_BF16>(g, (hipStream_t)hip_stream);
    return linear_run<true, true>(g, dtype, (hipStream_t)hip_stream);
}

mlmc_status mlmc_linear_dgrad(const void* dy, int64_t lddy, const void* weight, int64_t ldw, int64_t rows, int64_t outputs, int64_t inputs,
                              int dtype, int act, const void* z, int64_t ldz, const void* residual, int64_t ldr, void* dx, int64_t lddx,
                              void* ws, size_t ws_bytes, void* hip_stream) {
    if (!linear_sizes_ok(rows, outputs, inputs) || !entry_dtype_ok(dtype) || !act_ok(act) || lddy < outputs || ldw < inputs || lddx < inputs) return MLMC_EINVAL;
    if ((residual && ldr < inputs) || (act != MLMC_ACT_NONE && ldz < inputs)) return MLMC_EINVAL;
    if (rows == 0) return MLMC_OK;
    if (!entry_ptr_ok(dy, dtype) || !entry_ptr_ok(weight, dtype) || !entry_ptr_ok(dx, dtype)) return MLMC_EINVAL;
    if ((residual && !entry_ptr_ok(residual, dtype)) || (act != MLMC_ACT_NONE && !entry_ptr_ok(z, dtype))) return MLMC_EINVAL;
    LinearArgs g = {};
    g.a = dy; g.lda = lddy; g.b = weight; g.ldb = ldw; g.I = rows; g.J = inputs; g.C = outputs;
    g.act = act; g.slope_z = act != MLMC_ACT_NONE ? z : nullptr; g.ld_slope = ldz; g.residual = residual; g.ldr = ldr;
    g.out = dx; g.ldo = lddx; g.out_dtype = dtype; g.part = (float*)ws; g.ws_bytes = ws_bytes;
    return linear_run<true, false>(g, dtype, (hipStream_t)hip_stream);
}

mlmc_status mlmc_linear_wgrad(const void* dy, int64_t lddy, const void* x, int64_t ldx, int64_t rows, int64_t outputs, int64_t inputs, int dtype,
                              void* dweight, int64_t lddw, void* dbias, int grad_dtype, void* ws, size_t ws_bytes, void* hip_stream) {
    if (!linear_sizes_ok(rows, outputs, inputs) || !entry_dtype_ok(dtype) || !entry_dtype_ok(grad_dtype) || lddy < outputs || ldx < inputs || lddw < inputs) return MLMC_EINVAL;
    if (!entry_ptr_ok(dweight, grad_dtype) || (dbias && !entry_ptr_ok(dbias, grad_dtype))) return MLMC_EINVAL;
    if (rows > 0 && (!entry_ptr_ok(dy, dtype) || !entry_ptr_ok(x, dtype))) return MLMC_EINVAL;
    LinearArgs g = {};
    g.a = dy; g.lda = lddy; g.b = x; g.ldb = ldx; g.I = outputs; g.J = inputs; g.C = rows;
    g.act = MLMC_ACT_NONE; g.out = dweight; g.ldo = lddw; g.out_dtype = grad_dtype; g.row_sum = dbias; g.part = (float*)ws; g.ws_bytes = ws_bytes;
    return linear_run<false, false>(g, dtype, (hipStream_t)hip_stream);
}

}  // extern "C"
