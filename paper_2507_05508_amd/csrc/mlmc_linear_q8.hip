// Linear layer of matrices in 8 bits with a scale for every row (entry point mlmc_linear_q8): y = act((x_scale_n w_scale_m) x W^T + b) + r.
//
// The tiles, ways and epilogue are those of the linear layer (mlmc_linear.h).  A step of 128 bytes has 128 entries of the contraction instead of 64, and the matrix instructions for 8 bits
// take twice as many in the same time, so that loads and products keep their proportion.  Those instructions add the products of eight entries with what lies within 12 binary
// places of the greatest of them and cut the rest (measured: a product 2^-12 of the greatest is kept, one of 2^-14 lost): 1.5e-5 of a result of normal entries, a hundredth of its rounding to 16 bits.
// Accumulators are fp32.
#include "mlmc_linear.h"

using namespace mlmc;

extern "C" {

size_t mlmc_linear_q8_workspace(int64_t rows, int64_t outputs, int64_t inputs) {
    if (!linear_sizes_ok(rows, outputs, inputs) || rows == 0 || few_rows(rows, outputs, inputs, DT_E4M3)) return 0;
    size_t most = 0;
    for (bool fast : {false, true}) {
        const size_t need = align256(linear_part_bytes(linear_plan(rows, outputs, inputs, DT_E4M3, fast), rows, outputs));
        most = need > most ? need : most;
    }
    for (int which = 1; which < 4; ++which) {
        const PackPlan k = pack_plan(rows, outputs, inputs, DT_E4M3, true, true, WAY_REGISTERS, which & 1, which & 2);
        const size_t need = align256(linear_part_bytes(k.plan, rows, outputs)) + align256(k.bytes[0]) + k.bytes[1];
        most = need > most ? need : most;
    }
    return most;
}

mlmc_status mlmc_linear_q8(const uint8_t* x, int64_t ldx, const float* x_scale, const uint8_t* weight, int64_t ldw, const float* w_scale, int64_t rows, int64_t outputs,
                           int64_t inputs, const float* bias, int act, const void* residual, int64_t ldr, void* y, int64_t ldy, void* ws, size_t ws_bytes, void* hip_stream) {
    if (!linear_sizes_ok(rows, outputs, inputs) || !act_ok(act) || ldx < inputs || ldw < inputs || ldy < outputs || (residual && ldr < outputs)) return MLMC_EINVAL;
    if (rows == 0) return MLMC_OK;
    if (!x || !weight || !x_scale || !w_scale || !f32_ptr_ok(x_scale) || !f32_ptr_ok(w_scale) || !f32_ptr_ok(bias) || !entry_ptr_ok(y, MLMC_BF16)) return MLMC_EINVAL;
    if (residual && !entry_ptr_ok(residual, MLMC_BF16)) return MLMC_EINVAL;
    LinearArgs g = {};
    g.a = x; g.lda = ldx; g.row_scale = x_scale; g.b = weight; g.ldb = ldw; g.col_scale = w_scale; g.I = rows; g.J = outputs; g.C = inputs;
    g.act = act; g.bias = bias; g.residual = residual; g.ldr = ldr; g.out = y; g.ldo = ldy; g.out_dtype = MLMC_BF16; g.part = (float*)ws; g.ws_bytes = ws_bytes;
    if (few_rows(rows, outputs, inputs, DT_E4M3)) return linear_few<DT_E4M3>(g, (hipStream_t)hip_stream);
    return linear_layout<DT_E4M3, true, true>(g, (hipStream_t)hip_stream);
}

}  // extern "C"
