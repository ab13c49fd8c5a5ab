// Distillation from a teacher's top logits: the loss of every row and its gradient (entry point mlmc_distill).
//
// A row has logits s_0..s_{V-1} and the teacher's K entries (i_k, t_k).  With T the temperature,
//   q_k = exp(t_k / T) / sum_k' exp(t_k' / T),   p_j = exp(s_j / T) / sum_j' exp(s_j' / T),
//   loss = T^2 sum_k q_k (log q_k - log p_{i_k}),   d loss / d s_j = T (p_j - sum over k with i_k = j of q_k).
// Entries of an index below zero are padding.  A row with no entry, or whose entries are all -Inf, is masked: its logits are not
// read, its loss and gradient are zero.
#include "mlmc_worker.h"

namespace mlmc {

constexpr int DIS_WG = 256;
constexpr int DIS_TOP = MLMC_MAX_TEACHER;

struct DistillArgs {
    const void* s;
    int64_t lds, rows, vocab;
    const int32_t* t_idx;
    const float* t_val;
    int top;
    float temp, inv_temp;
    const float* dloss;
    float scale;
    float* loss;
    void* ds;
    int64_t ldds;
    int32_t* dev_status;
};

__global__ void k_distill_clear(int32_t* dev_status) { *dev_status = 0; }

// One workgroup per row, which it reads three times (greatest entry, sum, gradient).
template <int DT> __global__ __launch_bounds__(DIS_WG) void k_distill(DistillArgs a) {
    __shared__ float part[6][DIS_WG / 64];
    __shared__ float q[DIS_TOP], gather[DIS_TOP];
    __shared__ int32_t at[DIS_TOP];
    __shared__ int bad, live;
    const int64_t row = blockIdx.x;
    const entry_t<DT>* s = (const entry_t<DT>*)a.s + row * a.lds;
    entry_t<DT>* ds = a.ds ? (entry_t<DT>*)a.ds + row * a.ldds : nullptr;
    if (threadIdx.x == 0) bad = live = 0;
    __syncthreads();
    float tmax = -INFINITY;
    for (int k = threadIdx.x; k < a.top; k += DIS_WG) {
        const int32_t i = a.t_idx[row * a.top + k];
        const float t = a.t_val[row * a.top + k];
        if (i >= a.vocab) bad = 1;
        const bool here = i >= 0 && i < a.vocab;
        at[k] = here ? i : -1;
        q[k] = t;
        gather[k] = here ? to_f32(s[i]) : 0.f;
        if (here && t != -INFINITY) live = 1;   // a NaN too: it reaches the sum
        if (here) tmax = fmaxf(tmax, t);
    }
    tmax = group_max<DIS_WG / 64>(tmax, part[0]);
    float sum = 0.f;
    for (int k = threadIdx.x; k < a.top; k += DIS_WG) {
        const float u = (q[k] - tmax) * a.inv_temp;
        q[k] = u;
        if (at[k] >= 0) sum += expf(u);
    }
    const float qsum = group_sum<DIS_WG / 64>(sum, part[1]);   // its barrier is also the one after `bad` and `live`
    const float w = a.dloss ? a.dloss[row] * a.scale : a.scale;
    const bool masked = !live, zero = masked || bad || w == 0.f;
    if (bad && threadIdx.x == 0 && a.dev_status) atomicOr(a.dev_status, MLMC_DEV_RANGE);
    if (masked || bad) {
        if (threadIdx.x == 0) a.loss[row] = bad ? __builtin_nanf("") : 0.f;
        if (ds) for (int64_t j = threadIdx.x; j < a.vocab; j += DIS_WG) ds[j] = from_f32<DT>(0.f);
        return;
    }
    float m = -INFINITY;
    for (int64_t j = threadIdx.x; j < a.vocab; j += DIS_WG) m = fmaxf(m, to_f32(s[j]));
    m = group_max<DIS_WG / 64>(m, part[2]);
    sum = 0.f;
    for (int64_t j = threadIdx.x; j < a.vocab; j += DIS_WG) sum += expf((to_f32(s[j]) - m) * a.inv_temp);
    const float psum = group_sum<DIS_WG / 64>(sum, part[3]);
    const float log_q = logf(qsum), log_p = logf(psum);
    float l = 0.f;
    for (int k = threadIdx.x; k < a.top; k += DIS_WG) {
        const float u = q[k];
        q[k] = at[k] >= 0 ? expf(u) / qsum : 0.f;
        if (q[k] != 0.f) l += q[k] * ((u - log_q) - ((gather[k] - m) * a.inv_temp - log_p));
    }
    l = group_sum<DIS_WG / 64>(l, part[4]);
    if (threadIdx.x == 0) a.loss[row] = a.temp * a.temp * l;
    if (!ds) return;
    const float c = a.temp * w, inv = 1.0f / psum;
    for (int64_t j = threadIdx.x; j < a.vocab; j += DIS_WG) ds[j] = from_f32<DT>(zero ? 0.f : c * (expf((to_f32(s[j]) - m) * a.inv_temp) * inv));
    if (zero) return;
    __syncthreads();
    for (int k = threadIdx.x; k < a.top; k += DIS_WG) {
        if (at[k] < 0) continue;
        float qs = 0.f;   // an index may be there twice: each of its threads writes the same sum
        for (int o = 0; o < a.top; ++o) qs += at[o] == at[k] ? q[o] : 0.f;
        ds[at[k]] = from_f32<DT>(c * (expf((gather[k] - m) * a.inv_temp) * inv - qs));
    }
}

}  // namespace mlmc

using namespace mlmc;

extern "C" {

size_t mlmc_distill_workspace(int64_t rows, int64_t vocab, int top) {
    (void)rows; (void)vocab; (void)top;
    return 0;
}

mlmc_status mlmc_distill(const void* logits, int64_t ldl, int64_t rows, int64_t vocab, int dtype, const int32_t* t_idx, const float* t_val, int top,
                         float temperature, const float* dloss, float scale, float* loss, void* dlogits, int64_t ldd, int32_t* dev_status,
                         void* ws, size_t ws_bytes, void* hip_stream) {
    if (rows < 0 || rows >= ((int64_t)1 << 31) || vocab < 1 || vocab >= ((int64_t)1 << 31) || !entry_dtype_ok(dtype) || top < 1 || top > MLMC_MAX_TEACHER) return MLMC_EINVAL;
    if (!(temperature > 0.0f) || temperature > 3.402823e38f || !(1.0f / temperature <= 3.402823e38f) || ldl < vocab || (dlogits && ldd < vocab)) return MLMC_EINVAL;
    hipStream_t st = (hipStream_t)hip_stream;
    if (!f32_ptr_ok(dev_status)) return MLMC_EINVAL;
    if (rows > 0) {
        if (!entry_ptr_ok(logits, dtype) || !t_idx || !f32_ptr_ok(t_idx) || !t_val || !f32_ptr_ok(t_val) || !f32_ptr_ok(dloss) || !loss || !f32_ptr_ok(loss)) return MLMC_EINVAL;
        if (dlogits && !entry_ptr_ok(dlogits, dtype)) return MLMC_EINVAL;
    }
    const size_t need = mlmc_distill_workspace(rows, vocab, top);
    if (need && (!ws || (uintptr_t)ws % 256 || ws_bytes < need)) return MLMC_EINVAL;
    if (dev_status) MLMC_LAUNCH(K_ZERO, st, (k_distill_clear<<<1, 1, 0, st>>>(dev_status)));
    if (rows == 0) return MLMC_OK;
    DistillArgs a = {};
    a.s = logits; a.lds = ldl; a.rows = rows; a.vocab = vocab; a.t_idx = t_idx; a.t_val = t_val; a.top = top; a.temp = temperature;
    a.inv_temp = 1.0f / temperature; a.dloss = dloss; a.scale = scale; a.loss = loss; a.ds = dlogits; a.ldds = ldd; a.dev_status = dev_status;
    if (dtype == MLMC_F32) MLMC_LAUNCH(K_DISTILL, st, (k_distill<MLMC_F32><<<(unsigned)rows, DIS_WG, 0, st>>>(a)));
    else MLMC_LAUNCH(K_DISTILL, st, (k_distill<MLMC_BF16><<<(unsigned)rows, DIS_WG, 0, st>>>(a)));
    return MLMC_OK;
}

}  // extern "C"
