// Distillation from a teacher's top logits: the loss of every row and its gradient (entry point mlmc_distill).
//
// A row has logits s_0..s_{V-1} and the teacher's K entries (i_k, t_k).  With T the temperature,
//   q_k = exp(t_k / T) / sum_k' exp(t_k' / T),   p_j = exp(s_j / T) / sum_j' exp(s_j' / T),
//   loss = T^2 sum_k q_k (log q_k - log p_{i_k}),   d loss / d s_j = T (p_j - sum over k with i_k = j of q_k).
// Entries of an index below zero are padding.  A row with no entry, or whose entries are all -Inf, is masked: whatever its
// logits, its loss and gradient are zero.
//
// Bound by memory: the logits are read once and their gradient is written once, where a row fits in a workgroup's registers.  Kernel times: 4096 x 32768 bf16 112 us (0.54 GB,
// 4.8 TB/s, the rate of a plain copy), the loss alone 49 us (5.4); 1021 x 50021 fp32 97 us (4.2; three of sixteen chunks of a thread are past the row's end); rows in parts: 4 x 131072 bf16
// 3.5 + 6.6 us, 512 x 262144 207 us (2.6, its logits are read twice).
#include "mlmc_worker.h"

namespace mlmc {

constexpr int DIS_TOP = MLMC_MAX_TEACHER;

struct DistillArgs {
    const void* s;
    int64_t lds, rows, vocab;
    int64_t row0;                 // first row of a launch of a workgroup a row
    const int32_t* t_idx;
    const float* t_val;
    int top;
    float temp, inv_temp, unit;   // unit = log2(e) / T: exp(x / T) = 2^(x unit)
    const float* dloss;
    float scale;
    float* loss;
    void* ds;
    int64_t ldds;
    int32_t* dev_status;
    // rows in parts
    int parts;
    int64_t part_len;             // entries of a part, a multiple of 8
    float2* stats;                // [rows][parts] greatest entry, sum of 2^((s - greatest) unit)
    float* gather;                // [rows][top] the logits at the teacher's indices
};

__global__ void k_distill_clear(int32_t* dev_status) { *dev_status = 0; }

constexpr int T_LIVE = 1, T_BAD = 2;

// The teacher's entries of a row into LDS (index -1: padding, also up to a multiple of four) and, with them, the logits at their places; a thread's greatest value and what it has seen.
template <int DT, int T> __device__ inline void teacher_load(const DistillArgs& a, int64_t row, int32_t* at, float* u, float* gather, const float* gathered, float& tmax, int& seen) {
    const entry_t<DT>* s = (const entry_t<DT>*)a.s + row * a.lds;
    tmax = -INFINITY;
    seen = 0;
    if (threadIdx.x < 3 && a.top + threadIdx.x < DIS_TOP) at[a.top + threadIdx.x] = -1;
    for (int k = threadIdx.x; k < a.top; k += T) {
        const int32_t i = a.t_idx[row * a.top + k];
        const float t = a.t_val[row * a.top + k];
        const bool here = i >= 0 && i < a.vocab;
        at[k] = here ? i : -1;
        u[k] = t;
        gather[k] = gathered ? gathered[k] : here ? to_f32(s[i]) : 0.f;
        if (i >= a.vocab) seen |= T_BAD;
        if (here) {
            if (t != -INFINITY) seen |= T_LIVE;   // a NaN too: it reaches the sum
            tmax = fmaxf(tmax, t);
        }
    }
}

// exp((t - greatest) / T) of the thread's entries, their sum; u becomes t - greatest.
template <int T> __device__ inline float teacher_sum(const DistillArgs& a, const int32_t* at, float* u, float tmax) {
    float sum = 0.f;
    for (int k = threadIdx.x; k < a.top; k += T) {
        u[k] -= tmax;
        if (at[k] >= 0) sum += expf(u[k] * a.inv_temp);
    }
    return sum;
}

// The thread's part of sum_k q_k T (log q_k - log p_{i_k}), the loss over T; u becomes q.  With T inside the logarithms nothing is divided by it, and its square, which small ones do not
// have in fp32, is not needed.
template <int T> __device__ inline float teacher_loss(const DistillArgs& a, const int32_t* at, float* u, const float* gather, float qsum, float m, float psum) {
    const float logs = a.temp * (logf(psum) - logf(qsum));
    float l = 0.f;
    for (int k = threadIdx.x; k < a.top; k += T) {
        const float v = u[k], q = at[k] >= 0 ? expf(v * a.inv_temp) / qsum : 0.f;
        u[k] = q;
        if (q != 0.f) l += q * ((v - (gather[k] - m)) + logs);
    }
    return l;
}

// The gradient at the teacher's indices in [first, last), over what the dense pass has written there.  An index may be there twice: each of its threads writes
// the same sum.
template <int DT, int T> __device__ inline void teacher_gradient(const DistillArgs& a, entry_t<DT>* ds, const int32_t* at, const float* q, const float* gather, float m, float coef, float c,
                                                                int64_t first, int64_t last) {
    for (int k = threadIdx.x; k < a.top; k += T) {
        const int32_t i = at[k];
        if (i < first || i >= last) continue;
        float qs = 0.f;
        for (int o = 0; o < a.top; o += 4) {   // padded with -1 to fours
            const int4 w = *(const int4*)(at + o);
            const float4 v = *(const float4*)(q + o);
            qs += w.x == i ? v.x : 0.f;
            qs += w.y == i ? v.y : 0.f;
            qs += w.z == i ? v.z : 0.f;
            qs += w.w == i ? v.w : 0.f;
        }
        ds[i] = from_f32<DT>(fmaf(power(gather[k] - m, a.unit), coef, -c * qs));
    }
}

// ---- a row that fits in the registers of T threads, N chunks of 16 bytes each -------------------------------------------
// It is read once and its gradient written once.  Two exponentials an entry: keeping the first would take twice the registers of 16-bit entries.  Several
// workgroups share a CU, so that one loads or stores while another computes.
template <int DT, int T, int N> __global__ __launch_bounds__(T, N <= 8 ? 8 : 4) void k_distill_row(DistillArgs a) {
    constexpr int E = DT == MLMC_BF16 ? 8 : 4, W = T / 64;
    __shared__ __align__(16) float q[DIS_TOP], gather[DIS_TOP];
    __shared__ __align__(16) int32_t at[DIS_TOP];
    __shared__ float part[5][W];
    __shared__ int flags[W];
    const int64_t row = a.row0 + blockIdx.x;
    const int wave = threadIdx.x >> 6, V = (int)a.vocab, lane_col = threadIdx.x * E;
    const bool first_lane = (threadIdx.x & 63) == 0;
    const entry_t<DT>* s = (const entry_t<DT>*)a.s + row * a.lds;
    entry_t<DT>* ds = a.ds ? (entry_t<DT>*)a.ds + row * a.ldds : nullptr;
    constexpr float none = -INFINITY;
    chunk_t v[N];
#pragma unroll
    for (int n = 0; n < N; ++n)
        if (n * T * E < V) v[n] = load_chunk<DT>(s, lane_col + n * T * E, V);
    float tmax, m = none, f[E];
    int seen;
    teacher_load<DT, T>(a, row, at, q, gather, nullptr, tmax, seen);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n * T * E >= V) continue;
        chunk_floats<DT>(f, v[n]);
#pragma unroll
        for (int e = 0; e < E; ++e) m = fmaxf(m, f[e]);
    }
    m = wave_max(m);
    tmax = wave_max(tmax);
    const uint64_t live = __ballot(seen & T_LIVE), wrong = __ballot(seen & T_BAD);
    if (first_lane) {
        part[0][wave] = m;
        part[1][wave] = tmax;
        flags[wave] = (live ? T_LIVE : 0) | (wrong ? T_BAD : 0);
    }
    __syncthreads();
    seen = 0;
#pragma unroll 4
    for (int w = 0; w < W; ++w) {
        m = fmaxf(m, part[0][w]);
        tmax = fmaxf(tmax, part[1][w]);
        seen |= flags[w];
    }
    const bool bad = seen & T_BAD, masked = !(seen & T_LIVE);
    const float weight = a.dloss ? a.dloss[row] * a.scale : a.scale;
    if (bad || masked) {
        if (threadIdx.x == 0) {
            a.loss[row] = bad ? __builtin_nanf("") : 0.f;
            if (bad && a.dev_status) atomicOr(a.dev_status, MLMC_DEV_RANGE);
        }
    } else {
        float sum = 0.f, qsum = teacher_sum<T>(a, at, q, tmax);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (n * T * E >= V) continue;
            chunk_floats<DT>(f, v[n]);
#pragma unroll
            for (int e = 0; e < E; ++e) sum += power(f[e] - m, a.unit);
        }
        sum = wave_sum(sum);
        qsum = wave_sum(qsum);
        if (first_lane) {
            part[2][wave] = sum;
            part[3][wave] = qsum;
        }
        __syncthreads();
        sum = qsum = 0.f;
#pragma unroll 4
        for (int w = 0; w < W; ++w) {
            sum += part[2][w];
            qsum += part[3][w];
        }
        const float l = wave_sum(teacher_loss<T>(a, at, q, gather, qsum, m, sum));
        if (first_lane) part[4][wave] = l;
        const bool zero = weight == 0.f;
        const float c = a.temp * weight, coef = c / sum;
        if (ds && !zero) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (n * T * E >= V) continue;
                chunk_floats<DT>(f, v[n]);
#pragma unroll
                for (int e = 0; e < E; ++e) f[e] = power(f[e] - m, a.unit) * coef;
                if (lane_col + n * T * E < V) store_chunk<DT>(ds, lane_col + n * T * E, V, f);
            }
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            float loss = 0.f;
#pragma unroll 4
            for (int w = 0; w < W; ++w) loss += part[4][w];
            a.loss[row] = a.temp * loss;
        }
        if (ds && !zero) teacher_gradient<DT, T>(a, ds, at, q, gather, m, coef, c, 0, V);
        if (!zero) return;
    }
    if (!ds) return;
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = 0.f;
    for (int col = lane_col; col < V; col += T * E) store_chunk<DT>(ds, col, V, f);
}

// ---- rows in parts: few rows, each spread over many workgroups, and rows that are too long for one --------------------------
// k_distill_stats leaves every part's greatest entry and sum, k_distill_finish joins them (each workgroup by itself, in the order of the parts) and reads the part again, out of
// the caches: the rows of a launch are as many as those hold.
constexpr int PART_T = 256;

template <int DT> __global__ __launch_bounds__(PART_T) void k_distill_stats(DistillArgs a, int64_t row0) {
    constexpr int E = DT == MLMC_BF16 ? 8 : 4, U = 4;
    __shared__ float2 each[PART_T / 64];
    const int64_t row = row0 + blockIdx.y, first = (int64_t)blockIdx.x * a.part_len, last = min(a.vocab, first + a.part_len);
    const entry_t<DT>* s = (const entry_t<DT>*)a.s + row * a.lds;
    float m = -INFINITY, sum = 0.f, f[E];
    for (int64_t col = first + threadIdx.x * E; col < last; col += PART_T * E * U) {
        chunk_t v[U];
        float big = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (col + u * PART_T * E < last) v[u] = load_chunk<DT>(s, col + u * PART_T * E, last);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (col + u * PART_T * E < last) {
                chunk_floats<DT>(f, v[u]);
#pragma unroll
                for (int e = 0; e < E; ++e) big = fmaxf(big, f[e]);
            }
        if (big > m) {
            sum *= power(m - big, a.unit);   // the first time 0 times 0
            m = big;
        }
        const float from = m == -INFINITY ? 0.f : m;   // nothing but -Inf so far: they add nothing
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (col + u * PART_T * E < last) {
                chunk_floats<DT>(f, v[u]);
#pragma unroll
                for (int e = 0; e < E; ++e) sum += power(f[e] - from, a.unit);
            }
    }
    const float top = wave_max(m);
    sum = wave_sum(m == -INFINITY ? sum : sum * power(m - top, a.unit));   // (a lane of -Inf has 0, or the NaN that it met)
    if ((threadIdx.x & 63) == 0) each[threadIdx.x >> 6] = make_float2(top, sum);
    __syncthreads();
    if (threadIdx.x == 0) {
        float g = -INFINITY, t = 0.f;
#pragma unroll
        for (int w = 0; w < PART_T / 64; ++w) g = fmaxf(g, each[w].x);
#pragma unroll
        for (int w = 0; w < PART_T / 64; ++w) t += each[w].x == -INFINITY ? each[w].y : each[w].y * power(each[w].x - g, a.unit);
        a.stats[row * a.parts + blockIdx.x] = make_float2(g, t);
    }
    if (blockIdx.x == 0)   // before the gradient takes the logits' place
        for (int k = threadIdx.x; k < a.top; k += PART_T) {
            const int32_t i = a.t_idx[row * a.top + k];
            a.gather[row * a.top + k] = i >= 0 && i < a.vocab ? to_f32(s[i]) : 0.f;
        }
}

template <int DT> __global__ __launch_bounds__(PART_T) void k_distill_finish(DistillArgs a, int64_t row0) {
    constexpr int E = DT == MLMC_BF16 ? 8 : 4, W = PART_T / 64;
    __shared__ __align__(16) float q[DIS_TOP], gather[DIS_TOP];
    __shared__ float part[5][W];
    __shared__ __align__(16) int32_t at[DIS_TOP];
    __shared__ int flags[W];
    const int64_t row = row0 + blockIdx.y, first = (int64_t)blockIdx.x * a.part_len, last = min(a.vocab, first + a.part_len);
    const int wave = threadIdx.x >> 6;
    const bool first_lane = (threadIdx.x & 63) == 0;
    const entry_t<DT>* s = (const entry_t<DT>*)a.s + row * a.lds;
    entry_t<DT>* ds = a.ds ? (entry_t<DT>*)a.ds + row * a.ldds : nullptr;
    float tmax, m = -INFINITY, f[E];
    int seen;
    teacher_load<DT, PART_T>(a, row, at, q, gather, a.gather + row * a.top, tmax, seen);
    for (int p = threadIdx.x; p < a.parts; p += PART_T) m = fmaxf(m, a.stats[row * a.parts + p].x);
    m = wave_max(m);
    tmax = wave_max(tmax);
    const uint64_t live = __ballot(seen & T_LIVE), wrong = __ballot(seen & T_BAD);
    if (first_lane) {
        part[0][wave] = m;
        part[1][wave] = tmax;
        flags[wave] = (live ? T_LIVE : 0) | (wrong ? T_BAD : 0);
    }
    __syncthreads();
    seen = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        m = fmaxf(m, part[0][w]);
        tmax = fmaxf(tmax, part[1][w]);
        seen |= flags[w];
    }
    const bool bad = seen & T_BAD, masked = !(seen & T_LIVE);
    const float weight = a.dloss ? a.dloss[row] * a.scale : a.scale;
    bool zero = true;
    if (bad || masked) {
        if (threadIdx.x == 0 && blockIdx.x == 0) {
            a.loss[row] = bad ? __builtin_nanf("") : 0.f;
            if (bad && a.dev_status) atomicOr(a.dev_status, MLMC_DEV_RANGE);
        }
    } else {
        float sum = 0.f, qsum = wave_sum(teacher_sum<PART_T>(a, at, q, tmax));
        for (int p = threadIdx.x; p < a.parts; p += PART_T) {
            const float2 v = a.stats[row * a.parts + p];
            sum += v.x == -INFINITY && m != -INFINITY ? v.y : v.y * power(v.x - m, a.unit);   // nothing but -Inf in the whole row: NaN
        }
        sum = wave_sum(sum);
        if (first_lane) {
            part[2][wave] = sum;
            part[3][wave] = qsum;
        }
        __syncthreads();
        sum = qsum = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            sum += part[2][w];
            qsum += part[3][w];
        }
        const float l = wave_sum(teacher_loss<PART_T>(a, at, q, gather, qsum, m, sum));
        if (first_lane) part[4][wave] = l;
        zero = weight == 0.f;
        const float c = a.temp * weight, coef = c / sum;
        if (ds && !zero) {
#pragma unroll 4
            for (int64_t col = first + threadIdx.x * E; col < last; col += PART_T * E) {
                chunk_floats<DT>(f, load_chunk<DT>(s, col, last));
#pragma unroll
                for (int e = 0; e < E; ++e) f[e] = power(f[e] - m, a.unit) * coef;
                store_chunk<DT>(ds, col, last, f);
            }
        }
        __syncthreads();
        if (threadIdx.x == 0 && blockIdx.x == 0) {
            float loss = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) loss += part[4][w];
            a.loss[row] = a.temp * loss;
        }
        if (ds && !zero) teacher_gradient<DT, PART_T>(a, ds, at, q, gather, m, coef, c, first, last);
    }
    if (!ds || !zero) return;
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = 0.f;
    for (int64_t col = first + threadIdx.x * E; col < last; col += PART_T * E) store_chunk<DT>(ds, col, last, f);
}

// Parts of a row: none (1) where a row fits in a workgroup's registers and there are rows enough for the CUs; else as many as fill the chip twice, of at least 8192 entries.
constexpr int64_t ROWS_MANY = 128, PART_MIN = 8192, GROUP_BYTES = (int64_t)96 << 20;
static int64_t row_capacity(int dtype) { return dtype == MLMC_BF16 ? 131072 : 65536; }
struct DistillPlan { int64_t rows; int parts; };   // rows of a launch; parts 0: a workgroup per row
static DistillPlan distill_plan(int64_t rows, int64_t vocab, int dtype) {
    if (vocab <= row_capacity(dtype) && (rows >= ROWS_MANY || vocab <= PART_MIN)) return {rows, 0};
    const int64_t fit = GROUP_BYTES / (vocab * (dtype == MLMC_BF16 ? 2 : 4)), group = rows < fit ? rows : fit > 1 ? fit : 1;
    const int64_t want = (512 + group - 1) / group, most = (vocab + PART_MIN - 1) / PART_MIN;
    return {group < 65535 ? group : 65535, (int)(want < most ? want : most)};
}

}  // namespace mlmc

using namespace mlmc;

template <int DT, int T, int N> static mlmc_status distill_rows(DistillArgs& a, hipStream_t st) {
    constexpr int64_t slice = LAUNCH_THREADS / T;
    for (; a.row0 < a.rows; a.row0 += slice) {
        const unsigned rows = (unsigned)(a.rows - a.row0 < slice ? a.rows - a.row0 : slice);
        MLMC_LAUNCH(K_DISTILL, st, (k_distill_row<DT, T, N><<<rows, T, 0, st>>>(a)));
    }
    return MLMC_OK;
}
template <int DT> static mlmc_status distill_run(DistillArgs& a, const DistillPlan& p, hipStream_t st) {
    constexpr int64_t E = DT == MLMC_BF16 ? 8 : 4;
    if (p.parts == 0) {
        if (a.vocab <= 256 * 4 * E) return distill_rows<DT, 256, 4>(a, st);
        if (a.vocab <= 512 * 8 * E) return distill_rows<DT, 512, 8>(a, st);
        if (a.vocab <= 1024 * 8 * E) return distill_rows<DT, 1024, 8>(a, st);
        return distill_rows<DT, 1024, 16>(a, st);
    }
    a.part_len = ((a.vocab + p.parts - 1) / p.parts + 7) / 8 * 8;
    a.parts = (int)((a.vocab + a.part_len - 1) / a.part_len);
    for (int64_t row = 0; row < a.rows; row += p.rows) {
        const dim3 grid((unsigned)a.parts, (unsigned)(a.rows - row < p.rows ? a.rows - row : p.rows));
        MLMC_LAUNCH(K_DISTILL_STATS, st, (k_distill_stats<DT><<<grid, PART_T, 0, st>>>(a, row)));
        MLMC_LAUNCH(K_DISTILL, st, (k_distill_finish<DT><<<grid, PART_T, 0, st>>>(a, row)));
    }
    return MLMC_OK;
}

extern "C" {

size_t mlmc_distill_workspace(int64_t rows, int64_t vocab, int top) {
    if (rows <= 0 || rows >= ((int64_t)1 << 31) || vocab < 1 || vocab >= ((int64_t)1 << 31) || top < 1 || top > MLMC_MAX_TEACHER) return 0;
    int parts = 0;
    for (int dtype : {MLMC_F32, MLMC_BF16}) {
        const int p = distill_plan(rows, vocab, dtype).parts;
        parts = p > parts ? p : parts;
    }
    return parts ? (size_t)rows * (parts * sizeof(float2) + top * sizeof(float)) : 0;
}

mlmc_status mlmc_distill(const void* logits, int64_t ldl, int64_t rows, int64_t vocab, int dtype, const int32_t* t_idx, const float* t_val, int top,
                         float temperature, const float* dloss, float scale, float* loss, void* dlogits, int64_t ldd, int32_t* dev_status,
                         void* ws, size_t ws_bytes, void* hip_stream) {
    if (rows < 0 || rows >= ((int64_t)1 << 31) || vocab < 1 || vocab >= ((int64_t)1 << 31) || !entry_dtype_ok(dtype) || top < 1 || top > MLMC_MAX_TEACHER) return MLMC_EINVAL;
    if (!(temperature > 0.0f) || temperature > 3.402823e38f || !(1.4426950408889634f / temperature <= 3.402823e38f) || ldl < vocab || (dlogits && ldd < vocab)) return MLMC_EINVAL;
    hipStream_t st = (hipStream_t)hip_stream;
    if (!f32_ptr_ok(dev_status)) return MLMC_EINVAL;
    if (rows > 0) {
        if (!entry_ptr_ok(logits, dtype) || !t_idx || !f32_ptr_ok(t_idx) || !t_val || !f32_ptr_ok(t_val) || !f32_ptr_ok(dloss) || !loss || !f32_ptr_ok(loss)) return MLMC_EINVAL;
        if (dlogits && !entry_ptr_ok(dlogits, dtype)) return MLMC_EINVAL;
    }
    const DistillPlan p = rows > 0 ? distill_plan(rows, vocab, dtype) : DistillPlan{0, 0};
    const size_t need = p.parts ? (size_t)rows * (p.parts * sizeof(float2) + top * sizeof(float)) : 0;
    if (need && (!ws || (uintptr_t)ws % 256 || ws_bytes < need)) return MLMC_EINVAL;
    if (dev_status) MLMC_LAUNCH(K_ZERO, st, (k_distill_clear<<<1, 1, 0, st>>>(dev_status)));
    if (rows == 0) return MLMC_OK;
    DistillArgs a = {};
    a.s = logits; a.lds = ldl; a.rows = rows; a.vocab = vocab; a.t_idx = t_idx; a.t_val = t_val; a.top = top; a.temp = temperature;
    a.inv_temp = 1.0f / temperature; a.dloss = dloss; a.scale = scale; a.loss = loss; a.ds = dlogits; a.ldds = ldd; a.dev_status = dev_status;
    a.unit = 1.4426950408889634f / temperature;
    a.stats = (float2*)ws;
    a.gather = (float*)ws + 2 * rows * p.parts;
    return dtype == MLMC_F32 ? distill_run<MLMC_F32>(a, p, st) : distill_run<MLMC_BF16>(a, p, st);
}

}  // extern "C"
