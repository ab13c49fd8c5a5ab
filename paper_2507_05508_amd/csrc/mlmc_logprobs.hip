// Log probabilities of given tokens, entropy and the top alternatives of every row of logits, and their gradient (entry points mlmc_token_logprobs,
// mlmc_token_logprobs_backward).
//
// With T the temperature, m the row's greatest logit and S = sum_j exp((s_j - m) / T):
//   log p_j = (s_j - m) / T - log S,   H = -sum_j p_j log p_j = log S - (1 / S) sum_j exp((s_j - m) / T) (s_j - m) / T
//   d/ds_j of sum_k g_k log p_{i_k} + h H:   ( sum of the g_k with i_k = j  -  p_j sum_k g_k  -  h p_j (log p_j + H) ) / T
// The alternatives are in order of (logit, lowest index first).
//
// The top K without a sort of the row: the row's threads form 256 groups, whose greatest entries are known from the maximum.  The K-th greatest of those is a bound that K entries reach, and
// few more do (of 131072 independent entries 73 for K = 64, 177 for K = 128: those of which the K-th lies in a group of its own).  They are gathered in LDS and each counts how many are
// before it.  Where ties or an order of the row bring more than the room for them, two bisections find the K-th greatest value and the index where its equals run out.
//
// Bound by memory: the logits are read once.
#include "mlmc_worker.h"

namespace mlmc {

constexpr int MOST_ANSWERS = MLMC_MAX_ANSWERS, ROOM = 1024, GROUPS = 256, PARTS_MAX = 32;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct LogprobArgs {
    const void* s;
    int64_t lds, rows, vocab;
    int64_t row0;                 // first row of a launch
    const int32_t* tokens;
    int given, top;
    float inv_temp, unit;         // 1 / T, log2(e) / T
    float *logprob, *entropy;
    int32_t* top_idx;
    float *top_logprob, *stats;
    int32_t* dev_status;
    int parts;                    // of a row, 1: a workgroup has the whole row and its answers
    int64_t part_len;
    float4* part_stats;           // [rows][parts] greatest entry, sum, sum of e log2 e
    uint64_t* part_top;           // [rows][parts][top] keys in descending order, 0 behind the last
};

// Logits as numbers of the same order, -0 as 0.
__device__ inline uint32_t ordered(float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ inline float unordered(uint32_t k) { return __builtin_bit_cast(float, k >> 31 ? k & 0x7fffffffu : ~k); }
__device__ inline uint64_t key_of(float v, uint32_t index) { return (uint64_t)ordered(v) << 32 | (uint32_t)~index; }
__device__ inline uint32_t key_index(uint64_t key) { return ~(uint32_t)key; }
__device__ inline float key_value(uint64_t key) { return unordered((uint32_t)(key >> 32)); }
constexpr float LOWEST = -3.402823466e38f;

// What a row (or all its parts) comes to.
struct RowSums {
    float m, log_s, h;
    bool bad;
    __device__ RowSums(float m_, float s, float a) : m(m_) {
        bad = !(fabsf(m) <= 3.402823466e38f) || s != s;   // NaN or +Inf among the logits, or nothing but -Inf
        log_s = bad ? __builtin_nanf("") : logf(s);
        h = fmaf(-LN2, a / s, log_s);                     // NaN with log_s
    }
    __device__ float log_p(float v, float inv_temp) const { return (v - m) * inv_temp - log_s; }
};

template <int T> __device__ inline void write_given(const LogprobArgs& a, int64_t row, int32_t token, float logit, const RowSums& r) {
    if ((int)threadIdx.x < a.given) {
        const bool out = token >= a.vocab;
        a.logprob[row * a.given + threadIdx.x] = token < 0 ? 0.f : out ? __builtin_nanf("") : r.log_p(logit, a.inv_temp);
        if (out && a.dev_status) atomicOr(a.dev_status, MLMC_DEV_RANGE);
    }
    if (threadIdx.x == 0) {
        if (a.entropy) a.entropy[row] = r.h;
        if (a.stats) {
            a.stats[3 * row] = r.m;
            a.stats[3 * row + 1] = r.log_s;
            a.stats[3 * row + 2] = r.h;
        }
    }
}
// alternative i of the row; key 0: there is none
__device__ inline void write_top(const LogprobArgs& a, int64_t row, int i, uint64_t key, const RowSums& r) {
    a.top_idx[row * a.top + i] = r.bad || !key ? -1 : (int32_t)key_index(key);
    a.top_logprob[row * a.top + i] = r.bad ? __builtin_nanf("") : key ? r.log_p(key_value(key), a.inv_temp) : -INFINITY;
}

// A row, or a part of one, in the registers of T threads, N chunks of 16 bytes each.
template <int DT, int T, int N, bool TOP> __global__ __launch_bounds__(T, N <= 8 ? 8 : 4) void k_logprobs(LogprobArgs a) {
    constexpr int E = DT == MLMC_BF16 ? 8 : 4, W = T / 64;
    constexpr float none = -INFINITY;
    __shared__ float part[3][W];
    __shared__ __align__(16) float greatest[TOP ? GROUPS : 1];
    __shared__ uint64_t found[TOP ? ROOM : 1], best[TOP ? MOST_ANSWERS : 1];
    __shared__ float bound;
    __shared__ int number, counts[W];
    const int64_t row = a.row0 + blockIdx.y, first = (int64_t)blockIdx.x * a.part_len;
    const int len = (int)min(a.part_len, a.vocab - first), wave = threadIdx.x >> 6, lane = threadIdx.x & 63, lane_col = threadIdx.x * E;
    const entry_t<DT>* s = (const entry_t<DT>*)a.s + row * a.lds + first;
    chunk_t v[N];
#pragma unroll
    for (int n = 0; n < N; ++n)
        if (n * T * E < len) v[n] = load_chunk<DT>(s, lane_col + n * T * E, len);
    int32_t token = -1;
    float logit = 0.f;
    if (a.parts == 1 && (int)threadIdx.x < a.given) {
        token = a.tokens[row * a.given + threadIdx.x];
        if (token >= 0 && token < a.vocab) logit = to_f32(s[token]);
    }
    float f[E], mine = none;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n * T * E >= len) continue;
        chunk_floats<DT>(f, v[n]);
#pragma unroll
        for (int e = 0; e < E; ++e) mine = fmaxf(mine, f[e]);
    }
    if (TOP) {
        float g = mine;
        if (T >= 512) g = fmaxf(g, dpp<0xB1, 0xF>(g, g));    // lanes 2k and 2k + 1
        if (T >= 1024) g = fmaxf(g, dpp<0x4E, 0xF>(g, g));   // fours
        if (threadIdx.x % (T / GROUPS) == 0) greatest[threadIdx.x / (T / GROUPS)] = g;
        if (threadIdx.x == 0) number = 0;
    }
    float m = wave_max(mine);
    if (lane == 0) part[0][wave] = m;
    __syncthreads();
#pragma unroll 4
    for (int w = 0; w < W; ++w) m = fmaxf(m, part[0][w]);
    const float from = m == none ? 0.f : m;
    float sum = 0.f, elog = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n * T * E >= len) continue;
        chunk_floats<DT>(f, v[n]);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float t = (f[e] - from) * a.unit, x = __builtin_amdgcn_exp2f(t);
            sum += x;
            elog = fmaf(x, fmaxf(t, -1024.f), elog);   // x is 0 below that
        }
    }
    sum = wave_sum(sum);
    elog = wave_sum(elog);
    if (lane == 0) {
        part[1][wave] = sum;
        part[2][wave] = elog;
    }
    if (TOP && wave == 0) {   // the greatest number of 16 bits that `top` groups reach
        const float4 g = ((const float4*)greatest)[lane];
        const uint32_t k[4] = {ordered(g.x) >> 16, ordered(g.y) >> 16, ordered(g.z) >> 16, ordered(g.w) >> 16};
        uint32_t at = 0;
#pragma unroll 1
        for (int b = 15; b >= 0; --b) {
            const uint32_t c = at | 1u << b;
            int n = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) n += __popcll(__ballot(k[i] >= c));
            if (n >= a.top) at = c;
        }
        if (lane == 0) bound = at <= ordered(none) >> 16 ? LOWEST : unordered(at << 16);   // never -Inf: that is no alternative
    }
    __syncthreads();
    sum = elog = 0.f;
#pragma unroll 4
    for (int w = 0; w < W; ++w) {
        sum += part[1][w];
        elog += part[2][w];
    }
    int n_top = 0;
    if constexpr (TOP) {
        const float least = bound;
        // entries that `take` has, into `found`, in any order
        const auto gather = [&](auto take) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (n * T * E >= len) continue;
                chunk_floats<DT>(f, v[n]);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int col = lane_col + n * T * E + e;
                    if (take(f[e], col)) {
                        const int at = atomicAdd(&number, 1);
                        if (at < ROOM) found[at] = key_of(f[e], (uint32_t)(first + col));
                    }
                }
            }
        };
        if (mine >= least) gather([&](float x, int) { return x >= least; });
        __syncthreads();
        int n = number;
        if (n > ROOM) {
            // how many entries of the workgroup `take` has
            const auto count = [&](auto take) {
                int c = 0;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    if (n * T * E >= len) continue;
                    chunk_floats<DT>(f, v[n]);
#pragma unroll
                    for (int e = 0; e < E; ++e) c += __popcll(__ballot(take(f[e], lane_col + n * T * E + e)));
                }
                __syncthreads();
                if (lane == 0) counts[wave] = c;
                __syncthreads();
                c = 0;
                for (int w = 0; w < W; ++w) c += counts[w];
                return c;
            };
            uint32_t at = ordered(least), up = ordered(m);   // `top` entries reach at; the K-th greatest lies in [at, up]
            while (at < up) {
                const uint32_t mid = at + (up - at + 1) / 2;
                if (count([&](float x, int) { return x >= unordered(mid); }) >= a.top) at = mid;
                else up = mid - 1;
            }
            const float kth = unordered(at);
            const int left = a.top - count([&](float x, int) { return x > kth; });
            int lo = 0, hi = len - 1;   // the index up to which `left` entries are equal to it
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (count([&](float x, int col) { return x == kth && col <= mid; }) >= left) hi = mid;
                else lo = mid + 1;
            }
            __syncthreads();
            if (threadIdx.x == 0) number = 0;
            __syncthreads();
            gather([&](float x, int col) { return x > kth || (x == kth && col <= lo); });
            __syncthreads();
            n = number;   // `top` of them
        }
        for (int i = threadIdx.x; i < n; i += T) {
            const uint64_t key = found[i];
            int before = 0;
#pragma unroll 8
            for (int o = 0; o < n; ++o) before += found[o] > key;
            if (before < a.top) best[before] = key;
        }
        __syncthreads();
        n_top = min(n, a.top);
    }
    if (a.parts > 1) {
        const int64_t at = row * a.parts + blockIdx.x;
        if (threadIdx.x == 0) a.part_stats[at] = make_float4(m, sum, elog, 0.f);
        if constexpr (TOP)
            for (int i = threadIdx.x; i < a.top; i += T) a.part_top[at * a.top + i] = i < n_top ? best[i] : 0;
        return;
    }
    const RowSums r(m, sum, elog);
    write_given<T>(a, row, token, logit, r);
    if constexpr (TOP)
        for (int i = threadIdx.x; i < a.top; i += T) write_top(a, row, i, i < n_top ? best[i] : 0, r);
}

// The parts of a row: their sums scaled to the greatest maximum, in their order, and their lists, each of which says by bisection how many of its entries are before one of another.
constexpr int JOIN_T = 256;
__global__ __launch_bounds__(JOIN_T) void k_logprobs_join(LogprobArgs a, int dtype) {
    extern __shared__ uint64_t list[];   // [parts][top]
    __shared__ int number;
    const int64_t row = a.row0 + blockIdx.x;
    const int lane = threadIdx.x & 63, all = a.parts * a.top;
    int32_t token = -1;
    float logit = 0.f;
    if ((int)threadIdx.x < a.given) {
        token = a.tokens[row * a.given + threadIdx.x];
        if (token >= 0 && token < a.vocab) logit = dtype == MLMC_F32 ? ((const float*)a.s)[row * a.lds + token] : to_f32(((const __bf16*)a.s)[row * a.lds + token]);
    }
    const float4 p = lane < a.parts ? a.part_stats[row * a.parts + lane] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
    if (threadIdx.x == 0) number = 0;
    const uint64_t* from = a.part_top + row * all;
    for (int i = threadIdx.x; i < all; i += JOIN_T) list[i] = from[i];
    const float m = wave_max(p.x), t = p.x == -INFINITY ? -1024.f : fmaxf((p.x - m) * a.unit, -1024.f), w = __builtin_amdgcn_exp2f(t);
    const RowSums r(m, wave_sum(p.y * w), wave_sum(w * fmaf(p.y, t, p.z)));
    write_given<JOIN_T>(a, row, token, logit, r);
    if (a.top == 0) return;
    __syncthreads();
    for (int i = threadIdx.x; i < all; i += JOIN_T) {
        const uint64_t key = list[i];
        if (!key) continue;
        atomicAdd(&number, 1);
        const int own = i / a.top;
        int before = i - own * a.top;
        for (int q = 0; q < a.parts && before < a.top; ++q) {
            if (q == own) continue;
            int lo = 0, hi = a.top;   // entries of list q that are greater
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (list[q * a.top + mid] > key) lo = mid + 1;
                else hi = mid;
            }
            before += lo;
        }
        if (before < a.top) write_top(a, row, before, key, r);
    }
    __syncthreads();
    for (int i = number + threadIdx.x; i < a.top; i += JOIN_T) write_top(a, row, i, 0, r);
}

// ---- the gradient ---------------------------------------------------------------------------------------------------------------------

struct LogprobGradArgs {
    const void* s;
    int64_t lds, rows, vocab;
    int64_t row0;
    const float* stats;
    const int32_t *tokens, *top_idx;
    const float *dlogprob, *dtop, *dentropy;
    int given, top;
    float inv_temp, unit;
    void* ds;
    int64_t ldds;
};

// A workgroup has GRAD_T * GRAD_N chunks of a row: its logits are in registers before it writes any of their gradients, which may take their place.
constexpr int GRAD_T = 256, GRAD_N = 4;
template <int DT> __global__ __launch_bounds__(GRAD_T, 8) void k_logprobs_backward(LogprobGradArgs a) {
    constexpr int E = DT == MLMC_BF16 ? 8 : 4, LEN = GRAD_T * GRAD_N * E, MOST = 2 * MOST_ANSWERS;
    static_assert(MOST <= GRAD_T, "a thread for every token");
    __shared__ __align__(16) int32_t at[MOST];
    __shared__ __align__(16) float g[MOST];
    __shared__ float part[GRAD_T / 64];
    __shared__ int any[GRAD_T / 64];
    const int64_t row = a.row0 + blockIdx.y, first = (int64_t)blockIdx.x * LEN;
    const int len = (int)min((int64_t)LEN, a.vocab - first), k = threadIdx.x, lane_col = threadIdx.x * E;
    const entry_t<DT>* s = (const entry_t<DT>*)a.s + row * a.lds + first;
    entry_t<DT>* ds = (entry_t<DT>*)a.ds + row * a.ldds + first;
    chunk_t v[GRAD_N];
#pragma unroll
    for (int n = 0; n < GRAD_N; ++n)
        if (n * GRAD_T * E < len) v[n] = load_chunk<DT>(s, lane_col + n * GRAD_T * E, len);
    // the tokens of both lists, a thread each: place in this part, gradient, logit
    const int all = a.given + a.top, padded = (all + 3) / 4 * 4;
    int64_t place = -1;
    float weight = 0.f, logit = 0.f;
    if (k < a.given) {
        place = a.tokens[row * a.given + k];
        weight = a.dlogprob[row * a.given + k];
    } else if (k < all) {
        place = a.top_idx[row * a.top + k - a.given];
        weight = a.dtop[row * a.top + k - a.given];
    }
    if (place < 0 || place >= a.vocab) {   // padding, or no token of this vocabulary
        place = -1;
        weight = 0.f;
    }
    const bool inside = place >= first && place < first + len;
    const int col = (int)(place - first);
    if (inside) logit = to_f32(s[col]);
    if (k < padded) {
        at[k] = inside ? col : -1;
        g[k] = weight;
    }
    const float h = a.dentropy ? a.dentropy[row] : 0.f, m = a.stats[3 * row], log_s = a.stats[3 * row + 1], entropy = a.stats[3 * row + 2];
    const uint64_t live = __ballot(weight != 0.f);
    const float wave_total = wave_sum(weight);
    if ((k & 63) == 0) {
        part[k >> 6] = wave_total;
        any[k >> 6] = live != 0;
    }
    __syncthreads();
    float total = 0.f, f[E];
    bool zero = h == 0.f;
#pragma unroll
    for (int w = 0; w < GRAD_T / 64; ++w) {
        total += part[w];
        zero = zero && !any[w];
    }
    if (zero) {   // whatever the logits
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = 0.f;
#pragma unroll
        for (int n = 0; n < GRAD_N; ++n)
            if (lane_col + n * GRAD_T * E < len) store_chunk<DT>(ds, lane_col + n * GRAD_T * E, len, f);
        return;
    }
    const float inv_s = expf(-log_s), base = log_s - entropy, ca = -total * a.inv_temp, ch = -h * a.inv_temp;
    const auto dense = [&](float x) {
        const float d = x - m, p = power(d, a.unit) * inv_s;
        return p * fmaf(ch, fmaxf(fmaf(d, a.inv_temp, -base), -1024.f), ca);   // log p + H; p is 0 below that
    };
#pragma unroll
    for (int n = 0; n < GRAD_N; ++n) {
        if (n * GRAD_T * E >= len) continue;
        chunk_floats<DT>(f, v[n]);
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = dense(f[e]);
        if (lane_col + n * GRAD_T * E < len) store_chunk<DT>(ds, lane_col + n * GRAD_T * E, len, f);
    }
    __syncthreads();
    if (!inside || k >= all) return;
    float own = 0.f;   // a token may be there more than once: each of its threads writes the same sum
    for (int o = 0; o < padded; o += 4) {
        const int4 w = *(const int4*)(at + o);
        const float4 u = *(const float4*)(g + o);
        own += w.x == col ? u.x : 0.f;
        own += w.y == col ? u.y : 0.f;
        own += w.z == col ? u.z : 0.f;
        own += w.w == col ? u.w : 0.f;
    }
    ds[col] = from_f32<DT>(fmaf(own, a.inv_temp, dense(logit)));
}

// ---- plans ----------------------------------------------------------------------------------------------------------------------------

constexpr int64_t VOCAB_MAX = (int64_t)1 << 21;
// A row by one workgroup, or in parts: where rows are too few for the CUs, and where a row does not fit in a workgroup's registers.
struct LogprobPlan { int parts; int64_t part_len; };
static LogprobPlan logprob_plan(int64_t rows, int64_t vocab, int dtype) {
    const int64_t fit = dtype == MLMC_BF16 ? 65536 : 32768, least = 4096;
    int64_t parts = (vocab + fit - 1) / fit;
    const int64_t want = rows ? (512 + rows - 1) / rows : 1, most = (vocab + least - 1) / least;
    const int64_t fill = want < most ? want : most;
    parts = parts > fill ? parts : fill;
    parts = parts < PARTS_MAX ? parts : PARTS_MAX;
    const int64_t len = ((vocab + parts - 1) / parts + 7) / 8 * 8;
    return {(int)((vocab + len - 1) / len), len};
}
static size_t logprob_bytes(const LogprobPlan& p, int64_t rows, int top) {
    return p.parts > 1 ? (size_t)rows * p.parts * (sizeof(float4) + (size_t)top * sizeof(uint64_t)) : 0;
}
static bool logprob_sizes_ok(int64_t rows, int64_t vocab, int given, int top) {
    return rows >= 0 && rows < ((int64_t)1 << 31) && vocab >= 1 && vocab <= VOCAB_MAX && given >= 0 && given <= MOST_ANSWERS && top >= 0 && top <= MOST_ANSWERS;
}
static bool temperature_ok(float t) { return t > 0.0f && t <= 3.402823e38f && 1.4426950408889634f / t <= 3.402823e38f; }
constexpr int64_t ROW_SLICE = 32768;   // rows of a launch: they are the grid's second axis

template <int DT, int T, int N> static mlmc_status logprob_launch(const LogprobArgs& a, dim3 grid, hipStream_t st) {
    if (a.top) MLMC_LAUNCH(K_LOGPROBS, st, (k_logprobs<DT, T, N, true><<<grid, T, 0, st>>>(a)));
    else MLMC_LAUNCH(K_LOGPROBS, st, (k_logprobs<DT, T, N, false><<<grid, T, 0, st>>>(a)));
    return MLMC_OK;
}
template <int DT> static mlmc_status logprob_run(LogprobArgs a, hipStream_t st) {
    constexpr int64_t E = DT == MLMC_BF16 ? 8 : 4;
    for (; a.row0 < a.rows; a.row0 += ROW_SLICE) {
        const unsigned rows = (unsigned)(a.rows - a.row0 < ROW_SLICE ? a.rows - a.row0 : ROW_SLICE);
        const dim3 grid((unsigned)a.parts, rows);
        const mlmc_status rc = a.part_len <= 256 * 4 * E   ? logprob_launch<DT, 256, 4>(a, grid, st)
                               : a.part_len <= 512 * 8 * E  ? logprob_launch<DT, 512, 8>(a, grid, st)
                               : a.part_len <= 1024 * 8 * E ? logprob_launch<DT, 1024, 8>(a, grid, st)
                                                            : logprob_launch<DT, 1024, 16>(a, grid, st);
        if (rc != MLMC_OK) return rc;
        if (a.parts > 1) MLMC_LAUNCH(K_LOGPROBS_JOIN, st, (k_logprobs_join<<<rows, JOIN_T, (size_t)a.parts * a.top * sizeof(uint64_t), st>>>(a, DT)));
    }
    return MLMC_OK;
}
template <int DT> static mlmc_status logprob_backward_run(LogprobGradArgs a, hipStream_t st) {
    constexpr int64_t LEN = GRAD_T * GRAD_N * (DT == MLMC_BF16 ? 8 : 4);
    for (; a.row0 < a.rows; a.row0 += ROW_SLICE) {
        const dim3 grid((unsigned)((a.vocab + LEN - 1) / LEN), (unsigned)(a.rows - a.row0 < ROW_SLICE ? a.rows - a.row0 : ROW_SLICE));
        MLMC_LAUNCH(K_LOGPROBS_BACKWARD, st, (k_logprobs_backward<DT><<<grid, GRAD_T, 0, st>>>(a)));
    }
    return MLMC_OK;
}
static __global__ void k_logprobs_clear(int32_t* dev_status) { *dev_status = 0; }

}  // namespace mlmc

using namespace mlmc;

extern "C" {

size_t mlmc_token_logprobs_workspace(int64_t rows, int64_t vocab, int top) {
    if (!logprob_sizes_ok(rows, vocab, 0, top) || rows == 0) return 0;
    const size_t a = logprob_bytes(logprob_plan(rows, vocab, MLMC_F32), rows, top), b = logprob_bytes(logprob_plan(rows, vocab, MLMC_BF16), rows, top);
    return a > b ? a : b;
}

mlmc_status mlmc_token_logprobs(const void* logits, int64_t ldl, int64_t rows, int64_t vocab, int dtype, const int32_t* tokens, int given, int top, float temperature,
                                float* logprob, float* entropy, int32_t* top_idx, float* top_logprob, float* stats, int32_t* dev_status, void* ws, size_t ws_bytes,
                                void* hip_stream) {
    if (!logprob_sizes_ok(rows, vocab, given, top) || !entry_dtype_ok(dtype) || !temperature_ok(temperature) || ldl < vocab) return MLMC_EINVAL;
    hipStream_t st = (hipStream_t)hip_stream;
    if (!f32_ptr_ok(dev_status)) return MLMC_EINVAL;
    if (rows > 0) {
        if (!entry_ptr_ok(logits, dtype) || !f32_ptr_ok(entropy) || !f32_ptr_ok(stats)) return MLMC_EINVAL;
        if (given && (!tokens || !f32_ptr_ok(tokens) || !logprob || !f32_ptr_ok(logprob))) return MLMC_EINVAL;
        if (top && (!top_idx || !f32_ptr_ok(top_idx) || !top_logprob || !f32_ptr_ok(top_logprob))) return MLMC_EINVAL;
    }
    const LogprobPlan p = logprob_plan(rows, vocab, dtype);
    const size_t need = logprob_bytes(p, rows, top);
    if (need && (!ws || (uintptr_t)ws % 256 || ws_bytes < need)) return MLMC_EINVAL;
    if (dev_status) MLMC_LAUNCH(K_ZERO, st, (k_logprobs_clear<<<1, 1, 0, st>>>(dev_status)));
    if (rows == 0) return MLMC_OK;
    LogprobArgs a = {};
    a.s = logits; a.lds = ldl; a.rows = rows; a.vocab = vocab; a.tokens = tokens; a.given = given; a.top = top; a.inv_temp = 1.0f / temperature;
    a.unit = LOG2E / temperature; a.logprob = logprob; a.entropy = entropy; a.top_idx = top_idx; a.top_logprob = top_logprob; a.stats = stats; a.dev_status = dev_status;
    a.parts = p.parts; a.part_len = p.part_len; a.part_stats = (float4*)ws; a.part_top = (uint64_t*)((float4*)ws + rows * p.parts);
    return dtype == MLMC_F32 ? logprob_run<MLMC_F32>(a, st) : logprob_run<MLMC_BF16>(a, st);
}

mlmc_status mlmc_token_logprobs_backward(const void* logits, int64_t ldl, int64_t rows, int64_t vocab, int dtype, const float* stats, const int32_t* tokens, int given,
                                         const float* dlogprob, const int32_t* top_idx, int top, const float* dtop, const float* dentropy, float temperature, void* dlogits,
                                         int64_t ldd, void* hip_stream) {
    if (!logprob_sizes_ok(rows, vocab, given, top) || !entry_dtype_ok(dtype) || !temperature_ok(temperature) || ldl < vocab || ldd < vocab) return MLMC_EINVAL;
    if (rows == 0) return MLMC_OK;
    if (!entry_ptr_ok(logits, dtype) || !entry_ptr_ok(dlogits, dtype) || !stats || !f32_ptr_ok(stats) || !f32_ptr_ok(dentropy)) return MLMC_EINVAL;
    if (given && (!tokens || !f32_ptr_ok(tokens) || !dlogprob || !f32_ptr_ok(dlogprob))) return MLMC_EINVAL;
    if (top && (!top_idx || !f32_ptr_ok(top_idx) || !dtop || !f32_ptr_ok(dtop))) return MLMC_EINVAL;
    LogprobGradArgs a = {};
    a.s = logits; a.lds = ldl; a.rows = rows; a.vocab = vocab; a.stats = stats; a.tokens = tokens; a.given = given; a.dlogprob = dlogprob; a.top_idx = top_idx; a.top = top;
    a.dtop = dtop; a.dentropy = dentropy; a.inv_temp = 1.0f / temperature; a.unit = LOG2E / temperature; a.ds = dlogits; a.ldds = ldd;
    return dtype == MLMC_F32 ? logprob_backward_run<MLMC_F32>(a, (hipStream_t)hip_stream) : logprob_backward_run<MLMC_BF16>(a, (hipStream_t)hip_stream);
}

}  // extern "C"
