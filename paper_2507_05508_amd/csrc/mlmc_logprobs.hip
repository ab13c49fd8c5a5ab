// Log probabilities of given tokens, entropy and the top alternatives of every row of logits, and their gradient (entry points mlmc_token_logprobs,
// mlmc_token_logprobs_backward).
//
// With T the temperature, m the row's greatest logit and S = sum_j exp((s_j - m) / T):
//   log p_j = (s_j - m) / T - log S,   H = -sum_j p_j log p_j = log S - (1 / S) sum_j exp((s_j - m) / T) (s_j - m) / T
//   d/ds_j of sum_k g_k log p_{i_k} + h H:   ( sum of the g_k with i_k = j  -  p_j sum_k g_k  -  h p_j (log p_j + H) ) / T
// The alternatives are in order of (logit, lowest index first).
//
// Bound by memory: the logits are read once.  One launch of waves without barriers, each with a stretch of a row in its registers, leaves the stretch's maximum and sums and the greatest entry
// of every group of neighbouring entries; a wave a row then joins the sums and has the top K without a look at the whole row: K groups reach the K-th greatest of the groups' greatest entries, so
// that no entry below it is among the top K, and none of the groups that do not reach it holds one.  Those K groups are read again, of 1024 groups at most; a few more than K of their entries
// reach the bound (of 131072 independent entries 66 for K = 64), and each counts how many are before it.  Of equal entries the first K are enough; where an order of the row brings more than the
// room for them (a row in ascending order), those found so far are cut to the top K by bisection.
// The histogram ends 64 temperatures below the greatest logit: where the K-th alternative lies further down, all groups reach the bound, and a row takes a search by one wave instead.  Results are the
// same, the time is not (us, one logit raised by 20 over normal ones of deviation 2.5, T = 1 / 0.3 / 0.1, bf16): 4 x 131072 with 20 alternatives 12 / 12 / 90, 2048 x 131072 with 64 112 / 198 / 238,
// 512 x 32000 with 20 16 / 134 / 237, 2048 x 32000 39 / 104 / 143; without the raised logit only 2048 x 131072 with 64 at T = 0.1, 175.
// Shorter rows are held by one workgroup each (k_logprobs_short): its chunks are the groups, and one launch does all.
#include "mlmc_worker.h"

namespace mlmc {

constexpr int MOST_ANSWERS = MLMC_MAX_ANSWERS;
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
    int stretches;                // of a row, a wave each
    int groups, lanes;            // of a row, 0 without alternatives; lanes of a group, a power of two
    float* stretch_stats;         // [rows][stretches][3] greatest entry, sum, sum of e log2 e
    float* greatest;              // [rows][groups]
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

// (s - m) / T in the base of `unit`, m being at least s.  Differences below the range of fp32 are taken of halves, where the temperature may bring them back into it; where it is too small for
// that they are -Inf, as they have to be.  As many instructions as the difference.
struct Scaled {
    float half, m, unit;
    __device__ Scaled(float m_, float unit_) : half(m_ > 1e31f && unit_ < 1e38f ? 0.5f : 1.0f), m(m_ * half), unit(half == 1.0f ? unit_ : unit_ + unit_) {}
    __device__ float difference(float s) const { return fmaf(s, half, -m); }
    __device__ float operator()(float s) const { return difference(s) * unit; }
};

// What a row comes to.
struct RowSums {
    float m, log_s, h;
    bool bad;
    __device__ RowSums(float m_, float s, float a) : m(m_) {
        bad = !(fabsf(m) <= 3.402823466e38f) || s != s;   // NaN or +Inf among the logits, or nothing but -Inf
        log_s = bad ? __builtin_nanf("") : logf(s);
        h = fmaf(-LN2, a / s, log_s);                     // NaN with log_s
    }
    __device__ float log_p(float v, float inv_temp) const { return Scaled(m, inv_temp)(v) - log_s; }
};

// alternative i of the row; key 0: there is none
__device__ inline void write_top(const LogprobArgs& a, int64_t row, int i, uint64_t key, const RowSums& r) {
    a.top_idx[row * a.top + i] = r.bad || !key ? -1 : (int32_t)key_index(key);
    a.top_logprob[row * a.top + i] = r.bad ? __builtin_nanf("") : key ? r.log_p(key_value(key), a.inv_temp) : -INFINITY;
}

// ---- stretches --------------------------------------------------------------------------------------------------------------------------

constexpr int STRETCH_N = 4, STRETCH_WG = 256;
template <int DT> constexpr int STRETCH = 64 * STRETCH_N * ENTRIES<DT>;   // entries of a wave

// A wave's stretch as floats, its maximum and sums.  As much arithmetic as memory: ten vector instructions an entry (the exponential counts four).  2048 x 131072 bf16 take 91 us, 5.9 TB/s, and vector
// instructions are busy in 96 % of the cycles.
template <int DT> __global__ __launch_bounds__(STRETCH_WG, 8) void k_logprobs(LogprobArgs a) {
    constexpr int E = ENTRIES<DT>, N = STRETCH_N;
    const int at = blockIdx.x * (blockDim.x / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (at >= a.stretches) return;
    const int64_t row = a.row0 + blockIdx.y;
    const int first = at * STRETCH<DT>, lane = threadIdx.x & 63, lane_col = lane * E, vocab = (int)a.vocab;
    const entry_t<DT>* s = (const entry_t<DT>*)a.s + row * a.lds;
    chunk_t v[N];
    if (first + STRETCH<DT> <= vocab) {
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = *(const chunk_u*)(s + first + lane_col + n * 64 * E);
    } else {
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = load_chunk<DT>(s, first + lane_col + n * 64 * E, vocab);
    }
    float f[N][E], g[N], m = -INFINITY;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        chunk_floats<DT>(f[n], v[n]);
        g[n] = -INFINITY;   // a NaN among numbers is passed over, a chunk of nothing else has -Inf
#pragma unroll
        for (int e = 0; e < E; ++e) g[n] = fmaxf(g[n], f[n][e]);
        m = fmaxf(m, g[n]);
    }
    m = wave_max(m);
    if (a.groups) {
        const auto join = [&](auto other) {
#pragma unroll
            for (int n = 0; n < N; ++n) g[n] = fmaxf(g[n], other(g[n]));
        };
        if (a.lanes >= 2) join([](float x) { return dpp<0xB1, 0xF>(x, x); });     // lanes 2k and 2k + 1
        if (a.lanes >= 4) join([](float x) { return dpp<0x4E, 0xF>(x, x); });     // the pairs of four
        if (a.lanes >= 8) join([](float x) { return dpp<0x141, 0xF>(x, x); });    // eight, mirrored
        if (a.lanes >= 16) join([](float x) { return dpp<0x140, 0xF>(x, x); });   // sixteen
        if (a.lanes >= 32) join([](float x) { return __shfl_xor(x, 16); });
        if (a.lanes >= 64) join([](float x) { return __shfl_xor(x, 32); });
        if ((lane & (a.lanes - 1)) == 0) {
            const int shift = __builtin_ctz(a.lanes);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int chunk = (at * N + n) * 64 + lane;
                if (chunk * E < vocab) a.greatest[row * a.groups + (chunk >> shift)] = g[n];
            }
        }
    }
    const float from = m == -INFINITY ? 0.f : m, c = from * a.unit;
    float sum = 0.f, elog = 0.f;
    if (fabsf(c) < 65536.f) {
        // (s - m) / T in one instruction.  What c was rounded by, at most 2^-8, scales all of them alike, and is taken out of the sums.
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float t = fmaf(f[n][e], a.unit, -c), x = __builtin_amdgcn_exp2f(t);
                sum += x;
                elog = fmaf(x, fmaxf(t, -1024.f), elog);   // x is 0 below that
            }
        const float off = -fmaf(from, a.unit, -c), scale = __builtin_amdgcn_exp2f(off);
        elog = scale * fmaf(sum, off, elog);
        sum *= scale;
    } else {   // (a difference of -Inf: next to c it is thousands below)
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float t = (f[n][e] - from) * a.unit, x = __builtin_amdgcn_exp2f(t);
                sum += x;
                elog = fmaf(x, fmaxf(t, -1024.f), elog);
            }
    }
    sum = wave_sum(sum);
    elog = wave_sum(elog);
    float* p = a.stretch_stats + 3 * (row * a.stretches + at);
    if (lane < 3) p[lane] = lane == 0 ? m : lane == 1 ? sum : elog;
}

// ---- rows ---------------------------------------------------------------------------------------------------------------------------------

constexpr int ROOM = 1024, LIST = 512, BATCH = 4;   // keys found, groups listed; loads in flight
constexpr int SHORT_N = 4, SHORT_CHUNKS = 1024 * SHORT_N;   // chunks of a thread, and of a row, that one workgroup has in its registers

// Lanes below this one that are in the mask.
__device__ inline int lanes_before(uint64_t mask) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)); }
// Sums over the lanes up to this one.
template <int CTRL, int ROWS> __device__ inline int dpp_add(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false); }
__device__ inline int wave_prefix(int v) {
    v = dpp_add<0x111, 0xF>(v);
    v = dpp_add<0x112, 0xF>(v);
    v = dpp_add<0x114, 0xF>(v);
    v = dpp_add<0x118, 0xF>(v);
    v = dpp_add<0x142, 0xA>(v);
    return dpp_add<0x143, 0xC>(v);
}
// What the wave has written to LDS is there for all its lanes.
__device__ inline void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    __builtin_amdgcn_wave_barrier();
}

// The top keys among n of them (n > top), into the front of `found`, in any order; the least of them is returned.  One wave.
__device__ inline uint64_t cut_to_top(uint64_t* found, int n, int top) {
    constexpr int J = ROOM / 64;
    const int lane = threadIdx.x;
    uint64_t key[J];
    wave_sync();
#pragma unroll
    for (int j = 0; j < J; ++j) key[j] = j * 64 + lane < n ? found[j * 64 + lane] : 0;
    uint64_t least = 0;
    for (int b = 63; b >= 0; --b) {
        const uint64_t c = least | 1ull << b;
        int reach = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) reach += __popcll(__ballot(key[j] >= c));
        if (reach >= top) least = c;
        if (reach == top) break;
    }
    wave_sync();
    int at = 0;
    uint64_t smallest = ~0ull;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const bool keep = key[j] >= least;   // no two keys are equal: exactly `top`
        const uint64_t mask = __ballot(keep);
        if (keep) {
            found[at + lanes_before(mask)] = key[j];
            smallest = key[j] < smallest ? key[j] : smallest;
        }
        at += __popcll(mask);
    }
    wave_sync();
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const uint64_t other = (uint64_t)__shfl_xor((unsigned long long)smallest, o);
        smallest = other < smallest ? other : smallest;
    }
    return smallest;
}

// The top keys of a row by one wave, whatever ties and order it has, into the front of `found`: their number is returned.
template <int DT> __device__ inline int top_by_bisection(const LogprobArgs& a, const entry_t<DT>* s, const float* g, uint64_t* found, uint32_t* list) {
    constexpr int E = ENTRIES<DT>;
    const int lane = threadIdx.x;
    const auto group = [&](int r) { return r + lane < a.groups ? ordered(g[r + lane]) : 0u; };
    // the greatest number that `top` groups reach; below that of the lowest logit there is no alternative
    uint32_t bound = 0;
    for (int b = 31; b >= 0; --b) {
        const uint32_t c = bound | 1u << b;
        int reach = 0;
        for (int r = 0; r < a.groups; r += 64) reach += __popcll(__ballot(group(r) >= c));
        if (reach >= a.top) bound = c;
        if (reach == a.top) break;
    }
    bound = max(bound, ordered(LOWEST));
    // the groups, in order: all that are above the bound, of those that reach it the first `top`
    int listed = 0, ties = 0;
    for (int r = 0; r < a.groups; r += 64) {
        const uint32_t k = group(r);
        const bool tie = k == bound;
        const uint64_t tied = __ballot(tie);
        const bool take = k > bound || (tie && ties + lanes_before(tied) < a.top);
        const uint64_t mask = __ballot(take);
        const int at = listed + lanes_before(mask);
        if (take && at < 2 * MOST_ANSWERS) list[at] = r + lane;
        listed += __popcll(mask);
        ties += __popcll(tied);
    }
    listed = min(listed, 2 * MOST_ANSWERS);   // (never more)
    wave_sync();
    // their entries that reach the bound, 64 / lanes groups at a time
    float b = unordered(bound);
    bool equals = true;   // whether entries equal to b are still taken
    int n = 0, equal = 0;
    const int each = 64 / a.lanes, mine = lane / a.lanes, place = lane & (a.lanes - 1);
    for (int i = 0; i < listed; i += each) {
        const int at = i + mine;
        const unsigned col = at < listed ? (list[at] * a.lanes + place) * E : (unsigned)a.vocab;
        float f[E];
        chunk_floats<DT>(f, load_chunk<DT>(s, col, a.vocab));   // -Inf past the row's end
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool hit = f[e] > b || (equals && f[e] == b);
            const uint64_t mask = __ballot(hit);
            if (hit) found[n + lanes_before(mask)] = key_of(f[e], col + e);
            n += __popcll(mask);
            equal += __popcll(__ballot(f[e] == b));
        }
        if (equal >= a.top) equals = false;   // what follows has higher indices
        if (n > ROOM - 64 * E) {   // the next load may bring 64 * E
            static_assert(ROOM - 64 * E >= MOST_ANSWERS, "there are more than `top`");
            b = key_value(cut_to_top(found, n, a.top));
            n = a.top;
            equals = false;   // what follows and is equal to the last of them comes behind it
        }
    }
    if (n > a.top) {
        cut_to_top(found, n, a.top);
        n = a.top;
    }
    return n;
}

// The bound that the top K reach, by a histogram of the groups' greatest entries over their range, which ends 64 temperatures below the greatest (a mask's lowest value would leave all others one bin):
// 256 bins, of which a lower one holds greater entries.  `edge`: the bin in which the K-th lies (BINS: there are fewer), `upto`: the groups in it and above.  Each wave finds it by itself.
constexpr int ROWS_T = 256, BINS = 256;
struct Bound {
    float m, scale;
    int edge, upto;
    __device__ Bound(float m_, float low, float inv_temp) : m(m_), scale((BINS - 0.5f) / fminf(m_ - low, 64.f / inv_temp)), edge(0), upto(0) {}
    // (equal groups are all in the last one: fminf takes 0 times infinity for no number)
    __device__ int bin(float g) const { return g == -INFINITY ? BINS : (int)fminf((m - g) * scale, BINS - 1.f); }
    __device__ void count(int* bins, int b) const {
        if (b < BINS) atomicAdd(&bins[b], 1);
    }
    __device__ void find(const int* bins, int top) {
        const int lane = threadIdx.x & 63;
        const int4 own = ((const int4*)bins)[lane];
        const int four = own.x + own.y + own.z + own.w, behind = wave_prefix(four);
        const uint64_t reach = __ballot(behind >= top);
        edge = BINS;
        upto = __builtin_amdgcn_readlane(behind, 63);
        if (!reach) return;
        const int at = __ffsll((unsigned long long)reach) - 1, each[4] = {own.x, own.y, own.z, own.w};
        int e = 0, n = behind - four;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (n < top) {
                n += each[k];
                e = 4 * lane + k;
            }
        edge = __builtin_amdgcn_readlane(e, at);
        upto = __builtin_amdgcn_readlane(n, at);
    }
    // a number that the groups up to the edge reach, a little below the bin's end for what its arithmetic is rounded by; never -Inf, which is no alternative
    __device__ float least() const { return edge >= BINS - 1 ? LOWEST : fmaxf(m - (edge + 1.01f) / scale - fabsf(m) * 0x1p-22f, LOWEST); }
};

// Entries of a thread's chunks that reach `least`, into `found` as far as there is room.
template <int N, int E> __device__ inline void collect(const float (&f)[N][E], float least, const unsigned (&col)[N], uint64_t* found, int* number) {
    int hits = 0;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < E; ++e) hits += f[n][e] >= least;
    if (!hits) return;
    int at = atomicAdd(number, hits);
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (f[n][e] >= least) {
                if (at < ROOM) found[at] = key_of(f[n][e], col[n] + e);
                ++at;
            }
}
// The n keys found, each at its place.
template <int T> __device__ inline void write_found(const LogprobArgs& a, int64_t row, const uint64_t* found, int n, const RowSums& sums) {
    for (int i = threadIdx.x; i < n; i += T) {
        const uint64_t key = found[i];
        int before = 0;
#pragma unroll 8
        for (int o = 0; o < n; ++o) before += found[o] > key;
        if (before < a.top) write_top(a, row, before, key, sums);
    }
    for (int i = n + threadIdx.x; i < a.top; i += T) write_top(a, row, i, 0, sums);
}
__device__ inline void write_sums(const LogprobArgs& a, int64_t row, int32_t token, float logit, const RowSums& sums) {
    const int t = threadIdx.x;
    if (t < a.given) {
        const bool out = token >= a.vocab;
        a.logprob[row * a.given + t] = token < 0 ? 0.f : out ? __builtin_nanf("") : sums.log_p(logit, a.inv_temp);
        if (out && a.dev_status) atomicOr(a.dev_status, MLMC_DEV_RANGE);
    }
    if (t == 0 && a.entropy) a.entropy[row] = sums.h;
    if (a.stats && t < 3) a.stats[3 * row + t] = t == 0 ? sums.m : t == 1 ? sums.log_s : sums.h;
}
template <int DT> __device__ inline int32_t load_token(const LogprobArgs& a, int64_t row, float& logit) {
    int32_t token = -1;
    logit = 0.f;
    if ((int)threadIdx.x < a.given) {
        token = a.tokens[row * a.given + threadIdx.x];
        if (token >= 0 && token < a.vocab) logit = to_f32(((const entry_t<DT>*)a.s)[row * a.lds + token]);
    }
    return token;
}

// A row of several stretches by a workgroup.  Rows that have too many groups or entries at the bound, as with ties, go to one wave.  R: groups of a thread, 0 without alternatives.
template <int DT, int R> __global__ __launch_bounds__(ROWS_T) void k_logprobs_rows(LogprobArgs a) {
    constexpr int E = ENTRIES<DT>, W = ROWS_T / 64;
    __shared__ uint64_t found[R ? ROOM : 1];
    __shared__ uint32_t list[R ? LIST : 1];
    __shared__ __align__(16) int bins[R ? BINS : 1];
    __shared__ float lows[W], total[3];
    __shared__ int listed, number;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t row = a.row0 + blockIdx.x;
    const entry_t<DT>* s = (const entry_t<DT>*)a.s + row * a.lds;
    const float* groups = a.greatest + row * a.groups;
    float g[R ? R : 1];
    if constexpr (R > 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) g[r] = r * ROWS_T + t < a.groups ? groups[r * ROWS_T + t] : -INFINITY;
        bins[t] = 0;
    }
    float logit;
    const int32_t token = load_token<DT>(a, row, logit);
    const float* stretch = a.stretch_stats + 3 * row * a.stretches;
    float m = -INFINITY;
    if (R > 0 || wave == 0) {
        for (int p = lane; p < a.stretches; p += 64) m = fmaxf(m, stretch[3 * p]);
        m = wave_max(m);
    }
    if (wave == 0) {   // the stretches' sums: each lane's, one after the other, then the lanes'
        float sum = 0.f, elog = 0.f;
        const Scaled scaled(m, a.unit);
        for (int p = lane; p < a.stretches; p += 64) {
            const float from = stretch[3 * p], part = stretch[3 * p + 1];
            const float x = from == -INFINITY ? -1024.f : fmaxf(scaled(from), -1024.f), w = __builtin_amdgcn_exp2f(x);
            sum = fmaf(part, w, sum);
            elog = fmaf(w, fmaf(part, x, stretch[3 * p + 2]), elog);
        }
        sum = wave_sum(sum);
        elog = wave_sum(elog);
        if (lane == 0) {
            total[0] = m;
            total[1] = sum;
            total[2] = elog;
            listed = number = 0;
        }
    }
    if constexpr (R > 0) {
        float low = m;
#pragma unroll
        for (int r = 0; r < R; ++r) low = fminf(low, g[r] == -INFINITY ? m : g[r]);
        low = -wave_max(-low);
        if (lane == 0) lows[wave] = low;
    }
    __syncthreads();
    const RowSums sums(total[0], total[1], total[2]);
    write_sums(a, row, token, logit, sums);
    if constexpr (R > 0) {
        if (sums.bad) {
            for (int i = t; i < a.top; i += ROWS_T) write_top(a, row, i, 0, sums);
            return;
        }
        float low = m;
#pragma unroll
        for (int w = 0; w < W; ++w) low = fminf(low, lows[w]);
        Bound bound(m, low, a.inv_temp);
        int bin[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            bin[r] = bound.bin(g[r]);
            bound.count(bins, bin[r]);
        }
        __syncthreads();
        bound.find(bins, a.top);
        int n = ROOM + 1;
        if (bound.upto <= LIST) {
            int takes = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) takes += bin[r] <= bound.edge && bin[r] < BINS;
            int at = takes ? atomicAdd(&listed, takes) : 0;
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (bin[r] <= bound.edge && bin[r] < BINS) list[at++] = r * ROWS_T + t;
            __syncthreads();
            const float least = bound.least();
            const int each = 64 / a.lanes, mine = lane / a.lanes, place = lane & (a.lanes - 1);
            for (int i = wave * each; i < bound.upto; i += W * each * BATCH) {
                chunk_t v[BATCH];
                unsigned col[BATCH];
#pragma unroll
                for (int u = 0; u < BATCH; ++u) {
                    const int at = i + u * W * each + mine;
                    col[u] = at < bound.upto ? (list[at] * a.lanes + place) * E : (unsigned)a.vocab;
                    v[u] = load_chunk<DT>(s, col[u], a.vocab);   // -Inf past the row's end
                }
                float f[BATCH][E];
#pragma unroll
                for (int u = 0; u < BATCH; ++u) chunk_floats<DT>(f[u], v[u]);
                collect(f, least, col, found, &number);
            }
            __syncthreads();
            n = number;
        }
        if (n > ROOM) {
            __syncthreads();   // all waves have read the number
            if (wave == 0) {
                n = top_by_bisection<DT>(a, s, groups, found, list);
                if (lane == 0) number = n;
            }
            __syncthreads();
            n = number;
        }
        write_found<ROWS_T>(a, row, found, n, sums);
    }
}

// A short row (up to 4 T chunks of 16 bytes) by a workgroup of T threads, all of it in its registers: a chunk is a group, and its entries are at hand.
template <int DT, int T, bool TOP> __global__ __launch_bounds__(T, 8) void k_logprobs_short(LogprobArgs a) {
    constexpr int E = ENTRIES<DT>, N = SHORT_N, W = T / 64;
    __shared__ uint64_t found[TOP ? ROOM : 1];
    __shared__ uint32_t list[TOP ? 2 * MOST_ANSWERS : 1];
    __shared__ float groups[TOP ? N * T : 1];
    __shared__ __align__(16) int bins[TOP ? BINS : 1];
    __shared__ float most[W], lows[W], part[2][W];
    __shared__ int number;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, vocab = (int)a.vocab;
    const int64_t row = a.row0 + blockIdx.x;
    const entry_t<DT>* s = (const entry_t<DT>*)a.s + row * a.lds;
    chunk_t v[N];
#pragma unroll
    for (int n = 0; n < N; ++n)
        if (n * T * E < vocab) v[n] = load_chunk<DT>(s, (n * T + t) * E, vocab);
    float logit;
    const int32_t token = load_token<DT>(a, row, logit);
    float f[E], g[N], m = -INFINITY, low = INFINITY;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        g[n] = -INFINITY;
        if (n * T * E >= vocab) continue;
        chunk_floats<DT>(f, v[n]);
#pragma unroll
        for (int e = 0; e < E; ++e) g[n] = fmaxf(g[n], f[e]);
        m = fmaxf(m, g[n]);
        if (TOP && g[n] != -INFINITY) low = fminf(low, g[n]);
    }
    m = wave_max(m);
    if (TOP) low = -wave_max(-low);
    if (lane == 0) {
        most[wave] = m;
        lows[wave] = low;
    }
    if (TOP) {
        if (t < BINS) bins[t] = 0;
        if (t == 0) number = 0;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) {
        m = fmaxf(m, most[w]);
        low = fminf(low, lows[w]);
    }
    Bound bound(m, low, a.inv_temp);
    if (TOP) {
#pragma unroll
        for (int n = 0; n < N; ++n) bound.count(bins, bound.bin(g[n]));
    }
    const Scaled scaled(m == -INFINITY ? 0.f : m, a.unit);
    float sum = 0.f, elog = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n * T * E >= vocab) continue;
        chunk_floats<DT>(f, v[n]);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = scaled(f[e]), p = __builtin_amdgcn_exp2f(x);
            sum += p;
            elog = fmaf(p, fmaxf(x, -1024.f), elog);
        }
    }
    sum = wave_sum(sum);
    elog = wave_sum(elog);
    if (lane == 0) {
        part[0][wave] = sum;
        part[1][wave] = elog;
    }
    __syncthreads();
    sum = elog = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        sum += part[0][w];
        elog += part[1][w];
    }
    const RowSums sums(m, sum, elog);
    write_sums(a, row, token, logit, sums);
    if constexpr (TOP) {
        if (sums.bad) {
            for (int i = t; i < a.top; i += T) write_top(a, row, i, 0, sums);
            return;
        }
        bound.find(bins, a.top);
        const float least = bound.least();
        float most_here = g[0];
#pragma unroll
        for (int n = 1; n < N; ++n) most_here = fmaxf(most_here, g[n]);
        if (most_here >= least) {
            float all[N][E];
            unsigned col[N];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                col[n] = (unsigned)((n * T + t) * E);
                if (n * T * E < vocab) chunk_floats<DT>(all[n], v[n]);
                else {
#pragma unroll
                    for (int e = 0; e < E; ++e) all[n][e] = -INFINITY;
                }
            }
            collect(all, least, col, found, &number);
        }
        __syncthreads();
        int n = number;
        if (n > ROOM) {
#pragma unroll
            for (int k = 0; k < N; ++k) groups[k * T + t] = g[k];
            __syncthreads();
            if (wave == 0) {
                n = top_by_bisection<DT>(a, s, groups, found, list);
                if (lane == 0) number = n;
            }
            __syncthreads();
            n = number;
        }
        write_found<T>(a, row, found, n, sums);
    }
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
    const Scaled scaled(m, a.unit);
    const float unit = scaled.half == 1.0f ? a.inv_temp : a.inv_temp + a.inv_temp;
    const auto dense = [&](float x) {
        const float d = scaled.difference(x), p = power(d, scaled.unit) * inv_s;
        return p * fmaf(ch, fmaxf(fmaf(d, unit, -base), -1024.f), ca);   // log p + H; p is 0 below that
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

constexpr int64_t VOCAB_MAX = (int64_t)1 << 20;
constexpr int GROUPS_MOST = 1024;   // more only of rows that have them with all lanes of a wave

struct LogprobPlan { int stretches, groups, lanes; };
// Rows of up to 2048 chunks by one workgroup each; up to 4096 where all workgroups of 1024 threads are on the chip at once, or without alternatives, whose search holds up the next row's loads.
// In one launch / in two, us: 4 x 32000 bf16 with 20 13.1 / 15.6 (bound by the host), 512 x 32768 with 128 19.5 / 21.6, 2048 x 32000 with 20 51.8 / 40.1, without 4000 x 32000 49.9 / 51.4;
// of 512 threads 8000 x 8000 fp32 with 20 63 / 80, 8000 x 12000 bf16 with 64 80 / 91.
static LogprobPlan logprob_plan(int64_t rows, int64_t vocab, int dtype, int top) {
    const int64_t E = dtype == MLMC_BF16 ? 8 : 4, stretch = 64 * STRETCH_N * E, chunks = (vocab + E - 1) / E;
    LogprobPlan p = {(int)((vocab + stretch - 1) / stretch), 0, 1};
    if (chunks <= (rows <= 512 || !top ? SHORT_CHUNKS : SHORT_CHUNKS / 2)) return {0, (int)chunks, 1};   // by one workgroup, without a workspace
    while (p.lanes < 64 && (chunks + p.lanes - 1) / p.lanes > GROUPS_MOST) p.lanes *= 2;
    if (top) p.groups = (int)((chunks + p.lanes - 1) / p.lanes);
    return p;
}
static size_t logprob_bytes(const LogprobPlan& p, int64_t rows) { return p.stretches == 0 ? 0 : (size_t)rows * ((size_t)p.stretches * 3 + p.groups) * sizeof(float); }
static bool logprob_sizes_ok(int64_t rows, int64_t vocab, int given, int top) {
    return rows >= 0 && rows < ((int64_t)1 << 31) && vocab >= 1 && vocab <= VOCAB_MAX && given >= 0 && given <= MOST_ANSWERS && top >= 0 && top <= MOST_ANSWERS;
}
static bool temperature_ok(float t) { return t > 0.0f && t <= 3.402823e38f && 1.4426950408889634f / t <= 3.402823e38f; }
constexpr int64_t ROW_SLICE = 32768;   // rows of a launch: they are the grid's second axis

template <int DT, int T> static mlmc_status logprob_short(const LogprobArgs& a, unsigned rows, hipStream_t st) {
    if (a.top) MLMC_LAUNCH(K_LOGPROBS, st, (k_logprobs_short<DT, T, true><<<rows, T, 0, st>>>(a)));
    else MLMC_LAUNCH(K_LOGPROBS, st, (k_logprobs_short<DT, T, false><<<rows, T, 0, st>>>(a)));
    return MLMC_OK;
}
template <int DT> static mlmc_status logprob_run(LogprobArgs a, hipStream_t st) {
    const int each = a.stretches < STRETCH_WG / 64 ? a.stretches : STRETCH_WG / 64;
    for (; a.row0 < a.rows; a.row0 += ROW_SLICE) {
        const unsigned rows = (unsigned)(a.rows - a.row0 < ROW_SLICE ? a.rows - a.row0 : ROW_SLICE);
        if (a.stretches == 0) {
            const mlmc_status rc = a.groups <= 256 * SHORT_N ? logprob_short<DT, 256>(a, rows, st) : a.groups <= 512 * SHORT_N ? logprob_short<DT, 512>(a, rows, st) : logprob_short<DT, 1024>(a, rows, st);
            if (rc != MLMC_OK) return rc;
            continue;
        }
        MLMC_LAUNCH(K_LOGPROBS, st, (k_logprobs<DT><<<dim3((unsigned)((a.stretches + each - 1) / each), rows), each * 64, 0, st>>>(a)));
        if (a.groups == 0) MLMC_LAUNCH(K_LOGPROBS_ROWS, st, (k_logprobs_rows<DT, 0><<<rows, ROWS_T, 0, st>>>(a)));
        else if (a.groups <= 4 * ROWS_T) MLMC_LAUNCH(K_LOGPROBS_ROWS, st, (k_logprobs_rows<DT, 4><<<rows, ROWS_T, 0, st>>>(a)));
        else MLMC_LAUNCH(K_LOGPROBS_ROWS, st, (k_logprobs_rows<DT, 16><<<rows, ROWS_T, 0, st>>>(a)));
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
    const size_t a = logprob_bytes(logprob_plan(rows, vocab, MLMC_F32, top), rows), b = logprob_bytes(logprob_plan(rows, vocab, MLMC_BF16, top), rows);
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
    const LogprobPlan p = logprob_plan(rows, vocab, dtype, top);
    const size_t need = logprob_bytes(p, rows);
    if (rows > 0 && need && (!ws || (uintptr_t)ws % 256 || ws_bytes < need)) return MLMC_EINVAL;
    if (dev_status) MLMC_LAUNCH(K_ZERO, st, (k_logprobs_clear<<<1, 1, 0, st>>>(dev_status)));
    if (rows == 0) return MLMC_OK;
    LogprobArgs a = {};
    a.s = logits; a.lds = ldl; a.rows = rows; a.vocab = vocab; a.tokens = tokens; a.given = given; a.top = top; a.inv_temp = 1.0f / temperature;
    a.unit = LOG2E / temperature; a.logprob = logprob; a.entropy = entropy; a.top_idx = top_idx; a.top_logprob = top_logprob; a.stats = stats; a.dev_status = dev_status;
    a.stretches = p.stretches; a.groups = p.groups; a.lanes = p.lanes; a.stretch_stats = (float*)ws; a.greatest = (float*)ws + rows * 3 * p.stretches;
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
