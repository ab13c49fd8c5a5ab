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
#include <type_traits>

#include "mlmc_worker.h"

namespace mlmc {

// C[i][j] = sum_c A(i, c) B(j, c).  An operand lies along the contraction (A(i, c) at a[i * lda + c]) or across it (at a[c * lda + i]).
struct LinearArgs {
    const void *a, *b;
    int64_t lda, ldb, I, J, C;
    int act;
    const float* bias;     // forward: of column j
    const void* slope_z;   // dgrad: C is multiplied with act' of this
    int64_t ld_slope;
    const void* residual;
    int64_t ldr;
    void* z;               // forward: receives C + bias
    int64_t ldz;
    void* out;
    int64_t ldo;
    int out_dtype;
    void* row_sum;         // wgrad: sum_c A(i, c), in out_dtype
    int tiles_i, tiles_j;
    int splits;            // the contraction is cut into this many parts, whose sums are joined by k_linear_join
    int split_len;         // entries of the contraction of a part, a multiple of a step's
    float* part;           // the workspace: [splits][I][J], then [splits][I] for row_sum
    size_t ws_bytes;
};

// The tail of the normal distribution, Phi(-|z|) = erfc(|z| / sqrt 2) / 2, and its density's exponential e^(-z^2 / 2), which the slope of gelu needs as well.  For 32-bit results by
// the library's functions, so that gelu and its slope are no further off than elementary operations (2048 x 2048 x 2048 with gelu 131 us, its input gradient 134; by the approximation
// 127 and 128, and two to three times as far off).  For 16-bit ones by the rational approximation 7.1.26 of Abramowitz and Stegun,
// Handbook of Mathematical Functions: off by at most 1.5e-7, half of which reaches Phi, less than such a result's rounding down to z = -4 and about as much at -5.  It takes 15 to 40 us
// less on the largest products, which have 16 bits.
template <int DT> __device__ inline float normal_tail(float z, float& e) {
    if constexpr (DT == MLMC_F32) {
        e = expf(-0.5f * z * z);
        return 0.5f * erfcf(fabsf(z) * 0.70710678118654752f);
    }
    e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.3275911f * 0.70710678118654752f, 1.0f));
    const float p = fmaf(fmaf(fmaf(fmaf(0.5f * 1.061405429f, t, 0.5f * -1.453152027f), t, 0.5f * 1.421413741f), t, 0.5f * -0.284496736f), t, 0.5f * 0.254829592f);
    return p * (t * e);
}
__device__ inline float relu(float z) { return z > 0.f || z != z ? z : 0.f; }   // a NaN stays one
template <int DT> __device__ inline float gelu(float z) {
    float e;
    const float tail = normal_tail<DT>(z, e);
    return fmaf(-fminf(fabsf(z), 64.f), tail, fmaxf(z, 0.f));   // z Phi(z); the tail is 0 from 14 on, and infinity times it would be NaN
}
template <int DT> __device__ inline float gelu_slope(float z) {
    float e;
    const float tail = normal_tail<DT>(z, e);
    const float d = __builtin_amdgcn_fmed3f(z, -64.f, 64.f) * 0.39894228040143268f;   // z within +-64 for the same reason; a NaN comes by e
    if constexpr (DT == MLMC_BF16) return fmaf(d, e, z > 0.f ? 1.0f - tail : tail);
    const float s = fmaf(d, e, z > 0.f ? -tail : tail);   // one rounding less next to 1
    return z > 0.f ? 1.0f + s : s;
}
__device__ inline void store_as(void* p, int64_t at, int dtype, float v) {
    if (dtype == MLMC_F32) ((float*)p)[at] = v;
    else ((__bf16*)p)[at] = (__bf16)v;
}


using v16f = float __attribute__((ext_vector_type(16)));
using v4s = short __attribute__((ext_vector_type(4)));
using lds_void = __attribute__((address_space(3))) void;

template <int DT> __device__ inline void load8(float (&v)[8], const void* p, int64_t at, int n) {
    if constexpr (DT == MLMC_BF16) {
        const __bf16* q = (const __bf16*)p + at;
        if (n == 8) {
            const v8b w = __builtin_bit_cast(v8b, (chunk_t) * (const chunk_u*)q);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)w[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < n ? (float)q[e] : 0.f;
        }
    } else {
        const float* q = (const float*)p + at;
        if (n == 8) {
            const v4f w0 = __builtin_bit_cast(v4f, (chunk_t) * (const chunk_u*)q), w1 = __builtin_bit_cast(v4f, (chunk_t) * (const chunk_u*)(q + 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] = w0[e]; v[4 + e] = w1[e]; }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < n ? q[e] : 0.f;
        }
    }
}
__device__ inline void store8(const float (&v)[8], void* p, int64_t at, int n, int dtype) {
    if (n < 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) store_as(p, at + e, dtype, v[e]);
    } else if (dtype == MLMC_BF16) {
        v8b w;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = (__bf16)v[e];
        *(chunk_u*)((__bf16*)p + at) = __builtin_bit_cast(chunk_t, w);
    } else {
        const v4f w0 = {v[0], v[1], v[2], v[3]}, w1 = {v[4], v[5], v[6], v[7]};
        *(chunk_u*)((float*)p + at) = __builtin_bit_cast(chunk_t, w0);
        *(chunk_u*)((float*)p + at + 4) = __builtin_bit_cast(chunk_t, w1);
    }
}

// The epilogue of n <= 8 neighbouring entries of a row of the product, cut in two so that the loads of several rows are in flight together.
struct Epilogue {
    float slope[8], residual[8];
    template <int DT> __device__ void load(const LinearArgs& g, int64_t i, int64_t j, int n) {
        if (g.slope_z) load8<DT>(slope, g.slope_z, i * g.ld_slope + j, n);
        if (g.residual) load8<DT>(residual, g.residual, i * g.ldr + j, n);
    }
    template <int DT> __device__ void finish(const LinearArgs& g, int64_t i, int64_t j, float (&v)[8], const float (&bias)[8], int n) const {
        if (g.bias) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += bias[e];
        }
        if (g.z) store8(v, g.z, i * g.ldz + j, n, DT);
        if (g.act == MLMC_ACT_GELU) {   // the branches outside of the loops: inside they took longer than the arithmetic
            if (g.slope_z) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= gelu_slope<DT>(slope[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = gelu<DT>(v[e]);
            }
        } else if (g.act == MLMC_ACT_RELU) {
            if (g.slope_z) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = slope[e] > 0.f ? v[e] : 0.f * v[e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = relu(v[e]);
            }
        }
        if (g.residual) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += residual[e];
        }
        store8(v, g.out, i * g.ldo + j, n, g.out_dtype);
    }
};

// Where a step's operand lies in LDS, in 16-byte slots.  ALONG: a row of LDS is an index's 128 bytes of the contraction; else it is a
// contraction index's T entries.  The slot in a row is exclusive-ored so that the lanes that read at once (eight rows' slots; or, transposing,
// four rows' pairs of slots and the same eight rows below) lie in different banks.
template <int DT, bool ALONG, int T> struct Lds {
    static constexpr int E = DT == MLMC_BF16 ? 8 : 4, W = ALONG ? 8 : T / E;   // slots of a row
    __device__ static int swizzle(int r) {
        if (ALONG) return r & 7;
        return DT == MLMC_BF16 ? (((r & 3) << 1) | (r & 8)) & (W - 1) : 0;
    }
    __device__ static int slot(int r, int c) { return r * W + (c ^ swizzle(r)); }
};

// Operand fragments of the matrix instructions for a quarter q of a step: of index (f0 + f) * 32 + lane % 32 and, per half of the wave, 16 bytes of
// the contraction.  The lane's places are kept; f or q, whichever the slots' exclusive-or does not reach, goes into the instruction's offset.
template <int DT, bool ALONG, int T, int F> struct Fragments {
    using L = Lds<DT, ALONG, T>;
    static constexpr int N = ALONG ? 4 : DT == MLMC_BF16 ? F : 1;
    int place[N];   // bytes
    __device__ void init(int f0) {
        const int lane = threadIdx.x & 63, half = lane >> 5, i = lane & 15;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (ALONG) place[n] = L::slot(f0 * 32 + (lane & 31), n * 2 + half) * 16;
            else if (DT == MLMC_BF16) {
                const int col = (f0 + n) * 32 + (lane & 16) + (i & 3) * 4;
                place[n] = L::slot(half * 8 + (i >> 2), col >> 3) * 16 + ((col & 4) << 1);
            } else place[n] = (half * 4 * T + f0 * 32 + (lane & 31)) * 4;
        }
    }
    __device__ chunk_t get(const chunk_t* s, int f, int q) const {
        const char* p = (const char*)s;
        if constexpr (ALONG) {
            return *(const chunk_t*)(p + place[q] + f * 32 * 128);
        } else if constexpr (DT == MLMC_BF16) {
            v4s h[2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
                h[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(p + place[f] + (q * 16 + 4 * k) * T * 2));
            return __builtin_bit_cast(chunk_t, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            v4f v;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = *(const float*)(p + place[0] + ((q * 8 + k) * T + f * 32) * 4);
            return __builtin_bit_cast(chunk_t, v);
        }
    }
};

template <int DT> __device__ inline v16f multiply(chunk_t a, chunk_t b, v16f c) {
    if constexpr (DT == MLMC_BF16) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
    } else {
        const v4f x = __builtin_bit_cast(v4f, a), y = __builtin_bit_cast(v4f, b);
#pragma unroll
        for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[k], y[k], c, 0, 0, 0);
        return c;
    }
}

template <int DT> __device__ inline float chunk_sum(chunk_t a) {
    float s = 0.f;
    if constexpr (DT == MLMC_BF16) {
        const v8b v = __builtin_bit_cast(v8b, a);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += (float)v[e];
    } else {
        const v4f v = __builtin_bit_cast(v4f, a);
#pragma unroll
        for (int e = 0; e < 4; ++e) s += v[e];
    }
    return s;
}

// How steps come to LDS: through registers (any entry's place); by loads that go there by themselves, of 16 bytes a lane, or of 4 (fp32 of any place, bf16 whose rows
// begin and end at 4 bytes: four times the loads).  Through registers / by words, us: fp32 1000 x 2049 x 1537 88 / 80; bf16 1000 x 2050 x 1538 forward 27.5 / 23.1,
// input gradient 43.5 / 25.9, weight gradient 30.5 / 21.7; 4098 x 4098 over 4096 298 / 200.
enum LinearWay { WAY_REGISTERS = 0, WAY_CHUNKS, WAY_WORDS };

// One operand's way from memory to LDS: 128 bytes of the contraction (a step) for T indices, by NT threads.
template <int DT, bool ALONG, int T, int NT, int WAY> struct Operand {
    static constexpr bool WIDE = WAY == WAY_CHUNKS;   // a row has 16 bytes
    static constexpr int E = DT == MLMC_BF16 ? 8 : 4, STEP = 8 * E, N = T * 8 / NT;   // N: chunks a thread moves
    const void* p;
    int64_t ld, i0, I, C;
    using off_t = std::conditional_t<WAY != WAY_REGISTERS, unsigned, int64_t>;
    static constexpr int LOADS = WAY == WAY_WORDS ? 4 * N : N;
    off_t off[LOADS];   // byte offsets from the tile's base

    using L = Lds<DT, ALONG, T>;
    __device__ static int row(int q) { return q / L::W; }
    __device__ static int chunk(int q) { return (q % L::W) ^ L::swizzle(q / L::W); }   // which chunk of the row slot q holds
    __device__ void init(const void* p_, int64_t ld_, int64_t i0_, int64_t I_, int64_t C_) {
        p = p_; ld = ld_; i0 = i0_; I = I_; C = C_;
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int at = u * NT + threadIdx.x, q = WAY == WAY_WORDS ? at >> 2 : at, r = row(q), c = chunk(q) * E + (WAY == WAY_WORDS ? (at & 3) * (E / 4) : 0), e = WAY == WAY_WORDS ? E / 4 : E;
            // what lies past the matrix repeats its last entries: it reaches only results that are not stored
            if (ALONG) off[u] = (off_t)(((i0 + r < I ? r : I - 1 - i0) * ld + c) * (16 / E));
            else off[u] = (off_t)((r * ld + (i0 + c < I ? c : (I - 1) / e * e - i0)) * (16 / E));
        }
    }
    // a whole step, straight into LDS; `c` its first contraction index.  From `end` on nothing is read (the buffer has no entries, zeros arrive).
    __device__ void fetch(chunk_t* s, int c, int end) const {
        // a buffer load and not a global one: behind the latter the compiler takes every wait for LDS reads to be one for all of them
        const __amdgpu_buffer_rsrc_t rsrc =
            __builtin_amdgcn_make_buffer_rsrc((char*)p + (ALONG ? i0 * ld + c : (int64_t)c * ld + i0) * (16 / E), 0,
                                              __builtin_amdgcn_readfirstlane(c < end ? -1 : 0) /* the select is compiled into a vector one */, 0x00027000);
        const int wave0 = __builtin_amdgcn_readfirstlane(threadIdx.x) & ~63;
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            if constexpr (WAY == WAY_WORDS) __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)((int*)s + u * NT + wave0), 4, (int)off[u], 0, 0, 0);
            else __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(s + u * NT + wave0), 16, (int)off[u], 0, 0, 0);
        }
    }
    // any step, by way of registers, zeros outside
    __device__ bool inside(int64_t c) const { return WAY != WAY_WORDS && c + STEP <= C && (ALONG || i0 + T <= I); }
    __device__ void load(chunk_t (&v)[N], int64_t c) const {
        if (inside(c)) {
            const char* base = (const char*)p + (ALONG ? i0 * ld + c : c * ld + i0) * (16 / E);
#pragma unroll
            for (int u = 0; u < N; ++u) v[u] = *(const chunk_u*)(base + off[u]);
            return;
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int q = u * NT + threadIdx.x;
            if (ALONG) v[u] = raw_chunk<DT, WIDE>(p, ld, i0 + row(q), I, c + chunk(q) * E, C);
            else v[u] = raw_chunk<DT, WIDE>(p, ld, c + row(q), C, i0 + chunk(q) * E, I);
        }
    }
    __device__ void store(chunk_t* s, const chunk_t (&v)[N], int64_t c) const {
        if (inside(c)) {
#pragma unroll
            for (int u = 0; u < N; ++u) s[u * NT + threadIdx.x] = v[u];
            return;
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int q = u * NT + threadIdx.x;
            if (ALONG) s[q] = cut_chunk<DT, WIDE>(v[u], i0 + row(q), I, c + chunk(q) * E, C);
            else s[q] = cut_chunk<DT, WIDE>(v[u], c + row(q), C, i0 + chunk(q) * E, I);
        }
    }
};

// A tile of the product.  WM x WN waves, each FM x FN matrix instructions of 32 x 32.  AA, BA: the contraction is contiguous in A, B.
// The large tile (256 x 256, bf16) has 8 waves of 128 x 64: two a SIMD, so that one multiplies while the other waits to issue loads or is in the epilogue.  Four waves of
// 128 x 128 read a third less from LDS and are no faster (gelu, z stored: 8192 x 4096 x 4096 240 and 240 us, 8192 x 4096 x 1024 102 and 92; weight gradient of the former 251
// and 228).  Four steps of 64 bytes in flight instead of two of 128 have twice the barriers, and the loads are not what is waited for (247 and 236 us for
// 8192 x 4096 x 4096).  With no loads that product would take two thirds of the time, with nothing but loads also: what is left is that the two do not overlap fully.
// The small tile of 32-bit entries is held to the registers of four waves a SIMD, which its LDS allows and gelu's constants would not.
template <int DT, int WM, int WN, int FM, int FN, bool AA, bool BA, int WAY>
__global__ __launch_bounds__(WM * WN * 64, DT == MLMC_F32 && FM * FN == 1 ? 4 : 1) void k_linear_tile(LinearArgs g) {
    constexpr int NT = WM * WN * 64, TM = WM * FM * 32, TN = WN * FN * 32;
    constexpr bool FAST = WAY != WAY_REGISTERS;   // whole steps come straight into LDS
    __shared__ chunk_t a0[TM * 8], b0[TN * 8], a1[TM * 8], b1[TN * 8];
    using OpA = Operand<DT, AA, TM, NT, WAY>;
    using OpB = Operand<DT, BA, TN, NT, WAY>;
    constexpr int STEP = OpA::STEP;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave % WM, wn = wave / WM;
    // neighbouring tiles to the workgroups of one die (workgroups go round the 8 dies), eight tile rows at a time
    int t = blockIdx.x;
    {
        const int n = gridDim.x, q = n / 8, r = n % 8, x = t & 7;
        t = x * q + (x < r ? x : r) + (t >> 3);
    }
    // (divisions run on the vector unit; what follows from them is uniform, which the buffers' descriptors have to be)
    const auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    const int tiles = g.tiles_i * g.tiles_j, split = uniform(t / tiles);
    t -= split * tiles;
    const int band = uniform(t / (8 * g.tiles_j)), in_band = t - band * 8 * g.tiles_j, high = min(8, g.tiles_i - band * 8);
    const int tj = uniform(in_band / high), ti = band * 8 + in_band - tj * high;
    const int64_t i0 = (int64_t)ti * TM, j0 = (int64_t)tj * TN;
    const int C = (int)g.C, c_begin = split * g.split_len, c_end = min(C, c_begin + g.split_len);   // at most 2^21
    OpA A;
    OpB B;
    A.init(g.a, g.lda, i0, g.I, g.C);
    B.init(g.b, g.ldb, j0, g.J, g.C);

    v16f acc[FM][FN];
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int n = 0; n < FN; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[m][n][r] = 0.f;
    float sums[FM] = {};
    const bool rows = !AA && g.row_sum && tj == 0;   // this workgroup adds up A's entries; wave wn takes quarter wn of every step

    Fragments<DT, AA, TM, FM> FA;
    Fragments<DT, BA, TN, FN> FB;
    FA.init(wm * FM);
    FB.init(wn * FN);
    chunk_t fa[2][FM], fb[2][FN];
    const auto read = [&](const chunk_t* sa, const chunk_t* sb, int q) {
#pragma unroll
        for (int m = 0; m < FM; ++m) fa[q & 1][m] = FA.get(sa, m, q);
#pragma unroll
        for (int n = 0; n < FN; ++n) fb[q & 1][n] = FB.get(sb, n, q);
    };
    const auto multiply_quarter = [&](int q) {
#pragma unroll
        for (int m = 0; m < FM; ++m)
#pragma unroll
            for (int n = 0; n < FN; ++n) acc[m][n] = multiply<DT>(fb[q & 1][n], fa[q & 1][m], acc[m][n]);
        // the reads and the loads between the matrix instructions: left alone they sink behind them
        constexpr int READS = FM * (AA ? 1 : DT == MLMC_BF16 ? 2 : 4) + FN * (BA ? 1 : DT == MLMC_BF16 ? 2 : 4);
#pragma unroll
        for (int i = 0; i < READS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            if (FAST && (q == 3 || q == 0)) __builtin_amdgcn_sched_group_barrier(0x10, WAY == WAY_WORDS ? 4 : 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto add_rows = [&](const chunk_t* sa) {
        if (!AA && rows)
            for (int q = wn; q < 4; q += WN)
#pragma unroll
                for (int m = 0; m < FM; ++m) sums[m] += chunk_sum<DT>(FA.get(sa, m, q));
    };
    const auto arrived = [&] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0): also what goes to LDS by itself
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // The step at c from one pair of buffers.  Fragments are read a quarter ahead of the matrix instructions; before the last quarter's the wave waits for the other
    // pair to be full and for the others to have read this one, so that the next step's first fragments go out under it.  The step after next comes into the
    // pair that this frees, A's part under the last quarter, B's under the next step's first: a CU takes in 16 bytes a lane at 4 lanes a clock, and all
    // of a step's loads at once hold up the matrix instructions behind them (8192 x 4096 x 4096: 250 us, spread 235).  No branch around the loads: it would
    // keep them from between the matrix instructions.
    const int c_whole = FAST ? c_end - (c_end - c_begin) % STEP : c_end;
    const auto step = [&](int c, chunk_t* sa, chunk_t* sb, chunk_t* na, chunk_t* nb) {
        chunk_t va[OpA::N], vb[OpB::N];
        if constexpr (!FAST) {
            A.load(va, c + STEP);
            B.load(vb, c + STEP);
        }
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            read(sa, sb, q + 1);
            if (FAST && q == 0) B.fetch(nb, c + STEP, c_whole);
            multiply_quarter(q);
        }
        add_rows(sa);
        if constexpr (!FAST) {
            A.store(na, va, c + STEP);
            B.store(nb, vb, c + STEP);
        }
        arrived();
        if constexpr (FAST) A.fetch(sa, c + 2 * STEP, c_whole);
        read(na, nb, 0);
        multiply_quarter(3);
    };
    const auto guarded = [&](int c, chunk_t* sa, chunk_t* sb) {
        chunk_t va[OpA::N], vb[OpB::N];
        A.load(va, c);
        B.load(vb, c);
        A.store(sa, va, c);
        B.store(sb, vb, c);
    };
    if (c_begin < c_whole) {
        if constexpr (FAST) {
            A.fetch(a0, c_begin, c_whole);
            B.fetch(b0, c_begin, c_whole);
        } else guarded(c_begin, a0, b0);
        arrived();
        if constexpr (FAST) A.fetch(a1, c_begin + STEP, c_whole);
        read(a0, b0, 0);
        int c = c_begin;
        for (; c + STEP < c_whole; c += 2 * STEP) {
            step(c, a0, b0, a1, b1);
            step(c + STEP, a1, b1, a0, b0);
        }
        if (c < c_whole) step(c, a0, b0, a1, b1);
        arrived();
    }
    if (c_whole < c_end) {   // a step that is not whole
        guarded(c_whole, a0, b0);
        arrived();
        read(a0, b0, 0);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (q < 3) read(a0, b0, q + 1);
            multiply_quarter(q);
        }
        add_rows(a0);
        arrived();
    }

    if (!AA && rows) {   // the halves of a wave, then the waves of a row of waves
        float* s = (float*)b0;
#pragma unroll
        for (int m = 0; m < FM; ++m) {
            const float v = sums[m] + __shfl_xor(sums[m], 32);
            if (lane < 32) s[wn * TM + (wm * FM + m) * 32 + lane] = v;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < TM; i += NT) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < WN; ++w) v += s[w * TM + i];
            if (i0 + i < g.I) {
                if (g.splits > 1) g.part[(int64_t)g.splits * g.I * g.J + split * g.I + i0 + i] = v;
                else store_as(g.row_sum, i0 + i, g.out_dtype, v);
            }
        }
        __syncthreads();
    }
    // A wave's results 32 rows at a time through its own LDS, so that a lane has neighbouring entries of a row: a register of the matrix instruction holds
    // four of them, which would store 32 bytes of a row at a time.
    constexpr int WJ = FN * 32, SLOTS = WJ / 4;
    static_assert(WM * WN / 2 * 32 * SLOTS <= (TM > TN ? TM : TN) * 8, "half the waves' results fit in one buffer");
    chunk_t* stage = (wave < WM * WN / 2 ? (TM > TN ? a0 : b0) : (TM > TN ? a1 : b1)) + (wave % (WM * WN / 2)) * 32 * SLOTS;
    constexpr int PER = WJ / 8;   // lanes of a row
    constexpr int BATCH = FM * FN >= 8 || WJ < 64 ? 2 : 4;   // the large tile's registers are full of results
    const int c8 = lane % PER;
    const int64_t oj = j0 + wn * WJ + c8 * 8;
    const int n8 = (int)max((int64_t)0, min((int64_t)8, g.J - oj));
    float bias[8];
    if (g.bias && n8 > 0) load8<MLMC_F32>(bias, g.bias, oj, n8);
#pragma unroll 1
    for (int mm = 0; mm < FM; ++mm) {   // not unrolled: what follows the stores is long
        const int64_t im = i0 + (wm * FM + mm) * 32;
#pragma unroll
        for (int m = 0; m < FM; ++m) {
            if (m != mm) continue;
#pragma unroll
            for (int n = 0; n < FN; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const v4f v = {acc[m][n][4 * r], acc[m][n][4 * r + 1], acc[m][n][4 * r + 2], acc[m][n][4 * r + 3]};
                    const int slot = n * 8 + r * 2 + (lane >> 5), i = lane & 31;
                    stage[i * SLOTS + (slot ^ (i & 7))] = __builtin_bit_cast(chunk_t, v);
                }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        const auto rows_of = [&](int p, auto batch, auto cut) __attribute__((always_inline)) {
            constexpr int K = decltype(batch)::value;
            const int n = decltype(cut)::value ? n8 : 8;
            float v[K][8];
            Epilogue ep[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int i = (p + k) * (64 / PER) + lane / PER;
                const v4f v0 = __builtin_bit_cast(v4f, stage[i * SLOTS + ((2 * c8) ^ (i & 7))]), v1 = __builtin_bit_cast(v4f, stage[i * SLOTS + ((2 * c8 + 1) ^ (i & 7))]);
#pragma unroll
                for (int e = 0; e < 4; ++e) { v[k][e] = v0[e]; v[k][4 + e] = v1[e]; }
                if (g.splits == 1 && im + i < g.I && n8 > 0) ep[k].template load<DT>(g, im + i, oj, n);
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int64_t oi = im + (p + k) * (64 / PER) + lane / PER;
                if (oi >= g.I || n8 <= 0) continue;
                if (g.splits > 1) store8(v[k], g.part, ((int64_t)split * g.I + oi) * g.J + oj, n, MLMC_F32);
                else ep[k].template finish<DT>(g, oi, oj, v[k], bias, n);
            }
        };
        if (j0 + TN <= g.J) {
#pragma unroll 1
            for (int p = 0; p < WJ / 16; p += BATCH) rows_of(p, std::integral_constant<int, BATCH>{}, std::false_type{});
        } else {
#pragma unroll 1
            for (int p = 0; p < WJ / 16; ++p) rows_of(p, std::integral_constant<int, 1>{}, std::true_type{});
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// The sums of the contraction's parts, in their order, and the epilogue.
template <int DT> __global__ __launch_bounds__(256) void k_linear_join(LinearArgs g) {
    const int64_t per_row = (g.J + 7) / 8, t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= g.I * per_row) {
        const int64_t i = t - g.I * per_row;
        if (g.row_sum && i < g.I) {
            float v = 0.f;
            for (int s = 0; s < g.splits; ++s) v += g.part[(int64_t)g.splits * g.I * g.J + s * g.I + i];
            store_as(g.row_sum, i, g.out_dtype, v);
        }
        return;
    }
    const int64_t i = t / per_row, j = (t - i * per_row) * 8;
    const int n = (int)min((int64_t)8, g.J - j);
    float v[8] = {};
    for (int s = 0; s < g.splits; ++s) {
        float u[8];
        load8<MLMC_F32>(u, g.part, ((int64_t)s * g.I + i) * g.J + j, n);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += u[e];
    }
    float bias[8];
    if (g.bias) load8<MLMC_F32>(bias, g.bias, j, n);
    Epilogue ep;
    ep.load<DT>(g, i, j, n);
    ep.finish<DT>(g, i, j, v, bias, n);
}

// The forward product of up to 16 rows: bound by reading the weight once.  A workgroup has 16 outputs, its waves share the contraction and each has many
// 16-byte loads in flight, straight into the registers of the matrix instructions (16 x 16): no LDS, no second launch.  One row of 4096 x 4096 bf16, 33.6 MB: 8.6 us,
// a call again and again 8.1 to 10.4 (by tiles in parts, with the join, 12.6).
constexpr int FEW_ROWS = 16, FEW_WAVES = 8, FEW_DEPTH = 8;
template <int DT, bool WIDE> __global__ __launch_bounds__(FEW_WAVES * 64) void k_linear_few(LinearArgs g) {
    constexpr int E = DT == MLMC_BF16 ? 8 : 4, STEP = 4 * E;   // entries of the contraction a load of a wave covers, 64 bytes of each of 16 rows
    __shared__ float part[FEW_WAVES][FEW_ROWS][FEW_ROWS + 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, chunk = lane >> 4;
    const int64_t j0 = (int64_t)blockIdx.x * 16, jr = min(j0 + r, g.J - 1);
    const bool row = r < g.I;
    v4f acc = {0.f, 0.f, 0.f, 0.f};
    const auto product = [&](chunk_t w, chunk_t x) {
        if constexpr (DT == MLMC_BF16) {
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, w), __builtin_bit_cast(v8b, x), acc, 0, 0, 0);
        } else {
            const v4f u = __builtin_bit_cast(v4f, w), v = __builtin_bit_cast(v4f, x);
#pragma unroll
            for (int k = 0; k < 4; ++k) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(u[k], v[k], acc, 0, 0, 0);
        }
    };
    const char* pw = (const char*)((const entry_t<DT>*)g.b + jr * g.ldb + chunk * E);
    const char* px = (const char*)((const entry_t<DT>*)g.a + (row ? r : 0) * g.lda + chunk * E);
    const int C = (int)g.C, whole = C / STEP;   // C is at most 2^21
    constexpr chunk_t zero = {0, 0, 0, 0};
    for (int s = wave; s < whole; s += FEW_WAVES * FEW_DEPTH) {
        chunk_t w[FEW_DEPTH], x[FEW_DEPTH];
#pragma unroll
        for (int u = 0; u < FEW_DEPTH; ++u) {
            const int at = s + u * FEW_WAVES;
            const bool in = at < whole;
            w[u] = in ? (chunk_t) * (const chunk_u*)(pw + (int64_t)at * 64) : zero;
            x[u] = in && row ? (chunk_t) * (const chunk_u*)(px + (int64_t)at * 64) : zero;
        }
#pragma unroll
        for (int u = 0; u < FEW_DEPTH; ++u) product(w[u], x[u]);
    }
    if (wave == FEW_WAVES - 1 && whole * STEP < C) {   // the rest
        const int64_t c = whole * STEP + chunk * E;
        const chunk_t w = cut_chunk<DT, WIDE>(raw_chunk<DT, WIDE>(g.b, g.ldb, jr, g.J, c, C), jr, g.J, c, C);
        const chunk_t x = cut_chunk<DT, WIDE>(raw_chunk<DT, WIDE>(g.a, g.lda, r, g.I, c, C), r, g.I, c, C);
        product(w, x);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) part[wave][r][chunk * 4 + k] = acc[k];
    __syncthreads();
    const int64_t i = threadIdx.x >> 4, j = j0 + (threadIdx.x & 15);
    if (threadIdx.x >= 256 || i >= g.I || j >= g.J) return;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < FEW_WAVES; ++w) v += part[w][i][threadIdx.x & 15];
    if (g.bias) v += g.bias[j];
    if (g.z) store_as(g.z, i * g.ldz + j, DT, v);
    if (g.act == MLMC_ACT_GELU) v = gelu<DT>(v);
    else if (g.act == MLMC_ACT_RELU) v = relu(v);
    if (g.residual) v += to_f32(((const entry_t<DT>*)g.residual)[i * g.ldr + j]);
    store_as(g.out, i * g.ldo + j, DT, v);
}

template <int DT> static mlmc_status linear_few(const LinearArgs& g, hipStream_t st) {
    const unsigned grid = (unsigned)((g.J + 15) / 16);
    if (g.C >= (DT == MLMC_BF16 ? 8 : 4)) MLMC_LAUNCH(K_LINEAR_FEW, st, (k_linear_few<DT, true><<<grid, FEW_WAVES * 64, 0, st>>>(g)));
    else MLMC_LAUNCH(K_LINEAR_FEW, st, (k_linear_few<DT, false><<<grid, FEW_WAVES * 64, 0, st>>>(g)));
    return MLMC_OK;
}

// The tiles: rows and columns; microseconds of a step of a tile that has a CU to itself, of one among others, of the beginning and end of a round of tiles.
// Fitted to sweeps of tiles and parts, microseconds of the best of either side: 2048 x 2048 x 2048 bf16, tiles 32 / 64 / 128 / 256: 34 / 25 / 28 / 43; 4096 x 1024 over
// 8192: 166 / 97 / 84 (2 parts) / 83 (4); 1 x 4096 x 4096: 13.1 (8 parts) / 13.5 / 14.1 / 20.5; 4096 x 4096 x 512: 39 / 34 / 32 / 28; 200 x 8192 x 2048: 20 / 22 / 23 / 31;
// fp32 512 x 512 over 8192: 43 (8) / 43 (8) / 47 (16); 1000 x 2049 x 1537: 91 (2) / 87 (4) / 86 (3); 2048 x 2048 x 2048: 139 / 129 / 126.
enum LinearTile { TILE_32 = 0, TILE_64, TILE_128, TILE_256, TILES };
struct TileCost { int rows, cols; float alone_us[2], among_us[2], round_us; };   // [dtype]
constexpr TileCost tile_costs[TILES] = {{32, 128, {0.55f, 0.42f}, {0.53f, 0.28f}, 0.7f}, {64, 128, {0.95f, 0.44f}, {0.95f, 0.33f}, 1.3f},
                                        {128, 128, {1.85f, 0.70f}, {1.85f, 0.50f}, 2.5f}, {256, 256, {0.f, 1.50f}, {0.f, 1.60f}, 11.f}};
constexpr float LAUNCH_US = 5.f, JOIN_US = 3.f, JOIN_ENTRY_US = 1.6e-6f;
constexpr int LINEAR_CUS = 256, SPLITS_MAX = 32;

struct LinearPlan { int tile, splits, split_len; float us; };

// The tile and the number of parts of the contraction that the costs above say to be the fastest: tiles come in rounds of one for every CU, a part more
// makes the rounds finer and the join longer.
static LinearPlan linear_plan(int64_t I, int64_t J, int64_t C, int dtype, bool fast) {
    const int step = dtype == MLMC_BF16 ? 64 : 32;
    const int64_t steps = (C + step - 1) / step;
    LinearPlan best = {TILE_128, 1, (int)C, 0.f};
    float least = 3.0e38f;
    for (int t = 0; t < TILES; ++t) {
        if (t == TILE_256 && (dtype != MLMC_BF16 || !fast)) continue;
        const TileCost& k = tile_costs[t];
        const int64_t tiles = ((I + k.rows - 1) / k.rows) * ((J + k.cols - 1) / k.cols);
        for (int s = 1; s <= SPLITS_MAX && (s == 1 || (s * 2 <= steps && tiles * (s - 1) < 2 * LINEAR_CUS)); ++s) {
            const int64_t len = (steps + s - 1) / s, parts = steps ? (steps + len - 1) / len : 1, rounds = (tiles * parts + LINEAR_CUS - 1) / LINEAR_CUS;
            if (parts != s) continue;
            const float us = LAUNCH_US + (float)rounds * (k.round_us + (float)len * (rounds == 1 ? k.alone_us : k.among_us)[dtype]) +
                             (s > 1 ? JOIN_US + JOIN_ENTRY_US * (float)(s * I) * (float)J : 0.f);
            if (us < least) {
                least = us;
                best = {t, s, (int)(len * step), us};
            }
        }
    }
    return best;
}
// Whether k_linear_few takes a forward product: its workgroups read 16 rows of the weight each, at 30 KB a us by itself and 5 TB/s in all, and with few outputs there are few of them
// (time of a call, and by tiles in parts: 5 x 512 x 7104 fp32 22.8 us and 17.3, 9 x 295 x 3200 13.4 and 17.7; bf16 1 x 1024 x 4096 7.5 and 14.5, 4 x 256 x 8192 11.8 and 14.9,
// 16 x 4096 x 4096 10.4 and 11.7, 1 x 8192 x 8192 27.2 and 24.6).  The costs of tiles have no term for memory, so that beyond those sizes they promise tiles less than the weight's bytes
// take, and the rule goes to tiles (weights in turn, more than the caches hold; 1 row of 4096 inputs: 11008 outputs 18.8 and 21.6, 14336 23.9 and 25.6, 32000 45.7 and 64.0,
// 131072 169.6 and 176.4; 16 rows: 26.7 and 22.0, where it stays with the few, 32000 65.4 and 65.7, 131072 251 and 182; 4 x 50021 x 512 16.0 and 12.3, where it stays;
// fp32 1 x 32000 x 1024 29.0 and 36.9): at one row it gives away up to two fifths, at 16 it is right for the longest.
static bool few_rows(int64_t I, int64_t J, int64_t C, int dtype) {
    if (I > FEW_ROWS) return false;
    const float row = (float)C * (dtype == MLMC_BF16 ? 2.f : 4.f), alone = 16.f * row / 3.0e4f, all = (float)J * row / 5.0e6f;
    return LAUNCH_US + (alone > all ? alone : all) <= linear_plan(I, J, C, dtype, false).us + 6.f;   // small calls wait for the second launch longer than it takes
}
static size_t linear_part_bytes(const LinearPlan& p, int64_t I, int64_t J) { return p.splits > 1 ? (size_t)p.splits * (size_t)(I * J + I) * sizeof(float) : 0; }

template <int DT, int WM, int WN, int FM, int FN, bool AA, bool BA, int WAY> static mlmc_status launch_tile(LinearArgs& g, hipStream_t st) {
    constexpr int TM = WM * FM * 32, TN = WN * FN * 32;
    g.tiles_i = (int)((g.I + TM - 1) / TM);
    g.tiles_j = (int)((g.J + TN - 1) / TN);
    const unsigned grid = (unsigned)((int64_t)g.tiles_i * g.tiles_j * g.splits);
    MLMC_LAUNCH(K_LINEAR, st, (k_linear_tile<DT, WM, WN, FM, FN, AA, BA, WAY><<<grid, WM * WN * 64, 0, st>>>(g)));
    if (g.splits > 1) {
        const unsigned groups = (unsigned)((g.I * ((g.J + 7) / 8) + g.I + 255) / 256);
        MLMC_LAUNCH(K_LINEAR_JOIN, st, (k_linear_join<DT><<<groups, 256, 0, st>>>(g)));
    }
    return MLMC_OK;
}

// The way of an operand: aligned chunks or words, which across the contraction have to lie inside the matrix or outside (along it, whole steps do); offsets within a tile have to
// fit 32 bits for either.
static int operand_way(const void* p, int64_t ld, int64_t width, bool along, int esize) {
    const int E = 16 / esize;
    if (ld > ((int64_t)1 << 22) / esize) return WAY_REGISTERS;
    if ((uintptr_t)p % 16 == 0 && ld % E == 0 && width >= E && (along || width % E == 0)) return WAY_CHUNKS;
    return (uintptr_t)p % 4 == 0 && ld % (E / 4) == 0 && (along || width % (E / 4) == 0) ? WAY_WORDS : WAY_REGISTERS;
}

// bf16 matrices whose rows are no multiple of 16 bytes are copied to ones that are (zeros behind the rows) where the copy costs less than the slower ways: measured, those take
// `slower` times what the tiles' costs say.  Forward, input gradient, weight gradient, us, through registers / by a copy and chunks: 4096 x 4095 x 4097 218 / 152, 304 / 201, 322 / 198;
// 1001 x 1999 x 1535 23 / 20, 48 / 32, 32 / 26; 12175 x 1037 x 613 50 / 48, 50 / 44, 73 / 52.
struct PackPlan { bool pack; LinearPlan plan; size_t bytes[2]; };
static size_t packed_bytes(int64_t rows, int64_t cols) { return (size_t)rows * (size_t)((cols + 7) / 8) * 16; }
static PackPlan pack_plan(int64_t I, int64_t J, int64_t C, bool aa, bool ba, int way, bool pack_a, bool pack_b) {
    PackPlan r = {false, linear_plan(I, J, C, MLMC_BF16, false), {0, 0}};
    const int64_t a_cols = aa ? C : I, a_rows = aa ? I : C, b_cols = ba ? C : J, b_rows = ba ? J : C;
    if ((a_cols % 8 == 0 && b_cols % 8 == 0) || a_cols < 8 || b_cols < 8 || a_rows * ((a_cols + 7) / 8) >= ((int64_t)1 << 30) || b_rows * ((b_cols + 7) / 8) >= ((int64_t)1 << 30)) return r;
    const LinearPlan fast = linear_plan(I, J, C, MLMC_BF16, true);
    const size_t a = pack_a ? packed_bytes(a_rows, a_cols) : 0, b = pack_b ? packed_bytes(b_rows, b_cols) : 0;
    const float slower = way == WAY_WORDS || (aa && ba) ? 1.5f : 2.1f, copy_us = LAUNCH_US + 2.0f * (float)(a + b) / 3.0e6f;
    if (fast.us + copy_us >= slower * r.plan.us) return r;
    r = {true, fast, {a, b}};
    return r;
}
static size_t align256(size_t n) { return (n + 255) / 256 * 256; }

struct PackArgs { const void* from[2]; int64_t ld[2], rows[2], cols[2]; chunk_t* to[2]; unsigned groups_a; };
__global__ __launch_bounds__(256) void k_linear_pack(PackArgs p) {
    const int which = blockIdx.x >= p.groups_a;
    const unsigned per_row = (unsigned)((p.cols[which] + 7) / 8), t = (blockIdx.x - (which ? p.groups_a : 0)) * 256 + threadIdx.x;
    const unsigned r = t / per_row, c = t - r * per_row;
    if (r >= p.rows[which]) return;
    const chunk_t v = raw_chunk<MLMC_BF16, true>(p.from[which], p.ld[which], r, p.rows[which], (int64_t)c * 8, p.cols[which]);
    p.to[which][t] = cut_chunk<MLMC_BF16, true>(v, r, p.rows[which], (int64_t)c * 8, p.cols[which]);
}

template <int DT, bool AA, bool BA, int WAY> static mlmc_status linear_tile(LinearArgs& g, int tile, hipStream_t st) {
    if constexpr (DT == MLMC_BF16 && WAY == WAY_CHUNKS)
        if (tile == TILE_256) return launch_tile<DT, 2, 4, 4, 2, AA, BA, WAY>(g, st);
    if (tile == TILE_128) return launch_tile<DT, 2, 2, 2, 2, AA, BA, WAY>(g, st);
    if (tile == TILE_64) return launch_tile<DT, 1, 4, 2, 1, AA, BA, WAY>(g, st);
    return launch_tile<DT, 1, 4, 1, 1, AA, BA, WAY>(g, st);
}

template <int DT, bool AA, bool BA> static mlmc_status linear_layout(LinearArgs g, hipStream_t st) {
    constexpr int esize = DT == MLMC_BF16 ? 2 : 4;
    const int wa = operand_way(g.a, g.lda, AA ? g.C : g.I, AA, esize), wb = operand_way(g.b, g.ldb, BA ? g.C : g.J, BA, esize);
    int way = wa == WAY_REGISTERS || wb == WAY_REGISTERS ? WAY_REGISTERS : wa == WAY_CHUNKS && wb == WAY_CHUNKS ? WAY_CHUNKS : WAY_WORDS;
    LinearPlan p;
    size_t packed[2] = {0, 0};
    if (DT == MLMC_BF16 && way != WAY_CHUNKS && g.C > 0) {
        const PackPlan k = pack_plan(g.I, g.J, g.C, AA, BA, way, wa != WAY_CHUNKS, wb != WAY_CHUNKS);
        p = k.plan;
        if (k.pack) {
            way = WAY_CHUNKS;
            packed[0] = k.bytes[0];
            packed[1] = k.bytes[1];
        }
    } else p = linear_plan(g.I, g.J, g.C, DT, way == WAY_CHUNKS);
    g.splits = p.splits;
    g.split_len = p.split_len;
    const size_t parts = align256(linear_part_bytes(p, g.I, g.J)), need = parts + align256(packed[0]) + packed[1];
    if (need && (!g.part || (uintptr_t)g.part % 256 || g.ws_bytes < need)) return MLMC_EINVAL;
    if (packed[0] || packed[1]) {
        char* to = (char*)g.part + parts;
        PackArgs k = {{g.a, g.b}, {g.lda, g.ldb}, {AA ? g.I : g.C, BA ? g.J : g.C}, {AA ? g.C : g.I, BA ? g.C : g.J}, {(chunk_t*)to, (chunk_t*)(to + align256(packed[0]))}, 0};
        const unsigned groups_b = (unsigned)((packed[1] / 16 + 255) / 256);
        k.groups_a = (unsigned)((packed[0] / 16 + 255) / 256);
        MLMC_LAUNCH(K_LINEAR_PACK, st, (k_linear_pack<<<k.groups_a + groups_b, 256, 0, st>>>(k)));
        if (packed[0]) { g.a = k.to[0]; g.lda = (k.cols[0] + 7) / 8 * 8; }
        if (packed[1]) { g.b = k.to[1]; g.ldb = (k.cols[1] + 7) / 8 * 8; }
    }
    if (way == WAY_CHUNKS) return linear_tile<DT, AA, BA, WAY_CHUNKS>(g, p.tile, st);
    if (way == WAY_WORDS) return linear_tile<DT, AA, BA, WAY_WORDS>(g, p.tile, st);
    return linear_tile<DT, AA, BA, WAY_REGISTERS>(g, p.tile, st);
}

template <bool AA, bool BA> static mlmc_status linear_run(const LinearArgs& g, int dtype, hipStream_t st) {
    return dtype == MLMC_F32 ? linear_layout<MLMC_F32, AA, BA>(g, st) : linear_layout<MLMC_BF16, AA, BA>(g, st);
}

// Sizes go up to this: indices of the contraction, two steps past its end, and numbers of tiles are int, offsets in a tile of copied rows (4 MB each) 32 bits; a product whose matrices fit
// in memory has at most 2^31 threads.
constexpr int64_t LINEAR_ROWS_MAX = (int64_t)1 << 21;
static bool linear_sizes_ok(int64_t n, int64_t m, int64_t k) {
    return n >= 0 && n <= LINEAR_ROWS_MAX && m >= 1 && m <= LINEAR_ROWS_MAX && k >= 1 && k <= LINEAR_ROWS_MAX;
}
static bool act_ok(int act) { return act == MLMC_ACT_NONE || act == MLMC_ACT_RELU || act == MLMC_ACT_GELU; }

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
                const PackPlan k = pack_plan(size[c][0], size[c][1], size[c][2], c < 2, c == 0, way, which & 1, which & 2);
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
