// Linear layer of matrices in 8 bits with a scale for every row (entry point mlmc_linear_q8): y = act((x_scale_n w_scale_m) x W^T + b) + r.
//
// The tiles, ways and epilogue are those of the linear layer (mlmc_linear.h).  A step of 128 bytes has 128 entries of the contraction instead of 64, and the matrix instructions for 8 bits
// take twice as many in the same time, so that loads and products keep their proportion.  Those instructions add the products of eight entries with what lies within 12 binary
// places of the greatest of them and cut the rest (measured: a product 2^-12 of the greatest is kept, one of 2^-14 lost): 1.5e-5 of a result of normal entries, a hundredth of its rounding to 16 bits.
// Accumulators are fp32.
#include "mlmc_linear.h"

namespace mlmc {

// The large tile of matrices whose rows are aligned: 256 x 256 by 4 waves of 128 x 128, a workgroup for every CU with tile after tile, the first loads of the next one ahead of the stores of the last.
// Loads and barriers as in k_linear_tile; a wave's fragments of the next half step are read over those of this one, A's as soon as its instructions have gone out.
// 8192 x 4096 x 4096: 107 to 119 us by the card's clock (2.57 to 2.31 PFLOP/s; a library product without the epilogue 89 to 98), with gelu 121 to 136; by 8 waves of 128 x 64 (k_linear_tile) 20 more; by two workgroups a CU, 128 x 256 each and
// steps of 64 bytes, 45 more: half as much again comes from the L2.
constexpr int BIG = 256, BIG_T = 256, BIG_F = 4, AHEAD = 2;   // (a thread for every row of the tile)
using v2b = __bf16 __attribute__((ext_vector_type(2)));

// Chunk k of lane l of four becomes chunk l of lane k.
__device__ inline void transpose_fours(chunk_t (&c)[4], int lane) {
    const auto from = [](int v, auto ctrl) { return __builtin_amdgcn_update_dpp(v, v, decltype(ctrl)::value, 0xF, 0xF, false); };
    constexpr std::integral_constant<int, 0xB1> next;   // lanes 2k and 2k + 1
    constexpr std::integral_constant<int, 0x4E> pair;   // the pairs of four
    const bool one = lane & 1, two = lane & 2;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        int v[4] = {c[0][d], c[1][d], c[2][d], c[3][d]}, u[4];
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
            const int a = from(v[k], next), b = from(v[k + 1], next);   // by all lanes, ahead of the choice
            u[k] = one ? b : v[k];
            u[k + 1] = one ? v[k + 1] : a;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int a = from(u[k], pair), b = from(u[k + 2], pair);
            c[k][d] = two ? b : u[k];
            c[k + 2][d] = two ? u[k + 2] : a;
        }
    }
}

__global__ __launch_bounds__(BIG_T, 1) void k_linear_q8(LinearArgs g) {
    using Op = Operand<DT_E4M3, true, BIG, BIG_T, WAY_CHUNKS>;
    constexpr int STEP = Op::STEP, F = BIG_F;
    __shared__ chunk_t a0[BIG * 8], b0[BIG * 8], a1[BIG * 8], b1[BIG * 8];
    __shared__ __align__(16) float scales[BIG], biases[BIG];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1, half = lane >> 5;
    const auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    const auto fresh_thread = [] {   // what follows from it is not kept in registers through the loop
        int t = threadIdx.x;
        asm volatile("" : "+v"(t));
        return t;
    };
    const int tiles = g.tiles_i * g.tiles_j, C = (int)g.C, c_whole = C - C % STEP;
    Op A, B;
    int64_t i0, j0;
    const auto place = [&](int k) {   // neighbouring tiles to the workgroups of one die (workgroups go round the 8 dies), eight tile rows at a time
        const int q = tiles / 8, r = tiles % 8, x = k & 7, t = x * q + (x < r ? x : r) + (k >> 3);
        const int band = uniform(t / (8 * g.tiles_j)), in_band = t - band * 8 * g.tiles_j, high = min(8, g.tiles_i - band * 8);
        const int tj = uniform(in_band / high), ti = band * 8 + in_band - tj * high;
        i0 = (int64_t)ti * BIG;
        j0 = (int64_t)tj * BIG;
        const int thread = fresh_thread();
        A.init(g.a, g.lda, i0, g.I, g.C, thread);
        B.init(g.b, g.ldb, j0, g.J, g.C, thread);
    };
    v16f acc[F][F];
    Fragments<DT_E4M3, true, BIG, F> FA;
    FA.init(wm * F);
    // B's fragments in pairs, of 64 columns: n even has columns 0 to 15 and 32 to 47, n odd the others, so that in the end a lane's results of a pair are 32 neighbouring ones
    int place_b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) place_b[k] = Op::L::slot(wn * 128 + (lane & 16) * 2 + (lane & 15), k * 2 + half);
    const auto fragment_b = [&](const chunk_t* s, int n, int q) {
        const int at = ((n >> 1) * 64 + (n & 1) * 16) * 8;
        return __builtin_shufflevector(s[place_b[2 * q] + at], s[place_b[2 * q + 1] + at], 0, 1, 2, 3, 4, 5, 6, 7);
    };
    v8i fa[F], fb[2][F];
    const auto read = [&](const chunk_t* sa, const chunk_t* sb) {
#pragma unroll
        for (int n = 0; n < F; ++n) fb[0][n] = fragment_b(sb, n, 0);
#pragma unroll
        for (int m = 0; m < F; ++m) fa[m] = FA.get(sa, m, 0);
    };
    // the products of half q of a step; the other half of a pair of buffers is read meanwhile, if there is more
    const auto multiply_half = [&](int q, auto more, const chunk_t* sa, const chunk_t* sb) __attribute__((always_inline)) {
        constexpr bool MORE = decltype(more)::value;
#pragma unroll
        for (int n = 0; n < F; ++n)
            if (MORE) fb[1 - q][n] = fragment_b(sb, n, 1 - q);
#pragma unroll
        for (int m = 0; m < F; ++m) {
#pragma unroll
            for (int n = 0; n < F; ++n) acc[m][n] = multiply<DT_E4M3>(fb[q][n], fa[m], acc[m][n]);
            if (MORE) fa[m] = FA.get(sa, m, 1 - q);
        }
#pragma unroll
        for (int i = 0; i < F * F; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x10, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr std::true_type more;
    const auto arrived = [&] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0): also what goes to LDS by itself
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    const auto step = [&](int c, chunk_t* sa, chunk_t* sb, chunk_t* na, chunk_t* nb) {
        B.fetch(nb, c + STEP, c_whole);
        multiply_half(0, more, sa, sb);
        arrived();
        A.fetch(sa, c + 2 * STEP, c_whole);
        multiply_half(1, more, na, nb);
    };
    int k = blockIdx.x;
    place(k);
    A.fetch(a0, 0, c_whole);
    B.fetch(b0, 0, c_whole);
    while (true) {
        {
            const int64_t j = min(j0 + threadIdx.x, g.J - 1);
            scales[threadIdx.x] = g.col_scale[j];
            biases[threadIdx.x] = g.bias ? g.bias[j] : 0.f;
        }
#pragma unroll
        for (int m = 0; m < F; ++m)
#pragma unroll
            for (int n = 0; n < F; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[m][n][r] = 0.f;
        arrived();
        A.fetch(a1, STEP, c_whole);
        read(a0, b0);
        int c = 0;
        for (; c + STEP < c_whole; c += 2 * STEP) {
            step(c, a0, b0, a1, b1);
            step(c + STEP, a1, b1, a0, b0);
        }
        if (c < c_whole) step(c, a0, b0, a1, b1);
        arrived();
        if (c_whole < C) {   // a step that is not whole
            const int t = fresh_thread();
            const int left = C - c_whole, cut = c_whole + left / 16 * 16, slot = Op::L::slot(t, left / 16);
            A.fetch_rest(a0, c_whole, left, t);
            B.fetch_rest(b0, c_whole, left, t);
            arrived();
            if (left % 16) {   // the chunk that the end cuts, a row a thread
                const chunk_t u = raw_chunk<DT_E4M3, true>(g.a, g.lda, i0 + t, g.I, cut, C), v = raw_chunk<DT_E4M3, true>(g.b, g.ldb, j0 + t, g.J, cut, C);
                a0[slot] = cut_chunk<DT_E4M3, true>(u, i0 + t, g.I, cut, C);
                b0[slot] = cut_chunk<DT_E4M3, true>(v, j0 + t, g.J, cut, C);
                arrived();
            }
            read(a0, b0);
            multiply_half(0, more, a0, b0);
            multiply_half(1, std::false_type{}, a0, b0);
            arrived();
        }
        const int64_t i0_done = i0, oi = i0 + wm * 128 + (lane & 31), oj = j0 + wn * 128;
        float rs[F];   // ahead of the next tile's loads: what is waited for comes in order
#pragma unroll
        for (int m = 0; m < F; ++m) rs[m] = g.row_scale[min(oi + m * 32, g.I - 1)];
        // A lane has four neighbouring entries of a row in four registers (the operands are exchanged).  Rounded and exchanged between the halves of the wave they are 64 bytes of a pair of fragments,
        // and transposed among four lanes, 16 bytes each of the 64 of one row: a store has whole sectors of 16 rows.  (16 bytes of each of 64 places a store: 126 us instead of 115, and twice
        // the bytes written to HBM; by way of LDS the waits of the one wave a SIMD took more than that gave.)
        // The residual comes the same way back, loaded two blocks of 32 rows and 64 columns ahead of its use (more spill registers; by way of the free pair of buffers all of it took half as long again).
        // 8192 x 4096 x 4096 with residual 136 us (by 8 bytes a lane of 32 rows, without loads ahead, 150), 4000 x 4001 x 1072 50 (86).
        const int64_t is = i0_done + wm * 128 + (lane & 28), js = oj + half * 32 + (lane & 3) * 8;
        chunk_t ahead[AHEAD][4];
        const auto load_residual = [&](int block) __attribute__((always_inline)) {
            const int p = block / F, m = block % F;
            const int left = (int)min(g.J - js - p * 64, (int64_t)8);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const __bf16* from = (const __bf16*)g.residual + min(is + m * 32 + r, g.I - 1) * g.ldr + js + p * 64;
                if (left == 8) ahead[block % AHEAD][r] = *(const chunk_u*)from;
                else {
                    v8b u = {};
#pragma unroll
                    for (int e = 0; e < 7; ++e)
                        if (e < left) u[e] = from[e];
                    ahead[block % AHEAD][r] = __builtin_bit_cast(chunk_t, u);
                }
            }
        };
        if (g.residual) {
#pragma unroll
            for (int b = 0; b < AHEAD; ++b) load_residual(b);
        }
        k += gridDim.x;
        const bool again = k < tiles;
        if (again) {
            place(k);
            A.fetch(a0, 0, c_whole);
            B.fetch(b0, 0, c_whole);
        }
        const auto results = [&](auto act, auto residual) __attribute__((always_inline)) {
            constexpr int ACT = decltype(act)::value;
            constexpr bool RES = decltype(residual)::value;
            __bf16* const y = (__bf16*)g.out + is * g.ldo + js;
#pragma unroll
            for (int p = 0; p < F / 2; ++p)
#pragma unroll
                for (int m = 0; m < F; ++m) {
                    __builtin_amdgcn_sched_barrier(0);   // one after the other: there are no registers for more
                    chunk_t out[4], add[4];
                    if (RES) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) add[r] = ahead[(p * F + m) % AHEAD][r];
                        transpose_fours(add, lane);
                        if (p * F + m + AHEAD < F * F / 2) load_residual(p * F + m + AHEAD);
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int n = 2 * p + k;
                        unsigned packed[4][2], added[4][2];
                        if (RES) {
#pragma unroll
                            for (int h = 0; h < 2; ++h)
#pragma unroll
                                for (int w = 0; w < 2; ++w) {
                                    const auto both = __builtin_amdgcn_permlane32_swap(add[2 * k + h][w], add[2 * k + h][2 + w], false, false);
                                    added[h][w] = both[0];
                                    added[2 + h][w] = both[1];
                                }
                        }
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int col = p * 64 + (q >> 1) * 32 + k * 16 + (q & 1) * 8 + half * 4;
                            const v4f cs = *(const v4f*)(scales + wn * 128 + col), bs = *(const v4f*)(biases + wn * 128 + col);
                            float v[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                v[e] = fmaf(acc[m][n][q * 4 + e], rs[m] * cs[e], bs[e]);
                                if (ACT == MLMC_ACT_GELU) v[e] = gelu<MLMC_BF16>(v[e]);
                                if (ACT == MLMC_ACT_RELU) v[e] = relu(v[e]);
                                if (RES) v[e] += (float)__builtin_bit_cast(v2b, added[q][e / 2])[e & 1];
                            }
#pragma unroll
                            for (int w = 0; w < 2; ++w) packed[q][w] = __builtin_bit_cast(unsigned, v2b{(__bf16)v[2 * w], (__bf16)v[2 * w + 1]});
                        }
#pragma unroll
                        for (int h = 0; h < 2; ++h)   // lanes 0 to 31 get the first sixteen columns, the others the second
#pragma unroll
                            for (int w = 0; w < 2; ++w) {
                                const auto both = __builtin_amdgcn_permlane32_swap(packed[h][w], packed[2 + h][w], false, false);
                                out[2 * k + h][w] = (int)both[0];
                                out[2 * k + h][2 + w] = (int)both[1];
                            }
                    }
                    transpose_fours(out, lane);
                    const int left = (int)min(g.J - js - p * 64, (int64_t)8);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (is + m * 32 + r >= g.I) continue;
                        __bf16* to = y + (m * 32 + r) * g.ldo + p * 64;
                        if (left == 8) *(chunk_u*)to = out[r];
                        else {
                            const v8b u = __builtin_bit_cast(v8b, out[r]);
#pragma unroll
                            for (int e = 0; e < 7; ++e)
                                if (e < left) to[e] = u[e];
                        }
                    }
                }
        };
        const auto results_of = [&](auto act) __attribute__((always_inline)) {
            if (g.residual) results(act, std::true_type{});
            else results(act, std::false_type{});
        };
        if (g.act == MLMC_ACT_GELU) results_of(std::integral_constant<int, MLMC_ACT_GELU>{});
        else if (g.act == MLMC_ACT_RELU) results_of(std::integral_constant<int, MLMC_ACT_RELU>{});
        else results_of(std::integral_constant<int, MLMC_ACT_NONE>{});
        if (!again) return;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();   // scales and biases have been read
        asm volatile("" ::: "memory");
    }
}

static mlmc_status linear_q8_big(LinearArgs& g, hipStream_t st) {
    g.tiles_i = (int)((g.I + BIG - 1) / BIG);
    g.tiles_j = (int)((g.J + BIG - 1) / BIG);
    const int tiles = g.tiles_i * g.tiles_j;
    MLMC_LAUNCH(K_LINEAR_Q8, st, (k_linear_q8<<<tiles < LINEAR_CUS ? tiles : LINEAR_CUS, BIG_T, 0, st>>>(g)));
    return MLMC_OK;
}

}  // namespace mlmc

using namespace mlmc;

extern "C" {

size_t mlmc_linear_q8_workspace(int64_t rows, int64_t outputs, int64_t inputs) {
    if (!linear_sizes_ok(rows, outputs, inputs) || rows == 0 || few_rows(rows, outputs, inputs, DT_E4M3)) return 0;
    size_t most = 0;
    for (int epilogue = 0; epilogue < 4; ++epilogue) {
        for (bool fast : {false, true}) {
            const size_t need = align256(linear_part_bytes(linear_plan(rows, outputs, inputs, DT_E4M3, fast, epilogue), rows, outputs));
            most = need > most ? need : most;
        }
        for (int which = 1; which < 4; ++which) {
            const PackPlan k = pack_plan(rows, outputs, inputs, DT_E4M3, true, true, WAY_REGISTERS, which & 1, which & 2, epilogue);
            const size_t need = align256(linear_part_bytes(k.plan, rows, outputs)) + align256(k.bytes[0]) + k.bytes[1];
            most = need > most ? need : most;
        }
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
