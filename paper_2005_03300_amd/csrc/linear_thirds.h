// Products of fp32 matrices on the bf16 matrix units.  An fp32 number is the sum of three bf16 numbers exactly (x = h + m + l: each the nearest bf16 number to
// what is left, 8 + 8 + 8 bits), and the product of two such sums has nine products of bf16 numbers, which the matrix unit multiplies exactly and adds in fp32.  Three of the
// nine are left out: m l' and l m', at most 2^-25 of x x' each, and l l', at most 2^-34; together they are up to 2^-24 of it, as the rounding of an fp32 product is, and
// 2^-27.5 in the root mean square over random mantissas.  The other six take 96 cycles for what the fp32 units
// take 256 for.  8192 x 8192 x 8192 takes 5.2 ms (210 TFLOP/s; on the fp32 units at most 157, the library's product 151), 232965 x 602 x 128 270 us.
// Infinities and NaN have no such sum, nor have numbers that round to infinity as bf16: with them m, and with it the result, is NaN; and a finite product of
// numbers whose h are rounded up can become infinite.  A workgroup that has results that are not finite computes its tile again on the fp32 units, and takes these
// results from there (and no other, so that none depends on another row's numbers).  Numbers below 2^-100 lose bits of m and l below the smallest bf16 number, 2^-133.
#pragma once
#include "linear_tile.h"

namespace gcn {


// One operand of a stage: 32 values of k of R rows (of A) or columns (of B), as three planes of bf16.
//   BY_K   64 bytes per row; its four pieces of 8 k are moved about by bits of the row
//   BY_MN  one row per k of R elements, whose blocks of 16 are moved about as in Operand
template <int R, int LIES, int THREADS>
struct Thirds {
    using Plain = Operand<float, R, LIES, THREADS>;
    static constexpr int PLANE = R * 64, PER = Plain::PER;
    static constexpr int BLOCKS = R / 16 < 8 ? R / 16 : 8;
    __device__ static int twist(int k) { return ((k & 3) | ((k >> 3 & 1) << 2)) & (BLOCKS - 1); }
    __device__ static void put(const Vec<float> (&v)[PER], char* lds, int tid) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            int row, piece;
            Plain::at(i * THREADS + tid, row, piece);
            const int at = LIES == BY_K ? row * 64 + (((piece >> 1) ^ ((row >> 2) & 3)) << 4) + (piece & 1) * 8
                                        : row * (R * 2) + (((piece >> 2) ^ twist(row)) << 5) + (piece & 3) * 8;
            float x[4] = {v[i][0], v[i][1], v[i][2], v[i][3]};
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                uint2 words;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    typedef float f2 __attribute__((ext_vector_type(2)));
                    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
                    const uint32_t w = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{x[2 * h], x[2 * h + 1]}), b2));
                    (h ? words.y : words.x) = w;
                    x[2 * h] -= __builtin_bit_cast(float, w << 16);
                    x[2 * h + 1] -= __builtin_bit_cast(float, w & 0xffff0000u);
                }
                *reinterpret_cast<uint2*>(lds + p * PLANE + at) = words;
            }
        }
    }
    __device__ static Vec<__bf16> fragment(const char* lds, int plane, int r, int lane) {
        const char* const p = lds + plane * PLANE;
        if (LIES == BY_K) {
            const int row = r + (lane & 15);
            return *reinterpret_cast<const Vec<__bf16>*>(p + row * 64 + (((lane >> 4) ^ ((row >> 2) & 3)) << 4));
        }
#if defined(__HIP_DEVICE_COMPILE__)
        typedef short s4 __attribute__((ext_vector_type(4)));
        const int k = (lane >> 4) * 8 + ((lane & 15) >> 2);
        const char* const q = p + k * (R * 2) + ((((r >> 4) ^ twist(k)) << 5) + (lane & 3) * 8);      // (k + 4: the same block)
        const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(GCN_LDS(s4, q));
        const s4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(GCN_LDS(s4, q + 4 * R * 2));
        return __builtin_bit_cast(Vec<__bf16>, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
#else
        return Vec<__bf16>{};
#endif
    }
};

// As k_linear_tile through registers, for any alignment; one stage in LDS (three planes of 32 k: 48 KB of a 128 x 128 tile), the next one in registers, and another
// workgroup on the compute unit meanwhile.  Of the compute units' cycles the matrix units are busy in 40 % at 232965 x 602 x 128 (96 products of 16 cycles a stage and wavefront), and
// vector instructions are issued in 40 %: 22 split four numbers.  (A look at every number for infinities made them as many as the products take: 180 TFLOP/s.)  The second set of
// results for those that are not finite costs 16 and 18 spilled registers of the 128 x 128 forms whose B lies along n.
template <int BM, int BN, int WM, int WN, int LA, int LB>
__global__ __launch_bounds__(WM* WN * 64, 2) void k_linear_thirds(TileArgs a) {
    constexpr int THREADS = WM * WN * 64, BK = 32, E = 4;
    constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
    using OpA = Thirds<BM, LA, THREADS>;
    using OpB = Thirds<BN, LB, THREADS>;
    using PlainA = typename OpA::Plain;
    using PlainB = typename OpB::Plain;
    constexpr int STAGE = 3 * (OpA::PLANE + OpB::PLANE);
    __shared__ __attribute__((aligned(16))) char stage[STAGE];
    char* const stage_b = stage + 3 * OpA::PLANE;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int tm, tn;
    tile_place(a, tm, tn);
    const int64_t m0 = (int64_t)tm * BM;
    const int n0 = tn * BN;
    const int64_t kb = (int64_t)blockIdx.y * a.k_share, ke = kb + a.k_share < a.K ? kb + a.k_share : a.K;
    const float* const A = (const float*)a.A;
    const float* const B = (const float*)a.B;
    const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
    v4f acc[FM][FN] = {};
    // put(va, vb) and products() for all stages
    auto run = [&](auto put, auto products) {
        Vec<float> va[OpA::PER], vb[OpB::PER];
        int64_t k = kb;
        const int64_t end = (LA == BY_MN && a.M < E) || (LB == BY_MN && a.N < E) ? k : k + (ke - k) / BK * BK;
        typename PlainA::Source sa;
        typename PlainB::Source sb;
        if (k < end) {
            sa = PlainA::source(A, a.lda, m0, a.M, k, tid);
            sb = PlainB::source(B, a.ldb, n0, a.N, k, tid);
        }
        auto next = [&]() {
            if (k < end) {
                PlainA::fetch(sa, a.lda, va);
                PlainB::fetch(sb, a.ldb, vb);
            } else {
                PlainA::fetch_end(A, a.lda, m0, a.M, k, ke, va, tid);
                PlainB::fetch_end(B, a.ldb, n0, a.N, k, ke, vb, tid);
            }
        };
        next();
        while (true) {
            put(va, vb);
            __syncthreads();
            k += BK;
            if (k < ke) next();
            products();
            __syncthreads();
            if (k >= ke) break;
        }
    };
    run([&](const Vec<float>(&va)[OpA::PER], const Vec<float>(&vb)[OpB::PER]) {
            OpA::put(va, stage, tid);
            OpB::put(vb, stage_b, tid);
        },
        [&]() {
            Vec<__bf16> q[3][FM];
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
                for (int i = 0; i < FM; ++i) q[p][i] = OpA::fragment(stage, p, wm + i * 16, lane);
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                Vec<__bf16> b[3];
#pragma unroll
                for (int p = 0; p < 3; ++p) b[p] = OpB::fragment(stage_b, p, wn + j * 16, lane);
                // the small products first; the same accumulator is due again after FM products
#pragma unroll
                for (int t = 0; t < 6; ++t) {
                    constexpr int PB[6] = {2, 0, 1, 1, 0, 0}, PA[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
                    for (int i = 0; i < FM; ++i) acc[i][j] = mma(b[PB[t]], q[PA[t]][i], acc[i][j]);
                }
            }
        });
    bool lost = false;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) lost |= !(fabsf(acc[i][j][e]) < INFINITY);
    if (__syncthreads_or(lost)) {
        v4f plain[FM][FN] = {};
        run([&](const Vec<float>(&va)[OpA::PER], const Vec<float>(&vb)[OpB::PER]) {
                PlainA::put(va, stage, tid);
                PlainB::put(vb, stage + BM * 128, tid);
            },
            [&]() {
#pragma unroll
                for (int step = 0; step < 2; ++step) {
                    Vec<float> p[FN], q[FM];
#pragma unroll
                    for (int j = 0; j < FN; ++j) p[j] = PlainB::fragment(stage + BM * 128, wn + j * 16, step, lane);
#pragma unroll
                    for (int i = 0; i < FM; ++i) q[i] = PlainA::fragment(stage, wm + i * 16, step, lane);
#pragma unroll
                    for (int i = 0; i < FM; ++i)
#pragma unroll
                        for (int j = 0; j < FN; ++j) plain[i][j] = mma(p[j], q[i], plain[i][j]);
                }
            });
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!(fabsf(acc[i][j][e]) < INFINITY)) acc[i][j][e] = plain[i][j][e];
    }
    constexpr int PHASES = (BM * BN * 4 + STAGE - 1) / STAGE, PART = BM / WM / PHASES * (BN / WN) * 4;
    static_assert(WM * WN * PART <= STAGE && (BM + BN) * 128 <= STAGE, "results and plain stages have room");
    leave_tile<float, FM, FN, PHASES, LA == BY_MN, LB == BY_MN>(a, acc, stage + wave * PART, m0 + wm, n0 + wn, lane);
}

}  // namespace gcn
