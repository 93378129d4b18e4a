// A linear layer over few rows: one pass over the weights, whose reading is most of the time it takes.
#pragma once
#include "linear_tile.h"

namespace gcn {

constexpr int FEW_WAVES = 16;
// From so many strips on a workgroup takes all of k: one launch.  Below, the sum over k is split, and the partial results joined by a second one.  Microseconds with the split and
// without, of bf16 (and fp32), 16 rows: 512 columns, 32 strips, k of 16384 15.5 and 38.6 (19.3, 53.3), of 4096 7.1 and 7.9 (7.6, 11.8), of 1024, too short for a split in bf16, 4.0 (6.4,
// 5.0: the second launch costs more than it saves); 752 columns, 47 strips, k of 4096 9.5 and 10.0 (11.6, 13.7).  With 64 strips the other way round from k of about 8192 on:
// 1024 columns, k of 16384 23.8 with a split, 37.4 without (30.4, 49.9), of 4096 8.3 and 8.0 (12.1, 14.8), of 1024 4.1 and 4.1 (6.5, 5.0).
constexpr int FEW_STRIPS = 48;
template <typename T, int C, int RT>
constexpr size_t few_lds() { return (size_t)FEW_WAVES * RT * 16 * (16 * C + 4) * 4; }

// Y's rows are few, so the product is bound by reading W (and by about 4 us of start and end): 4096 x 4096 in bf16 for 16 rows 13.5 us, in fp32 for one row 14.5 us (4.6
// TB/s), 4096 x 16384 in bf16 26 to 28 us (4.8 to 5 TB/s).  What is left where strips are narrow: a wavefront waits for its two steps before it multiplies them and sends for the next two
// after, so at 4096 x 4096 in bf16, two bytes to a load, the weights come at 2.5 TB/s.
// A workgroup has a strip of 16 C columns; its wavefronts take the 4 E values of k of a step in turn, straight from memory into the operands of the matrix unit: a
// lane loads C neighbouring columns of E rows of W and has with them C fragments of E values of k.  Up to 16 RT rows of X, whose fragments are 16
// bytes of a row.  The wavefronts' results are added in order in LDS, and what the layer does with them follows.  Neighbouring strips run on the same XCD, since
// a strip can be half of a cache line wide.
// C is the widest that still leaves a strip for every compute unit: 4096 x 4096 in fp32 with 256 strips of 16 columns 14.5 us, with 128 of 32 18.8.
// Few strips: the steps are also shared by gridDim.y workgroups, whose partial results k_linear_join adds.
template <typename T, int C, int RT>
__global__ __launch_bounds__(FEW_WAVES * 64) void k_linear_few(TileArgs a, int strips) {
    constexpr int E = Elem<T>::E, STEP = 4 * E, AHEAD = 2, ROW = 16 * C + 4;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, quarter = lane >> 4;
    const int per = (strips + 7) / 8, strip = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
    if (strip >= strips || (int)(blockIdx.x >> 3) >= per) return;
    const int n0 = strip * 16 * C, n = n0 + r * C;
    const int there = a.N - n < 0 ? 0 : (a.N - n > C ? C : a.N - n);
    const T* const W = (const T*)a.B + n;
    const T* const X = (const T*)a.A;
    const int64_t kb = (int64_t)blockIdx.y * a.k_share, ke = kb + a.k_share < a.K ? kb + a.k_share : a.K;
    v4f acc[RT][C] = {};
    struct Step {
        Elems<T, C> w[E];
        Vec<T> x[RT];
    };
    // `whole`: all of the step's k and all of the wavefront's columns are there
    auto load = [&](int64_t k0, auto whole) {
        Step s = {};
        const int64_t k = k0 + quarter * E;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (decltype(whole)::value || (k + e < ke && there > 0)) s.w[e] = load_elems<C>(W + (k + e) * a.ldb, decltype(whole)::value ? C : there);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int64_t left = ke - k;
            if (t * 16 + r < a.M && left > 0) s.x[t] = load_vec_part(X + (t * 16 + r) * a.lda + k, decltype(whole)::value || left > E ? E : (int)left);
        }
        return s;
    };
    auto products = [&](const Step& s) {
#pragma unroll
        for (int q = 0; q < C; ++q) {
            Vec<T> f;
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] = s.w[e][q];
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[t][q] = mma(f, s.x[t], acc[t][q]);
        }
    };
    constexpr int ALL = FEW_WAVES * STEP;
    int64_t k = kb + wave * STEP;
    if (n0 + 16 * C <= a.N)
        for (; k + (AHEAD - 1) * ALL + STEP <= ke; k += AHEAD * ALL) {
            Step s[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) s[u] = load(k + u * ALL, std::true_type());
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) products(s[u]);
        }
    for (; k < ke; k += ALL) products(load(k, std::false_type()));
    float* const mine = (float*)lds + wave * (RT * 16 * ROW);
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int q = 0; q < C; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) mine[(t * 16 + r) * ROW + (quarter * 4 + e) * C + q] = acc[t][q][e];
    __syncthreads();
    // a thread for each result; the sum takes the place of the first wavefront's, which no other thread reads
    for (int i = threadIdx.x; i < RT * 16 * 16 * C; i += FEW_WAVES * 64) {
        float* const at = (float*)lds + i / (16 * C) * ROW + i % (16 * C);
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < FEW_WAVES; ++w) sum += at[w * RT * 16 * ROW];
        *at = sum;
    }
    __syncthreads();
    constexpr int PIECES = 16 * C / E;
    if constexpr (16 * C % E == 0) {
        for (int i = threadIdx.x; i < RT * 16 * PIECES; i += FEW_WAVES * 64) {
            const int row = i / PIECES, c = i % PIECES * E, count = a.N - n0 - c;
            if (row >= a.M || count <= 0) continue;
            float d[E];
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] = ((const float*)lds)[row * ROW + c + e];
            if (a.part) {
                float* const p = a.part + ((int64_t)blockIdx.y * a.M + row) * a.N + n0 + c;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e < count) p[e] = d[e];
            } else {
                float r_[E];
                finish<T>(a, row, n0 + c, count, d, false, r_);
            }
        }
    }
}

}  // namespace gcn
