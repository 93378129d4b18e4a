// Products with weights held in 4 bits, for one element type: Y = rho R + act(X W + 1 bias^T), and the gated block.  The matrix units take the places as bf16 (fp16 for fp16 elements) numbers, exactly,
// eight of a column from a word by four instructions; the sum over a group, in fp32, is multiplied by its scale where it leaves the unit.  So the weights are never rounded.  fp32 elements enter as the
// sum of three bf16 numbers, which is all of them: three products each.
#pragma once
#include "held.h"
#include "launch_rules.h"
#include "linear_few.h"

namespace gcn {

template <typename T> int linear4_of(const TileArgs& a, const Weights4& w, hipStream_t s);

template <typename T> using Unit4 = std::conditional_t<std::is_same<T, _Float16>::value, _Float16, __bf16>;      // what the matrix unit takes
// The places enter 2^-10 times as large: the sum over a group, of up to 128 places of up to 6, is then no larger than the largest x, which may be the largest number there is.  (fp16 elements are far
// from fp32's largest.)
template <typename T> constexpr float PLACE4 = std::is_same<T, _Float16>::value ? 1.f : 1.f / 1024;

template <typename U>
__device__ __forceinline__ Vec<U> places_of(uint32_t word, float times) {
    uint4 v = {};
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (std::is_same<U, _Float16>::value) {
        v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, times, 0));
        v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, times, 1));
        v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, times, 2));
        v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, times, 3));
    } else {
        v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, times, 0));
        v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, times, 1));
        v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, times, 2));
        v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, times, 3));
    }
#endif
    return __builtin_bit_cast(Vec<U>, v);
}

// Two fp32 numbers as three words of two bf16 numbers each.  Each number is what is left cut off behind eight bits, so that the three are all of it; an infinity or NaN is the first alone.
__device__ __forceinline__ void cut_in_three(float x, float y, uint32_t (&w)[3]) {
    auto first = [](float v) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        return v != v ? 0x7fc00000u : b & 0xffff0000u;
    };
    auto two = [](uint32_t lo, uint32_t hi) { return lo >> 16 | hi; };
    const uint32_t hx = first(x), hy = first(y);
    w[0] = two(hx, hy);
    x = fabsf(x) < INFINITY ? x - __builtin_bit_cast(float, hx) : 0.f;
    y = fabsf(y) < INFINITY ? y - __builtin_bit_cast(float, hy) : 0.f;
    const uint32_t mx = __builtin_bit_cast(uint32_t, x) & 0xffff0000u, my = __builtin_bit_cast(uint32_t, y) & 0xffff0000u;
    w[1] = two(mx, my);
    x -= __builtin_bit_cast(float, mx);
    y -= __builtin_bit_cast(float, my);
    w[2] = two(__builtin_bit_cast(uint32_t, x) & 0xffff0000u, __builtin_bit_cast(uint32_t, y) & 0xffff0000u);
}

// Eight elements of a row of X as the matrix unit takes them.
template <typename T> constexpr int PARTS4 = sizeof(T) == 4 ? 3 : 1;
template <typename T> struct Eight { Vec<T> v[8 / Elem<T>::E]; };
template <typename T>
__device__ __forceinline__ Eight<T> load_eight(const T* p, int64_t there) {
    Eight<T> x = {};
#pragma unroll
    for (int i = 0; i < 8 / Elem<T>::E; ++i) {
        const int64_t left = there - i * Elem<T>::E;
        if (left > 0) x.v[i] = load_vec_part(p + i * Elem<T>::E, left < Elem<T>::E ? (int)left : Elem<T>::E);
    }
    return x;
}
template <typename T>
__device__ __forceinline__ void parts_of(const Eight<T>& x, Vec<Unit4<T>> (&p)[PARTS4<T>]) {
    if constexpr (sizeof(T) == 2) {
        p[0] = x.v[0];
    } else {
        uint32_t w[4][3];
#pragma unroll
        for (int i = 0; i < 4; ++i) cut_in_three(x.v[i / 2][i % 2 * 2], x.v[i / 2][i % 2 * 2 + 1], w[i]);
#pragma unroll
        for (int k = 0; k < 3; ++k) p[k] = __builtin_bit_cast(Vec<__bf16>, (uint4{w[0][k], w[1][k], w[2][k], w[3][k]}));
    }
}

#if defined(__HIP_DEVICE_COMPILE__)
#define KEEP_ORDER() __builtin_amdgcn_sched_barrier(0)
#else
#define KEEP_ORDER() (void)0
#endif

// The number of the wavefront in its workgroup, as the scalar that it is.
__device__ __forceinline__ int wave_number() {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
#else
    return 0;
#endif
}

constexpr int BLOCK4 = 128;           // values of k that a wavefront takes at a time: a whole number of groups

// Few rows: the strips and their end are those of k_linear_few.  A lane loads C neighbouring words of four rows of words, which are C fragments of four steps of 32 values of k, and has the results of
// the same columns, so that it needs their scales and no others.  blockIdx.z: which 16 RT rows.
// Bound by memory where there are codes enough: 16 rows of a gated block, 8192 x 2*14336 in fp16, 29 us, 4.3 TB/s of codes and scales.  One row, 4096 x 4096 in bf16, 6 us, most of them the start and the
// joining of 16 wavefronts.
template <typename T, int C, int RT, int WAVES, bool GATED>
__global__ __launch_bounds__(WAVES * 64, WAVES == 16 || (sizeof(T) == 2 && RT == 1 && C <= 4) ? 4 : 2) void k_linear4_few(TileArgs a, Weights4 w, int strips) {
    using U = Unit4<T>;
    constexpr int PARTS = PARTS4<T>, WIDE = GATED ? 8 * C : 16 * C;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = wave_number(), r = lane & 15, quarter = lane >> 4;
    const int per = (strips + 7) / 8, strip = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
    if (strip >= strips || (int)(blockIdx.x >> 3) >= per) return;
    const int n0 = strip * WIDE, n = n0 + (GATED ? (r & 7) * C : r * C);
    const int there = a.N - n;                                    // of the lane's C columns
    const int64_t c = n + (GATED && r >= 8 ? (int64_t)a.N : 0);
    const uint32_t* const Q = w.Q + quarter * w.ldq + c;          // of the first step's word
    const uint16_t* const S = w.S + c;
    const int64_t m0 = (int64_t)blockIdx.z * (16 * RT);
    const T* const X = (const T*)a.A + m0 * a.lda;
    const int64_t rows = a.M;
    a.M -= m0;
    if (a.part) a.part += m0 * a.N * (GATED ? 2 : 1);
    a.Y = (T*)a.Y + m0 * a.ldy;
    if (a.R) a.R = (const T*)a.R + m0 * a.ldr;
    const int64_t kb = (int64_t)blockIdx.y * a.k_share, ke = kb + a.k_share < a.K ? kb + a.k_share : a.K;
    const int shift = w.group == 32 ? 5 : w.group == 64 ? 6 : 7, steps = 1 << (shift - 5);
    v4f acc[RT][C] = {};
    // `whole`: all of the block's k and all of the strip's columns are there
    auto block = [&](int64_t k0, auto whole) {
        constexpr bool ALL = decltype(whole)::value;
        Elems<uint32_t, C> word[4];
        Elems<uint16_t, C> scale[4];
        Eight<T> x[4][RT];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t k = k0 + i * 32 + quarter * 8;
            word[i] = load_elems<C>(Q + (k0 / 8 + i * 4) * w.ldq, ALL ? C : k < ke ? there : 0);
            scale[i] = {};
            if ((i & (steps - 1)) == 0) scale[i] = load_elems<C>(S + ((k0 + i * 32) >> shift) * w.lds, ALL ? C : k0 + i * 32 < ke ? there : 0);
#pragma unroll
            for (int t = 0; t < RT; ++t) x[i][t] = t * 16 + r < a.M ? load_eight(X + (t * 16 + r) * a.lda + k, ALL ? 8 : ke - k) : Eight<T>{};
        }
        v4f sum[RT][C] = {};
        Elems<uint16_t, C> of = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if ((i & (steps - 1)) == 0) of = scale[i];
            Vec<U> part[RT][PARTS];
#pragma unroll
            for (int t = 0; t < RT; ++t) parts_of<T>(x[i][t], part[t]);
#pragma unroll
            for (int q = 0; q < C; ++q) {
                const Vec<U> f = places_of<U>(word[i][q], PLACE4<T>);
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int p = PARTS - 1; p >= 0; --p) sum[t][q] = mma(part[t][p], f, sum[t][q]);
            }
            if (((i + 1) & (steps - 1)) == 0)
#pragma unroll
                for (int q = 0; q < C; ++q)
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[t][q][e] = fmaf(scale_value(of[q]), sum[t][q][e], acc[t][q][e]);
                        sum[t][q] = v4f{};
                    }
        }
    };
    int64_t k = kb + wave * BLOCK4;
    if (n0 + WIDE <= a.N)
        for (; k + BLOCK4 <= ke; k += WAVES * BLOCK4) block(k, std::true_type());
    for (; k < ke; k += WAVES * BLOCK4) block(k, std::false_type());
    leave_few<T, C, RT, GATED, WAVES, true>(a, acc, lds, n0, rows, 1.f / PLACE4<T>);
}

// Many rows: 128 x 128 results of four wavefronts, 64 values of k at a time, through registers: words become 16-byte pieces of places on their way to LDS, where X and W lie by k alike (see Operand).
// Two stages, of which one is fetched while the other is multiplied; fp32 elements are three planes of X, and one stage.  A lane has four rows of a column, so that a scale goes with all that it
// has of a fragment.  STEPS: of 32 values of k in a group.
// Bound by the vector instructions beside the matrix units': making places of words, and a multiplication of every sum for each group.  2048 x 4096 x 4096 in bf16 with groups of 64 and 128 85 us (0.81
// PFLOP/s), of 32 101 us (matrix units busy in 28 % of the cycles, vector instructions issued in 48 %); with weights of 16 bits k_linear_tile takes 68 us.
template <typename T, bool GATED, int STEPS>
__global__ __launch_bounds__(256, 2) void k_linear4_tile(TileArgs a, Weights4 w) {
    using U = Unit4<T>;
    constexpr int E = Elem<T>::E, BM = 128, BN = 128, THREADS = 256, PARTS = PARTS4<T>, BK = 64, PLANE = BM * 128, WORDS = BN * 8 / THREADS;
    constexpr int STAGE = PARTS * PLANE + BN * 128, STAGES = PARTS == 1 ? 2 : 1, WIDE = GATED ? BN / 2 : BN;
    using OpX = Operand<U, BM, BY_K, THREADS>;
    using OpW = Operand<U, BN, BY_K, THREADS>;
    __shared__ __attribute__((aligned(16))) char lds[STAGES * STAGE];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int tm, tn;
    tile_place(a, tm, tn);
    const int64_t m0 = (int64_t)tm * BM;
    const int n0 = tn * WIDE;
    // (k is 2^27 at most)
    const int K = (int)a.K, kb = (int)(blockIdx.y * a.k_share), ke = kb + a.k_share < a.K ? (int)(kb + a.k_share) : K;
    const int wm = (wave / 2) * 64, wn = (wave % 2) * 64;
    // a column of the tile: of each 64 of a gated block's the first 32 are the gate's; the last one's where there is none
    auto column = [&](int c) -> uint32_t {
        const int h = GATED ? n0 + c / 64 * 32 + c % 32 : n0 + c;
        return (uint32_t)(h < a.N ? h : a.N - 1) + (GATED && c % 64 >= 32 ? (uint32_t)a.N : 0u);
    };
    // what a thread takes of a stage: words of one column, and eight elements at one place of XS rows
    const uint32_t my_column = column(tid & (BN - 1)) * 4;        // bytes, as a scale's place below: 32 bits are enough for rows of up to 2^27
    const int my_word = wave_number() / (BN / 64);
    const int last_word = (ke - 1) >> 3, last_group = (ke - 1) / (32 * STEPS);
    constexpr int XS = BM * 8 / THREADS, VECS = 8 / E;
    int my_row, my_piece;
    OpX::at(tid, my_row, my_piece);                               // (32 rows on: the same piece)
    const T* rows[XS];
#pragma unroll
    for (int i = 0; i < XS; ++i) {
        const int64_t m = m0 + my_row + i * (THREADS / 8);
        rows[i] = (const T*)a.A + (m < a.M ? m : a.M - 1) * a.lda;
    }
    // the scales of a lane's column of each fragment
    uint32_t scale_at[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) scale_at[j] = column(wn + j * 16 + (lane & 15)) * 2;
    constexpr int GROUPS = STEPS == 1 ? 2 : 1;                    // that a stage has scales of
    // What is on its way: of two stages, with fp32 elements, which have the registers of one only, of one
    constexpr int SETS = PARTS == 1 ? 2 : 1;
    uint32_t word[SETS][WORDS];
    Words<T, E> x[SETS][XS][VECS];
    uint16_t scale[SETS][GROUPS][4];
    auto fetch = [&](auto of_set, int k) {
        constexpr int s = decltype(of_set)::value;
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            int j = (k >> 3) + i * (THREADS / BN) + my_word;
            j = j < last_word ? j : last_word;                    // (X is 0 behind it)
            word[s][i] = *reinterpret_cast<const uint32_t*>((const char*)(w.Q + j * w.ldq) + my_column);
        }
#pragma unroll
        for (int v = 0; v < VECS; ++v) {
            int at = k + my_piece * 8 + v * E;
            at = at < K - E ? at : K - E;                         // as load_near
#pragma unroll
            for (int i = 0; i < XS; ++i) x[s][i][v] = load_near<E>(rows[i] + at, 0, E);
        }
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            int at = k / (32 * STEPS) + g;
            at = at < last_group ? at : last_group;
#pragma unroll
            for (int j = 0; j < 4; ++j) scale[s][g][j] = *reinterpret_cast<const uint16_t*>((const char*)(w.S + at * w.lds) + scale_at[j]);
        }
    };
    float of[GROUPS][4];                                          // the scales of the stage in LDS
    auto put = [&](auto of_set, char* to, int k) {
        constexpr int s = decltype(of_set)::value;
        if (k + BK > K)                                           // the end of the rows: zeros behind it
#pragma unroll
            for (int v = 0; v < VECS; ++v) {
                const int by = settle_by<E>(k + my_piece * 8 + v * E, K);
#pragma unroll
                for (int i = 0; i < XS; ++i) x[s][i][v] = __builtin_bit_cast(Words<T, E>, settle<E, T>(x[s][i][v], by));
            }
#pragma unroll
        for (int i = 0; i < XS; ++i) {
            Eight<T> e;
#pragma unroll
            for (int v = 0; v < VECS; ++v) e.v[v] = __builtin_bit_cast(Vec<T>, x[s][i][v]);
            Vec<U> p[PARTS];
            parts_of<T>(e, p);
#pragma unroll
            for (int part = 0; part < PARTS; ++part) *reinterpret_cast<Vec<U>*>(to + part * PLANE + (i * THREADS + tid) * 16) = p[part];
        }
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            const int c = tid & (BN - 1), piece = i * (THREADS / BN) + my_word;
            *reinterpret_cast<Vec<U>*>(to + PARTS * PLANE + c * 128 + ((piece ^ (c & 7)) << 4)) = places_of<U>(word[s][i], PLACE4<T>);
        }
#pragma unroll
        for (int g = 0; g < GROUPS; ++g)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                of[g][j] = scale_value(scale[s][g][j]);
#if defined(__HIP_DEVICE_COMPILE__)
                asm volatile("" : "+v"(of[g][j]));                // now, or the next ones would have to be copied before they arrive
#endif
            }
    };
    // The sums of a group leave with its stage, or with its 32 values of k: longer groups would need a second set of all sums (128 values of k at a time: 93 us at 2048 x 4096 x 4096, 64 at a
    // time 86).  Those of fp32 elements, three products each, every 32.
    constexpr int AT_ONCE = PARTS == 3 || STEPS == 1 ? 1 : 2;     // steps
    v4f acc[4][4] = {};
    auto add = [&](int j, const v4f (&of)[4], float s) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(s, of[i][e], acc[i][j][e]);
#if defined(__HIP_DEVICE_COMPILE__)
        // here and not behind the branch that follows the stage, where the compiler would put all of it at once, and the matrix units wait
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(acc[i][j]));
#endif
    };
    auto multiply = [&](const char* stage, int k0) {
        auto row_fragments = [&](int part, int step, Vec<U> (&q)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = OpX::fragment(stage + part * PLANE, wm + i * 16, step, lane);
        };
        auto columns = [&](int j, int step) { return OpW::fragment(stage + PARTS * PLANE, wn + j * 16, step, lane); };
#pragma unroll
        for (int step = 0; step < 2; step += AT_ONCE) {
            Vec<U> q[AT_ONCE][PARTS][4], p[AT_ONCE][4];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
#pragma unroll
                for (int j = 0; j < 4; ++j) p[u][j] = columns(j, step + u);
#pragma unroll
                for (int part = 0; part < PARTS; ++part) row_fragments(part, step + u, q[u][part]);
            }
            v4f one[2][4];
#pragma unroll
            for (int j = 0; j < 5; ++j) {                     // a column's sums leave while the next one's products are made
                if (j < 4) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) one[j & 1][i] = v4f{};
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
                        for (int part = PARTS - 1; part >= 0; --part)
#pragma unroll
                            for (int i = 0; i < 4; ++i) one[j & 1][i] = mma(q[u][part][i], p[u][j], one[j & 1][i]);
                }
                if (j > 0) add(j - 1, one[(j - 1) & 1], of[STEPS == 1 ? step : 0][j - 1]);
                KEEP_ORDER();
            }
        }
    };
    // The stage at k is in LDS, the next one in the other set or, with one set, not on its way yet.
    int k = kb;
    auto turn = [&](auto mine, auto next, char* stage, char* other) {
        if (k + SETS * BK < ke) fetch(mine, k + SETS * BK);
        multiply(stage, k);
        k += BK;
        if (k >= ke) return false;
        if (STAGES == 1) __syncthreads();
        put(next, other, k);
        __syncthreads();
        return true;
    };
    constexpr std::integral_constant<int, 0> zero{};
    constexpr std::integral_constant<int, SETS - 1> last{};
    fetch(zero, k);
    if (SETS == 2 && k + BK < ke) fetch(last, k + BK);
    put(zero, lds, k);
    __syncthreads();
    char* const other = lds + (STAGES - 1) * STAGE;
    while (turn(zero, last, lds, other) && turn(last, zero, other, lds)) {}
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] *= 1.f / PLACE4<T>;
    constexpr int PART = 64 * 64 * 4;
    static_assert(4 * PART <= STAGES * STAGE, "results have room");
    __syncthreads();
    char* const mine = lds + wave * PART;
    if constexpr (GATED) leave_gated<T, 4, 4, 1, false, true>(a, acc, mine, m0 + wm, n0 + wn / 2, lane);
    else leave_tile<T, 4, 4, 1, false, false, true>(a, acc, mine, m0 + wm, n0 + wn, lane);
}

template <typename T, int C, int RT, bool GATED>
static int launch_few4(TileArgs a, const Weights4& w, int64_t splits, hipStream_t s) {
    constexpr int WAVES = few4_waves(C, RT), WIDE = GATED ? 8 * C : 16 * C, ALL = BLOCK4 * WAVES, ROWS = 16 * RT;
    const int strips = (a.N + WIDE - 1) / WIDE;
    if (a.M > 65535 * ROWS) splits = 1;                           // (more than one launch)
    const int64_t blocks = (a.K + ALL - 1) / ALL;
    a.k_share = (blocks + splits - 1) / splits * ALL;
    splits = (a.K + a.k_share - 1) / a.k_share;
    ScratchLease lease;
    if (splits > 1) {
        void* p = nullptr;
        GCN_TRY(lease.get(&p, (size_t)splits * a.M * a.N * (GATED ? 8 : 4), s));
        a.part = (float*)p;
    }
    for (int64_t m = 0; m < a.M; m += 65535 * ROWS) {             // (a launch has so many workgroups along a dimension)
        TileArgs b = a;
        b.A = (const T*)a.A + m * a.lda;
        b.Y = (T*)a.Y + m * a.ldy;
        if (a.R) b.R = (const T*)a.R + m * a.ldr;
        b.M = a.M - m;
        const int64_t blocks_m = (b.M + ROWS - 1) / ROWS;
        launch_lds<k_linear4_few<T, C, RT, WAVES, GATED>>(dim3((unsigned)((strips + 7) / 8 * 8), (unsigned)splits, (unsigned)(blocks_m < 65535 ? blocks_m : 65535)), WAVES * 64,
                                                          few_lds<C, RT, WAVES>(), s, b, w, strips);
        GCN_LAUNCH_CHECK();
    }
    return splits > 1 ? launch_join<T, GATED>(a, (int)splits, s) : GCN_OK;
}

template <typename T, bool GATED>
static int launch_tile4(TileArgs a, const Weights4& w, hipStream_t s) {
    constexpr int BM = 128, WIDE = GATED ? 64 : 128;
    const int64_t tm = (a.M + BM - 1) / BM, tn = (a.N + WIDE - 1) / WIDE;
    if (tm * tn * 256 > UINT32_MAX) return fail(GCN_ERR_RANGE, "linear: more results than one launch has threads for");
    a.tiles_m = (int32_t)tm;
    a.tiles_n = (int32_t)tn;
    int splits = splits_of_4(tm * tn, a.M * (GATED ? 2 * (int64_t)a.N : a.N), a.K, sizeof(T) == 4, device_info().cus);
    const int64_t blocks = (a.K + BLOCK4 - 1) / BLOCK4;
    a.k_share = (blocks + splits - 1) / splits * BLOCK4;
    splits = (int)((a.K + a.k_share - 1) / a.k_share);
    ScratchLease lease;
    if (splits > 1) {
        void* p = nullptr;
        GCN_TRY(lease.get(&p, (size_t)splits * a.M * a.N * (GATED ? 8 : 4), s));
        a.part = (float*)p;
    }
    const dim3 grid((unsigned)(tm * tn), (unsigned)splits);
    auto launch = [&](auto steps) { hipLaunchKernelGGL((k_linear4_tile<T, GATED, decltype(steps)::value>), grid, dim3(256), 0, s, a, w); };
    if (w.group == 32) launch(std::integral_constant<int, 1>());
    else if (w.group == 64) launch(std::integral_constant<int, 2>());
    else launch(std::integral_constant<int, 4>());
    GCN_LAUNCH_CHECK();
    return splits > 1 ? launch_join<T, GATED>(a, splits, s) : GCN_OK;
}

template <typename T, bool GATED>
static int linear4_impl(const TileArgs& a, const Weights4& w, hipStream_t s) {
    constexpr bool FP32 = sizeof(T) == 4;
    const Few4 f = few4_choice(a.M, GATED ? 2 * (int64_t)a.N : a.N, a.K, FP32, device_info().cus);
    if (f.rows == 0) return launch_tile4<T, GATED>(a, w, s);
    auto by_columns = [&](auto rt) {
        constexpr int RT = decltype(rt)::value;
        if constexpr (RT == 1 || (RT == 2 && !FP32))
            if (f.columns == 8) return launch_few4<T, 8, RT, GATED>(a, w, f.splits, s);
        if (f.columns >= 4) return launch_few4<T, 4, RT, GATED>(a, w, f.splits, s);
        if (f.columns == 2) return launch_few4<T, 2, RT, GATED>(a, w, f.splits, s);
        return launch_few4<T, 1, RT, GATED>(a, w, f.splits, s);
    };
    if (f.rows == 1) return by_columns(std::integral_constant<int, 1>());
    if constexpr (!FP32)
        if (f.rows == 4) return by_columns(std::integral_constant<int, 4>());
    return by_columns(std::integral_constant<int, 2>());
}

}  // namespace gcn
