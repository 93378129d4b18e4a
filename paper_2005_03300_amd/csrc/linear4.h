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

constexpr int BLOCK4 = 128;           // values of k that a wavefront takes at a time: a whole number of groups

// Few rows: the strips, wavefronts and their end are those of k_linear_few.  A lane loads C neighbouring words of four rows of words, which are C fragments of four steps of 32 values of k.
template <typename T, int C, int RT, bool GATED>
__global__ __launch_bounds__(FEW_WAVES * 64) void k_linear4_few(TileArgs a, Weights4 w, int strips) {
    using U = Unit4<T>;
    constexpr int PARTS = PARTS4<T>, WIDE = GATED ? 8 * C : 16 * C;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, quarter = lane >> 4;
    const int per = (strips + 7) / 8, strip = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
    if (strip >= strips || (int)(blockIdx.x >> 3) >= per) return;
    const int n0 = strip * WIDE;
    // where columns `c` on of the strip's 16 C are, and how many of C or 4 C of them are there
    auto column = [&](int c) { return GATED ? n0 + (c < 8 * C ? c : c - 8 * C) : n0 + c; };
    auto behind = [&](int c) { return GATED && c >= 8 * C ? (int64_t)a.N : (int64_t)0; };
    const int cq = r * C, cs = quarter * 4 * C;
    const int there_q = a.N - column(cq), there_s = a.N - column(cs);
    const uint32_t* const Q = w.Q + column(cq) + behind(cq);
    const uint16_t* const S = w.S + column(cs) + behind(cs);
    const T* const X = (const T*)a.A;
    const int64_t kb = (int64_t)blockIdx.y * a.k_share, ke = kb + a.k_share < a.K ? kb + a.k_share : a.K;
    const int steps = w.group / 32;
    v4f acc[RT][C] = {};
    // `whole`: all of the block's k and all of the strip's columns are there
    auto block = [&](int64_t k0, auto whole) {
        constexpr bool ALL = decltype(whole)::value;
        Elems<uint32_t, C> word[4];
        Elems<uint16_t, 4 * C> scale[4];
        Eight<T> x[4][RT];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t k = k0 + i * 32 + quarter * 8;
            word[i] = load_elems<C>(Q + k / 8 * w.ldq, ALL ? C : k < ke ? there_q : 0);
            scale[i] = {};
            if ((i & (steps - 1)) == 0) scale[i] = load_elems<4 * C>(S + (k0 + i * 32) / w.group * w.lds, ALL ? 4 * C : k0 + i * 32 < ke ? there_s : 0);
#pragma unroll
            for (int t = 0; t < RT; ++t) x[i][t] = t * 16 + r < a.M ? load_eight(X + (t * 16 + r) * a.lda + k, ALL ? 8 : ke - k) : Eight<T>{};
        }
        v4f sum[RT][C] = {};
        Elems<uint16_t, 4 * C> of = {};
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
                    for (int p = PARTS - 1; p >= 0; --p) sum[t][q] = mma(f, part[t][p], sum[t][q]);
            }
            if (((i + 1) & (steps - 1)) == 0)
#pragma unroll
                for (int q = 0; q < C; ++q)
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[t][q][e] = fmaf(scale_value(of[e * C + q]), sum[t][q][e], acc[t][q][e]);
                        sum[t][q] = v4f{};
                    }
        }
    };
    int64_t k = kb + wave * BLOCK4;
    if (n0 + WIDE <= a.N)
        for (; k + BLOCK4 <= ke; k += FEW_WAVES * BLOCK4) block(k, std::true_type());
    for (; k < ke; k += FEW_WAVES * BLOCK4) block(k, std::false_type());
    leave_few<T, C, RT, GATED>(a, acc, lds, n0, 1.f / PLACE4<T>);
}

// Many rows: 128 x 128 results of four wavefronts, 64 values of k at a time.  Words become 16-byte pieces of places on their way to LDS, where X and W lie by k alike (see Operand).  The sums over a
// group are held apart from those over all of them.  fp32 elements: three planes of X, one stage; else two stages, of which one is fetched while the other is multiplied.
template <typename T, bool DIRECT, bool GATED>
__global__ __launch_bounds__(256, 2) void k_linear4_tile(TileArgs a, Weights4 w) {
    using U = Unit4<T>;
    constexpr int BM = 128, BN = 128, THREADS = 256, PARTS = PARTS4<T>, BK = 64, PLANE = BM * 128, WORDS = BN * 8 / THREADS;
    constexpr int STAGE = PARTS * PLANE + BN * 128, STAGES = PARTS == 1 ? 2 : 1, WIDE = GATED ? BN / 2 : BN;
    using OpX = Operand<U, BM, BY_K, THREADS>;
    using OpW = Operand<U, BN, BY_K, THREADS>;
    __shared__ __attribute__((aligned(16))) char stage0[STAGE], stage1[STAGES == 2 ? STAGE : 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, quarter = lane >> 4;
    int tm, tn;
    tile_place(a, tm, tn);
    const int64_t m0 = (int64_t)tm * BM;
    const int n0 = tn * WIDE;
    const int64_t kb = (int64_t)blockIdx.y * a.k_share, ke = kb + a.k_share < a.K ? kb + a.k_share : a.K;
    const T* const A = (const T*)a.A;
    const int wm = (wave / 2) * 64, wn = (wave % 2) * 64;
    const int steps = w.group / 32;
    // a column of the tile: of each 64 of a gated block's the first 32 are the gate's
    auto column = [&](int c) -> int64_t {
        const int h = GATED ? n0 + c / 64 * 32 + c % 32 : n0 + c;
        return (h < a.N ? h : a.N - 1) + (GATED && c % 64 >= 32 ? (int64_t)a.N : 0);
    };
    const uint32_t* const Q = w.Q + column(tid & (BN - 1));
    const int64_t last_word = (ke - 1) / 8;
    uint32_t word[WORDS];
    auto send_words = [&](int64_t k) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            const int64_t j = k / 8 + (i * THREADS + tid) / BN;
            word[i] = Q[(j < last_word ? j : last_word) * w.ldq];             // (X is 0 behind the last)
        }
    };
    auto put_words = [&](char* to) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            const int c = tid & (BN - 1), piece = (i * THREADS + tid) / BN;
            *reinterpret_cast<Vec<U>*>(to + c * 128 + ((piece ^ (c & 7)) << 4)) = places_of<U>(word[i], PLACE4<T>);
        }
    };
    constexpr int XS = BM * BK / (8 * THREADS);                               // eight elements of X at a time for each thread
    Eight<T> x[XS];
    auto send_rows = [&](int64_t k) {
#pragma unroll
        for (int i = 0; i < XS; ++i) {
            int row, piece;
            OpX::at(i * THREADS + tid, row, piece);
            const int64_t m = m0 + row < a.M ? m0 + row : a.M - 1, at = k + piece * 8;
            x[i] = load_eight(A + m * a.lda + at, at + 8 <= ke ? 8 : ke - at);
        }
    };
    auto put_rows = [&](char* to) {
#pragma unroll
        for (int i = 0; i < XS; ++i) {
            Vec<U> p[PARTS];
            parts_of<T>(x[i], p);
#pragma unroll
            for (int k = 0; k < PARTS; ++k) *reinterpret_cast<Vec<U>*>(to + k * PLANE + (i * THREADS + tid) * 16) = p[k];
        }
    };
    v4f acc[4][4] = {}, sum[4][4] = {};
    auto multiply = [&](const char* stage, int64_t k0) {
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            const int64_t k = k0 + step * 32;
            Vec<U> p[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) p[j] = OpW::fragment(stage + PARTS * PLANE, wn + j * 16, step, lane);
#pragma unroll
            for (int part = PARTS - 1; part >= 0; --part) {
                Vec<U> q[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = OpX::fragment(stage + part * PLANE, wm + i * 16, step, lane);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[i][j] = mma(p[j], q[i], sum[i][j]);
            }
            if (((k / 32 + 1) & (steps - 1)) == 0 || k + 32 >= ke) {           // the end of a group
                if (k >= ke) continue;
                const uint16_t* const S = w.S + k / w.group * w.lds;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float s[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[e] = scale_value(S[column(wn + j * 16 + quarter * 4 + e)]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(s[e], sum[i][j][e], acc[i][j][e]);
                        sum[i][j] = v4f{};
                    }
                }
            }
        }
    };
    auto fetch = [&](char* stage, int64_t k) {
        send_words(k);
        if (DIRECT && k + BK <= ke) OpX::direct((const U*)A, a.lda, m0, a.M, k, stage, tid);
        else send_rows(k);
    };
    auto put = [&](char* stage, int64_t k) {
        if (!(DIRECT && k + BK <= ke)) put_rows(stage);
        put_words(stage + PARTS * PLANE);
        if (DIRECT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    fetch(stage0, kb);
    put(stage0, kb);
    int64_t k = kb;
    if constexpr (STAGES == 2) {
        while (true) {
            const bool more = k + BK < ke;
            if (more) fetch(stage1, k + BK);
            multiply(stage0, k);
            if (!more) break;
            k += BK;
            put(stage1, k);
            const bool again = k + BK < ke;
            if (again) fetch(stage0, k + BK);
            multiply(stage1, k);
            if (!again) break;
            k += BK;
            put(stage0, k);
        }
    } else {
        while (true) {
            const bool more = k + BK < ke;
            if (more) fetch(stage0, k + BK);
            multiply(stage0, k);
            if (!more) break;
            k += BK;
            __syncthreads();
            put(stage0, k);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] *= 1.f / PLACE4<T>;
    constexpr int PART = 64 * 64 * 4;
    static_assert(STAGES == 2 ? 2 * PART <= STAGE : 4 * PART <= STAGE, "results have room");
    __syncthreads();
    char* const mine = STAGES == 2 ? (wave < 2 ? stage0 : stage1) + (wave & 1) * PART : stage0 + wave * PART;
    if constexpr (GATED) leave_gated<T, 4, 4, 1, false>(a, acc, mine, m0 + wm, n0 + wn / 2, lane);
    else leave_tile<T, 4, 4, 1, false, false>(a, acc, mine, m0 + wm, n0 + wn, lane);
}

template <typename T, int C, int RT, bool GATED>
static int launch_few4(TileArgs a, const Weights4& w, hipStream_t s) {
    constexpr int WIDE = GATED ? 8 * C : 16 * C, ALL = BLOCK4 * FEW_WAVES;
    const int strips = (a.N + WIDE - 1) / WIDE;
    int64_t splits = 1;
    if (strips < FEW_STRIPS) {
        splits = 128 / strips;
        const int64_t most = (a.K + ALL - 1) / ALL;
        if (splits > most) splits = most;
    }
    const int64_t blocks = (a.K + ALL - 1) / ALL;
    a.k_share = (blocks + splits - 1) / splits * ALL;
    splits = (a.K + a.k_share - 1) / a.k_share;
    ScratchLease lease;
    if (splits > 1) {
        void* p = nullptr;
        GCN_TRY(lease.get(&p, (size_t)splits * a.M * a.N * (GATED ? 8 : 4), s));
        a.part = (float*)p;
    }
    launch_lds<k_linear4_few<T, C, RT, GATED>>(dim3((unsigned)((strips + 7) / 8 * 8), (unsigned)splits), FEW_WAVES * 64, few_lds<T, C, RT>(), s, a, w, strips);
    GCN_LAUNCH_CHECK();
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
    if (sizeof(T) == 2 && whole_pieces<T, BY_K>(a.A, a.lda, a.K)) hipLaunchKernelGGL((k_linear4_tile<T, sizeof(T) == 2, GATED>), grid, dim3(256), 0, s, a, w);
    else hipLaunchKernelGGL((k_linear4_tile<T, false, GATED>), grid, dim3(256), 0, s, a, w);
    GCN_LAUNCH_CHECK();
    return splits > 1 ? launch_join<T, GATED>(a, splits, s) : GCN_OK;
}

template <typename T, bool GATED>
static int linear4_impl(const TileArgs& a, const Weights4& w, hipStream_t s) {
    if (a.M > 32) return launch_tile4<T, GATED>(a, w, s);
    const int64_t cus = device_info().cus, cols = GATED ? 2 * (int64_t)a.N : a.N;
    const int c = cols >= 64 * cus ? 4 : cols >= 32 * cus ? 2 : 1;            // as k_linear_few: the widest strips that are one for every compute unit
    if (a.M <= 16) return c == 4 ? launch_few4<T, 4, 1, GATED>(a, w, s) : c == 2 ? launch_few4<T, 2, 1, GATED>(a, w, s) : launch_few4<T, 1, 1, GATED>(a, w, s);
    return c == 4 ? launch_few4<T, 4, 2, GATED>(a, w, s) : c == 2 ? launch_few4<T, 2, 2, GATED>(a, w, s) : launch_few4<T, 1, 2, GATED>(a, w, s);
}

}  // namespace gcn
