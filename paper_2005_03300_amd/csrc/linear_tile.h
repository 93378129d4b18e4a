// Tiles of a matrix product for the matrix units: D (M x N) = A (M x K) B (K x N), of 32- (see linear_thirds.h) or 16-bit elements, sums in 32 bits, with what a linear
// layer does to its result where a tile leaves.  One kernel serves the three products of a layer and its backward pass, which differ in which of
// their dimensions lies contiguous in memory:
//   forward  X W      A by k, B by n
//   dX       dZ W^T   A by k, B by k   (the stored W is N x K)
//   dW       X^T dZ   A by m, B by n   (the stored X is K x M)
#pragma once
#include "rows.h"

namespace gcn {

enum Lies { BY_K = 0, BY_MN = 1 };

struct TileArgs {
    const void* A = nullptr;
    const void* B = nullptr;
    int64_t lda = 0, ldb = 0;
    int64_t M = 0, K = 0;
    int64_t k_share = 0;          // of one split: a multiple of the tile's depth
    int32_t N = 0;
    int32_t tiles_m = 0, tiles_n = 0;
    float* part = nullptr;        // partial results, one M x N each split; NULL: the epilogue runs here
    // D' = rho R + act(D + 1 bias^T); the argument of act is Z
    const float* bias = nullptr;
    const void* R = nullptr;
    void* Z = nullptr;
    void* Y = nullptr;
    int64_t ldr = 0, ldz = 0, ldy = 0;
    float rho = 0;
    int act = GCN_ACT_NONE;
};

// The normal distribution function Phi(z) and its density.  For 16-bit elements erfc by Abramowitz and Stegun's formula 7.1.26, off by 1.5e-7 at most, whose
// exponential is the density's (erff's way through its ranges made the activation of 16384 x 4096 elements 100 us).
template <typename T>
__device__ __forceinline__ float normal_cdf(float z, float& density) {
    if (sizeof(T) == 4) {
        density = 0.39894228040143268f * expf(-0.5f * z * z);
        return 0.5f * (1.f + erff(z * 0.70710678118654752f));
    }
    const float g = exp_for<T>(-0.5f * z * z), t = inverse(fmaf(0.3275911f * 0.70710678118654752f, fabsf(z), 1.f));
    float p = fmaf(1.061405429f, t, -1.453152027f);
    p = fmaf(p, t, 1.421413741f);
    p = fmaf(p, t, -0.284496736f);
    p = fmaf(p, t, 0.254829592f);
    const float tail = 0.5f * p * t * g;
    density = 0.39894228040143268f * g;
    return z < 0.f ? tail : 1.f - tail;
}
// act and its derivative.  NaN stays NaN.
template <typename T>
__device__ __forceinline__ float act_of(float z, int act) {
    if (act == GCN_ACT_RELU) return z < 0.f ? 0.f : z;
    if (act == GCN_ACT_GELU) {
        float density;
        return z * normal_cdf<T>(z, density);
    }
    if (act == GCN_ACT_SILU) return z * sigmoid<T>(z);
    return z;
}
template <typename T>
__device__ __forceinline__ float slope_of(float z, int act) {
    if (act == GCN_ACT_RELU) return z > 0.f ? 1.f : (z <= 0.f ? 0.f : z);
    if (act == GCN_ACT_GELU) {
        float density;
        const float phi = normal_cdf<T>(z, density);
        return fmaf(z, density, phi);
    }
    if (act == GCN_ACT_SILU) {
        const float s = sigmoid<T>(z);
        return s * fmaf(z, 1.f - s, 1.f);
    }
    return 1.f;
}

// What becomes of the results of row m, columns n to n + E - 1, of which `count` are there; r: the residual's, where they have been loaded already.
template <typename T>
__device__ __forceinline__ void finish(const TileArgs& a, int64_t m, int n, int count, float (&d)[Elem<T>::E], bool loaded, float (&r)[Elem<T>::E]) {
    constexpr int E = Elem<T>::E;
    if (a.bias) {
        float b[E];
        load_floats<E>(a.bias, n, count, 0.f, b);
#pragma unroll
        for (int e = 0; e < E; ++e) d[e] += b[e];
    }
    if (a.Z) store_vec_part((T*)a.Z + m * a.ldz + n, from_floats<T>(d), count);
    if (a.act != GCN_ACT_NONE)
#pragma unroll
        for (int e = 0; e < E; ++e) d[e] = act_of<T>(d[e], a.act);
    if (a.R) {
        if (!loaded) to_floats<T>(load_vec_part((const T*)a.R + m * a.ldr + n, count), r);
#pragma unroll
        for (int e = 0; e < E; ++e) d[e] = fmaf(a.rho, r[e], d[e]);
    }
    store_vec_part((T*)a.Y + m * a.ldy + n, from_floats<T>(d), count);
}

#if defined(__HIP_DEVICE_COMPILE__)
#define GCN_LDS(T, p) ((__attribute__((address_space(3))) T*)(p))
#endif

// One operand of a tile in LDS: R rows (of A) or columns (of B) by 128 bytes of k, as 16-byte pieces.
//   BY_K   R rows of 8 pieces; piece c of row r lies at c ^ (r & 7), so that the 16 rows that a fragment takes one piece of each
//          come from all banks.
//   BY_MN  one row per k of R elements; blocks of 16 elements are moved about within a row by a few bits of k, so that the rows that
//          a fragment takes together (four, or four of eight) lie in different banks.
// The place is the same whether pieces come straight from memory or through registers.
template <typename T, int R, int LIES, int THREADS>
struct Operand {
    static constexpr int E = Elem<T>::E, BK = 8 * E, PIECES = R * 8, PER = PIECES / THREADS, ROW = R / E;   // ROW: pieces of a row, BY_MN
    static constexpr int BLOCKS = R / 16 < 8 ? R / 16 : 8;
    static_assert(PIECES % THREADS == 0, "whole pieces for every thread");
    __device__ static int twist(int k) {                          // which block a row's first lies at
        return (sizeof(T) == 2 ? (k & 3) | ((k >> 3 & 1) << 2) : (k >> 2) & 3) & (BLOCKS - 1);
    }
    // piece `slot` of LDS: its row (of r or k) and which piece of that row in memory
    __device__ static void at(int slot, int& row, int& piece) {
        if (LIES == BY_K) {
            row = slot >> 3;
            piece = (slot & 7) ^ (row & 7);
        } else {
            row = slot / ROW;
            piece = (slot % ROW) ^ (twist(row) * (16 / E));
        }
    }
    // All of a tile's k are there, and rows lie in whole pieces at 16-byte addresses: memory to LDS without registers.  What lies beyond the
    // matrix along the other dimension is a copy of its last row or piece; its results are not stored.
    __device__ static void direct(const T* p, int64_t ld, int64_t r0, int64_t rows, int64_t k0, char* lds, int tid) {
        const int wave = tid & ~63;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            int row, piece;
            at(i * THREADS + tid, row, piece);
            const T* src;
            if (LIES == BY_K) {
                int64_t r = r0 + row;
                r = r < rows ? r : rows - 1;
                src = p + r * ld + k0 + piece * E;
            } else {
                int64_t r = r0 + piece * E;
                r = r < rows ? r : rows - E;
                src = p + (k0 + row) * ld + r;
            }
#if defined(__HIP_DEVICE_COMPILE__)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                             GCN_LDS(void, lds + (i * THREADS + wave) * 16), 16, 0, 0);
#endif
        }
    }
    // Any alignment and any k: through registers.  What lies beyond the matrix along the other dimension is, as with `direct`, something else of it; a piece that its
    // end cuts is the last whole one (see `piece_at`).
    struct Source {                                               // where a thread's pieces of the next stage are
        const T* src[PER];
    };
    __device__ static Source source(const T* p, int64_t ld, int64_t r0, int64_t rows, int64_t k0, int tid) {
        Source s;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            int row, piece;
            at(i * THREADS + tid, row, piece);
            if (LIES == BY_K) s.src[i] = p + (r0 + row < rows ? r0 + row : rows - 1) * ld + k0 + piece * E;
            else s.src[i] = p + (k0 + row) * ld + piece_at(r0 + piece * E, rows);
        }
        return s;
    }
    __device__ static void fetch(Source& s, int64_t ld, Vec<T> (&v)[PER]) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            v[i] = load_vec(s.src[i]);
            s.src[i] += LIES == BY_K ? (int64_t)BK : BK * ld;
        }
    }
    // A stage of which not all k are there: zeros for the others, in both operands.  Also rows shorter than a piece.
    __device__ static void fetch_end(const T* p, int64_t ld, int64_t r0, int64_t rows, int64_t k0, int64_t K, Vec<T> (&v)[PER], int tid) {
        if (LIES == BY_K && K < E) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                int row, piece;
                at(i * THREADS + tid, row, piece);
                v[i] = load_vec_part(p + (r0 + row < rows ? r0 + row : rows - 1) * ld, piece == 0 ? (int)K : 0);
            }
            return;
        }
        if (LIES == BY_K) {
            Words<T, E> x[PER];
            int by[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                int row, piece;
                at(i * THREADS + tid, row, piece);
                x[i] = load_near<E>(p + (r0 + row < rows ? r0 + row : rows - 1) * ld, k0 + piece * E, K);
                by[i] = settle_by<E>(k0 + piece * E, K);
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) v[i] = settle<E, T>(x[i], by[i]);
            return;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            int row, piece;
            at(i * THREADS + tid, row, piece);
            const int64_t r = r0 + piece * E, k = k0 + row;
            if (rows >= E) v[i] = k < K ? load_vec(p + k * ld + piece_at(r, rows)) : Vec<T>{};
            else v[i] = k < K && r == 0 ? load_vec_part(p + k * ld, (int)rows) : Vec<T>{};
        }
    }
    // Where the piece from r on (a multiple of E) of a dimension that is contiguous in memory is taken from.
    __device__ static int64_t piece_at(int64_t r, int64_t rows) { return r + E <= rows ? r : rows - E; }
    __device__ static void put(const Vec<T> (&v)[PER], char* lds, int tid) {
#pragma unroll
        for (int i = 0; i < PER; ++i) *reinterpret_cast<Vec<T>*>(lds + (i * THREADS + tid) * 16) = v[i];
    }
    // The fragment of 16 rows (from r on) and the `step`th 64 bytes of k: lane l has row l % 16 and the E values of k that its quarter l / 16 stands for.
    __device__ static Vec<T> fragment(const char* lds, int r, int step, int lane) {
        if (LIES == BY_K) {
            const int row = r + (lane & 15);
            return *reinterpret_cast<const Vec<T>*>(lds + row * 128 + (((step * 4 + (lane >> 4)) ^ (row & 7)) << 4));
        }
#if defined(__HIP_DEVICE_COMPILE__)
        if constexpr (sizeof(T) == 2) {
            typedef short s4 __attribute__((ext_vector_type(4)));
            typedef short s8 __attribute__((ext_vector_type(8)));
            // Sixteen lanes read four rows of k by 16 columns, 8 bytes each, and receive a column each.
            const int k = step * 32 + (lane >> 4) * 8 + ((lane & 15) >> 2), c = (lane & 3) * 8;
            const char* const p0 = lds + (int64_t)k * (R * 2) + ((((r >> 4) ^ twist(k)) << 5) + c);
            const char* const p1 = lds + (int64_t)(k + 4) * (R * 2) + ((((r >> 4) ^ twist(k + 4)) << 5) + c);
            const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(GCN_LDS(s4, p0));
            const s4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(GCN_LDS(s4, p1));
            return __builtin_bit_cast(Vec<T>, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        }
#endif
        Vec<T> v = {};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int k = step * (4 * E) + (lane >> 4) * E + e;
            v[e] = *reinterpret_cast<const T*>(lds + (int64_t)k * (R * sizeof(T)) + ((((r >> 4) ^ twist(k)) * 16 + (lane & 15)) * sizeof(T)));
        }
        return v;
    }
};

// acc += P Q over 64 bytes of k: P 16 rows, Q 16 columns.  With f32 elements four products of four k each; the k of a lane's quarter are consecutive,
// which orders the sum's terms differently and needs one 16-byte read.
__device__ __forceinline__ v4f mma(Vec<__bf16> p, Vec<__bf16> q, v4f acc) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, q, acc, 0, 0, 0);
#else
    return acc;
#endif
}
__device__ __forceinline__ v4f mma(Vec<_Float16> p, Vec<_Float16> q, v4f acc) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(p, q, acc, 0, 0, 0);
#else
    return acc;
#endif
}
__device__ __forceinline__ v4f mma(Vec<float> p, Vec<float> q, v4f acc) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(p[e], q[e], acc, 0, 0, 0);
#endif
    return acc;
}

// The tile of a workgroup.  Neighbouring workgroups run on different XCDs, each with an L2 of its own: every XCD gets a contiguous share of the tiles, and walks it in
// groups of eight rows of tiles, column by column, so that what runs at one time shares operands.
__device__ __forceinline__ void tile_place(const TileArgs& a, int& tm, int& tn) {
    const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n, b = blockIdx.x, x = b & 7, q = tiles >> 3, r = tiles & 7;
    const int64_t t = (x < r ? x * (q + 1) : r * (q + 1) + (x - r) * q) + (b >> 3);
    const int64_t per = (int64_t)8 * a.tiles_n, g = t / per;
    const int first = (int)(g * 8), rows = a.tiles_m - first < 8 ? a.tiles_m - first : 8, in = (int)(t % per);
    tm = first + in % rows;
    tn = in / rows;
}

// A wavefront's results, 16 FM rows from m0 and 16 FN columns from n0 on, leave through LDS, its own part `mine` of it, in PHASES: what the matrix unit leaves with a
// lane are four columns of a row, and whole rows of the wavefront's tile go out together, 16 bytes per lane.  The pieces of a row are moved about by the row, so that
// the lanes' writes meet all banks.  CUT_M, CUT_N: pieces that the end of a dimension cuts were taken from its last whole one.
template <typename T, int FM, int FN, int PHASES, bool CUT_M, bool CUT_N>
__device__ __forceinline__ void leave_tile(const TileArgs& a, const v4f (&acc)[FM][FN], char* mine, int64_t m0, int n0, int lane) {
    constexpr int E = Elem<T>::E, FP = FM / PHASES, ROWS = FP * 16, PIECES = FN * 4;
    static_assert(FM % PHASES == 0, "whole phases");
    float* const part = a.part ? a.part + (int64_t)blockIdx.y * a.M * a.N : nullptr;
#pragma unroll
    for (int ph = 0; ph < PHASES; ++ph) {
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const int row = i * 16 + (lane & 15);
                *reinterpret_cast<v4f*>(mine + row * (PIECES * 16) + (((j * 4 + (lane >> 4)) ^ (row & (PIECES - 1))) << 4)) = acc[ph * FP + i][j];
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        constexpr int LANES = FN * 16 / E, STEP = 64 / LANES;     // lanes of a row, rows at a time
        const int c = (lane % LANES) * E, n = n0 + c, count = a.N - n;
        // a piece that the end of a dimension cut holds the last whole one: its last `count` columns, and likewise rows
        const bool shifted = CUT_N && count < E && a.N >= E;
        // the residual's pieces of several rows are on their way together (one after the other: 130 us of 16384 x 4096 x 4096 in bf16)
        constexpr int AHEAD = ROWS / STEP < 4 ? ROWS / STEP : 4;
        const bool ahead = !part && a.R && a.N >= E;
        const int by = settle_by<E>(n, a.N);
#pragma nounroll
        for (int row0 = lane / LANES; row0 < ROWS; row0 += AHEAD * STEP) {
            Words<T, E> near[AHEAD] = {};
            if (ahead)
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const int64_t m = m0 + ph * ROWS + row0 + u * STEP;
                    near[u] = load_near<E>((const T*)a.R + (m < a.M ? m : a.M - 1) * a.ldr, n, a.N);
                }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int row = row0 + u * STEP;
                int64_t m = m0 + ph * ROWS + row;
                float d[E];
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const v4f x = *reinterpret_cast<const v4f*>(mine + row * (PIECES * 16) + ((((c + e) / 4) ^ (row & (PIECES - 1))) << 4));
#pragma unroll
                    for (int q = 0; q < 4; ++q) d[e + q] = x[q];
                }
                if (CUT_M && a.M >= E) {
                    const int64_t first = m - row % E;             // of the piece (a wavefront's rows are whole ones)
                    if (first + E > a.M) {
                        if (first >= a.M) continue;
                        m += a.M - E - first;
                        if (m < first) continue;
                    }
                }
                if (m >= a.M || count <= 0) continue;
                if (shifted)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        float x = d[e];
#pragma unroll
                        for (int o = 1; o < E; ++o) x = e + o < E && E - count == o ? d[e + o < E ? e + o : e] : x;
                        d[e] = x;
                    }
                if (part) {
                    float* const p = part + m * a.N + n;
                    if (count >= E)
#pragma unroll
                        for (int e = 0; e < E; e += 4) *reinterpret_cast<f4u*>(p + e) = f4u{d[e], d[e + 1], d[e + 2], d[e + 3]};
                    else
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            if (e < count) p[e] = d[e];
                } else {
                    float r[E];
                    floats_of<E, T>(by ? settle<E, T>(near[u], by) : __builtin_bit_cast(Vec<T>, near[u]), r);
                    finish<T>(a, m, n, count, d, ahead, r);
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// D = A B for 16-bit elements: BM x BN results of a workgroup of WM x WN wavefronts, 128 bytes of k (64 values) at a time, two such stages in LDS: one is
// fetched while the other is multiplied.  A wavefront's results are the transpose of what the matrix unit is given (B's columns as its rows), so that a lane
// holds four neighbouring columns of one row.
// Large products: 16384 x 4096 x 4096 in bf16 435 to 475 us (1.16 to 1.27 PFLOP/s, the library's rate) in each of the three directions; the matrix units are busy in 47 % of the
// cycles, epilogue included, in the library's product of 8192 x 8192 x 8192 in 73 % at a lower clock.  A 256 x 256 tile reads
// each operand half as often from L2 as 128 x 128 and LDS as often per product as its wavefronts' 128 x 64 results ask for (the units take 2048 cycles of a stage, LDS
// 1536); 128 x 128 has two workgroups on a compute unit, so that one's end overlaps the other's products (1.05 PFLOP/s), and 64 x 64 is for results too small to fill
// the chip otherwise.  128 bytes of k are a cache line of a row, and one barrier for 64 (256 x 256) products of a wavefront.
// DIRECT: rows of both operands at 16-byte addresses in whole pieces: memory to LDS without registers.  (Through registers the 256 x 256 tile spills 23 of them forward and
// 60 for dW.)
template <typename T, int BM, int BN, int WM, int WN, int LA, int LB, bool DIRECT>
__global__ __launch_bounds__(WM* WN * 64, BM == 64 ? 4 : 2) void k_linear_tile(TileArgs a) {
    constexpr int THREADS = WM * WN * 64, E = Elem<T>::E, BK = 8 * E;
    constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
    constexpr int STAGE = (BM + BN) * 128;
    using OpA = Operand<T, BM, LA, THREADS>;
    using OpB = Operand<T, BN, LB, THREADS>;
    // Two arrays, so that the compiler can tell what is on its way to the one from what is read of the other: it makes a transposing read wait for everything
    // that may be on its way to the same array (16384 x 4096 x 4096 in bf16 with one: 935 TFLOP/s).
    __shared__ __attribute__((aligned(16))) char stage0[STAGE], stage1[STAGE];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int tm, tn;
    tile_place(a, tm, tn);
    const int64_t m0 = (int64_t)tm * BM;
    const int n0 = tn * BN;
    const int64_t kb = (int64_t)blockIdx.y * a.k_share, ke = kb + a.k_share < a.K ? kb + a.k_share : a.K;
    const T* const A = (const T*)a.A;
    const T* const B = (const T*)a.B;
    const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
    v4f acc[FM][FN] = {};

    auto multiply = [&](const char* stage) {
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            Vec<T> p[FN], q[FM];
#pragma unroll
            for (int j = 0; j < FN; ++j) p[j] = OpB::fragment(stage + BM * 128, wn + j * 16, step, lane);
#pragma unroll
            for (int i = 0; i < FM; ++i) q[i] = OpA::fragment(stage, wm + i * 16, step, lane);
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = mma(p[j], q[i], acc[i][j]);
        }
    };
    const int64_t whole = DIRECT ? (ke - kb) / BK : 0;
    if (DIRECT && whole > 0) {
        auto send = [&](char* stage, int64_t t) {
            OpA::direct(A, a.lda, m0, a.M, kb + t * BK, stage, tid);
            OpB::direct(B, a.ldb, n0, a.N, kb + t * BK, stage + BM * 128, tid);
        };
        auto arrived = []() {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
        };
        send(stage0, 0);
        arrived();
        for (int64_t t = 0; t < whole; t += 2) {
            if (t + 1 < whole) send(stage1, t + 1);
            multiply(stage0);
            arrived();
            if (t + 1 == whole) break;
            if (t + 2 < whole) send(stage0, t + 2);
            multiply(stage1);
            arrived();
        }
    }
    int64_t k = kb + whole * BK;
    if (k < ke) {
        Vec<T> va[OpA::PER], vb[OpB::PER];
        // whole stages one after the other, then what is left; none are whole where rows are shorter than a piece
        const int64_t end = DIRECT || (LA == BY_MN && a.M < E) || (LB == BY_MN && a.N < E) ? k : k + (ke - k) / BK * BK;
        typename OpA::Source sa;
        typename OpB::Source sb;
        if (!DIRECT && k < end) {
            sa = OpA::source(A, a.lda, m0, a.M, k, tid);
            sb = OpB::source(B, a.ldb, n0, a.N, k, tid);
        }
        auto next = [&]() {
            if (!DIRECT && k < end) {
                OpA::fetch(sa, a.lda, va);
                OpB::fetch(sb, a.ldb, vb);
            } else {
                OpA::fetch_end(A, a.lda, m0, a.M, k, ke, va, tid);
                OpB::fetch_end(B, a.ldb, n0, a.N, k, ke, vb, tid);
            }
        };
        auto step = [&](char* stage) {
            OpA::put(va, stage, tid);
            OpB::put(vb, stage + BM * 128, tid);
            __syncthreads();
            k += BK;
            if (!DIRECT && k < ke) next();
            multiply(stage);
        };
        next();
        step(stage0);                                             // (DIRECT: the only one)
        if (!DIRECT)
            while (k < ke) {
                step(stage1);
                if (k < ke) step(stage0);
            }
    }
    constexpr int PHASES = (BM * BN * 4 + 2 * STAGE - 1) / (2 * STAGE), PART = BM / WM / PHASES * (BN / WN) * 4;
    constexpr int HALF = WM * WN / 2;                             // wavefronts that have their part in the first stage
    static_assert(HALF * PART <= STAGE, "results have room");
    __syncthreads();
    leave_tile<T, FM, FN, PHASES, LA == BY_MN && !DIRECT, LB == BY_MN && !DIRECT>(a, acc, (wave < HALF ? stage0 : stage1) + (wave % HALF) * PART, m0 + wm,
                                                                                 n0 + wn, lane);
}

// The partial results of the splits, added in order, and what the layer does with the sum: 16 bytes of it per thread; SHARES threads, a wavefront apart, take a
// share of the splits each where there are many of them and few results (one thread after 211 of them: 60 us).
template <typename T, int SHARES>
__global__ __launch_bounds__(64 * (SHARES > 1 ? SHARES : 4)) void k_linear_join(TileArgs a, int splits) {
    constexpr int E = Elem<T>::E, PER = SHARES > 1 ? 64 : 256;
    __shared__ float add[SHARES > 1 ? SHARES : 1][SHARES > 1 ? 64 : 1][E + 1];
    const int64_t per = (a.N + E - 1) / E, t = (int64_t)blockIdx.x * PER + threadIdx.x % PER;
    const int share = threadIdx.x / PER;
    const int64_t m = t / per;
    const int n = (int)(t % per) * E, count = a.N - n;
    float d[E] = {};
    if (m < a.M) {
        const float* const p = a.part + m * a.N + n;
#pragma unroll 4
        for (int s = share; s < splits; s += SHARES) {
            float x[E];
            load_floats<E>(p + (int64_t)s * a.M * a.N, 0, count, 0.f, x);
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] += x[e];
        }
    }
    if constexpr (SHARES > 1) {
#pragma unroll
        for (int e = 0; e < E; ++e) add[share][threadIdx.x % PER][e] = d[e];
        __syncthreads();
        if (share) return;
        for (int w = 1; w < SHARES; ++w)
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] += add[w][threadIdx.x][e];
    }
    float r[E];
    if (m < a.M) finish<T>(a, m, n, count, d, false, r);
}

template <typename T> int linear_forward_of(const TileArgs& a, hipStream_t s);          // A by k, B by n, with the epilogue
template <typename T> int linear_dx_of(const TileArgs& a, hipStream_t s);               // A by k, B by k
template <typename T> int linear_dw_of(const TileArgs& a, hipStream_t s);               // A by m, B by n

}  // namespace gcn
