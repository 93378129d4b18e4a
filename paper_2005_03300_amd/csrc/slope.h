// The elementwise part of a backward pass: what the gradient of a layer's output becomes in front of its products.  Of a gated block, whose Z = [Zg Zu] has 2 N columns,
//   dZg = dH Zu act'(Zg),  dZu = dH act(Zg),  H = act(Zg) Zu again,
// and of a linear layer, dZ = dY act'(Z), dR = rho dY.  With the column sums of dZ, of the products before they are rounded.
#pragma once
#include "held.h"
#include "launch_rules.h"
#include "linear_tile.h"
#include "sum_parts.h"

namespace gcn {

// A matrix that the forward pass kept: elements, or a checkpoint of them.
struct Kept {
    const void* p = nullptr;          // elements, or codes where there are scales
    int64_t ld = 0;
    const uint16_t* scales = nullptr;
    int64_t lds = 0;
};

struct SlopeArgs {
    int64_t n = 0, rows_per_block = 0;
    int32_t N = 0;                    // columns of dY
    Kept Z;
    const void* dY = nullptr;
    void* dZ = nullptr;
    void* also = nullptr;             // H of a gated block, dR of a linear layer; or NULL
    int64_t lddy = 0, lddz = 0, ldalso = 0;
    int act = GCN_ACT_NONE;
    int lanes = 64;                   // of a wavefront for a row
    float rho = 1;
    float* part = nullptr;            // sums of each share of the rows, or NULL
};

// Of gated blocks, and of linear layers from a checkpoint of Z (from elements see k_linear_slope): one pass over the matrices, bound by memory.  A workgroup has 64 lanes of 16 bytes by four rows at a time, two
// or four such sets on their way, and a share of the rows; the four row sets are added in order.  A wavefront has several rows where they are short, `lanes`
// of it for each, a power of two, and folds their sums first (56450 x 20 of a gated block in fp16: all 64 lanes for a row 106 us, four 18);
// rows that would leave an eighth of the lanes idle are cut into strips of 32 or 16 (16384 x 720 in fp16 41 us with 64, 37 with 32; 16508 x 300 in bf16 from a checkpoint 39 and, with 16, 34).
// dZ is rounded to the element type here: both products take it from memory, and 16-bit matrix units take no more.  As the sum of two 16-bit numbers it would lose
// nothing that counts, and both products would be twice as long (8192 x 1024 x 4096 in fp16: 160 us more on 210).  So dX and dW are off by what the roundings of dZ come to, about as much as by their own
// (2.9e-4 of their norm in fp16 where the sum of an unrounded dZ has 2.1e-4, 2.3e-3 and 1.7e-3 in bf16); the bias's gradient is the sum of what was not rounded.
template <typename T, bool GATED, bool HELD>
__global__ __launch_bounds__(256) void k_slope(SlopeArgs a) {
    constexpr int E = Elem<T>::E, WAVES = 4, AHEAD = GATED ? 2 : 4, HALVES = GATED ? 2 : 1;
    static_assert(GATED || HELD, "linear layers from elements have k_linear_slope");
    __shared__ float sums[WAVES][64][HALVES * E + 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lanes = a.lanes, SETS = WAVES * (64 / lanes), set = (int)threadIdx.x / lanes;
    const int32_t N = a.N;
    const int64_t c = ((int64_t)blockIdx.x * lanes + (lane & (lanes - 1))) * E, width = (int64_t)HALVES * N;
    const int64_t rb = (int64_t)blockIdx.y * a.rows_per_block, re = rb + a.rows_per_block < a.n ? rb + a.rows_per_block : a.n;
    const int count = c >= N ? 0 : N - c < E ? (int)(N - c) : E;
    const bool apart = GATED && N % E != 0;                       // a piece of the second half can lie in two groups
    float sum[HALVES][E] = {};
    struct Piece {                                                // of a row: dY's elements, and Z's or their codes
        Vec<T> y, z[HALVES];
        Codes<E> q[HALVES];
        uint16_t s[HALVES][2];
    };
    auto load = [&](int64_t i, auto whole) {
        Piece p = {};
        // E elements of a row of `len` from `along` on; behind its end zeros, or what else the row has there
        auto part = [&](const T* row, int64_t along, int64_t len) {
            if (decltype(whole)::value) return load_vec(row + along);
            if (len >= E) return __builtin_bit_cast(Vec<T>, settle<E, T>(load_near<E>(row, along, len), settle_by<E>(along, len)));
            return load_vec_part(row + along, len - along < E ? (int)(len - along) : E);
        };
        p.y = part((const T*)a.dY + i * a.lddy, c, N);
        if (!GATED && a.act == GCN_ACT_NONE) return p;
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const int64_t at = (int64_t)h * N + c;
            if constexpr (HELD) {
                p.q[h] = load_codes<E>((const int8_t*)a.Z.p + i * a.Z.ld, at, width);
                const int64_t g = at / CHECKPOINT_GROUP, last = (at + count - 1) / CHECKPOINT_GROUP;
                p.s[h][0] = a.Z.scales[i * a.Z.lds + g];
                if (apart) p.s[h][1] = a.Z.scales[i * a.Z.lds + last];
            } else {
                p.z[h] = part((const T*)a.Z.p + i * a.Z.ld, at, width);
            }
        }
        return p;
    };
    auto row = [&](int64_t i, const Piece& p) {
        float g[E], z[HALVES][E], d[HALVES][E], other[E];
        to_floats<T>(p.y, g);
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
            if constexpr (HELD) {
                const float s0 = scale_value(p.s[h][0]);
                if (h == 1 && apart) {
                    const int here = CHECKPOINT_GROUP - (int)(((int64_t)h * N + c) % CHECKPOINT_GROUP);
                    const float s1 = scale_value(p.s[h][1]);
#pragma unroll
                    for (int e = 0; e < E; ++e) z[h][e] = (float)(T)((e < here ? s0 : s1) * code_value<E>(p.q[h], e));
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) z[h][e] = (float)(T)(s0 * code_value<E>(p.q[h], e));
                }
            } else {
                to_floats<T>(p.z[h], z[h]);
            }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if constexpr (GATED) {
                const float act = act_of<T>(z[0][e], a.act);
                d[0][e] = g[e] * z[1][e] * slope_of<T>(z[0][e], a.act);
                d[1][e] = g[e] * act;
                other[e] = act * z[1][e];
            } else {
                d[0][e] = a.act == GCN_ACT_NONE ? g[e] : g[e] * slope_of<T>(z[0][e], a.act);
                other[e] = a.rho * g[e];
            }
        }
        if (a.also) store_vec_part((T*)a.also + i * a.ldalso + c, from_floats<T>(other), count);
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            if (a.dZ) store_vec_part((T*)a.dZ + i * a.lddz + (int64_t)h * N + c, from_floats<T>(d[h]), count);
#pragma unroll
            for (int e = 0; e < E; ++e) sum[h][e] += d[h][e];
        }
    };
    auto rows = [&](auto whole) {
        for (int64_t i = rb + set; i < re; i += AHEAD * SETS) {
            Piece p[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) p[u] = load(i + u * SETS < re ? i + u * SETS : i, whole);       // (the first again where there is no second)
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (i + u * SETS < re) row(i + u * SETS, p[u]);
        }
    };
    // a workgroup whose columns are not all whole pieces goes the other way with all of them: two ways one after the other took twice as long (4099 x 1001 of a gated block from a checkpoint in bf16: 22 us, 32)
    if (((int64_t)blockIdx.x + 1) * lanes * E <= N || N % E == 0) {
        if (count > 0) rows(std::true_type());
    } else if (count > 0) {
        rows(std::false_type());
    }
    if (!a.part) return;
    for (int d = 32; d >= lanes; d >>= 1)                         // the rows of a wavefront
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
#pragma unroll
            for (int e = 0; e < E; ++e) sum[h][e] += __shfl_xor(sum[h][e], d);
#pragma unroll
    for (int h = 0; h < HALVES; ++h)
#pragma unroll
        for (int e = 0; e < E; ++e) sums[wave][lane][h * E + e] = sum[h][e];
    __syncthreads();
    if (wave || lane >= lanes) return;
#pragma unroll
    for (int h = 0; h < HALVES; ++h)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            for (int w = 1; w < WAVES; ++w) sum[h][e] += sums[w][lane][h * E + e];
            if (e < count) a.part[(int64_t)blockIdx.y * width + (int64_t)h * N + c + e] = sum[h][e];
        }
}

// The sums of the shares of the rows, added in order: 64 columns for each workgroup.
int launch_column_sums(const float* part, int parts, int32_t count, float* out, hipStream_t s);
// The elementwise part of a linear layer whose Z is elements.
int launch_linear_slope(int type, SlopeArgs a, float* dbias, hipStream_t s);

template <typename T, bool GATED, bool HELD>
static int launch_slope(SlopeArgs a, float* dbias, hipStream_t s) {
    constexpr int E = Elem<T>::E;
    auto taken = [&](int lanes) { return (a.N + lanes * E - 1) / (lanes * E) * lanes; };           // lanes for a row, idle ones among them
    for (; a.lanes > 1 && a.lanes / 2 * E >= a.N; a.lanes /= 2) {}
    for (int lanes = a.lanes / 2; lanes >= 16; lanes /= 2)
        if (8 * taken(lanes) <= 7 * taken(a.lanes)) a.lanes = lanes;
    const int64_t wide = a.lanes * E, across = (a.N + wide - 1) / wide, width = (int64_t)a.N * (GATED ? 2 : 1), together = 64 / a.lanes;
    RowShares shares = row_shares((a.n + together - 1) / together, across, device_info().cus);       // of as many rows as a wavefront has together
    a.rows_per_block = shares.rows *= together;
    shares.count = (a.n + shares.rows - 1) / shares.rows;
    ScratchLease lease;
    void* part = dbias;                                           // the sums of a single share of the rows are the result
    if (dbias && shares.count > 1) GCN_TRY(lease.get(&part, (size_t)shares.count * width * 4, s));
    a.part = (float*)part;
    hipLaunchKernelGGL((k_slope<T, GATED, HELD>), dim3((unsigned)across, (unsigned)shares.count), dim3(256), 0, s, a);
    GCN_LAUNCH_CHECK();
    return dbias && shares.count > 1 ? launch_column_sums(a.part, (int)shares.count, (int32_t)width, dbias, s) : GCN_OK;
}

// dX = G W^T and dW = X^T G, each where it is wanted, for the n x cols gradient G.
struct BackProducts {
    int64_t n = 0;
    int32_t f_in = 0, cols = 0;
    Kept X;
    const void* W = nullptr;
    const void* G = nullptr;
    void* dX = nullptr;
    void* dW = nullptr;
    int64_t ldw = 0, ldg = 0, lddx = 0, lddw = 0;
};
int back_products(int type, const BackProducts& b, hipStream_t s);

// The bytes of a kept matrix, for the checks of operands.
inline Span span_of(const Kept& k, int64_t rows, int64_t cols, size_t bytes) { return Span(k.p, rows, cols, k.ld, k.scales ? 1 : bytes); }
inline Span scales_of(const Kept& k, int64_t rows, int64_t cols) { return Span(k.scales, rows, groups_of(cols, CHECKPOINT_GROUP), k.lds, 2); }

}  // namespace gcn
