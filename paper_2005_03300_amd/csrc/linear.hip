// A linear layer with what follows it: Y = rho R + act(X W + 1 bias^T), and its gradients, on 32- and 16-bit elements.
#include "launch_rules.h"
#include "linear_tile.h"
#include "sum_parts.h"

namespace gcn {

// dZ = dY * act'(Z), dR = rho dY, and the column sums of dZ (the bias gradient, of the unrounded products): one pass over the matrices for the elementwise
// part, bound by memory (8192 x 4096 in fp16 with SiLU: 201 MB in 45 us, 4.5 TB/s).  A workgroup has 64 lanes of 16 bytes by four rows at a time, two such sets on their way,
// and a share of the rows; the four row sets are added in order.
// dZ is rounded to the element type here: both products take it from memory, and 16-bit matrix units take no more.  As the sum of two 16-bit numbers it would lose
// nothing that counts, and both products would be twice as long (8192 x 1024 x 4096 in fp16: 160 us more on 210).  So dX and dW are off by what the roundings of dZ come to, about as much as by their own
// (2.9e-4 of their norm in fp16 where the sum of an unrounded dZ has 2.1e-4, 2.3e-3 and 1.7e-3 in bf16); the bias's gradient is the sum of what was not rounded.
template <typename T>
__global__ __launch_bounds__(256) void k_linear_slope(int64_t n, int32_t N, int64_t rows_per_block, const T* Z, int64_t ldz,
                                                      const T* dY, int64_t lddy, int act, float rho, T* dZ, int64_t lddz, T* dR,
                                                      int64_t lddr, float* __restrict__ part) {
    constexpr int E = Elem<T>::E, SETS = 4, AHEAD = 2;
    __shared__ float sums[SETS][64][E + 1];
    const int lane = threadIdx.x & 63, set = threadIdx.x >> 6;
    const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * E;
    const int64_t rb = (int64_t)blockIdx.y * rows_per_block, re = rb + rows_per_block < n ? rb + rows_per_block : n;
    const int count = c >= N ? 0 : N - c < E ? (int)(N - c) : E;
    float sum[E] = {};
    auto row = [&](int64_t i, Vec<T> y, Vec<T> z) {
        float d[E], g[E];
        to_floats<T>(y, g);
#pragma unroll
        for (int e = 0; e < E; ++e) d[e] = g[e];
        if (act != GCN_ACT_NONE) {
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] *= slope_of<T>((float)z[e], act);
            if (dZ) store_vec_part(dZ + i * lddz + c, from_floats<T>(d), count);
        }
        if (dR) {
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] *= rho;
            store_vec_part(dR + i * lddr + c, from_floats<T>(g), count);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += d[e];
    };
    if (count == E) {
        for (int64_t i = rb + set; i < re; i += AHEAD * SETS) {
            Vec<T> y[AHEAD], z[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int64_t at = i + u * SETS < re ? i + u * SETS : i;           // (the first again where there is no second)
                y[u] = load_vec(dY + at * lddy + c);
                if (act != GCN_ACT_NONE) z[u] = load_vec(Z + at * ldz + c);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (i + u * SETS < re) row(i + u * SETS, y[u], z[u]);
        }
    } else if (count > 0 && N >= E) {
        const int by = settle_by<E>(c, N);
        for (int64_t i = rb + set; i < re; i += SETS) {
            const Words<T, E> y = load_near<E>(dY + i * lddy, c, N);
            Words<T, E> z = {};
            if (act != GCN_ACT_NONE) z = load_near<E>(Z + i * ldz, c, N);
            row(i, settle<E, T>(y, by), settle<E, T>(z, by));
        }
    } else if (count > 0) {
        for (int64_t i = rb + set; i < re; i += SETS)
            row(i, load_vec_part(dY + i * lddy + c, count), act != GCN_ACT_NONE ? load_vec_part(Z + i * ldz + c, count) : Vec<T>{});
    }
    if (!part) return;
#pragma unroll
    for (int e = 0; e < E; ++e) sums[set][lane][e] = sum[e];
    __syncthreads();
    if (set) return;
    for (int w = 1; w < SETS; ++w)
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += sums[w][lane][e];
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e < count) part[(int64_t)blockIdx.y * N + c + e] = sum[e];
}

// The partial results of the shares of the rows, added in order (see sum_of_parts): 64 columns for each workgroup.
__global__ __launch_bounds__(1024) void k_vector_sums(const float* __restrict__ part, int parts, int32_t count, float* __restrict__ out) {
    __shared__ float s_sum[16][64];
    sum_of_parts(blockIdx.x, 1, count, parts, 0, part, 16, s_sum, [&](int, int c, float s) { out[c] = s; });
}

template <typename T>
static int slope_launch(int64_t n, int32_t N, const void* Z, int64_t ldz, const void* dY, int64_t lddy, int act, float rho, void* dZ,
                        int64_t lddz, void* dR, int64_t lddr, float* dbias, hipStream_t s) {
    const int64_t wide = 64 * Elem<T>::E, across = (N + wide - 1) / wide;
    const RowShares shares = row_shares(n, across, device_info().cus);
    const int64_t per = shares.rows, blocks = shares.count;
    ScratchLease lease;
    void* part = dbias;                                           // the sums of a single share of the rows are the result
    if (dbias && blocks > 1) GCN_TRY(lease.get(&part, (size_t)blocks * N * 4, s));
    hipLaunchKernelGGL(k_linear_slope<T>, dim3((unsigned)across, (unsigned)blocks), dim3(256), 0, s, n, N, per, (const T*)Z, ldz,
                       (const T*)dY, lddy, act, rho, (T*)dZ, lddz, (T*)dR, lddr, (float*)part);
    GCN_LAUNCH_CHECK();
    if (dbias && blocks > 1) {
        hipLaunchKernelGGL(k_vector_sums, dim3((unsigned)column_sum_groups(N)), dim3(1024), 0, s, (const float*)part, (int)blocks, N, dbias);
        GCN_LAUNCH_CHECK();
    }
    return GCN_OK;
}

}  // namespace gcn

using namespace gcn;

static bool known_act(int act) { return act >= GCN_ACT_NONE && act <= GCN_ACT_SILU; }

extern "C" int gcn_linear_forward(int64_t n, int32_t f_in, int32_t f_out, int type, const void* X, int64_t ldx, const void* W,
                                  int64_t ldw, const float* bias, int act, const void* R, int64_t ldr, float rho, void* Z,
                                  int64_t ldz, void* Y, int64_t ldy, void* stream) {
    static const char* const who = "gcn_linear_forward";
    if (!X || !W || !Y) return fail(GCN_ERR_BADARG, "%s: NULL argument", who);
    if (!known_type(type)) return fail(GCN_ERR_BADARG, "%s: unknown element type %d", who, type);
    if (!known_act(act)) return fail(GCN_ERR_BADARG, "%s: unknown activation %d", who, act);
    if (n <= 0 || f_in <= 0 || f_out <= 0) return fail(GCN_ERR_BADARG, "%s: sizes must be positive", who);
    if (f_in > LINEAR_WIDEST || f_out > LINEAR_WIDEST) return fail(GCN_ERR_RANGE, "%s: widths go up to 2^27", who);
    if (ldx < f_in || ldw < f_out || ldy < f_out || (R && ldr < f_out) || (Z && ldz < f_out))
        return fail(GCN_ERR_BADARG, "%s: leading dimension below the width", who);
    const size_t b = elem_bytes(type);
    const Span x(X, n, f_in, ldx, b), w(W, f_in, f_out, ldw, b), y(Y, n, f_out, ldy, b), z(Z, n, f_out, ldz, b), r(R, n, f_out, ldr, b);
    const Span v(bias, 1, f_out, f_out, 4);
    if (y.meets(x) || y.meets(w) || z.meets(x) || z.meets(w) || z.meets(y) || z.meets(r) || y.meets(v) || z.meets(v) || (y.meets(r) && !y.is(r)))
        return fail(GCN_ERR_BADARG, "%s: an output overlaps an input or another output", who);
    TileArgs a;
    a.A = X; a.lda = ldx; a.B = W; a.ldb = ldw; a.M = n; a.N = f_out; a.K = f_in;
    a.bias = bias; a.act = act; a.R = R; a.ldr = ldr; a.rho = rho; a.Z = Z; a.ldz = ldz; a.Y = Y; a.ldy = ldy;
    return by_type(type, [&](auto t) { return linear_forward_of<decltype(t)>(a, (hipStream_t)stream); });
}

extern "C" int gcn_linear_backward(int64_t n, int32_t f_in, int32_t f_out, int type, const void* X, int64_t ldx, const void* W,
                                   int64_t ldw, const void* Z, int64_t ldz, const void* dY, int64_t lddy, int act, float rho, void* dZ,
                                   int64_t lddz, void* dX, int64_t lddx, void* dW, int64_t lddw, float* dbias, void* dR, int64_t lddr,
                                   void* stream) {
    static const char* const who = "gcn_linear_backward";
    const hipStream_t s = (hipStream_t)stream;
    if (!dY || (dW && !X) || (dX && !W)) return fail(GCN_ERR_BADARG, "%s: NULL argument", who);
    if (!known_type(type)) return fail(GCN_ERR_BADARG, "%s: unknown element type %d", who, type);
    if (!known_act(act)) return fail(GCN_ERR_BADARG, "%s: unknown activation %d", who, act);
    const bool curved = act != GCN_ACT_NONE, products = dX || dW;
    if (curved && (products || dbias || dZ) && !Z) return fail(GCN_ERR_BADARG, "%s: the activation's derivative needs Z", who);
    if (curved && products && !dZ) return fail(GCN_ERR_BADARG, "%s: the products need dZ as workspace", who);
    if (n <= 0 || f_in <= 0 || f_out <= 0) return fail(GCN_ERR_BADARG, "%s: sizes must be positive", who);
    if (f_in > LINEAR_WIDEST || f_out > LINEAR_WIDEST) return fail(GCN_ERR_RANGE, "%s: widths go up to 2^27", who);
    if (lddy < f_out || (X && ldx < f_in) || (W && ldw < f_out) || (Z && ldz < f_out) || (dZ && lddz < f_out) || (dX && lddx < f_in) ||
        (dW && lddw < f_out) || (dR && lddr < f_out))
        return fail(GCN_ERR_BADARG, "%s: leading dimension below the width", who);
    const size_t b = elem_bytes(type);
    if (!curved) dZ = nullptr;
    const Span in[] = {Span(X, n, f_in, ldx, b), Span(W, f_in, f_out, ldw, b), Span(curved ? Z : nullptr, n, f_out, ldz, b), Span(dY, n, f_out, lddy, b)};
    const Span out[] = {Span(dZ, n, f_out, lddz, b), Span(dR, n, f_out, lddr, b), Span(dX, n, f_in, lddx, b), Span(dW, f_in, f_out, lddw, b), Span(dbias, 1, f_out, f_out, 4)};
    bool bad = false;
    for (int o = 0; o < 5; ++o) {
        for (int i = 0; i < 4; ++i) {
            // an element of dZ may take the place of the one of Z or dY that it is made of, one of dR that of dY
            const bool may = (o == 0 && (i == 2 || i == 3)) || (o == 1 && i == 3 && (curved || !products));
            const bool same = may && out[o].is(in[i]);
            bad |= out[o].meets(in[i]) && !same;
        }
        for (int i = 0; i < o; ++i) bad |= out[o].meets(out[i]);
    }
    if (bad) return fail(GCN_ERR_BADARG, "%s: an output overlaps an input or another output", who);
    return by_type(type, [&](auto t) -> int {
        using T = decltype(t);
        if (dbias || dR || dZ)
            GCN_TRY(slope_launch<T>(n, f_out, Z, ldz, dY, lddy, dbias || dZ ? act : GCN_ACT_NONE, rho, dZ, lddz, dR, lddr, dbias, s));
        const void* const G = curved ? dZ : dY;
        const int64_t ldg = curved ? lddz : lddy;
        TileArgs a;
        if (dX) {
            a.A = G; a.lda = ldg; a.B = W; a.ldb = ldw; a.M = n; a.N = f_in; a.K = f_out; a.Y = dX; a.ldy = lddx;
            GCN_TRY(linear_dx_of<T>(a, s));
        }
        if (dW) {
            a.A = X; a.lda = ldx; a.B = G; a.ldb = ldg; a.M = f_in; a.N = f_out; a.K = n; a.Y = dW; a.ldy = lddw;
            GCN_TRY(linear_dw_of<T>(a, s));
        }
        return GCN_OK;
    });
}
