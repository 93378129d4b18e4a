// The norms around a block, with the block's gate and its residual scale, in one pass over a row:
//   V = N_post(U),  X' = X + scale * sigmoid(A) * V,  H = N_pre(X')
// where N(x) = w (x - mean) rstd + b, mean = 0 for the root-mean-square norm, rstd = 1 / sqrt(mean((x - mean)^2) + eps); and its gradients.
#include <initializer_list>
#include <type_traits>

#include "launch_rules.h"
#include "rows.h"
#include "sum_parts.h"

namespace gcn {

struct NormArgs {
    int64_t n = 0;
    int32_t f = 0;
    int layer = 0;                 // subtract the mean
    float eps = 0;
    int gate = 0;                  // columns of A: 0, 1 or f
    int64_t ldx = 0, ldu = 0, lda = 0, ldxo = 0, ldh = 0;
    const void *X = nullptr, *U = nullptr, *A = nullptr;
    const float *scale = nullptr, *w_post = nullptr, *b_post = nullptr, *w_pre = nullptr, *b_pre = nullptr;
    void *Xout = nullptr, *H = nullptr;
    float* stats = nullptr;        // n x 4: mean and rstd of U, mean and rstd of X'
    // backward
    int64_t lddxo = 0, lddh = 0, lddx = 0, lddu = 0, ldda = 0;
    const void *dXout = nullptr, *dH = nullptr;
    void *dX = nullptr, *dU = nullptr, *dA = nullptr;
    struct RowSums* rows = nullptr;    // rows longer than the registers hold, or shorter than a lane's elements
    float* part = nullptr;         // partial sums: of each workgroup (or share of the rows) `sums` vectors of f
    int sums = 0;
    int at[4] = {-1, -1, -1, -1};  // which of them are sum dX' a u^, sum dX' a, sum dH x^, sum dH
};

// L lanes (a power of two, up to 1024) hold a row, E neighbouring elements each; a workgroup has as many rows at a time as make 512 threads.  All of them
// go through the same number of steps, with zeros for a row that is not there.  A lane keeps its columns for all its rows, and what the vectors
// hold for them; columns behind the row's end have zeros there, which keeps what is computed for them out of every sum.
template <typename T, int L, int E>
struct NormRows {
    static constexpr int THREADS = L > 512 ? L : 512, ROWS = THREADS / L;
    __device__ static int column() { return (int)(threadIdx.x % L) * E; }
    __device__ static int row() { return (int)(threadIdx.x / L); }
};
__device__ __forceinline__ f4u zero4() { return f4u{0.f, 0.f, 0.f, 0.f}; }

// LAYER: with what a layer norm has beside the root-mean-square norm, the mean (where g.layer asks for it) and the biases.
// The next rows are on their way while these are worked on: one pass over the matrices, every statistic from the registers (the variance about the mean that is known by
// then).  Bound by memory: 232965 x 128 in fp32 118 us (5.1 TB/s), 16384 x 4096 in bf16 142 us (4.7 TB/s).
template <typename T, int L, int E, bool LAYER>
__global__ __launch_bounds__((NormRows<T, L, E>::THREADS), 4) void k_block_norm(NormArgs g) {
    using R = NormRows<T, L, E>;
    __shared__ float meet[2][16][4];
    int turn = 0;
    const int c = R::column(), count = g.f - c < 0 ? 0 : (g.f - c > E ? E : g.f - c);
    const float inv_f = 1.f / (float)g.f;
    const bool ragged = g.f != L * E;                            // lanes whose elements a row's end cuts
    const int by = settle_by<E>(c, g.f);
    auto floats = [&](Words<T, E> x, float(&v)[E]) { floats_of<E, T>(ragged ? settle<E, T>(x, by) : __builtin_bit_cast(Elems<T, E>, x), v); };
    struct Raw {
        Words<T, E> x, u, a;
        float gate;
    };
    auto load = [&](int64_t i) {
        Raw r = {};
        if (i >= g.n) return r;
        r.x = load_near<E>((const T*)g.X + i * g.ldx, c, g.f);
        if (g.U) r.u = load_near<E>((const T*)g.U + i * g.ldu, c, g.f);
        if (g.gate > 1) r.a = load_near<E>((const T*)g.A + i * g.lda, c, g.f);
        if (g.gate == 1) r.gate = (float)((const T*)g.A)[i * g.lda];
        return r;
    };
    const int64_t step = (int64_t)gridDim.x * R::ROWS;
    int64_t base = (int64_t)blockIdx.x * R::ROWS;
    Raw now = load(base + R::row());
    float sw[E], sb[E], w_pre[E], b_pre[E];                      // scale w_post, scale b_post
    load_floats<E>(g.scale, c, count, 1.f, sw);
    if (LAYER) load_floats<E>(g.b_post, c, count, 0.f, sb);
    {
        float w[E];
        load_floats<E>(g.w_post, c, count, 1.f, w);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (LAYER) sb[e] *= sw[e];
            sw[e] *= w[e];
        }
    }
    load_floats<E>(g.w_pre, c, count, 1.f, w_pre);
    if (LAYER) load_floats<E>(g.b_pre, c, count, 0.f, b_pre);
    // mean and deviation of the row's x
    auto statistics = [&](const float(&x)[E], float& mean, float& rstd) {
        float s[1] = {0.f};
        if (LAYER && g.layer) {
#pragma unroll
            for (int e = 0; e < E; ++e) s[0] += e < count ? x[e] : 0.f;
            join_lanes<L>(s, meet, turn);
            mean = s[0] * inv_f;
        }
        s[0] = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = e < count ? x[e] - mean : 0.f;
            s[0] = fmaf(d, d, s[0]);
        }
        join_lanes<L>(s, meet, turn);
        rstd = 1.f / sqrtf(fmaf(s[0], inv_f, g.eps));
    };
    for (; base < g.n; base += step) {
        const int64_t i = base + R::row();
        const Raw next = load(i + step);
        float x[E];
        floats(now.x, x);
        f4u st = zero4();
        if (g.U) {
            float u[E], a[E];
            floats(now.u, u);
            if (g.w_post) {
                statistics(u, st.x, st.y);
#pragma unroll
                for (int e = 0; e < E; ++e) u[e] = (u[e] - st.x) * st.y;
            }
            if (g.gate > 1) floats(now.a, a);
            const float row_gate = g.gate == 1 ? sigmoid<T>(now.gate) : 1.f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float gate = g.gate > 1 ? sigmoid<T>(a[e]) : row_gate;
                x[e] = fmaf(gate, LAYER ? fmaf(u[e], sw[e], sb[e]) : u[e] * sw[e], x[e]);
            }
            if (g.Xout && i < g.n) store_elems<E>((T*)g.Xout + i * g.ldxo + c, x, count);
        }
        if (g.H) {
            statistics(x, st.z, st.w);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = LAYER ? fmaf((x[e] - st.z) * st.w, w_pre[e], b_pre[e]) : x[e] * st.w * w_pre[e];
            if (i < g.n) store_elems<E>((T*)g.H + i * g.ldh + c, x, count);
        }
        if (g.stats && c == 0 && i < g.n) *reinterpret_cast<f4u*>(g.stats + 4 * i) = st;
        now = next;
    }
}

// With g = dH w_pre and x^ = (X' - mean) rstd:  dX = dX' + rstd (g - x^ mean(g x^) - mean(g)), the last for the layer norm; with u^ likewise, d = dX sigmoid(A) and
// e = d scale w_post:  dA = d scale (w_post u^ + b_post) (1 - sigmoid(A)),  dU = rstd_u (e - u^ mean(e u^) - mean(e)): two joins of the row's lanes.  The vectors' gradients are
// products of the vectors with four sums over the rows (see NormVectors), which are kept per column in registers and leave once per workgroup.
// Bound by memory: 16384 x 4096 in bf16 223 us (4.8 TB/s), in fp32 399 us (5.4 TB/s).  Four elements per lane in 128 registers (eight of 16
// bits spill: 410 us), but eight for rows longer than a workgroup holds otherwise (in fp32 with a mean three registers are spilled); these start the next row after this one where both do not fit
// (AHEAD; 8192 x 8192 in fp32 422 us against 623, layer norm 431 against 888, in bf16 246 against 466; without a mean in 16 bits both fit: 215 us against 230).
template <typename T, int L, int E, bool LAYER>
__global__ __launch_bounds__((NormRows<T, L, E>::THREADS), 4) void k_block_norm_back(NormArgs g) {
    using R = NormRows<T, L, E>;
    constexpr int SUMS = LAYER ? 4 : 2;
    constexpr bool AHEAD = E < 8 || (sizeof(T) == 2 && !LAYER);
    __shared__ float meet[2][16][4];
    int turn = 0;
    const int c = R::column(), count = g.f - c < 0 ? 0 : (g.f - c > E ? E : g.f - c);
    const float inv_f = 1.f / (float)g.f;
    const bool ragged = g.f != L * E;                            // lanes whose elements a row's end cuts
    const int by = settle_by<E>(c, g.f);
    auto floats = [&](Words<T, E> x, float(&v)[E]) { floats_of<E, T>(ragged ? settle<E, T>(x, by) : __builtin_bit_cast(Elems<T, E>, x), v); };
    struct Raw {
        Words<T, E> dxo, xo, dh, u, a;
        float gate;
        f4u st;
    };
    auto load = [&](int64_t i) {
        Raw r = {};
        if (i >= g.n) return r;
        r.st = *reinterpret_cast<const f4u*>(g.stats + 4 * i);
        if (g.dXout) r.dxo = load_near<E>((const T*)g.dXout + i * g.lddxo, c, g.f);
        if (g.dH) {
            r.xo = load_near<E>((const T*)g.Xout + i * g.ldxo, c, g.f);
            r.dh = load_near<E>((const T*)g.dH + i * g.lddh, c, g.f);
        }
        if (g.U) r.u = load_near<E>((const T*)g.U + i * g.ldu, c, g.f);
        if (g.gate > 1) r.a = load_near<E>((const T*)g.A + i * g.lda, c, g.f);
        if (g.gate == 1) r.gate = (float)((const T*)g.A)[i * g.lda];
        return r;
    };
    const int64_t step = (int64_t)gridDim.x * R::ROWS;
    int64_t base = (int64_t)blockIdx.x * R::ROWS;
    Raw now = load(base + R::row());
    float sw[E], sb[E], w_pre[E], sum[SUMS][E] = {};
    load_floats<E>(g.scale, c, count, 1.f, sw);
    if (LAYER) load_floats<E>(g.b_post, c, count, 0.f, sb);
    {
        float w[E];
        load_floats<E>(g.w_post, c, count, 1.f, w);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (LAYER) sb[e] *= sw[e];
            sw[e] = e < count ? sw[e] * w[e] : 0.f;
        }
    }
    load_floats<E>(g.w_pre, c, count, 0.f, w_pre);
    for (; base < g.n; base += step) {
        const int64_t i = base + R::row();
        Raw next;
        if (AHEAD) next = load(i + step);
        const bool there = i < g.n;
        float dx[E];
        floats(now.dxo, dx);
        if (g.dH) {
            float xh[E], gw[E], s[2] = {0.f, 0.f};
            floats(now.xo, xh);
            floats(now.dh, gw);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                xh[e] = (xh[e] - now.st.z) * now.st.w;
                sum[1][e] = fmaf(gw[e], xh[e], sum[1][e]);
                if (LAYER) sum[3][e] += gw[e];
                gw[e] *= w_pre[e];
                s[0] = fmaf(gw[e], xh[e], s[0]);
                s[1] += gw[e];
            }
            join_lanes<L>(s, meet, turn);
            const float along = s[0] * inv_f, mean = LAYER && g.layer ? s[1] * inv_f : 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) dx[e] = fmaf(now.st.w, gw[e] - fmaf(xh[e], along, mean), dx[e]);
        }
        if (g.dX && there) store_elems<E>((T*)g.dX + i * g.lddx + c, dx, count);
        if (g.U) {
            const float row_gate = g.gate == 1 ? sigmoid<T>(now.gate) : 1.f;
            const float mean_u = g.w_post ? now.st.x : 0.f, rstd_u = g.w_post ? now.st.y : 1.f;
            float u[E], a[E], s[3] = {0.f, 0.f, 0.f};
            floats(now.u, u);
            if (g.gate > 1) floats(now.a, a);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                u[e] = (u[e] - mean_u) * rstd_u;
                const float gate = g.gate > 1 ? sigmoid<T>(a[e]) : row_gate;
                const float d = dx[e] * gate;
                sum[0][e] = fmaf(d, u[e], sum[0][e]);
                if (LAYER) sum[2][e] += d;
                a[e] = d * (LAYER ? fmaf(u[e], sw[e], sb[e]) : u[e] * sw[e]) * (1.f - gate);
                s[2] += e < count ? a[e] : 0.f;
                dx[e] = d * sw[e];
                s[0] = fmaf(dx[e], u[e], s[0]);
                s[1] += dx[e];
            }
            if (g.dA && g.gate > 1 && there) store_elems<E>((T*)g.dA + i * g.ldda + c, a, count);
            if (g.w_post || g.gate == 1) join_lanes<L>(s, meet, turn);
            if (g.dA && g.gate == 1 && c == 0 && there) ((T*)g.dA)[i * g.ldda] = (T)s[2];
            if (g.w_post) {
                const float along = s[0] * inv_f, mean = LAYER && g.layer ? s[1] * inv_f : 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) dx[e] = rstd_u * (dx[e] - fmaf(u[e], along, mean));
            }
            if (g.dU && there) store_elems<E>((T*)g.dU + i * g.lddu + c, dx, count);
        }
        if (AHEAD) now = next;
        else now = load(i + step);
    }
    if (!g.part) return;
    // the rows of the workgroup in order, one of the sums at a time
    __shared__ float add[R::ROWS > 1 ? R::THREADS * E : 1];
    constexpr int AT[4] = {0, 2, 1, 3};                          // sum[] of NormArgs::at[]
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (AT[k] >= SUMS || g.at[k] < 0) continue;
        float(&mine)[E] = sum[AT[k] < SUMS ? AT[k] : 0];
        if constexpr (R::ROWS > 1) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e) add[threadIdx.x * E + e] = mine[e];
            __syncthreads();
            if (threadIdx.x < L)
#pragma nounroll
                for (int r = 1; r < R::ROWS; ++r)
#pragma unroll
                    for (int e = 0; e < E; ++e) mine[e] += add[(r * L + threadIdx.x) * E + e];
        }
        float* const out = g.part + ((int64_t)blockIdx.x * g.sums + g.at[k]) * g.f;
        if (threadIdx.x < L)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e < count) out[c + e] = mine[e];
    }
}

// Rows longer than the registers hold, and rows shorter than a lane's elements: a workgroup reads its row again for every sum, from the caches.
// 4096 x 16384 in bf16 263 us (2.6 TB/s of one reading and writing), in fp32 382 us (3.5 TB/s).
template <typename T>
__global__ __launch_bounds__(1024) void k_block_norm_long(NormArgs g) {
    constexpr int E = Elem<T>::E, STEP = 1024 * E;
    __shared__ float meet[2][16][4];
    int turn = 0;
    const float inv_f = 1.f / (float)g.f;
    for (int64_t i = blockIdx.x; i < g.n; i += gridDim.x) {
        const T* const X = (const T*)g.X + i * g.ldx;
        const T* const U = g.U ? (const T*)g.U + i * g.ldu : nullptr;
        const float row_gate = g.gate == 1 ? sigmoid<T>((float)((const T*)g.A)[i * g.lda]) : 1.f;
        float umean = 0.f, urstd = 0.f, xmean = 0.f, xrstd = 0.f;
        // each(value, column, elements there) for the thread's columns of U, then of X'
        auto each_u = [&](auto f) {
            for (int64_t c = (int64_t)threadIdx.x * E; c < g.f; c += STEP) {
                const int count = g.f - c < E ? (int)(g.f - c) : E;
                float u[E];
                to_floats<T>(load_vec_part(U + c, count), u);
                f(u, c, count);
            }
        };
        auto each_x = [&](auto f) {
            for (int64_t c = (int64_t)threadIdx.x * E; c < g.f; c += STEP) {
                const int count = g.f - c < E ? (int)(g.f - c) : E;
                float x[E];
                to_floats<T>(load_vec_part(X + c, count), x);
                if (U) {
                    float u[E], w[E], b[E], sc[E], a[E];
                    to_floats<T>(load_vec_part(U + c, count), u);
                    load_floats<E>(g.scale, c, count, 1.f, sc);
                    load_floats<E>(g.w_post, c, count, 1.f, w);
                    load_floats<E>(g.b_post, c, count, 0.f, b);
                    if (g.gate > 1) to_floats<T>(load_vec_part((const T*)g.A + i * g.lda + c, count), a);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float v = g.w_post ? fmaf((u[e] - umean) * urstd, w[e], b[e]) : u[e];
                        x[e] = fmaf(sc[e] * (g.gate > 1 ? sigmoid<T>(a[e]) : row_gate), v, x[e]);
                    }
                }
                f(x, c, count);
            }
        };
        auto statistics = [&](auto each, float& mean, float& rstd) {
            float s[1] = {0.f};
            if (g.layer) {
                each([&](float(&v)[E], int64_t, int count) {
#pragma unroll
                    for (int e = 0; e < E; ++e) s[0] += e < count ? v[e] : 0.f;
                });
                join_lanes<1024>(s, meet, turn);
                mean = s[0] * inv_f;
            }
            s[0] = 0.f;
            each([&](float(&v)[E], int64_t, int count) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float d = e < count ? v[e] - mean : 0.f;
                    s[0] = fmaf(d, d, s[0]);
                }
            });
            join_lanes<1024>(s, meet, turn);
            rstd = 1.f / sqrtf(fmaf(s[0], inv_f, g.eps));
        };
        if (U && g.w_post) statistics(each_u, umean, urstd);
        if (g.H) statistics(each_x, xmean, xrstd);
        each_x([&](float(&x)[E], int64_t c, int count) {          // what is written may take the place of what is read here
            if (U && g.Xout) store_vec_part((T*)g.Xout + i * g.ldxo + c, from_floats<T>(x), count);
            if (!g.H) return;
            float w[E], b[E];
            load_floats<E>(g.w_pre, c, count, 1.f, w);
            load_floats<E>(g.b_pre, c, count, 0.f, b);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = fmaf((x[e] - xmean) * xrstd, w[e], b[e]);
            store_vec_part((T*)g.H + i * g.ldh + c, from_floats<T>(x), count);
        });
        if (g.stats && threadIdx.x == 0) *reinterpret_cast<f4u*>(g.stats + 4 * i) = f4u{umean, urstd, xmean, xrstd};
    }
}

// Their gradients: what a row's elements have to know of the whole row is found by a workgroup, which then has the rest of the row too where no vector's gradient is
// wanted.  With these the rest is a launch of its own, in strips of columns, where a thread keeps its columns' sums over the rows in registers: a workgroup's sums over
// whole rows would be as long as the rows (four of 2^24 columns from 256 workgroups 64 GB), and in memory.  Three readings of the operands either way,
// the last one from the caches only in the one launch: 4096 x 16384 in bf16 382 us without the vectors (564 in two launches), 617 with them (a copy of as
// many bytes takes 224).
struct RowSums {
    float along, mean;             // of g x^ and g over the row: mean(g x^), and mean(g) for the layer norm
    float along_u, mean_u;         // likewise of e u^ and e
    float gate, dgate;             // with one gate per row: sigmoid(A), and dA
};
// dX of E elements from column c of row i on, with x^ and dH, zeros behind the row's end
template <typename T, int E>
__device__ __forceinline__ void long_stream_side(const NormArgs& g, int64_t i, int64_t c, int count, const f4u& st, const float (&w_pre)[E], float along, float mean,
                                                 float (&dx)[E], float (&xh)[E], float (&dh)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) dx[e] = xh[e] = dh[e] = 0.f;
    if (g.dXout) to_floats<T>(load_vec_part((const T*)g.dXout + i * g.lddxo + c, count), dx);
    if (!g.dH) return;
    to_floats<T>(load_vec_part((const T*)g.Xout + i * g.ldxo + c, count), xh);
    to_floats<T>(load_vec_part((const T*)g.dH + i * g.lddh + c, count), dh);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        xh[e] = e < count ? (xh[e] - st.z) * st.w : 0.f;
        dx[e] = fmaf(st.w, dh[e] * w_pre[e] - fmaf(xh[e], along, mean), dx[e]);
    }
}
// The block's side from it: u^, d = dX sigmoid(A), dA, and e = d scale w_post
template <typename T, int E>
__device__ __forceinline__ void long_block_side(const NormArgs& g, int64_t i, int64_t c, int count, const f4u& st, float row_gate, const float (&scale)[E],
                                                const float (&w_post)[E], const float (&b_post)[E], const float (&dx)[E], float (&uh)[E], float (&d)[E],
                                                float (&da)[E], float (&de)[E]) {
    float a[E];
    to_floats<T>(load_vec_part((const T*)g.U + i * g.ldu + c, count), uh);
    if (g.gate > 1) to_floats<T>(load_vec_part((const T*)g.A + i * g.lda + c, count), a);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (g.w_post) uh[e] = e < count ? (uh[e] - st.x) * st.y : 0.f;
        const float gate = g.gate > 1 ? sigmoid<T>(a[e]) : row_gate;
        d[e] = e < count ? dx[e] * gate : 0.f;
        da[e] = d[e] * scale[e] * fmaf(uh[e], w_post[e], b_post[e]) * (1.f - gate);
        de[e] = d[e] * scale[e] * w_post[e];
    }
}
// The gradients of E elements of the matrices.  What is written may take the place of what has been read; dA of one gate per row, of a row of one element, too.
template <typename T, int E>
__device__ __forceinline__ void long_matrices(const NormArgs& g, int64_t i, int64_t c, int count, const f4u& st, const RowSums& r, const float (&dx)[E],
                                              const float (&uh)[E], const float (&da)[E], float (&de)[E]) {
    if (g.dX) store_vec_part((T*)g.dX + i * g.lddx + c, from_floats<T>(dx), count);
    if (!g.U) return;
    if (g.dA && g.gate > 1) store_vec_part((T*)g.dA + i * g.ldda + c, from_floats<T>(da), count);
    if (g.dA && g.gate == 1 && c == 0) ((T*)g.dA)[i * g.ldda] = (T)r.dgate;
    if (!g.dU) return;
    if (g.w_post)
#pragma unroll
        for (int e = 0; e < E; ++e) de[e] = st.y * (de[e] - fmaf(uh[e], r.along_u, r.mean_u));
    store_vec_part((T*)g.dU + i * g.lddu + c, from_floats<T>(de), count);
}
template <int E>
__device__ __forceinline__ void long_vectors(const NormArgs& g, int64_t c, int count, float (&scale)[E], float (&w_post)[E], float (&b_post)[E]) {
    load_floats<E>(g.scale, c, count, 1.f, scale);
    load_floats<E>(g.w_post, c, count, 1.f, w_post);
    load_floats<E>(g.b_post, c, count, 0.f, b_post);
}

template <typename T>
__global__ __launch_bounds__(1024) void k_block_norm_back_rows(NormArgs g) {
    constexpr int E = Elem<T>::E, STEP = 1024 * E;
    __shared__ float meet[2][16][4];
    int turn = 0;
    const float inv_f = 1.f / (float)g.f;
    for (int64_t i = blockIdx.x; i < g.n; i += gridDim.x) {
        const f4u st = *reinterpret_cast<const f4u*>(g.stats + 4 * i);
        RowSums r = {0.f, 0.f, 0.f, 0.f, 1.f, 0.f};
        if (g.gate == 1) r.gate = sigmoid<T>((float)((const T*)g.A)[i * g.lda]);
        if (g.dH) {
            float s[2] = {0.f, 0.f};
            for (int64_t c = (int64_t)threadIdx.x * E; c < g.f; c += STEP) {
                const int count = g.f - c < E ? (int)(g.f - c) : E;
                float dx[E], xh[E], dh[E], w_pre[E];
                load_floats<E>(g.w_pre, c, count, 1.f, w_pre);
                long_stream_side<T, E>(g, i, c, count, st, w_pre, 0.f, 0.f, dx, xh, dh);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    s[0] = fmaf(dh[e] * w_pre[e], xh[e], s[0]);
                    s[1] += dh[e] * w_pre[e];
                }
            }
            join_lanes<1024>(s, meet, turn);
            r.along = s[0] * inv_f;
            r.mean = g.layer ? s[1] * inv_f : 0.f;
        }
        if (g.U && (g.w_post || g.gate == 1)) {
            float s[3] = {0.f, 0.f, 0.f};
            for (int64_t c = (int64_t)threadIdx.x * E; c < g.f; c += STEP) {
                const int count = g.f - c < E ? (int)(g.f - c) : E;
                float dx[E], xh[E], dh[E], w_pre[E], scale[E], w_post[E], b_post[E], uh[E], d[E], da[E], de[E];
                load_floats<E>(g.w_pre, c, count, 1.f, w_pre);
                long_vectors<E>(g, c, count, scale, w_post, b_post);
                long_stream_side<T, E>(g, i, c, count, st, w_pre, r.along, r.mean, dx, xh, dh);
                long_block_side<T, E>(g, i, c, count, st, r.gate, scale, w_post, b_post, dx, uh, d, da, de);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    s[0] = fmaf(de[e], uh[e], s[0]);
                    s[1] += de[e];
                    s[2] += da[e];
                }
            }
            join_lanes<1024>(s, meet, turn);
            r.along_u = s[0] * inv_f;
            r.mean_u = g.layer ? s[1] * inv_f : 0.f;
            r.dgate = s[2];
        }
        if (g.rows) {
            if (threadIdx.x == 0) g.rows[i] = r;
            continue;
        }
        for (int64_t c = (int64_t)threadIdx.x * E; c < g.f; c += STEP) {
            const int count = g.f - c < E ? (int)(g.f - c) : E;
            float dx[E], xh[E], dh[E], w_pre[E], scale[E], w_post[E], b_post[E], uh[E], d[E], da[E], de[E];
            load_floats<E>(g.w_pre, c, count, 1.f, w_pre);
            long_stream_side<T, E>(g, i, c, count, st, w_pre, r.along, r.mean, dx, xh, dh);
            if (g.U) {
                long_vectors<E>(g, c, count, scale, w_post, b_post);
                long_block_side<T, E>(g, i, c, count, st, r.gate, scale, w_post, b_post, dx, uh, d, da, de);
            }
            long_matrices<T, E>(g, i, c, count, st, r, dx, uh, da, de);
        }
    }
}

// 64 lanes of E columns by four rows at a time; a share of the rows, whose sums are the four row sets' in order.  What is written may take the place of what is read here.
template <typename T>
__global__ __launch_bounds__(256) void k_block_norm_back_columns(NormArgs g, int64_t rows_per_block) {
    constexpr int E = Elem<T>::E, SETS = 4;
    __shared__ float add[SETS][64][E + 1];
    const int lane = threadIdx.x & 63, set = threadIdx.x >> 6;
    const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * E;
    const int64_t rb = (int64_t)blockIdx.y * rows_per_block, re = rb + rows_per_block < g.n ? rb + rows_per_block : g.n;
    const int count = c >= g.f ? 0 : g.f - c < E ? (int)(g.f - c) : E;
    float sum[4][E] = {};
    if (count > 0) {
        float w_pre[E], scale[E], w_post[E], b_post[E];
        load_floats<E>(g.w_pre, c, count, 1.f, w_pre);
        long_vectors<E>(g, c, count, scale, w_post, b_post);
        for (int64_t i = rb + set; i < re; i += SETS) {
            const f4u st = *reinterpret_cast<const f4u*>(g.stats + 4 * i);
            RowSums r = {0.f, 0.f, 0.f, 0.f, 1.f, 0.f};
            if (g.rows) r = g.rows[i];
            float dx[E], xh[E], dh[E], uh[E], d[E], da[E], de[E];
            long_stream_side<T, E>(g, i, c, count, st, w_pre, r.along, r.mean, dx, xh, dh);
            if (g.U) long_block_side<T, E>(g, i, c, count, st, r.gate, scale, w_post, b_post, dx, uh, d, da, de);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                sum[2][e] = fmaf(dh[e], xh[e], sum[2][e]);
                sum[3][e] += dh[e];
                if (!g.U) continue;
                sum[0][e] = fmaf(d[e], uh[e], sum[0][e]);
                sum[1][e] += d[e];
            }
            long_matrices<T, E>(g, i, c, count, st, r, dx, uh, da, de);
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (g.at[k] < 0) continue;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e) add[set][lane][e] = sum[k][e];
        __syncthreads();
        if (set) continue;
        float* const out = g.part + ((int64_t)blockIdx.y * g.sums + g.at[k]) * g.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            float s = add[0][lane][e];
            for (int w = 1; w < SETS; ++w) s += add[w][lane][e];
            if (e < count) out[c + e] = s;
        }
    }
}

// The sums of the workgroups, added in order, and the vectors' gradients from them:
//   dscale = w_post S0 + b_post S1, dw_post = scale S0, db_post = scale S1, dw_pre = S2, db_pre = S3
struct NormVectors {
    const float *scale, *w_post, *b_post;
    float *dscale, *dw_post, *db_post, *dw_pre, *db_pre;
};
// Sixteen columns by 64 shares of the workgroups, the shares in order.  (A second dimension of workgroups for more columns than one has threads for: a loop over the
// columns took 1 us longer.)
__global__ __launch_bounds__(1024) void k_block_norm_vectors(NormArgs g, int blocks, NormVectors v) {
    __shared__ float shares[4][64][17];
    const int col = threadIdx.x & 15, share = threadIdx.x >> 4;
    const int64_t c = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 16 + col;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (g.at[k] >= 0) shares[k][share][col] = c < g.f ? strided_sum(g.part + (int64_t)g.at[k] * g.f + c, (int64_t)g.sums * g.f, share, 64, blocks) : 0.f;
    __syncthreads();
    // (sum, column) of a thread; the others are done
    __shared__ float total[4][16];
    if (threadIdx.x < 64) {
        float s = 0.f;
        if (g.at[share] >= 0)
            for (int w = 0; w < 64; ++w) s += shares[share][w][col];
        total[share][col] = s;
    }
    __syncthreads();
    if (threadIdx.x >= 16 || c >= g.f) return;
    const float s0 = total[0][col], s1 = total[1][col], sc = v.scale ? v.scale[c] : 1.f;
    if (v.dscale) v.dscale[c] = v.w_post ? fmaf(v.w_post[c], s0, v.b_post ? v.b_post[c] * s1 : 0.f) : s0;
    if (v.dw_post) v.dw_post[c] = sc * s0;
    if (v.db_post) v.db_post[c] = sc * s1;
    if (v.dw_pre) v.dw_pre[c] = total[2][col];
    if (v.db_pre) v.db_pre[c] = total[3][col];
}

// The fewest lanes that hold a row with E elements each, a workgroup's 1024 with twice as many for longer rows; call(lanes, elements), or call(0, 0) for rows longer than
// that or shorter than E.
template <int E, typename F>
static int by_row(int32_t f, const F& call) {
    const int64_t pieces = f < E ? INT64_MAX : (f + E - 1) / E;
#define GCN_LANES(L) if (pieces <= (int64_t)(L)) return call(std::integral_constant<int, L>(), std::integral_constant<int, E>())
    GCN_LANES(4); GCN_LANES(8); GCN_LANES(16); GCN_LANES(32); GCN_LANES(64); GCN_LANES(128); GCN_LANES(256); GCN_LANES(512); GCN_LANES(1024);
#undef GCN_LANES
    if constexpr (E < 8)
        if (f >= 8 && f <= 8192) return call(std::integral_constant<int, 1024>(), std::integral_constant<int, 8>());
    return call(std::integral_constant<int, 0>(), std::integral_constant<int, 0>());
}

template <typename T>
static int norm_forward(const NormArgs& g, hipStream_t s) {
    return by_row<Elem<T>::E>(g.f, [&](auto l, auto elements) -> int {
        constexpr int L = decltype(l)::value, E = decltype(elements)::value;
        const int64_t cus = device_info().cus;
        if constexpr (L == 0) {
            hipLaunchKernelGGL((k_block_norm_long<T>), dim3((unsigned)(g.n < 16 * cus ? g.n : 16 * cus)), dim3(1024), 0, s, g);
        } else {
            using R = NormRows<T, L, E>;
            const int64_t groups = (g.n + R::ROWS - 1) / R::ROWS, most = cus * (2048 / R::THREADS);
            const dim3 grid((unsigned)(groups < most ? groups : most));
            // (LAYER: a mean or biases; the norm without either has a kernel of its own)
            if (g.layer || g.b_post || g.b_pre) hipLaunchKernelGGL((k_block_norm<T, L, E, true>), grid, dim3(R::THREADS), 0, s, g);
            else hipLaunchKernelGGL((k_block_norm<T, L, E, false>), grid, dim3(R::THREADS), 0, s, g);
        }
        GCN_LAUNCH_CHECK();
        return GCN_OK;
    });
}

template <typename T>
static int norm_backward(NormArgs g, const NormVectors& v, hipStream_t s) {
    // (16-bit elements too by four: eight of them, with the sums, are more than a lane's 128 registers)
    return by_row<4>(g.f, [&](auto l, auto elements) -> int {
        constexpr int L = decltype(l)::value, E = decltype(elements)::value;
        const int64_t cus = device_info().cus;
        ScratchLease lease;
        int64_t blocks = 0;
        auto room = [&](size_t rows) -> int {                     // for `blocks` partial sums and, before them, what there is for each row
            void* mem = nullptr;
            const size_t bytes = rows + (size_t)blocks * g.sums * g.f * 4;      // (24 bytes for a row: the sums behind them are aligned)
            if (bytes) GCN_TRY(lease.get(&mem, bytes, s));
            if (rows) g.rows = (RowSums*)mem;
            if (g.sums) g.part = (float*)((char*)mem + rows);
            return GCN_OK;
        };
        if constexpr (L == 0) {
            const int64_t across = (g.f + 64 * Elem<T>::E - 1) / (64 * Elem<T>::E);
            const RowShares shares = row_shares(g.n, across, cus);
            blocks = shares.count;
            const bool rows = !g.sums || g.dH || g.w_post || g.gate == 1;
            GCN_TRY(room(rows && g.sums ? (size_t)g.n * sizeof(RowSums) : 0));
            if (rows) {
                hipLaunchKernelGGL((k_block_norm_back_rows<T>), dim3((unsigned)(g.n < 2 * cus ? g.n : 2 * cus)), dim3(1024), 0, s, g);
                GCN_LAUNCH_CHECK();
            }
            if (g.sums) hipLaunchKernelGGL((k_block_norm_back_columns<T>), dim3((unsigned)across, (unsigned)blocks), dim3(256), 0, s, g, shares.rows);
        } else {
            // as many workgroups as run at one time: each leaves partial sums, which are read again
            using R = NormRows<T, L, E>;
            const int64_t groups = (g.n + R::ROWS - 1) / R::ROWS, most = cus * (1024 / R::THREADS);
            blocks = groups < most ? groups : most;
            GCN_TRY(room(0));
            if (g.layer || g.b_post || v.db_post || v.db_pre) hipLaunchKernelGGL((k_block_norm_back<T, L, E, true>), dim3((unsigned)blocks), dim3(R::THREADS), 0, s, g);
            else hipLaunchKernelGGL((k_block_norm_back<T, L, E, false>), dim3((unsigned)blocks), dim3(R::THREADS), 0, s, g);
        }
        GCN_LAUNCH_CHECK();
        if (g.sums) {
            const LaunchGroups groups = norm_vector_groups(g.f);
            hipLaunchKernelGGL(k_block_norm_vectors, dim3(groups.x, groups.y), dim3(1024), 0, s, g, (int)blocks, v);
            GCN_LAUNCH_CHECK();
        }
        return GCN_OK;
    });
}

}  // namespace gcn

using namespace gcn;

// Whether outputs overlap inputs or each other otherwise than element by element: an output of the rows' size may be an input of that size
// (same address and, of several rows, leading dimension).
struct Place {
    const void* p;
    int64_t cols, ld;
};
static bool misplaced(int64_t n, int32_t f, size_t b, std::initializer_list<Place> in, std::initializer_list<Place> out,
                      std::initializer_list<const void*> vectors_in, std::initializer_list<const void*> vectors_out, const void* stats, bool stats_out) {
    auto span = [&](const Place& x) { return Span(x.p, n, x.cols, x.ld, b); };
    const Span st(stats, n, 4, 4, 4);
    for (const Place* o = out.begin(); o != out.end(); ++o) {
        for (const Place& i : in)
            if (span(*o).meets(span(i)) && !span(*o).is(span(i))) return true;
        for (const Place* q = out.begin(); q != o; ++q)
            if (span(*o).meets(span(*q))) return true;
        for (const void* v : vectors_in)
            if (span(*o).meets(Span(v, 1, f, f, 4))) return true;
        for (const void* v : vectors_out)
            if (span(*o).meets(Span(v, 1, f, f, 4))) return true;
        if (span(*o).meets(st)) return true;
    }
    for (const void* const* o = vectors_out.begin(); o != vectors_out.end(); ++o) {
        const Span v(*o, 1, f, f, 4);
        for (const Place& i : in)
            if (v.meets(span(i))) return true;
        for (const void* x : vectors_in)
            if (v.meets(Span(x, 1, f, f, 4))) return true;
        for (const void* const* q = vectors_out.begin(); q != o; ++q)
            if (v.meets(Span(*q, 1, f, f, 4))) return true;
        if (v.meets(st)) return true;
    }
    if (stats_out) {
        for (const Place& i : in)
            if (st.meets(span(i))) return true;
        for (const void* v : vectors_in)
            if (st.meets(Span(v, 1, f, f, 4))) return true;
    }
    return false;
}

static int norm_checks(const char* who, int64_t n, int32_t f, int type, int kind, int32_t gate_cols, const void* A, int64_t lda) {
    if (!known_type(type)) return fail(GCN_ERR_BADARG, "%s: unknown element type %d", who, type);
    if (kind != GCN_NORM_RMS && kind != GCN_NORM_LAYER) return fail(GCN_ERR_BADARG, "%s: unknown norm %d", who, kind);
    if (n <= 0 || f <= 0) return fail(GCN_ERR_BADARG, "%s: sizes must be positive", who);
    if (f > NORM_WIDEST) return fail(GCN_ERR_RANGE, "%s: rows go up to 2^26", who);
    if (A && gate_cols != 1 && gate_cols != f) return fail(GCN_ERR_BADARG, "%s: the gate has 1 or f columns", who);
    if (A && lda < gate_cols) return fail(GCN_ERR_BADARG, "%s: leading dimension below the width", who);
    return GCN_OK;
}

extern "C" int gcn_block_norm_forward(int64_t n, int32_t f, int type, int kind, float eps, const void* X, int64_t ldx, const void* U,
                                      int64_t ldu, const void* A, int32_t gate_cols, int64_t lda, const float* scale, const float* w_post,
                                      const float* b_post, const float* w_pre, const float* b_pre, void* Xout, int64_t ldxo, void* H,
                                      int64_t ldh, float* stats, void* stream) {
    static const char* const who = "gcn_block_norm_forward";
    GCN_TRY(norm_checks(who, n, f, type, kind, gate_cols, A, lda));
    if (!X || (!H && !(U && Xout))) return fail(GCN_ERR_BADARG, "%s: NULL argument", who);
    if (!U && (A || scale || w_post || b_post || Xout)) return fail(GCN_ERR_BADARG, "%s: a gate, a scale, a post-norm and X' need U", who);
    if (b_post && !w_post) return fail(GCN_ERR_BADARG, "%s: b_post without w_post", who);
    if ((H && !w_pre) || (!H && (w_pre || b_pre))) return fail(GCN_ERR_BADARG, "%s: H and w_pre go together", who);
    if (!(eps >= 0.f)) return fail(GCN_ERR_BADARG, "%s: eps must not be negative", who);
    if (ldx < f || (U && ldu < f) || (Xout && ldxo < f) || (H && ldh < f))
        return fail(GCN_ERR_BADARG, "%s: leading dimension below the width", who);
    if (misplaced(n, f, elem_bytes(type), {{X, f, ldx}, {U, f, ldu}, {A, gate_cols, lda}}, {{Xout, f, ldxo}, {H, f, ldh}},
                  {scale, w_post, b_post, w_pre, b_pre}, {}, stats, true))
        return fail(GCN_ERR_BADARG, "%s: an output overlaps an input or another output", who);
    NormArgs g;
    g.n = n; g.f = f; g.layer = kind == GCN_NORM_LAYER; g.eps = eps; g.gate = A ? (gate_cols == f && f > 1 ? f : 1) : 0;
    g.X = X; g.ldx = ldx; g.U = U; g.ldu = ldu; g.A = A; g.lda = lda; g.scale = scale; g.w_post = w_post; g.b_post = b_post;
    g.w_pre = w_pre; g.b_pre = b_pre; g.Xout = Xout; g.ldxo = ldxo; g.H = H; g.ldh = ldh; g.stats = stats;
    return by_type(type, [&](auto t) { return norm_forward<decltype(t)>(g, (hipStream_t)stream); });
}

extern "C" int gcn_block_norm_backward(int64_t n, int32_t f, int type, int kind, const void* U, int64_t ldu, const void* A,
                                       int32_t gate_cols, int64_t lda, const float* scale, const float* w_post, const float* b_post,
                                       const float* w_pre, const void* Xout, int64_t ldxo, const float* stats, const void* dXout,
                                       int64_t lddxo, const void* dH, int64_t lddh, void* dX, int64_t lddx, void* dU, int64_t lddu,
                                       void* dA, int64_t ldda, float* dscale, float* dw_post, float* db_post, float* dw_pre, float* db_pre,
                                       void* stream) {
    static const char* const who = "gcn_block_norm_backward";
    GCN_TRY(norm_checks(who, n, f, type, kind, gate_cols, A, lda));
    if ((!dXout && !dH) || !stats) return fail(GCN_ERR_BADARG, "%s: NULL argument", who);
    if (!U && (A || scale || w_post || b_post || dU || dA || dscale || dw_post || db_post))
        return fail(GCN_ERR_BADARG, "%s: a gate, a scale, a post-norm and their gradients need U", who);
    if (b_post && !w_post) return fail(GCN_ERR_BADARG, "%s: b_post without w_post", who);
    if (dH && (!w_pre || !Xout)) return fail(GCN_ERR_BADARG, "%s: dH needs w_pre and X'", who);
    if (!dH && (dw_pre || db_pre)) return fail(GCN_ERR_BADARG, "%s: the pre-norm's gradients need dH", who);
    if ((dA && !A) || (dw_post && !w_post) || (db_post && !w_post))
        return fail(GCN_ERR_BADARG, "%s: the gradient of an operand that is not there", who);
    if ((U && ldu < f) || (dH && (ldxo < f || lddh < f)) || (dXout && lddxo < f) || (dX && lddx < f) || (dU && lddu < f) || (dA && ldda < gate_cols))
        return fail(GCN_ERR_BADARG, "%s: leading dimension below the width", who);
    if (misplaced(n, f, elem_bytes(type), {{U, f, ldu}, {A, gate_cols, lda}, {dH ? Xout : nullptr, f, ldxo}, {dXout, f, lddxo}, {dH, f, lddh}},
                  {{dX, f, lddx}, {dU, f, lddu}, {dA, gate_cols, ldda}}, {scale, w_post, b_post, w_pre},
                  {dscale, dw_post, db_post, dw_pre, db_pre}, stats, false))
        return fail(GCN_ERR_BADARG, "%s: an output overlaps an input or another output", who);
    NormArgs g;
    g.n = n; g.f = f; g.layer = kind == GCN_NORM_LAYER; g.gate = A ? (gate_cols == f && f > 1 ? f : 1) : 0;
    g.U = U; g.ldu = ldu; g.A = A; g.lda = lda; g.scale = scale; g.w_post = w_post; g.b_post = b_post; g.w_pre = w_pre;
    g.Xout = const_cast<void*>(Xout); g.ldxo = ldxo; g.stats = const_cast<float*>(stats); g.dXout = dXout; g.lddxo = lddxo; g.dH = dH; g.lddh = lddh;
    g.dX = dX; g.lddx = lddx; g.dU = dU; g.lddu = lddu; g.dA = dA; g.ldda = ldda;
    const bool want[4] = {dscale || dw_post, (dscale && b_post) || db_post, dw_pre != nullptr, db_pre != nullptr};
    for (int k = 0; k < 4; ++k)
        if (want[k]) g.at[k] = g.sums++;
    const NormVectors v{scale, w_post, b_post, dscale, dw_post, db_post, dw_pre, db_pre};
    return by_type(type, [&](auto t) { return norm_backward<decltype(t)>(g, v, (hipStream_t)stream); });
}
