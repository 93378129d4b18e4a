// Distillation from a teacher's largest logits: with S the entries of a row's list (index >= 0, logit above -inf), p = softmax over S of t / T and
// q = softmax over all classes of z / T,
//   loss = 1/m sum over rows [ wt T^2 sum over S of p (log p - log q) - wl log softmax(z)_y ]
//   G    = 1/m [ wt T (q - p) where S is not empty, + wl (softmax(z) - onehot(y)) where y >= 0 ]
// A row of up to 16 KB is read once, held in registers in its own type, and its gradient written once: bound by memory and, where rows are short, by the instructions of a row
// (its list, two joins, the list again; vector instructions are issued in 83 % of the cycles): 232965 x 41 in fp32 35 us, x 128 55 us (4.3 TB/s).  Longer rows: 4096 x 100,000 in bf16
// 403 us, 3 x 819 MB from and to memory and caches, with vector instructions in 75 % of the cycles.  Double entries are looked for by every entry in the whole list, which long
// lists feel: 4096 rows of 100,000 with 1500 entries 2.0 ms, without a gradient 0.24.
#include <type_traits>

#include "rows.h"
#include "sum_parts.h"

namespace gcn {

struct DistillArgs {
    int64_t n = 0;
    int32_t C = 0, k = 0;
    const void* Z = nullptr;
    void* G = nullptr;
    int64_t ldz = 0, ldg = 0, ldtop = 0, ldt = 0;
    const int32_t* top = nullptr;
    const void* t = nullptr;
    const int32_t* labels = nullptr;
    float inv_T = 1, wt = 0, wl = 0;          // wt, wl: of the loss over T, which joins 1 / m: w_teacher T, w_label / T
    float gt = 0, gl = 0;                     // of the gradient: grad_scale / m times wt T and wl
    double* part = nullptr;
};

// e^((x - high) / T) by the instruction that raises 2 to a power, c = log2(e) / T: difference and product are rounded, so the result is off by 2^-23 of itself for each
// unit d of the exponent.  In a row's sum, which is 1 at least, that is at most d e^-d 2^-23 of it, less than an fp32 rounding; what is relative to itself is the gradient of a
// class far below the largest.  (With the lost bits, as exp_for has them for fp32 elements, 232965 x 41 took 34.0 us, without 31.0.)
__device__ __forceinline__ float power(float x, float high, float c) { return power_of_2((x - high) * c); }
// e^(x - high) from et = e^((x - high) / T): itself at the temperature 1, its square at 2 and that one's at 4 (POWER), else a second exponential.  Microseconds at 1, 2, 4 and, with
// a second one, 3: 4096 x 100,000 in bf16 399, 404, 422, 458 (exponentials of a quarter of the vector rate, twice for each element, beside the memory); 65536 x 1000 in bf16 70, 74, 75, 77;
// 232965 x 41 in fp32 30.2, 31.3, 31.0, 31.8.  Further whole powers would take as many products as a second exponential takes.
template <int POWER>
__device__ __forceinline__ float plain_power(float et, float x, float high) {
    if (POWER == 1) return et;
    if (POWER == 2) return et * et;
    if (POWER == 4) return (et * et) * (et * et);
    return power(x, high, LOG2E);
}

// P = 0: rows longer than the registers hold are read twice, for the sums and for the gradient; what a thread has of a row is summed as it comes, with
// its running maximum.
// Elements that are not there count as -inf, so that only loads and stores look at a row's end.
template <typename T, int L, int P, int POWER>
__global__ __launch_bounds__((Rows<T, L, P>::THREADS), P == 0 ? 8 : 4) void k_distill(DistillArgs a) {
    using R = Rows<T, L, P>;
    constexpr int E = R::E;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float meet[2][16][4];
    __shared__ double s_w[16];
    int turn = 0;
    const int li = threadIdx.x % L, entries = a.k + 1;
    // the row's list: index (-1: none), logit of the student, p; the label is its last entry, with p = 0
    int32_t* const l_at = (int32_t*)lds + (int64_t)(threadIdx.x / L) * 3 * entries;
    float* const l_z = (float*)(l_at + entries);
    float* const l_p = l_z + entries;
    const float cT = LOG2E * a.inv_T;
    double mine = 0.0;
    auto lanes_meet = [&]() {                                    // what the row's lanes have written, to LDS or to G, comes before what follows
        if constexpr (L > 64) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };
    // (the fewest lanes also have the rows that are shorter than a piece)
    auto load = [&](const T* z, int64_t c) -> Words<T, E> {
        if constexpr (L == 4 && P == 1) return __builtin_bit_cast(Words<T, E>, load_elems<E>(z + c, R::there((int)c, a.C)));
        else return load_near<E>(z, c, a.C);
    };
    // behind the row's end: -inf
    auto whole = [&](Words<T, E> x, int64_t c) {
        const int64_t left = a.C - c;
        if (left >= E) return __builtin_bit_cast(Vec<T>, x);
        Vec<T> v = __builtin_bit_cast(Vec<T>, x);
        if constexpr (!(L == 4 && P == 1)) v = settle<E, T>(x, settle_by<E>(c, a.C));
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = e < left ? v[e] : (T)-INFINITY;
        return v;
    };
    auto highest = [](Vec<T> v, float m) {
#pragma unroll
        for (int e = 0; e < E; ++e) m = fmaxf(m, (float)v[e]);
        return m;
    };
    for (int64_t i = (int64_t)blockIdx.x * R::ROWS + threadIdx.x / L; i < a.n; i += (int64_t)gridDim.x * R::ROWS) {
        const T* const z = (const T*)a.Z + i * a.ldz;
        Vec<T> held[P ? P : 1];
        Words<T, E> near[P ? P : 1];
        if constexpr (P != 0)
#pragma unroll
            for (int p = 0; p < P; ++p) near[p] = load(z, R::column(p));
        const int32_t y = a.labels ? a.labels[i] : -1;
        const bool labelled = y >= 0 && y < a.C;
        // the list, and the maxima of both sides
        float high[3] = {-INFINITY, -INFINITY, 0.f};             // of z, of t, whether there is an entry
        for (int j = li; j < entries; j += L) {
            int32_t at = labelled ? y : -1;
            float t = 0.f;
            if (j < a.k) {
                at = a.top[i * a.ldtop + j];
                t = (float)((const T*)a.t)[i * a.ldt + j];
                if (at >= a.C || t == -INFINITY) at = -1;
                if (at >= 0) {
                    high[1] = fmaxf(high[1], t);
                    high[2] = 1.f;
                }
            }
            l_at[j] = at;
            l_p[j] = t;
            if (at >= 0) l_z[j] = (float)z[at];
        }
        float sum[3] = {0.f, 0.f, 0.f};                          // of e^((z - zh) / T), of e^(z - zh), of the list's e^((t - th) / T)
        float m = -INFINITY;                                     // P = 0: what the thread's sums are relative to
        if constexpr (P != 0) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                held[p] = whole(near[p], R::column(p));
                m = highest(held[p], m);
            }
        } else {
            for (int64_t c = (int64_t)li * E; c < a.C; c += (int64_t)L * E) {
                const Vec<T> v = whole(load(z, c), c);
                const float now = highest(v, m);
                if (now > m) {
                    const float by = power(m, now, cT);          // (nothing before: 0)
                    sum[0] *= by;
                    if (POWER != 1) sum[1] *= plain_power<POWER>(by, m, now);
                    m = now;
                }
                const float from = m == -INFINITY ? 0.f : m;     // (nothing yet: -inf adds 0, and NaN is not lost)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float et = power((float)v[e], from, cT);
                    sum[0] += et;
                    if (POWER != 1) sum[1] += plain_power<POWER>(et, (float)v[e], from);
                }
            }
        }
        high[0] = m;
        join_lanes<L, 3, 3>(high, meet, turn);
        const bool taught = high[2] > 0.f;
        const float zh = high[0], th = high[1];
        if constexpr (P != 0) {
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float et = power((float)held[p][e], zh, cT);
                    sum[0] += et;
                    if (POWER != 1) sum[1] += plain_power<POWER>(et, (float)held[p][e], zh);
                }
        } else if (m == -INFINITY) {                             // nothing in it: 0 (or NaN), and NaN where the whole row is so
            if (zh == -INFINITY) sum[0] = sum[1] = NAN;
        } else {
            const float by = power(m, zh, cT);
            sum[0] *= by;
            if (POWER != 1) sum[1] *= plain_power<POWER>(by, m, zh);
        }
        for (int j = li; j < a.k; j += L)
            if (l_at[j] >= 0) {
                const float e = expf((l_p[j] - th) * a.inv_T);
                l_p[j] = e;
                sum[2] += e;
            }
        join_lanes<L, 3>(sum, meet, turn);
        if (POWER == 1) sum[1] = sum[0];
        const float over = taught ? 1.f / sum[2] : 0.f;
        // sum of p (log p - log q), the list's constant part log(sum of e^((z - zh) / T)) - log(sum of e^((t - th) / T)) taken out of the logarithms; log p is that of
        // the p that counts, and where p is 0 nothing does
        const float apart = taught ? logf(sum[0]) - logf(sum[2]) : 0.f;
        float kl = 0.f;
        for (int j = li; j < a.k; j += L) {
            if (l_at[j] < 0) continue;
            const float p = l_p[j] * over, t = (float)((const T*)a.t)[i * a.ldt + j];
            l_p[j] = p;
            if (p != 0.f) kl = fmaf(p, fmaf((t - th) - (l_z[j] - zh), a.inv_T, apart), kl);
        }
        mine += (double)a.wt * (double)kl;
        if (labelled && li == a.k % L) mine -= (double)a.wl * (double)((l_z[a.k] - zh) - logf(sum[1]));
        lanes_meet();                                            // all of the list is there; the next row writes it anew
        if (!a.G) continue;
        T* const G = (T*)a.G + i * a.ldg;
        const float ct = taught ? a.gt / sum[0] : 0.f, cl = labelled ? a.gl / sum[1] : 0.f;
        const bool any = taught || labelled;                     // the row's powers may be NaN where it is neither: not multiplied away
        auto smooth = [&](float x) {                             // the gradient where the list and the label are not
            const float et = power(x, zh, cT);
            const float g = POWER == 1 ? (ct + cl) * et : fmaf(cl, plain_power<POWER>(et, x, zh), ct * et);
            return any ? g : 0.f;
        };
        auto put = [&](Vec<T> v, int64_t c) {
            Vec<T> out;
#pragma unroll
            for (int e = 0; e < E; ++e) out[e] = (T)smooth((float)v[e]);
            const int64_t left = a.C - c;
            // (a long row's gradient is not for the caches, which hold the rows that are to be read again: 4096 rows of 100,000 in bf16 431 us without)
            if (left >= E && P == 0) stream_vec(G + c, out);
            else if (left >= E) store_vec(G + c, out);
            else if (left > 0) store_vec_part(G + c, out, (int)left);
        };
        if constexpr (P != 0) {
#pragma unroll
            for (int p = 0; p < P; ++p) put(held[p], R::column(p));
        } else {
            for (int64_t c = (int64_t)li * E; c < a.C; c += (int64_t)L * E) put(whole(load(z, c), c), c);
        }
        lanes_meet();                                            // the list's columns are written again, by other lanes
        for (int j = li; j < entries; j += L) {
            const int32_t at = l_at[j];
            if (at < 0) continue;
            float p = 0.f;                                       // of all entries that name this column
            for (int o = 0; o < a.k; ++o) p += l_at[o] == at ? l_p[o] : 0.f;
            G[at] = (T)(smooth(l_z[j]) - fmaf(a.gt, p, labelled && at == y ? a.gl : 0.f));
        }
        lanes_meet();
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) mine += __shfl_xor(mine, d, 64);
    if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        double total = s_w[0];
        for (int w = 1; w < R::THREADS / 64; ++w) total += s_w[w];
        a.part[blockIdx.x] = total;
    }
}

__global__ __launch_bounds__(256) void k_distill_loss(int64_t parts, const double* __restrict__ part, double scale, float* __restrict__ loss) {
    __shared__ double s[256];
    sum_of_losses(part, parts, scale, loss, s);
}

template <typename T>
static int distill_of(DistillArgs a, int64_t m, float T_, float* loss, hipStream_t s) {
    auto launch = [&](auto l, auto p, auto power) -> int {
        constexpr int L = decltype(l)::value, P = decltype(p)::value;
        using R = Rows<T, L, P>;
        const int64_t groups = (a.n + R::ROWS - 1) / R::ROWS, most = (int64_t)device_info().cus * (L <= 64 ? 16 : 2048 / R::THREADS);
        const int blocks = (int)(groups < most ? groups : most);
        ScratchLease lease;
        void* part = nullptr;
        GCN_TRY(lease.get(&part, (size_t)blocks * 8, s));
        a.part = (double*)part;
        launch_lds<k_distill<T, L, P, decltype(power)::value>>(dim3((unsigned)blocks), R::THREADS, (size_t)R::ROWS * (a.k + 1) * 12, s, a);
        GCN_LAUNCH_CHECK();
        hipLaunchKernelGGL(k_distill_loss, dim3(1), dim3(256), 0, s, (int64_t)blocks, (const double*)part, (double)T_ / (double)m, loss);
        GCN_LAUNCH_CHECK();
        return GCN_OK;
    };
    auto with = [&](auto l, auto p) -> int {
        if (T_ == 1.f) return launch(l, p, std::integral_constant<int, 1>());
        if (T_ == 2.f) return launch(l, p, std::integral_constant<int, 2>());
        if (T_ == 4.f) return launch(l, p, std::integral_constant<int, 4>());
        return launch(l, p, std::integral_constant<int, 0>());
    };
    // The fewest lanes that hold a row with four pieces each: more lanes have less to do between the same number of joins (65536 x 1000 in bf16 with 64 lanes 101 us,
    // with 32 68; 65536 x 2000 in fp32 with 256 442, with 128 296).  Short rows are rather bound by what a lane does one piece after the other, and by their lists, of which a
    // lane of few has more: up to 16 pieces eight lanes with two (232965 x 41 in fp32 31.4 us, with four of four 34.8, with eight of four 40.6; x 64 in bf16 39.5, 39.9 and
    // 55; but x 32 in fp32 25.4 and 24.9 with four of four), up to four pieces four lanes with one (232965 x 16 in fp32 17.6, with eight of two 24.4, in bf16 x 32 19.6 and 32.5).
    // Rows of over 16 KB are read twice; the longer, the more lanes: the rows in work at one
    // time, as many as workgroups fit, stay in the caches until they are read again (4096 x 100,000 in bf16 with 512 lanes 493 us, with 1024 431).
    const int64_t pieces = (a.C + Elem<T>::E - 1) / Elem<T>::E;
#define GCN_LANES(L, P) if (pieces <= (int64_t)(L) * (P)) return with(std::integral_constant<int, L>(), std::integral_constant<int, P>())
    GCN_LANES(4, 1); GCN_LANES(8, 2); GCN_LANES(8, 4); GCN_LANES(16, 4); GCN_LANES(32, 4); GCN_LANES(64, 4); GCN_LANES(128, 4); GCN_LANES(256, 4);
    if (pieces <= 8192) return with(std::integral_constant<int, 256>(), std::integral_constant<int, 0>());
#undef GCN_LANES
    return with(std::integral_constant<int, 1024>(), std::integral_constant<int, 0>());
}

}  // namespace gcn

using namespace gcn;

extern "C" int gcn_distill(int64_t n, int32_t C, int type, const void* Z, int64_t ldz, int32_t k, const int32_t* top, int64_t ldtop,
                           const void* t, int64_t ldt, const int32_t* labels, float temperature, float w_teacher, float w_label,
                           int64_t m, float grad_scale, float* loss, void* G, int64_t ldg, void* stream) {
    static const char* const who = "gcn_distill";
    if (!Z || !top || !t || !loss) return fail(GCN_ERR_BADARG, "%s: NULL argument", who);
    if (!known_type(type)) return fail(GCN_ERR_BADARG, "%s: unknown element type %d", who, type);
    if (n <= 0 || C <= 0) return fail(GCN_ERR_BADARG, "%s: sizes must be positive", who);
    if (C > (1 << 30)) return fail(GCN_ERR_RANGE, "%s: there are up to 2^30 classes", who);
    if (k <= 0 || k > C || k > GCN_DISTILL_MOST) return fail(GCN_ERR_BADARG, "%s: a list has 1 to %d entries, and no more than there are classes", who, GCN_DISTILL_MOST);
    if (ldz < C || ldtop < k || ldt < k || (G && ldg < C)) return fail(GCN_ERR_BADARG, "%s: leading dimension below the width", who);
    if (!(temperature > 0.f) || !(temperature < INFINITY)) return fail(GCN_ERR_BADARG, "%s: the temperature must be positive", who);
    if (temperature < 0x1p-126f) return fail(GCN_ERR_RANGE, "%s: temperatures begin at 2^-126", who);
    if (m <= 0) return fail(GCN_ERR_BADARG, "%s: m must be positive", who);
    const size_t b = elem_bytes(type);
    const Span z(Z, n, C, ldz, b), g(G, n, C, ldg, b), at(top, n, k, ldtop, 4), tt(t, n, k, ldt, b), y(labels, 1, n, n, 4), l(loss, 1, 1, 1, 4);
    if ((g.meets(z) && !g.is(z)) || g.meets(at) || g.meets(tt) || g.meets(y) || l.meets(z) || l.meets(g) || l.meets(at) || l.meets(tt) || l.meets(y))
        return fail(GCN_ERR_BADARG, "%s: an output overlaps an input or another output", who);
    DistillArgs a;
    a.n = n; a.C = C; a.k = w_teacher != 0.f ? k : 0; a.Z = Z; a.ldz = ldz; a.G = G; a.ldg = ldg; a.top = top; a.ldtop = ldtop; a.t = t; a.ldt = ldt;
    a.labels = w_label != 0.f ? labels : nullptr;                 // (a part of weight 0 is none, whatever it is: not multiplied away)
    a.inv_T = 1.f / temperature;
    a.wt = w_teacher * temperature;                               // (T^2 in fp32 is 0 below 2^-75, and infinite from 2^64 on)
    a.wl = w_label / temperature;
    const double scale = (double)grad_scale / (double)m;
    a.gt = (float)(scale * w_teacher * temperature);
    a.gl = (float)(scale * w_label);
    return by_type(type, [&](auto e) { return distill_of<decltype(e)>(a, m, temperature, loss, (hipStream_t)stream); });
}
