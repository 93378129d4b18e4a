// Checkpoints of activations in 8 bits: stored, restored, and read by the backward pass of a linear layer.
#include "slope.h"

namespace gcn {

// The largest of the bits of L lanes' numbers without their signs (NaN and infinities are the largest).
template <int L>
__device__ __forceinline__ uint32_t most_of_lanes(uint32_t v) {
    auto with = [&](float p) {
        const uint32_t o = __builtin_bit_cast(uint32_t, p);
        v = v > o ? v : o;
    };
    with(partner<1>(__builtin_bit_cast(float, v)));
    with(partner<2>(__builtin_bit_cast(float, v)));
    with(partner<4>(__builtin_bit_cast(float, v)));
    if constexpr (L == 16) with(partner<8>(__builtin_bit_cast(float, v)));
    return v;
}

// The largest of the bits of 16 bytes of elements without their signs, as those of an fp32 number; of 16-bit ones two at a time.
template <typename T>
__device__ __forceinline__ uint32_t most_of(Vec<T> x) {
    if constexpr (sizeof(T) == 4) {
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float v = x[e];                                 // (the bits of a vector's element taken in place are those of its first)
            const uint32_t b = __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
            most = most > b ? most : b;
        }
        return most;
    } else {
        typedef unsigned short u2 __attribute__((ext_vector_type(2)));
        const Words<T, 8> w = __builtin_bit_cast(Words<T, 8>, x);
        u2 most = __builtin_bit_cast(u2, w[0] & 0x7fff7fffu);
#pragma unroll
        for (int e = 1; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(u2, w[e] & 0x7fff7fffu));
        const uint16_t m = most[0] > most[1] ? most[0] : most[1];
        return __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(T, m));
    }
}
// The lowest bytes of four words.
__device__ __forceinline__ uint32_t lowest_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
#if defined(__HIP_DEVICE_COMPILE__)
    const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), cd = __builtin_amdgcn_perm(d, c, 0x0c0c0400u);
    return __builtin_amdgcn_perm(cd, ab, 0x05040100u);
#else
    return (a & 255u) | (b & 255u) << 8 | (c & 255u) << 16 | d << 24;
#endif
}

// The pieces of a matrix, `per` of each row, that a lane comes to: the lane's own and then as many further on as there are lanes, which are `rows` rows and `pieces` pieces.
struct Walk {
    int64_t row;
    int32_t piece, per, pieces;
    int64_t rows;
    __device__ Walk(int32_t per, int32_t lanes) : per(per) {
        const uint32_t t = blockIdx.x * 256 + threadIdx.x;       // (a launch has up to 2^20 lanes)
        row = t / (uint32_t)per;
        piece = (int32_t)(t % (uint32_t)per);
        rows = lanes / per;
        pieces = lanes % per;
    }
    __device__ void next() {
        row += rows;
        piece += pieces;
        if (piece >= per) {
            piece -= per;
            ++row;
        }
    }
};

// 16 bytes of a row for each lane, 8 lanes (fp32: 16) for a group, whose largest number they find together.  A piece that a row's end cuts is the row's last whole one instead, where that lies in the
// same group: its codes are written twice, the same.  Bound by memory and, with 12 vector instructions an element, nearly as much by these: 232965 x 602 in bf16 103 us,
// 4.2 TB/s, vector instructions issued in 65 % of the cycles.
template <typename T>
__global__ __launch_bounds__(256) void k_checkpoint_pack(int64_t n, int32_t f, const T* X, int64_t ldx, int8_t* C, int64_t ldc, uint16_t* S, int64_t lds) {
    constexpr int E = Elem<T>::E, L = CHECKPOINT_GROUP / E, A = 2;
    const int32_t per = (int32_t)groups_of(f, CHECKPOINT_GROUP) * L;          // lanes of a row
    const int32_t end = f % CHECKPOINT_GROUP, last = end == 0 || end >= E ? f - E : f;         // where the last whole piece of the last group begins
    Walk at(per, gridDim.x * 256);
    while (at.row < n) {                                          // (a group's lanes go together)
        Vec<T> x[A];
        int64_t row[A];
        int32_t col[A];
#pragma unroll
        for (int u = 0; u < A; ++u) {
            row[u] = at.row;
            col[u] = at.piece * E;
            at.next();
            const T* const from = X + (row[u] < n ? row[u] : n - 1) * ldx;
            if (last < f) x[u] = load_vec(from + (col[u] < last ? col[u] : last));
            else x[u] = load_vec_part(from + col[u], f - col[u] < 0 ? 0 : f - col[u]);
        }
#pragma unroll
        for (int u = 0; u < A; ++u) {
            const uint32_t bits = scale_of<T>(most_of_lanes<L>(most_of<T>(x[u])), CHECKPOINT_TOP);
            const int64_t i = row[u];
            if (i >= n || col[u] >= f) continue;
            const float s = scale_value(bits), inv = inverse(s);
            float v[E];
            to_floats<T>(x[u], v);
            if (bits == largest_scale<T>(CHECKPOINT_TOP)) {       // numbers beyond what that reaches
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = fminf(fmaxf(v[e], -CHECKPOINT_TOP * s), CHECKPOINT_TOP * s);
            }
            uint32_t code[E];
#pragma unroll
            for (int e = 0; e < E; ++e) code[e] = checkpoint_code<T>(v[e], s, inv);
            int8_t* const to = C + i * ldc;
            if (last < f) {
                LooseCodes<E> q;
#pragma unroll
                for (int w = 0; w < E / 4; ++w) q.w[w] = lowest_bytes(code[4 * w], code[4 * w + 1], code[4 * w + 2], code[4 * w + 3]);
                *reinterpret_cast<LooseCodes<E>*>(to + (col[u] < last ? col[u] : last)) = q;
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (col[u] + e < f) to[col[u] + e] = (int8_t)code[e];
            }
            if (col[u] % CHECKPOINT_GROUP == 0) S[i * lds + col[u] / CHECKPOINT_GROUP] = (uint16_t)bits;
        }
    }
}

// A lane has 16 bytes of a row; those that its end cuts are the row's last whole ones, of which some lie in the group before.  Four rows' loads are on their way at a time.  Bound by memory: 232965 x 602
// in bf16 100 us, 4.45 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void k_checkpoint_unpack(int64_t n, int32_t f, const int8_t* C, int64_t ldc, const uint16_t* S, int64_t lds, T* X, int64_t ldx) {
    constexpr int E = Elem<T>::E, A = 4;
    const int32_t last = f - E;
    Walk at((int32_t)groups_of(f, E), gridDim.x * 256);
    while (at.row < n) {
        Codes<E> q[A];
        uint16_t s[A][2];
        int64_t row[A];
        int32_t col[A];
#pragma unroll
        for (int u = 0; u < A; ++u) {
            row[u] = at.row;
            col[u] = at.piece * E;
            if (last >= 0 && col[u] > last) col[u] = last;
            at.next();
            const int64_t i = row[u] < n ? row[u] : n - 1;
            q[u] = load_codes<E>(C + i * ldc, col[u], f);
            s[u][0] = S[i * lds + col[u] / CHECKPOINT_GROUP];
            s[u][1] = S[i * lds + (last >= 0 ? col[u] + E - 1 : f - 1) / CHECKPOINT_GROUP];
        }
#pragma unroll
        for (int u = 0; u < A; ++u) {
            if (row[u] >= n) break;
            const int here = CHECKPOINT_GROUP - col[u] % CHECKPOINT_GROUP;
            const float s0 = scale_value(s[u][0]), s1 = scale_value(s[u][1]);
            float v[E];
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = (e < here ? s0 : s1) * code_value<E>(q[u], e);
            T* const to = X + row[u] * ldx + col[u];
            if (last >= 0) store_vec(to, from_floats<T>(v));
            else store_vec_part(to, from_floats<T>(v), f);
        }
    }
}

static unsigned passes(int64_t pieces) {                          // workgroups of a pass over matrices: two pieces for each lane, and more
    const int64_t blocks = (pieces + 511) / 512, most = 16 * (int64_t)device_info().cus;
    return (unsigned)(blocks < most ? blocks : most);
}

template <typename T>
static int unpack_launch(int64_t n, int32_t f, const Kept& k, void* X, int64_t ldx, hipStream_t s) {
    hipLaunchKernelGGL(k_checkpoint_unpack<T>, dim3(passes(n * groups_of(f, Elem<T>::E))), dim3(256), 0, s, n, f, (const int8_t*)k.p, k.ld, k.scales, k.lds, (T*)X, ldx);
    GCN_LAUNCH_CHECK();
    return GCN_OK;
}

int back_products(int type, const BackProducts& b, hipStream_t s) {
    return by_type(type, [&](auto t) -> int {
        using T = decltype(t);
        if (b.dX) {
            TileArgs a;
            a.A = b.G; a.lda = b.ldg; a.B = b.W; a.ldb = b.ldw; a.M = b.n; a.N = b.f_in; a.K = b.cols; a.Y = b.dX; a.ldy = b.lddx;
            GCN_TRY(linear_dx_of<T>(a, s));
        }
        if (b.dW) {
            TileArgs a;
            const void* X = b.X.p;
            int64_t ldx = b.X.ld;
            ScratchLease lease;
            if (b.X.scales && sizeof(T) == 4 && b.f_in % 4 == 0) {             // fp32 products split their operands on the way to LDS, and codes as well
                a.a_scales = b.X.scales;
                a.lda_scales = b.X.lds;
            } else if (b.X.scales) {                              // into rows of whole pieces, which the tiles take straight to LDS (dW of 25809 x 2271 x 800 in fp16 127 us, 166 in rows of 2271)
                void* p = nullptr;
                ldx = groups_of(b.f_in, Elem<T>::E) * Elem<T>::E;
                GCN_TRY(lease.get(&p, (size_t)b.n * ldx * sizeof(T), s));
                GCN_TRY(unpack_launch<T>(b.n, b.f_in, b.X, p, ldx, s));
                X = p;
            }
            a.a_wide = X == b.X.p ? 0 : ldx;
            a.A = X; a.lda = ldx; a.B = b.G; a.ldb = b.ldg; a.M = b.f_in; a.N = b.cols; a.K = b.n; a.Y = b.dW; a.ldy = b.lddw;
            GCN_TRY(linear_dw_of<T>(a, s));
        }
        return GCN_OK;
    });
}

}  // namespace gcn

using namespace gcn;

static int check_pack(const char* who, int64_t n, int32_t f, int type, const void* X, int64_t ldx, const Kept& k) {
    if (!X || !k.p || !k.scales) return fail(GCN_ERR_BADARG, "%s: NULL argument", who);
    if (!known_type(type)) return fail(GCN_ERR_BADARG, "%s: unknown element type %d", who, type);
    if (n <= 0 || f <= 0) return fail(GCN_ERR_BADARG, "%s: sizes must be positive", who);
    if (f > LINEAR_WIDEST) return fail(GCN_ERR_RANGE, "%s: widths go up to 2^27", who);
    if (ldx < f || k.ld < f || k.lds < groups_of(f, CHECKPOINT_GROUP)) return fail(GCN_ERR_BADARG, "%s: leading dimension below the width", who);
    const Span x(X, n, f, ldx, elem_bytes(type)), c = span_of(k, n, f, 1), s = scales_of(k, n, f);
    if (x.meets(c) || x.meets(s) || c.meets(s)) return fail(GCN_ERR_BADARG, "%s: an output overlaps an input or another output", who);
    return GCN_OK;
}

extern "C" int gcn_checkpoint_pack(int64_t n, int32_t f, int type, const void* X, int64_t ldx, int8_t* codes, int64_t ldc, uint16_t* scales, int64_t lds, void* stream) {
    GCN_TRY(check_pack("gcn_checkpoint_pack", n, f, type, X, ldx, {codes, ldc, scales, lds}));
    return by_type(type, [&](auto t) -> int {
        using T = decltype(t);
        hipLaunchKernelGGL(k_checkpoint_pack<T>, dim3(passes(n * groups_of(f, CHECKPOINT_GROUP) * (CHECKPOINT_GROUP / Elem<T>::E))), dim3(256), 0, (hipStream_t)stream, n, f,
                           (const T*)X, ldx, codes, ldc, scales, lds);
        GCN_LAUNCH_CHECK();
        return GCN_OK;
    });
}

extern "C" int gcn_checkpoint_unpack(int64_t n, int32_t f, int type, const int8_t* codes, int64_t ldc, const uint16_t* scales, int64_t lds, void* X, int64_t ldx, void* stream) {
    const Kept k{codes, ldc, scales, lds};
    GCN_TRY(check_pack("gcn_checkpoint_unpack", n, f, type, X, ldx, k));
    return by_type(type, [&](auto t) { return unpack_launch<decltype(t)>(n, f, k, X, ldx, (hipStream_t)stream); });
}

extern "C" int gcn_checkpoint_linear_backward(int64_t n, int32_t f_in, int32_t f_out, int type, const void* X, int64_t ldx, const uint16_t* x_scales, int64_t ldxs, const void* W,
                                              int64_t ldw, const void* Z, int64_t ldz, const uint16_t* z_scales, int64_t ldzs, const void* dY, int64_t lddy, int act, float rho, void* dZ,
                                              int64_t lddz, void* dX, int64_t lddx, void* dW, int64_t lddw, float* dbias, void* dR, int64_t lddr, void* stream) {
    static const char* const who = "gcn_checkpoint_linear_backward";
    const hipStream_t s = (hipStream_t)stream;
    if (!dY || (dW && !X) || (dX && !W)) return fail(GCN_ERR_BADARG, "%s: NULL argument", who);
    if (!known_type(type)) return fail(GCN_ERR_BADARG, "%s: unknown element type %d", who, type);
    if (!known_act(act)) return fail(GCN_ERR_BADARG, "%s: unknown activation %d", who, act);
    const bool curved = act != GCN_ACT_NONE, products = dX || dW;
    if (curved && (products || dbias || dZ) && !Z) return fail(GCN_ERR_BADARG, "%s: the activation's derivative needs Z", who);
    if (curved && products && !dZ) return fail(GCN_ERR_BADARG, "%s: the products need dZ as workspace", who);
    if (n <= 0 || f_in <= 0 || f_out <= 0) return fail(GCN_ERR_BADARG, "%s: sizes must be positive", who);
    if (f_in > LINEAR_WIDEST || f_out > LINEAR_WIDEST) return fail(GCN_ERR_RANGE, "%s: widths go up to 2^27", who);
    const Kept x{X, ldx, X ? x_scales : nullptr, ldxs}, z{curved ? Z : nullptr, ldz, curved && Z ? z_scales : nullptr, ldzs};
    if (lddy < f_out || (x.p && ldx < f_in) || (x.scales && ldxs < groups_of(f_in, CHECKPOINT_GROUP)) || (W && ldw < f_out) || (z.p && ldz < f_out) ||
        (z.scales && ldzs < groups_of(f_out, CHECKPOINT_GROUP)) || (curved && dZ && lddz < f_out) || (dX && lddx < f_in) || (dW && lddw < f_out) || (dR && lddr < f_out))
        return fail(GCN_ERR_BADARG, "%s: leading dimension below the width", who);
    const size_t b = elem_bytes(type);
    if (!curved) dZ = nullptr;
    const Span in[] = {span_of(x, n, f_in, b), scales_of(x, n, f_in), Span(W, f_in, f_out, ldw, b), span_of(z, n, f_out, b), scales_of(z, n, f_out), Span(dY, n, f_out, lddy, b)};
    const Span out[] = {Span(dZ, n, f_out, lddz, b), Span(dR, n, f_out, lddr, b), Span(dX, n, f_in, lddx, b), Span(dW, f_in, f_out, lddw, b), Span(dbias, 1, f_out, f_out, 4)};
    bool bad = false;
    for (int o = 0; o < 5; ++o) {
        for (int i = 0; i < 6; ++i) {
            // an element of dZ may take the place of the one of Z or dY that it is made of, one of dR that of dY
            const bool may = (o == 0 && ((i == 3 && !z.scales) || i == 5)) || (o == 1 && i == 5 && (curved || !products));
            bad |= out[o].meets(in[i]) && !(may && out[o].is(in[i]));
        }
        for (int i = 0; i < o; ++i) bad |= out[o].meets(out[i]);
    }
    if (bad) return fail(GCN_ERR_BADARG, "%s: an output overlaps an input or another output", who);
    if (dbias || dR || dZ) {
        SlopeArgs a;
        a.n = n; a.N = f_out; a.Z = z; a.dY = dY; a.lddy = lddy; a.dZ = dZ; a.lddz = lddz; a.also = dR; a.ldalso = lddr; a.rho = rho;
        a.act = dbias || dZ ? act : GCN_ACT_NONE;
        GCN_TRY(z.scales ? by_type(type, [&](auto t) { return launch_slope<decltype(t), false, true>(a, dbias, s); }) : launch_linear_slope(type, a, dbias, s));
    }
    BackProducts p;
    p.n = n; p.f_in = f_in; p.cols = f_out; p.X = x; p.W = W; p.ldw = ldw; p.G = curved ? dZ : dY; p.ldg = curved ? lddz : lddy;
    p.dX = dX; p.lddx = lddx; p.dW = dW; p.lddw = lddw;
    return back_products(type, p, s);
}
