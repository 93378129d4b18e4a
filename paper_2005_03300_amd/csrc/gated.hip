// A gated block over the rows of X: Z = X W + 1 bias^T with W of 2 N columns, H = act(Z's first N columns) (Hadamard) the others, and its gradients.
#include "slope.h"

using namespace gcn;

extern "C" int gcn_gated_forward(int64_t n, int32_t f_in, int32_t f_out, int type, const void* X, int64_t ldx, const void* W, int64_t ldw, const float* bias, int act, void* Z,
                                 int64_t ldz, void* H, int64_t ldh, void* stream) {
    static const char* const who = "gcn_gated_forward";
    if (!X || !W || !H) return fail(GCN_ERR_BADARG, "%s: NULL argument", who);
    if (!known_type(type)) return fail(GCN_ERR_BADARG, "%s: unknown element type %d", who, type);
    if (!known_act(act)) return fail(GCN_ERR_BADARG, "%s: unknown activation %d", who, act);
    if (n <= 0 || f_in <= 0 || f_out <= 0) return fail(GCN_ERR_BADARG, "%s: sizes must be positive", who);
    if (f_in > LINEAR_WIDEST || f_out > LINEAR_WIDEST / 2) return fail(GCN_ERR_RANGE, "%s: f_in goes up to 2^27, f_out to 2^26", who);
    const int64_t cols = 2 * (int64_t)f_out;
    if (ldx < f_in || ldw < cols || ldh < f_out || (Z && ldz < cols)) return fail(GCN_ERR_BADARG, "%s: leading dimension below the width", who);
    const size_t b = elem_bytes(type);
    const Span x(X, n, f_in, ldx, b), w(W, f_in, cols, ldw, b), v(bias, 1, cols, cols, 4), z(Z, n, cols, ldz, b), h(H, n, f_out, ldh, b);
    if (h.meets(x) || h.meets(w) || h.meets(v) || z.meets(x) || z.meets(w) || z.meets(v) || z.meets(h))
        return fail(GCN_ERR_BADARG, "%s: an output overlaps an input or another output", who);
    TileArgs a;
    a.A = X; a.lda = ldx; a.B = W; a.ldb = ldw; a.M = n; a.N = f_out; a.K = f_in; a.bias = bias; a.act = act; a.Z = Z; a.ldz = ldz; a.Y = H; a.ldy = ldh;
    return by_type(type, [&](auto t) { return gated_forward_of<decltype(t)>(a, (hipStream_t)stream); });
}

extern "C" int gcn_gated_backward(int64_t n, int32_t f_in, int32_t f_out, int type, const void* X, int64_t ldx, const uint16_t* x_scales, int64_t ldxs, const void* W, int64_t ldw,
                                  const void* Z, int64_t ldz, const uint16_t* z_scales, int64_t ldzs, const void* dH, int64_t lddh, int act, void* dZ, int64_t lddz, void* dX,
                                  int64_t lddx, void* dW, int64_t lddw, float* dbias, void* H, int64_t ldh, void* stream) {
    static const char* const who = "gcn_gated_backward";
    const hipStream_t s = (hipStream_t)stream;
    if (!dH || !Z || (dW && !X) || (dX && !W)) return fail(GCN_ERR_BADARG, "%s: NULL argument", who);
    if (!known_type(type)) return fail(GCN_ERR_BADARG, "%s: unknown element type %d", who, type);
    if (!known_act(act)) return fail(GCN_ERR_BADARG, "%s: unknown activation %d", who, act);
    if ((dX || dW) && !dZ) return fail(GCN_ERR_BADARG, "%s: the products need dZ as workspace", who);
    if (n <= 0 || f_in <= 0 || f_out <= 0) return fail(GCN_ERR_BADARG, "%s: sizes must be positive", who);
    if (f_in > LINEAR_WIDEST || f_out > LINEAR_WIDEST / 2) return fail(GCN_ERR_RANGE, "%s: f_in goes up to 2^27, f_out to 2^26", who);
    const int64_t cols = 2 * (int64_t)f_out;
    const Kept x{X, ldx, X ? x_scales : nullptr, ldxs}, z{Z, ldz, z_scales, ldzs};
    if (lddh < f_out || (x.p && ldx < f_in) || (x.scales && ldxs < groups_of(f_in, CHECKPOINT_GROUP)) || (W && ldw < cols) || ldz < cols ||
        (z.scales && ldzs < groups_of(cols, CHECKPOINT_GROUP)) || (dZ && lddz < cols) || (dX && lddx < f_in) || (dW && lddw < cols) || (H && ldh < f_out))
        return fail(GCN_ERR_BADARG, "%s: leading dimension below the width", who);
    const size_t b = elem_bytes(type);
    const Span in[] = {span_of(x, n, f_in, b), scales_of(x, n, f_in), Span(W, f_in, cols, ldw, b), span_of(z, n, cols, b), scales_of(z, n, cols), Span(dH, n, f_out, lddh, b)};
    const Span out[] = {Span(dZ, n, cols, lddz, b), Span(H, n, f_out, ldh, b), Span(dX, n, f_in, lddx, b), Span(dW, f_in, cols, lddw, b), Span(dbias, 1, cols, cols, 4)};
    bool bad = false;
    for (int o = 0; o < 5; ++o) {
        // an element of dZ may take the place of the one of Z that it is made of, one of H that of dH
        for (int i = 0; i < 6; ++i) bad |= out[o].meets(in[i]) && !(((o == 0 && i == 3 && !z.scales) || (o == 1 && i == 5)) && out[o].is(in[i]));
        for (int i = 0; i < o; ++i) bad |= out[o].meets(out[i]);
    }
    if (bad) return fail(GCN_ERR_BADARG, "%s: an output overlaps an input or another output", who);
    if (dbias || H || dZ) {
        SlopeArgs a;
        a.n = n; a.N = f_out; a.Z = z; a.dY = dH; a.lddy = lddh; a.act = act; a.dZ = dZ; a.lddz = lddz; a.also = H; a.ldalso = ldh;
        GCN_TRY(by_type(type, [&](auto t) {
            using T = decltype(t);
            return z.scales ? launch_slope<T, true, true>(a, dbias, s) : launch_slope<T, true, false>(a, dbias, s);
        }));
    }
    BackProducts p;
    p.n = n; p.f_in = f_in; p.cols = (int32_t)cols; p.X = x; p.W = W; p.ldw = ldw; p.G = dZ; p.ldg = lddz; p.dX = dX; p.lddx = lddx; p.dW = dW; p.lddw = lddw;
    return back_products(type, p, s);
}
