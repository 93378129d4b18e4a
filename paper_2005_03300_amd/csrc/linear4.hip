// Linear layers and gated blocks whose weights are held in 4 bits: laid out once, and multiplied as they are.
#include "held.h"
#include "linear_tile.h"

namespace gcn {

// The place of |w| among {0, 1/2, 1, 3/2, 2, 3, 4, 6} s, as many as there are borders below it; a border goes to the even place beside it.  Products with a scale are exact.
__device__ __forceinline__ uint32_t weight4_code(float w, float s) {
    const float a = fabsf(w);
    uint32_t c = a > 0.25f * s;
    c += a >= 0.75f * s;
    c += a > 1.25f * s;
    c += a >= 1.75f * s;
    c += a > 2.5f * s;
    c += a >= 3.5f * s;
    c += a > 5.f * s;
    return c ? c | (w < 0.f ? 8u : 0u) : 0u;
}
__device__ __forceinline__ float weight4_value(uint32_t code) {
    const uint32_t c = code & 7u;
    const float v = c < 4 ? 0.5f * c : (c == 7 ? 6.f : (float)c - 2.f);
    return code & 8u ? -v : v;
}

// A thread has a group of a column, read twice: the largest first.
template <typename T>
__global__ __launch_bounds__(256) void k_linear4_pack(int32_t K, int64_t cols, const T* W, int64_t ldw, int group, uint32_t* Q, int64_t ldq, uint16_t* S, int64_t lds) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= cols) return;
    const int64_t groups = groups_of(K, group);
    for (int64_t g = blockIdx.y; g < groups; g += gridDim.y) {
        const int64_t k0 = g * group, k1 = k0 + group < K ? k0 + group : K;
        uint32_t most = 0;
        for (int64_t k = k0; k < k1; ++k) {
            const uint32_t b = __builtin_bit_cast(uint32_t, (float)W[k * ldw + c]) & 0x7fffffffu;
            most = most > b ? most : b;
        }
        const uint32_t bits = scale_of<T>(most, WEIGHT4_TOP);
        const float s = scale_value(bits);
        for (int64_t k = k0; k < k1; k += 8) {
            uint32_t word = 0;
            for (int e = 0; e < 8; ++e)
                if (k + e < k1) word |= weight4_code((float)W[(k + e) * ldw + c], s) << (4 * e);
            Q[k / 8 * ldq + c] = word;
        }
        S[g * lds + c] = (uint16_t)bits;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_linear4_unpack(int32_t K, int64_t cols, const uint32_t* Q, int64_t ldq, const uint16_t* S, int64_t lds, int group, T* W, int64_t ldw) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x, words = groups_of(K, 8);
    if (c >= cols) return;
    for (int64_t j = blockIdx.y; j < words; j += gridDim.y) {
        const uint32_t q = Q[j * ldq + c];
        const float s = scale_value(S[j * 8 / group * lds + c]);
        for (int e = 0; e < 8; ++e)
            if (j * 8 + e < K) W[(j * 8 + e) * ldw + c] = (T)(s * weight4_value(q >> (4 * e)));
    }
}

template <typename T> int linear4_of(const TileArgs& a, const Weights4& w, hipStream_t s);

}  // namespace gcn

using namespace gcn;

static int check_weights(const char* who, int32_t f_in, int64_t cols, const Weights4& w) {
    if (w.group != 32 && w.group != 64 && w.group != 128) return fail(GCN_ERR_BADARG, "%s: groups are of 32, 64 or 128 weights, not %d", who, w.group);
    if (f_in <= 0 || cols <= 0) return fail(GCN_ERR_BADARG, "%s: sizes must be positive", who);
    if (f_in > LINEAR_WIDEST || cols > LINEAR_WIDEST) return fail(GCN_ERR_RANGE, "%s: widths go up to 2^27", who);
    if (w.ldq < cols || w.lds < cols) return fail(GCN_ERR_BADARG, "%s: leading dimension below the width", who);
    return GCN_OK;
}
static Span words_of(const Weights4& w, int32_t f_in, int64_t cols) { return Span(w.Q, groups_of(f_in, 8), cols, w.ldq, 4); }
static Span scales_of(const Weights4& w, int32_t f_in, int64_t cols) { return Span(w.S, groups_of(f_in, w.group), cols, w.lds, 2); }

static int check_layout(const char* who, int32_t f_in, int32_t cols, int type, const void* W, int64_t ldw, const Weights4& w) {
    if (!W || !w.Q || !w.S) return fail(GCN_ERR_BADARG, "%s: NULL argument", who);
    if (!known_type(type)) return fail(GCN_ERR_BADARG, "%s: unknown element type %d", who, type);
    GCN_TRY(check_weights(who, f_in, cols, w));
    if (ldw < cols) return fail(GCN_ERR_BADARG, "%s: leading dimension below the width", who);
    const Span m(W, f_in, cols, ldw, elem_bytes(type)), q = words_of(w, f_in, cols), s = scales_of(w, f_in, cols);
    if (m.meets(q) || m.meets(s) || q.meets(s)) return fail(GCN_ERR_BADARG, "%s: an output overlaps an input or another output", who);
    return GCN_OK;
}
static dim3 columns_and_steps(int64_t cols, int64_t steps) { return dim3((unsigned)((cols + 255) / 256), (unsigned)(steps < 65535 ? steps : 65535)); }

extern "C" int gcn_linear4_pack(int32_t f_in, int32_t cols, int type, const void* W, int64_t ldw, int group, uint32_t* Q, int64_t ldq, uint16_t* S, int64_t lds, void* stream) {
    GCN_TRY(check_layout("gcn_linear4_pack", f_in, cols, type, W, ldw, {Q, S, ldq, lds, group}));
    return by_type(type, [&](auto t) -> int {
        using T = decltype(t);
        hipLaunchKernelGGL(k_linear4_pack<T>, columns_and_steps(cols, groups_of(f_in, group)), dim3(256), 0, (hipStream_t)stream, f_in, cols, (const T*)W, ldw, group, Q, ldq, S, lds);
        GCN_LAUNCH_CHECK();
        return GCN_OK;
    });
}

extern "C" int gcn_linear4_unpack(int32_t f_in, int32_t cols, int type, const uint32_t* Q, int64_t ldq, const uint16_t* S, int64_t lds, int group, void* W, int64_t ldw, void* stream) {
    GCN_TRY(check_layout("gcn_linear4_unpack", f_in, cols, type, W, ldw, {Q, S, ldq, lds, group}));
    return by_type(type, [&](auto t) -> int {
        using T = decltype(t);
        hipLaunchKernelGGL(k_linear4_unpack<T>, columns_and_steps(cols, groups_of(f_in, 8)), dim3(256), 0, (hipStream_t)stream, f_in, cols, Q, ldq, S, lds, group, (T*)W, ldw);
        GCN_LAUNCH_CHECK();
        return GCN_OK;
    });
}

extern "C" int gcn_linear4_forward(int64_t n, int32_t f_in, int32_t f_out, int type, const void* X, int64_t ldx, const uint32_t* Q, int64_t ldq, const uint16_t* S, int64_t lds, int group,
                                   int gated, const float* bias, int act, const void* R, int64_t ldr, float rho, void* Y, int64_t ldy, void* stream) {
    static const char* const who = "gcn_linear4_forward";
    if (!X || !Q || !S || !Y) return fail(GCN_ERR_BADARG, "%s: NULL argument", who);
    if (!known_type(type)) return fail(GCN_ERR_BADARG, "%s: unknown element type %d", who, type);
    if (!known_act(act)) return fail(GCN_ERR_BADARG, "%s: unknown activation %d", who, act);
    if (n <= 0 || f_out <= 0) return fail(GCN_ERR_BADARG, "%s: sizes must be positive", who);
    const int64_t cols = (int64_t)f_out * (gated ? 2 : 1);
    const Weights4 w{Q, S, ldq, lds, group, gated != 0};
    GCN_TRY(check_weights(who, f_in, cols, w));
    if (ldx < f_in || ldy < f_out || (R && ldr < f_out)) return fail(GCN_ERR_BADARG, "%s: leading dimension below the width", who);
    const size_t b = elem_bytes(type);
    const Span x(X, n, f_in, ldx, b), y(Y, n, f_out, ldy, b), r(R, n, f_out, ldr, b), v(bias, 1, cols, cols, 4);
    if (y.meets(x) || y.meets(words_of(w, f_in, cols)) || y.meets(scales_of(w, f_in, cols)) || y.meets(v) || (y.meets(r) && !y.is(r)))
        return fail(GCN_ERR_BADARG, "%s: an output overlaps an input or another output", who);
    TileArgs a;
    a.A = X; a.lda = ldx; a.M = n; a.N = f_out; a.K = f_in; a.bias = bias; a.act = act; a.R = R; a.ldr = ldr; a.rho = rho; a.Y = Y; a.ldy = ldy;
    return by_type(type, [&](auto t) { return linear4_of<decltype(t)>(a, w, (hipStream_t)stream); });
}
