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
// A place as a number: from 2 on bits 1 and 2 are its exponent and bit 0 is its mantissa; below it is half of itself.
__device__ __forceinline__ float weight4_value(uint32_t code) {
    const uint32_t c = code & 7u;
    const float v = c < 2 ? 0.5f * (float)c : __builtin_bit_cast(float, (c << 22) + (126u << 23));
    return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, v) | (code & 8u) << 28);
}
template <int E>
__device__ __forceinline__ void store_words(uint32_t* p, Elems<uint32_t, E> x, int there) {
    if (there >= E) {
        *reinterpret_cast<LooseElems<uint32_t, E>*>(p) = __builtin_bit_cast(LooseElems<uint32_t, E>, x);
        return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e < there) p[e] = x[e];
}

// A lane has four columns, a wavefront eight rows of them, which are a word each (of groups of 128 two times eight): read once, and held until the workgroup's wavefronts have found the largest
// numbers of the groups in LDS.  Bound by memory and vector instructions: 4099 x 4096 in fp32 25 us, 3.0 TB/s, these issued in 59 % of
// the cycles.
template <typename T>
__global__ __launch_bounds__(512) void k_linear4_pack(int32_t K, int64_t cols, const T* W, int64_t ldw, int group, uint32_t* Q, int64_t ldq, uint16_t* S, int64_t lds) {
    constexpr int E = 4, WAVES = 8;
    __shared__ uint32_t found[WAVES][64][E];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * E;
    const int count = cols - c < 0 ? 0 : cols - c < E ? (int)(cols - c) : E;
    auto unit = [&](int64_t k0, auto words_of_wave) {
        constexpr int WORDS = decltype(words_of_wave)::value;
        Elems<T, E> v[WORDS][8];
        uint32_t most[E] = {};
#pragma unroll
        for (int w = 0; w < WORDS; ++w)
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const int64_t k = k0 + (w * WAVES + wave) * 8 + r;
                v[w][r] = load_elems<E>(W + k * ldw + c, k < K ? count : 0);
            }
#pragma unroll
        for (int w = 0; w < WORDS; ++w)
#pragma unroll
            for (int r = 0; r < 8; ++r)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint32_t b = __builtin_bit_cast(uint32_t, (float)v[w][r][e]) & 0x7fffffffu;
                    most[e] = most[e] > b ? most[e] : b;
                }
#pragma unroll
        for (int e = 0; e < E; ++e) found[wave][lane][e] = most[e];
        __syncthreads();
        const int slices = group == 32 ? 4 : WAVES, first = wave & ~(slices - 1);
        for (int w = 0; w < slices; ++w)
#pragma unroll
            for (int e = 0; e < E; ++e) most[e] = most[e] > found[first + w][lane][e] ? most[e] : found[first + w][lane][e];
        __syncthreads();
        uint32_t bits[E];
        float s[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            bits[e] = scale_of<T>(most[e], WEIGHT4_TOP);
            s[e] = scale_value(bits[e]);
        }
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            const int64_t k = k0 + (w * WAVES + wave) * 8;
            if (k >= K) continue;
            Elems<uint32_t, E> word = {};
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int r = 0; r < 8; ++r) word[e] |= weight4_code((float)v[w][r][e], s[e]) << (4 * r);     // (rows behind the last are zeros, of code 0)
            store_words(Q + k / 8 * ldq + c, word, count);
            if (k % group == 0)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e < count) S[k / group * lds + c + e] = (uint16_t)bits[e];
        }
    };
    const int64_t rows = group == 128 ? 128 : 64;
    for (int64_t k0 = (int64_t)blockIdx.y * rows; k0 < K; k0 += gridDim.y * rows) {
        if (group == 128) unit(k0, std::integral_constant<int, 2>());
        else unit(k0, std::integral_constant<int, 1>());
    }
}

// A lane has the words of 16 bytes of columns, a wavefront all rows of a word, so that each is read once.  Bound by memory: 4099 x 4096 in fp32 13 us, 5.7 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void k_linear4_unpack(int32_t K, int64_t cols, const uint32_t* Q, int64_t ldq, const uint16_t* S, int64_t lds, int group, T* W, int64_t ldw) {
    constexpr int E = Elem<T>::E;
    const int64_t c = ((int64_t)blockIdx.x * 64 + (threadIdx.x & 63)) * E, words = groups_of(K, 8);
    const int count = cols - c < 0 ? 0 : cols - c < E ? (int)(cols - c) : E, shift = group == 32 ? 2 : group == 64 ? 3 : 4;
    if (count == 0) return;
    for (int64_t j = (int64_t)blockIdx.y * 4 + (threadIdx.x >> 6); j < words; j += (int64_t)gridDim.y * 4) {
        const Elems<uint32_t, E> word = load_elems<E>(Q + j * ldq + c, count);
        const Elems<uint16_t, E> bits = load_elems<E>(S + (j >> shift) * lds + c, count);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            if (j * 8 + r >= K) break;
            float v[E];
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = scale_value(bits[e]) * weight4_value(word[e] >> (4 * r));
            store_vec_part(W + (j * 8 + r) * ldw + c, from_floats<T>(v), count);
        }
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
// Workgroups of 64 lanes of so many columns, and enough along k
static dim3 across_and_down(int64_t cols, int64_t each, int64_t down) {
    const int64_t wide = 64 * each;
    return dim3((unsigned)((cols + wide - 1) / wide), (unsigned)(down < 65535 ? down : 65535));
}

extern "C" int gcn_linear4_pack(int32_t f_in, int32_t cols, int type, const void* W, int64_t ldw, int group, uint32_t* Q, int64_t ldq, uint16_t* S, int64_t lds, void* stream) {
    GCN_TRY(check_layout("gcn_linear4_pack", f_in, cols, type, W, ldw, {Q, S, ldq, lds, group}));
    return by_type(type, [&](auto t) -> int {
        using T = decltype(t);
        hipLaunchKernelGGL(k_linear4_pack<T>, across_and_down(cols, 4, groups_of(f_in, group == 128 ? 128 : 64)), dim3(512), 0, (hipStream_t)stream, f_in, cols, (const T*)W, ldw, group, Q, ldq, S, lds);
        GCN_LAUNCH_CHECK();
        return GCN_OK;
    });
}

extern "C" int gcn_linear4_unpack(int32_t f_in, int32_t cols, int type, const uint32_t* Q, int64_t ldq, const uint16_t* S, int64_t lds, int group, void* W, int64_t ldw, void* stream) {
    GCN_TRY(check_layout("gcn_linear4_unpack", f_in, cols, type, W, ldw, {Q, S, ldq, lds, group}));
    return by_type(type, [&](auto t) -> int {
        using T = decltype(t);
        hipLaunchKernelGGL(k_linear4_unpack<T>, across_and_down(cols, Elem<T>::E, groups_of(f_in, 32)), dim3(256), 0, (hipStream_t)stream, f_in, cols, Q, ldq, S, lds, group, (T*)W, ldw);
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
