// Rows that a group of lanes holds in registers: L lanes (a power of two), each with P times the elements of 16 bytes, `L * E` elements apart.  Up to 64 lanes
// are a part of a wavefront, and a workgroup of 256 threads has several rows; more are a workgroup, which has one.
#pragma once
#include <type_traits>

#include "elem.h"

namespace gcn {

template <typename T, int L, int P>
struct Rows {
    static constexpr int E = Elem<T>::E, THREADS = L <= 64 ? 256 : L, ROWS = THREADS / L;
    __device__ static int column(int p) { return (p * L + (int)(threadIdx.x % L)) * E; }
    // of the E elements from column c on, how many a row of f has
    __device__ static int there(int c, int32_t f) { return f - c < 0 ? 0 : (f - c > E ? E : f - c); }
};

template <typename T>
__device__ __forceinline__ void to_floats(Vec<T> x, float (&v)[Elem<T>::E]) {
#pragma unroll
    for (int e = 0; e < Elem<T>::E; ++e) v[e] = (float)x[e];
}
template <typename T>
__device__ __forceinline__ Vec<T> from_floats(const float (&v)[Elem<T>::E]) {
    Vec<T> x;
#pragma unroll
    for (int e = 0; e < Elem<T>::E; ++e) x[e] = (T)v[e];
    return x;
}
// E floats of a vector that goes with the columns; zeros (or `fill`) where there is none
template <int E>
__device__ __forceinline__ void load_floats(const float* p, int64_t c, int count, float fill, float (&v)[E]) {
    if (!p || count <= 0) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = p ? 0.f : fill;
        return;
    }
    if (count >= E) {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            const f4u t = *reinterpret_cast<const f4u*>(p + c + e);
            v[e] = t.x; v[e + 1] = t.y; v[e + 2] = t.z; v[e + 3] = t.w;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e < count ? p[c + e] : 0.f;
}

// The value of the lane whose number differs in bit D (all lanes take part; with D = 4 and 8 of the lane mirrored in 8 and 16, which is the same once
// the lower bits are joined).  Register moves between lanes: through LDS, as a shuffle goes, each took six times as long.
template <int D>
__device__ __forceinline__ float partner(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
    const int x = __builtin_bit_cast(int, v);
    if constexpr (D == 1) return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, true));
    if constexpr (D == 2) return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, true));
    if constexpr (D == 4) return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, true));
    if constexpr (D == 8) return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, x, 0x140, 0xf, 0xf, true));
#endif
    return v;
}
// v of this lane and of its partner, joined
template <int D, bool MAX>
__device__ __forceinline__ float with_partner(float v) {
    auto join = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
#if defined(__HIP_DEVICE_COMPILE__)
    const unsigned x = __builtin_bit_cast(unsigned, v);
    if constexpr (D == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return join(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
    }
    if constexpr (D == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return join(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
    }
#endif
    return join(v, partner<D>(v));
}

template <int L, int N, int MAXES>
__device__ __forceinline__ void fold_lanes(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        auto fold = [&](auto is_max) {
            constexpr bool M = decltype(is_max)::value;
            if constexpr (L >= 2) v[i] = with_partner<1, M>(v[i]);
            if constexpr (L >= 4) v[i] = with_partner<2, M>(v[i]);
            if constexpr (L >= 8) v[i] = with_partner<4, M>(v[i]);
            if constexpr (L >= 16) v[i] = with_partner<8, M>(v[i]);
            if constexpr (L >= 32) v[i] = with_partner<16, M>(v[i]);
            if constexpr (L >= 64) v[i] = with_partner<32, M>(v[i]);
        };
        if (i < MAXES) fold(std::true_type());
        else fold(std::false_type());
    }
}

// N numbers of every lane joined over the L lanes of a row, the first MAXES by their maximum, the others by their sum; every lane receives the results, in an
// order that the sizes alone decide.  Wavefronts meet in LDS; two places in turn, so that one barrier is enough: a place is written again only behind the
// barrier of the other.
template <int L, int N, int MAXES = 0>
__device__ __forceinline__ void join_lanes(float (&v)[N], float (*meet)[16][4], int& turn) {
    fold_lanes<(L < 64 ? L : 64), N, MAXES>(v);
    if constexpr (L > 64) {
        constexpr int WAVES = L / 64;
        const int lane = threadIdx.x & 63, first = (int)(threadIdx.x >> 6) & ~(WAVES - 1);    // of the row's wavefronts
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) meet[turn][threadIdx.x >> 6][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = meet[turn][first + (lane & (WAVES - 1))][i];
        fold_lanes<WAVES, N, MAXES>(v);
        turn ^= 1;
    }
}

}  // namespace gcn
