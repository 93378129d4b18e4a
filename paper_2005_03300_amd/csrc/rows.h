// Rows that a group of lanes holds in registers: L lanes (a power of two), each with P times the elements of 16 bytes, `L * E` elements apart.  Up to 64 lanes
// are a part of a wavefront, and a workgroup of 256 threads has several rows; more are a workgroup, which has one.
#pragma once
#include "elem.h"

namespace gcn {

template <typename T, int L, int P>
struct Rows {
    static constexpr int E = Elem<T>::E, THREADS = L <= 64 ? 256 : L, ROWS = THREADS / L, WAVES = L <= 64 ? 1 : L / 64;
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

// N numbers of every lane joined over the L lanes of a row, by a sum or a maximum; every lane receives the results, in an order that the sizes alone
// decide.  Wavefronts meet in LDS; two places in turn, so that one barrier is enough: a place is written again only behind the barrier of the other.
template <int L, int N, int MAXES = 0>                          // the first MAXES of them by their maximum
__device__ __forceinline__ void join_lanes(float (&v)[N], float (*meet)[16][4], int& turn) {
    constexpr int W = L < 64 ? L : 64;
#pragma unroll
    for (int d = W / 2; d >= 1; d >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float o = __shfl_xor(v[i], d, 64);
            v[i] = i < MAXES ? fmaxf(v[i], o) : v[i] + o;
        }
    if constexpr (L > 64) {
        constexpr int WAVES = L / 64;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) meet[turn][wave][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = meet[turn][0][i];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s = i < MAXES ? fmaxf(s, meet[turn][w][i]) : s + meet[turn][w][i];
            v[i] = s;
        }
        turn ^= 1;
    }
}

}  // namespace gcn
