// Elements of 32 and 16 bits: 16 bytes of them at a time, at any address that the type itself is aligned for, and as floats.
#pragma once
#include <type_traits>

#include "common.h"
#include "places.h"

namespace gcn {

typedef float v4f __attribute__((ext_vector_type(4)));

template <typename T> struct Elem;
template <> struct Elem<float> {
    static constexpr int E = 4;                                  // elements of 16 bytes
    typedef float V __attribute__((ext_vector_type(4)));
    struct __attribute__((packed, aligned(4))) Loose { uint32_t w[4]; };
};
template <> struct Elem<__bf16> {
    static constexpr int E = 8;
    typedef __bf16 V __attribute__((ext_vector_type(8)));
    struct __attribute__((packed, aligned(2))) Loose { uint32_t w[4]; };
};
template <> struct Elem<_Float16> {
    static constexpr int E = 8;
    typedef _Float16 V __attribute__((ext_vector_type(8)));
    struct __attribute__((packed, aligned(2))) Loose { uint32_t w[4]; };
};
template <typename T> using Vec = typename Elem<T>::V;

template <typename T>
__device__ __forceinline__ Vec<T> load_vec(const T* p) {
    return __builtin_bit_cast(Vec<T>, *reinterpret_cast<const typename Elem<T>::Loose*>(p));
}
template <typename T>
__device__ __forceinline__ void store_vec(T* p, Vec<T> v) {
    *reinterpret_cast<typename Elem<T>::Loose*>(p) = __builtin_bit_cast(typename Elem<T>::Loose, v);
}
typedef float v4f_loose __attribute__((ext_vector_type(4), aligned(2)));
template <typename T>
__device__ __forceinline__ void stream_vec(T* p, Vec<T> v) {       // past the caches
    __builtin_nontemporal_store((v4f_loose)__builtin_bit_cast(v4f, v), reinterpret_cast<v4f_loose*>(p));
}
// The first `count` elements of 16 bytes; the others are zero.
template <typename T>
__device__ __forceinline__ Vec<T> load_vec_part(const T* p, int count) {
    if (count >= Elem<T>::E) return load_vec(p);
    Vec<T> v = {};
#pragma unroll
    for (int e = 0; e < Elem<T>::E; ++e)
        if (e < count) v[e] = p[e];
    return v;
}
template <typename T>
__device__ __forceinline__ void store_vec_part(T* p, Vec<T> v, int count) {
    if (count >= Elem<T>::E) {
        store_vec(p, v);
        return;
    }
#pragma unroll
    for (int e = 0; e < Elem<T>::E; ++e)
        if (e < count) p[e] = v[e];
}

inline size_t elem_bytes(int type) { return type == GCN_F32 ? 4 : 2; }
// Count elements, at any address that the type itself is aligned for; those that are not there are zero.
template <typename T, int COUNT> using Elems = T __attribute__((ext_vector_type(COUNT)));
template <typename T, int COUNT>
struct __attribute__((packed, aligned(sizeof(T)))) LooseElems { uint32_t w[COUNT * sizeof(T) / 4]; };
template <int COUNT, typename T>
__device__ __forceinline__ Elems<T, COUNT> load_elems(const T* p, int there) {
    if constexpr (COUNT * sizeof(T) >= 4) {
        if (there >= COUNT) return __builtin_bit_cast(Elems<T, COUNT>, *reinterpret_cast<const LooseElems<T, COUNT>*>(p));
    }
    Elems<T, COUNT> v = {};
#pragma unroll
    for (int e = 0; e < COUNT; ++e)
        if (e < there) v[e] = p[e];
    return v;
}
// The elements of a row of `len` from `along` on, zeros behind the row's end, in two steps, so that nothing waits for the load: `load_near` takes any COUNT elements of
// the row that hold them, one load without a mask, and `settle` moves them to their place.  (An element at a time under masks, each load waits for the one before.)
// For rows of COUNT elements at least: another way for shorter ones beside it, chosen at run time, brings the waits back.
template <int COUNT>
__device__ __forceinline__ int settle_by(int64_t along, int64_t len) {        // 0: nothing to move; COUNT: nothing there
    if (along + COUNT <= len) return 0;
    return along - (len - COUNT) < COUNT ? (int)(along - (len - COUNT)) : COUNT;
}
// (Words, not elements: of 16-bit elements the compiler would take the loaded registers apart at once.)
template <typename T, int COUNT> using Words = uint32_t __attribute__((ext_vector_type(COUNT * sizeof(T) / 4)));
template <int COUNT, typename T>
__device__ __forceinline__ Words<T, COUNT> load_near(const T* row, int64_t along, int64_t len) {
    const int64_t at = along + COUNT <= len ? along : len - COUNT;
    return __builtin_bit_cast(Words<T, COUNT>, *reinterpret_cast<const LooseElems<T, COUNT>*>(row + at));
}
template <int COUNT, typename T>
__device__ __forceinline__ Elems<T, COUNT> settle(Words<T, COUNT> x, int by) {
    constexpr int BYTES = COUNT * sizeof(T);
    if constexpr (BYTES == 8 || BYTES == 16) {
        using Bits = std::conditional_t<BYTES == 8, uint64_t, unsigned __int128>;
        const Bits bits = __builtin_bit_cast(Bits, x) >> ((by < COUNT ? by : 0) * (int)sizeof(T) * 8);
        return __builtin_bit_cast(Elems<T, COUNT>, by < COUNT ? bits : (Bits)0);
    } else {
        const Elems<T, COUNT> y = __builtin_bit_cast(Elems<T, COUNT>, x);
        Elems<T, COUNT> v = {};
#pragma unroll
        for (int e = 0; e < COUNT; ++e)
#pragma unroll
            for (int o = 0; e + o < COUNT; ++o)
                if (by == o) v[e] = y[e + o];
        return v;
    }
}
template <int COUNT, typename T>
__device__ __forceinline__ void store_elems(T* p, const float (&v)[COUNT], int there) {
    Elems<T, COUNT> x;
#pragma unroll
    for (int e = 0; e < COUNT; ++e) x[e] = (T)v[e];
    if (there >= COUNT) {
        *reinterpret_cast<LooseElems<T, COUNT>*>(p) = __builtin_bit_cast(LooseElems<T, COUNT>, x);
        return;
    }
#pragma unroll
    for (int e = 0; e < COUNT; ++e)
        if (e < there) p[e] = x[e];
}
template <int COUNT, typename T>
__device__ __forceinline__ void floats_of(Elems<T, COUNT> x, float (&v)[COUNT]) {
#pragma unroll
    for (int e = 0; e < COUNT; ++e) v[e] = (float)x[e];
}
// 2^x and 1/x by the instructions, each off by a unit in the last place.
constexpr float LOG2E = (float)1.4426950408889634, LOG2E_LOW = (float)(1.4426950408889634 - (double)LOG2E);
__device__ __forceinline__ float power_of_2(float x) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_exp2f(x);
#else
    return 0.f;
#endif
}
__device__ __forceinline__ float inverse(float x) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_rcpf(x);
#else
    return 0.f;
#endif
}
// e^x for elements T.  The argument times log2(e) is rounded, which the power feels as 2^-24 of itself for each unit of the argument: nothing to 16-bit elements, but
// 2^-18 of an fp32 result at -80.  For fp32 elements therefore with what was lost: 2^(t + l) = 2^t (1 + l ln 2) for the small l.  Beyond 2^200 nothing is left of
// it, and infinities have no such rest; NaN stays NaN.  SiLU of 65536 x 128 x 256 in fp32 82.4 us, without the rest 81.1, with expf 84.2; the norms around a block of
// 232965 x 128 118.5, 118.4 and 119.1.
template <typename T>
__device__ __forceinline__ float exp_for(float x) {
    const float t = x * LOG2E;
    if (sizeof(T) == 2) return power_of_2(t);
    const float low = fmaf(x, LOG2E_LOW, fmaf(x, LOG2E, -t));
    return power_of_2(t) * fmaf(fabsf(t) > 200.f ? 0.f : low, 0.69314718055994531f, 1.f);
}
template <typename T>
__device__ __forceinline__ float sigmoid(float z) { return inverse(1.f + exp_for<T>(-z)); }
// Calls f with a value of the element type.
template <typename F>
int by_type(int type, const F& f) {
    if (type == GCN_F32) return f(float());
    if (type == GCN_BF16) return f(__bf16());
    return f(_Float16());
}
inline bool known_type(int type) { return type == GCN_F32 || type == GCN_BF16 || type == GCN_F16; }

}  // namespace gcn
