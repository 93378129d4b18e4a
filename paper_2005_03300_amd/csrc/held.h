// Matrices held in 8 and in 4 bits, with a scale for each group of neighbours.
//   checkpoint (8 bits)  64 neighbours of a row; x is held as the whole number c nearest to x / s, -127 to 127, and stands for s c rounded to the element type
//   weights (4 bits)     32, 64 or 128 neighbours of a column; w is held as a sign and the nearest of {0, 1/2, 1, 3/2, 2, 3, 4, 6} times s
// In both s is the smallest bf16 number with which the largest place of the list reaches the largest |x| of the group, so that nothing is cut off.  Of eight bits: products of a scale
// and a place, or the middle between two places, are exact in fp32, and which place is the nearest (of two that are as near the even one) has one answer, however it is computed.
#pragma once
#include "launch_rules.h"
#include "rows.h"

namespace gcn {

constexpr int CHECKPOINT_GROUP = GCN_CHECKPOINT_GROUP;
constexpr float CHECKPOINT_TOP = 127.f, WEIGHT4_TOP = 6.f;

__host__ __device__ constexpr int64_t groups_of(int64_t f, int64_t group) { return (f + group - 1) / group; }

// Weights held in 4 bits, as gcn_linear4_pack lays them out.
struct Weights4 {
    const uint32_t* Q = nullptr;
    const uint16_t* S = nullptr;
    int64_t ldq = 0, lds = 0;
    int group = 0;
    bool gated = false;
};

// A scale's bits as a number, and 2 of them in a word.
__device__ __forceinline__ float scale_value(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }

// The largest scale: TOP times it is the largest number of the type that the places reach (a number beyond that is held as the largest place).
template <typename T>
constexpr uint32_t largest_scale(float top) {
    // 127 2^121, 127 2^9 (65024); 6 x 1.328125 x 2^125, 6 x 1.328125 x 2^13 (65280)
    return top == CHECKPOINT_TOP ? (std::is_same<T, _Float16>::value ? 0x4400u : 0x7c00u) : (std::is_same<T, _Float16>::value ? 0x462au : 0x7e2au);
}
// The bits of the scale of a group whose largest |x| has the bits `most`: the smallest bf16 number, 2^-126 at least, with TOP s >= |x|; NaN where the group holds an infinity or NaN.
template <typename T>
__device__ __forceinline__ uint32_t scale_of(uint32_t most, float top) {
    if (most >= 0x7f800000u) return 0x7fc0u;
    const float a = __builtin_bit_cast(float, most);
    uint32_t s = __builtin_bit_cast(uint32_t, a * (1.f / top)) >> 16;          // at most two steps below it
    s = s < 0x80u ? 0x80u : s;
    s += top * scale_value(s) < a;
    s += top * scale_value(s) < a;
    const uint32_t most_of_type = largest_scale<T>(top);
    return s < most_of_type ? s : most_of_type;
}

// x / s, between -127 and 127, to the nearest whole number: the bits of 1.5 2^23 plus it, whose lowest byte is the code.  `inv`: 1 / s to a few 2^-24.  One correction of the product x inv makes a quotient that has few
// bits exact, so that the middle between two numbers, x = (c + 1/2) s, goes to the even one.  Other quotients are no nearer to a middle than 2^-9 (bf16 x) or 2^-13 (fp16) and the
// correction is off by 2^-17 at most; fp32 numbers can be as near as 2^-25, so there the remainder, which is exact, decides.
template <typename T>
__device__ __forceinline__ uint32_t checkpoint_code(float x, float s, float inv) {
    const float q = x * inv;
    const float t = fmaf(fmaf(-q, s, x), inv, q);
    constexpr float MAGIC = 12582912.f;
    const float m = t + MAGIC;
    if (sizeof(T) == 4) {
        const float c = m - MAGIC, rest = fmaf(-c, s, x);
        return __builtin_bit_cast(uint32_t, fabsf(rest) > 0.5f * s ? m + (rest > 0.f ? 1.f : -1.f) : m);
    }
    return __builtin_bit_cast(uint32_t, m);
}

// E codes of a row of `len`, from `along` on, zeros behind its end; at any address.  As load_near and settle: any E codes of the row that hold them, then moved to their place.
template <int E> struct Codes { uint32_t w[E / 4]; };
template <int E> struct __attribute__((packed, aligned(1))) LooseCodes { uint32_t w[E / 4]; };
template <int E>
__device__ __forceinline__ Codes<E> load_codes(const int8_t* row, int64_t along, int64_t len) {
    Codes<E> c = {};
    if (len >= E) {
        const LooseCodes<E> x = *reinterpret_cast<const LooseCodes<E>*>(row + (along + E <= len ? along : len - E));
        const int by = settle_by<E>(along, len);
        if constexpr (E == 8) {
            uint64_t bits = (uint64_t)x.w[1] << 32 | x.w[0];
            bits = by < E ? bits >> (by * 8) : 0;
            c.w[0] = (uint32_t)bits;
            c.w[1] = (uint32_t)(bits >> 32);
        } else {
            c.w[0] = by < E ? x.w[0] >> (by * 8) : 0;
        }
        return c;
    }
    for (int e = 0; e < E; ++e)
        if (along + e < len) c.w[e / 4] |= (uint32_t)(uint8_t)row[along + e] << (e % 4 * 8);
    return c;
}
template <int E>
__device__ __forceinline__ float code_value(const Codes<E>& c, int e) { return (float)(int8_t)(c.w[e / 4] >> (e % 4 * 8)); }

}  // namespace gcn
