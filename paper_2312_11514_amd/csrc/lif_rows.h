// Rows in 8 and 4 bits: what the norm, the packed weights and their products share.
#pragma once

#include "lif_common.h"

namespace lif {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// Eight consecutive elements, as they lie in memory, and as fp32.
template <typename T> struct Eight {
    typedef T Raw __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ Raw load(const T* p) { return *reinterpret_cast<const Raw*>(p); }
};
template <> struct Eight<float> {
    struct Raw { f32x4 v[2]; __device__ __forceinline__ float operator[](int e) const { return v[e >> 2][e & 3]; } };
    static __device__ __forceinline__ Raw load(const float* p) {
        return Raw{{reinterpret_cast<const f32x4*>(p)[0], reinterpret_cast<const f32x4*>(p)[1]}};
    }
};
template <typename T>
__device__ __forceinline__ void store_eight(T* p, const float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        reinterpret_cast<f32x4*>(p)[0] = f32x4{v[0], v[1], v[2], v[3]};
        reinterpret_cast<f32x4*>(p)[1] = f32x4{v[4], v[5], v[6], v[7]};
    } else {
        typename Eight<T>::Raw r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = (T)v[e];
        *reinterpret_cast<typename Eight<T>::Raw*>(p) = r;
    }
}
template <int N>
__device__ __forceinline__ void load_floats8(const float* p, float (&v)[N]) {
    static_assert(N == 8, "eight");
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
    const f4 a = reinterpret_cast<const f4*>(p)[0], b = reinterpret_cast<const f4*>(p)[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
}

// The bits of |v|: as whole numbers they are ordered as the values are, infinity above them and NaN above that, so that a maximum keeps both.
__device__ __forceinline__ unsigned magnitude_bits(float v) { return __builtin_bit_cast(unsigned, v) & 0x7fffffffu; }

// maximum over groups of `lanes` consecutive lanes (4, 8, 16 or 64), in every one of them
template <int CTRL>
__device__ __forceinline__ unsigned max_with(unsigned v) { return max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false)); }
__device__ __forceinline__ unsigned lanes_max(unsigned v, int lanes) {
    v = max_with<0xb1>(v);                                   // pairs swapped
    v = max_with<0x4e>(v);                                   // pairs of pairs
    if (lanes >= 8) v = max_with<0x141>(v);                  // mirrored in 8 lanes
    if (lanes >= 16) v = max_with<0x140>(v);                 // mirrored in 16 lanes
    if (lanes >= 64) {
        v = max(v, (unsigned)__builtin_amdgcn_ds_swizzle((int)v, 0x401f));      // lanes 16 apart
        v = max(v, (unsigned)__shfl_xor((int)v, 32));
    }
    return v;
}

// fp32 to 16 significant bits, halves up; not finite: NaN.
__device__ __forceinline__ float sixteen_bits(float v) {
    const unsigned bits = __builtin_bit_cast(unsigned, v);
    if ((bits & 0x7fffffffu) >= 0x7f7fff80u) return __builtin_nanf("");
    return __builtin_bit_cast(float, (bits + 0x80u) & ~0xffu);
}
// A step of a grid of whole numbers: (k + 1/2) * step is then exact for |k| <= 127, and which whole number is nearest to v / step can be told exactly, by a
// comparison.  Steps below 2^-110, where that would end, are 0: everything is 0.
__device__ __forceinline__ float grid_step(float v) {
    const float s = sixteen_bits(v);
    return __builtin_fabsf(s) < 0x1p-110f ? 0.f : s;
}

// The whole number nearest to v / step, of two the even one, exactly; `inverse` is 1 / step to 2^-22, |v / step| < 128, step > 0.
__device__ __forceinline__ float nearest(float v, float step, float inverse) {
    const float below = __builtin_floorf(v * inverse);       // may be off by one where v is next to a multiple: nearest to the half, all the same
    const float half = (below + 0.5f) * step;
    const bool odd = ((int)below & 1) != 0;
    return v > half || (v == half && odd) ? below + 1.f : below;
}
// The lowest bytes of four.
__device__ __forceinline__ unsigned low_bytes(float a, float b, float c, float d) {
    auto two = [](float x, float y) { return __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, y), __builtin_bit_cast(unsigned, x), 0x0c0c0400u); };
    return __builtin_amdgcn_perm(two(c, d), two(a, b), 0x05040100u);
}
// The same of eight, as t with t - kWhole the whole number and its two's complement in the lowest bits of t.  Nearly always the product with the inverse is
// further from a half than the 2^-15 it may be off by, and adding kWhole rounds it; a wave that has one nearer to a half looks at its own again.
// No step (0, or not a number): 0.
constexpr float kWhole = 12582912.f;         // 1.5 * 2^23: its neighbours are whole numbers
__device__ __forceinline__ void nearest_of(const float (&v)[8], float step, float (&t)[8]) {
#pragma clang fp contract(off)
    const bool some = step > 0.f;
    const float inverse = __builtin_amdgcn_rcpf(step);
    float far = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float q = v[e] * inverse;
        t[e] = q + kWhole;
        far = fmaxf(far, __builtin_fabsf(q - (t[e] - kWhole)));
    }
    if (far > 0.4999f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = nearest(v[e], step, inverse) + kWhole;
    }
    if (!some) {
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = kWhole;
    }
}

}  // namespace lif
