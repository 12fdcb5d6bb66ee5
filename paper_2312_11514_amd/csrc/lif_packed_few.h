// Products of rows with weights in 4 bits, on the matrix cores.
//
//   y[t, n] = sum over groups g of step[n, g] * sum_{k in g} x[t, k] * (code[n, k] - zero[n, g])   (+ bias[n])
//
// A tile of 16 outputs is one operand, 16 rows of x the other, and the lane (r, q) gets row r of the outputs 4 q .. 4 q + 3: with one row in use of 16 the
// products still cost less than the bytes.  Codes become elements by a mask and, where it takes one, an addition, exactly:
//   fp16  1024 + c and 1024 + 16 c are patterns of bits; minus 1032, or times 1/16 minus 72, is c - 8
//   bf16  (16 + c) / 2^12 is a pattern of bits; what is too much comes off with the zero point, by the sum of x
//   fp32  c - 8 in bf16; x / 2^11 is three bf16 pieces of 8 bits each, which are exact together
//   8 bits  16 (c - 8), whole numbers throughout
// Every group's sum is fp32 (or whole), and its step and zero point are applied to that: weights are not rounded.  bf16 and fp32 rows may be as large as what
// sums are held in: with 2^-12 or 2^-11 on one side no group's sum is infinite before its step is applied, and an output gets the factor back at its end.
#pragma once

#include <type_traits>

#include "lif_packed.h"

namespace lif {

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct ProductArgs {
    PackedView w;
    const char* x;
    char* out;
    const float* x_scales;           // rows in 8 bits: [rows][x_groups]
    const float* bias;
    long long x_stride, out_stride;  // elements
    int32_t rows, x_groups, out_type;      // x_groups: 1, or as many as the matrix has; out_type: enum lif_dtype
};

// Eight inputs of a row as the matrix cores take them, and the codes beside them.
template <typename X> struct Operand;
template <> struct Operand<_Float16> {
    typedef f32x4 Acc;
    static constexpr int kPieces = 1;
    static constexpr float kUp = 1.f;        // what an output is multiplied by at its end
    static constexpr float kMiddle = 8.f;    // the code that counts 0
    typedef f16x8 Word;
    static __device__ __forceinline__ Word codes(unsigned w) {
        const unsigned u = w >> 8;
        const f16x2 minus{(_Float16)-1032.f, (_Float16)-1032.f}, part{(_Float16)0.0625f, (_Float16)0.0625f}, less{(_Float16)-72.f, (_Float16)-72.f};
        auto low = [&](unsigned v) { return __builtin_bit_cast(f16x2, (v & 0x000f000fu) ^ 0x64086408u) + minus; };
        auto high = [&](unsigned v) { return __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (v & 0x00f000f0u) ^ 0x64806480u), part, less); };
        const f16x2 a = low(w), b = high(w), c = low(u), d = high(u);
        return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    static __device__ __forceinline__ Word ones() { const _Float16 o = (_Float16)1.f; return Word{o, o, o, o, o, o, o, o}; }
    static __device__ __forceinline__ Acc mul(Word a, f16x8 b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Operand<__bf16> {
    typedef f32x4 Acc;
    static constexpr int kPieces = 1;
    static constexpr float kUp = 4096.f, kMiddle = -16.f;
    typedef bf16x8 Word;
    static __device__ __forceinline__ Word codes(unsigned w) {
        auto pair = [](unsigned v) { return (v & 0x00780078u) ^ 0x3bc03bc0u; };
        return __builtin_bit_cast(Word, u32x4{pair(w << 3), pair(w >> 1), pair(w >> 5), pair(w >> 9)});
    }
    static __device__ __forceinline__ Word ones() { return __builtin_bit_cast(Word, u32x4{0x39803980u, 0x39803980u, 0x39803980u, 0x39803980u}); }     // 2^-12
    static __device__ __forceinline__ Acc mul(Word a, bf16x8 b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Operand<float> {
    typedef f32x4 Acc;
    static constexpr int kPieces = 3;
    static constexpr float kUp = 2048.f, kMiddle = 8.f;
    typedef bf16x8 Word;
    static __device__ __forceinline__ Word codes(unsigned w) {
        auto pair = [&](int p) {
            const float a = (float)code_of(w, 2 * p), b = (float)code_of(w, 2 * p + 1);      // no more than 4 bits: the upper half has all of it
            return __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, a), 0x07060302u);
        };
        return __builtin_bit_cast(Word, u32x4{pair(0), pair(1), pair(2), pair(3)});
    }
    static __device__ __forceinline__ Word ones() { return __builtin_bit_cast(Word, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u}); }
    static __device__ __forceinline__ Acc mul(Word a, bf16x8 b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

// Rows of x: eight inputs of an fp32 row as three pieces, cut off and not rounded, so that what is left is exact and nothing becomes infinite.
struct Pieces {
    bf16x8 p[3];
};
__device__ __forceinline__ Pieces pieces_of(const Eight<float>::Raw& v) {
    u32x4 w[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = v[2 * i] * (1.f / Operand<float>::kUp), b = v[2 * i + 1] * (1.f / Operand<float>::kUp);
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            const unsigned ua = __builtin_bit_cast(unsigned, a), ub = __builtin_bit_cast(unsigned, b);
            w[j][i] = __builtin_amdgcn_perm(ub, ua, 0x07060302u);
            a -= __builtin_bit_cast(float, ua & 0xffff0000u);
            b -= __builtin_bit_cast(float, ub & 0xffff0000u);
        }
    }
    return Pieces{{__builtin_bit_cast(bf16x8, w[0]), __builtin_bit_cast(bf16x8, w[1]), __builtin_bit_cast(bf16x8, w[2])}};
}

// A tile's products: c[s] += of the sub-group s = word * S / 4, S = 128 / G sub-groups, and the sums of x beside them.
template <typename X>
struct Rows {
    typename Eight<X>::Raw v[4];
    __device__ __forceinline__ void load(const X* row, int at, int n_in, bool in) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (in && at + 32 * j < n_in) v[j] = Eight<X>::load(row + at + 32 * j);
            else v[j] = typename Eight<X>::Raw{};
        }
    }
};
template <>
struct Rows<signed char> {
    u32x2 v[4];
    __device__ __forceinline__ void load(const signed char* row, int at, int n_in, bool in) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (in && at + 32 * j < n_in) v[j] = *reinterpret_cast<const u32x2*>(row + at + 32 * j);
            else v[j] = u32x2{0, 0};
        }
    }
};

template <typename X>
__device__ __forceinline__ void store_as(char* out, int type, long long at, float v) {
    if constexpr (sizeof(X) != 1) reinterpret_cast<X*>(out)[at] = (X)v;
    else if (type == 0) reinterpret_cast<float*>(out)[at] = v;
    else if (type == 1) reinterpret_cast<_Float16*>(out)[at] = (_Float16)v;
    else reinterpret_cast<__bf16*>(out)[at] = (__bf16)v;
}

// One workgroup: 16 outputs, 16 * NT rows; its waves take the tiles of the inputs in turn and add up in LDS.
template <typename X, int G, bool ZEROS, int NT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_packed_few(ProductArgs a) {
    constexpr int S = kTileIn / G, PER = 4 / S;              // groups of a tile, words of a group
    constexpr bool kBytes = sizeof(X) == 1, kSums = ZEROS || (!kBytes && Operand<std::conditional_t<kBytes, float, X>>::kMiddle != 8.f);
    __shared__ float part[WAVES][NT * 4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int tile_out = blockIdx.x, first = blockIdx.y * (16 * NT);
    const PackedView& w = a.w;
    const u32x4* codes = reinterpret_cast<const u32x4*>(w.codes) + (size_t)tile_out * w.in_tiles * 64 + lane;
    const u32x4* groups = reinterpret_cast<const u32x4*>(w.groups) + (size_t)tile_out * w.n_groups * 4 + q;
    float y[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[t][i] = 0.f;
    const X* rows[NT];
    bool in[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = first + 16 * t + r;
        in[t] = row < a.rows;
        rows[t] = reinterpret_cast<const X*>(a.x) + (long long)min(row, a.rows - 1) * a.x_stride;
    }
    for (int it = wave; it < w.in_tiles; it += WAVES) {
        const u32x4 tile = codes[(size_t)it * 64];
        u32x4 gw[S];
#pragma unroll
        for (int s = 0; s < S; ++s) gw[s] = groups[(it * S + s) * 4];
        Rows<X> x[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) x[t].load(rows[t], it * kTileIn + 8 * q, w.n_in, in[t]);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if constexpr (kBytes) {
                i32x4 acc[NT], sum[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t] = sum[t] = i32x4{0, 0, 0, 0};
#pragma unroll
                for (int j = s * PER; j < (s + 1) * PER; j += 2) {
                    // of a group of 32, the second half of the instruction's inputs is 0
                    constexpr unsigned m = 0xf0f0f0f0u;
                    const unsigned w0 = tile[j], w1 = PER == 1 ? 0u : tile[(j + 1) & 3];
                    const i32x4 c{(int)(w0 << 4 & m), (int)(w0 & m), (int)(w1 << 4 & m), (int)(w1 & m)};
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const u32x2 x0 = x[t].v[j], x1 = PER == 1 ? u32x2{0, 0} : x[t].v[(j + 1) & 3];
                        const i32x4 b{(int)__builtin_amdgcn_perm(x0[1], x0[0], 0x05010400u), (int)__builtin_amdgcn_perm(x0[1], x0[0], 0x07030602u),
                                      (int)__builtin_amdgcn_perm(x1[1], x1[0], 0x05010400u), (int)__builtin_amdgcn_perm(x1[1], x1[0], 0x07030602u)};
                        acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(c, b, acc[t], 0, 0, 0);
                        if constexpr (ZEROS) {
                            constexpr int o = 0x10101010;
                            sum[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(i32x4{o, o, o, o}, b, sum[t], 0, 0, 0);
                        }
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float xs = 0.0625f;
                    if (a.x_groups > 1) {
                        const int row = first + 16 * t + r, g = it * S + s;
                        xs *= in[t] && g < a.x_groups ? a.x_scales[(long long)row * a.x_groups + g] : 0.f;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        int v = acc[t][i];
                        if constexpr (ZEROS) v -= ((int)(gw[s][i] & 0xffu) - 8) * sum[t][i];
                        y[t][i] = __builtin_fmaf(step_of(gw[s][i]), (float)v * xs, y[t][i]);
                    }
                }
            } else {
                using O = Operand<X>;
                f32x4 acc[NT], sum[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t] = sum[t] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int j = s * PER; j < (s + 1) * PER; ++j) {
                    const auto c = O::codes(tile[j]);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        if constexpr (O::kPieces == 3) {
                            const Pieces b = pieces_of(x[t].v[j]);
#pragma unroll
                            for (int k = 2; k >= 0; --k) {
                                acc[t] = O::mul(c, b.p[k], acc[t]);
                                if constexpr (kSums) sum[t] = O::mul(O::ones(), b.p[k], sum[t]);
                            }
                        } else {
                            acc[t] = O::mul(c, x[t].v[j], acc[t]);
                            if constexpr (kSums) sum[t] = O::mul(O::ones(), x[t].v[j], sum[t]);
                        }
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float v = acc[t][i];
                        if constexpr (kSums) v = __builtin_fmaf(O::kMiddle - (ZEROS ? zero_of(gw[s][i]) : 8.f), sum[t][i], v);
                        y[t][i] = __builtin_fmaf(step_of(gw[s][i]), v, y[t][i]);
                    }
            }
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[wave][4 * t + i][lane] = y[t][i];
    lds_barrier();
    for (int o = threadIdx.x; o < NT * 256; o += WAVES * 64) {
        const int t = o >> 8, row = first + 16 * t + ((o >> 4) & 15), n = o & 15, out = tile_out * kTileOut + n;
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) v += part[k][4 * t + (n & 3)][(n >> 2) * 16 + ((o >> 4) & 15)];
        if (row < a.rows && out < w.n_out) {
            if constexpr (kBytes) {
                if (a.x_groups == 1) v *= a.x_scales[row];
            } else {
                v *= Operand<X>::kUp;
            }
            if (a.bias) v += a.bias[out];
            store_as<X>(a.out, a.out_type, row * a.out_stride + out, v);
        }
    }
}

void launch_product_f32(const ProductArgs& a, bool zeros, hipStream_t s);
void launch_product_f16(const ProductArgs& a, bool zeros, hipStream_t s);
void launch_product_bf16(const ProductArgs& a, bool zeros, hipStream_t s);
void launch_product_i8(const ProductArgs& a, bool zeros, hipStream_t s);

template <typename X, int G, bool ZEROS>
void launch_product_form(const ProductArgs& a, hipStream_t s) {
    constexpr int NT = 1, WAVES = 8;
    hipLaunchKernelGGL((k_packed_few<X, G, ZEROS, NT, WAVES>), dim3((a.w.n_out + kTileOut - 1) / kTileOut, (a.rows + 16 * NT - 1) / (16 * NT)),
                       dim3(WAVES * 64), 0, s, a);
}
template <typename X>
void launch_product_as(const ProductArgs& a, bool zeros, hipStream_t s) {
    if (a.w.group == 32) zeros ? launch_product_form<X, 32, true>(a, s) : launch_product_form<X, 32, false>(a, s);
    else if (a.w.group == 64) zeros ? launch_product_form<X, 64, true>(a, s) : launch_product_form<X, 64, false>(a, s);
    else zeros ? launch_product_form<X, 128, true>(a, s) : launch_product_form<X, 128, false>(a, s);
}

}  // namespace lif
