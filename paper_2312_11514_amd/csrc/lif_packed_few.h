// Products of rows with weights in 4 bits, on the matrix cores.
//
//   y[t, n] = sum over groups g of step[n, g] * sum_{k in g} x[t, k] * (code[n, k] - zero[n, g])   (+ bias[n])
//
// A tile of 16 outputs is one operand, 16 rows of x the other, and the lane (r, q) gets row r of the outputs 4 q .. 4 q + 3: with one row in use of 16 the
// products still cost less than the bytes.  Codes become elements by masks, exactly:
//   fp16  64 + c is a pattern of bits, an instruction further 16 + c; so is 1024 + c or 1024 + 16 c, and minus 1032, or times 1/16 minus 72, that is c - 8
//   bf16  (16 + c) / 2^16 is a pattern of bits
//   fp32  (c - 8) / 2^15 in bf16; x is three bf16 pieces of 8 bits each, which are exact together down to 2^-133
//   8 bits  16 (c - 8), whole numbers throughout
// What is too much comes off with the sum of x: little of it, so that a group's sum is not much smaller than what it is rounded as on its way, by 32 inputs in
// turn without zero points, by the group with them.  Of 11008 inputs with a common offset of a fifth of their spread sums are off by up to 1.0e-6 of them in
// fp16, 1.6e-6 with zero points in groups of 64, 0.8e-6 in groups of 128, where codes are 16 + c; 0.5e-6 in bf16.  One addition after the other in fp32 leaves
// 2.6e-6.  (64 + c and 128 + c throughout: 2.8e-6 and 3.7e-6.  16 + c in fp16 throughout: at most 0.8e-6, but one row by 50001 outputs 22.4 us instead of 21.9.)
// Every group's sum is fp32 (or whole), and its step and zero point are applied to that: weights are not rounded.
// bf16 and fp32 rows, and rows in 8 bits with scales by groups, may be as large as what sums are held in: with 2^-16 or 2^-15 on the codes, or 2^-20 on the
// scales, no group's sum is infinite before its step is applied (128 inputs, zero points to 255), and an output gets the factor back at its end.
//
// What bounds it, up to 16 rows: the launch and one round trip to memory where the matrix is small (one row of 4096 by 4096, fp16: 3.6 us, 1.8 of them the launch,
// 4.8 where no cache has the codes), the bytes where it is large (one row by 50001 outputs, groups of 64 with zero points: 19.2 us, 22.3 from memory, 116 MB at
// 5.2 TB/s of the 6.3 that a plain read reaches), and between them what a tile costs in instructions: a SIMD issues one in four cycles, and the bytes of a tile
// take a compute unit 100 cycles.  So codes take seven or eight instructions for eight of them, the offset of their patterns comes off on the matrix cores, which have
// the time, and groups stand side by side in columns that rows have no use for (with an addition for every two codes and steps group by group 27 us instead of
// 19.9).  16 rows by 11008 outputs: 9.0 us, 11.6 from memory.  fp32 pays for its conversions: 8 rows of 2560 by 10240, groups of 32: 10.5 us for 16 MB.
// Four waves instead of eight: the same for 50001 outputs, 3.7 us instead of 3.55 for 4096; sixteen: 30 and 4.1.
#pragma once

#include <type_traits>

#include "lif_packed.h"
#include "lif_packed_form.h"

namespace lif {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

struct ProductArgs {
    PackedView w;
    const char* x;
    char* out;
    const float* x_scales;           // rows in 8 bits: [rows][x_groups]
    const float* bias;
    long long x_stride, out_stride;  // elements
    int32_t rows, x_groups, out_type;      // x_groups: 1, or as many as a row of the matrix has; out_type: enum lif_dtype
};

// Eight codes as the matrix cores take them: codes() counts kMiddle as 0; all(v) in the place of codes adds v times the sum of x.
template <typename X> struct Operand;
template <> struct Operand<_Float16> {
    static constexpr int kPieces = 1;
    static constexpr float kUp = 1.f;        // what an output is multiplied by at its end
    static constexpr float kMiddle = -64.f;  // the code that counts 0
    typedef f16x8 Word;
    static __device__ __forceinline__ Word codes(unsigned w) {
        auto pair = [](unsigned v) { return (v & 0x00f000f0u) ^ 0x54805480u; };
        return __builtin_bit_cast(Word, u32x4{pair(w << 4), pair(w), pair(w >> 4), pair(w >> 8)});
    }
    static __device__ __forceinline__ Word all(float v) { const _Float16 o = (_Float16)v; return Word{o, o, o, o, o, o, o, o}; }
    static __device__ __forceinline__ f32x4 mul(Word a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Operand<__bf16> {
    static constexpr int kPieces = 1;
    static constexpr float kUp = 65536.f, kMiddle = -16.f;
    typedef bf16x8 Word;
    static __device__ __forceinline__ Word codes(unsigned w) {
        auto pair = [](unsigned v) { return (v & 0x00780078u) ^ 0x39c039c0u; };      // (16 + c) / 2^16
        return __builtin_bit_cast(Word, u32x4{pair(w << 3), pair(w >> 1), pair(w >> 5), pair(w >> 9)});
    }
    static __device__ __forceinline__ Word all(float v) { const __bf16 o = (__bf16)(v / kUp); return Word{o, o, o, o, o, o, o, o}; }
    static __device__ __forceinline__ f32x4 mul(Word a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Operand<float> {
    static constexpr int kPieces = 3;
    static constexpr float kUp = 32768.f, kMiddle = 8.f;
    typedef bf16x8 Word;
    static __device__ __forceinline__ Word codes(unsigned w) {
        // 16 (c - 8) by bytes of both halves: codes 0, 4, 1, 5 and 2, 6, 3, 7
        const int low = (int)(w << 4 & 0xf0f0f0f0u), high = (int)(w & 0xf0f0f0f0u);
        auto byte = [](int v, int i) { return __builtin_bit_cast(unsigned, (float)(signed char)(v >> 8 * i)); };
        auto pair = [&](int v, int i) {                      // no more than 4 bits: the upper halves have all of it; 19 off each exponent, and 0 stays 0
            const unsigned both = __builtin_amdgcn_perm(byte(v, i + 2), byte(v, i), 0x07060302u);
            return __builtin_bit_cast(unsigned, __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, both), u16x2{19 << 7, 19 << 7}));
        };
        return __builtin_bit_cast(Word, u32x4{pair(low, 0), pair(high, 0), pair(low, 1), pair(high, 1)});
    }
    static __device__ __forceinline__ Word all(float v) { const __bf16 o = (__bf16)(v / kUp); return Word{o, o, o, o, o, o, o, o}; }
    static __device__ __forceinline__ f32x4 mul(Word a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Operand<signed char> {    // 16 (c - 8)
    static constexpr float kUp = 0.0625f, kMiddle = 8.f;
};
// an element of a row in 8 bits that has a scale for each group of the weights: divided by kDown when a group's sum is multiplied by it
struct ByGroup {
    signed char code;
};
template <> struct Operand<ByGroup> {
    static constexpr float kUp = 65536.f, kMiddle = 8.f, kDown = 16.f * kUp;
};

// The same for a group and its zero points.
template <typename X, int G, bool ZEROS> struct Near : Operand<X> {};
template <> struct Near<_Float16, 128, true> : Operand<_Float16> {
    static constexpr float kMiddle = -16.f;
    static __device__ __forceinline__ Word codes(unsigned w) {
        auto pair = [](unsigned v) { return (v & 0x03c003c0u) ^ 0x4e004e00u; };
        return __builtin_bit_cast(Word, u32x4{pair(w << 6), pair(w << 2), pair(w >> 2), pair(w >> 6)});
    }
};

// Rows first .. first + n - 1 of x as a buffer: what lies behind the last of them is 0, and so is every row that is not there.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_buffer(const ProductArgs& a, int bytes, int first, int n) {
    const int rows = min(n, a.rows - first);
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(a.x) + (long long)first * a.x_stride * bytes, 0,
                                             (int)((rows - 1) * (int)a.x_stride * bytes + a.w.n_in * bytes), 0x00027000);
}

// sum of eight elements, each divided by kUp before it is added: it may be the largest of its type
__device__ __forceinline__ float sum_of(const f16x8& v) {
    static_assert(Operand<_Float16>::kUp == 1.f, "not divided here");
    const f16x2 one{(_Float16)1.f, (_Float16)1.f};
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_fdot2(f16x2{v[2 * i], v[2 * i + 1]}, one, s, false);
    return s;
}
__device__ __forceinline__ float sum_of(const bf16x8& v) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fmaf((float)v[i], 1.f / Operand<__bf16>::kUp, s);
    return s;
}
__device__ __forceinline__ float sum_of(const Eight<float>::Raw& v) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fmaf(v[i], 1.f / Operand<float>::kUp, s);
    return s;
}

// Rows of x: eight inputs of an fp32 row as three pieces, cut off and not rounded, so that what is left is exact and nothing becomes infinite.
struct Pieces {
    bf16x8 p[3];
};
__device__ __forceinline__ Pieces pieces_of(const Eight<float>::Raw& v) {
    u32x4 w[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = v[2 * i], b = v[2 * i + 1];
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

template <typename X>
__device__ __forceinline__ void store_as(char* out, int type, long long at, float v) {
    if constexpr (sizeof(X) != 1) reinterpret_cast<X*>(out)[at] = (X)v;
    else if (type == 0) reinterpret_cast<float*>(out)[at] = v;
    else if (type == 1) reinterpret_cast<_Float16*>(out)[at] = (_Float16)v;
    else reinterpret_cast<__bf16*>(out)[at] = (__bf16)v;
}

// A tile of the inputs of 4 * MQ rows, of one wave: asked for row by row, 16 lanes each, and handed to the lanes that the matrix cores want them from
// through LDS, where rows are a chunk longer than they need, so that the 16 lanes that read one chunk of 16 rows meet different banks.  (A load whose neighbouring
// lanes are in 16 different rows takes a compute unit 65 cycles, row by row 17: 16 rows by 11008 outputs 14.4 us instead of 9.4.)
template <typename X, int MQ>
struct FewRows {
    static constexpr bool kBytes = sizeof(X) == 1;
    static constexpr int kRows = 4 * MQ, kSlots = 4 / MQ, kChunks = kBytes ? 8 : 16, kPlanes = sizeof(X) == 4 ? 3 : 1;
    struct Buffer {
        u32x4 x[kPlanes][kRows + (kSlots > 1)][kChunks + 1];      // (the last row is zeros)
    };
    std::conditional_t<kBytes, u32x2, typename Eight<std::conditional_t<kBytes, float, X>>::Raw> v[MQ];

    // k: of this lane, inside the row
    __device__ __forceinline__ void ask(const X* const (&from)[MQ], int k) {
#pragma unroll
        for (int i = 0; i < MQ; ++i) {
            if constexpr (kBytes) v[i] = *reinterpret_cast<const u32x2*>(from[i] + k);
            else v[i] = Eight<X>::load(from[i] + k);
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < MQ; ++i) {
            if constexpr (kBytes) v[i] = u32x2{0, 0};
            else v[i] = typename Eight<X>::Raw{};
        }
    }
    __device__ __forceinline__ void put(Buffer& b, int lane) const {
        const int c = lane & 15;
#pragma unroll
        for (int i = 0; i < MQ; ++i) {
            const int row = 4 * i + (lane >> 4);
            if constexpr (kBytes) {
                // word j = c / 4 of the lane group q = c mod 4: half j mod 2 of the chunk 4 (j / 2) + q
                u32x2* at = reinterpret_cast<u32x2*>(&b.x[0][row][4 * (c >> 3) + (c & 3)]) + (c >> 2 & 1);
                *at = u32x2{__builtin_amdgcn_perm(v[i][1], v[i][0], 0x05010400u), __builtin_amdgcn_perm(v[i][1], v[i][0], 0x07030602u)};
            } else if constexpr (sizeof(X) == 4) {
                const Pieces p = pieces_of(v[i]);
#pragma unroll
                for (int k = 0; k < 3; ++k) b.x[k][row][c] = __builtin_bit_cast(u32x4, p.p[k]);
            } else {
                b.x[0][row][c] = __builtin_bit_cast(u32x4, v[i]);
            }
        }
    }
};

// One workgroup: 16 outputs, up to 4 * MQ rows; its waves take the tiles of the inputs in turn, each with DEPTH of them on their way, and add up in LDS.
// The matrix cores have 16 columns: with 4 or 8 rows the others go to the next groups.  Column r is row r mod 4 MQ of every (4 / MQ)-th group and zero in the
// others', so that the sums of up to four groups stand side by side and get their steps and zero points in one go.
template <typename X, int G, bool ZEROS, int MQ, int DEPTH, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_packed_few(ProductArgs a) {
    constexpr int S = kTileIn / G, PER = 4 / S;              // groups of a tile, words of a group
    using Rows = FewRows<X, MQ>;
    constexpr int SLOTS = Rows::kSlots, ROWS = Rows::kRows;
    constexpr int UNIT = S >= SLOTS ? 1 : SLOTS / S, SETS = S >= SLOTS ? S / SLOTS : 1;     // tiles that share sums; sets of sums of a tile
    static_assert(DEPTH % UNIT == 0, "whole units on their way");
    constexpr bool kBytes = sizeof(X) == 1, kByGroup = std::is_same_v<X, ByGroup>;
    __shared__ typename Rows::Buffer buffers[WAVES];
    __shared__ float part[WAVES][4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    const int tile_out = blockIdx.x, first = blockIdx.y * 16, mine = r & (ROWS - 1), slot = r / ROWS;
    const PackedView& w = a.w;
    const int last = w.in_tiles - 1, tail = w.n_in - 8 - last * kTileIn;
    const char* codes = reinterpret_cast<const char*>(w.codes) + (size_t)tile_out * w.in_tiles * 1024;
    const char* groups = reinterpret_cast<const char*>(w.groups) + (size_t)tile_out * w.n_groups * 64;
    typename Rows::Buffer& buffer = buffers[wave];
    if constexpr (SLOTS > 1) {
#pragma unroll
        for (int p = 0; p < Rows::kPlanes; ++p)
            if (lane <= Rows::kChunks) buffer.x[p][ROWS][lane] = u32x4{0, 0, 0, 0};
    }
    const u32x4* column[SLOTS];                              // chunk q of the row, or of the zeros, by the group's slot
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) column[i] = &buffer.x[0][SLOTS == 1 || slot == i ? mine : ROWS][q];
    constexpr int kPlane = (ROWS + (SLOTS > 1)) * (Rows::kChunks + 1);
    // (of rows behind the last one the last one: their columns count for nothing)
    const X* from[MQ];
#pragma unroll
    for (int i = 0; i < MQ; ++i) from[i] = reinterpret_cast<const X*>(a.x) + (long long)min(first + 4 * i + (lane >> 4), a.rows - 1) * a.x_stride;
    const float* scales = kByGroup ? a.x_scales + (long long)min(first + mine, a.rows - 1) * a.x_groups : nullptr;

    float y[4] = {0.f, 0.f, 0.f, 0.f};
    u32x4 tile[DEPTH], gw[DEPTH / UNIT][SETS];
    float xs[kByGroup ? DEPTH / UNIT : 1][SETS];
    Rows rows[DEPTH];
    auto ask = [&](int d, int it) {
        const int safe = min(it, last);
        tile[d] = reinterpret_cast<const u32x4*>(codes + (size_t)safe * 1024)[lane];
        rows[d].ask(from, safe * kTileIn + min(8 * r, safe == last ? tail : kTileIn));
        if (d % UNIT == 0) {
#pragma unroll
            for (int v = 0; v < SETS; ++v) {
                // the group that this lane's column belongs to
                const int g = UNIT == 1 ? safe * S + v * SLOTS + slot : min(it + (slot / S) * WAVES, last) * S + slot % S;
                gw[d / UNIT][v] = *reinterpret_cast<const u32x4*>(groups + (unsigned)(g * 64 + q * 16));
                if constexpr (kByGroup) xs[d / UNIT][v] = scales[min(g, a.x_groups - 1)];      // (behind the last group: of a step of 0)
            }
        }
    };
    using Acc = std::conditional_t<kBytes, i32x4, f32x4>;
    Acc acc[SETS], sum[SETS];
    auto take = [&](int d, int it) {
        if (it == last && 8 * r > tail) rows[d].clear();
        rows[d].put(buffer, lane);
        lds_wave_fence();
        if (d % UNIT == 0) {
#pragma unroll
            for (int v = 0; v < SETS; ++v) acc[v] = sum[v] = Acc{0, 0, 0, 0};
        }
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int v = UNIT == 1 ? s / SLOTS : 0;
            const u32x4* from_column = column[(d * S + s) % SLOTS];
            if constexpr (kBytes) {
#pragma unroll
                for (int h = 0; h < (PER + 1) / 2; ++h) {
                    const int pair = PER == 1 ? s / 2 : s * PER / 2 + h;       // words 2 pair, 2 pair + 1
                    constexpr unsigned m = 0xf0f0f0f0u;
                    // of a group of 32 the other half of the instruction's inputs counts nothing
                    const bool no0 = PER == 1 && s % 2, no1 = PER == 1 && s % 2 == 0;
                    const unsigned w0 = no0 ? 0u : tile[d][2 * pair], w1 = no1 ? 0u : tile[d][2 * pair + 1];
                    const i32x4 c{(int)(w0 << 4 & m), (int)(w0 & m), (int)(w1 << 4 & m), (int)(w1 & m)};
                    const i32x4 x = __builtin_bit_cast(i32x4, from_column[4 * pair]);
                    acc[v] = __builtin_amdgcn_mfma_i32_16x16x64_i8(c, x, acc[v], 0, 0, 0);
                    if constexpr (ZEROS) {
                        const int o0 = no0 ? 0 : 0x10101010, o1 = no1 ? 0 : 0x10101010;
                        sum[v] = __builtin_amdgcn_mfma_i32_16x16x64_i8(i32x4{o0, o0, o1, o1}, x, sum[v], 0, 0, 0);
                    }
                }
            } else {
                using O = Near<X, G, ZEROS>;
#pragma unroll
                for (int j = s * PER; j < (s + 1) * PER; ++j) {
                    const auto c = O::codes(tile[d][j]);
#pragma unroll
                    for (int p = O::kPieces - 1; p >= 0; --p) {
                        const auto x = __builtin_bit_cast(typename O::Word, from_column[p * kPlane + 4 * j]);
                        acc[v] = O::mul(c, x, acc[v]);
                        if constexpr (ZEROS) sum[v] = O::mul(O::all(1.f), x, sum[v]);
                        else if constexpr (O::kMiddle != 8.f) acc[v] = O::mul(O::all(O::kMiddle - 8.f), x, acc[v]);
                    }
                }
            }
        }
        lds_wave_fence();
    };
    auto finish = [&](int d) {                               // behind the last tile of a unit, d its first one
#pragma unroll
        for (int v = 0; v < SETS; ++v) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned word = gw[d / UNIT][v][i];
                float s = (float)acc[v][i];
                if constexpr (ZEROS) s = __builtin_fmaf(Near<X, G, ZEROS>::kMiddle - zero_of(word), (float)sum[v][i], s);
                if constexpr (kByGroup) s *= xs[d / UNIT][v] * (1.f / Operand<X>::kDown);
                y[i] = __builtin_fmaf(step_of(word), s, y[i]);
            }
        }
    };
    // (loads without branches around them: the compiler waits for all of them where it cannot tell how many are on their way)
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) ask(d, wave + d * WAVES);
    int it = wave;
    for (; it + DEPTH * WAVES <= last; it += DEPTH * WAVES) {
#pragma unroll
        for (int d = 0; d < DEPTH; d += UNIT) {
#pragma unroll
            for (int u = 0; u < UNIT; ++u) take(d + u, it + (d + u) * WAVES);
            finish(d);
#pragma unroll
            for (int u = 0; u < UNIT; ++u) ask(d + u, it + (d + u + DEPTH) * WAVES);
        }
    }
#pragma unroll
    for (int d = 0; d < DEPTH; d += UNIT) {
        if (it + d * WAVES > last) continue;
#pragma unroll
        for (int u = 0; u < UNIT; ++u)
            if (u == 0 || it + (d + u) * WAVES <= last) take(d + u, it + (d + u) * WAVES);
        finish(d);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) part[wave][i][lane] = y[i];
    lds_barrier();
    if (threadIdx.x < 16 * ROWS) {
        const int t = threadIdx.x >> 4, row = first + t, n = threadIdx.x & 15, out = tile_out * kTileOut + n;
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < WAVES; ++k)
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) v += part[k][n & 3][(n >> 2) * 16 + i * ROWS + t];
        if (row < a.rows && out < w.n_out) {
            v *= Operand<X>::kUp;
            if constexpr (kBytes && !kByGroup) v *= a.x_scales[row];
            if (a.bias) v += a.bias[out];
            store_as<X>(a.out, a.out_type, row * a.out_stride + out, v);
        }
    }
}

// per type of the rows; false: there is no such form, nothing was launched
bool launch_product_f32(const ProductArgs& a, PackedForm f, bool zeros, hipStream_t s);
bool launch_product_f16(const ProductArgs& a, PackedForm f, bool zeros, hipStream_t s);
bool launch_product_bf16(const ProductArgs& a, PackedForm f, bool zeros, hipStream_t s);
bool launch_product_i8(const ProductArgs& a, PackedForm f, bool zeros, hipStream_t s);
bool launch_product_i8_groups(const ProductArgs& a, PackedForm f, bool zeros, hipStream_t s);

}  // namespace lif
