// Making packed weights, from full ones or from codes as checkpoints hold them, and what they stand for.
#pragma once

#include "lif_packed.h"

namespace lif {

// a word of 8 codes - 8 from two's complements in v[0..8)
__device__ __forceinline__ unsigned word_of(const int (&v)[8]) {
    unsigned w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) w |= ((unsigned)v[i] & 15u) << (4 * (i >> 1) + 16 * (i & 1));
    return w;
}
// 256 threads have a tile: thread (r, c) = (tid / 16, tid mod 16) the inputs 8 c .. 8 c + 7 of output r.
struct TilePlace {
    int row, chunk, at;                                  // output, chunk, input
    bool in;
};
__device__ __forceinline__ TilePlace tile_place(const PackedView& w, int tile) {
    const int ot = tile / w.in_tiles, it = tile - ot * w.in_tiles, r = threadIdx.x >> 4, c = threadIdx.x & 15;
    TilePlace p{ot * kTileOut + r, c, it * kTileIn + 8 * c, false};
    p.in = p.row < w.n_out && p.at < w.n_in;
    return p;
}
// where the word of a thread lies
__device__ __forceinline__ unsigned* tile_word(const PackedView& w, int tile) {
    const int r = threadIdx.x >> 4, c = threadIdx.x & 15;
    return w.codes + (size_t)tile * 256 + ((c & 3) * 16 + r) * 4 + (c >> 2);
}
__device__ __forceinline__ unsigned* group_word(const PackedView& w, int tile, int at) {
    const int ot = tile / w.in_tiles, r = threadIdx.x >> 4;
    return w.groups + ((size_t)ot * w.n_groups + at / w.group) * kTileOut + r;
}

// Symmetric: step = max |w| * (1 / 7), zero 8.  Otherwise step = (max(w, 0) - min(w, 0)) * (1 / 15), zero = -min / step to the nearest whole number.
template <typename T, bool ZEROS>
__global__ __launch_bounds__(256) void k_packed_quantize(PackedView w, const T* __restrict__ from, long long stride, int tiles) {
#pragma clang fp contract(off)
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const TilePlace p = tile_place(w, tile);
        float v[8];
        if (p.in) {
            const auto raw = Eight<T>::load(from + p.row * stride + p.at);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)raw[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.f;
        }
        const int lanes = w.group / 8;
        int code[8];
        float step, zero = 8.f;
        if constexpr (ZEROS) {
            unsigned low = 0, high = 0;                      // magnitudes of the lowest below zero and of the highest above
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (v[e] < 0.f) low = max(low, magnitude_bits(v[e]));
                else high = max(high, magnitude_bits(v[e]));      // (NaN among them)
            }
            low = lanes_max(low, lanes);
            high = lanes_max(high, lanes);
            const float lowest = __builtin_bit_cast(float, low), highest = __builtin_bit_cast(float, high);
            step = grid_step((highest + lowest) * (1.f / 15.f));
            const float inverse = 1.f / step;
            if (step > 0.f) zero = fminf(nearest(lowest, step, inverse), 15.f);
#pragma unroll
            for (int e = 0; e < 8; ++e) code[e] = step > 0.f ? min(max((int)nearest(v[e], step, inverse) + (int)zero, 0), 15) - 8 : (int)zero - 8;
        } else {
            unsigned most = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, magnitude_bits(v[e]));
            most = lanes_max(most, lanes);
            step = grid_step(__builtin_bit_cast(float, most) * (1.f / 7.f));
            const float inverse = 1.f / step;
#pragma unroll
            for (int e = 0; e < 8; ++e) code[e] = step > 0.f ? (int)nearest(v[e], step, inverse) : 0;
        }
        *tile_word(w, tile) = word_of(code);
        if (p.chunk % lanes == 0) *group_word(w, tile, p.at) = (__builtin_bit_cast(unsigned, step) & ~0xffu) | (unsigned)zero;
    }
}

// From codes as checkpoints hold them, two in a byte, the lower input in the lower half.
__global__ __launch_bounds__(256) void k_packed_pack(PackedView w, const unsigned char* __restrict__ codes, const float* __restrict__ scales,
                                                     const unsigned char* __restrict__ zeros, int tiles) {
    const int row_groups = (w.n_in + w.group - 1) / w.group;
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const TilePlace p = tile_place(w, tile);
        unsigned four = 0x88888888u;
        if (p.in) four = *reinterpret_cast<const unsigned*>(codes + (size_t)p.row * (w.n_in / 2) + p.at / 2);
        int code[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) code[e] = (int)(four >> 4 * e & 15u) - 8;
        *tile_word(w, tile) = word_of(code);
        if (p.chunk % (w.group / 8) == 0) {
            const size_t g = (size_t)p.row * row_groups + p.at / w.group;
            float step = 0.f;
            unsigned zero = 8;
            if (p.in) {
                const float s = scales[g];
                step = grid_step(s);
                if (zeros) zero = zeros[g];
            }
            *group_word(w, tile, p.at) = (__builtin_bit_cast(unsigned, step) & ~0xffu) | zero;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_packed_dequantize(PackedView w, T* __restrict__ to, long long stride, int tiles) {
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const TilePlace p = tile_place(w, tile);
        if (!p.in) continue;
        const unsigned word = *tile_word(w, tile), g = *group_word(w, tile, p.at);
        const float step = step_of(g);
        const int zero = (int)(g & 0xffu) - 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = step * (float)(code_of(word, e) - zero);
        store_eight<T>(to + p.row * stride + p.at, v);
    }
}

}  // namespace lif
