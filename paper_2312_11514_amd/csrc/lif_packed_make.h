// Making packed weights, from full ones or from codes as checkpoints hold them, and what they stand for.
// A tile of 16 outputs x 128 inputs at a time, a word of eight codes to a thread; its group's largest weight by register moves between the lanes.  What bounds it:
// 16384 x 4096 in fp16, the bytes and some arithmetic (38 us, 4.4 TB/s of the 5.2 that a large copy reaches; 47 with each weight compared with the half and codes
// put together one by one); what the weights stand for 29 us, 5.8 TB/s; from codes 22 us, 3.2 TB/s, 4 bytes
// a thread.
#pragma once

#include "lif_packed.h"

namespace lif {

// a word of eight codes - 8, two's complements in the lowest bits
__device__ __forceinline__ unsigned word_of(const float (&t)[8]) {
    const unsigned low = low_bytes(t[0], t[4], t[1], t[5]), high = low_bytes(t[2], t[6], t[3], t[7]);
    return (low & 0x0f0f0f0fu) | (high << 4 & 0xf0f0f0f0u);
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
    typename Eight<T>::Raw next{};
    auto ask = [&](int tile) {
        const TilePlace p = tile_place(w, min(tile, tiles - 1));
        next = Eight<T>::load(from + min(p.row, w.n_out - 1) * stride + min(p.at, w.n_in - 8));
    };
    ask(blockIdx.x);
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const TilePlace p = tile_place(w, tile);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = p.in ? (float)next[e] : 0.f;
        ask(tile + gridDim.x);
        const int lanes = w.group / 8;
        float step, zero = 8.f, t[8];
        if constexpr (ZEROS) {
            // Bits of numbers above zero are ordered as whole numbers, those below zero, as unsigned ones, by their magnitudes; NaN is beyond infinity in both.
            unsigned low = 0;
            int high = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                low = max(low, __builtin_bit_cast(unsigned, v[e]));
                high = max(high, __builtin_bit_cast(int, v[e]));
            }
            low = lanes_max(low, lanes);
            const float highest = __builtin_bit_cast(float, lanes_max((unsigned)high, lanes)), lowest = low >> 31 ? __builtin_bit_cast(float, low & 0x7fffffffu) : 0.f;
            step = grid_step((highest + lowest) * (1.f / 15.f));
            if (step > 0.f) zero = fminf(nearest(lowest, step, 1.f / step), 15.f);
            nearest_of(v, step, t);
            // a code between 0 and 15, and 8 less than that: the whole number between -zero and 15 - zero, and zero - 8 more
#pragma unroll
            for (int e = 0; e < 8; ++e) t[e] = __builtin_amdgcn_fmed3f(t[e], kWhole - zero, kWhole + (15.f - zero)) + (zero - 8.f);
        } else {
            unsigned most = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, magnitude_bits(v[e]));
            most = lanes_max(most, lanes);
            step = grid_step(__builtin_bit_cast(float, most) * (1.f / 7.f));
            nearest_of(v, step, t);
        }
        *tile_word(w, tile) = word_of(t);
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
        // pairs (2 p, 2 p + 1) lie side by side, and go to bits 4 p and 16 + 4 p; a code's two's complement less 8 has its upper bit turned over
        unsigned word = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) word |= (four >> 4 * i & 15u) << (4 * (i >> 1) + 16 * (i & 1));
        *tile_word(w, tile) = word ^ 0x88888888u;
        if (p.chunk % (w.group / 8) == 0) {
            const size_t g = (size_t)p.row * row_groups + p.at / w.group;
            float step = 0.f;
            unsigned zero = 8;
            if (p.in) {
                step = sixteen_bits(scales[g]);              // (no weight is looked for on its grid: small ones are kept)
                if (zeros) zero = zeros[g];
            }
            *group_word(w, tile, p.at) = (__builtin_bit_cast(unsigned, step) & ~0xffu) | zero;
        }
    }
}

// 16 bytes of a row to a thread, so that its neighbours' stores lie beside them (fp32 with 32 bytes a thread in two stores: 18176 x 4544 111 us).
template <typename T>
__global__ __launch_bounds__(256) void k_packed_dequantize(PackedView w, T* __restrict__ to, long long stride, int tiles) {
    constexpr int PER = 16 / sizeof(T), ACROSS = kTileIn / PER;
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int ot = tile / w.in_tiles, it = tile - ot * w.in_tiles;
#pragma unroll
        for (int place = threadIdx.x; place < kTileOut * ACROSS; place += 256) {
            const int r = place / ACROSS, k = place % ACROSS * PER, row = ot * kTileOut + r, at = it * kTileIn + k, c = k / 8;
            if (row >= w.n_out || at >= w.n_in) continue;
            const unsigned word = w.codes[(size_t)tile * 256 + ((c & 3) * 16 + r) * 4 + (c >> 2)];
            const unsigned g = w.groups[((size_t)ot * w.n_groups + at / w.group) * kTileOut + r];
            const float step = step_of(g);
            const int zero = (int)(g & 0xffu) - 8;
            typedef T Some __attribute__((ext_vector_type(PER)));
            Some v;
#pragma unroll
            for (int e = 0; e < PER; ++e) v[e] = (T)(step * (float)(code_of(word, (k & 7) + e) - zero));
            *reinterpret_cast<Some*>(to + row * stride + at) = v;
        }
    }
}

}  // namespace lif
