// Weights in 4 bits, a step and a zero point for every group of inputs: layout, packing, and what they stand for.
//
//   weight[n, k] = step[n, k / G] * (code[n, k] - zero[n, k / G]),   code 0..15,   G = 32, 64 or 128 inputs
//
// Layout: tiles of 16 outputs x 128 inputs, 1 KiB each, [output / 16][input / 128][64 lanes][16 bytes], so that a wave asks for a tile with one
// instruction and every lane has what the matrix cores take from it: lane (r, q) = (lane mod 16, lane div 16) holds output r, its word j = 0..3 the inputs
// 32 j + 8 q + i, i = 0..7.  A code is kept as the two's complement of code - 8, i = 2 p at bit 4 p and i = 2 p + 1 at bit 16 + 4 p: one mask takes a pair
// (2 p, 2 p + 1) out as the halves of a register, or four as its bytes.  What lies behind the last input or output is 0 (code 8) with a step of 0.
// Beside them a word for every group, [output / 16][group][16 outputs]: the step in fp32 to 16 significant bits (fp16 and bf16 ones fit exactly), the zero
// point in the 8 bits below.
#pragma once

#include "lif_rows.h"

namespace lif {

constexpr int kTileOut = 16, kTileIn = 128;

// What the kernels know of a matrix.
struct PackedView {
    unsigned* codes;
    unsigned* groups;
    int32_t n_out, n_in, group, in_tiles, n_groups;      // n_groups: of a row, whole tiles
};

__device__ __forceinline__ float step_of(unsigned word) { return __builtin_bit_cast(float, word & ~0xffu); }
__device__ __forceinline__ float zero_of(unsigned word) { return (float)(word & 0xffu); }
__device__ __forceinline__ int code_of(unsigned word, int i) { return (int)(word << (28 - 4 * (i >> 1) - 16 * (i & 1))) >> 28; }

}  // namespace lif
