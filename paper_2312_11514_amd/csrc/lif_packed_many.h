// Products of many rows with weights in 4 bits (the formula, the operands and their rounding: lif_packed_few.h).
//
// A workgroup has 16 * NT rows and 16 * WN outputs, a tile of 16 to a wave, and WK sets of such waves that take the tiles of the inputs in turn.  The rows go
// through LDS in pieces of 128 inputs, as the matrix cores take them (fp32 cut in three, bytes in the order of the codes), double buffered, with the sums that
// zero points need beside them; the codes go from memory to the registers of the one wave that has use for them, and are unpacked once for 16 * NT rows.
//
// What bounds it: the instructions of a SIMD.  By measurement a matrix instruction takes two issue slots of four cycles of the sixteen that it works, an
// arithmetic one about one, a read of LDS two, and a wave alone has one slot in two; with 64 rows there are four arithmetic instructions and one read to a
// matrix instruction, with 16 rows nine.  1024 rows of 4096 by 11008, fp16: 128 to 139 us, 0.66 to 0.72 PFLOP/s of the 1.37 that a library's large product
// reaches; rows in 8 bits 94 us, 1.0 PFLOP/s; 777 rows by 4096 with zero points 48 to 49 us (0.53; a library's fp16 product of these sizes 42); 48 rows of 4544 in
// 8 bits with scales by groups by 18176 outputs 26 us; 64 rows by 4096 8.1 us, 60 rows of 11008 in groups of 32, bf16, 20 to 21 us.
#pragma once

#include "lif_packed_few.h"

namespace lif {

// The codes as they come, where the sum of x is taken off anyway; in fp16 without zero points c - 8 itself, from which nothing has to be.  (With zero points
// c itself, two instructions more for a pair: 777 rows by 4096 50 us instead of 48.)
template <typename X, int G, bool ZEROS>
struct Exact : Near<X, G, ZEROS> {};
template <int G>
struct Exact<_Float16, G, false> {
    static constexpr float kMiddle = 8.f;
    static __device__ __forceinline__ f16x8 codes(unsigned w) {
        const unsigned u = w >> 8;
        const _Float16 m = (_Float16)-1032.f, l = (_Float16)-72.f;
        const f16x2 minus{m, m}, part{(_Float16)0.0625f, (_Float16)0.0625f}, less{l, l};
        auto low = [&](unsigned v) { return __builtin_bit_cast(f16x2, (v & 0x000f000fu) ^ 0x64086408u) + minus; };
        auto high = [&](unsigned v) { return __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (v & 0x00f000f0u) ^ 0x64806480u), part, less); };
        const f16x2 a = low(w), b = high(w), c = low(u), d = high(u);
        return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
};

// sum over LANES consecutive lanes (1, 4, 8 or 16), in every one of them
template <int LANES, typename V>
__device__ __forceinline__ V lanes_sum(V v) {
    auto add = [&](auto ctrl) {
        constexpr int kCtrl = decltype(ctrl)::value;
        v += __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kCtrl, 0xf, 0xf, false));
    };
    if constexpr (LANES >= 4) {
        add(std::integral_constant<int, 0xb1>());
        add(std::integral_constant<int, 0x4e>());
    }
    if constexpr (LANES >= 8) add(std::integral_constant<int, 0x141>());
    if constexpr (LANES >= 16) add(std::integral_constant<int, 0x140>());
    return v;
}

// How 16 * NT rows of X lie in LDS: pieces of 16 bytes, the chunk c of a row at c ^ (row mod CHUNKS), so that the 16 lanes that read one chunk of
// 16 rows meet different banks.  THREADS put them there.
template <typename X, int G, bool SUMS, int NT, int THREADS>
struct Staged {
    static constexpr bool kBytes = sizeof(X) == 1, kByGroup = std::is_same_v<X, ByGroup>;
    static constexpr int kRows = 16 * NT, kChunks = kBytes ? 8 : 16, kPlanes = sizeof(X) == 4 ? 3 : 1, kUnits = kRows * kChunks;
    static constexpr int kEach = (kUnits + THREADS - 1) / THREADS, S = kTileIn / G, kScales = kByGroup ? (S * kRows + THREADS - 1) / THREADS : 1;
    struct Buffer {
        u32x4 x[kPlanes][kRows][kChunks];
        float sum[SUMS ? S : 1][SUMS ? kRows : 1];
        float scale[kByGroup ? S : 1][kByGroup ? kRows : 1];
    };
    // what a thread has on its way
    std::conditional_t<kBytes, u32x4, typename Eight<std::conditional_t<kBytes, float, X>>::Raw> v[kEach];
    float scales[kScales];

    // where a thread's pieces lie in the first tile
    static __device__ __forceinline__ void place(const ProductArgs& a, unsigned (&offset)[kEach], int tid) {
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const int unit = u * THREADS + tid, row = unit / kChunks, c = unit % kChunks;
            offset[u] = (unsigned)row * (unsigned)a.x_stride * sizeof(X) + (kBytes ? 64 * (c >> 2) + 8 * (c & 3) : 8 * c * sizeof(X));
        }
    }
    // (inputs behind the last one are those of the next row: put clears them)
    __device__ __forceinline__ void ask(const ProductArgs& a, __amdgpu_buffer_rsrc_t x, const unsigned (&offset)[kEach], int first, int it, int tid) {
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const int at = (int)(offset[u] + (unsigned)it * (kTileIn * sizeof(X)));
            if constexpr (kBytes) {
                const u32x2 p = __builtin_amdgcn_raw_buffer_load_b64(x, at, 0, 0), n = __builtin_amdgcn_raw_buffer_load_b64(x, at + 32, 0, 0);
                v[u] = u32x4{p[0], p[1], n[0], n[1]};
            } else if constexpr (sizeof(X) == 4) {
                v[u].v[0] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(x, at, 0, 0));
                v[u].v[1] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(x, at + 16, 0, 0));
            } else {
                v[u] = __builtin_bit_cast(typename Eight<X>::Raw, __builtin_amdgcn_raw_buffer_load_b128(x, at, 0, 0));
            }
        }
        if constexpr (kByGroup) {
#pragma unroll
            for (int u = 0; u < kScales; ++u) {
                const int i = u * THREADS + tid, g = it * S + min(i / kRows, S - 1);       // (behind the last group: of a step of 0)
                scales[u] = a.x_scales[(long long)min(first + i % kRows, a.rows - 1) * a.x_groups + min(g, a.x_groups - 1)];
            }
        }
    }
    __device__ __forceinline__ void put(const ProductArgs& a, Buffer& b, int it, int tid) {
        if ((it + 1) * kTileIn > a.w.n_in) {
#pragma unroll
            for (int u = 0; u < kEach; ++u) {
                const int c = (u * THREADS + tid) % kChunks;
                if constexpr (kBytes) {
                    const int k = it * kTileIn + 64 * (c >> 2) + 8 * (c & 3);
                    if (k >= a.w.n_in) v[u][0] = v[u][1] = 0;
                    if (k + 32 >= a.w.n_in) v[u][2] = v[u][3] = 0;
                } else {
                    if (it * kTileIn + 8 * c >= a.w.n_in) v[u] = typename Eight<X>::Raw{};
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const int unit = u * THREADS + tid, row = unit / kChunks, c = unit % kChunks;
            const bool in = kUnits % THREADS == 0 || unit < kUnits;
            const int at = c ^ (row & (kChunks - 1));
            if constexpr (kBytes) {
                const u32x4 x = v[u];
                if (in)
                    b.x[0][row][at] = u32x4{__builtin_amdgcn_perm(x[1], x[0], 0x05010400u), __builtin_amdgcn_perm(x[1], x[0], 0x07030602u),
                                            __builtin_amdgcn_perm(x[3], x[2], 0x05010400u), __builtin_amdgcn_perm(x[3], x[2], 0x07030602u)};
                if constexpr (SUMS) {
                    constexpr int o = 0x10101010;
                    int p = __builtin_amdgcn_sdot4((int)x[1], o, __builtin_amdgcn_sdot4((int)x[0], o, 0, false), false);
                    int n = __builtin_amdgcn_sdot4((int)x[3], o, __builtin_amdgcn_sdot4((int)x[2], o, 0, false), false);
                    if constexpr (G == 32) {
                        p = lanes_sum<4>(p);
                        n = lanes_sum<4>(n);
                        if (in && (c & 3) == 0) b.sum[(c >> 2) * 2][row] = (float)p, b.sum[(c >> 2) * 2 + 1][row] = (float)n;
                    } else {
                        p = lanes_sum<G / 16>(p + n);
                        if (in && c % (G / 16) == 0) b.sum[c / (G / 16)][row] = (float)p;
                    }
                }
            } else {
                if constexpr (sizeof(X) == 4) {
                    const Pieces p = pieces_of(v[u]);
#pragma unroll
                    for (int i = 0; i < 3; ++i)
                        if (in) b.x[i][row][at] = __builtin_bit_cast(u32x4, p.p[i]);
                } else if (in) {
                    b.x[0][row][at] = __builtin_bit_cast(u32x4, v[u]);
                }
                if constexpr (SUMS) {
                    const float s = lanes_sum<G / 8>(sum_of(v[u]));
                    if (in && c % (G / 8) == 0) b.sum[c / (G / 8)][row] = s;
                }
            }
        }
        if constexpr (kByGroup) {
#pragma unroll
            for (int u = 0; u < kScales; ++u) {
                const int i = u * THREADS + tid;
                if (i < S * kRows) b.scale[i / kRows][i % kRows] = scales[u] * (1.f / Operand<X>::kDown);
            }
        }
    }
};

template <typename X, int G, bool ZEROS, int NT, int WN, int WK>
__global__ __launch_bounds__(64 * WN * WK, 4) void k_packed_many(ProductArgs a) {
    constexpr int S = kTileIn / G, PER = 4 / S, THREADS = 64 * WN;
    constexpr bool kBytes = sizeof(X) == 1, kByGroup = std::is_same_v<X, ByGroup>;
    // What codes are off by comes off with the sum of x, once per group, or on the matrix cores, once per word: in groups of one word these have the time.
    constexpr bool kOff = !ZEROS && Exact<X, G, ZEROS>::kMiddle != 8.f, kShift = kOff && PER == 1, kSums = ZEROS || (kOff && !kShift);
    using Stage = Staged<X, G, kSums, NT, THREADS>;
    union Shared {
        typename Stage::Buffer x[WK][2];
        float part[WK > 1 ? WK - 1 : 1][WN][NT * 4][64];
    };
    static_assert(sizeof(Shared) <= 160 * 1024, "LDS of a compute unit");
    __shared__ Shared shared;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    const int set = wave / WN, tid = threadIdx.x - set * THREADS;
    const PackedView& w = a.w;
    const int first = blockIdx.y * (16 * NT), tile_out = blockIdx.x * WN + wave % WN, tiles = (w.n_out + kTileOut - 1) / kTileOut;
    const int last = w.in_tiles - 1, rounds = (w.in_tiles + WK - 1) / WK;
    const size_t safe = min(tile_out, tiles - 1);            // (a wave behind the last output works for nothing, in bounds)
    const char* codes = reinterpret_cast<const char*>(w.codes) + safe * w.in_tiles * 1024;
    const char* groups = reinterpret_cast<const char*>(w.groups) + safe * w.n_groups * 64;
    const __amdgpu_buffer_rsrc_t x = rows_buffer(a, sizeof(X), first, 16 * NT);
    unsigned offset[Stage::kEach];
    Stage::place(a, offset, tid);

    float y[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[t][i] = 0.f;
    Stage stage;
    u32x4 tile[2], gw[2][S];
    auto tile_of = [&](int i) { return min(i * WK + set, last); };
    auto ask = [&](int d, int i) {
        const int it = tile_of(i);
        tile[d] = reinterpret_cast<const u32x4*>(codes + (size_t)it * 1024)[lane];
#pragma unroll
        for (int s = 0; s < S; ++s) gw[d][s] = reinterpret_cast<const u32x4*>(groups + (size_t)(it * S + s) * 64)[q];
    };
    auto ask_rows = [&](int i) { stage.ask(a, x, offset, first, tile_of(i), tid); };
    auto put = [&](int d, int i) { stage.put(a, shared.x[set][d], tile_of(i), tid); };
    auto take = [&](int d) {
        const typename Stage::Buffer& now = shared.x[set][d];
#pragma unroll
        for (int s = 0; s < S; ++s) {
            using Acc = std::conditional_t<kBytes, i32x4, f32x4>;
            Acc acc[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = Acc{0, 0, 0, 0};
            if constexpr (kBytes) {
#pragma unroll
                for (int h = 0; h < (PER + 1) / 2; ++h) {
                    const int pair = PER == 1 ? s / 2 : s * PER / 2 + h;       // words 2 pair, 2 pair + 1
                    constexpr unsigned m = 0xf0f0f0f0u;
                    // of a group of 32 the other half of the instruction's inputs counts nothing
                    const unsigned w0 = PER == 1 && s % 2 ? 0u : tile[d][2 * pair], w1 = PER == 1 && s % 2 == 0 ? 0u : tile[d][2 * pair + 1];
                    const i32x4 c{(int)(w0 << 4 & m), (int)(w0 & m), (int)(w1 << 4 & m), (int)(w1 & m)};
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(c, __builtin_bit_cast(i32x4, now.x[0][16 * t + r][(4 * pair + q) ^ (r & 7)]), acc[t], 0, 0, 0);
                }
            } else {
                using O = Operand<X>;
#pragma unroll
                for (int j = s * PER; j < (s + 1) * PER; ++j) {
                    const typename O::Word c = Exact<X, G, ZEROS>::codes(tile[d][j]);
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int p = O::kPieces - 1; p >= 0; --p) {
                            const auto v = __builtin_bit_cast(typename O::Word, now.x[p][16 * t + r][(4 * j + q) ^ r]);
                            acc[t] = O::mul(c, v, acc[t]);
                            if constexpr (kShift) acc[t] = O::mul(O::all(O::kMiddle - 8.f), v, acc[t]);
                        }
                }
            }
            float step[4], off[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                step[i] = step_of(gw[d][s][i]);
                off[i] = Exact<X, G, ZEROS>::kMiddle - (ZEROS ? zero_of(gw[d][s][i]) : 8.f);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float sum = kSums ? now.sum[s][16 * t + r] : 0.f, xs = kByGroup ? now.scale[s][16 * t + r] : 1.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = (float)acc[t][i];
                    if constexpr (kSums) v = __builtin_fmaf(off[i], sum, v);
                    if constexpr (kByGroup) v *= xs;
                    y[t][i] = __builtin_fmaf(step[i], v, y[t][i]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);               // one group after the other: the sums of several do not fit
        }
    };
    // Codes are asked for two rounds ahead of their use; rows one round ahead of being handed over, and that one round ahead of their use, so that no one waits
    // for LDS at the barrier.  (Without branches around the loads: the compiler waits for all of them where it cannot tell how many are on their way.)
    ask_rows(0);
    ask(0, 0);
    ask(1, 1);
    put(0, 0);
    ask_rows(1);
    for (int i = 0; i < rounds; i += 2) {
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            if (d == 1 && i + 1 >= rounds) break;            // (for all waves)
            lds_barrier();
            put(d ^ 1, i + d + 1);
            ask_rows(i + d + 2);
            if ((i + d) * WK + set <= last) take(d);
            ask(d, i + d + 2);
        }
    }
    if constexpr (WK > 1) {
        lds_barrier();
        if (set > 0) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) shared.part[set - 1][wave % WN][4 * t + i][lane] = y[t][i];
        }
        lds_barrier();
        if (set > 0) return;
#pragma unroll
        for (int k = 0; k + 1 < WK; ++k)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) y[t][i] += shared.part[k][wave % WN][4 * t + i][lane];
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = first + 16 * t + r;
        if (row >= a.rows) continue;
        float up = Operand<X>::kUp;
        if constexpr (kBytes && !kByGroup) up *= a.x_scales[row];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = tile_out * kTileOut + 4 * q + i;
            if (n < w.n_out) store_as<X>(a.out, a.out_type, row * a.out_stride + n, a.bias ? y[t][i] * up + a.bias[n] : y[t][i] * up);
        }
    }
}

}  // namespace lif
