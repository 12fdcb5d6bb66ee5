// The residual's addition, the norm of the sum and its rounding to 8 bits, in one pass over the rows.
//
//   h = residual + x      RMS  h / sqrt(mean h^2 + eps) * w      LAYER  (h - mean h) / sqrt(var h + eps) * w + b      NONE  h
//   8 bits: step = max |y| * (1 / 127) (of the row, or of every `group` elements), code = y / step to the nearest whole number
//
// A workgroup has one row, in registers.  The sums are fp64, in an order that the width alone decides, and everything else is a fixed chain of fp32
// operations: rows and codes do not depend on how many rows there are.
// What bounds it: one row, the launch (1.8 of 2.4 us, 3.2 in 8 bits) and what a wave does one after the other; many, the bytes: 2048 rows of 4544 in bf16 with a
// layer norm 15.9 us where the last-level cache has them, 20 from memory (74 MB, 3.7 TB/s of the 5.2 that a large copy reaches; 8 bits 18.7 and 22); 4096 rows of
// 8192 fp16 48.4 us, 5.5 TB/s; 512 rows of 65536 fp32 with a layer norm 113 us, 4.8 TB/s.  (With everything in fp64 and a mean of 0 taken off in RMS norms, and
// codes that compare each element with the half: 2.8, 3.8, 18.4 and 22.4 us.)
#pragma once

#include "lif_rows.h"

namespace lif {

struct NormArgs {
    const char *x, *residual;
    char *total, *out;
    float* scales;
    const float *weight, *bias;
    long long x_stride, residual_stride, total_stride, out_stride, scales_stride;      // elements
    int32_t rows, width, norm, group;                                                     // group: 0 where a row has one scale
    float eps;
};

constexpr int kNormMaxWaves = 16;

// Which piece of a row a thread has.  With one or two a thread the order of the sums is the same: pieces 32 apart, within each run of 64 of them, are added
// first (two lanes of a wave, or one lane's two), then the 32 sums of a run, and then runs by twos, fours and so on (waves, or the halves of one).
template <int V>
__device__ __forceinline__ int piece_of(int v, int tid, int threads) {
    if constexpr (V == 2) return (tid & ~31) * 2 + 32 * v + (tid & 31);
    return v * threads + tid;
}
// Sum over 16 or 32 lanes, by twos, fours and so on; `lane` is the last of them.
template <int LANES>
__device__ __forceinline__ double lanes_sum_at(double v, int lane) {
    v += dpp_from<0x111, 0xf>(v);                            // row_shr:1, 2, 4, 8
    v += dpp_from<0x112, 0xf>(v);
    v += dpp_from<0x114, 0xf>(v);
    v += dpp_from<0x118, 0xf>(v);
    if constexpr (LANES == 32) v += dpp_from<0x142, 0xa>(v); // row_bcast:15 into rows 1 and 3
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)u, lane), hi = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(u >> 32), lane);
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
// Sum over the workgroup of what threads have of V pieces each, in every thread.  `slot` holds a value per wave; every call has slots of its own.
template <int V>
__device__ __forceinline__ double block_sum(double v, double* slot, int waves) {
    if constexpr (V == 1) v = lanes_sum_at<32>(swap_add<32>(v, v), 31);
    else v = wave_sum(v);
    if (waves == 1) return v;
    const int lane = threadIdx.x & 63;
    if (lane == 0) slot[threadIdx.x >> 6] = v;
    lds_barrier();
    return lanes_sum_at<16>(lane < waves ? slot[lane] : 0., 15);
}
__device__ __forceinline__ unsigned block_max(unsigned v, unsigned* slot, int waves) {
    v = lanes_max(v, 64);
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    lds_barrier();
    unsigned m = 0;
    for (int i = 0; i < waves; ++i) m = max(m, slot[i]);
    return m;
}

// V: pieces of 8 elements that a thread has; EIGHT: codes and scales instead of rows of T; NORM: enum lif_norm
template <typename T, int V, bool EIGHT, int NORM>
__global__ void k_add_norm(NormArgs a) {
#pragma clang fp contract(off)
    __shared__ double sums[2][kNormMaxWaves];
    __shared__ unsigned largest[kNormMaxWaves];
    const int tid = threadIdx.x, threads = blockDim.x, waves = threads >> 6, width = a.width;
    const long long row = blockIdx.x;
    float h[V][8];
    double s = 0, second = 0;                                // of a thread's pieces; with two of them, of the second
    // Pieces on their way at a time: with eight a thread, rows as they come and as fp32 do not fit the 128 registers of 16 waves.
    constexpr int ASKED = V < 8 ? V : sizeof(T) == 4 ? 2 : 4;
#pragma unroll
    for (int first = 0; first < V; first += ASKED) {
        typename Eight<T>::Raw xs[ASKED], rs[ASKED];
#pragma unroll
        for (int u = 0; u < ASKED; ++u) {
            const int at = 8 * piece_of<V>(first + u, tid, threads);
            xs[u] = rs[u] = typename Eight<T>::Raw{};
            if (at < width) {
                xs[u] = Eight<T>::load((const T*)a.x + row * a.x_stride + at);
                if (a.residual) rs[u] = Eight<T>::load((const T*)a.residual + row * a.residual_stride + at);
            }
        }
#pragma unroll
        for (int u = 0; u < ASKED; ++u) {
            const int v = first + u, at = 8 * piece_of<V>(v, tid, threads);
            double& sum = V == 2 && v == 1 ? second : s;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[v][e] = a.residual ? (float)rs[u][e] + (float)xs[u][e] : (float)xs[u][e];
                if constexpr (NORM == 1) sum = __builtin_fma((double)h[v][e], (double)h[v][e], sum);
                if constexpr (NORM == 2) sum += (double)h[v][e];
            }
            if (a.total && at < width) store_eight<T>((T*)a.total + row * a.total_stride + at, h[v]);
        }
        if constexpr (ASKED < V) __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (NORM != 0) {
        if constexpr (NORM == 2) {
            const double mean = block_sum<V>(s + second, sums[0], waves) / width;
            s = second = 0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                double& sum = V == 2 && v == 1 ? second : s;
                // (widened anew: the compiler would keep what the first sum has made of it, in twice the registers)
                if constexpr (V == 8) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(h[v][e]));
                }
                if (8 * piece_of<V>(v, tid, threads) < width) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const double d = (double)h[v][e] - mean;
                        h[v][e] = (float)d;
                        sum = __builtin_fma(d, d, sum);
                    }
                }
            }
        }
        const float inverse = (float)(1.0 / __builtin_sqrt(block_sum<V>(s + second, sums[1], waves) / width + (double)a.eps));
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = 8 * piece_of<V>(v, tid, threads);
            if (at < width) {
                float w[8], b[8];
                if (a.weight) load_floats8(a.weight + at, w);
                if (NORM == 2 && a.bias) load_floats8(a.bias + at, b);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float y = h[v][e] * inverse;
                    if (a.weight) y = y * w[e];
                    if (NORM == 2 && a.bias) y = y + b[e];
                    h[v][e] = y;
                }
            }
        }
    }
    if constexpr (!EIGHT) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = 8 * piece_of<V>(v, tid, threads);
            if (at < width) store_eight<T>((T*)a.out + row * a.out_stride + at, h[v]);
        }
    } else {
        unsigned most[V], all = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            most[v] = 0;
            if (8 * piece_of<V>(v, tid, threads) < width) {
#pragma unroll
                for (int e = 0; e < 8; ++e) most[v] = max(most[v], magnitude_bits(h[v][e]));
            }
            all = max(all, most[v]);
        }
        if (a.group == 0) all = block_max(all, largest, waves);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = 8 * piece_of<V>(v, tid, threads);
            const unsigned top = a.group ? lanes_max(most[v], a.group / 8) : all;
            const float step = grid_step(__builtin_bit_cast(float, top) * (1.f / 127.f));
            float t[8];
            nearest_of(h[v], step, t);
            if (at < width) {
                *reinterpret_cast<u32x2*>(a.out + row * a.out_stride + at) = u32x2{low_bytes(t[0], t[1], t[2], t[3]), low_bytes(t[4], t[5], t[6], t[7])};
                if (a.group ? at % a.group == 0 : at == 0) a.scales[row * a.scales_stride + (a.group ? at / a.group : 0)] = step;
            }
        }
    }
}

void launch_add_norm_f32(const NormArgs& a, hipStream_t s);
void launch_add_norm_f16(const NormArgs& a, hipStream_t s);
void launch_add_norm_bf16(const NormArgs& a, hipStream_t s);

template <typename T, int V>
void launch_add_norm_pieces(const NormArgs& a, int threads, hipStream_t s) {
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a.rows), dim3(threads), 0, s, a); };
    if (a.scales) a.norm == 0 ? go(k_add_norm<T, V, true, 0>) : a.norm == 1 ? go(k_add_norm<T, V, true, 1>) : go(k_add_norm<T, V, true, 2>);
    else a.norm == 0 ? go(k_add_norm<T, V, false, 0>) : a.norm == 1 ? go(k_add_norm<T, V, false, 1>) : go(k_add_norm<T, V, false, 2>);
}
// Few rows last as long as one of them: a piece a thread (one row of 4096, fp16: 2.5 us, with two 2.7, with eight 5.5).  Many are bound by what all threads
// do together, and two pieces a thread share sums and barriers (2048 rows of 4544, bf16, layer norm: 17.5 us with one, 15.9 with two, 17.1 with four).
template <typename T>
void launch_add_norm_as(const NormArgs& a, hipStream_t s) {
    const int pieces = a.width / 8;
    int v = a.rows >= 1024 ? 2 : 1;
    while (v < 8 && 64 * kNormMaxWaves * v < pieces) v *= 2;
    const int threads = (pieces + 64 * v - 1) / (64 * v) * 64;
    if (v == 1) launch_add_norm_pieces<T, 1>(a, threads, s);
    else if (v == 2) launch_add_norm_pieces<T, 2>(a, threads, s);
    else if (v == 4) launch_add_norm_pieces<T, 4>(a, threads, s);
    else launch_add_norm_pieces<T, 8>(a, threads, s);
}

}  // namespace lif
