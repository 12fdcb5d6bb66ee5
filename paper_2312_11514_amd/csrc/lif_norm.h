// The residual's addition, the norm of the sum and its rounding to 8 bits, in one pass over the rows.
//
//   h = residual + x      RMS  h / sqrt(mean h^2 + eps) * w      LAYER  (h - mean h) / sqrt(var h + eps) * w + b      NONE  h
//   8 bits: step = max |y| * (1 / 127) (of the row, or of every `group` elements), code = y / step to the nearest whole number
//
// A workgroup has one row, in registers.  The sums are fp64 and everything else is a fixed chain of fp32 operations, so that codes do not depend on
// how a row is dealt to threads.
#pragma once

#include "lif_rows.h"

namespace lif {

struct NormArgs {
    const char *x, *residual;
    char *total, *out;
    float* scales;
    const float *weight, *bias;
    long long x_stride, residual_stride, total_stride, out_stride, scales_stride;      // elements
    int32_t width, norm, group;                                                        // group: 0 where a row has one scale
    float eps;
};

constexpr int kNormMaxWaves = 16;

// sum over the workgroup, in every thread, in a fixed order.  `slot` holds a double per wave; every call has one of its own.
__device__ __forceinline__ double block_sum(double v, double* slot, int waves) {
    v = wave_sum(v);
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    lds_barrier();
    double s = 0;
    for (int i = 0; i < waves; ++i) s += slot[i];
    return s;
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

// V: pieces of 8 elements that a thread has; EIGHT: codes and scales instead of rows of T
template <typename T, int V, bool EIGHT>
__global__ void k_add_norm(NormArgs a) {
#pragma clang fp contract(off)
    __shared__ double sums[2][kNormMaxWaves];
    __shared__ unsigned largest[kNormMaxWaves];
    const int tid = threadIdx.x, threads = blockDim.x, waves = threads >> 6, width = a.width;
    const long long row = blockIdx.x;
    const T* x = (const T*)a.x + row * a.x_stride;
    float h[V][8];
    typename Eight<T>::Raw xs[V], rs[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int at = 8 * (v * threads + tid);
        if (at < width) {
            xs[v] = Eight<T>::load(x + at);
            if (a.residual) rs[v] = Eight<T>::load((const T*)a.residual + row * a.residual_stride + at);
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const bool in = 8 * (v * threads + tid) < width;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[v][e] = !in ? 0.f : a.residual ? (float)rs[v][e] + (float)xs[v][e] : (float)xs[v][e];
        if (in && a.total) store_eight<T>((T*)a.total + row * a.total_stride + 8 * (v * threads + tid), h[v]);
    }
    if (a.norm != 0) {
        double mean = 0, s = 0;
        if (a.norm == 2) {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) s += (double)h[v][e];
            mean = block_sum(s, sums[0], waves) / width;
            s = 0;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const bool in = 8 * (v * threads + tid) < width;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double d = (double)h[v][e] - mean;
                h[v][e] = (float)d;
                if (in) s += d * d;
            }
        }
        const float inverse = (float)(1.0 / __builtin_sqrt(block_sum(s, sums[1], waves) / width + (double)a.eps));
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = 8 * (v * threads + tid);
            float w[8], b[8];
            if (at < width && a.weight) load_floats8(a.weight + at, w);
            if (at < width && a.bias) load_floats8(a.bias + at, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float y = h[v][e] * inverse;
                if (a.weight) y = y * w[e];
                if (a.bias) y = y + b[e];
                h[v][e] = at < width ? y : 0.f;
            }
        }
    }
    if constexpr (!EIGHT) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = 8 * (v * threads + tid);
            if (at < width) store_eight<T>((T*)a.out + row * a.out_stride + at, h[v]);
        }
    } else {
        unsigned most[V], all = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            most[v] = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) most[v] = max(most[v], magnitude_bits(h[v][e]));
            all = max(all, most[v]);
        }
        if (a.group == 0) all = block_max(all, largest, waves);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = 8 * (v * threads + tid);
            const unsigned top = a.group ? lanes_max(most[v], a.group / 8) : all;
            const float step = grid_step(__builtin_bit_cast(float, top) * (1.f / 127.f)), inverse = 1.f / step;
            unsigned word[2] = {0, 0};
            if (step > 0.f) {
#pragma unroll
                for (int e = 0; e < 8; ++e) word[e >> 2] |= ((unsigned)(int)nearest(h[v][e], step, inverse) & 0xffu) << 8 * (e & 3);
            }
            if (at < width) {
                *reinterpret_cast<u32x2*>(a.out + row * a.out_stride + at) = u32x2{word[0], word[1]};
                if (a.group ? at % a.group == 0 : at == 0) a.scales[row * a.scales_stride + (a.group ? at / a.group : 0)] = step;
            }
        }
    }
}

void launch_add_norm_f32(const NormArgs& a, int rows, hipStream_t s);
void launch_add_norm_f16(const NormArgs& a, int rows, hipStream_t s);
void launch_add_norm_bf16(const NormArgs& a, int rows, hipStream_t s);

template <typename T, int V>
void launch_add_norm_pieces(const NormArgs& a, int rows, int threads, hipStream_t s) {
    if (a.scales) hipLaunchKernelGGL((k_add_norm<T, V, true>), dim3(rows), dim3(threads), 0, s, a);
    else hipLaunchKernelGGL((k_add_norm<T, V, false>), dim3(rows), dim3(threads), 0, s, a);
}
template <typename T>
void launch_add_norm_as(const NormArgs& a, int rows, hipStream_t s) {
    const int pieces = a.width / 8;
    int v = 1;
    while (v < 8 && 1024 * v < pieces) v *= 2;
    const int threads = (pieces + 64 * v - 1) / (64 * v) * 64;
    if (v == 1) launch_add_norm_pieces<T, 1>(a, rows, threads, s);
    else if (v == 2) launch_add_norm_pieces<T, 2>(a, rows, threads, s);
    else if (v == 4) launch_add_norm_pieces<T, 4>(a, rows, threads, s);
    else launch_add_norm_pieces<T, 8>(a, rows, threads, s);
}

}  // namespace lif
