// Queries and keys of the new tokens: norm per head and rotation; keys and values into their pages.
//
//   RMS  x / sqrt(mean x^2 + eps) * w      LAYER  (x - mean) / sqrt(var + eps) * w + b      then, of the first r dimensions, pairs
//   (x, y) -> (x cos a - y sin a, x sin a + y cos a) * magnitude with a = position * frequency.
//
// What bounds it: for a few tokens the chain slot -> length -> table entry -> store (three dependent round trips) and the launch; for
// prompts the bytes, each read and written once.  A lane holds 16 bytes of a head, a power of two of lanes a head, so the sums of a norm
// are a few lane exchanges; the other half of a pair (half layout) is a second 16-byte load of the same line and not an exchange,
// since it is normalised with other weights anyway.  The angles belong to the lane's dimensions and the token, not to the head: a wave
// computes them once and goes through its heads with them.
#pragma once

#include "lif_kv.h"

namespace lif {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
template <> struct Vec<__bf16> {
    using type = bf16x8;
    static constexpr int N = 8;
};

struct AppendArgs {
    const char *q, *k, *v;
    char* q_out;
    long long q_stride, k_stride, v_stride, q_out_stride;      // elements
    const float *q_weight, *q_bias, *k_weight, *k_bias;
    const double* frequencies;
    const int32_t* positions;
    const int32_t* slots;
    int32_t n_tokens, heads, kv_heads, dim, layer, rotary_dim, norm, heads_per_block;
    float eps, magnitude;
};

void launch_append_f16(const KvView& kv, const AppendArgs& a, bool interleaved, int rows, int blocks, hipStream_t s);
void launch_append_bf16(const KvView& kv, const AppendArgs& a, bool interleaved, int rows, int blocks, hipStream_t s);
void launch_append_f32(const KvView& kv, const AppendArgs& a, bool interleaved, int rows, int blocks, hipStream_t s);

// lanes that share a head: the pieces of 16 bytes, rounded up to a power of two
__host__ __device__ __forceinline__ int lanes_of_head(int dim, int per_piece) {
    int lanes = 1;
    while (lanes * per_piece < dim) lanes *= 2;
    return lanes;
}

__device__ __forceinline__ float group_sum(float v, int lanes) {
    for (int m = 1; m < lanes; m *= 2) v += __shfl_xor(v, m);
    return v;
}

// cos and sin of 2 pi * position * frequency / (2 pi): reduced in fp64, where position * frequency is good to 2^-52 of itself
__device__ __forceinline__ void turn(double position, double frequency, float magnitude, float& c, float& s) {
    const double half_turns = position * frequency * 0.31830988618379067154;       // angle / pi
    const double rest = half_turns - 2.0 * __builtin_rint(0.5 * half_turns);       // -1 .. 1
    sincospif((float)rest, &s, &c);
    c *= magnitude;
    s *= magnitude;
}

// grid = (rows, blocks of heads), block = 256.  Heads are numbered queries, keys, values; a workgroup takes heads_per_block of them.
template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(256) void k_kv_append(const KvView kv, const AppendArgs a) {
    using V = typename Vec<T>::type;
    constexpr int N = Vec<T>::N;
    const int row = blockIdx.x, i = row / a.n_tokens, t = row % a.n_tokens;
    const int error = kv.st->error;
    const int slot = a.slots ? a.slots[i] : i;
    int length = 0, fresh = 0;
    if ((unsigned)slot < (unsigned)kv.max_seqs) {
        length = length_of(kv, slot);
        fresh = min(max(kv.fresh[slot], 0), length);
    }
    if (error) return;
    const bool there = t < fresh;
    const int at = there ? length - fresh + t : 0;
    int page = -1;
    if (there) page = kv.table[(size_t)slot * kv.max_pages + (at >> kv.log_page)];
    const int offset = at & ((1 << kv.log_page) - 1);
    const bool store = there && page_ok(kv, page);

    const int lanes = lanes_of_head(a.dim, N), lane = threadIdx.x & (lanes - 1), group = threadIdx.x / lanes, groups = 256 / lanes;
    const int d0 = lane * N, half = a.rotary_dim / 2;
    const bool mine = d0 < a.dim;
    // half layout: all of the lane's dimensions turn or none, all on one side of their pairs
    const bool turns = mine && d0 < a.rotary_dim, upper = !INTERLEAVED && d0 >= half;
    const int d1 = !turns || INTERLEAVED ? d0 : upper ? d0 - half : d0 + half;
    constexpr int PAIRS = INTERLEAVED ? N / 2 : N;
    float c[PAIRS], s[PAIRS];
    if (turns) {
        const double position = a.positions ? a.positions[row] : at;
#pragma unroll
        for (int e = 0; e < PAIRS; ++e) {
            const int pair = INTERLEAVED ? d0 / 2 + e : (upper ? d1 : d0) + e;
            c[e] = 1.f;
            s[e] = 0.f;
            if (pair < half) turn(position, a.frequencies[pair], a.magnitude, c[e], s[e]);
        }
    }
    const int first = blockIdx.y * a.heads_per_block, last = min(first + a.heads_per_block, a.heads + 2 * a.kv_heads);
    for (int base = first; base < last; base += groups) {
        const int head = base + group;
        const bool ok = head < last && mine;
        const int kind = head < a.heads ? 0 : head < a.heads + a.kv_heads ? 1 : 2;
        const int h = kind == 0 ? head : kind == 1 ? head - a.heads : head - a.heads - a.kv_heads;
        if (!there) {                                          // (the whole workgroup)
            if (ok && kind == 0)
                *reinterpret_cast<V*>((T*)a.q_out + (size_t)row * a.q_out_stride + (size_t)h * a.dim + d0) = V{};
            continue;
        }
        const T* x = kind == 0 ? (const T*)a.q + (size_t)row * a.q_stride
                               : kind == 1 ? (const T*)a.k + (size_t)row * a.k_stride : (const T*)a.v + (size_t)row * a.v_stride;
        x += (size_t)h * a.dim;
        V own = {}, other = {};
        if (ok) {
            own = *reinterpret_cast<const V*>(x + d0);
            if (!INTERLEAVED && kind != 2) other = *reinterpret_cast<const V*>(x + d1);
        }
        if (kind == 2) {                                       // (lanes of one head go one way; the exchanges below stay inside it)
            if (ok && store) {
                T* to = (T*)kv.v + ((((size_t)a.layer * kv.pages + page) * a.kv_heads + h) << kv.log_page) * a.dim +
                        ((size_t)(offset / N) * a.dim + d0) * N + offset % N;
#pragma unroll
                for (int e = 0; e < N; ++e) to[e * N] = own[e];
            }
            continue;
        }
        float f[N], g[N];                                      // the lane's dimensions, and those they are paired with
#pragma unroll
        for (int e = 0; e < N; ++e) {
            f[e] = (float)own[e];
            g[e] = (float)other[e];
        }
        if (a.norm) {
            float mean = 0.f;
            if (a.norm == 2) {
#pragma unroll
                for (int e = 0; e < N; ++e) mean += f[e];
                mean = group_sum(mean, lanes) / a.dim;
            }
            float square = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float v = mine ? f[e] - mean : 0.f;
                square += v * v;
            }
            const float inv = 1.f / sqrtf(group_sum(square, lanes) / a.dim + a.eps);
            const float* w = kind == 0 ? a.q_weight : a.k_weight;
            const float* b = a.norm == 2 ? (kind == 0 ? a.q_bias : a.k_bias) : nullptr;
            if (mine) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    f[e] = (f[e] - mean) * inv * (w ? w[d0 + e] : 1.f) + (b ? b[d0 + e] : 0.f);
                    if (!INTERLEAVED) g[e] = (g[e] - mean) * inv * (w ? w[d1 + e] : 1.f) + (b ? b[d1 + e] : 0.f);
                }
            }
        }
        V out;
#pragma unroll
        for (int e = 0; e < N; ++e) out[e] = (T)f[e];
        if (turns) {
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int e = 0; e < N; e += 2)
                    if (d0 + e < a.rotary_dim) {
                        out[e] = (T)(f[e] * c[e / 2] - f[e + 1] * s[e / 2]);
                        out[e + 1] = (T)(f[e] * s[e / 2] + f[e + 1] * c[e / 2]);
                    }
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) out[e] = (T)(upper ? g[e] * s[e] + f[e] * c[e] : f[e] * c[e] - g[e] * s[e]);
            }
        }
        if (!ok) continue;
        if (kind == 0)
            *reinterpret_cast<V*>((T*)a.q_out + (size_t)row * a.q_out_stride + (size_t)h * a.dim + d0) = out;
        else if (store)
            *reinterpret_cast<V*>((T*)kv.k + (((((size_t)a.layer * kv.pages + page) * a.kv_heads + h) << kv.log_page) + offset) * a.dim + d0) = out;
    }
}

template <typename T>
void launch_append_as(const KvView& kv, const AppendArgs& a, bool interleaved, int rows, int blocks, hipStream_t s) {
    if (interleaved) hipLaunchKernelGGL((k_kv_append<T, true>), dim3(rows, blocks), dim3(256), 0, s, kv, a);
    else hipLaunchKernelGGL((k_kv_append<T, false>), dim3(rows, blocks), dim3(256), 0, s, kv, a);
}

}  // namespace lif
