// Queries and keys of the new tokens: norm per head and rotation; keys and values into their pages.
//
//   RMS  x / sqrt(mean x^2 + eps) * w      LAYER  (x - mean) / sqrt(var + eps) * w + b      then, of the first r dimensions, pairs
//   (x, y) -> (x cos a - y sin a, x sin a + y cos a) * magnitude with a = position * frequency.
//
// What bounds it: for a few tokens the chain slot -> length -> table entry -> store (three dependent round trips) and the launch; for
// prompts the bytes, each read and written once.
// Queries and keys: a workgroup has one token, and computes its angles once, one pair to a thread, for all heads.  A lane holds 16 bytes of
// a head, a power of two of lanes a head, so the sums of a norm are a few lane exchanges; the other half of a pair (half layout) is a second
// 16-byte load of the same line and not an exchange, since it is normalised with other weights anyway.
// Values: the cache keeps N consecutive tokens of a dimension in 16 bytes.  Written token by token, from workgroups on different XCDs,
// those are N writes of a part of a line each; a workgroup takes the N tokens of a piece together and writes it whole where it has all of them.
// What it measured: one token of 32 heads of 128 3.1 us in a graph (6.5 as called from Python, which is what a launch costs there); 32 prompts of up to
// 64 tokens, 64 heads of 64, bf16, layer norms, half of a head turned: 58 MB in 19.5 us where the last-level cache has them, 23.5 from memory, 2.5 TB/s of
// the 4.8 a large copy reaches (66 us with values token by token and angles per lane).  117 registers in that form leave a compute unit four
// workgroups of 4352, so they come in more than four rounds, each a chain of five round trips.
#pragma once

#include "lif_kv.h"

namespace lif {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
template <> struct Vec<__bf16> {
    using type = bf16x8;
    static constexpr int N = 8;
};

constexpr int kAppendAhead = 4;           // heads that a thread asks for at once

struct AppendArgs {
    const char *q, *k, *v;
    char* q_out;
    long long q_stride, k_stride, v_stride, q_out_stride;      // elements
    const float *q_weight, *q_bias, *k_weight, *k_bias;
    const double* frequencies;
    const int32_t* positions;
    const int32_t* slots;
    int32_t batch, n_tokens, heads, kv_heads, dim, layer, rotary_dim, norm;
    int32_t log_lanes;                         // lanes that share a head: the pieces of 16 bytes, rounded up to a power of two
    int32_t head_blocks, heads_per_block;      // workgroups of a token for its queries and keys, and heads of each
    int32_t pieces, value_blocks;              // pieces of N positions that a batch row's new tokens may lie in, workgroups of a piece
    float eps, magnitude, inv_dim;
};

void launch_append_f16(const KvView& kv, const AppendArgs& a, bool interleaved, hipStream_t s);
void launch_append_bf16(const KvView& kv, const AppendArgs& a, bool interleaved, hipStream_t s);
void launch_append_f32(const KvView& kv, const AppendArgs& a, bool interleaved, hipStream_t s);

// sum over groups of `lanes` lanes (the same number everywhere), in every one of them: register moves, no round trips through the LDS
__device__ __forceinline__ float group_sum(float v, int lanes) {
    if (lanes >= 2) v += dpp_from<0xb1, 0xf>(v);               // pairs swapped
    if (lanes >= 4) v += dpp_from<0x4e, 0xf>(v);               // pairs of pairs
    if (lanes >= 8) v += from_xor<4>(v);
    if (lanes >= 16) v += from_xor<8>(v);
    if (lanes >= 32) v = swap_add<16>(v, v);
    if (lanes >= 64) v = swap_add<32>(v, v);
    return v;
}

// N floats at any float's address
template <int N>
__device__ __forceinline__ void load_floats(const float* from, float (&to)[N]) {
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
    for (int e = 0; e < N; e += 4) {
        const f4 v = *reinterpret_cast<const f4*>(from + e);
#pragma unroll
        for (int j = 0; j < 4; ++j) to[e + j] = v[j];
    }
}

// cos and sin of position * frequency: reduced in fp64, where the product is good to 2^-52 of itself
__device__ __forceinline__ void turn(double position, double frequency, float magnitude, float& c, float& s) {
    const double half_turns = position * frequency * 0.31830988618379067154;       // angle / pi
    const double rest = half_turns - 2.0 * __builtin_rint(0.5 * half_turns);       // -1 .. 1
    sincospif((float)rest, &s, &c);
    c *= magnitude;
    s *= magnitude;
}

// new tokens of batch row i: slot, length, how many
struct NewTokens {
    int slot, length, fresh;
};
__device__ __forceinline__ NewTokens new_tokens(const KvView& kv, const AppendArgs& a, int i) {
    NewTokens t{a.slots ? a.slots[i] : i, 0, 0};
    if ((unsigned)t.slot < (unsigned)kv.max_seqs) {
        t.length = length_of(kv, t.slot);
        t.fresh = min(max(kv.fresh[t.slot], 0), t.length);
    }
    return t;
}

// Values of the positions N p .. N p + N - 1 of a batch row, p counted from the piece of its first new token on; 256 threads, each
// 4 bytes of a token at a time.
template <typename T>
__device__ __forceinline__ void append_values(const KvView& kv, const AppendArgs& a, int i, int unit) {
    using V = typename Vec<T>::type;
    constexpr int N = Vec<T>::N, W = 4 / (int)sizeof(T);       // dimensions in 4 bytes
    const int p = (int)((unsigned)unit / (unsigned)a.value_blocks), block = unit - p * a.value_blocks;
    const int error = kv.st->error;
    const NewTokens n = new_tokens(kv, a, i);
    const int first = n.length - n.fresh, low = (first / N + p) * N;                  // position of the piece's first token
    if (error || n.fresh == 0 || low >= min(n.length, first + a.n_tokens)) return;
    const int page = kv.table[(size_t)n.slot * kv.max_pages + (low >> kv.log_page)], width = a.kv_heads * a.dim;
    if (!page_ok(kv, page)) return;
    const int t0 = low - first, t_end = min(n.fresh, a.n_tokens);                     // token of the piece's first position; negative: an older one
    const T* from = (const T*)a.v + ((long long)i * a.n_tokens + t0) * a.v_stride;
    T* page_at = (T*)kv.v + (((size_t)a.layer * kv.pages + page) * a.kv_heads << kv.log_page) * a.dim;
    const int piece = (low & ((1 << kv.log_page) - 1)) / N;
    for (int c = (block * 256 + (int)threadIdx.x) * W; c < width; c += a.value_blocks * 256 * W) {
        const int h = (int)((unsigned)c / (unsigned)a.dim), d = c - h * a.dim;
        T* to = page_at + ((size_t)h << kv.log_page) * a.dim + (size_t)(piece * a.dim + d) * N;
        unsigned w[N];
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = t0 + e >= 0 && t0 + e < t_end ? *reinterpret_cast<const unsigned*>(from + e * a.v_stride + c) : 0u;
        V out[W];
#pragma unroll
        for (int e = 0; e < N; ++e)
#pragma unroll
            for (int j = 0; j < W; ++j) {
                if constexpr (W == 1) out[j][e] = __builtin_bit_cast(T, w[e]);
                else out[j][e] = __builtin_bit_cast(T, (unsigned short)(w[e] >> (16 * j)));
            }
        if (t0 >= 0 && t0 + N <= t_end) {
#pragma unroll
            for (int j = 0; j < W; ++j) *reinterpret_cast<V*>(to + j * N) = out[j];
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (t0 + e >= 0 && t0 + e < t_end) {
#pragma unroll
                    for (int j = 0; j < W; ++j) to[j * N + e] = out[j][e];
                }
        }
    }
}

// grid = (n_tokens * head_blocks workgroups for queries and keys, then pieces * value_blocks for values; batch), block = 256
template <typename T, bool INTERLEAVED, bool NORM>
__global__ __launch_bounds__(256) void k_kv_append(const KvView kv, const AppendArgs a) {
    using V = typename Vec<T>::type;
    constexpr int N = Vec<T>::N;
    __shared__ float cosine[128], sine[128];                   // of the token's pairs
    const int unit = blockIdx.x, i = blockIdx.y;
    if (unit >= a.n_tokens * a.head_blocks) {
        append_values<T>(kv, a, i, unit - a.n_tokens * a.head_blocks);
        return;
    }
    const int t = a.head_blocks == 1 ? unit : (int)((unsigned)unit / (unsigned)a.head_blocks), row = i * a.n_tokens + t, half = a.rotary_dim / 2;
    const int lanes = 1 << a.log_lanes, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.log_lanes, groups = 256 >> a.log_lanes;
    const int d0 = lane * N;
    const bool mine = d0 < a.dim;
    // half layout: all of the lane's dimensions turn or none, all on one side of their pairs
    const bool turns = mine && d0 < a.rotary_dim, upper = !INTERLEAVED && d0 >= half;
    const int d1 = !turns || INTERLEAVED ? d0 : upper ? d0 - half : d0 + half;
    const int first = (unit - t * a.head_blocks) * a.heads_per_block, last = min(first + a.heads_per_block, a.heads + a.kv_heads);
    // The lane's dimensions of its next heads, and those they are paired with.  Of single tokens the first ones are asked for before it is
    // known whether the token is there; of several many may not be, and reading all of them costs more than the wait (from memory 25.7 us against
    // 23.5 in the case above, where half are padding; 32.5 against 30.8 where none is).
    const T *q_row = (const T*)a.q + (size_t)row * a.q_stride, *k_row = (const T*)a.k + (size_t)row * a.k_stride;
    T* q_to = (T*)a.q_out + (size_t)row * a.q_out_stride + d0;
    V own[kAppendAhead], other[kAppendAhead];
    auto ask = [&](int base) {
#pragma unroll
        for (int u = 0; u < kAppendAhead; ++u) {
            const int head = base + u * groups + group;
            own[u] = other[u] = V{};
            if (head < last && mine) {
                const T* from = (head < a.heads ? q_row : k_row) + (unsigned)((head < a.heads ? head : head - a.heads) * a.dim);
                own[u] = *reinterpret_cast<const V*>(from + d0);
                if (!INTERLEAVED && half) other[u] = *reinterpret_cast<const V*>(from + d1);
            }
        }
    };
    if (a.n_tokens == 1) ask(first);
    float w[N], b[N], w1[N], b1[N];                            // norm: weights of these dimensions, of queries or of keys
    bool weights_of = false;
    auto ask_weights = [&](bool key) {
        weights_of = key;
        const float* weight = key ? a.k_weight : a.q_weight;
        const float* bias = a.norm == 2 ? (key ? a.k_bias : a.q_bias) : nullptr;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            w[e] = w1[e] = 1.f;
            b[e] = b1[e] = 0.f;
        }
        if (mine && weight) {
            load_floats(weight + d0, w);
            if (!INTERLEAVED) load_floats(weight + d1, w1);
        }
        if (mine && bias) {
            load_floats(bias + d0, b);
            if (!INTERLEAVED) load_floats(bias + d1, b1);
        }
    };
    if constexpr (NORM) ask_weights(first + group >= a.heads);

    const double frequency = (int)threadIdx.x < half ? a.frequencies[threadIdx.x] : 0.;
    const int error = kv.st->error;
    const NewTokens n = new_tokens(kv, a, i);
    if (error) return;
    const bool there = t < n.fresh;
    const int at = there ? n.length - n.fresh + t : 0, offset = at & ((1 << kv.log_page) - 1);
    int page = -1;
    if (there) page = kv.table[(size_t)n.slot * kv.max_pages + (at >> kv.log_page)];
    if (there && (int)threadIdx.x < half)
        turn(a.positions ? a.positions[row] : at, frequency, a.magnitude, cosine[threadIdx.x], sine[threadIdx.x]);
    __syncthreads();
    if (!there) {                                              // (the whole workgroup)
        for (int head = first + group; head < min(last, a.heads); head += groups)
            if (mine) *reinterpret_cast<V*>(q_to + (unsigned)(head * a.dim)) = V{};
        return;
    }
    if (a.n_tokens > 1) ask(first);
    const bool store = page_ok(kv, page);
    T* k_to = (T*)kv.k + (((((size_t)a.layer * kv.pages + (store ? page : 0)) * a.kv_heads) << kv.log_page) + offset) * a.dim + d0;
    constexpr int PAIRS = INTERLEAVED ? N / 2 : N;
    float c[PAIRS], s[PAIRS];
#pragma unroll
    for (int e = 0; e < PAIRS; ++e) {
        const int pair = INTERLEAVED ? d0 / 2 + e : (upper ? d1 : d0) + e;
        const bool there_is = turns && pair < half;
        c[e] = there_is ? cosine[pair] : 1.f;
        s[e] = there_is ? sine[pair] : 0.f;
    }
    for (int base = first;;) {
#pragma unroll
      for (int u = 0; u < kAppendAhead; ++u) {
        if (base + u * groups >= last) return;                 // (the whole workgroup)
        const int head = base + u * groups + group;
        const bool ok = head < last && mine, key = head >= a.heads;
        float f[N], g[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            f[e] = (float)own[u][e];
            g[e] = (float)other[u][e];
        }
        if constexpr (NORM) {
            if (weights_of != key) ask_weights(key);
            float mean = 0.f;
            if (a.norm == 2) {
#pragma unroll
                for (int e = 0; e < N; ++e) mean += mine ? f[e] : 0.f;
                mean = group_sum(mean, lanes) * a.inv_dim;
            }
            float square = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float v = mine ? f[e] - mean : 0.f;
                square += v * v;
            }
            const float inv = __builtin_amdgcn_rsqf(group_sum(square, lanes) * a.inv_dim + a.eps);      // (good to one unit in the last place)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                f[e] = (f[e] - mean) * inv * w[e] + b[e];
                if (!INTERLEAVED) g[e] = (g[e] - mean) * inv * w1[e] + b1[e];
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
        if (!key)
            *reinterpret_cast<V*>(q_to + (unsigned)(head * a.dim)) = out;
        else if (store)
            *reinterpret_cast<V*>(k_to + (unsigned)(((head - a.heads) * a.dim) << kv.log_page)) = out;
      }
      base += kAppendAhead * groups;
      if (base >= last) return;
      ask(base);
    }
}

template <typename T>
void launch_append_as(const KvView& kv, const AppendArgs& a, bool interleaved, hipStream_t s) {
    const dim3 grid(a.n_tokens * a.head_blocks + a.pieces * a.value_blocks, a.batch);
    auto kernel = a.norm ? (interleaved ? k_kv_append<T, true, true> : k_kv_append<T, false, true>)
                         : (interleaved ? k_kv_append<T, true, false> : k_kv_append<T, false, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, kv, a);
}

}  // namespace lif
