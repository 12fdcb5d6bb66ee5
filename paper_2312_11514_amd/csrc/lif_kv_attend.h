// Attention of the newest tokens of every sequence over the pages of its cache.
//
//   out = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m),   s_j = scale * q . k_j        over the visible positions j
//
// in one pass over keys and values with the running maximum m and sum of the softmax.  The queries that read the same keys, tokens x
// query heads of a key head, are the rows of one item; 16 of them make a tile of the matrix cores:
//
//   S^T [16 positions x 16 rows] = K Q^T        the lane (n, g) = (lane mod 16, lane div 16) gets row n of the positions 4g .. 4g+3
//   O^T [16 dims x 16 rows]     += V^T P^T      where it hands in row n of N consecutive positions, the ones of its group g
//
// Which position a row of a K tile stands for is free: tile a takes position N g + 4 a + i as its row 4 g + i, so that what a lane gets
// out of the first products is what it has to hand into the second.  The weights never leave its registers; keys and values come
// straight from their pages, 16 bytes a lane, in the order the products take them (values are stored with N consecutive positions
// together for that), and no LDS is used before the end.  With one row in use of 16 the products cost a fifteenth of the
// time that the bytes take, so one token of an unshared head takes the same path.
//
// What bounds it: reading keys and values once.  Sequences differ in length, and the host does not know them: the steps of all items, one
// after the other, are dealt to a fixed number of workgroups in equal contiguous runs, each of which works out its own from the
// lengths.  A run that is a whole item writes its output, a part leaves m, the sum and the unscaled output behind, and k_kv_join adds them.
#pragma once

#include "lif_kv.h"
#include "lif_kv_append.h"

namespace lif {

constexpr int kAttendGroups = 512;       // workgroups at most: two per compute unit
constexpr int kAttendWaves = 4;
constexpr float kLog2e = 1.44269504088896340736f;
// added to the exponent of every weight, and taken out of the sums: fp16 has no exponents below 2^-24, and of a long sequence many small
// weights count; none can pass 2^15
constexpr float kWeightBias = 15.f;

struct AttendArgs {
    const char* q;
    char* out;
    float* lse;
    long long q_stride, out_stride;        // elements
    const int32_t* slots;
    const int32_t* starts;
    const unsigned long long* tree;
    float* parts;                          // [2 * groups][rows of a block][dim_pad] sums, unscaled
    float2* stats;                         // [2 * groups][rows of a block] maximum (log2), sum
    int32_t batch, n_tokens, heads, kv_heads, share, dim, layer, window, row_blocks;
    float scale_log2;                      // scale * log2 e
};

void launch_attend_f16(const KvView& kv, const AttendArgs& a, int dim_pad, int tiles, int groups, hipStream_t s);
void launch_attend_bf16(const KvView& kv, const AttendArgs& a, int dim_pad, int tiles, int groups, hipStream_t s);
void launch_attend_f32(const KvView& kv, const AttendArgs& a, int dim_pad, int tiles, int groups, hipStream_t s);

// head_dim rounded up to what the kernels are compiled for
__host__ __device__ __forceinline__ int attend_dim_pad(int dim) { return dim <= 32 ? 32 : dim <= 64 ? 64 : dim <= 96 ? 96 : dim <= 128 ? 128 : 256; }
// tiles of 16 rows that a workgroup takes over the same keys: as many as there are, up to what the registers hold
__host__ __device__ __forceinline__ int attend_tiles(int rows, int dim_pad) {
    const int most = dim_pad > 128 ? 2 : 4;
    const int tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    return tiles < most ? tiles : most;
}

template <typename T> struct Mat;
template <> struct Mat<_Float16> {
    static __device__ __forceinline__ f32x4 mul(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Mat<__bf16> {
    static __device__ __forceinline__ f32x4 mul(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mat<float> {
    static __device__ __forceinline__ f32x4 mul(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};

// max and sum over the four lanes of a row (16 and 32 apart); every one of them gets the result
__device__ __forceinline__ float row_max(float v) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const float w = fmaxf(__builtin_bit_cast(float, (unsigned)a[0]), __builtin_bit_cast(float, (unsigned)a[1]));
    const unsigned x = __builtin_bit_cast(unsigned, w);
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return fmaxf(__builtin_bit_cast(float, (unsigned)b[0]), __builtin_bit_cast(float, (unsigned)b[1]));
}
__device__ __forceinline__ float row_sum(float v) { return swap_add<32>(swap_add<16>(v, v), swap_add<16>(v, v)); }

// factor on sums over the maximum m for the larger maximum `most`: with nothing visible (m = -inf) the sums are zeros, or NaN, which stays
__device__ __forceinline__ float rescale(float m, float most) { return m == most ? 1.f : exp2f(m - most); }

// ---- how the steps are dealt -------------------------------------------------------------------------------------------------
// A batch row of length n, f of its tokens new, has the positions [low, n) to go through, in steps of STEP positions from low rounded down
// to a stage on; a row with nothing to do has one step (it writes zeros).  Its items, key heads x blocks of rows, have the same.
struct RowRange {
    int n, fresh, low;                     // length, new tokens, first position any of them may see
};
__device__ __forceinline__ RowRange row_range(const KvView& kv, const AttendArgs& a, int i) {
    RowRange r{0, 0, 0};
    const int slot = a.slots ? a.slots[i] : i;
    const int start = a.starts ? max(a.starts[i], 0) : 0;
    if ((unsigned)slot < (unsigned)kv.max_seqs) {
        r.n = length_of(kv, slot);
        r.fresh = min(min(max(kv.fresh[slot], 0), r.n), a.n_tokens);
        // (more new tokens than the call has room for: the call's are the first of them)
        const int all = min(max(kv.fresh[slot], 0), r.n);
        r.n -= all - r.fresh;
    }
    r.low = a.window ? max(start, r.n - r.fresh + 1 - a.window) : start;
    if (r.fresh == 0 || r.low >= r.n) r.low = r.n = 0;
    return r;
}
template <int STAGE, int STEP>
__device__ __forceinline__ int row_steps(const RowRange& r) { return max(1, (r.n - r.low / STAGE * STAGE + STEP - 1) / STEP); }

// first[i] = steps of the batch rows before i, first[batch] = all; per key head and block.  By a workgroup of 256.
template <int STAGE, int STEP>
__device__ __forceinline__ void plan_steps(const KvView& kv, const AttendArgs& a, int* first, int* wave_tot) {
    const int per = (a.batch + 255) / 256, i0 = threadIdx.x * per;
    int sum = 0;
    for (int e = 0; e < per; ++e)
        if (i0 + e < a.batch) sum += row_steps<STAGE, STEP>(row_range(kv, a, i0 + e));
    int total;
    int at = block_exclusive_scan<4>(sum, wave_tot, &total);
    for (int e = 0; e < per; ++e)
        if (i0 + e < a.batch) {
            first[i0 + e] = at;
            at += row_steps<STAGE, STEP>(row_range(kv, a, i0 + e));
        }
    if (threadIdx.x == 0) first[a.batch] = total;
    __syncthreads();
}

// ---- the pass over keys and values -------------------------------------------------------------------------------------------
// grid = groups, block = 256.  HDP: head_dim rounded up (FULL: head_dim itself); QT: tiles of 16 rows.
template <typename T, int HDP, int QT, bool FULL>
__global__ __launch_bounds__(256, QT * HDP <= 128 ? 2 : 1) void k_kv_attend(const KvView kv, const AttendArgs a) {
    using V = typename Vec<T>::type;
    constexpr int N = Vec<T>::N;               // elements of 16 bytes; positions of a lane in the second products
    constexpr int TILES = N / 4;               // K tiles of a stage
    constexpr int STAGE = 4 * N, STEP = STAGE * kAttendWaves;
    constexpr int CH = HDP / (4 * N);          // pieces of a key that a lane holds
    constexpr int DT = HDP / 16;               // tiles of dimensions
    constexpr int HALF = HDP > 128 ? 2 : 1;    // the waves' sums meet in LDS, up to 128 dimensions at a time
    constexpr int PITCH = HDP / HALF + 4;
    __shared__ int first[kKvMaxSeqs + 1];
    __shared__ int wave_tot[4];
    __shared__ float wave_max[kAttendWaves][16 * QT], wave_sum_[kAttendWaves][16 * QT];
    __shared__ float sums[kAttendWaves][16][PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, n = lane & 15, g = lane >> 4, dim = FULL ? HDP : a.dim;
    if (kv.st->error) return;
    plan_steps<STAGE, STEP>(kv, a, first, wave_tot);
    const int per_row = a.kv_heads * a.row_blocks;
    const long long all = (long long)first[a.batch] * per_row;
    const long long groups = min((long long)gridDim.x, all);      // (every one of them gets a step)
    if (blockIdx.x >= groups) return;
    long long at = all * blockIdx.x / groups;
    const long long end = all * (blockIdx.x + 1) / groups;
    int i = last_not_above(first, a.batch, (int)(at / per_row));
    bool first_segment = true;

    while (at < end) {
        while (i + 1 < a.batch && (long long)first[i + 1] * per_row <= at) ++i;
        const int steps = first[i + 1] - first[i];
        const long long in_row = at - (long long)first[i] * per_row;
        const int item = (int)(in_row / steps), s0 = (int)(in_row % steps);
        const int s1 = (int)min((long long)steps, s0 + (end - at));
        const int kvh = item / a.row_blocks, rb = item % a.row_blocks;
        const RowRange r = row_range(kv, a, i);
        const int slot = a.slots ? a.slots[i] : i;
        const int start = a.starts ? max(a.starts[i], 0) : 0;
        const int rows = a.n_tokens * a.share, row0 = rb * 16 * QT, base = r.n - r.fresh;

        // the lane's rows: token, what it sees, query
        int token[QT], low[QT];
        unsigned long long seen[QT];
        V q[QT][CH];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const int row = row0 + 16 * t + n;
            token[t] = row / a.share;
            const bool ok = row < rows && token[t] < r.fresh;
            if (!ok) token[t] = -1;
            low[t] = a.window ? max(start, base + token[t] + 1 - a.window) : start;
            seen[t] = 0;
            if (ok && a.tree) seen[t] = a.tree[(size_t)i * a.n_tokens + token[t]];
            const T* from = (const T*)a.q + ((size_t)i * a.n_tokens + (ok ? token[t] : 0)) * a.q_stride +
                            (unsigned)((kvh * a.share + (ok ? row % a.share : 0)) * dim);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int d = (4 * c + g) * N;
                q[t][c] = ok && (FULL || d < dim) ? *reinterpret_cast<const V*>(from + d) : V{};
            }
        }
        f32x4 o[QT][DT];
        float top[QT], off[QT], sum[QT];       // running maximum (log2), what is taken from the exponents, sum of the lane's weights
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            top[t] = -INFINITY;
            off[t] = 0.f;
            sum[t] = 0.f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        const int origin = r.low / STAGE * STAGE;
        const int p_end = min(r.n, origin + s1 * STEP);
        int p = origin + s0 * STEP + wv * STAGE;
        const int32_t* row_table = kv.table + (size_t)((unsigned)slot < (unsigned)kv.max_seqs ? slot : 0) * kv.max_pages;
        // positions in [sure, sure_end) are visible to all rows of the block
        const int sure = a.window ? max(start, r.n - a.window) : start, sure_end = a.tree ? base : base + 1;
        const size_t head_bytes = (size_t)kv.page_bytes / a.kv_heads;
        const size_t layer0 = (size_t)a.layer * kv.pages;
        const int page_mask = (1 << kv.log_page) - 1;

        // whether the lane's row of tile t sees a position
        auto sees = [&](int t, int pos) {
            const int own = pos - base;
            const bool new_ok = a.tree ? own < 64 && (seen[t] >> (own & 63) & 1ull) : own <= token[t];
            return token[t] >= 0 && pos >= low[t] && pos < r.n && (own < 0 || new_ok);
        };

        while (p < p_end) {
            // keys: row n of tile e is position p + N (n div 4) + 4 e + n mod 4; values: positions p + N g ..
            const int kp = p + N * (n >> 2), vp = p + N * g;
            int k_page = row_table[min(kp, r.n - 1) >> kv.log_page], v_page = row_table[min(vp, r.n - 1) >> kv.log_page];
            if (!page_ok(kv, k_page)) k_page = 0;
            if (!page_ok(kv, v_page)) v_page = 0;
            const char* k_at = kv.k + (layer0 + k_page) * kv.page_bytes + kvh * head_bytes;
            const char* v_at = kv.v + (layer0 + v_page) * kv.page_bytes + kvh * head_bytes;
            V k[TILES][CH], v[DT];
#pragma unroll
            for (int e = 0; e < TILES; ++e)
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const int d = (4 * c + g) * N;
                    const T* from = (const T*)k_at + (unsigned)(((kp & page_mask) + 4 * e + (n & 3)) * dim);
                    k[e][c] = *reinterpret_cast<const V*>(from + (FULL || d < dim ? d : 0));
                    if (!FULL && d >= dim) k[e][c] = V{};
                }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const T* from = (const T*)v_at + (unsigned)((vp & page_mask) * dim);
                v[d] = *reinterpret_cast<const V*>(from + (FULL || 16 * d + n < dim ? 16 * d + n : 0) * N);
                if (!FULL && 16 * d + n >= dim) v[d] = V{};
            }
            const bool edge = p < sure || p + STAGE > sure_end;
            if (edge) {                        // what no row may see is not there, whatever it holds
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const bool in = vp + e >= r.low && vp + e < r.n;
#pragma unroll
                    for (int d = 0; d < DT; ++d) v[d][e] = in ? v[d][e] : (T)0.f;
                }
            }
            V w[QT];
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                float x[N];
#pragma unroll
                for (int e = 0; e < TILES; ++e) {
                    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = 0; c < CH; ++c) s = Mat<T>::mul(k[e][c], q[t][c], s);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[4 * e + j] = s[j] * a.scale_log2;
                }
                if (edge) {
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        x[e] = sees(t, vp + e) ? x[e] : -INFINITY;
                    }
                }
                float most = x[0];
#pragma unroll
                for (int e = 1; e < N; ++e) most = fmaxf(most, x[e]);
                if (__any(most > top[t])) {
                    most = fmaxf(row_max(most), top[t]);
                    const float scale = most == -INFINITY ? 1.f : exp2f(top[t] - most);
                    off[t] = most == -INFINITY ? 0.f : most - kWeightBias;
                    top[t] = most;
                    sum[t] *= scale;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[t][d] *= scale;
                }
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float weight = __builtin_amdgcn_exp2f(x[e] - off[t]);
                    sum[t] += weight;
                    w[t][e] = (T)weight;
                }
            }
            // A weight of zero does not keep a value out that is not finite.  Where rows see different positions of a stage, such values are
            // taken out of the products and added to the rows that see them.
            if (edge && r.fresh > 1) {
                bool finite = true;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int e = 0; e < N; ++e) finite = finite && __builtin_isfinite((float)v[d][e]);
                if (__any(!finite)) {
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int e = 0; e < N; ++e) v[d][e] = __builtin_isfinite((float)v[d][e]) ? v[d][e] : (T)0.f;
#pragma unroll 1
                    for (int pos = max(p, r.low); pos < min(p + STAGE, r.n); ++pos) {
                        int page = row_table[pos >> kv.log_page];
                        if (!page_ok(kv, page)) page = 0;
                        const T* from = (const T*)(kv.v + (layer0 + page) * kv.page_bytes + kvh * head_bytes) +
                                        (unsigned)((pos & page_mask) / N * dim * N) + pos % N;
                        bool seen_here[QT];
#pragma unroll
                        for (int t = 0; t < QT; ++t) seen_here[t] = sees(t, pos);
#pragma unroll
                        for (int d = 0; d < DT; ++d)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const int at_dim = 16 * d + 4 * g + j;
                                const float value = (float)from[(FULL || at_dim < dim ? at_dim : 0) * N];
                                const bool add = !__builtin_isfinite(value) && (FULL || at_dim < dim);
#pragma unroll
                                for (int t = 0; t < QT; ++t) o[t][d][j] += add && seen_here[t] ? value : 0.f;
                            }
                    }
                }
            }
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int t = 0; t < QT; ++t) o[t][d] = Mat<T>::mul(v[d], w[t], o[t][d]);
            p += STEP;
        }

        // the waves' sums meet
        __syncthreads();                       // (the last segment's readers are done)
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const float total = row_sum(sum[t]);
            if (g == 0) {
                wave_max[wv][16 * t + n] = top[t];
                wave_sum_[wv][16 * t + n] = total;
            }
        }
        __syncthreads();
        const bool whole = s0 == 0 && s1 == steps;
        const int part_slot = 2 * blockIdx.x + (first_segment ? 0 : 1);
        const int rows_here = min(16 * QT, rows - row0);
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            float most = -INFINITY;
#pragma unroll
            for (int w = 0; w < kAttendWaves; ++w) most = fmaxf(most, wave_max[w][16 * t + n]);
            const float scale = rescale(top[t], most);
#pragma unroll
            for (int half = 0; half < HALF; ++half) {
                if (t || half) __syncthreads();
#pragma unroll
                for (int d = 0; d < DT / HALF; ++d) {
                    *reinterpret_cast<f32x4*>(&sums[wv][n][16 * d + 4 * g]) = o[t][half * (DT / HALF) + d] * scale;
                }
                __syncthreads();
                // thread -> row tid / 16 of the tile, four dimensions at a time
                const int rr = tid >> 4, row = 16 * t + rr;
                float m = -INFINITY, total = 0.f;
#pragma unroll
                for (int w = 0; w < kAttendWaves; ++w) m = fmaxf(m, wave_max[w][row]);
#pragma unroll
                for (int w = 0; w < kAttendWaves; ++w) total += wave_sum_[w][row] * rescale(wave_max[w][row], m);
                if (row < rows_here) {
                    const int abs_row = row0 + row, tok = abs_row / a.share, head = kvh * a.share + abs_row % a.share;
                    const size_t out_row = (size_t)i * a.n_tokens + tok;
                    const bool padding = tok >= r.fresh, none = padding || total == 0.f;
                    const float inv = 1.f / total;
                    for (int d = 4 * (tid & 15); d < HDP / HALF; d += 64) {
                        f32x4 v = *reinterpret_cast<const f32x4*>(&sums[0][rr][d]);
#pragma unroll
                        for (int w = 1; w < kAttendWaves; ++w) v += *reinterpret_cast<const f32x4*>(&sums[w][rr][d]);
                        const int to_dim = half * (HDP / HALF) + d;
                        if (whole) {
                            if (FULL || to_dim < dim) {
                                T* to = (T*)a.out + out_row * a.out_stride + (unsigned)(head * dim + to_dim);
#pragma unroll
                                for (int j = 0; j < 4; ++j) to[j] = none ? (T)0.f : (T)(v[j] * inv);
                            }
                        } else {
                            *reinterpret_cast<f32x4*>(a.parts + ((size_t)part_slot * 16 * QT + row) * HDP + to_dim) = padding ? f32x4{} : v;
                        }
                    }
                    if (half == 0 && (tid & 15) == 0) {
                        if (!whole) a.stats[(size_t)part_slot * 16 * QT + row] = padding ? make_float2(-INFINITY, 0.f) : make_float2(m, total);
                        else if (a.lse) a.lse[out_row * a.heads + head] = none ? -INFINITY : (m - kWeightBias + log2f(total)) / kLog2e;
                    }
                }
            }
        }
        at += s1 - s0;
        first_segment = false;
    }
}

// ---- parts of items are added ------------------------------------------------------------------------------------------------
// grid = (rows of a batch row's items x key heads, batch), block = 256: a workgroup per output row; its waves take the parts in turn.
template <typename T, int HDP, int QT>
__global__ __launch_bounds__(256) void k_kv_join(const KvView kv, const AttendArgs a, int grid) {
    constexpr int N = Vec<T>::N, STAGE = 4 * N, STEP = STAGE * kAttendWaves, PER = (HDP + 63) / 64;
    __shared__ int first[kKvMaxSeqs + 1];
    __shared__ int wave_tot[4];
    __shared__ float wave_m[4], wave_l[4], acc[4][HDP];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    if (kv.st->error) return;
    plan_steps<STAGE, STEP>(kv, a, first, wave_tot);
    const int i = blockIdx.y, rows = a.n_tokens * a.share, kvh = blockIdx.x / rows, abs_row = blockIdx.x % rows;
    const int rb = abs_row / (16 * QT), row = abs_row % (16 * QT);
    const int per_row = a.kv_heads * a.row_blocks, steps = first[i + 1] - first[i];
    const long long all = (long long)first[a.batch] * per_row;
    const long long groups = min((long long)grid, all);
    const long long begin = (long long)first[i] * per_row + (long long)(kvh * a.row_blocks + rb) * steps;
    // the workgroup that has step s: the last one whose first step is not above s
    const int w0 = (int)(((begin + 1) * groups - 1) / all), w1 = (int)(((begin + steps) * groups - 1) / all);
    if (w0 == w1) return;                      // the item was whole
    float m = -INFINITY, l = 0.f, o[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = 0.f;
    for (int w = w0 + wv; w <= w1; w += 4) {
        const size_t slot = 2 * (size_t)w + (all * w / groups >= begin ? 0 : 1), at = slot * 16 * QT + row;
        const float2 s = a.stats[at];
        float v[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) v[e] = lane * PER + e < HDP ? a.parts[at * HDP + lane * PER + e] : 0.f;
        const float most = fmaxf(m, s.x), mine = rescale(m, most), theirs = rescale(s.x, most);
        m = most;
        l = l * mine + s.y * theirs;
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] = o[e] * mine + v[e] * theirs;
    }
    if (lane == 0) {
        wave_m[wv] = m;
        wave_l[wv] = l;
    }
#pragma unroll
    for (int e = 0; e < PER; ++e)
        if (lane * PER + e < HDP) acc[wv][lane * PER + e] = o[e];
    __syncthreads();
    float most = -INFINITY, total = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) most = fmaxf(most, wave_m[w]);
    const int tok = abs_row / a.share, head = kvh * a.share + abs_row % a.share;
    const size_t out_row = (size_t)i * a.n_tokens + tok;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float scale = rescale(wave_m[w], most);
        total += wave_l[w] * scale;
        if (tid < HDP) v += acc[w][tid] * scale;
    }
    if (tid < a.dim) ((T*)a.out)[out_row * a.out_stride + (size_t)head * a.dim + tid] = (T)(total == 0.f ? 0.f : v / total);
    if (tid == 0 && a.lse) a.lse[out_row * a.heads + head] = total == 0.f ? -INFINITY : (most - kWeightBias + log2f(total)) / kLog2e;
}

template <typename T, int HDP, int QT>
void launch_attend(const KvView& kv, const AttendArgs& a, int groups, hipStream_t s) {
    if (a.dim == HDP) hipLaunchKernelGGL((k_kv_attend<T, HDP, QT, true>), dim3(groups), dim3(256), 0, s, kv, a);
    else hipLaunchKernelGGL((k_kv_attend<T, HDP, QT, false>), dim3(groups), dim3(256), 0, s, kv, a);
    if (groups > 1)
        hipLaunchKernelGGL((k_kv_join<T, HDP, QT>), dim3(a.n_tokens * a.heads, a.batch), dim3(256), 0, s, kv, a, groups);
}

template <typename T, int HDP>
void launch_attend_tiles(const KvView& kv, const AttendArgs& a, int tiles, int groups, hipStream_t s) {
    if (tiles == 1) return launch_attend<T, HDP, 1>(kv, a, groups, s);
    if constexpr (HDP <= 128)
        if (tiles == 4) return launch_attend<T, HDP, 4>(kv, a, groups, s);
    launch_attend<T, HDP, 2>(kv, a, groups, s);
}

template <typename T>
void launch_attend_as(const KvView& kv, const AttendArgs& a, int dim_pad, int tiles, int groups, hipStream_t s) {
    switch (dim_pad) {
        case 32: return launch_attend_tiles<T, 32>(kv, a, tiles, groups, s);
        case 64: return launch_attend_tiles<T, 64>(kv, a, tiles, groups, s);
        case 96: return launch_attend_tiles<T, 96>(kv, a, tiles, groups, s);
        case 128: return launch_attend_tiles<T, 128>(kv, a, tiles, groups, s);
        default: return launch_attend_tiles<T, 256>(kv, a, tiles, groups, s);
    }
}

}  // namespace lif
