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
// together for that).  With one row in use of 16 the products cost a fifteenth of the time that the bytes take, so one token of an
// unshared head takes the same path.
//
// Rounding: scores, maxima, sums and outputs are fp32; a weight is rounded to E for the second products, which take nothing wider at their
// rate (relative error of an output 2.3e-4 in fp16, 2e-3 in bf16, half of it the rounding of the output itself; fp32 4e-7).
//
// What bounds it: reading keys and values once, and for short sequences the chain slot -> length -> table entry -> keys -> sums.  Sequences
// differ in length, and the host does not know them: the steps of all items, one after the other, are dealt to a fixed number of
// workgroups in equal contiguous runs, each of which works out its own from the lengths.  A run that is a whole item writes its
// output; of an item's parts every workgroup leaves the maximum, the sum and the unscaled output behind, and the last one to do so adds them.
// What that leaves, with tables about as wide as the sequences: one sequence of 200003, 32 heads of 128 on 8, bf16: 819 MB in 146 us, 5.6 TB/s (a plain
// streaming read reaches 6.3); 64 of up to 8192, fp16: 794 MB in 147 us; 16 of up to 6001 with 5 tokens each: 120 MB in 37.5 us; one of 2048, 32 heads:
// 33.6 MB in 12 us, where a plain read in a launch of its own takes 7.3; one of 77: 5.8 us.  Of those 12 the launch has 1.8, lengths and first table
// entries 2.5, the merge of the waves 0.8, the count of parts 0.7, adding the parts 2.
// Many rows are bound by the matrix cores and the arithmetic on scores between them, with one or two waves a SIMD: 20 tokens of 64 sequences of 8000, 71
// heads of 64 on one, 186 GFLOP in 367 us, 0.51 PFLOP/s (a library's large product reaches 1.16); 64 tokens of 4 sequences of 4000, 32 heads of 128 on 8:
// bf16 49 us, 0.34 PFLOP/s, fp32 180 us, 0.093 of 0.154.
// Registers go to memory in fp32 for dimensions that are not compiled: 188 to 196 bytes a lane for 104, 112 and 120, 312 for 136 to 248 (one token of 8
// sequences of 1000, 16 heads of 112: 52 us, of 128: 31.5), and 12 bytes in bf16 with eight waves for 104 to 120.
#pragma once

#include "lif_kv.h"
#include "lif_kv_append.h"

namespace lif {

constexpr int kAttendUnits = 256;        // compute units
constexpr int kAttendMost = 2048;        // workgroups of a call that may leave parts
constexpr int kAttendFan = 16;           // parts that one workgroup adds at most; of more, such sums are added again (4: one stream of 2048 12.4 -> 14.8 us)
constexpr int kAttendAsk = 8;            // ... and asks for at once (16: no difference beyond 3 %, in both directions)
constexpr float kLog2e = 1.44269504088896340736f;
// Weights are relative to a reference that follows the maximum of their row.  Every change of it multiplies all sums, and a maximum creeps up for most of a
// sequence: with tiles of 64 rows, whose time is arithmetic, it follows only once the maximum is more than this far ahead (as an exponent of two; 60 tokens
// of 64 sequences of 8000, 71 heads on one: 1050 us instead of 1195).  Otherwise at once: the largest weight is then a power of two, and not rounded.
constexpr float attend_slack(int tiles) { return tiles == 4 ? 4.f : 0.f; }

struct AttendArgs {
    const char* q;
    char* out;
    float* lse;
    long long q_stride, out_stride;        // elements
    const int32_t* slots;
    const int32_t* starts;
    const unsigned long long* tree;
    const char* k;                         // of the layer
    const char* v;
    const int32_t* table;
    const int32_t* lengths;
    const int32_t* fresh;
    const int32_t* error;
    float* parts;                          // [2][2 * workgroups][rows of a block][dim_pad + 4] sums, unscaled; maximum and sum behind
                                           // them; of the parts, and of their runs
    unsigned* arrived;                     // [2][2 * workgroups] parts written; zero between calls
    unsigned part_bytes;                   // of `parts`
    unsigned page_bytes, head_bytes;       // of the keys of a page, and of one head of them
    int32_t pages, max_seqs, max_pages, log_page;
    int32_t batch, n_tokens, heads, kv_heads, share, dim, window;
    int32_t units;                         // workgroups of a block of rows
    int32_t round_units, round_steps;      // of them, so many that all blocks' run at once; steps of a block below which only those work
    int32_t row_blocks, block_rows;        // blocks of 16 * tiles rows of an item; rows of a block that are there at most
    float scale_log2;                      // scale * log2 e
};

// per element type and tiles of 16 rows that a wave takes over the same keys; false: there is no such form, nothing was launched
bool launch_attend_f16_1(const AttendArgs& a, int groups, int waves, hipStream_t s);
bool launch_attend_f16_2(const AttendArgs& a, int groups, int waves, hipStream_t s);
bool launch_attend_f16_4(const AttendArgs& a, int groups, int waves, hipStream_t s);
bool launch_attend_bf16_1(const AttendArgs& a, int groups, int waves, hipStream_t s);
bool launch_attend_bf16_2(const AttendArgs& a, int groups, int waves, hipStream_t s);
bool launch_attend_bf16_4(const AttendArgs& a, int groups, int waves, hipStream_t s);
bool launch_attend_f32_1(const AttendArgs& a, int groups, int waves, hipStream_t s);
bool launch_attend_f32_2(const AttendArgs& a, int groups, int waves, hipStream_t s);
bool launch_attend_f32_4(const AttendArgs& a, int groups, int waves, hipStream_t s);

// head_dim rounded up to what the kernels are compiled for
__host__ __device__ __forceinline__ int attend_dim_pad(int dim) {
    return dim <= 32 ? 32 : dim <= 64 ? 64 : dim == 80 ? 80 : dim <= 96 ? 96 : dim <= 128 ? 128 : 256;
}
// most tiles of 16 rows that a wave has registers for: dimensions that are not the compiled ones take some for their bounds
__host__ __device__ __forceinline__ int attend_most_tiles(int dim) { return dim == 256 ? 2 : dim > 128 ? 1 : dim == attend_dim_pad(dim) ? 4 : 2; }

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// c + a b by one instruction of kParts
template <typename T> struct Mat;
template <> struct Mat<_Float16> {
    static constexpr int kParts = 1;
    static constexpr bool kFewExponents = true;
    static __device__ __forceinline__ f32x4 mul(f16x8 a, f16x8 b, f32x4 c, int) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Mat<__bf16> {
    static constexpr int kParts = 1;
    static constexpr bool kFewExponents = false;
    static __device__ __forceinline__ f32x4 mul(bf16x8 a, bf16x8 b, f32x4 c, int) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mat<float> {
    static constexpr int kParts = 4;
    static constexpr bool kFewExponents = false;
    static __device__ __forceinline__ f32x4 mul(f32x4 a, f32x4 b, f32x4 c, int e) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0); }
};

// Added to the exponent of every weight, and taken out of the sums.  fp16 has no exponents below 2^-24, and of a long sequence many small weights count:
// as large as it goes, none passes 2^15 with the slack.  bf16 and fp32 have the exponents, but values as large as what the sums are held in: -k for more
// than 2^(k-1) positions, up to 2^k, so that weights add up to one at most and sums stay below the largest value (with 15 as in fp16 a single
// value above 1.04e34 came out infinite, and 200000 alike above 5e28).
template <typename T>
__device__ __forceinline__ int attend_bias(int tiles, int positions) {
    const int slack = (int)attend_slack(tiles);
    if constexpr (Mat<T>::kFewExponents) return 15 - slack;
    else return (positions > 1 ? __builtin_clz(positions - 1) - 32 : 0) - slack;
}

typedef float f32x2 __attribute__((ext_vector_type(2)));

// load_through of eight bytes
__device__ __forceinline__ f32x2 load_through2(const float* base, unsigned off, unsigned bytes) {
    constexpr int kFlags = 0x00027000, kPast = 1 << 4;           // a raw buffer of dwords; the cache policy bit sc1
    return __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(
                                         __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(base), 0, (int)bytes, kFlags), (int)off, 0, kPast));
}

// whether a wave has 256 registers for its tiles, so that a compute unit has room for eight
__host__ __device__ constexpr bool attend_lean(int dim_pad, bool exact, int tiles, int bytes) {
    return exact ? dim_pad <= 128 && dim_pad * tiles * bytes <= 512 : dim_pad * tiles <= 128;
}
// workgroups that fit a compute unit
__host__ __device__ constexpr int attend_resident(bool lean, int waves) { return lean ? 8 / waves : 1; }

// max and sum over the four lanes of a row (16 and 32 apart); every one of them gets the result
__device__ __forceinline__ float row_max(float v) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const float w = fmaxf(__builtin_bit_cast(float, (unsigned)a[0]), __builtin_bit_cast(float, (unsigned)a[1]));
    const unsigned x = __builtin_bit_cast(unsigned, w);
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return fmaxf(__builtin_bit_cast(float, (unsigned)b[0]), __builtin_bit_cast(float, (unsigned)b[1]));
}
__device__ __forceinline__ float row_sum(float v) {
    const float w = swap_add<16>(v, v);
    return swap_add<32>(w, w);
}

// factor on sums over the maximum m for the larger maximum `most`: with nothing visible (m = -inf) the sums are zeros, or NaN, which stays.
// Maxima are kept as the products give them and scaled after the subtraction, which is exact: of large scores the scaled ones would differ by
// more than their rounding.
__device__ __forceinline__ float rescale(float m, float most, float scale_log2) {
    return m == most ? 1.f : __builtin_amdgcn_exp2f((m - most) * scale_log2);
}

// ---- how the steps are dealt -------------------------------------------------------------------------------------------------
// A batch row of length n, f of its tokens new, has the positions [low, n) to go through, in steps from low rounded down to a stage on; a
// row with nothing to do has one step (it writes zeros).  Its items, one per key head, have the same.  The steps of all items, by
// batch row, key head and position, are dealt to the `units` workgroups of a block of rows in runs:
//   by items    every item in as many equal parts as it takes for none to be longer than the even share (or an eighth more), if that needs
//               no more workgroups than there are: a workgroup then begins and ends one part.  16 sequences of 15 steps of 128, 8 key
//               heads, 512 workgroups: 29.5 us against 31.1 with runs that go on into the next item
//   evenly      else: runs of equal length across the items (many items, or few steps for each workgroup)
// Every wave works this out by itself, 64 batch rows at a time, one to a lane: for up to 64 that is no LDS and no barrier.
struct RowRange {
    int n, fresh, start, slot;             // length, new tokens, first visible position, slot
};
__device__ __forceinline__ int low_of(const RowRange& r, int token, int window) {
    return window ? max(r.start, r.n - r.fresh + token + 1 - window) : r.start;
}
__device__ __forceinline__ RowRange row_range(const AttendArgs& a, int i) {
    RowRange r{0, 0, 0, 0};
    const int slot = a.slots ? a.slots[i] : i;
    if (a.starts) r.start = max(a.starts[i], 0);
    if ((unsigned)slot < (unsigned)a.max_seqs) {
        r.slot = slot;
        const int length = a.lengths[slot], fresh = a.fresh[slot];
        r.n = min(max(length, 0), a.max_pages << a.log_page);
        const int all = min(max(fresh, 0), r.n);
        r.fresh = min(all, a.n_tokens);
        r.n -= all - r.fresh;              // (more new tokens than the call has rows for: the call's are the first of them)
    }
    if (r.fresh == 0 || low_of(r, 0, a.window) >= r.n) r.n = r.start = 0;
    return r;
}

// values that are the same in all lanes, as ones of the wave: what follows from them then runs on the scalar unit
__device__ __forceinline__ int whole_wave(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ RowRange of_lane(const RowRange& r, int lane) {
    return RowRange{__builtin_amdgcn_readlane(r.n, lane), __builtin_amdgcn_readlane(r.fresh, lane), __builtin_amdgcn_readlane(r.start, lane),
                    __builtin_amdgcn_readlane(r.slot, lane)};
}

// a / b rounded up, for 0 < a < 2^24, b > 0: by the reciprocal, a dozen instructions instead of thirty
__device__ __forceinline__ int small_ceil(int a, int b) {
    if (b >= a) return 1;
    const int up = a + b - 1;
    int q = (int)((float)up * __builtin_amdgcn_rcpf((float)b));
    const int rest = up - q * b;
    q += rest >= b ? 1 : 0;
    return rest < 0 ? q - 1 : q;
}

// a / b, the same in all lanes
__device__ __forceinline__ int quotient(int a, int b) { return whole_wave((int)((unsigned)a / (unsigned)b)); }

// 64 batch rows from `first` on, one to a lane
struct RowChunk {
    RowRange range;
    int first, steps, before;              // first batch row; steps per item of the lane's row, and of the rows before it (all of them)
    int after;                             // steps per item up to the chunk's end
};
__device__ __forceinline__ RowChunk row_chunk(const AttendArgs& a, int stage, int step, int first, int before) {
    RowChunk c;
    c.first = first;
    c.range = RowRange{0, 0, 0, 0};
    c.steps = 0;
    const int lane = threadIdx.x & 63;
    if (first + lane < a.batch) {
        c.range = row_range(a, first + lane);
        const int low = c.range.n ? low_of(c.range, 0, a.window) : 0;
        c.steps = max(1, (c.range.n - (low & -stage) + step - 1) / step);        // (stage and step are powers of two)
    }
    const int up_to = wave_inclusive_scan(c.steps, lane);
    c.before = before + up_to - c.steps;
    c.after = before + __builtin_amdgcn_readlane(up_to, 63);
    return c;
}

// ---- the pass over keys and values -------------------------------------------------------------------------------------------
// grid = groups, block = 64 * WAVES.  HDP: head_dim rounded up (FULL: head_dim itself).  QT: tiles of 16 rows of a wave.
template <typename T, int HDP, bool FULL, int QT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, attend_lean(HDP, FULL, QT, sizeof(T)) ? 2 : 1) void k_kv_attend(const AttendArgs a) {
    using V = typename Vec<T>::type;
    using M = Mat<T>;
    constexpr int THREADS = 64 * WAVES;
    constexpr int N = Vec<T>::N;               // elements of 16 bytes; positions of a lane in the second products
    constexpr int TILES = N / 4;               // K tiles of a stage
    constexpr int STAGE = 4 * N;
    constexpr int CH = (HDP + 4 * N - 1) / (4 * N);          // pieces of a key that a lane holds
    constexpr int DT = HDP / 16;               // tiles of dimensions
    constexpr int HALF = HDP > 128 ? 2 : 1;    // the waves' sums meet in LDS, up to 128 dimensions at a time
    constexpr int COLS = HDP / HALF, PITCH = COLS + 4;
    constexpr int ROW = HDP + 4;               // floats of a row of a part
    __shared__ int last;
    __shared__ float wave_max[WAVES][16 * QT], wave_sum_[WAVES][16 * QT];
    __shared__ float sums[WAVES][16][PITCH];
    // What a wave needs of its rows only now and then is not kept in registers: their place in `out` (a row, negative for padding, and the
    // head), of the first segment and of later ones; first position, last new token, and which of those they see.  Queries of several
    // tiles neither: 128 dimensions by 32 rows fit 256 registers then, and eight waves a compute unit.
    // (64 rows by 128 dimensions have a wave a SIMD either way, and are slower so: 77 -> 80 us for 60 tokens of 4 sequences of 8000.)
    constexpr bool QLDS = QT > 1 && (attend_lean(HDP, FULL, QT, sizeof(T)) || (HDP == 256 && CH <= 8));
    __shared__ int2 out_at[2][16 * QT], sees_at[WAVES][16 * QT];
    __shared__ unsigned long long seen_at[WAVES][16 * QT];
    __shared__ V q_at[QLDS ? WAVES : 1][QLDS ? QT : 1][QLDS ? CH : 1][64];
    __shared__ int4 join_of[WAVES][2];         // parts to add behind the loop: w0, count, begins_before, bias
    const int tid = threadIdx.x, lane = tid & 63, wv = whole_wave(tid >> 6), n = lane & 15, g = lane >> 4, dim = FULL ? HDP : a.dim;
    constexpr int STEP = STAGE * WAVES;
    const int error = *a.error;
    RowChunk rc = row_chunk(a, STAGE, STEP, 0, 0);
    if (whole_wave(error)) return;
    int total = rc.after;
    for (int c0 = 64; c0 < a.batch; c0 += 64) total = row_chunk(a, STAGE, STEP, c0, total).after;
    const int all = total * a.kv_heads;        // (below 2^31: lif_kv_attend has seen to it)
    // which block of rows, and which of its workgroups: those that read the same keys are eight apart, on one XCD
    int block = 0, unit = blockIdx.x, units = a.units;
    if (a.row_blocks > 1) {
        if (all < a.round_steps) {             // all blocks' at once, each workgroup with more steps
            units = a.round_units;
            block = quotient(blockIdx.x, units);
            if (block >= a.row_blocks) return;
            unit = (int)blockIdx.x - block * units;
        } else if (a.units % 8 == 0) {
            const int eights = (int)blockIdx.x >> 3, high = quotient(eights, a.row_blocks);
            block = eights - high * a.row_blocks;
            unit = high * 8 + ((int)blockIdx.x & 7);
        } else {
            block = quotient(blockIdx.x, a.units);
            unit = (int)blockIdx.x - block * a.units;
        }
    }
    const int slots0 = 2 * block * a.units;    // the block's first place for a part
    const int rows = a.n_tokens * a.share, row0 = block * QT * 16;
    // Rows that are not there compute with one that is, and are not looked at; but where the reference lags, they have a say in when it moves.  There it is the
    // first row of the block, which no other item writes where `out` is q itself.
    constexpr bool LAGS = attend_slack(QT) > 0.f;
    const int tok0 = LAGS && row0 ? quotient(row0, a.share) : 0, share0 = row0 - tok0 * a.share;
    int run_steps = quotient(all + units - 1, units);
    // by items: parts of the lane's row, steps of each, parts of the rows before
    int parts_of_row = 0, part_steps = 1, parts_before = 0;
    bool by_items = false;
    if (a.batch <= 64) {
        for (int tries = 0; tries < 2 && !by_items; ++tries) {
            const int most = run_steps + (tries ? run_steps / 8 : 0);
            part_steps = small_ceil(rc.steps, small_ceil(rc.steps, most));
            parts_of_row = rc.steps > 0 ? small_ceil(rc.steps, part_steps) : 0;
            const int up_to = wave_inclusive_scan(parts_of_row, lane);
            parts_before = up_to - parts_of_row;
            const int needed = __builtin_amdgcn_readlane(up_to, 63) * a.kv_heads;
            by_items = needed <= units;
            if (by_items && unit >= needed) return;
            if (run_steps < 8) break;
        }
    }
    const int end = by_items ? 1 : (int)min((unsigned)run_steps * ((unsigned)unit + 1u), (unsigned)all);
    int at = by_items ? 0 : (int)min((unsigned)run_steps * (unsigned)unit, (unsigned)all);
    bool first_segment = true;
    bool arrived = false;                      // the first segment's part was the last of its run to be left
    int joins = 0;                             // bits of the segments that are parts
    const float scale_log2 = a.scale_log2, slack = fminf(attend_slack(QT) / scale_log2, 1e30f);
    const int rows_here = min(16 * QT, rows - row0);
    // four dimensions of a row of the output
    auto finish = [&](int seg, int r0, int d, f32x4 v, float m, float total, float bias) {
        const int2 to = out_at[seg][r0];
        const size_t out_row = (unsigned)to.x & 0x7fffffffu;
        const bool none = to.x < 0 || total == 0.f;
        const float inv = 1.f / total;
        if (FULL || d < dim) {
            typedef T T4 __attribute__((ext_vector_type(4)));
            T4 y;
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = none ? (T)0.f : (T)(v[j] * inv);
            *reinterpret_cast<T4*>((T*)a.out + out_row * a.out_stride + (unsigned)(to.y * dim + d)) = y;
        }
        if (a.lse && d == 0) a.lse[out_row * a.heads + to.y] = none ? -INFINITY : (m * scale_log2 - bias + log2f(total)) / kLog2e;
    };
    char* parts = reinterpret_cast<char*>(a.parts);
    const int level2 = 2 * (int)gridDim.x;     // places of parts; those of runs are behind them
    // place of the k-th part of an item whose first workgroup is w0
    auto part_of = [&](int w0, bool begins_before, int k) { return slots0 + 2 * (w0 + k) + (k == 0 && begins_before ? 1 : 0); };
    // whether this workgroup is the last of `n` to have left its part; `place`: of the first of them
    auto arrive = [&](int level, int place, int n) -> bool {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                     // this wave's stores are acknowledged,
        __syncthreads();                                                     // and those of the others
        if (tid == 0) last = n == 1 || (int)atomicInc(a.arrived + level * level2 + place, (unsigned)n - 1u) == n - 1;
        __syncthreads();
        return whole_wave(last);
    };
    auto part_at = [&](int slot, int r0) { return (unsigned)(((unsigned)slot * a.block_rows + r0) * ROW * 4u); };

    while (at < end) {
        int il, s0, s1, steps, kvh, w0, count;             // lane of the batch row, steps, key head, workgroups that share the item
        bool begins_before = false;                        // the first of them has steps of another item before
        if (by_items) {
            il = __popcll(__ballot(parts_before * a.kv_heads <= unit && rc.steps > 0)) - 1;
            steps = __builtin_amdgcn_readlane(rc.steps, il);
            count = __builtin_amdgcn_readlane(parts_of_row, il);
            const int in_row = unit - __builtin_amdgcn_readlane(parts_before, il) * a.kv_heads, each = __builtin_amdgcn_readlane(part_steps, il);
            kvh = quotient(in_row, count);
            w0 = unit - (in_row - kvh * count);
            s0 = (unit - w0) * each;
            s1 = min(steps, s0 + each);
        } else {
            while (rc.after * a.kv_heads <= at) rc = row_chunk(a, STAGE, STEP, rc.first + 64, rc.after);
            // the last row that begins at or before the step (rows behind the batch have no steps, and begin behind it)
            il = __popcll(__ballot(rc.before * a.kv_heads <= at && rc.steps > 0)) - 1;
            steps = __builtin_amdgcn_readlane(rc.steps, il);
            const int in_row = at - __builtin_amdgcn_readlane(rc.before, il) * a.kv_heads;
            kvh = quotient(in_row, steps);
            s0 = in_row - kvh * steps;
            s1 = min(steps, s0 + end - at);
            const int begin = at - s0;
            w0 = quotient(begin, run_steps);
            count = quotient(begin + steps - 1, run_steps) - w0 + 1;
            begins_before = w0 * run_steps < begin;
        }
        const int i = rc.first + il;
        const RowRange r = of_lane(rc.range, il);
        const int base = r.n - r.fresh, low_all = low_of(r, 0, a.window);
        const int bias_exp = attend_bias<T>(QT, r.n - low_all);
        const float bias = (float)bias_exp;

        const int seg = first_segment ? 0 : 1;
        if (!first_segment) lds_barrier();     // (the last segment's readers are done)
        V q[QLDS ? 1 : QT][CH];
        int2 my_sees;
        unsigned long long my_seen;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const int row = row0 + 16 * t + n;
            const int tok = (int)((unsigned)row / (unsigned)a.share), head = kvh * a.share + row - tok * a.share;
            const bool ok = row < rows && tok < r.fresh;
            if (g == 0) {
                if (wv == 0) out_at[seg][16 * t + n] = make_int2((i * a.n_tokens + tok) | (ok ? 0 : 1 << 31), head);
                if (QT > 1) sees_at[wv][16 * t + n] = make_int2(ok ? low_of(r, tok, a.window) : 0x7fffffff, a.tree ? 63 : tok);
                if (QT > 1) seen_at[wv][16 * t + n] = ok && a.tree ? a.tree[(size_t)i * a.n_tokens + tok] : ~0ull;
            }
            if (QT == 1) {
                my_sees = make_int2(ok ? low_of(r, tok, a.window) : 0x7fffffff, a.tree ? 63 : tok);
                my_seen = ~0ull;
                if (ok && a.tree) my_seen = a.tree[(size_t)i * a.n_tokens + tok];
            }
            const T* from = (const T*)a.q + ((size_t)i * a.n_tokens + (ok ? tok : tok0)) * a.q_stride + (unsigned)((ok ? head : LAGS ? kvh * a.share + share0 : 0) * dim);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const bool sure_in = FULL && (4 * c + 4) * N <= HDP;
                const int d = (4 * c + g) * N;
                V held = *reinterpret_cast<const V*>(from + (sure_in || d < dim ? d : 0));
                if (!sure_in && d >= dim) held = V{};
                if constexpr (QLDS) q_at[wv][t][c][lane] = held;
                else q[t][c] = held;
            }
        }
        f32x4 o[QT][DT];
        float top[QT], ref[QT], sum[QT];       // reference (-inf: nothing seen), the same or 0 there, sum of the lane's weights
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            top[t] = -INFINITY;
            ref[t] = sum[t] = 0.f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        const int origin = low_all / STAGE * STAGE;
        const int p_end = min(r.n, origin + s1 * STEP), p_last = r.n - 1;
        int p = origin + s0 * STEP + wv * STAGE;
        const int32_t* row_table = a.table + (size_t)r.slot * a.max_pages;
        // positions in [sure, sure_end) are visible to all rows of the item
        const int sure = a.window ? max(r.start, r.n - a.window) : r.start, sure_end = a.tree ? base : base + 1;
        const char* k_pool = a.k + kvh * (size_t)a.head_bytes;
        const char* v_pool = a.v + kvh * (size_t)a.head_bytes;
        const int page_mask = (1 << a.log_page) - 1;
        // whether the lane's row of tile t sees a position
        auto sees = [&](int2 at, unsigned long long seen, int pos) -> bool {
            const int own = pos - base;
            return (int)(pos >= at.x) & (int)(pos < r.n) & ((int)(own < 0) | ((int)(own <= at.y) & (int)(seen >> (own & 63) & 1ull)));
        };
        auto page_at = [&](int pos) { return row_table[min(pos, p_last) >> a.log_page]; };
        auto in_pool = [&](int page) { return (size_t)((unsigned)page < (unsigned)a.pages ? page : 0) * a.page_bytes; };
        // keys of a stage: row n of tile e is position p + N (n div 4) + 4 e + n mod 4; values: positions p + N g ..
        auto load_k = [&](V (&k)[TILES][CH], int p, int page) {
            const T* from = (const T*)(k_pool + in_pool(page)) + (unsigned)((((p + N * (n >> 2)) & page_mask) + (n & 3)) * dim);
#pragma unroll
            for (int e = 0; e < TILES; ++e)
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const bool sure_in = FULL && (4 * c + 4) * N <= HDP;
                    const int d = (4 * c + g) * N;
                    k[e][c] = *reinterpret_cast<const V*>(from + 4 * e * dim + (sure_in || d < dim ? d : 0));
                    if (!sure_in && d >= dim) k[e][c] = V{};
                }
        };
        auto v_from = [&](int p, int page) { return (const T*)(v_pool + in_pool(page)) + (unsigned)(((p + N * g) & page_mask) * dim); };
        auto load_v = [&](V (&v)[DT], const T* from) {
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                v[d] = *reinterpret_cast<const V*>(from + (FULL || 16 * d + n < dim ? 16 * d + n : 0) * N);
                if (!FULL && 16 * d + n >= dim) v[d] = V{};
            }
        };

        // Keys of the next stage are asked for as soon as this stage's are used up, values likewise, table entries a stage ahead of both: a
        // wave always has something on its way.  Loads come back in the order they were asked for in, so that order is keys, table entries,
        // values, everywhere: a wait for one of them is then no wait for the next (the barriers keep the compiler to it).
        if (p < p_end) {
            V k[TILES][CH], v[DT];
            const int k0 = page_at(p + N * (n >> 2)), v0 = page_at(p + N * g);
            load_k(k, p, k0);
            __builtin_amdgcn_sched_barrier(0);
            int k_page = page_at(p + STEP + N * (n >> 2)), v_page = page_at(p + STEP + N * g);
            __builtin_amdgcn_sched_barrier(0);
            load_v(v, v_from(p, v0));
            __builtin_amdgcn_sched_barrier(0);
            bool more;
            do {
                more = p + STEP < p_end;
                int here = lane;
                if constexpr (QLDS) asm volatile("" : "+v"(here));       // (read anew every time, and not kept in registers after all)
                float x[QT][N];
                {
                    // (two sums where one chain of products would be long)
                    constexpr int CHAINS = QT == 1 && M::kParts > 1 ? 2 : 1;
                    f32x4 s[QT][TILES][CHAINS];
#pragma unroll
                    for (int t = 0; t < QT; ++t)
#pragma unroll
                        for (int e = 0; e < TILES; ++e)
#pragma unroll
                            for (int h = 0; h < CHAINS; ++h) s[t][e][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = 0; c < CH; ++c) {
                        V qc[QT];
#pragma unroll
                        for (int t = 0; t < QT; ++t) {
                            if constexpr (QLDS) qc[t] = q_at[wv][t][c][here];
                            else qc[t] = q[t][c];
                        }
#pragma unroll
                        for (int u = 0; u < M::kParts; ++u)
#pragma unroll
                            for (int e = 0; e < TILES; ++e)
#pragma unroll
                                for (int t = 0; t < QT; ++t) s[t][e][u % CHAINS] = M::mul(k[e][c], qc[t], s[t][e][u % CHAINS], u);
                    }
#pragma unroll
                    for (int t = 0; t < QT; ++t)
#pragma unroll
                        for (int e = 0; e < TILES; ++e)
#pragma unroll
                            for (int j = 0; j < 4; ++j) x[t][4 * e + j] = CHAINS == 2 ? s[t][e][0][j] + s[t][e][CHAINS - 1][j] : s[t][e][0][j];
                }
                if (more) load_k(k, p + STEP, k_page);
                const T* v_next = v_from(p + STEP, v_page);
                __builtin_amdgcn_sched_barrier(0);
                k_page = page_at(p + 2 * STEP + N * (n >> 2));
                v_page = page_at(p + 2 * STEP + N * g);
                __builtin_amdgcn_sched_barrier(0);
                const int vp = p + N * g;
                const bool edge = p < sure || p + STAGE > sure_end;
                if (edge) {
                    if (QT > 1) lds_wave_fence();          // (sees_at, seen_at: stored by the lanes of the first group)
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        const int2 at = QT == 1 ? my_sees : sees_at[wv][16 * t + n];
                        const unsigned long long seen = QT == 1 ? my_seen : seen_at[wv][16 * t + n];
#pragma unroll
                        for (int e = 0; e < N; ++e) x[t][e] = sees(at, seen, vp + e) ? x[t][e] : -INFINITY;
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u) {          // what no row may see is not there, whatever it holds
                        auto in = [&](int e) { return vp + e >= low_all && vp + e < r.n; };
                        const unsigned mask = N == 4 ? (in(u) ? ~0u : 0u) : (in(2 * u) ? 0xffffu : 0u) | (in(2 * u + 1) ? 0xffff0000u : 0u);
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            u32x4 bits = __builtin_bit_cast(u32x4, v[d]);
                            bits[u] &= mask;
                            v[d] = __builtin_bit_cast(V, bits);
                        }
                    }
                }
                V w[QT];
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    float most = x[t][0];
#pragma unroll
                    for (int e = 1; e < N; ++e) most = fmaxf(most, x[t][e]);
                    if (__any(most > (attend_slack(QT) > 0.f ? top[t] + slack : top[t]))) {
                        most = fmaxf(row_max(most), top[t]);
                        const float scale = rescale(top[t], most, scale_log2);
                        ref[t] = most == -INFINITY ? 0.f : most;
                        top[t] = most;
                        sum[t] *= scale;
#pragma unroll
                        for (int d = 0; d < DT; ++d) o[t][d] *= scale;
                    }
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float weight = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][e] - ref[t], scale_log2, bias));
                        sum[t] += weight;
                        w[t][e] = (T)weight;
                    }
                }
                // A weight of zero does not keep a value out that is not finite.  Where rows see different positions of a stage, or none of them
                // sees one (by a tree, a single new token its own), such values are taken out of the products and added to the rows that see them.
                if (edge && (r.fresh > 1 || a.tree)) {
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
                        for (int pos = max(p, low_all); pos < min(p + STAGE, r.n); ++pos) {
                            const T* from = (const T*)(v_pool + in_pool(page_at(pos))) + (unsigned)((pos & page_mask) / N * dim * N) + pos % N;
                            bool seen_here[QT];
#pragma unroll
                            for (int t = 0; t < QT; ++t) seen_here[t] = QT == 1 ? sees(my_sees, my_seen, pos) : sees(sees_at[wv][16 * t + n], seen_at[wv][16 * t + n], pos);
#pragma unroll
                            for (int d = 0; d < DT; ++d)
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const int at_dim = 16 * d + 4 * g + j;
                                    const float value = (float)from[(FULL || at_dim < dim ? at_dim : 0) * N];
                                    const float add = __builtin_isfinite(value) || (!FULL && at_dim >= dim) ? 0.f : value;
#pragma unroll
                                    for (int t = 0; t < QT; ++t) o[t][d][j] += seen_here[t] ? add : 0.f;
                                }
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < M::kParts; ++u)
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int t = 0; t < QT; ++t) o[t][d] = M::mul(v[d], w[t], o[t][d], u);
                if (more) load_v(v, v_next);
                p += STEP;
            } while (more);
        }

        // the waves' sums meet
        const bool whole = s0 == 0 && s1 == steps;
        const int part = slots0 + 2 * unit + seg;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const float total = row_sum(sum[t]);
            if (g == 0) {
                wave_max[wv][16 * t + n] = top[t];
                wave_sum_[wv][16 * t + n] = total;
            }
        }
#pragma unroll
        for (int t = 0; t < QT; ++t) {
#pragma unroll
            for (int half = 0; half < HALF; ++half) {
                if (t || half) lds_barrier();
#pragma unroll
                for (int d = 0; d < DT / HALF; ++d)
                    *reinterpret_cast<f32x4*>(&sums[wv][n][16 * d + 4 * g]) = o[t][half * (DT / HALF) + d];
                lds_barrier();
                for (int u = tid; u < 16 * (COLS / 4); u += THREADS) {
                    const int rr = u / (COLS / 4), d = u % (COLS / 4) * 4, r0 = 16 * t + rr;
                    if (r0 >= rows_here) break;
                    float wm[WAVES], wl[WAVES];
                    f32x4 wy[WAVES];
#pragma unroll
                    for (int w = 0; w < WAVES; ++w) {
                        wm[w] = wave_max[w][r0];
                        wl[w] = wave_sum_[w][r0];
                        wy[w] = *reinterpret_cast<const f32x4*>(&sums[w][rr][d]);
                    }
                    float m = wm[0], l = 0.f;
#pragma unroll
                    for (int e = 1; e < WAVES; ++e) m = fmaxf(m, wm[e]);
                    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int e = 0; e < WAVES; ++e) {
                        const float f = rescale(wm[e], m, scale_log2);
                        l += wl[e] * f;
                        y += wy[e] * f;
                    }
                    if (whole) {
                        finish(seg, r0, half * COLS + d, y, m, l, bias);
                    } else {
                        store_through(parts, part_at(part, r0) + (half * COLS + d) * 4, a.part_bytes, y);
                        if (half == 0 && d == 0) store_through(parts, part_at(part, r0) + HDP * 4, a.part_bytes, f32x4{m, l, 0.f, 0.f});
                    }
                }
            }
        }

        if (!whole) {
            joins |= 1 << seg;
            if (lane == 0) join_of[wv][seg] = make_int4(w0, count, begins_before, bias_exp);
        }
        if (by_items) break;
        at += s1 - s0;
        if (!whole && at < end) {              // (others may be waiting for this one's first part)
            const int from = (unit - w0) / kAttendFan * kAttendFan;
            arrived = arrive(0, part_of(w0, begins_before, from), min(kAttendFan, count - from));
            joins = arrived ? 1 : 0;
        }
        first_segment = false;
    }

    // Parts: each of the `count` workgroups from w0 on has left one (the first of them its last segment, if it began before the item).
    // Runs of kAttendFan of them are added by the last one of the run, into the place of the run's first part, and the runs by the last run.
    // (Behind the loop: inside, what this needs of registers would be kept through the pass over the keys.)
#pragma unroll 1
    for (int seg = 0; seg < 2; ++seg) {
        if (!(joins >> seg & 1)) continue;
        lds_wave_fence();
        const int4 of = join_of[wv][seg];
        const int w0 = whole_wave(of.x), count = whole_wave(of.y), runs = (count + kAttendFan - 1) / kAttendFan;
        const bool begins_before = whole_wave(of.z);
        const float bias = (float)(M::kFewExponents ? attend_bias<T>(QT, 0) : whole_wave(of.w));
        int level = 0, from = (unit - w0) / kAttendFan * kAttendFan, stride = 1, n_parts = min(kAttendFan, count - from);
        while (true) {
            if (!arrived && !arrive(level, part_of(w0, begins_before, from), n_parts)) break;
            arrived = false;
            const bool done = level == 1 || runs == 1;
            // Rows x four dimensions to the threads, and what is left of them shares the parts of a row.  A thread asks for kAttendAsk parts
            // at once, those of its next rows among them.
            constexpr int QUADS = HDP / 4, TEAMS = THREADS / QUADS >= 32 ? 32 : THREADS / QUADS >= 16 ? 16 : THREADS / QUADS >= 8 ? 8 : 4;
            int log_once = 0;
            while ((1 << log_once) < TEAMS && (1 << log_once) < rows_here) ++log_once;
            const int shares = TEAMS >> log_once, per = (n_parts + shares - 1) >> (__builtin_ctz(TEAMS) - log_once);
            const int team = tid / QUADS, d = tid % QUADS * 4, share = team >> log_once, row_in = team & ((1 << log_once) - 1);
            const int units = ((rows_here + (1 << log_once) - 1) >> log_once) * per;
            auto leave = [&](int r0, f32x4 y, float m, float l) {
                if (done) {
                    finish(seg, r0, d, y, m, l, bias);
                } else {
                    const unsigned b = part_at(level2 + part_of(w0, begins_before, from), r0);
                    store_through(parts, b + d * 4, a.part_bytes, y);
                    if (d == 0) store_through(parts, b + HDP * 4, a.part_bytes, f32x4{m, l, 0.f, 0.f});
                }
            };
            float m = -INFINITY, l = 0.f;
            f32x4 y = {0.f, 0.f, 0.f, 0.f};
            int r_ask = row_in, e_ask = 0, r0 = row_in, e_now = 0;           // row and part of the next one to ask for, and to add
            for (int u0 = 0; u0 < units; u0 += kAttendAsk) {
                f32x2 s[kAttendAsk];
                f32x4 v[kAttendAsk];
#pragma unroll
                for (int e = 0; e < kAttendAsk; ++e)
                    if (u0 + e < units) {
                        const unsigned b = part_at(level * level2 + part_of(w0, begins_before, from + min(share * per + e_ask, n_parts - 1) * stride),
                                                   min(r_ask, rows_here - 1));
                        s[e] = load_through2(a.parts, b + HDP * 4, a.part_bytes);
                        v[e] = load_through(a.parts, b + d * 4, a.part_bytes);
                        if (++e_ask == per) {
                            e_ask = 0;
                            r_ask += 1 << log_once;
                        }
                    }
#pragma unroll
                for (int e = 0; e < kAttendAsk; ++e)
                    if (u0 + e < units) {
                        if (share * per + e_now < n_parts) {
                            const float most = fmaxf(m, s[e][0]), old = rescale(m, most, scale_log2), f = rescale(s[e][0], most, scale_log2);
                            m = most;
                            l = l * old + s[e][1] * f;
                            y = y * old + v[e] * f;
                        }
                        if (++e_now == per) {
                            if (shares == 1) {
                                if (team < TEAMS && r0 < rows_here) leave(r0, y, m, l);
                                r0 += 1 << log_once;
                                m = -INFINITY;
                                l = 0.f;
                                y = f32x4{0.f, 0.f, 0.f, 0.f};
                            }
                            e_now = 0;
                        }
                    }
            }
            if (shares > 1) {                    // (one round of rows)
                const int taken = small_ceil(n_parts, per);              // shares that have parts
                float* mine = &sums[0][0][0] + (team < TEAMS ? team : 0) * ROW;
                const bool here = team < TEAMS && r0 < rows_here;
                __syncthreads();
                if (here) {
                    *reinterpret_cast<f32x4*>(mine + d) = y;
                    if (d == 0) {
                        mine[HDP] = m;
                        mine[HDP + 1] = l;
                    }
                }
                __syncthreads();
                if (here && share == 0) {
                    float most = m;
#pragma unroll 4
                    for (int k = 1; k < taken; ++k) most = fmaxf(most, mine[(k << log_once) * ROW + HDP]);
                    const float f0 = rescale(m, most, scale_log2);
                    l *= f0;
                    y *= f0;
#pragma unroll 4
                    for (int k = 1; k < taken; ++k) {
                        const float* theirs = mine + (k << log_once) * ROW;
                        const float f = rescale(theirs[HDP], most, scale_log2);
                        l += theirs[HDP + 1] * f;
                        y += *reinterpret_cast<const f32x4*>(theirs + d) * f;
                    }
                    leave(r0, y, most, l);
                }
            }
            if (done) break;
            level = 1;
            from = 0;
            stride = kAttendFan;
            n_parts = runs;
        }
    }
}

template <typename T, int HDP, bool FULL, int QT>
bool launch_attend_waves(const AttendArgs& a, int groups, int waves, hipStream_t s) {
    constexpr bool lean = attend_lean(HDP, FULL, QT, sizeof(T));
    if constexpr (lean)
        if (waves == 8) {
            hipLaunchKernelGGL((k_kv_attend<T, HDP, FULL, QT, 8>), dim3(groups), dim3(512), 0, s, a);
            return true;
        }
    if constexpr (!lean || QT == 1)
        if (waves == 4) {
            hipLaunchKernelGGL((k_kv_attend<T, HDP, FULL, QT, 4>), dim3(groups), dim3(256), 0, s, a);
            return true;
        }
    return false;
}

template <typename T, int HDP, int QT>
bool launch_attend(const AttendArgs& a, int groups, int waves, hipStream_t s) {
    if (a.dim == HDP) return launch_attend_waves<T, HDP, true, QT>(a, groups, waves, s);
    if constexpr (HDP != 80 && QT <= (HDP == 256 ? 1 : 2)) return launch_attend_waves<T, HDP, false, QT>(a, groups, waves, s);
    return false;
}

template <typename T, int QT>
bool launch_attend_tiles(const AttendArgs& a, int groups, int waves, hipStream_t s) {
    switch (attend_dim_pad(a.dim)) {
        case 32: return launch_attend<T, 32, QT>(a, groups, waves, s);
        case 64: return launch_attend<T, 64, QT>(a, groups, waves, s);
        case 80: return launch_attend<T, 80, QT>(a, groups, waves, s);
        case 96: return launch_attend<T, 96, QT>(a, groups, waves, s);
        case 128: return launch_attend<T, 128, QT>(a, groups, waves, s);
        default:
            if constexpr (QT <= 2) return launch_attend<T, 256, QT>(a, groups, waves, s);
            return false;
    }
}

}  // namespace lif
