// The calls on the pages of a key-value cache: reset, adopt, reserve, truncate, fork, compact.
//
// A page is free iff refs[page] == 0.  The same as one bit per page, set where it is free, is what the calls look for pages in: 64
// pages a word and a word a thread, so that one workgroup sees 16384 pages a pass with 256 threads, 65536 with 1024.  The plans (which page goes where) are made by one workgroup, whose
// time is a few dependent memory round trips; the copies that follow from them by a launch over the whole chip (k_kv_move).  A reservation,
// which every step of a program makes, is a single launch.
#pragma once

#include "lif_kv.h"

namespace lif {

// threads of the planning workgroup, one per slot: 256 or 1024 (max_seqs).  A barrier among 16 waves costs more than one among 4; a pool of more
// than 16384 pages takes more passes with 256 (one of 200000 whose first pages are in use 9.7 us for reserve + truncate, one of 8192 9.5).
constexpr int kKvPlanFew = 256;

// Walks the set bits of the words [w0, w1) in ascending order by the whole workgroup: emit(rank, page) for those of rank < total, and
// keep(word index, word, taken bits) for every word that had one of them.  select(word index, word) picks the bits that count.  A thread
// counts the bits of a word; a word with bits that are wanted is then dealt to a wave, one bit to a lane: pages come in runs, and
// one thread that goes through 64 bits by itself is what the others wait for.
// Returns the bits seen (all of them if total is not reached).  Every thread of the workgroup has to call it.
// `ahead`: the word of the thread in the first pass.
template <int THREADS>
struct WalkScratch {
    int wave_tot[THREADS / 64];
    unsigned long long word[THREADS];
    int before[THREADS];
};
__device__ __forceinline__ unsigned long long word_ahead(const unsigned long long* bits, int w0, int w1) {
    return w0 + (int)threadIdx.x < w1 ? bits[w0 + threadIdx.x] : 0ull;
}
template <int THREADS, typename Select, typename Emit, typename Keep>
__device__ __forceinline__ int walk_bits(const unsigned long long* bits, int w0, int w1, int total, unsigned long long ahead, WalkScratch<THREADS>& ws,
                                         Select select, Emit emit, Keep keep) {
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    int seen = 0;
    for (int base = w0; base < w1 && seen < total; base += THREADS) {
        const int at = base + tid;
        const unsigned long long w = at < w1 ? select(at, base == w0 ? ahead : bits[at]) : 0ull;
        int all;
        const int before = block_exclusive_scan<THREADS / 64>(__popcll(w), ws.wave_tot, &all);
        ws.word[tid] = w;
        ws.before[tid] = seen + before;
        __syncthreads();
        for (int i = wv; i < min(THREADS, w1 - base); i += THREADS / 64) {
            const unsigned long long word = ws.word[i];
            const int first = ws.before[i];
            if (first >= total) break;
            if (!word) continue;
            const int rank = first + __popcll(word & ((1ull << lane) - 1ull));
            const bool take = (word >> lane & 1ull) && rank < total;
            if (take) emit(rank, (base + i) * 64 + lane);
            const unsigned long long taken = __ballot(take);
            if (lane == 0) keep(base + i, taken);
        }
        seen += all;
        __syncthreads();
    }
    return seen;
}

// ---- reset, adopt: grid over the pages and the slots, block = 256 ---------------------------------------------------------------

__device__ __forceinline__ unsigned long long free_word(int w, int pages) {
    const int left = pages - w * 64;
    return left >= 64 ? ~0ull : (1ull << left) - 1ull;
}

// RESET: no sequences.  Else only what k_kv_adopt counts afresh.
template <bool RESET>
__global__ __launch_bounds__(256) void k_kv_clear(const KvView kv) {
    const long long step = (long long)gridDim.x * 256, at = (long long)blockIdx.x * 256 + threadIdx.x;
    if (at == 0) *kv.st = KvState{0, 0, 0, 0, 0};
    for (long long i = at; i < kv.n_arrived; i += step) kv.arrived[i] = 0;
    for (long long i = at; i < kv.pages; i += step) kv.refs[i] = 0;
    for (long long i = at; i < (kv.pages + 63) / 64; i += step) kv.free_bits[i] = free_word((int)i, kv.pages);
    if (RESET) {
        for (long long i = at; i < kv.max_seqs; i += step) kv.lengths[i] = kv.fresh[i] = 0;
        for (long long i = at; i < (long long)kv.max_seqs * kv.max_pages; i += step) kv.table[i] = -1;
    }
}

// grid = max_seqs; a workgroup per slot
__global__ __launch_bounds__(256) void k_kv_adopt(const KvView kv) {
    const int slot = blockIdx.x, n = kv.lengths[slot], f = kv.fresh[slot];
    int32_t* row = kv.table + (size_t)slot * kv.max_pages;
    bool bad = n < 0 || (long long)n > (long long)kv.max_pages << kv.log_page || f < 0 || f > n;
    const int held = bad ? 0 : pages_of(n, kv.log_page);
    int used = 0;
    for (int j = threadIdx.x; j < kv.max_pages; j += 256) {
        if (j >= held) {
            if (!bad) row[j] = -1;
            continue;
        }
        const int page = row[j];
        if (!page_ok(kv, page)) {
            bad = true;
        } else if (atomicAdd(&kv.refs[page], 1) == 0) {
            atomicAnd(&kv.free_bits[page >> 6], ~(1ull << (page & 63)));
            ++used;
        } else {
            kv.st->shares = 1;
        }
    }
    if (used) atomicAdd(&kv.st->used, used);
    if (bad) atomicExch(&kv.st->error, 2 /* LIF_BAD_STATE */);
}

// ---- copies of pages ------------------------------------------------------------------------------------------------------------
// kKvPiece bytes of one page of one layer at a time by 256 threads: 16-byte loads, four in flight per thread, neighbouring workgroups on
// neighbouring pieces; the pieces first, first + step, ..  (compaction of 470 MB read and written: 97 us, 4.9 TB/s, what a large copy reaches; a fork
// of 537 MB: 54 us, since its sources lie in the last-level cache)
constexpr int kKvPiece = 256 * 16 * 4;

__device__ __forceinline__ void copy_pages(const KvView& kv, const int2* moves, int n_moves, unsigned first, unsigned step) {
    const unsigned pieces = (unsigned)((kv.page_bytes + kKvPiece - 1) / kKvPiece), per_move = pieces * 2u * (unsigned)kv.layers;
    const unsigned long long units = (unsigned long long)n_moves * per_move;
    for (unsigned long long u = first; u < units; u += step) {
        const unsigned move = (unsigned)(u / per_move), rest = (unsigned)(u % per_move), piece = rest % pieces, part = rest / pieces;
        const int2 m = moves[move];
        char* pool = (part & 1) ? kv.v : kv.k;
        const size_t layer = (size_t)(part >> 1) * kv.pages;
        const char* from = pool + (layer + m.x) * kv.page_bytes;
        char* to = pool + (layer + m.y) * kv.page_bytes;
        const size_t at = (size_t)piece * kKvPiece + (size_t)(threadIdx.x & 255) * 16;
        f32x4 held[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (at + q * 4096 < kv.page_bytes) held[q] = *reinterpret_cast<const f32x4*>(from + at + q * 4096);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (at + q * 4096 < kv.page_bytes) *reinterpret_cast<f32x4*>(to + at + q * 4096) = held[q];
    }
}

// ---- reserve: grid = the first workgroup, and those that copy if there may be something to ----------------------------------------
// Without sharing the first workgroup does everything.  With it every workgroup works out the same plan for itself, and copies its
// part of the pages; nothing that the plan follows from may change before all of them have read it, so it is the last one to have
// planned that writes it down.  One launch, and no workgroup waits for another (reserve + truncate of 64 slots, called one after the other:
// 8.8 us a pair; 12.2 with the copies in a launch of their own).  After a fork a page may have several holders, and stays counted as such until
// lif_kv_reset or lif_kv_adopt: 32 sequences of 2000, 9.5 us a pair before a fork, 12.0 after it, also when the beam is gone.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_kv_reserve(const KvView kv, const int32_t* __restrict__ counts) {
    __shared__ WalkScratch<THREADS> ws;
    __shared__ int first[THREADS], had_of[THREADS], copy_of[THREADS], last;
    __shared__ int2 moves[THREADS];                      // the copies
    const int slot = threadIdx.x, words = (kv.pages + 63) / 64;
    KvState* st = kv.st;
    const int error = st->error, used = st->used, shares = st->shares;
    if (blockIdx.x > 0 && !shares) return;
    const unsigned long long ahead = word_ahead(kv.free_bits, 0, words);
    int length = 0, count = 0;
    if (slot < kv.max_seqs) {
        length = length_of(kv, slot);
        count = max(counts[slot], 0);
    }
    if (error) return;                                   // (the same for all threads)
    const long long end = (long long)length + count;
    const int had = pages_of(length, kv.log_page);
    const bool fits = end <= (long long)kv.max_pages << kv.log_page;
    int32_t* row = kv.table + (size_t)(slot < kv.max_seqs ? slot : 0) * kv.max_pages;
    // tokens that go behind others into a page that is not this sequence's alone: a copy of it
    int shared = -1;
    if (shares && fits && count > 0 && (length & ((1 << kv.log_page) - 1))) {
        const int page = row[had - 1];
        if (page_ok(kv, page) && kv.refs[page] > 1) shared = page;
    }
    const int need = fits ? pages_of(end, kv.log_page) - had + (shared >= 0) : 0;
    int total, copies;
    const int rank0 = block_exclusive_scan<THREADS / 64>(need, ws.wave_tot, &total);
    int copy0 = copies = 0;
    if (shares) copy0 = block_exclusive_scan<THREADS / 64>(shared >= 0, ws.wave_tot, &copies);
    first[slot] = rank0;
    had_of[slot] = had - (shared >= 0);
    copy_of[slot] = shared >= 0 ? copy0 : -1;
    if (__syncthreads_or(!fits) || total > kv.pages - used) {
        if (slot == 0 && blockIdx.x == 0) {
            st->error = 3 /* LIF_CAPACITY */;            // (who reads it before the counts comes to the same end)
            st->n_moves = 0;
        }
        return;
    }
    const int slots = min(THREADS, kv.max_seqs);
    if (shares) {
        if (shared >= 0) moves[copy0].x = shared;
        if (copies > 0)
            walk_bits(
                kv.free_bits, 0, words, total, ahead, ws, [](int, unsigned long long w) { return w; },
                [&](int rank, int page) {
                    const int s = last_not_above(first, slots, rank);
                    if (rank == first[s] && copy_of[s] >= 0) moves[copy_of[s]].y = page;
                },
                [](int, unsigned long long) {});
        __syncthreads();                                 // (what this workgroup read has arrived)
        if (slot == 0) last = atomicInc(&st->planned, gridDim.x - 1) == gridDim.x - 1;
        __syncthreads();
        copy_pages(kv, moves, copies, blockIdx.x * (THREADS / 256) + threadIdx.x / 256, gridDim.x * (THREADS / 256));
        if (!last) return;
    }
    if (total > 0) {
        walk_bits(
            kv.free_bits, 0, words, total, ahead, ws, [](int, unsigned long long w) { return w; },
            [&](int rank, int page) {
                const int s = last_not_above(first, slots, rank), j = rank - first[s];
                kv.table[(size_t)s * kv.max_pages + had_of[s] + j] = page;
                kv.refs[page] = 1;
            },
            [&](int w, unsigned long long taken) { kv.free_bits[w] &= ~taken; });
    }
    int all_freed = 0, freed = 0;
    if (shared >= 0 && atomicSub(&kv.refs[shared], 1) == 1) {        // (everyone who held it has a copy)
        atomicOr(&kv.free_bits[shared >> 6], 1ull << (shared & 63));
        freed = 1;
    }
    if (shares) all_freed = __syncthreads_count(freed);
    if (slot < kv.max_seqs) {
        kv.lengths[slot] = (int)end;
        kv.fresh[slot] = count;
    }
    if (slot == 0) {
        st->used = used + total - all_freed;
        st->n_moves = copies;
        st->ok = 1;
    }
}

// ---- truncate: grid = max_seqs, a workgroup per slot ------------------------------------------------------------------------

__global__ __launch_bounds__(256) void k_kv_truncate(const KvView kv, const int32_t* __restrict__ to) {
    const int slot = blockIdx.x, length = length_of(kv, slot), want = to[slot];
    const int error = kv.st->error;
    if (error == 2 /* LIF_BAD_STATE */) return;
    const int keep = want < 0 || want > length ? length : want;
    int32_t* row = kv.table + (size_t)slot * kv.max_pages;
    __syncthreads();                                     // (every thread has read the length)
    int freed = 0;
    for (int j = pages_of(keep, kv.log_page) + threadIdx.x; j < pages_of(length, kv.log_page); j += 256) {
        const int page = row[j];
        row[j] = -1;
        if (page_ok(kv, page) && atomicSub(&kv.refs[page], 1) == 1) {
            atomicOr(&kv.free_bits[page >> 6], 1ull << (page & 63));
            ++freed;
        }
    }
    if (freed) atomicSub(&kv.st->used, freed);
    if (threadIdx.x == 0) {
        kv.lengths[slot] = keep;
        kv.fresh[slot] = 0;
        if (error && slot == 0) kv.st->error = 0;
    }
}

// ---- fork: one workgroup plans, k_kv_move does ------------------------------------------------------------------------------

template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_kv_fork(const KvView kv, const int32_t* __restrict__ src, const int32_t* __restrict__ dst, int n) {
    __shared__ WalkScratch<THREADS> ws;
    __shared__ unsigned named[kKvMaxSeqs / 32];
    const int i = threadIdx.x, words = (kv.pages + 63) / 64;
    KvState* st = kv.st;
    const unsigned long long ahead = word_ahead(kv.free_bits, 0, words);
    const int error = st->error, used = st->used;
    if (i < kKvMaxSeqs / 32) named[i] = 0;
    __syncthreads();
    bool bad = false;
    int s = 0, d = 0, length = 0;
    if (i < n) {
        s = src[i];
        d = dst[i];
        bad = (unsigned)s >= (unsigned)kv.max_seqs || (unsigned)d >= (unsigned)kv.max_seqs;
        if (!bad) {
            length = length_of(kv, s);
            bad = kv.lengths[d] != 0 || (atomicOr(&named[d / 32], 1u << (d % 32)) >> (d % 32) & 1u);
        }
    }
    const bool partial = i < n && !bad && (length & ((1 << kv.log_page) - 1));
    int total;
    const int rank0 = block_exclusive_scan<THREADS / 64>(partial, ws.wave_tot, &total);
    const bool any_bad = __syncthreads_or(bad);
    if (error || any_bad || total > kv.pages - used) {
        if (i == 0) {
            st->ok = 0;
            if (!error) {
                st->error = any_bad ? 1 /* LIF_INVALID_ARG */ : 3 /* LIF_CAPACITY */;
                st->n_moves = 0;
            }
        }
        return;
    }
    // the page of rank r is the copy of the last page of the r-th pair that has a partly filled one
    if (total > 0)
        walk_bits(
            kv.free_bits, 0, words, total, ahead, ws, [](int, unsigned long long w) { return w; },
            [&](int rank, int page) {
                kv.moves[rank].y = page;
                kv.refs[page] = 1;
            },
            [&](int w, unsigned long long taken) { kv.free_bits[w] &= ~taken; });
    if (i < n) {
        const int held = pages_of(length, kv.log_page);
        if (partial) {
            const int page = kv.table[(size_t)s * kv.max_pages + held - 1];
            kv.moves[rank0].x = page_ok(kv, page) ? page : 0;
        }
        kv.remap[i] = partial ? rank0 : -1;              // which copy the last page of pair i is (max_seqs entries are there)
        kv.lengths[d] = length;
        kv.fresh[d] = 0;
    }
    if (i == 0) {
        st->used = used + total;
        st->n_moves = total;
        st->ok = 1;
        st->shares = 1;
    }
}

// ---- compact: one workgroup plans -------------------------------------------------------------------------------------------

template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_kv_compact(const KvView kv) {
    __shared__ WalkScratch<THREADS> ws;
    KvState* st = kv.st;
    const int error = st->error, used = st->used, words = (kv.pages + 63) / 64, edge = used >> 6;
    if (error) {
        if (threadIdx.x == 0) st->ok = 0;
        return;
    }
    auto below = [&](int w) { return w < edge ? ~0ull : w > edge ? 0ull : (1ull << (used & 63)) - 1ull; };   // pages < used
    auto nothing = [](int, unsigned long long) {};
    const int holes = walk_bits(
        kv.free_bits, 0, min(edge + 1, words), 0x7fffffff, word_ahead(kv.free_bits, 0, words), ws, [&](int w, unsigned long long v) { return v & below(w); },
        [&](int rank, int page) { kv.moves[rank].y = page; }, nothing);
    if (holes > 0) {
        // as many used pages lie at or above `used` as free ones below; the highest goes to the lowest hole
        const int movers = walk_bits(
            kv.free_bits, edge, words, holes, word_ahead(kv.free_bits, edge, words), ws, [&](int w, unsigned long long v) { return ~v & ~below(w) & free_word(w, kv.pages); },
            [&](int rank, int page) { kv.moves[holes - 1 - rank].x = page; }, nothing);
        if (movers < holes) {                            // (counts that do not belong together: the state was written over)
            if (threadIdx.x == 0) st->error = 2 /* LIF_BAD_STATE */;
            return;
        }
        for (int j = threadIdx.x; j < holes; j += THREADS) {
            const int2 m = kv.moves[j];
            kv.refs[m.y] = kv.refs[m.x];
            kv.refs[m.x] = 0;
            kv.remap[m.x] = m.y;
        }
        for (int w = threadIdx.x; w < words; w += THREADS) kv.free_bits[w] = free_word(w, kv.pages) & ~below(w);
    }
    if (threadIdx.x == 0) {
        st->n_moves = holes;
        st->ok = 1;
    }
}

// ---- what the plans leave to the whole chip ---------------------------------------------------------------------------------
// The first `table_blocks` workgroups bring the tables in line, the others copy pages.
enum { KV_FORK = 1, KV_COMPACT = 2 };

template <int JOB>
__global__ __launch_bounds__(256) void k_kv_move(const KvView kv, const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                 int table_blocks) {
    const KvState* st = kv.st;
    const int n_moves = st->n_moves;
    if (st->error || !st->ok) return;
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < table_blocks) {
        if constexpr (JOB == KV_FORK) {                  // a pair: full pages shared, the copy behind them
            const int i = blockIdx.x, copy = kv.remap[i], held = pages_of(length_of(kv, dst[i]), kv.log_page);
            const int32_t* from = kv.table + (size_t)src[i] * kv.max_pages;
            int32_t* to = kv.table + (size_t)dst[i] * kv.max_pages;
            for (int j = tid; j < held; j += 256) {
                if (copy >= 0 && j == held - 1) {
                    to[j] = kv.moves[copy].y;
                } else {
                    const int page = from[j];
                    to[j] = page;
                    if (page_ok(kv, page)) atomicAdd(&kv.refs[page], 1);
                }
            }
        } else {                                         // a slot: pages at or above the count have moved
            const int held = pages_of(length_of(kv, blockIdx.x), kv.log_page), used = st->used;
            int32_t* row = kv.table + (size_t)blockIdx.x * kv.max_pages;
            if (n_moves)
                for (int j = tid; j < held; j += 256) {
                    const int page = row[j];
                    if (page >= used && page_ok(kv, page)) row[j] = kv.remap[page];
                }
        }
        return;
    }
    copy_pages(kv, kv.moves, n_moves, blockIdx.x - table_blocks, gridDim.x - table_blocks);
}

}  // namespace lif
