// The paged key-value cache as the kernels see it.
#pragma once

#include "lif_common.h"

namespace lif {

constexpr int kKvMaxSeqs = 1024;

struct KvState {
    int32_t used;            // pages in use
    int32_t error;           // sticky lif_status
    int32_t n_moves;         // pages to copy by the launch that follows a plan
    int32_t ok;              // whether the plan of a fork or a compaction stands
    int32_t shares;          // whether a page may have several holders: since a fork, or tables that were adopted so
    unsigned planned;        // workgroups of a reservation that have planned; zero between calls
};

// What the kernels know of a cache.
struct KvView {
    char* k;
    char* v;
    int32_t* table;
    int32_t* lengths;
    int32_t* fresh;
    int32_t* refs;
    KvState* st;
    unsigned* arrived;               // counts of lif_kv_attend, zero between calls
    unsigned long long* free_bits;   // [ceil(pages / 64)]
    int2* moves;                     // [pages] from, to
    int32_t* remap;                  // [pages or max_seqs] where a moved page went; which copy a pair of a fork gets
    int32_t pages, max_seqs, max_pages, log_page, layers, n_arrived;
    unsigned long long page_bytes;   // of the keys of one page of one layer (and of the values)
};

__device__ __forceinline__ int pages_of(long long tokens, int log_page) { return (int)((tokens + (1 << log_page) - 1) >> log_page); }
// the length of a slot, inside the table whatever the array holds
__device__ __forceinline__ int length_of(const KvView& kv, int slot) { return min(max(kv.lengths[slot], 0), kv.max_pages << kv.log_page); }
__device__ __forceinline__ bool page_ok(const KvView& kv, int page) { return (unsigned)page < (unsigned)kv.pages; }

// the last entry of first[0..n) that is <= v; first[0] = 0, ascending
__device__ __forceinline__ int last_not_above(const int* first, int n, int v) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (first[mid] <= v) lo = mid;
        else hi = mid;
    }
    return lo;
}

}  // namespace lif
