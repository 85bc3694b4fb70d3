// What the kernels of the paged cache share: where a row of a batch belongs, and where a position lies.
#pragma once
#include "launch.h"

namespace spd {

// positions that sequence `seq` has cached, as the calls count them
__device__ __forceinline__ int paged_len(const PagedBatchArgs &b, int seq) { return min(max(b.lens[seq], 0), b.capacity); }
// rows of sequence `seq`: first and behind the last, inside the call's rows whatever row_start holds
__device__ __forceinline__ void paged_rows(const PagedBatchArgs &b, int seq, int &first, int &last) {
    if (b.row_start) {
        first = min(max(b.row_start[seq], 0), b.n_rows);
        last = min(max(b.row_start[seq + 1], first), b.n_rows);
    } else {
        first = seq * b.each;
        last = first + b.each;
    }
}
// the page of positions p .. with p / page_size alike; -1: none
__device__ __forceinline__ int paged_page(const PagedBatchArgs &b, const PagedCacheArgs &c, int seq, int at) {
    if (at >= b.max_pages) return -1;
    const int page = b.page_table[(size_t)seq * b.table_stride + at];
    return (unsigned)page < (unsigned)c.n_pages ? page : -1;
}

// The same in two parts: the table's entry, whose load may be under way while other things are done, and what it says.  (Looked at in the step that loads it,
// an entry makes that step wait for every load before it.)
__device__ __forceinline__ int paged_entry(const PagedBatchArgs &b, const PagedCacheArgs &c, int seq, int position) {
    return b.page_table[(size_t)seq * b.table_stride + min(position >> c.page_bits, b.max_pages - 1)];
}
__device__ __forceinline__ int paged_entry_page(const PagedBatchArgs &b, const PagedCacheArgs &c, int entry, int position) {
    return position < b.capacity && (unsigned)entry < (unsigned)c.n_pages ? entry : -1;
}

}  // namespace spd
