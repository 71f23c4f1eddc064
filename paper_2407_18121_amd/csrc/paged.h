// Caches whose rows lie in pages of a pool: what the kernels that read and write them share.
#pragma once

#include "ec_common.h"

namespace ec {

// Slot s of sequence b is row s % page of page table[b][s / page]; page = 1 << shift, pools are [n_pages, heads, page, ...].
struct Pages {
    const int32_t* table;  // [B, max_pages]
    int n_pages, max_pages, shift;
    __host__ __device__ __forceinline__ int slots() const { return max_pages << shift; }
    __host__ __device__ __forceinline__ int page() const { return 1 << shift; }
    // Page of a slot of sequence b, or -1 where the table names none: whatever the table holds, nothing outside the pool is touched.
    __device__ __forceinline__ int page_of(int b, int slot) const
    {
        const int id = table[(size_t)b * max_pages + (slot >> shift)];
        return (unsigned)id < (unsigned)n_pages ? id : -1;
    }
    // Number of a head's row in a pool of `heads` heads a page.
    __device__ __forceinline__ size_t row(int id, int heads, int head, int slot) const
    {
        return (((size_t)id * heads + head) << shift) + (slot & ((1 << shift) - 1));
    }
};

}  // namespace ec
