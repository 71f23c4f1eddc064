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

// Sum over the wave's lanes up to this one, of int or uint32_t.
template <typename T> __device__ __forceinline__ T wave_scan(T x_)
{
    static_assert(sizeof(T) == 4);
    int x = (int)x_;
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // the last lane of a row to the next one (rows 1, 3)
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to rows 2, 3
    return (T)x;
}

}  // namespace ec
