// The paged cache as the kernels see it (include/cats.h: cats_paged_kv): where a row of a sequence lies.
#pragma once

#include "cats_kernels.cuh"

namespace cats {

// n / d for 0 <= n < 2^31 and 1 <= d <= 2^26: with 2^(L-1) < d <= 2^L, mul = ceil(2^(31+L) / d) fits 32 bits and is less than
// 2^L / d over, so n mul / 2^(31+L) is less than 1 / d over n / d.
struct Divisor {
    uint32_t mul;
    int shift;
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (uint32_t)(((uint64_t)n * mul) >> shift); }
};
inline Divisor divisor(uint32_t d) {
    int l = 0;
    while ((1u << l) < d) ++l;
    return {(uint32_t)((((uint64_t)1 << (31 + l)) + d - 1) / d), 31 + l};
}

// Whether a row that starts at unit `at` lies `behind` units behind one at `at0`.  The last unit of a cache of 2^36 bytes is 2^32 - 1, and at0 + behind may pass it:
// the sum is 0 then, where another row may lie.
__host__ __device__ __forceinline__ bool lies_behind(uint32_t at0, uint32_t at, uint32_t behind) { return at >= at0 && at - at0 == behind; }

struct PagedDev {
    uint8_t *k, *v;
    float *ks, *vs;                         // int8 caches
    uint32_t page16, row16, head16;         // strides in units of 16 bytes
    uint32_t s_page, s_row, s_head;         // strides of the scales in elements
    int n_pages, page_size, n_kv;
    Divisor by_page;
    const int32_t* table;
    long long ld_table;
    int width, n_seqs;

    struct Row { uint32_t at, s; };         // of head 0: in units of 16 bytes behind k and v, and in elements behind ks and vs
    __device__ __forceinline__ Row row_of(uint32_t page, uint32_t in_page) const { return {page * page16 + in_page * row16, page * s_page + in_page * s_row}; }
    // false: outside the tables
    __device__ __forceinline__ bool locate(int seq, int pos, Row& r) const {
        if ((unsigned)seq >= (unsigned)n_seqs) return false;
        const uint32_t nth = by_page((uint32_t)pos);
        if (nth >= (uint32_t)width) return false;
        const int page = table[seq * ld_table + nth];
        if ((unsigned)page >= (unsigned)n_pages) return false;
        r = row_of((uint32_t)page, (uint32_t)pos - nth * (uint32_t)page_size);
        return true;
    }
};

}  // namespace cats
