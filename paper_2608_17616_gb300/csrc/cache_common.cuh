// What the kernels over a paged cache (cache.cu, cache_attention.cu) share: a context's length and the place of a
// position, both from device memory and checked in every build.
#pragma once

#include "mone_common.cuh"

namespace mone {

__device__ __forceinline__ void cache_fail(int* status, int site) {
    atomicOr(status, DEV_CHECK);
    atomicCAS(status + 1, 0, site);
}

// Positions that context c holds; a length that its table cannot cover counts as what it covers.
__device__ __forceinline__ int cache_len(const CacheView& v, int c) {
    const int n = v.lens[c];
    if (n < 0 || n > v.cap) {
        cache_fail(v.status, DS_CACHE_LEN);
        return n < 0 ? 0 : (int)v.cap;
    }
    return n;
}

// Page of a table entry, -1 (and an error latched) where it is outside the pool.
__device__ __forceinline__ int cache_page(const CacheView& v, const int* table, int block) {
    const int p = table[block];
    if ((unsigned)p < (unsigned)v.n_pages) return p;
    cache_fail(v.status, DS_CACHE_PAGE);
    return -1;
}

// Whether every row of head_dim elements of the pools starts on a 16-byte boundary.
inline bool cache_vec(const CacheView& v, int el) {
    return (((uintptr_t)v.K | (uintptr_t)v.V) & 15u) == 0 && v.s_layer * el % 16 == 0 && v.s_page * el % 16 == 0 &&
           v.s_head * el % 16 == 0 && v.s_pos * el % 16 == 0;
}

}  // namespace mone
