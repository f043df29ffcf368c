// Caches of the drafted-token calls: where an entry lies, head-major or in pages.
#pragma once

#include "common.h"

namespace lvlm {

struct CachePlace {
    const int32_t *pages;   // null: head-major
    int Lmax, shift;        // slots per head; log2 of the page size
    int n_pages, per_head;  // pages of the pool, table places of a head
#if defined(__HIPCC__)
    // Row of the cache, seen as [rows][hd], that holds `slot` (in [0, Lmax)) of head hg; -1: a page outside the pool.
    __device__ __forceinline__ long long row(int hg, int slot) const {
        if (!pages) return (long long)hg * Lmax + slot;
        const int page = pages[(long long)hg * per_head + (slot >> shift)];
        return (unsigned)page < (unsigned)n_pages ? ((long long)page << shift) + (slot & ((1 << shift) - 1)) : -1;
    }
#endif
};
inline CachePlace cache_place(const lvlm_cache &c) {
    int shift = 0;
    while (c.pages && (1 << shift) < c.page_size) ++shift;
    return {c.pages, c.Lmax, shift, c.pages ? c.n_pages : 0, c.pages ? c.Lmax >> shift : 0};
}

}  // namespace lvlm
