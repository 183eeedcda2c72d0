// What the calls over caches held in pages share: where a row of a sequence stands, and the checks of the pages.
//
// A pool is [n_pages, Hkv, page_size, D]; row j of sequence b stands in page page_table[b, j / page_size], and a page holds a power of two of rows, so that it is found by shifts.  An entry of
// the table is clamped into the pool where it is read, and refused where it is written through, so that no table makes a call leave the pool.
#pragma once
#include "common.h"

namespace dream {

constexpr int MIN_PAGE = 16, MAX_PAGE = 256;

int paged_attn_init();      // part of dream_init()
int check_pages(const char *who, const dream_attn_desc *desc, const dream_page_desc *pages);

inline int log2_of(int32_t power) { return __builtin_ctz((unsigned)power); }

// A value that every lane of a wave wants and this launch does not write, by the scalar unit.
__device__ __forceinline__ int uniform_load(const int32_t *p) { return *(const __attribute__((address_space(4))) int32_t *)(uintptr_t)p; }

// Rows a sequence's pages hold
inline int64_t paged_rows(const dream_page_desc *pages) { return (int64_t)pages->max_pages * pages->page_size; }

}  // namespace dream
