// kv4.h -- layout of the paged cache of 4-bit keys and values (iseg.h), shared
// by the kernels that write and read it.
#pragma once

#include "rowops.h"

constexpr float kKvScaleMin = 8.67361738e-19f;     // 2^-60: the least scale the writer leaves

// stored width of a row of D codes
static inline int kv4_width(int64_t D) { return (int)(D <= 128 ? ceil_div64(D, 32) * 32 : ceil_div64(D, 64) * 64); }

// whether a cache's pages can be addressed by slots of 32 bits
static inline bool kv4_pages_ok(int64_t n_pages, int64_t page)
{
    return n_pages >= 0 && page >= 1 && n_pages <= ((int64_t)1 << 31) / page;
}
