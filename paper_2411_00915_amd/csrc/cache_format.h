// The format of the cache's pages (include/lora_abi.h, THE CACHE) as the kernels address it, and what they read of the
// descriptor's device arrays, kept within its bounds.
#pragma once
#include "device_util.h"
#include "kernels_attention.h"

struct cache_rows {
    int first, count;      // packed rows of a sequence
};

__device__ __forceinline__ cache_rows rows_of(const cache_args& c, int s)
{
    if (!c.indptr) return cache_rows{s, s < c.num_tokens ? 1 : 0};
    const int first = min(max(c.indptr[s], 0), c.num_tokens);
    return cache_rows{first, min(max(c.indptr[s + 1], first), c.num_tokens) - first};
}

__device__ __forceinline__ int length_of(const cache_args& c, int s) { return min(max(c.length[s], 0), c.max_length); }

// the page that a slot is in (pages are mostly powers of two)
__device__ __forceinline__ int page_number(const cache_args& c, int slot)
{
    return (c.page_tokens & (c.page_tokens - 1)) == 0 ? slot >> __builtin_ctz(c.page_tokens) : slot / c.page_tokens;
}

// page number `page` of sequence s in the pool, or -1.  page < table_stride: slots are below max_length
__device__ __forceinline__ int64_t page_of(const cache_args& c, int s, int page)
{
    const int id = c.page_table[(int64_t)s * c.table_stride + page];
    return id >= 0 && id < c.num_pages ? id : -1;
}

// bytes from the start of a page of one head: lane r's codes of the token at place `at`, dims (DP/16) r ...
template <int DP>
__device__ __forceinline__ int key_offset(int at, int r) { return at * (DP / 2) + r * (DP / 32); }
template <int DP>
__device__ __forceinline__ int value_offset(int page_tokens, int at, int r)
{
    return page_tokens * (DP / 2) + (at >> 5) * (DP * 16) + ((((at >> 3) & 3) * 16 + r) * 8 + (at & 7)) * (DP / 32);
}
// part 0: of the keys, 1: of the values
template <int DP>
__device__ __forceinline__ int word_offset(int page_tokens, int at, int part) { return page_tokens * DP + (part * page_tokens + at) * 4; }

// DP/16 codes of a lane
template <int DP>
__device__ __forceinline__ void load_codes(const unsigned char* p, uint32_t* w)
{
    if constexpr (DP == 64) w[0] = *reinterpret_cast<const uint16_t*>(p);
    else
#pragma unroll
        for (int i = 0; i < DP / 128; ++i) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
}
template <int DP>
__device__ __forceinline__ void store_codes(unsigned char* p, const uint32_t* w)
{
    if constexpr (DP == 64) *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
    else
#pragma unroll
        for (int i = 0; i < DP / 128; ++i) reinterpret_cast<uint32_t*>(p)[i] = w[i];
}
