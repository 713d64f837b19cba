// Launch interface between the entry points of attention and of the cache (attention.hip) and the kernels.  Every function
// enqueues on `stream` and returns the HIP status of the launch.
#pragma once
#include <hip/hip_runtime.h>

#include "attention_internal.h"

struct attention_args {
    const attention_tile* items;
    int32_t num_items, most_rows, group, head_dim;      // most_rows: see lora_attention_plan; group: query heads of a kv head
    const void *q, *k, *v;
    void* o;
    int64_t ldq, ldk, ldv, ldo;
    float scale;
};

hipError_t launch_attention(const attention_args& a, int32_t dtype, hipStream_t stream);

// What the kernels of the cache take: the descriptor's fields by value
struct cache_args {
    unsigned char* pages;
    float* weight;
    const int32_t* page_table;
    const int32_t* length;
    const int32_t* indptr;       // null: one token a sequence
    int64_t num_pages;
    int64_t page_bytes;          // of one head
    int32_t num_seqs, table_stride, max_length, page_tokens, kv_heads, head_dim;
    int32_t num_tokens, max_new;
};

struct cache_attention_args {
    cache_args c;
    const void* q;
    void* o;
    int64_t ldq, ldo;
    int32_t num_heads, group;
    float scale, decay;          // decay < 0: weights are left alone
    int32_t row_tiles, splits, split_tokens, waves;
    float2* stats;               // [num_tokens * num_heads][splits] maximum and sum
    float* partial;              // [num_tokens * num_heads][splits][head_dim], where splits > 1
    float* scores;               // [num_tokens * num_heads][score_stride], where weights are wanted
    int64_t score_stride;
};

// The cache's tokens go in and out in tiles of 32 packed rows, a workgroup one of a head
inline int64_t tiles_of_tokens(int64_t tokens) { return (tokens + 31) / 32; }

hipError_t launch_cache_append(const cache_args& c, int32_t dtype, const void* k, int64_t ldk, const void* v, int64_t ldv, hipStream_t stream);
hipError_t launch_cache_read(const cache_args& c, int32_t dtype, void* k, int64_t ldk, void* v, int64_t ldv, hipStream_t stream);
hipError_t launch_cache_attention(const cache_attention_args& a, int32_t dtype, hipStream_t stream);
hipError_t launch_cache_evict(const cache_args& source, const cache_args& target, int32_t* target_length, int32_t budget, int32_t recent, int32_t* kept,
                              hipStream_t stream);
