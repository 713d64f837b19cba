// Launch interface of the pages' bounds and of the choice among them (kernels_choose.hip).
#pragma once
#include "kernels_attention.h"

enum { LORA_CACHE_DIGEST_THREADS = 256, LORA_CACHE_CHOOSE_THREADS = 512 };

// pages that hold some of n tokens in a row, at most
inline int32_t digest_pages(int32_t n, int32_t page_tokens) { return (int32_t)(((int64_t)n + 2 * page_tokens - 2) / page_tokens); }

struct choose_args {
    cache_args c;
    const void* q;
    int64_t ldq;
    int32_t group, budget, first, recent;
    const int8_t* bounds;
    const float* steps;
    int32_t* chosen;
    uint32_t* keys;          // workspace: [num_tokens][kv_heads][key_stride]; null: in LDS
    int64_t key_stride;
    int32_t pieces, piece_pages;       // of a token's pages, a workgroup each, in a launch before the choice's; 1: one launch
};

// pages of the longest sequence, whose keys LDS holds up to (beside 9 KB of queries and counts)
constexpr int32_t LORA_CACHE_CHOOSE_NEAR = 12288;

// Pieces of a token's pages: of the longest sequence's (strides of keys, whole 32s) at least 256 each, as many as make two workgroups a compute unit
inline int32_t choose_pieces(int64_t workgroups, int64_t stride)
{
    const int64_t most = stride / 256, wanted = workgroups > 0 ? 512 / workgroups : 1;
    return (int32_t)(most < 2 || wanted < 2 ? 1 : most < wanted ? most : wanted);
}

hipError_t launch_cache_digest(const cache_args& c, int8_t* bounds, float* steps, hipStream_t stream);
hipError_t launch_cache_choose(const choose_args& a, int32_t dtype, hipStream_t stream);
