// Plans of prompt attention and the division of the cache's attention: host code, no HIP (attention_plan.cpp).
#pragma once
#include <vector>

#include "../../include/lora_abi.h"

// Some queries of one sequence, at most LORA_ATTENTION_ROWS
struct attention_tile {
    int32_t q_row0;      // first row of q and o
    int32_t rows;
    int32_t kv_row0;     // first row of k and v of the sequence
    int32_t num_kv;      // keys of the sequence
    int32_t ahead;       // query i of the tile sees the keys [0, clamp(ahead + i + 1, 0, num_kv)); not causal: num_kv all along
    int32_t max_kv;      // keys that the last query sees
    int32_t heads;       // heads of one kv head that a workgroup takes together: 1, or 2 or 4 where the queries are few (a tile: at most so many)
    int32_t head;        // in a workgroup's item: the first of its heads
};

#define LORA_ATTENTION_ROWS 128
#define LORA_ATTENTION_MAX_ROWS (1 << 30)      /* of a batch: row numbers and sums of two stay below 2^31 */

// Threads of a workgroup, and how many workgroups of them a launch holds: fewer than 2^32 threads in all
enum { LORA_ATTENTION_THREADS = 256, LORA_CACHE_APPEND_THREADS = 320, LORA_CACHE_READ_THREADS = 256, LORA_CACHE_FINISH_THREADS = 512, LORA_CACHE_SELECT_THREADS = 1024,
       LORA_CACHE_MOVE_THREADS = 256 };
constexpr int64_t most_workgroups(int64_t threads) { return (((int64_t)1 << 32) - 1) / threads; }

struct lora_attention_plan {
    int32_t num_heads = 0, num_kv_heads = 0, head_dim = 0, dtype = 0;
    int32_t num_queries = 0, num_keys = 0;
    int32_t most_rows = LORA_ATTENTION_ROWS;      // of a tile, where wavefronts may share a tile's keys
    std::vector<attention_tile> tiles;      // most keys first
    std::vector<attention_tile> items;      // tiles with their heads, in the order of the workgroups of the tiled kernel; heads 0: nothing

    int device = -1;
    size_t d_bytes = 0;
    void* d_buf = nullptr;
    void* h_stage = nullptr;
};

// The instance of the prompts' kernel that a call takes: dims that it is made for, keys of a tile, wavefronts that share a tile's keys;
// aligned: keys and values straight to LDS
struct attention_instance {
    int32_t dims, keys, sharing, aligned;
};
// aligned: rows and heads of the call are to 16 bytes; pitch: the greater of the bytes between rows of k and between rows of v
attention_instance choose_attention(int32_t dtype, int32_t head_dim, int32_t most_rows, bool aligned, int64_t pitch);

// Rows in memory: `width` bytes each, `pitch` apart
struct memory_rows {
    int64_t at, rows, pitch, width;
    memory_rows(const void* p, int64_t rows_, int64_t ld, int64_t width_, size_t element)
        : at((int64_t)reinterpret_cast<uintptr_t>(p)), rows(rows_), pitch(ld * (int64_t)element), width(width_ * (int64_t)element) {}
    bool one_piece() const { return rows == 1 || pitch == width; }
    int64_t end() const { return at + (rows - 1) * pitch + width; }
};

// Whether an output's rows and an input's have bytes in common.  Columns of one buffer, side by side in each of its rows, have
// not.  (Rows of two different pitches, neither of them in one piece, are not looked at.)
bool share_bytes(const memory_rows& a, const memory_rows& b);

// set by the device side, so that the host code of plans links without it
extern void (*lora_attention_plan_device_release)(lora_attention_plan*);

// head_dim as the cache and the kernels hold it
inline int32_t padded_head_dim(int32_t d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

// Query rows of a tile of the cache's attention, where there are more than 16.  fp32 and 256 dims: 32 rows in three terms are more
// registers than there are (64 requests of 1000 tokens, 8 new ones, 16 heads on 4: 96 us with 32 rows, 66 with 16).
constexpr int32_t cache_tile_rows(bool f32, int32_t head_dim) { return f32 && head_dim > 128 ? 16 : 32; }

// how lora_cache_attention divides its work, from what the host knows; the workspace's parts follow from it
struct cache_division {
    int32_t row_tiles, splits, split_tokens, waves;      // waves: wavefronts of a workgroup
    size_t stats, partial, scores, total;      // bytes before each part, in all
    int64_t score_stride;
};
cache_division divide_cache_attention(const lora_cache* c, int32_t num_heads, int32_t num_tokens, int32_t max_new, bool weights);
