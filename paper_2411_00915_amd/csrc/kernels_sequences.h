// Launch interface between the entry points of pages and beams (sequences.hip) and the kernels, and what the host decides for them.
// Every launch function enqueues on `stream` and returns the HIP status.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/lora_abi.h"

constexpr int32_t LORA_PAGES_MAX_SEQS = 1 << 14;

// The descriptor by value, and where the workspace's parts are
struct pages_args {
    int32_t *page_table, *length, *users;
    int32_t num_pages, num_seqs, table_stride, max_length, page_tokens;
};

// What a sequence gets, from the launch that decides to the one that writes it down
struct page_grant {
    int32_t from, to;       // length before and after
    int32_t first;          // of its new pages in the list of free pages; bit 31: the first of them is a copy
    int32_t row;            // of its first new token
    // (before the launch that decides: lengths held and wanted, the page that would be written and has other users or -1, and whether the wanted one is a length)
};

struct resize_args {
    pages_args p;
    const int32_t* wanted;
    int32_t num_tokens;
    int32_t *granted, *indptr, *token_seq, *token_position;
    int64_t* token_slot;
    int32_t* copies;
    page_grant* grants;     // workspace: [num_seqs]
    int32_t* part_first;    // workspace: [free_parts]
    int32_t* list;          // workspace: [num_pages] free pages in order, each part of the pool's at its place, or all from the start
};

// Parts of the pool whose free pages a workgroup looks for
constexpr int FREE_PART = 4096;
constexpr int free_parts(int64_t num_pages) { return (int)((num_pages + FREE_PART - 1) / FREE_PART); }

// workspace of the two calls: grants, parts and list; the new table, new and old lengths
inline size_t pages_parts_offset(int64_t num_seqs) { return ((size_t)num_seqs * sizeof(page_grant) + 255) / 256 * 256; }
inline size_t pages_list_offset(int64_t num_seqs, int64_t num_pages) { return pages_parts_offset(num_seqs) + ((size_t)free_parts(num_pages) * 4 + 255) / 256 * 256; }
inline size_t pages_workspace(int64_t num_pages, int64_t num_seqs, int64_t table_stride)
{
    const size_t resize = pages_list_offset(num_seqs, num_pages) + (size_t)num_pages * 4, fork = (size_t)num_seqs * (size_t)table_stride * 4 + (size_t)num_seqs * 8;
    return ((resize > fork ? resize : fork) + 255) / 256 * 256;
}

// Whether one workgroup does all of a resize: 1024 sequences, and as many entries and tokens as it writes in the time of another launch
inline bool one_workgroup_resizes(int64_t num_seqs, int64_t table_stride, int64_t num_tokens)
{
    return num_seqs <= 1024 && num_seqs * table_stride <= 32 * 1024 && num_tokens <= 16 * 1024;
}
// Else wavefronts of a sequence's entries, 1024 each, and of its new tokens, too, where these are wanted
constexpr int PAGES_CHUNK = 1024;
inline int64_t entry_chunks(int64_t table_stride) { return table_stride < PAGES_CHUNK ? 1 : (table_stride + PAGES_CHUNK - 1) / PAGES_CHUNK; }
inline int64_t write_chunks(int64_t table_stride, int64_t max_length, int64_t num_tokens, bool tokens)
{
    const int64_t rows = tokens ? ((num_tokens < max_length ? num_tokens : max_length) + PAGES_CHUNK - 1) / PAGES_CHUNK : 0, entries = entry_chunks(table_stride);
    return rows > entries ? rows : entries;
}

hipError_t launch_pages_resize(const resize_args& a, hipStream_t stream);
hipError_t launch_pages_none(int32_t* indptr, hipStream_t stream);
hipError_t launch_pages_fork(const pages_args& p, const int32_t* parent, int32_t* workspace, hipStream_t stream);

struct beam_sum {
    double sum, ref;         // of exp(logit - ref); no finite number where one of the logits is NaN or +inf
};
struct beam_entry {
    float logit;
    int32_t token;           // -1: none
};

// Beams.  A workgroup takes `chunk` tokens of a row, a unit at a time
struct beam_args {
    const void* logits;
    int64_t ld;
    const float* score;
    const int32_t* last_token;
    int32_t end_token, num_groups, beams, vocab, num_out, unit, chunk, splits;
    float* out_score;
    int32_t *out_parent, *out_token;
    beam_sum* sums;                 // workspace: [rows][splits]
    beam_entry* entries;            // workspace: [rows][splits][num_out], greatest first
};
constexpr int BEAM_THREADS = 256, BEAM_JOIN_THREADS = 512, BEAM_FEW = 8, BEAM_MANY = 16;      // (the last two: tokens a thread takes)

// Chunks of a row: units of 4096 tokens, or of 2048 where those would be fewer than two workgroups a compute unit; and as many units a
// workgroup, one after the other, as leave four workgroups a compute unit (bounds carry on, and there is less to join)
inline void divide_beams(int64_t rows, int32_t vocab, int32_t* unit, int32_t* chunk, int32_t* splits)
{
    const int32_t many = BEAM_THREADS * BEAM_MANY, few = BEAM_THREADS * BEAM_FEW, units = (vocab + many - 1) / many;
    if (rows * units < 512 || vocab < many) {
        *unit = *chunk = few;
    } else {
        const int64_t together = rows * units / 1024 < 1 ? 1 : rows * units / 1024 < units ? rows * units / 1024 : units;
        const int32_t pieces = (int32_t)((units + together - 1) / together);
        *unit = many;
        *chunk = (units + pieces - 1) / pieces * many;             // (evenly)
    }
    *splits = (vocab + *chunk - 1) / *chunk;
}
inline size_t beam_entries_offset(int64_t rows, int32_t splits) { return ((size_t)rows * splits * sizeof(beam_sum) + 255) / 256 * 256; }
inline size_t beam_workspace(int64_t rows, int32_t splits, int32_t num_out)
{
    return (beam_entries_offset(rows, splits) + (size_t)rows * splits * num_out * sizeof(beam_entry) + 255) / 256 * 256;
}

hipError_t launch_beam_select(const beam_args& a, int32_t dtype, hipStream_t stream);
