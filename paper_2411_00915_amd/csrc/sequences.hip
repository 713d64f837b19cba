// C-ABI entry points of pages and of beams: argument checks, what is launched.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>

#include "attention_internal.h"
#include "kernels_sequences.h"

namespace {
bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
lora_status status_of(hipError_t e)
{
    if (e == hipSuccess) return LORA_OK;
    (void)hipGetLastError();
    return LORA_ERR_DEVICE;
}

lora_status check_pages(const lora_pages* p)
{
    if (!p || p->num_seqs < 0 || p->num_pages < 0 || p->table_stride < 0 || p->max_length < 0) return LORA_ERR_INVALID_ARG;
    if (lora_cache_page_bytes(p->page_tokens, 1) == 0 || p->max_length > (int64_t)p->table_stride * p->page_tokens) return LORA_ERR_INVALID_ARG;
    if (p->num_seqs == 0) return LORA_OK;
    if (!p->length || (p->table_stride > 0 && !p->page_table) || (p->num_pages > 0 && !p->users)) return LORA_ERR_INVALID_ARG;
    if (misaligned(p->page_table, 4) || misaligned(p->length, 4) || misaligned(p->users, 4)) return LORA_ERR_INVALID_ARG;
    if (p->num_seqs > LORA_PAGES_MAX_SEQS || p->max_length > LORA_ATTENTION_MAX_ROWS) return LORA_ERR_UNSUPPORTED;
    if (p->num_pages > INT32_MAX / p->page_tokens - p->num_seqs) return LORA_ERR_UNSUPPORTED;
    // (launches of a thread an entry)
    return (int64_t)p->num_seqs * p->table_stride > most_workgroups(256) * 256 ? LORA_ERR_UNSUPPORTED : LORA_OK;
}

pages_args args_of(const lora_pages* p)
{
    return pages_args{p->page_table, p->length, p->users, (int32_t)p->num_pages, p->num_seqs, p->table_stride, p->max_length, p->page_tokens};
}

// some memory of the call: nothing where there is none
struct piece {
    const void* at;
    int64_t bytes;
};
bool share(const piece& a, const piece& b)
{
    if (!a.at || !b.at || a.bytes < 1 || b.bytes < 1) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
    return x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes;
}
// the first `outputs` of the pieces with any of them
bool share_any(std::initializer_list<piece> pieces, int outputs)
{
    for (int i = 0; i < outputs; ++i)
        for (int j = i + 1; j < (int)pieces.size(); ++j)
            if (share(pieces.begin()[i], pieces.begin()[j])) return true;
    return false;
}
}  // namespace

extern "C" lora_status lora_pages_workspace(const lora_pages* p, size_t* bytes)
{
    if (!bytes) return LORA_ERR_INVALID_ARG;
    *bytes = 0;
    const lora_status st = check_pages(p);
    if (st == LORA_OK && p->num_seqs > 0) *bytes = pages_workspace(p->num_pages, p->num_seqs, p->table_stride);
    return st;
}

extern "C" lora_status lora_pages_resize(const lora_pages* p, const int32_t* wanted, int32_t num_tokens, int32_t* granted, int32_t* indptr, int32_t* token_seq,
                                         int32_t* token_position, int64_t* token_slot, int32_t* copies, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    const lora_status st = check_pages(p);
    if (st != LORA_OK) return st;
    if (num_tokens < 0 || misaligned(wanted, 4) || misaligned(granted, 4) || misaligned(indptr, 4) || misaligned(token_seq, 4) || misaligned(token_position, 4) ||
        misaligned(token_slot, 8) || misaligned(copies, 4))
        return LORA_ERR_INVALID_ARG;
    if (p->num_seqs == 0) return indptr ? status_of(launch_pages_none(indptr, static_cast<hipStream_t>(hip_stream))) : LORA_OK;
    if (!wanted || !copies) return LORA_ERR_INVALID_ARG;
    const size_t need = pages_workspace(p->num_pages, p->num_seqs, p->table_stride);
    if (!workspace || workspace_bytes < need || misaligned(workspace, 256)) return LORA_ERR_WORKSPACE;
    const int64_t S = p->num_seqs, T = num_tokens;
    if (share_any({{granted, 4 * S}, {indptr, 4 * S + 4}, {token_seq, 4 * T}, {token_position, 4 * T}, {token_slot, 8 * T}, {copies, 8 * S}, {workspace, (int64_t)need},
                   {p->page_table, 4 * S * p->table_stride}, {p->length, 4 * S}, {p->users, 4 * p->num_pages}, {wanted, 4 * S}}, 10))
        return LORA_ERR_INVALID_ARG;
    // (the last of its launches: refused before the first has changed anything)
    if (!one_workgroup_resizes(S, p->table_stride, T) && S * write_chunks(p->table_stride, p->max_length, T, token_seq || token_position || token_slot) > most_workgroups(64) - 4)
        return LORA_ERR_UNSUPPORTED;
    char* const w = static_cast<char*>(workspace);
    const resize_args a{args_of(p), wanted, num_tokens, granted, indptr, token_seq, token_position, token_slot, copies, reinterpret_cast<page_grant*>(w),
                        reinterpret_cast<int32_t*>(w + pages_parts_offset(p->num_seqs)), reinterpret_cast<int32_t*>(w + pages_list_offset(p->num_seqs, p->num_pages))};
    return status_of(launch_pages_resize(a, static_cast<hipStream_t>(hip_stream)));
}

extern "C" lora_status lora_pages_fork(const lora_pages* p, const int32_t* parent, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    const lora_status st = check_pages(p);
    if (st != LORA_OK) return st;
    if (misaligned(parent, 4)) return LORA_ERR_INVALID_ARG;
    if (p->num_seqs == 0) return LORA_OK;
    if (!parent) return LORA_ERR_INVALID_ARG;
    const size_t need = pages_workspace(p->num_pages, p->num_seqs, p->table_stride);
    if (!workspace || workspace_bytes < need || misaligned(workspace, 256)) return LORA_ERR_WORKSPACE;
    const int64_t S = p->num_seqs;
    if (share_any({{workspace, (int64_t)need}, {p->page_table, 4 * S * p->table_stride}, {p->length, 4 * S}, {p->users, 4 * p->num_pages}, {parent, 4 * S}}, 4))
        return LORA_ERR_INVALID_ARG;
    return status_of(launch_pages_fork(args_of(p), parent, static_cast<int32_t*>(workspace), static_cast<hipStream_t>(hip_stream)));
}

namespace {
lora_status check_beams(int32_t num_groups, int32_t beams, int32_t vocab, int32_t num_out)
{
    if (num_groups < 0 || beams < 1 || beams > LORA_MAX_BEAMS || vocab < 1 || vocab > 1 << 24 || num_out < 1 || num_out > LORA_MAX_BEAMS) return LORA_ERR_INVALID_ARG;
    if ((int64_t)num_groups * beams > LORA_ATTENTION_MAX_ROWS) return LORA_ERR_UNSUPPORTED;
    int32_t unit, chunk, splits;
    divide_beams((int64_t)num_groups * beams, vocab, &unit, &chunk, &splits);
    return (int64_t)num_groups * beams > most_workgroups(BEAM_THREADS) / splits || num_groups > most_workgroups(BEAM_JOIN_THREADS) ? LORA_ERR_UNSUPPORTED : LORA_OK;
}
}  // namespace

extern "C" lora_status lora_beam_workspace(int32_t num_groups, int32_t beams, int32_t vocab, int32_t num_out, size_t* bytes)
{
    if (!bytes) return LORA_ERR_INVALID_ARG;
    *bytes = 0;
    const lora_status st = check_beams(num_groups, beams, vocab, num_out);
    if (st != LORA_OK || num_groups == 0) return st;
    int32_t unit, chunk, splits;
    divide_beams((int64_t)num_groups * beams, vocab, &unit, &chunk, &splits);
    *bytes = beam_workspace((int64_t)num_groups * beams, splits, num_out);
    return LORA_OK;
}

extern "C" lora_status lora_beam_select(int32_t dtype, int32_t num_groups, int32_t beams, int32_t vocab, const void* logits, int64_t ld, const float* score,
                                        const int32_t* last_token, int32_t end_token, int32_t num_out, float* out_score, int32_t* out_parent, int32_t* out_token,
                                        void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (dtype != LORA_F32 && dtype != LORA_BF16) return LORA_ERR_INVALID_ARG;
    const lora_status st = check_beams(num_groups, beams, vocab, num_out);
    if (st != LORA_OK) return st;
    if (end_token >= 1 << 24) return LORA_ERR_INVALID_ARG;
    if (num_groups == 0) return LORA_OK;
    const size_t e = dtype == LORA_F32 ? 4 : 2;
    if (!logits || !score || !out_score || !out_parent || !out_token || ld < vocab || misaligned(logits, e) || misaligned(score, 4) || misaligned(last_token, 4) ||
        misaligned(out_score, 4) || misaligned(out_parent, 4) || misaligned(out_token, 4))
        return LORA_ERR_INVALID_ARG;
    beam_args a{};
    const int64_t rows = (int64_t)num_groups * beams, out = 4 * (int64_t)num_groups * num_out;
    divide_beams(rows, vocab, &a.unit, &a.chunk, &a.splits);
    const size_t need = beam_workspace(rows, a.splits, num_out);
    if (!workspace || workspace_bytes < need || misaligned(workspace, 256)) return LORA_ERR_WORKSPACE;
    if (ld > ((int64_t)1 << 60) / rows) return LORA_ERR_UNSUPPORTED;
    if (share_any({{out_score, out}, {out_parent, out}, {out_token, out}, {workspace, (int64_t)need}, {score, 4 * rows}, {last_token, 4 * rows}}, 4))
        return LORA_ERR_INVALID_ARG;
    const memory_rows in(logits, rows, ld, vocab, e);
    for (const piece& x : {piece{out_score, out}, piece{out_parent, out}, piece{out_token, out}, piece{workspace, (int64_t)need}})
        if (share_bytes(memory_rows(x.at, 1, 1, x.bytes, 1), in)) return LORA_ERR_INVALID_ARG;
    char* const w = static_cast<char*>(workspace);
    a.logits = logits;
    a.ld = ld;
    a.score = score;
    a.last_token = last_token;
    a.end_token = end_token;
    a.num_groups = num_groups;
    a.beams = beams;
    a.vocab = vocab;
    a.num_out = num_out;
    a.out_score = out_score;
    a.out_parent = out_parent;
    a.out_token = out_token;
    a.sums = reinterpret_cast<beam_sum*>(w);
    a.entries = reinterpret_cast<beam_entry*>(w + beam_entries_offset(rows, a.splits));
    return status_of(launch_beam_select(a, dtype, static_cast<hipStream_t>(hip_stream)));
}
