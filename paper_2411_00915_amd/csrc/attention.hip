// C-ABI entry points of attention and of its cache: argument checks, plan upload, what is launched.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "kernels.h"
#include "kernels_attention.h"

namespace {
bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
size_t elem_bytes(int32_t dtype) { return dtype == LORA_F32 ? 4 : 2; }
bool known(int32_t dtype) { return dtype == LORA_F32 || dtype == LORA_BF16; }
lora_status status_of(hipError_t e)
{
    if (e == hipSuccess) return LORA_OK;
    (void)hipGetLastError();
    return LORA_ERR_DEVICE;
}

void release_tiles(lora_attention_plan* p)
{
    lora_give_tables(p->device, p->d_bytes, p->d_buf, p->h_stage);
    p->d_buf = p->h_stage = nullptr;
}
struct install_release { install_release() { lora_attention_plan_device_release = release_tiles; } } g_install_release;

lora_status ensure_uploaded(lora_attention_plan* p, hipStream_t stream)
{
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return LORA_ERR_DEVICE;
    if (p->d_buf) return p->device == dev ? LORA_OK : LORA_ERR_INVALID_ARG;      // a plan lives on one device
    const size_t items = p->items.size() * sizeof(attention_tile), bytes = std::max<size_t>(items, 64);
    size_t cls = 0;
    void *dbuf = nullptr, *hbuf = nullptr;
    const lora_status st = lora_take_tables(dev, bytes, &cls, &dbuf, &hbuf);
    if (st != LORA_OK) return st;
    std::memcpy(hbuf, p->items.data(), items);
    if (hipMemcpyAsync(dbuf, hbuf, bytes, hipMemcpyHostToDevice, stream) != hipSuccess) {
        (void)hipGetLastError();
        lora_give_tables(dev, cls, dbuf, hbuf);
        return LORA_ERR_DEVICE;
    }
    p->device = dev;
    p->d_buf = dbuf;
    p->d_bytes = cls;
    p->h_stage = hbuf;
    return LORA_OK;
}

// the descriptor's own consistency; LORA_OK also where there is no sequence
lora_status check_cache(const lora_cache* c)
{
    if (!c || c->num_seqs < 0 || c->num_pages < 0 || c->table_stride < 0 || c->max_length < 0 || c->num_kv_heads < 1) return LORA_ERR_INVALID_ARG;
    if (lora_cache_page_bytes(c->page_tokens, c->head_dim) == 0) return LORA_ERR_INVALID_ARG;
    if (c->max_length > (int64_t)c->table_stride * c->page_tokens) return LORA_ERR_INVALID_ARG;
    if (c->num_seqs == 0) return LORA_OK;
    if (!c->pages || !c->page_table || !c->length) return LORA_ERR_INVALID_ARG;
    if (misaligned(c->pages, 16) || misaligned(c->weight, 4) || misaligned(c->page_table, 4) || misaligned(c->length, 4)) return LORA_ERR_INVALID_ARG;
    if (c->num_pages >= (int64_t)1 << 31 || c->max_length > LORA_ATTENTION_MAX_ROWS) return LORA_ERR_UNSUPPORTED;
    return LORA_OK;
}

// of the last tokens' packing
lora_status check_tokens(const lora_cache* c, int32_t dtype, int32_t num_tokens, int32_t max_new, const int32_t* d_indptr)
{
    if (!known(dtype) || num_tokens < 0 || max_new < 0 || misaligned(d_indptr, 4)) return LORA_ERR_INVALID_ARG;
    if (num_tokens > LORA_ATTENTION_MAX_ROWS) return LORA_ERR_UNSUPPORTED;
    return check_cache(c);
}

// of lora_cache_attention: rows, workgroups and the workspace's parts that the kernels' 32- and 64-bit numbers hold
lora_status check_rows(const lora_cache* c, int32_t num_heads, int32_t num_tokens, int32_t max_new)
{
    if (num_heads < 1 || num_heads % c->num_kv_heads != 0) return LORA_ERR_INVALID_ARG;
    const int64_t rows = (int64_t)num_tokens * num_heads;
    if (rows > INT32_MAX || (int64_t)c->num_seqs * max_new > INT32_MAX / num_heads) return LORA_ERR_UNSUPPORTED;
    // (the launch behind the attention's: up to a workgroup for 2048 slots, beside those of the rows to be joined, which are fewer)
    if ((int64_t)c->num_seqs * c->num_kv_heads > most_workgroups(2 * LORA_CACHE_FINISH_THREADS) / (c->max_length / 2048 + 1)) return LORA_ERR_UNSUPPORTED;
    if (rows > ((int64_t)1 << 40) / std::max<int64_t>(c->max_length, 1)) return LORA_ERR_UNSUPPORTED;
    return LORA_OK;
}

// of the cache's pages
bool share_bytes(const memory_rows& a, const lora_cache* c)
{
    const int64_t page = (int64_t)lora_cache_page_bytes(c->page_tokens, c->head_dim), most = INT64_MAX / 2 / page / c->num_kv_heads;
    return c->num_pages > 0 && share_bytes(a, memory_rows(c->pages, 1, 1, std::min(c->num_pages, most) * c->num_kv_heads * page, 1));
}

cache_args args_of(const lora_cache* c, int32_t num_tokens, int32_t max_new, const int32_t* d_indptr)
{
    cache_args a{};
    a.pages = static_cast<unsigned char*>(c->pages);
    a.weight = c->weight;
    a.page_table = c->page_table;
    a.length = c->length;
    a.indptr = d_indptr;
    a.num_pages = c->num_pages;
    a.page_bytes = (int64_t)lora_cache_page_bytes(c->page_tokens, c->head_dim);
    a.num_seqs = c->num_seqs;
    a.table_stride = c->table_stride;
    a.max_length = c->max_length;
    a.page_tokens = c->page_tokens;
    a.kv_heads = c->num_kv_heads;
    a.head_dim = c->head_dim;
    a.num_tokens = num_tokens;
    a.max_new = max_new;
    return a;
}
}  // namespace

extern "C" lora_status lora_attention_plan_upload(lora_attention_plan* p, void* hip_stream)
{
    return p ? ensure_uploaded(p, static_cast<hipStream_t>(hip_stream)) : LORA_ERR_INVALID_ARG;
}

extern "C" lora_status lora_attention(lora_attention_plan* p, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                                      void* o, int64_t ldo, float scale, void* hip_stream)
{
    if (!p || !std::isfinite(scale)) return LORA_ERR_INVALID_ARG;
    if (p->items.empty()) return LORA_OK;
    const int64_t q_row = (int64_t)p->num_heads * p->head_dim, kv_row = (int64_t)p->num_kv_heads * p->head_dim;
    const size_t e = elem_bytes(p->dtype);
    if (!q || !o || ldq < q_row || ldo < q_row || misaligned(q, e) || misaligned(o, e)) return LORA_ERR_INVALID_ARG;
    if (p->num_keys > 0 && (!k || !v || ldk < kv_row || ldv < kv_row || misaligned(k, e) || misaligned(v, e))) return LORA_ERR_INVALID_ARG;
    const memory_rows out(o, p->num_queries, ldo, q_row, e);
    if (share_bytes(out, memory_rows(q, p->num_queries, ldq, q_row, e)) || share_bytes(out, memory_rows(k, p->num_keys, ldk, kv_row, e)) ||
        share_bytes(out, memory_rows(v, p->num_keys, ldv, kv_row, e)))
        return LORA_ERR_INVALID_ARG;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const lora_status st = ensure_uploaded(p, stream);
    if (st != LORA_OK) return st;
    const attention_args a{static_cast<const attention_tile*>(p->d_buf), (int32_t)p->items.size(), p->most_rows, p->num_heads / p->num_kv_heads, p->head_dim,
                           q, k, v, o, ldq, ldk, ldv, ldo, scale};
    return status_of(launch_attention(a, p->dtype, stream));
}

extern "C" lora_status lora_cache_append(const lora_cache* c, int32_t dtype, int32_t num_tokens, int32_t max_new, const int32_t* d_indptr, const void* k,
                                         int64_t ldk, const void* v, int64_t ldv, void* hip_stream)
{
    const lora_status st = check_tokens(c, dtype, num_tokens, max_new, d_indptr);
    if (st != LORA_OK) return st;
    if (num_tokens == 0 || max_new == 0 || c->num_seqs == 0) return LORA_OK;
    const int64_t row = (int64_t)c->num_kv_heads * c->head_dim;
    if (!k || !v || ldk < row || ldv < row || misaligned(k, elem_bytes(dtype)) || misaligned(v, elem_bytes(dtype))) return LORA_ERR_INVALID_ARG;
    if (tiles_of_tokens(num_tokens) > most_workgroups(LORA_CACHE_APPEND_THREADS) / c->num_kv_heads) return LORA_ERR_UNSUPPORTED;
    const memory_rows keys(k, num_tokens, ldk, row, elem_bytes(dtype)), values(v, num_tokens, ldv, row, elem_bytes(dtype));
    if (share_bytes(keys, c) || share_bytes(values, c)) return LORA_ERR_INVALID_ARG;
    return status_of(launch_cache_append(args_of(c, num_tokens, std::min(max_new, num_tokens), d_indptr), dtype, k, ldk, v, ldv, static_cast<hipStream_t>(hip_stream)));
}

extern "C" lora_status lora_cache_read(const lora_cache* c, int32_t dtype, int32_t num_tokens, int32_t max_new, const int32_t* d_indptr, void* k, int64_t ldk,
                                       void* v, int64_t ldv, void* hip_stream)
{
    const lora_status st = check_tokens(c, dtype, num_tokens, max_new, d_indptr);
    if (st != LORA_OK) return st;
    if (num_tokens == 0 || max_new == 0 || c->num_seqs == 0) return LORA_OK;
    const int64_t row = (int64_t)c->num_kv_heads * c->head_dim;
    if (!k || !v || ldk < row || ldv < row || misaligned(k, elem_bytes(dtype)) || misaligned(v, elem_bytes(dtype))) return LORA_ERR_INVALID_ARG;
    if (tiles_of_tokens(num_tokens) > most_workgroups(LORA_CACHE_READ_THREADS) / c->num_kv_heads) return LORA_ERR_UNSUPPORTED;
    const memory_rows keys(k, num_tokens, ldk, row, elem_bytes(dtype)), values(v, num_tokens, ldv, row, elem_bytes(dtype));
    if (share_bytes(keys, c) || share_bytes(values, c) || share_bytes(keys, values)) return LORA_ERR_INVALID_ARG;
    return status_of(launch_cache_read(args_of(c, num_tokens, std::min(max_new, num_tokens), d_indptr), dtype, k, ldk, v, ldv, static_cast<hipStream_t>(hip_stream)));
}

extern "C" lora_status lora_cache_workspace(const lora_cache* c, int32_t num_heads, int32_t num_tokens, int32_t max_new, int32_t weights, size_t* bytes)
{
    if (!bytes) return LORA_ERR_INVALID_ARG;
    *bytes = 0;
    lora_status st = check_tokens(c, LORA_BF16, num_tokens, max_new, nullptr);
    if (st != LORA_OK) return st;
    max_new = std::min(max_new, num_tokens);                   // (no sequence has more)
    st = check_rows(c, num_heads, num_tokens, max_new);
    if (st != LORA_OK) return st;
    if (num_tokens > 0 && max_new > 0 && c->num_seqs > 0) *bytes = divide_cache_attention(c, num_heads, num_tokens, max_new, weights != 0).total;
    return LORA_OK;
}

extern "C" lora_status lora_cache_attention(const lora_cache* c, int32_t dtype, int32_t num_heads, int32_t num_tokens, int32_t max_new,
                                            const int32_t* d_indptr, const void* q, int64_t ldq, void* o, int64_t ldo, float scale, float decay,
                                            void* workspace, size_t workspace_bytes, void* hip_stream)
{
    lora_status st = check_tokens(c, dtype, num_tokens, max_new, d_indptr);
    if (st != LORA_OK) return st;
    if (!std::isfinite(scale) || !(decay <= 1.f)) return LORA_ERR_INVALID_ARG;
    max_new = std::min(max_new, num_tokens);
    st = check_rows(c, num_heads, num_tokens, max_new);
    if (st != LORA_OK) return st;
    const bool weights = decay >= 0.f;
    if (weights && c->num_seqs > 0 && !c->weight) return LORA_ERR_INVALID_ARG;
    if (num_tokens == 0 || max_new == 0 || c->num_seqs == 0) return LORA_OK;
    const int64_t row = (int64_t)num_heads * c->head_dim;
    if (!q || !o || ldq < row || ldo < row || misaligned(q, elem_bytes(dtype)) || misaligned(o, elem_bytes(dtype))) return LORA_ERR_INVALID_ARG;
    const memory_rows out(o, num_tokens, ldo, row, elem_bytes(dtype));
    if (share_bytes(out, memory_rows(q, num_tokens, ldq, row, elem_bytes(dtype))) || share_bytes(out, c)) return LORA_ERR_INVALID_ARG;
    const cache_division v = divide_cache_attention(c, num_heads, num_tokens, max_new, weights);
    if (v.total > 0 && (!workspace || workspace_bytes < v.total || misaligned(workspace, 256))) return LORA_ERR_WORKSPACE;
    const int64_t rows = (int64_t)num_heads / c->num_kv_heads * max_new, tile = cache_tile_rows(dtype == LORA_F32, c->head_dim), row_tiles = (rows + tile - 1) / tile;
    if ((int64_t)c->num_seqs * c->num_kv_heads * v.splits > most_workgroups(64 * v.waves) / std::max<int64_t>(1, row_tiles)) return LORA_ERR_UNSUPPORTED;
    char* const w = static_cast<char*>(workspace);
    cache_attention_args a{};
    a.c = args_of(c, num_tokens, max_new, d_indptr);
    a.q = q;
    a.o = o;
    a.ldq = ldq;
    a.ldo = ldo;
    a.num_heads = num_heads;
    a.group = num_heads / c->num_kv_heads;
    a.scale = scale;
    a.decay = decay;
    a.row_tiles = (int32_t)row_tiles;
    a.splits = v.splits;
    a.split_tokens = v.split_tokens;
    a.waves = v.waves;
    a.stats = v.splits > 1 || weights ? reinterpret_cast<float2*>(w + v.stats) : nullptr;
    a.partial = v.splits > 1 ? reinterpret_cast<float*>(w + v.partial) : nullptr;
    a.scores = weights ? reinterpret_cast<float*>(w + v.scores) : nullptr;
    a.score_stride = v.score_stride;
    return status_of(launch_cache_attention(a, dtype, static_cast<hipStream_t>(hip_stream)));
}

extern "C" lora_status lora_cache_evict(const lora_cache* source, const lora_cache* target, int32_t budget, int32_t recent, int32_t* kept, void* hip_stream)
{
    lora_status st = check_cache(source);
    if (st == LORA_OK) st = check_cache(target);
    if (st != LORA_OK) return st;
    if (budget < 0 || recent < 0 || recent > budget) return LORA_ERR_INVALID_ARG;
    if (source->num_seqs != target->num_seqs || source->num_kv_heads != target->num_kv_heads || source->head_dim != target->head_dim ||
        source->page_tokens != target->page_tokens || target->max_length < budget)
        return LORA_ERR_INVALID_ARG;
    if (source->num_seqs == 0) return LORA_OK;
    if (!source->weight || !target->weight || (budget > 0 && !kept) || misaligned(kept, 4) || source->length == target->length) return LORA_ERR_INVALID_ARG;
    const int64_t heads = (int64_t)source->num_seqs * source->num_kv_heads;
    if (heads > most_workgroups(LORA_CACHE_SELECT_THREADS) || heads > most_workgroups(LORA_CACHE_MOVE_THREADS) / (budget / 32 + 1)) return LORA_ERR_UNSUPPORTED;
    return status_of(launch_cache_evict(args_of(source, 0, 0, nullptr), args_of(target, 0, 0, nullptr), target->length, budget, recent, kept,
                                        static_cast<hipStream_t>(hip_stream)));
}
