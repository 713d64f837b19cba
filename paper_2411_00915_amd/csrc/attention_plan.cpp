// Host side of attention: the tiles of a batch of prompts, and how the cache's attention divides its work.  No HIP calls in
// this file: everything here runs, and is tested, without a GPU.
#include <algorithm>
#include <new>

#include "attention_internal.h"

void (*lora_attention_plan_device_release)(lora_attention_plan*) = nullptr;

namespace {
bool offsets_ok(const int32_t* p, int32_t n)
{
    if (p[0] != 0) return false;
    for (int32_t i = 0; i < n; ++i)
        if (p[i + 1] < p[i]) return false;
    return true;
}

// The workgroups' work.  Workgroups go round the 8 XCDs, so every eighth item is one XCD's: it gets whole heads, one behind the
// other, so that the workgroups that run beside each other there read the same keys and values; heads that are left over
// go to the XCD that has the least to do.  Tiles of a head: most keys first.  False: more workgroups than a launch holds.
bool order_items(lora_attention_plan* p)
{
    constexpr int X = 8;
    std::vector<attention_tile> list[X];
    int64_t cost[X] = {};
    auto add = [&](int x, int32_t tile, int32_t head, int32_t heads) {
        list[x].push_back(p->tiles[tile]);
        list[x].back().head = head;
        list[x].back().heads = heads;
        cost[x] += (int64_t)p->tiles[tile].max_kv + 64;
    };
    const int32_t H = p->num_heads, group = H / p->num_kv_heads, T = (int32_t)p->tiles.size();
    // Runs of heads that belong together stay together: of 4, 2 or 1, of which a tile takes as many as it may -- but one by one
    // where that makes no more than two workgroups a compute unit (4 requests of 20 queries behind 1000 keys, 32 heads on 8: 17.0 us
    // by four, 16.2 by one).  Where most tiles have few queries, and 4 does not divide the heads of a kv head, a run is all of
    // them, taken by fours, twos and one (150 of 40 queries behind 1000 keys, 40 heads on 8: 324 us by one, 146 by four and one).
    const bool many = (int64_t)T * H > 512;
    // No more workgroups than compute units, few queries each and many keys: the wavefronts of one share its keys (8 requests of 20
    // queries behind 1000 keys, 32 heads on 8: 20.6 us without, 15.9 shared, fp32 133 and 79; 15 of them 22.7 and 26.8, as a
    // compute unit then holds one workgroup; 70 keys: 6.8 and 7.7).
    if (T > 0 && (int64_t)T * H <= 256 && p->tiles[0].max_kv > 256)
        p->most_rows = std::max_element(p->tiles.begin(), p->tiles.end(), [](const attention_tile& a, const attention_tile& b) { return a.rows < b.rows; })->rows;
    const int64_t few = std::count_if(p->tiles.begin(), p->tiles.end(), [](const attention_tile& t) { return t.heads > 1; });
    const int32_t unit = group % 4 == 0 ? 4 : many && 2 * few >= T ? group : group % 2 == 0 ? 2 : 1, units = H / unit, whole = units / X;
    auto taken = [&](int32_t t, int32_t h) {                   // from head h of a run on
        const int32_t left = unit - h;
        return !many ? 1 : std::min(p->tiles[t].heads, left >= 4 ? 4 : left >= 2 ? 2 : 1);
    };
    for (int32_t u = 0; u < whole * X; ++u)
        for (int32_t t = 0; t < T; ++t)
            for (int32_t h = 0, n; h < unit; h += n) add(u / whole, t, u * unit + h, n = taken(t, h));
    for (int32_t t = 0; t < T; ++t)
        for (int32_t u = whole * X; u < units; ++u)
            for (int32_t h = 0, n; h < unit; h += n)
                add((int)(std::min_element(cost, cost + X) - cost), t, u * unit + h, n = taken(t, h));
    size_t longest = 0;
    for (const auto& l : list) longest = std::max(longest, l.size());
    if ((int64_t)longest > most_workgroups(LORA_ATTENTION_THREADS) / X) return false;
    p->items.assign(longest * X, attention_tile{});
    for (int x = 0; x < X; ++x)
        for (size_t i = 0; i < list[x].size(); ++i) p->items[i * X + x] = list[x][i];
    return true;
}
}  // namespace

// A tile's loads straight to LDS address its rows by 32-bit offsets below 2^31 (what is behind that reads as zeros, and the chunks
// past head_dim are put there), so all rows of an aligned instance's tile have to lie within 2 GB; rows further apart than that go
// through registers.
attention_instance choose_attention(int32_t dtype, int32_t head_dim, int32_t most_rows, bool aligned, int64_t pitch)
{
    const bool f32 = dtype == LORA_F32;
    auto fits = [&](int32_t keys) { return aligned && pitch < ((int64_t)1 << 31) / keys; };
    // few queries on a chip that is not full: a workgroup's wavefronts share the keys, as many as 128 KB of LDS hold a tile for
    if (most_rows <= 32 && head_dim <= (f32 ? 64 : 128) && fits(128)) return {head_dim <= 64 ? 64 : head_dim <= 96 ? 96 : 128, 128, 4, 1};
    if (most_rows <= 64 && head_dim <= 128 && fits(f32 ? 64 : 128)) return {128, f32 ? 64 : 128, 2, 1};
    const int32_t dims = !f32 && head_dim > 64 && head_dim <= 96 ? 96 : padded_head_dim(head_dim), keys = f32 || dims == 256 ? 32 : 64;
    return {dims, keys, 1, fits(keys)};
}

bool share_bytes(const memory_rows& a, const memory_rows& b)
{
    if (a.rows < 1 || b.rows < 1 || a.end() <= b.at || b.end() <= a.at) return false;
    auto one_in_rows = [](const memory_rows& x, const memory_rows& y) {       // y's first row that ends behind x's start, if it starts before x's end
        const int64_t behind = x.at - y.at - y.width, i = behind < 0 ? 0 : y.rows == 1 ? 1 : behind / y.pitch + 1;
        return i < y.rows && y.at + i * y.pitch < x.end();
    };
    if (a.one_piece()) return one_in_rows(a, b);
    if (b.one_piece()) return one_in_rows(b, a);
    if (a.pitch != b.pitch) return false;
    const int64_t d = b.at - a.at, k = d >= 0 ? d / a.pitch : -((-d + a.pitch - 1) / a.pitch), ahead = d - k * a.pitch;      // b's row j is `ahead` behind a's row k + j
    auto both = [&](int64_t n) { return std::max<int64_t>(0, -n) < std::min(b.rows, a.rows - n); };                        // some j with 0 <= n + j < a.rows
    return (ahead < a.width && both(k)) || (ahead + b.width > a.pitch && both(k + 1));
}

extern "C" lora_status lora_attention_plan_create(const lora_attention_desc* d, lora_attention_plan** out)
{
    if (out) *out = nullptr;
    if (!d || !out || d->num_seqs < 0 || !d->q_indptr) return LORA_ERR_INVALID_ARG;
    if (d->num_heads < 1 || d->num_kv_heads < 1 || d->num_heads % d->num_kv_heads != 0) return LORA_ERR_INVALID_ARG;
    if (d->head_dim < 1 || d->head_dim > LORA_MAX_HEAD_DIM) return LORA_ERR_INVALID_ARG;
    if ((d->dtype != LORA_F32 && d->dtype != LORA_BF16) || (d->causal != 0 && d->causal != 1)) return LORA_ERR_INVALID_ARG;
    const int32_t* kv = d->kv_indptr ? d->kv_indptr : d->q_indptr;
    if (!offsets_ok(d->q_indptr, d->num_seqs) || !offsets_ok(kv, d->num_seqs)) return LORA_ERR_INVALID_ARG;
    if (d->q_indptr[d->num_seqs] > LORA_ATTENTION_MAX_ROWS || kv[d->num_seqs] > LORA_ATTENTION_MAX_ROWS) return LORA_ERR_UNSUPPORTED;
    lora_attention_plan* p = nullptr;
    try {
        p = new lora_attention_plan;
        p->num_heads = d->num_heads;
        p->num_kv_heads = d->num_kv_heads;
        p->head_dim = d->head_dim;
        p->dtype = d->dtype;
        p->num_queries = d->q_indptr[d->num_seqs];
        p->num_keys = kv[d->num_seqs];
        const int32_t group = d->num_heads / d->num_kv_heads;
        for (int32_t s = 0; s < d->num_seqs; ++s) {
            const int32_t nq = d->q_indptr[s + 1] - d->q_indptr[s], nk = kv[s + 1] - kv[s];
            for (int32_t r = 0; r < nq; r += LORA_ATTENTION_ROWS) {
                attention_tile t{};
                t.q_row0 = d->q_indptr[s] + r;
                t.rows = std::min(LORA_ATTENTION_ROWS, nq - r);
                t.kv_row0 = kv[s];
                t.num_kv = nk;
                t.ahead = d->causal ? nk - nq + r : nk;
                t.heads = group == 1 ? 1 : t.rows <= LORA_ATTENTION_ROWS / 4 ? 4 : t.rows <= LORA_ATTENTION_ROWS / 2 ? 2 : 1;
                t.max_kv = (int32_t)std::max<int64_t>(0, std::min<int64_t>(nk, (int64_t)t.ahead + t.rows));
                p->tiles.push_back(t);
            }
        }
        std::stable_sort(p->tiles.begin(), p->tiles.end(), [](const attention_tile& a, const attention_tile& b) { return a.max_kv != b.max_kv ? a.max_kv > b.max_kv : a.rows < b.rows; });
        if ((int64_t)p->tiles.size() * p->num_heads > most_workgroups(LORA_ATTENTION_THREADS) || !order_items(p)) {
            delete p;
            return LORA_ERR_UNSUPPORTED;
        }
    } catch (const std::bad_alloc&) {
        delete p;
        return LORA_ERR_NOMEM;
    }
    *out = p;
    return LORA_OK;
}

extern "C" void lora_attention_plan_destroy(lora_attention_plan* p)
{
    if (!p) return;
    if (p->d_buf && lora_attention_plan_device_release) lora_attention_plan_device_release(p);
    delete p;
}

// Not part of the ABI: the workgroups' work of the tiled kernel, eight int32 an item (attention_tile), for the plan's tests
extern "C" int32_t lora_attention_plan_items(const lora_attention_plan* p, const int32_t** items)
{
    *items = reinterpret_cast<const int32_t*>(p->items.data());
    return (int32_t)p->items.size();
}

// Not part of the ABI: the instance that a call with this plan takes (attention_instance), for tests
extern "C" void lora_attention_plan_instance(const lora_attention_plan* p, int32_t aligned, int64_t pitch, int32_t* instance)
{
    const attention_instance n = choose_attention(p->dtype, p->head_dim, p->most_rows, aligned != 0, pitch);
    instance[0] = n.dims;
    instance[1] = n.keys;
    instance[2] = n.sharing;
    instance[3] = n.aligned;
}

extern "C" size_t lora_cache_page_bytes(int32_t page_tokens, int32_t head_dim)
{
    if (page_tokens < 32 || page_tokens > 1024 || page_tokens % 32 != 0 || head_dim < 1 || head_dim > LORA_MAX_HEAD_DIM) return 0;
    return (size_t)page_tokens * (size_t)(padded_head_dim(head_dim) + 8);
}

cache_division divide_cache_attention(const lora_cache* c, int32_t num_heads, int32_t num_tokens, int32_t max_new, bool weights)
{
    const int64_t rows = (int64_t)num_heads / c->num_kv_heads * max_new;          // of a kv head and a sequence
    cache_division v{};
    v.row_tiles = (int32_t)((rows + 31) / 32);
    const int64_t wgs = (int64_t)c->num_seqs * c->num_kv_heads * v.row_tiles;
    // Long contexts are split where there are fewer workgroups than compute units: into 512, of at least 256 tokens (two blocks a
    // wavefront; 512 where there are 128 workgroups already: 160 of 260 tokens 7.8 us in one piece, 15.7 in two); and, where the
    // pieces keep 2048 tokens, beside which joining them costs little, into the 1024 that the chip holds at a time (12 requests of
    // 20000 tokens, 8 heads: 62 us in six pieces, 55 in ten; 40 of 8000: 92 in one, 79 in four; where the workgroups fill the
    // compute units evenly it is the other way round: 8 of 8000, 32 heads, 50 in one and 55 in four).
    auto pieces = [&](int64_t total, int64_t tokens) {
        return std::min<int64_t>((total + wgs - 1) / std::max<int64_t>(wgs, 1), (c->max_length + tokens - 1) / tokens);
    };
    const int64_t splits = std::max<int64_t>(1, std::max(wgs < 256 ? pieces(512, wgs < 128 ? 256 : 512) : 1, pieces(1024, 2048)));
    // In one piece, and fewer than two workgroups a compute unit: eight wavefronts each (one tile of rows, heads of up to 128; 8
    // requests of 700 tokens, 32 heads: 11.7 us with four, 10.3 with eight; with pieces to join there is nothing in it, 11.2
    // and 11.1 for one request of 2000, 55.5 and 56.4 for 12 of 20000).
    v.waves = splits == 1 && wgs < 512 && rows <= 16 && padded_head_dim(c->head_dim) <= 128 ? 8 : 4;
    v.split_tokens = (int32_t)std::max<int64_t>(128, ((c->max_length + splits - 1) / splits + 127) / 128 * 128);
    v.splits = (int32_t)std::max<int64_t>(1, ((int64_t)c->max_length + v.split_tokens - 1) / v.split_tokens);
    const size_t out_rows = (size_t)num_tokens * num_heads;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off = (off + bytes + 255) / 256 * 256; return o; };
    v.stats = take(v.splits > 1 || weights ? out_rows * v.splits * 8 : 0);
    v.partial = take(v.splits > 1 ? out_rows * v.splits * c->head_dim * 4 : 0);
    v.score_stride = ((int64_t)c->max_length + 31) / 32 * 32;
    v.scores = take(weights ? out_rows * (size_t)v.score_stride * 4 : 0);
    v.total = off;
    return v;
}
