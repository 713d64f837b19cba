// Host side of attention under sanitizers (tests/test_attention_sanitizers.py): plans of random and of extreme batches, whose items
// have to cover every query of every head once, and the division of the cache's attention.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "../paper_2411_00915_amd/csrc/attention_internal.h"

#define CHECK(x)                                                              \
    do {                                                                      \
        if (!(x)) {                                                           \
            std::fprintf(stderr, "line %d: %s\n", __LINE__, #x);              \
            std::exit(1);                                                     \
        }                                                                     \
    } while (0)

static void plans(std::mt19937& rng)
{
    auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
    for (int round = 0; round < 300; ++round) {
        const int S = pick(0, 90), kv = pick(1, 9), group = pick(1, 9), H = kv * group;
        std::vector<int32_t> q(S + 1, 0), k(S + 1, 0);
        for (int s = 0; s < S; ++s) {
            q[s + 1] = q[s] + (pick(0, 3) ? pick(0, 40) : pick(0, 600));
            k[s + 1] = k[s] + (pick(0, 3) ? pick(0, 300) : pick(0, 9) ? 0 : 1 << 20);
        }
        const lora_attention_desc d{S, q.data(), round % 2 ? k.data() : nullptr, H, kv, pick(1, 256), pick(0, 1), pick(0, 1)};
        lora_attention_plan* p = nullptr;
        CHECK(lora_attention_plan_create(&d, &p) == LORA_OK && p);
        std::vector<int> seen((size_t)q[S] * H, 0);
        for (const attention_tile& t : p->items) {
            if (t.heads == 0) continue;
            CHECK(t.rows >= 1 && t.rows * t.heads <= LORA_ATTENTION_ROWS && t.head / group == (t.head + t.heads - 1) / group);
            for (int r = 0; r < t.rows; ++r)
                for (int h = 0; h < t.heads; ++h) ++seen[(size_t)(t.q_row0 + r) * H + t.head + h];
        }
        for (int n : seen) CHECK(n == 1);
        lora_attention_plan_destroy(p);
    }
    // a query and the longest rows there are
    for (int32_t keys : {0, 1, LORA_ATTENTION_MAX_ROWS}) {
        const int32_t q[] = {0, 1, 300}, k[] = {0, 0, keys};
        for (int causal = 0; causal < 2; ++causal) {
            const lora_attention_desc d{2, q, k, 8, 2, 64, LORA_BF16, causal};
            lora_attention_plan* p = nullptr;
            CHECK(lora_attention_plan_create(&d, &p) == LORA_OK);
            for (const attention_tile& t : p->items) CHECK(t.heads == 0 || (t.max_kv >= 0 && t.max_kv <= t.num_kv));
            lora_attention_plan_destroy(p);
        }
    }
}

static void divisions(std::mt19937& rng)
{
    auto upto = [&](double most) { return (int64_t)std::exp2(std::uniform_real_distribution<double>(0, most)(rng)); };
    for (int round = 0; round < 20000; ++round) {
        lora_cache c{};
        c.num_seqs = (int32_t)upto(13);
        c.num_kv_heads = (int32_t)upto(6);
        c.head_dim = (int32_t)(1 + rng() % 256);
        c.page_tokens = 32;
        c.max_length = round % 9 ? (int32_t)upto(30) : round % 2 ? 1 << 30 : 0;
        const int32_t H = c.num_kv_heads * (int32_t)upto(4), max_new = (int32_t)upto(10), tokens = (int32_t)std::min<int64_t>((int64_t)c.num_seqs * max_new, 1 << 30);
        if ((int64_t)tokens * H > INT32_MAX || (int64_t)tokens * H > ((int64_t)1 << 40) / std::max(1, c.max_length)) continue;
        const bool weights = rng() % 2;
        const cache_division v = divide_cache_attention(&c, H, tokens, max_new, weights);
        CHECK(v.splits >= 1 && v.split_tokens >= 128 && v.split_tokens % 128 == 0 && (int64_t)v.splits * v.split_tokens >= c.max_length);
        CHECK((int64_t)(v.splits - 1) * v.split_tokens <= c.max_length && (int64_t)v.splits * v.split_tokens <= INT32_MAX);
        CHECK((int64_t)v.row_tiles * 32 >= (int64_t)(H / c.num_kv_heads) * max_new);
        CHECK(v.waves == 4 || (v.waves == 8 && v.splits == 1));
        const size_t rows = (size_t)tokens * H;
        CHECK(v.partial - v.stats >= (v.splits > 1 || weights ? rows * v.splits * 8 : 0));
        CHECK(v.scores - v.partial >= (v.splits > 1 ? rows * v.splits * c.head_dim * 4 : 0));
        CHECK(v.total - v.scores >= (weights ? rows * (size_t)v.score_stride * 4 : 0) && v.score_stride >= c.max_length);
        CHECK(v.total % 256 == 0 && (v.total == 0) == (v.splits == 1 && !weights));
    }
}

int main()
{
    std::mt19937 rng(24);
    plans(rng);
    divisions(rng);
    std::printf("sanitize_attention: ok\n");
}
