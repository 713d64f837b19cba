// The pages that a query attends to: bounds of a page's keys, and the choice by them (include/lora_abi.h, ATTENTION OVER CHOSEN PAGES).
//
// A key of the page has upper[d] >= k[d] >= lower[d], so q . k <= sum max(q[d], 0) upper[d] + min(q[d], 0) lower[d]: what the choice
// orders pages by.  Bounds and queries are whole numbers of 8 bits, so the sums are exact whatever their order, and what follows is
// one rounding each: the choice is the definition's, page by page, which a sum in floating point would not be.
//
// Bounds of 8192 tokens' pages, 8 heads of 128: 10.6 us, of which the trips offsets -> length -> table -> codes are most.  The choice for 8
// requests of 8000 tokens, 8 kv heads: 6.4 us (lengths 0.6, table and bounds 2.4, products 1, the choice 2); 32 of 16384,
// 17 MB of bounds, 11; four tokens over 131072, in pieces: 6.4 and 8.5 (in one launch 32: a compute unit reads 512 KB in 21 us).
#include <hip/hip_runtime.h>

#include "cache_format.h"
#include "kernels_choose.h"
#include "launch.h"

namespace {

typedef __attribute__((__vector_size__(4 * sizeof(int)))) int int4v;

// ---------------------------------------------------------------------------
// Bounds: a wavefront a page of one head.  A lane has 8 dims of every so-manieth token (DP/8 lanes a token), the lanes of the same dims
// meet by exchange.
__device__ __forceinline__ float max_of_wave(float x)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off, 64));
    return x;
}

template <int DP>
__global__ __launch_bounds__(256) void cache_digest_kernel(cache_args c, int8_t* bounds, float* steps, int pages)
{
    constexpr int LANES = DP / 8, TOKENS = 64 / LANES;         // lanes a token, tokens at a time
    const int lane = threadIdx.x & 63;
    int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int head = (int)(id % c.kv_heads);
    id /= c.kv_heads;
    const int i = (int)(id % pages);
    if (id / pages >= c.num_seqs) return;
    const int s = (int)(id / pages);
    const cache_rows rows = rows_of(c, s);
    const int length = length_of(c, s), n = min(rows.count, c.max_new);
    if (n == 0 || length == 0) return;
    // (as many tokens as the call's are the last ones; of those that are left out past max_new the last are)
    const int number = page_number(c, max(0, length - rows.count)) + i, first = number * c.page_tokens;
    if (first >= length - rows.count + n) return;
    const int64_t page = page_of(c, s, number);
    if (page < 0) return;
    const int held = min(c.page_tokens, length - first), word = lane % LANES, token = lane / LANES;
    const unsigned char* const base = c.pages + (page * c.kv_heads + head) * c.page_bytes;
    float high[8], low[8];
    bool wild = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        high[e] = -INFINITY;
        low[e] = INFINITY;
    }
    // 32 tokens at a time, the next ones' loads on their way
    constexpr int LOADS = 32 / TOKENS;
    uint32_t codes[LOADS], words[LOADS];
    auto load = [&](int first_token) {
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            const int at = min(first_token + k * TOKENS + token, held - 1);        // (those behind the last: the last once more)
            codes[k] = *reinterpret_cast<const uint32_t*>(base + at * (DP / 2) + 4 * word);
            words[k] = *reinterpret_cast<const uint32_t*>(base + word_offset<DP>(c.page_tokens, at, 0));
        }
    };
    load(0);
#pragma unroll 1
    for (int t = 0; t < held; t += 32) {
        uint32_t now[LOADS], w[LOADS];
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            now[k] = codes[k];
            w[k] = words[k];
        }
        if (t + 32 < held) load(t + 32);
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            const float step = __uint_as_float(w[k] << 16), zero = __uint_as_float(w[k] & 0xffff0000u);
            wild |= !(fabsf(step) < INFINITY && fabsf(zero) < INFINITY);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = (float)(now[k] >> (4 * e) & 15u) * step + zero;
                high[e] = fmaxf(high[e], x);
                low[e] = fminf(low[e], x);
            }
        }
    }
    float most = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int off = LANES; off < 64; off <<= 1) {
            high[e] = fmaxf(high[e], __shfl_xor(high[e], off, 64));
            low[e] = fminf(low[e], __shfl_xor(low[e], off, 64));
        }
        if (8 * word + e < c.head_dim) most = fmaxf(most, fmaxf(fabsf(high[e]), fabsf(low[e])));
    }
    most = max_of_wave(most);
    float step = most * (1.f / 127.f);
    if (step < 0x1p-100f) step = 0.f;
    if (__ballot(wild) || !(most < INFINITY)) step = __builtin_nanf("");
    const bool none = !(step > 0.f);
    if (lane >= LANES) return;
    uint32_t up[2] = {0, 0}, down[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const bool there = !none && 8 * word + e < c.head_dim;
        const int u = there ? (int)fminf(ceilf(high[e] / step), 127.f) : 0, d = there ? (int)fmaxf(floorf(low[e] / step), -127.f) : 0;
        up[e / 4] |= (uint32_t)(u & 255) << (8 * (e % 4));
        down[e / 4] |= (uint32_t)(d & 255) << (8 * (e % 4));
    }
    int8_t* const out = bounds + (page * c.kv_heads + head) * (2 * DP) + 8 * word;
    *reinterpret_cast<uint2*>(out) = uint2{up[0], up[1]};
    *reinterpret_cast<uint2*>(out + DP) = uint2{down[0], down[1]};
    if (lane == 0) steps[page * c.kv_heads + head] = step;
}

// ---------------------------------------------------------------------------
// The choice: a workgroup a token and kv head.  Its queries' codes, parted by sign, are rows of a product with the pages' bounds as columns, 16
// queries and 16 pages at a time, on the matrix cores in whole numbers; a column's greatest goes to LDS as a whole number in the
// order of the scores (or to the workspace, where there are more pages than LDS holds, or several workgroups share a token's pages).  Then
// the last page chosen is found and the pages are written in order: by one wavefront, bit by bit, without a barrier (up to 256 pages: 2 us; 5.5 for
// 400), or by all, by bins (2.7 and 0.8).

// scores in their order as whole numbers above 0; NaN above them, what is chosen in any case above all
constexpr uint32_t kForced = 0xffffffffu, kNan = 0xfffffffeu;
__device__ __forceinline__ uint32_t order_of(float x)
{
    if (x != x) return kNan;
    const uint32_t u = __float_as_uint(x + 0.f);               // (-0 is +0)
    return u >> 31 ? ~u : u | 0x80000000u;
}

// the greater, NaN above all
__device__ __forceinline__ float greater(float x, float y) { return y > x || y != y ? y : x; }

constexpr int kThreads = LORA_CACHE_CHOOSE_THREADS, kWaves = kThreads / 64;

// 16 codes of a page's bounds, and what makes a score of them, for 16 pages a wavefront at a time, ROUNDS of them on their way together (four: 0.8 us
// more for 125 pages, whose table entries are then asked for in vain)
template <int DP>
struct bounds_block {
    static constexpr int NS = 2 * DP / 64, ROUNDS = 2, PAGES = ROUNDS * kWaves * 16;
    int4v b[ROUNDS][NS];
    float step[ROUNDS];
    bool there[ROUNDS];

    // pages first ... of `end`; what is not there is loaded from page 0
    __device__ __forceinline__ void load(const choose_args& a, const int32_t* table, int head, int first, int end, int wave, int lane)
    {
        const cache_args& c = a.c;
        int64_t at[ROUNDS];
#pragma unroll
        for (int u = 0; u < ROUNDS; ++u) {
            const int n = first + (u * kWaves + wave) * 16 + (lane & 15);
            const int page = n < end ? table[n] : -1;
            there[u] = page >= 0 && page < c.num_pages;
            at[u] = (int64_t)(there[u] ? page : 0) * c.kv_heads + head;
        }
#pragma unroll
        for (int u = 0; u < ROUNDS; ++u) {
            if (first + (u * kWaves + wave) * 16 >= end) continue;             // (the wavefront's 16 together)
            const int8_t* const p = a.bounds + at[u] * (2 * DP) + 16 * (lane >> 4);
#pragma unroll
            for (int m = 0; m < NS; ++m) b[u][m] = *reinterpret_cast<const int4v*>(p + 64 * m);
            step[u] = a.steps[at[u]];
        }
    }
};

// The queries' codes, parted by sign: 16 lanes a query, DP/16 dims each
template <typename T, int DP>
struct query_codes {
    static constexpr int E = DP / 16;
    float x[E];
    __device__ __forceinline__ void load(const choose_args& a, int row, int head, int h0, int tid)
    {
        const int D = a.c.head_dim, l = tid & 15, h = min(h0 + (tid >> 4 & 15), a.group - 1);
        const T* const q = static_cast<const T*>(a.q) + (int64_t)row * a.ldq + (int64_t)(head * a.group + h) * D;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = elem<T>::load(q + min(l * E + e, D - 1));
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = l * E + e < D ? x[e] : 0.f;
    }
    __device__ __forceinline__ void make(int8_t (*codes)[2 * DP], float* units, int tid) const
    {
        if (tid >= 256) return;
        const int l = tid & 15, h = tid >> 4;
        float most = 0.f, wild = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            most = fmaxf(most, fabsf(x[e]));
            wild = __builtin_fmaf(x[e], 0.f, wild);
        }
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) {
            most = fmaxf(most, __shfl_xor(most, off, 16));
            wild += __shfl_xor(wild, off, 16);
        }
        float unit = most * (1.f / 127.f);
        if (unit < 0x1p-100f) unit = 0.f;
        if (wild != 0.f) unit = __builtin_nanf("");
        uint32_t up[(E + 3) / 4] = {}, down[(E + 3) / 4] = {};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int v = unit > 0.f ? (int)fminf(fmaxf(rintf(x[e] / unit), -127.f), 127.f) : 0;
            up[e / 4] |= (uint32_t)max(v, 0) << (8 * (e % 4));
            down[e / 4] |= ((uint32_t)min(v, 0) & 255u) << (8 * (e % 4));
        }
#pragma unroll
        for (int w = 0; w < E / 4; ++w) {
            *reinterpret_cast<uint32_t*>(&codes[h][l * E + 4 * w]) = up[w];
            *reinterpret_cast<uint32_t*>(&codes[h][DP + l * E + 4 * w]) = down[w];
        }
        if (l == 0) units[h] = unit;
    }
};

// The budget-th largest of `pages` keys, and how many of its like are wanted, 8 bits at a time (workgroup)
__device__ __forceinline__ void threshold_by_bins(const uint32_t* keys, int pages, int budget, int* bins, uint32_t* found, int tid, uint32_t* threshold, int* equal)
{
    const int lane = tid & 63;
    uint32_t prefix = 0;
    int wanted = budget;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int n = tid; n < 256; n += kThreads) bins[n] = 0;
        __syncthreads();
        const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
        for (int n = tid; n < pages; n += kThreads) {
            const uint32_t key = keys[n];
            if ((key & mask) == prefix) atomicAdd(&bins[key >> shift & 255], 1);
        }
        __syncthreads();
        if (tid < 64) {                                        // from the top: the bin in which the wanted number is reached
            int mine[4], sum = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += mine[e] = bins[255 - (4 * lane + e)];
            const int upto = wave_sum_upto(sum);
            int above = upto - sum;
            if (above < wanted && upto >= wanted)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (above < wanted && above + mine[e] >= wanted) {
                        found[0] = prefix | (uint32_t)(255 - (4 * lane + e)) << shift;
                        found[1] = wanted - above;
                    }
                    above += mine[e];
                }
        }
        __syncthreads();
        prefix = found[0];
        wanted = (int)found[1];
    }
    *threshold = prefix;
    *equal = wanted;
}

// how many lanes before this one are in the mask, on top of n
__device__ __forceinline__ int lanes_before(uint64_t mask, int n)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, (uint32_t)n));
#else
    return n;
#endif
}

// The choice among up to 64 N keys, by one wavefront without a barrier: the budget-th largest bit by bit, done as soon as as many as wanted are not
// below a number; then the pages in order.  (Eight wavefronts, each for itself, are in each other's way in the scalar unit: 3.9 us for 400 keys;
// counts in lanes that are summed up across them, for up to 256 pages 0.4 us slower, for up to 512 0.6 than by bins.)
template <int N>
__device__ __forceinline__ void choose_by_bits(const uint32_t* keys, int pages, int budget, bool all, int lane, int32_t* out)
{
    uint32_t k[N], t = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) k[i] = i * 64 + lane < pages ? keys[i * 64 + lane] : 0u;
    int equal = -1;                                            // of those that are t, so many are wanted
    if (!all) {
#pragma unroll 1
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t next = t | 1u << bit;
            int count = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) count += __popcll(__ballot(k[i] >= next));
            if (count >= budget) t = next;
            if (count == budget) {
                --t;                                           // (all that are above it)
                equal = 0;
                break;
            }
        }
        if (equal < 0) {
            equal = budget;
#pragma unroll
            for (int i = 0; i < N; ++i) equal -= __popcll(__ballot(k[i] > t));
        }
    }
    int at = 0, same = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        bool is = k[i] > t;
        if (equal > 0) {
            const bool like = k[i] == t && k[i] != 0;          // (0: a page that is not there)
            const uint64_t mask = __ballot(like);
            is |= like && lanes_before(mask, same) < equal;
            same += __popcll(mask);
        }
        const uint64_t mask = __ballot(is);
        if (is) out[lanes_before(mask, at)] = i * 64 + lane;
        at += __popcll(mask);
    }
    for (int n = at + lane; n < budget; n += 64) out[n] = -1;
}

constexpr int kBoth = 0, kScores = 1, kChoice = 2;      // what a launch does: keys and choice; keys of a piece of the pages; the choice

template <typename T, int DP, int WHAT>
__global__ __launch_bounds__(kThreads, DP == 256 ? 2 : 4) void cache_choose_kernel(choose_args a)
{
    typedef bounds_block<DP> block;
    constexpr int NS = block::NS;
    extern __shared__ __align__(16) uint32_t near[];           // keys of the pages, where they fit
    __shared__ __align__(16) int8_t codes[WHAT == kChoice ? 1 : 16][2 * DP];
    __shared__ float units[16];
    __shared__ int bins[256], counts[2][kWaves];
    __shared__ uint32_t found[2];
    const cache_args& c = a.c;
    int id = blockIdx.x;
    const int piece = WHAT == kScores ? id % a.pieces : 0;
    if constexpr (WHAT == kScores) id /= a.pieces;
    const int head = id % c.kv_heads;
    id /= c.kv_heads;
    const int i = id % c.max_new, s = id / c.max_new;
    const cache_rows rows = rows_of(c, s);
    if (i >= rows.count) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = rows.first + i;
    const int sees = max(0, length_of(c, s) - rows.count + i + 1), pages = sees == 0 ? 0 : page_number(c, sees - 1) + 1;
    const int budget = a.budget, last = pages - a.recent;
    const int32_t* const table = c.page_table + (int64_t)s * c.table_stride;
    uint32_t* const keys = WHAT != kBoth || a.keys ? a.keys + ((int64_t)row * c.kv_heads + head) * a.key_stride : near;
    const bool all = pages <= budget || c.num_pages == 0;      // no need to know their order
    if constexpr (WHAT != kChoice) {
        const int begin = WHAT == kScores ? piece * a.piece_pages : 0, end = WHAT == kScores ? min(pages, begin + a.piece_pages) : pages;
        if (all) {
            for (int n = begin + tid; n < end; n += kThreads) keys[n] = table[n] < 0 || table[n] >= c.num_pages ? 0u : kForced;
        } else if (begin < end) {
            query_codes<T, DP> q;
            block now;
            q.load(a, row, head, 0, tid);                      // (asked for before the pages' bounds, and used while these are on their way)
            now.load(a, table, head, begin, end, wave, lane);
            for (int h0 = 0; h0 < a.group; h0 += 16) {
                if (h0 > 0) {
                    __syncthreads();
                    q.load(a, row, head, h0, tid);
                }
                q.make(codes, units, tid);
                __syncthreads();
                const int r = lane & 15, g = lane >> 4;
                int4v query[NS];
#pragma unroll
                for (int n = 0; n < NS; ++n) query[n] = *reinterpret_cast<const int4v*>(&codes[WHAT == kChoice ? 0 : r][64 * n + 16 * g]);
                float unit[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) unit[e] = units[4 * g + e];
                const int valid = a.group - h0 - 4 * g;        // of the lane's four rows
                for (int first = begin; first < end; first += block::PAGES) {
                    if (first > begin || h0 > 0) now.load(a, table, head, first, end, wave, lane);
#pragma unroll
                    for (int u = 0; u < block::ROUNDS; ++u) {
                        const int n = first + (u * kWaves + wave) * 16 + r;
                        if (n - r >= end) continue;
                        int4v sum = {0, 0, 0, 0};
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
                        for (int m = 0; m < NS; ++m) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(query[m], now.b[u][m], sum, 0, 0, 0);
#endif
                        float most = -INFINITY;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (e < valid) most = greater(most, (float)sum[e] * unit[e]);
                        most = greater(most, __shfl_xor(most, 16, 64));
                        most = greater(most, __shfl_xor(most, 32, 64));
                        if (g == 0 && n < end) {
                            uint32_t key = !now.there[u] ? 0u : n < a.first || n >= last ? kForced : order_of(most * now.step[u]);
                            if (h0 > 0) key = max(key, keys[n]);               // (products with a step not below 0 are in their order)
                            keys[n] = key;
                        }
                    }
                }
            }
        }
        if constexpr (WHAT == kScores) return;
        __syncthreads();
    }
    if constexpr (WHAT != kScores) {
        int32_t* const out = a.chosen + ((int64_t)row * c.kv_heads + head) * budget;
        if (pages <= 256) {
            if (wave == 0) choose_by_bits<4>(keys, pages, budget, all, lane, out);
            return;
        }
        uint32_t threshold = 1;
        int equal = budget;                                    // (all that are there)
        if (!all) threshold_by_bins(keys, pages, budget, bins, found, tid, &threshold, &equal);
        // in order, four pages a thread: above it, all; equal to it, the first few; a page that is not there never
        int written = 0, same = 0;
        for (int n0 = 0; n0 < pages; n0 += 4 * kThreads) {
            uint32_t above = 0, like = 0;                      // of the thread's four
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int n = n0 + 4 * tid + e;
                const uint32_t key = n < pages ? keys[n] : 0u;
                above |= (uint32_t)(key > threshold) << e;
                like |= (uint32_t)(key == threshold && key != 0) << e;
            }
            auto upto = [&](int n, int* into, int* base) {     // of the workgroup's threads before this one, on top of *base, which becomes all
                const int mine = wave_sum_upto(n);
                __syncthreads();
                if (lane == 63) into[wave] = mine;
                __syncthreads();
                int before = *base + mine - n;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    before += w < wave ? into[w] : 0;
                    *base += into[w];
                }
                return before;
            };
            if (equal > 0) {
                int before = upto(__popc(like), counts[0], &same);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (like >> e & 1) {
                        if (before < equal) above |= 1u << e;
                        ++before;
                    }
            }
            int at = upto(__popc(above), counts[1], &written);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (above >> e & 1) {
                    if (at < budget) out[at] = n0 + 4 * tid + e;
                    ++at;
                }
        }
        for (int n = written + tid; n < budget; n += kThreads) out[n] = -1;
    }
}

template <typename T, int DP>
void launch_dims(const choose_args& a, hipStream_t stream)
{
    const uint32_t wgs = (uint32_t)((int64_t)a.c.num_seqs * a.c.max_new * a.c.kv_heads);
    const dim3 block(kThreads);
    if (a.pieces > 1) {
        LORA_LAUNCH(LORA_K_CACHE_SCORES, (cache_choose_kernel<T, DP, kScores>), dim3(wgs * (uint32_t)a.pieces), block, 0, stream, a);
        LORA_LAUNCH(LORA_K_CACHE_CHOOSE, (cache_choose_kernel<T, DP, kChoice>), dim3(wgs), block, 0, stream, a);
    } else
        LORA_LAUNCH(LORA_K_CACHE_CHOOSE, (cache_choose_kernel<T, DP, kBoth>), dim3(wgs), block, a.keys ? 0u : (uint32_t)a.key_stride * 4, stream, a);
}

template <typename T>
hipError_t launch_choose(const choose_args& a, hipStream_t stream)
{
    switch (padded_head_dim(a.c.head_dim)) {
        case 64: launch_dims<T, 64>(a, stream); break;
        case 128: launch_dims<T, 128>(a, stream); break;
        default: launch_dims<T, 256>(a, stream);
    }
    return hipGetLastError();
}
}  // namespace

hipError_t launch_cache_digest(const cache_args& c, int8_t* bounds, float* steps, hipStream_t stream)
{
    const int pages = digest_pages(c.max_new, c.page_tokens);
    const dim3 grid((uint32_t)(((int64_t)c.num_seqs * pages * c.kv_heads + 3) / 4)), block(256);
    switch (padded_head_dim(c.head_dim)) {
        case 64: LORA_LAUNCH(LORA_K_CACHE_DIGEST, (cache_digest_kernel<64>), grid, block, 0, stream, c, bounds, steps, pages); break;
        case 128: LORA_LAUNCH(LORA_K_CACHE_DIGEST, (cache_digest_kernel<128>), grid, block, 0, stream, c, bounds, steps, pages); break;
        default: LORA_LAUNCH(LORA_K_CACHE_DIGEST, (cache_digest_kernel<256>), grid, block, 0, stream, c, bounds, steps, pages);
    }
    return hipGetLastError();
}

hipError_t launch_cache_choose(const choose_args& a, int32_t dtype, hipStream_t stream)
{
    return dtype == LORA_F32 ? launch_choose<float>(a, stream) : launch_choose<bf16_t>(a, stream);
}
