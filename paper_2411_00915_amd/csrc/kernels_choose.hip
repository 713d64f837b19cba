// The pages that a query attends to: bounds of a page's keys, and the choice by them (include/lora_abi.h, ATTENTION OVER CHOSEN PAGES).
//
// A key of the page has upper[d] >= k[d] >= lower[d], so q . k <= sum max(q[d], 0) upper[d] + min(q[d], 0) lower[d]: what the choice
// orders pages by.  Bounds and queries are whole numbers of 8 bits, so the sums are exact whatever their order, and what follows is
// one rounding each: the choice is the definition's, page by page, which a sum in floating point would not be.
#include <hip/hip_runtime.h>

#include "cache_format.h"
#include "kernels_choose.h"
#include "launch.h"

namespace {

typedef __attribute__((__vector_size__(4 * sizeof(int)))) int int4v;

// ---------------------------------------------------------------------------
// Bounds: a wavefront a page of one head.  A lane has 8 dims of every so-manieth token (DP/8 lanes a token), the lanes of the same dims
// meet by exchange.  Bound by the instructions that take the codes apart.
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
#pragma unroll 4
    for (int t = token; t < c.page_tokens; t += TOKENS) {
        const int at = min(t, held - 1);                       // (those behind the last: the last once more)
        const uint32_t codes = *reinterpret_cast<const uint32_t*>(base + at * (DP / 2) + 4 * word);
        const uint32_t w = *reinterpret_cast<const uint32_t*>(base + word_offset<DP>(c.page_tokens, at, 0));
        const float step = __uint_as_float(w << 16), zero = __uint_as_float(w & 0xffff0000u);
        wild |= !(fabsf(step) < INFINITY && fabsf(zero) < INFINITY);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = (float)(codes >> (4 * e) & 15u) * step + zero;
            high[e] = fmaxf(high[e], x);
            low[e] = fminf(low[e], x);
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
// order of the scores (or to the workspace, where there are more pages than LDS holds).  Then the number of the last page chosen
// is found 8 bits at a time, and the pages are written in order.

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

__device__ __forceinline__ int lanes_before(uint64_t mask, int n)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, (uint32_t)n));
#else
    return n;
#endif
}

constexpr int kThreads = LORA_CACHE_CHOOSE_THREADS, kWaves = kThreads / 64;

template <typename T, int DP>
__global__ __launch_bounds__(kThreads) void cache_choose_kernel(choose_args a)
{
    constexpr int NS = 2 * DP / 64;                            // products of 64 codes
    extern __shared__ __align__(16) uint32_t near[];           // keys of the pages, where they fit
    __shared__ __align__(16) int8_t codes[16][2 * DP];
    __shared__ float units[16];
    __shared__ int bins[256], counts[2][kWaves];
    __shared__ uint32_t found[2];
    const cache_args& c = a.c;
    int id = blockIdx.x;
    const int head = id % c.kv_heads;
    id /= c.kv_heads;
    const int i = id % c.max_new, s = id / c.max_new;
    const cache_rows rows = rows_of(c, s);
    if (i >= rows.count) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = rows.first + i;
    const int sees = max(0, length_of(c, s) - rows.count + i + 1), pages = sees == 0 ? 0 : page_number(c, sees - 1) + 1;
    const int budget = a.budget, last = pages - a.recent;
    int32_t* const out = a.chosen + ((int64_t)row * c.kv_heads + head) * budget;
    const int32_t* const table = c.page_table + (int64_t)s * c.table_stride;
    auto page_at = [&](int n) -> int64_t {
        const int64_t p = table[n];
        return p < 0 || p >= c.num_pages ? -1 : p;
    };
    uint32_t* const keys = a.keys ? a.keys + ((int64_t)row * c.kv_heads + head) * a.key_stride : near;
    const bool all = pages <= budget || c.num_pages == 0;      // no need to know their order
    if (all) {
        for (int n = tid; n < pages; n += kThreads) keys[n] = page_at(n) < 0 ? 0u : kForced;
    } else {
        for (int h0 = 0; h0 < a.group; h0 += 16) {
            // the queries' codes: 16 lanes a query, DP/16 dims each
            __syncthreads();
            constexpr int E = DP / 16;
            for (int h = tid >> 4; h < 16; h += kThreads / 16) {
                const int l = tid & 15;
                const T* const q = static_cast<const T*>(a.q) + (int64_t)row * a.ldq + (int64_t)(head * a.group + min(h0 + h, a.group - 1)) * c.head_dim;
                float x[E], most = 0.f, wild = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int d = l * E + e;
                    x[e] = d < c.head_dim ? elem<T>::load(q + d) : 0.f;
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
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int v = unit > 0.f ? (int)fminf(fmaxf(rintf(x[e] / unit), -127.f), 127.f) : 0;
                    codes[h][l * E + e] = (int8_t)max(v, 0);
                    codes[h][DP + l * E + e] = (int8_t)min(v, 0);
                }
                if (l == 0) units[h] = unit;
            }
            __syncthreads();
            const int r = lane & 15, g = lane >> 4;
            int4v query[NS];
#pragma unroll
            for (int n = 0; n < NS; ++n) query[n] = *reinterpret_cast<const int4v*>(&codes[r][64 * n + 16 * g]);
            float unit[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) unit[e] = units[4 * g + e];
            const int valid = a.group - h0 - 4 * g;            // of the lane's four rows
            for (int n0 = wave * 16; n0 < pages; n0 += kWaves * 16) {
                const int n = n0 + r;
                const int64_t page = n < pages ? page_at(n) : -1, at = max(page, (int64_t)0) * c.kv_heads + head;
                const int8_t* const p = a.bounds + at * (2 * DP) + 16 * g;
                int4v b[NS];
#pragma unroll
                for (int m = 0; m < NS; ++m) b[m] = *reinterpret_cast<const int4v*>(p + 64 * m);
                const float step = a.steps[at];
                int4v sum = {0, 0, 0, 0};
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
                for (int m = 0; m < NS; ++m) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(query[m], b[m], sum, 0, 0, 0);
#endif
                float most = -INFINITY;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < valid) most = greater(most, (float)sum[e] * unit[e]);
                most = greater(most, __shfl_xor(most, 16, 64));
                most = greater(most, __shfl_xor(most, 32, 64));
                if (g == 0 && n < pages) {
                    uint32_t key = page < 0 ? 0u : n < a.first || n >= last ? kForced : order_of(most * step);
                    if (h0 > 0) key = max(key, keys[n]);       // (products with a step not below 0 are in their order)
                    keys[n] = key;
                }
            }
        }
    }
    __syncthreads();
    // the budget-th largest key, and how many of its like are wanted
    uint32_t threshold = 1;
    int equal = budget;                                        // (all that are there)
    if (!all) {
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
            if (wave == 0) {                                   // from the top: the bin in which the wanted number is reached
                int mine[4], sum = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += mine[e] = bins[255 - (4 * lane + e)];
                int upto = sum;
#pragma unroll
                for (int off = 1; off < 64; off <<= 1) {
                    const int above = __shfl_up(upto, off, 64);
                    if (lane >= off) upto += above;
                }
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
        threshold = prefix;
        equal = wanted;
    }
    // in order: above it, all; equal to it, the first few; a page that is not there never
    int written = 0, same = 0;
    for (int n0 = 0; n0 < pages; n0 += kThreads) {
        const uint32_t key = n0 + tid < pages ? keys[n0 + tid] : 0u;
        const bool is_equal = key == threshold && key != 0, above = key > threshold;
        const uint64_t equals = __ballot(is_equal);
        __syncthreads();
        if (lane == 0) counts[0][wave] = __popcll(equals);
        __syncthreads();
        int before = same;
        for (int w = 0; w < kWaves; ++w) {
            before += w < wave ? counts[0][w] : 0;
            same += counts[0][w];
        }
        const bool is = above || (is_equal && lanes_before(equals, before) < equal);
        const uint64_t mask = __ballot(is);
        if (lane == 0) counts[1][wave] = __popcll(mask);
        __syncthreads();
        int at = written;
        for (int w = 0; w < kWaves; ++w) {
            at += w < wave ? counts[1][w] : 0;
            written += counts[1][w];
        }
        at = lanes_before(mask, at);
        if (is && at < budget) out[at] = n0 + tid;
    }
    for (int n = written + tid; n < budget; n += kThreads) out[n] = -1;
}

template <typename T>
hipError_t launch_choose(const choose_args& a, hipStream_t stream)
{
    const dim3 grid((uint32_t)((int64_t)a.c.num_seqs * a.c.max_new * a.c.kv_heads)), block(kThreads);
    const uint32_t lds = a.keys ? 0u : (uint32_t)a.key_stride * 4;
    switch (padded_head_dim(a.c.head_dim)) {
        case 64: LORA_LAUNCH(LORA_K_CACHE_CHOOSE, (cache_choose_kernel<T, 64>), grid, block, lds, stream, a); break;
        case 128: LORA_LAUNCH(LORA_K_CACHE_CHOOSE, (cache_choose_kernel<T, 128>), grid, block, lds, stream, a); break;
        default: LORA_LAUNCH(LORA_K_CACHE_CHOOSE, (cache_choose_kernel<T, 256>), grid, block, lds, stream, a);
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
