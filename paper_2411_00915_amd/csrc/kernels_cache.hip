// The cache in 4 bits: tokens into it, their values out of it, and eviction.  (Attention over it: kernels_cache_attention.hip.)
#include <hip/hip_runtime.h>

#include <climits>

#include "cache_format.h"
#include "launch.h"

// ---------------------------------------------------------------------------
// Tokens go in and out in tiles of 32 packed rows of one head.  16 lanes hold a token's keys and values, lane r the dims (DP/16) r
// ...: a lane's codes are whole words of the format in both parts, so nothing is exchanged but the least and the greatest
// element.  A token's keys are one run of bytes in its page; its values are 16 pieces that lie beside those of the seven
// tokens around it, so they pass through LDS and go 8 tokens at a time (4 bytes apart a lane, 32 bytes together).
// Bound by memory where there are many tokens (8 heads of 128, bf16: 8192 tokens in 17 and out in 10 us, 84 MB, 3.1 TB/s; 64000 out
// in 51, 332 MB, 6.5), by the chain offsets -> length -> page -> store where there are few (16 tokens: 5.7 in, 3.8 out).
namespace {

constexpr int kTile = 32;                                   // (tiles_of_tokens)

// where the tokens of a tile are: the head's page (from the pool's start; -1: nowhere) and the place in it
struct tile_places {
    int64_t page[kTile];
    int at[kTile];
    int known[kTile];      // the row is one of the call's tokens
};

// the last s with indptr[s] <= t, by all lanes of a wavefront together; t is the same in all of them
__device__ __forceinline__ int search_indptr(const cache_args& c, int t, int lane)
{
    int lo = 0, n = c.num_seqs;
    while (n > 1) {
        const int step = (n + 63) >> 6, i = lane * step;
        const int count = __popcll(__ballot(i < n && c.indptr[lo + min(i, n - 1)] <= t));
        const int skip = max(count - 1, 0) * step;
        lo += skip;
        n = min(step, n - skip);
    }
    return lo;
}

// Places of rows t0 ... by a wavefront (lanes 0 .. 31 a row each).  The trips to memory are what it takes: one for a window of
// 63 sequences' offsets and lengths (two more to find the window where there are many), one for the pages.
__device__ __forceinline__ void find_places(const cache_args& c, int t0, int head, int lane, tile_places& p)
{
    const int t = t0 + lane, S = c.num_seqs;
    const bool mine = lane < kTile && t < c.num_tokens;
    int s = -1, first = t, next = t + 1, length = 0;
    if (!c.indptr) {
        if (mine && t < S) {
            s = t;
            length = c.length[t];
        }
    } else {
        bool pending = mine;
        for (int base = S < 64 ? 0 : search_indptr(c, t0, lane);; base += 63) {
            const int starts = base + lane <= S ? c.indptr[base + lane] : INT_MAX, held = c.length[min(base + lane, S - 1)];
            int j = 0;                                         // starts are in order: of lanes 1 .. 63, how many are not behind t
#pragma unroll
            for (int step = 32; step > 0; step >>= 1)
                if (__shfl(starts, min(j + step, 63), 64) <= t) j += step;
            const int a = __shfl(starts, j, 64), b = __shfl(starts, min(j + 1, 63), 64), n = __shfl(held, j, 64);
            if (pending && j < 63) {
                s = base + j;
                first = a;
                next = b;
                length = n;
                pending = false;
            }
            if (!__ballot(pending) || base + 63 > S) break;
        }
    }
    if (lane >= kTile) return;
    int64_t page = -1;
    int at = 0, known = 0;
    if (s >= 0 && s < S) {
        first = min(max(first, 0), c.num_tokens);              // (as rows_of and length_of)
        const int count = min(max(next, first), c.num_tokens) - first, i = t - first;
        known = i >= 0 && i < min(count, c.max_new);
        const int slot = known ? min(max(length, 0), c.max_length) - count + i : -1;
        if (slot >= 0) {
            const int number = page_number(c, slot);
            at = slot - number * c.page_tokens;
            page = page_of(c, s, number);
            if (page >= 0) page = page * c.kv_heads + head;
        }
    }
    p.page[lane] = page;
    p.at[lane] = at;
    p.known[lane] = known;
}

template <typename T, int E>
__device__ __forceinline__ void load_elems(const T* p, int count, bool aligned, float* x)
{
    if (aligned && count >= E) {
        if constexpr (sizeof(T) == 2) {
            uint32_t w[E / 2];
#pragma unroll
            for (int i = 0; i < E / 2; i += (E == 4 ? 2 : 4))
                if constexpr (E == 4) *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(p);
                else *reinterpret_cast<uint4*>(w + i) = *reinterpret_cast<const uint4*>(p + 2 * i);
#pragma unroll
            for (int i = 0; i < E; ++i) x[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        } else {
#pragma unroll
            for (int i = 0; i < E; i += 4) *reinterpret_cast<float4*>(x + i) = *reinterpret_cast<const float4*>(p + i);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = i < count ? elem<T>::load(p + i) : 0.f;
}

template <typename T, int E>
__device__ __forceinline__ void store_elems(T* p, int count, bool aligned, const float* x)
{
    if (aligned && count >= E) {
        if constexpr (sizeof(T) == 2) {
            uint32_t w[E / 2];
#pragma unroll
            for (int i = 0; i < E / 2; ++i) w[i] = f32_to_bf16(x[2 * i]) | (uint32_t)f32_to_bf16(x[2 * i + 1]) << 16;
            if constexpr (E == 4) *reinterpret_cast<uint2*>(p) = uint2{w[0], w[1]};
            else
#pragma unroll
                for (int i = 0; i < E / 2; i += 4) *reinterpret_cast<uint4*>(p + 2 * i) = uint4{w[i], w[i + 1], w[i + 2], w[i + 3]};
        } else {
#pragma unroll
            for (int i = 0; i < E; i += 4) *reinterpret_cast<float4*>(p + i) = float4{x[i], x[i + 1], x[i + 2], x[i + 3]};
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (i < count) elem<T>::store(p + i, x[i]);
}

// codes (E per lane, packed low nibble first) and word of the elements that 16 lanes hold; count: how many of a lane's E there are
template <int E>
__device__ __forceinline__ uint32_t quantise(const float* x, int count, uint32_t* codes)
{
    float lo = INFINITY, hi = -INFINITY, wild = 0.f;           // wild: NaN where an element is not finite
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (i < count) {
            lo = fminf(lo, x[i]);
            hi = fmaxf(hi, x[i]);
            wild = __builtin_fmaf(x[i], 0.f, wild);
        }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) {
        lo = fminf(lo, __shfl_xor(lo, off, 16));
        hi = fmaxf(hi, __shfl_xor(hi, off, 16));
        wild += __shfl_xor(wild, off, 16);
    }
    uint32_t z = __float_as_uint(lo);                          // rounded down to bf16
    z = (z & 0xffff0000u) + ((z >> 31) && (z & 0xffffu) ? 0x10000u : 0u);
    const float zero = __uint_as_float(z), range = hi - zero;
    float step = bf16_to_f32(f32_to_bf16(range * (1.f / 15.f)));
    if (step < 0x1p-100f) step = 0.f;
    const bool bad = wild != 0.f || !(fabsf(zero) < INFINITY) || !(range < INFINITY);
    // (x - zero) / step, rounded as a division is: with the reciprocal rounded to nearest, one step of Newton's on the quotient
    // gives the nearest one (Markstein); step is a bf16 of 2^-100 and more, so nothing on the way is lost below the normal numbers
    const float inverse = 1.f / step;
    const bool none = step == 0.f || bad;
#pragma unroll
    for (int w = 0; w < (E + 7) / 8; ++w) {
        uint32_t u = 0;
#pragma unroll
        for (int i = 0; i < (E < 8 ? E : 8); ++i) {
            const float d = x[8 * w + i] - zero, q0 = d * inverse, q = __builtin_fmaf(__builtin_fmaf(-q0, step, d), inverse, q0);
            u |= (8 * w + i < count ? (uint32_t)__builtin_amdgcn_fmed3f(rintf(q), 0.f, 15.f) : 0u) << (4 * i);
        }
        codes[w] = none ? 0u : u;
    }
    return bad ? 0x7fc07fc0u : (z | __float_as_uint(step) >> 16);
}

// A fifth wavefront finds the places while four make the codes
constexpr int kAppendThreads = LORA_CACHE_APPEND_THREADS;
template <typename T, int DP>
__global__ __launch_bounds__(kAppendThreads) void cache_append_kernel(cache_args c, const T* k, int64_t ldk, const T* v, int64_t ldv, bool aligned)
{
    constexpr int E = DP / 16, W = (E + 7) / 8;                // elements and words of a lane
    __shared__ tile_places places;
    __shared__ uint32_t values[kTile][16 * W + 1];
    const int tid = threadIdx.x, r = tid & 15, head = blockIdx.x % c.kv_heads, t0 = blockIdx.x / c.kv_heads * kTile;
    const int d0 = r * E, count = min(E, c.head_dim - d0);
    uint32_t codes[2][W], words[2][2];                         // of the keys; of tokens tid / 16 and 16 on
    if (tid >= 256) find_places(c, t0, head, tid - 256, places);
    else {
        float x[2][2][E];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = min(t0 + (tid >> 4) + 16 * h, c.num_tokens - 1);
            load_elems<T, E>(k + (int64_t)t * ldk + head * c.head_dim + d0, count, aligned, x[h][0]);
            load_elems<T, E>(v + (int64_t)t * ldv + head * c.head_dim + d0, count, aligned, x[h][1]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t u[W];
            words[h][0] = quantise<E>(x[h][0], count, codes[h]);
            words[h][1] = quantise<E>(x[h][1], count, u);
#pragma unroll
            for (int w = 0; w < W; ++w) values[(tid >> 4) + 16 * h][W * r + w] = u[w];
        }
    }
    __syncthreads();
    if (tid >= 256) return;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = (tid >> 4) + 16 * h;
        const int64_t page = places.page[i];
        if (page < 0) continue;
        unsigned char* const base = c.pages + page * c.page_bytes;
        store_codes<DP>(base + key_offset<DP>(places.at[i], r), codes[h]);
        if (r < 2) *reinterpret_cast<uint32_t*>(base + word_offset<DP>(c.page_tokens, places.at[i], r)) = r ? words[h][1] : words[h][0];
        if (r == 2 && c.weight) c.weight[page * c.page_tokens + places.at[i]] = 0.f;
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const int i = tid & 31, q = (tid >> 5) + 8 * n;
        if (places.page[i] >= 0)
            store_codes<DP>(c.pages + places.page[i] * c.page_bytes + value_offset<DP>(c.page_tokens, places.at[i], q), &values[i][W * q]);
    }
}

template <typename T, int DP>
__global__ __launch_bounds__(LORA_CACHE_READ_THREADS) void cache_read_kernel(cache_args c, T* k, int64_t ldk, T* v, int64_t ldv, bool aligned)
{
    constexpr int E = DP / 16, W = (E + 7) / 8;
    __shared__ tile_places places;
    __shared__ uint32_t values[kTile][16 * W + 1];
    const int tid = threadIdx.x, r = tid & 15, head = blockIdx.x % c.kv_heads, t0 = blockIdx.x / c.kv_heads * kTile;
    const int d0 = r * E, count = min(E, c.head_dim - d0);
    if (tid < 64) find_places(c, t0, head, tid, places);
    __syncthreads();
    uint32_t codes[2][2][W], words[2][2];                      // a page that is not there: zeros
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const int i = tid & 31, q = (tid >> 5) + 8 * n;
        uint32_t u[W] = {};
        if (places.page[i] >= 0) load_codes<DP>(c.pages + places.page[i] * c.page_bytes + value_offset<DP>(c.page_tokens, places.at[i], q), u);
#pragma unroll
        for (int w = 0; w < W; ++w) values[i][W * q + w] = u[w];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = (tid >> 4) + 16 * h;
        const int64_t page = places.page[i];
        words[h][0] = words[h][1] = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) codes[h][0][w] = 0;
        if (page < 0) continue;
        const unsigned char* const base = c.pages + page * c.page_bytes;
        load_codes<DP>(base + key_offset<DP>(places.at[i], r), codes[h][0]);
#pragma unroll
        for (int part = 0; part < 2; ++part) words[h][part] = *reinterpret_cast<const uint32_t*>(base + word_offset<DP>(c.page_tokens, places.at[i], part));
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = (tid >> 4) + 16 * h;
        if (!places.known[i]) continue;
#pragma unroll
        for (int w = 0; w < W; ++w) codes[h][1][w] = values[i][W * r + w];
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const float step = __uint_as_float(words[h][part] << 16), zero = __uint_as_float(words[h][part] & 0xffff0000u);
            float x[E];
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = (float)(codes[h][part][e / 8] >> (4 * (e % 8)) & 15u) * step + zero;
            T* const out = (part ? v + (int64_t)(t0 + i) * ldv : k + (int64_t)(t0 + i) * ldk) + head * c.head_dim + d0;
            store_elems<T, E>(out, count, aligned, x);
        }
    }
}

// A page of one head to another page: bound by memory
__global__ __launch_bounds__(LORA_CACHE_COPY_THREADS) void cache_copy_kernel(cache_args c, const int32_t* copies)
{
    const int head = blockIdx.x % c.kv_heads, i = blockIdx.x / c.kv_heads, tid = threadIdx.x;
    const int64_t source = copies[2 * (int64_t)i], target = copies[2 * (int64_t)i + 1];
    if (source < 0 || source >= c.num_pages || target < 0 || target >= c.num_pages || source == target) return;
    const int64_t from = source * c.kv_heads + head, to = target * c.kv_heads + head;
    const uint4* const p = reinterpret_cast<const uint4*>(c.pages + from * c.page_bytes);
    uint4* const q = reinterpret_cast<uint4*>(c.pages + to * c.page_bytes);
    const int count = (int)(c.page_bytes / 16);
#pragma unroll 4
    for (int n = tid; n < count; n += LORA_CACHE_COPY_THREADS) q[n] = p[n];
    if (c.weight)
        for (int n = tid; n < c.page_tokens; n += LORA_CACHE_COPY_THREADS) c.weight[to * c.page_tokens + n] = c.weight[from * c.page_tokens + n];
}

bool rows_aligned(const void* k, int64_t ldk, const void* v, int64_t ldv, int32_t head_dim, int32_t dtype)
{
    const uintptr_t es = dtype == LORA_F32 ? 4 : 2;
    return ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | (uintptr_t)ldk * es | (uintptr_t)ldv * es | (uintptr_t)head_dim * es) & 15) == 0;
}

// ---------------------------------------------------------------------------
// Eviction, first step: a workgroup per sequence and head finds what is kept.  The weights as whole numbers in their order, NaN
// above all; the budget-th largest of them by three passes over their bits (histograms of 11, 11 and 10), then the slots in
// order: above it, all; equal to it, the first few.  A thread has four slots in a row at a time (one address, one load), 4 STEPS
// in all, whose numbers stay in registers (STEPS 0: they are read again in every pass).  Many weights share their first bits,
// the exponent's: a wavefront adds those of its first lane's bin in one go.  Bound by one compute unit's instructions: 32768
// weights 26.3 us (a slot at a time: 54), 1300 of 512 heads 11.3 in all.
__device__ __forceinline__ uint32_t order_of(float w)
{
    if (w != w) return 0xffffffffu;
    const uint32_t u = __float_as_uint(w + 0.f);               // (-0 is +0)
    return u >> 31 ? ~u : u | 0x80000000u;
}

// of the slots slot .. slot + 3 (in one page: below `end`, slot is a multiple of 4); 0, which no weight gives, from `end` on
__device__ __forceinline__ void keys_at(const cache_args& c, int s, int head, int slot, int end, uint32_t* keys)
{
    struct __attribute__((packed, aligned(4))) four { float w[4]; } x = {};
    if (slot < end) {
        const int page = page_number(c, slot);
        const int64_t id = page_of(c, s, page);
        if (id >= 0) x = *reinterpret_cast<const four*>(c.weight + (id * c.kv_heads + head) * c.page_tokens + slot - page * c.page_tokens);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) keys[e] = e < end - slot ? order_of(x.w[e]) : 0u;
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

constexpr int kSelectThreads = LORA_CACHE_SELECT_THREADS, kSelectWaves = kSelectThreads / 64, kSelectStep = 4 * kSelectThreads;
template <int STEPS>
__global__ __launch_bounds__(kSelectThreads) void cache_select_kernel(cache_args c, int32_t* target_length, int budget, int recent, int32_t* kept)
{
    constexpr int COUNTS = (STEPS > 0 ? STEPS : 1) * kSelectWaves;
    __shared__ int bins[2 * kSelectThreads], totals[kSelectWaves], counts[2][COUNTS];
    __shared__ uint32_t found[2];                              // prefix so far, how many are still wanted of it
    const int s = blockIdx.x / c.kv_heads, head = blockIdx.x % c.kv_heads, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int length = length_of(c, s);
    int32_t* const out = kept + (int64_t)blockIdx.x * budget;
    if (head == 0 && tid == 0) target_length[s] = min(length, budget);
    if (length <= budget) {
        for (int i = tid; i < budget; i += kSelectThreads) out[i] = i < length ? i : -1;
        return;
    }
    const int old = length - recent, wanted = budget - recent; // (wanted < old)
    for (int i = tid; i < recent; i += kSelectThreads) out[wanted + i] = old + i;
    if (wanted == 0) return;
    uint32_t held[STEPS > 0 ? STEPS : 1][4];                   // (the launch sees to it that STEPS are enough)
    if constexpr (STEPS > 0)
#pragma unroll
        for (int n = 0; n < STEPS; ++n) keys_at(c, s, head, n * kSelectStep + 4 * tid, old, held[n]);
    const int steps = (int)(((int64_t)old + kSelectStep - 1) / kSelectStep);
    // f(step, keys), slots of a step in the order of the threads
    auto each = [&](auto f) {
        if constexpr (STEPS > 0) {
#pragma unroll
            for (int n = 0; n < STEPS; ++n)
                if (n < steps) f(n, held[n]);
        } else
            for (int n = 0; n < steps; ++n) {
                keys_at(c, s, head, (int)min((int64_t)n * kSelectStep + 4 * tid, (int64_t)old), old, held[0]);
                f(n, held[0]);
            }
    };
    if (tid == 0) { found[0] = 0; found[1] = (uint32_t)wanted; }
#pragma unroll 1
    for (int shift = 21; shift >= 0; shift = shift == 21 ? 10 : shift - 10) {
        const uint32_t digit = shift == 0 ? 1023u : 2047u;     // 11, 11 and 10 bits
        bins[tid] = bins[tid + kSelectThreads] = 0;
        __syncthreads();
        const uint32_t prefix = found[0], still = found[1];
        if (shift == 21)                                       // (keys of 0 are the only ones in bin 0, and what is wanted is above it)
            each([&](int, const uint32_t* keys) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t at = keys[e] >> 21, first = (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
                    const int same = __popcll(__ballot(at == first));
                    if (lane == 0 || at != first) atomicAdd(&bins[at], lane == 0 ? same : 1);
                }
            });
        else {
            const int fixed = shift == 10 ? 21 : 10;
            each([&](int, const uint32_t* keys) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (keys[e] >> fixed == prefix >> fixed) atomicAdd(&bins[keys[e] >> shift & digit], 1);
            });
        }
        __syncthreads();
        // from the highest bin down, two a thread: the one at which what is wanted is reached
        const int b = 2047 - 2 * tid, high = bins[b], sum = high + bins[b - 1];
        int up = sum;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int x = __shfl_up(up, off, 64);
            if (lane >= off) up += x;
        }
        if (lane == 63) totals[wave] = up;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kSelectWaves; ++w) up += w < wave ? totals[w] : 0;
        if ((uint32_t)up >= still && (uint32_t)(up - sum) < still) {
            const uint32_t left = still - (uint32_t)(up - sum);
            const bool upper = (uint32_t)high >= left;
            found[0] = prefix | (uint32_t)(upper ? b : b - 1) << shift;
            found[1] = upper ? left : left - (uint32_t)high;
        }
        __syncthreads();
    }
    const uint32_t threshold = found[0];                       // (not 0: keys of 0 are neither above it nor equal)
    const int ties = (int)found[1];                            // of the slots at the threshold, the first so many
    auto put = [&](int n, const uint32_t* keys, int above, int equal) {      // above, equal: how many such come before this wavefront's
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            above = lanes_before(__ballot(keys[e] > threshold), above);
            equal = lanes_before(__ballot(keys[e] == threshold), equal);
        }
        const int slot = (int)((uint32_t)n * kSelectStep + 4u * tid);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool is_above = keys[e] > threshold, is_equal = keys[e] == threshold;
            if (is_above || (is_equal && equal < ties)) out[above + min(equal, ties)] = slot + e;
            above += is_above;
            equal += is_equal;
        }
    };
    auto count = [&](int n, const uint32_t* keys) {
        int a = 0, q = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            a += __popcll(__ballot(keys[e] > threshold));
            q += __popcll(__ballot(keys[e] == threshold));
        }
        if (lane == 0) { counts[0][n * kSelectWaves + wave] = a; counts[1][n * kSelectWaves + wave] = q; }
    };
    if constexpr (STEPS > 0) {
        each(count);
        __syncthreads();
        if (wave < 2) {                                        // sums over what comes before, in the order of the slots
            int before = 0;
            for (int i0 = 0; i0 < steps * kSelectWaves; i0 += 64) {
                const int mine = i0 + lane < steps * kSelectWaves ? counts[wave][i0 + lane] : 0;
                int up = mine;
#pragma unroll
                for (int off = 1; off < 64; off <<= 1) {
                    const int x = __shfl_up(up, off, 64);
                    if (lane >= off) up += x;
                }
                if (i0 + lane < steps * kSelectWaves) counts[wave][i0 + lane] = before + up - mine;
                before += __shfl(up, 63, 64);
            }
        }
        __syncthreads();
        each([&](int n, const uint32_t* keys) { put(n, keys, counts[0][n * kSelectWaves + wave], counts[1][n * kSelectWaves + wave]); });
    } else {
        int above = 0, equal = 0;
        each([&](int n, const uint32_t* keys) {
            __syncthreads();                                   // (the counts of the step before are read)
            count(0, keys);
            __syncthreads();
            int a = 0, e = 0;
            for (int w = 0; w < kSelectWaves; ++w) {
                if (w == wave) { a = above; e = equal; }
                above += counts[0][w];
                equal += counts[1][w];
            }
            put(n, keys, a, e);
        });
    }
}

// Second step: the kept tokens' codes, words and weights, a workgroup kMoved of them of a head: three trips to memory (what is
// kept, its pages, their contents).  64 at a time, values in the target's order: 64 caches of 1300 tokens to 1000, 8 heads of 128,
// 50 us for 139 MB, 2.8 TB/s; with selection and the values read back 132 (32 at a time 136; 128: 132, but one cache of 32768
// tokens to 4096 70 instead of 66).
constexpr int kMoved = 64;
template <int DP>
__global__ __launch_bounds__(LORA_CACHE_MOVE_THREADS) void cache_move_kernel(cache_args c, cache_args to, int budget, int tiles, const int32_t* kept)
{
    constexpr int E = DP / 16, W = (E + 7) / 8, N = kMoved / 16;
    __shared__ int64_t from[kMoved], where[kMoved];            // the head's page (-1: nowhere)
    __shared__ int from_at[kMoved], where_at[kMoved];
    const int tid = threadIdx.x, r = tid & 15;
    const int64_t group = blockIdx.x / tiles;                  // sequence and head
    const int j0 = (int)(blockIdx.x - group * tiles) * kMoved, s = (int)(group / c.kv_heads), head = (int)(group - (int64_t)s * c.kv_heads);
    if (tid < kMoved) {
        const int j = j0 + tid, slot = j < budget ? kept[group * budget + j] : -1;
        int64_t src = -1, dst = -1;
        int at = 0, there = 0;
        if (slot >= 0 && slot < c.max_length) {
            const int number = page_number(c, slot), page = page_number(c, j);
            at = slot - number * c.page_tokens;
            there = j - page * c.page_tokens;
            src = page_of(c, s, number);
            dst = page_of(to, s, page);
        }
        from[tid] = src < 0 ? -1 : src * c.kv_heads + head;
        from_at[tid] = at;
        where[tid] = dst < 0 ? -1 : dst * c.kv_heads + head;
        where_at[tid] = there;
    }
    __syncthreads();
    uint32_t v[N][W], k[N][W], words[N];                       // (a page that is not there reads as zeros)
    float weight[N];
#pragma unroll
    for (int h = 0; h < N; ++h) {
        const int at = tid + 256 * h, i = (at >> 7) * 8 + (at & 7), q = at >> 3 & 15, j = (tid >> 4) + 16 * h;      // values in the target's order
        const int64_t page = from[j];
        const unsigned char* const src = c.pages + max(page, (int64_t)0) * c.page_bytes;
#pragma unroll
        for (int w = 0; w < W; ++w) v[h][w] = k[h][w] = 0;
        if (from[i] >= 0) load_codes<DP>(c.pages + from[i] * c.page_bytes + value_offset<DP>(c.page_tokens, from_at[i], q), v[h]);
        if (page >= 0) load_codes<DP>(src + key_offset<DP>(from_at[j], r), k[h]);
        words[h] = page >= 0 && r < 2 ? *reinterpret_cast<const uint32_t*>(src + word_offset<DP>(c.page_tokens, from_at[j], r & 1)) : 0u;
        weight[h] = page >= 0 && r == 2 ? c.weight[page * c.page_tokens + from_at[j]] : 0.f;
    }
#pragma unroll
    for (int h = 0; h < N; ++h) {
        const int at = tid + 256 * h, i = (at >> 7) * 8 + (at & 7), q = at >> 3 & 15, j = (tid >> 4) + 16 * h;      // values in the target's order
        if (where[i] >= 0) store_codes<DP>(to.pages + where[i] * c.page_bytes + value_offset<DP>(c.page_tokens, where_at[i], q), v[h]);
        const int64_t page = where[j];
        if (page < 0) continue;
        unsigned char* const dst = to.pages + page * c.page_bytes;
        store_codes<DP>(dst + key_offset<DP>(where_at[j], r), k[h]);
        if (r < 2) *reinterpret_cast<uint32_t*>(dst + word_offset<DP>(c.page_tokens, where_at[j], r)) = words[h];
        if (r == 2) to.weight[page * c.page_tokens + where_at[j]] = weight[h];
    }
}

#define BY_HEAD_DIM(KERNEL, ...)                                                              \
    switch (padded_head_dim(c.head_dim)) {                                                    \
        case 64: KERNEL(64, __VA_ARGS__); break;                                              \
        case 128: KERNEL(128, __VA_ARGS__); break;                                            \
        default: KERNEL(256, __VA_ARGS__);                                                    \
    }
}  // namespace

hipError_t launch_cache_append(const cache_args& c, int32_t dtype, const void* k, int64_t ldk, const void* v, int64_t ldv, hipStream_t stream)
{
    const dim3 grid((uint32_t)(tiles_of_tokens(c.num_tokens) * c.kv_heads));
    const bool aligned = rows_aligned(k, ldk, v, ldv, c.head_dim, dtype);
#define APPEND(DP, T) LORA_LAUNCH(LORA_K_CACHE_APPEND, (cache_append_kernel<T, DP>), grid, dim3(kAppendThreads), 0, stream, c, static_cast<const T*>(k), ldk, static_cast<const T*>(v), ldv, aligned)
    if (dtype == LORA_F32) { BY_HEAD_DIM(APPEND, float) }
    else { BY_HEAD_DIM(APPEND, bf16_t) }
    return hipGetLastError();
}

hipError_t launch_cache_read(const cache_args& c, int32_t dtype, void* k, int64_t ldk, void* v, int64_t ldv, hipStream_t stream)
{
    const dim3 grid((uint32_t)(tiles_of_tokens(c.num_tokens) * c.kv_heads));
    const bool aligned = rows_aligned(k, ldk, v, ldv, c.head_dim, dtype);
#define READ(DP, T) LORA_LAUNCH(LORA_K_CACHE_READ, (cache_read_kernel<T, DP>), grid, dim3(LORA_CACHE_READ_THREADS), 0, stream, c, static_cast<T*>(k), ldk, static_cast<T*>(v), ldv, aligned)
    if (dtype == LORA_F32) { BY_HEAD_DIM(READ, float) }
    else { BY_HEAD_DIM(READ, bf16_t) }
    return hipGetLastError();
}

hipError_t launch_cache_evict(const cache_args& c, const cache_args& to, int32_t* target_length, int32_t budget, int32_t recent, int32_t* kept,
                              hipStream_t stream)
{
    const dim3 grid1((uint32_t)(c.num_seqs * c.kv_heads));
    const int32_t old = c.max_length - recent;
#define SELECT(STEPS) LORA_LAUNCH(LORA_K_CACHE_SELECT, (cache_select_kernel<STEPS>), grid1, dim3(kSelectThreads), 0, stream, c, target_length, budget, recent, kept)
    if (old <= kSelectStep) SELECT(1);
    else if (old <= 8 * kSelectStep) SELECT(8);
    else SELECT(0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || budget == 0) return e;
    const int32_t tiles = budget / kMoved + (budget % kMoved != 0);
    const dim3 grid((uint32_t)(c.num_seqs * c.kv_heads * tiles));
#define MOVE(DP, UNUSED) LORA_LAUNCH(LORA_K_CACHE_MOVE, (cache_move_kernel<DP>), grid, dim3(LORA_CACHE_MOVE_THREADS), 0, stream, c, to, budget, tiles, kept)
    BY_HEAD_DIM(MOVE, )
    return hipGetLastError();
}

hipError_t launch_cache_copy(const cache_args& c, int32_t num_copies, const int32_t* copies, hipStream_t stream)
{
    LORA_LAUNCH(LORA_K_CACHE_COPY, cache_copy_kernel, dim3((uint32_t)((int64_t)num_copies * c.kv_heads)), dim3(LORA_CACHE_COPY_THREADS), 0, stream, c, copies);
    return hipGetLastError();
}
