// The cache in 4 bits: tokens into it, their values out of it, and eviction.  (Attention over it: kernels_cache_attention.hip.)
#include <hip/hip_runtime.h>

#include "cache_format.h"
#include "launch.h"

// ---------------------------------------------------------------------------
// Append.  16 lanes hold a token's keys (then values) of one head, lane r the dims (DP/16) r ...: a lane's codes are whole words
// of the format in both parts, so nothing is exchanged but the least and the greatest element.  Memory bound: 4 D bytes of bf16
// in, D + 8 out.
namespace {

// sequence of packed row t, or -1: the last with indptr[s] <= t that has it
__device__ __forceinline__ int sequence_of(const cache_args& c, int t)
{
    if (!c.indptr) return t < c.num_seqs ? t : -1;
    int lo = 0, hi = c.num_seqs;                               // indptr[lo] <= t < indptr[hi], if the offsets are in order
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (c.indptr[mid] <= t) lo = mid; else hi = mid;
    }
    return t >= c.indptr[lo] && t < c.indptr[lo + 1] ? lo : -1;
}

// slot of packed row t of sequence s; -1 where there is none
__device__ __forceinline__ int slot_of(const cache_args& c, int s, int t)
{
    const cache_rows rows = rows_of(c, s);
    const int i = t - rows.first;
    return i >= 0 && i < min(rows.count, c.max_new) ? length_of(c, s) - rows.count + i : -1;
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
    float lo = INFINITY, hi = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (i < count) {
            lo = fminf(lo, x[i]);
            hi = fmaxf(hi, x[i]);
            bad |= !(fabsf(x[i]) < INFINITY);
        }
    int any = bad;
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) {
        lo = fminf(lo, __shfl_xor(lo, off, 16));
        hi = fmaxf(hi, __shfl_xor(hi, off, 16));
        any |= __shfl_xor(any, off, 16);
    }
    uint32_t z = __float_as_uint(lo);                          // rounded down to bf16
    z = (z & 0xffff0000u) + ((z >> 31) && (z & 0xffffu) ? 0x10000u : 0u);
    const float zero = __uint_as_float(z), range = hi - zero;
    float step = bf16_to_f32(f32_to_bf16(range * (1.f / 15.f)));
    if (step < 0x1p-100f) step = 0.f;
    any |= !(fabsf(zero) < INFINITY) || !(range < INFINITY);
#pragma unroll
    for (int w = 0; w < (E + 7) / 8; ++w) {
        uint32_t u = 0;
#pragma unroll
        for (int i = 0; i < (E < 8 ? E : 8); ++i) {
            const float c = fminf(fmaxf(rintf((x[8 * w + i] - zero) / step), 0.f), 15.f);
            u |= (8 * w + i < count && step > 0.f && !any ? (uint32_t)c : 0u) << (4 * i);
        }
        codes[w] = u;
    }
    return any ? 0x7fc07fc0u : (z | __float_as_uint(step) >> 16);
}

template <typename T, int DP>
__global__ __launch_bounds__(256) void cache_append_kernel(cache_args c, const T* k, int64_t ldk, const T* v, int64_t ldv, bool aligned)
{
    constexpr int E = DP / 16;
    const int64_t item = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    const int r = threadIdx.x & 15;
    if (item >= (int64_t)c.num_tokens * c.kv_heads) return;    // (whole groups of 16 lanes)
    const int t = (int)(item / c.kv_heads), head = (int)(item - (int64_t)t * c.kv_heads);
    const int s = sequence_of(c, t);
    const int slot = s < 0 ? -1 : slot_of(c, s, t);
    if (slot < 0) return;
    const int page = slot / c.page_tokens, at = slot - page * c.page_tokens;
    const int64_t id = page_of(c, s, page);
    if (id < 0) return;
    const int d0 = r * E, count = min(E, c.head_dim - d0);
    float x[2][E];
    load_elems<T, E>(k + (int64_t)t * ldk + head * c.head_dim + d0, count, aligned, x[0]);
    load_elems<T, E>(v + (int64_t)t * ldv + head * c.head_dim + d0, count, aligned, x[1]);
    unsigned char* const base = c.pages + (id * c.kv_heads + head) * c.page_bytes;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        uint32_t codes[(E + 7) / 8];
        const uint32_t word = quantise<E>(x[part], count, codes);
        store_codes<DP>(base + (part ? value_offset<DP>(c.page_tokens, at, r) : key_offset<DP>(at, r)), codes);
        if (r == 0) *reinterpret_cast<uint32_t*>(base + word_offset<DP>(c.page_tokens, at, part)) = word;
    }
    if (r == 0 && c.weight) c.weight[(id * c.kv_heads + head) * c.page_tokens + at] = 0.f;
}

template <typename T, int DP>
__global__ __launch_bounds__(256) void cache_read_kernel(cache_args c, T* k, int64_t ldk, T* v, int64_t ldv, bool aligned)
{
    constexpr int E = DP / 16;
    const int64_t item = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    const int r = threadIdx.x & 15;
    if (item >= (int64_t)c.num_tokens * c.kv_heads) return;
    const int t = (int)(item / c.kv_heads), head = (int)(item - (int64_t)t * c.kv_heads);
    const int s = sequence_of(c, t);
    if (s < 0) return;
    const cache_rows rows = rows_of(c, s);
    if (t - rows.first >= min(rows.count, c.max_new)) return;
    const int slot = slot_of(c, s, t);
    const int page = slot < 0 ? 0 : slot / c.page_tokens, at = slot - page * c.page_tokens;
    const int64_t id = slot < 0 ? -1 : page_of(c, s, page);
    const int d0 = r * E, count = min(E, c.head_dim - d0);
    const unsigned char* const base = c.pages + (max(id, (int64_t)0) * c.kv_heads + head) * c.page_bytes;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        float x[E];
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = 0.f;
        if (id >= 0) {
            uint32_t codes[(E + 7) / 8];
            load_codes<DP>(base + (part ? value_offset<DP>(c.page_tokens, at, r) : key_offset<DP>(at, r)), codes);
            const uint32_t word = *reinterpret_cast<const uint32_t*>(base + word_offset<DP>(c.page_tokens, at, part));
            const float step = __uint_as_float(word << 16), zero = __uint_as_float(word & 0xffff0000u);
#pragma unroll
            for (int i = 0; i < E; ++i) x[i] = (float)(codes[i / 8] >> (4 * (i % 8)) & 15u) * step + zero;
        }
        if (part) store_elems<T, E>(v + (int64_t)t * ldv + head * c.head_dim + d0, count, aligned, x);
        else store_elems<T, E>(k + (int64_t)t * ldk + head * c.head_dim + d0, count, aligned, x);
    }
}

bool rows_aligned(const void* k, int64_t ldk, const void* v, int64_t ldv, int32_t head_dim, int32_t dtype)
{
    const uintptr_t es = dtype == LORA_F32 ? 4 : 2;
    return ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | (uintptr_t)ldk * es | (uintptr_t)ldv * es | (uintptr_t)head_dim * es) & 15) == 0;
}

// ---------------------------------------------------------------------------
// Eviction, first step: a workgroup per sequence and head finds what is kept.  The weights as whole numbers in their order, NaN
// above all; the budget-th largest of them by four passes over their bytes (a histogram of 256 bins each), then the slots in
// order: above it, all; equal to it, the first few.
__device__ __forceinline__ uint32_t order_of(float w)
{
    if (w != w) return 0xffffffffu;
    const uint32_t u = __float_as_uint(w + 0.f);               // (-0 is +0)
    return u >> 31 ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ uint32_t key_at(const cache_args& c, int s, int head, int slot)
{
    const int page = slot / c.page_tokens;
    const int64_t id = page_of(c, s, page);
    return id < 0 ? order_of(0.f) : order_of(c.weight[(id * c.kv_heads + head) * c.page_tokens + slot - page * c.page_tokens]);
}

constexpr int kSelectThreads = 1024;

__global__ __launch_bounds__(kSelectThreads) void cache_select_kernel(cache_args c, int32_t* target_length, int budget, int recent, int32_t* kept)
{
    __shared__ int bins[256];
    __shared__ int counts[2][kSelectThreads / 64];
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
    uint32_t threshold = 0xffffffffu;
    int ties = 0;                                              // of the slots at the threshold, the first so many
    if (wanted > 0) {
        if (tid == 0) { found[0] = 0; found[1] = (uint32_t)wanted; }
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < 256; i += kSelectThreads) bins[i] = 0;
            __syncthreads();
            const uint32_t prefix = found[0], still = found[1];
            for (int i = tid; i < old; i += kSelectThreads) {
                const uint32_t key = key_at(c, s, head, i);
                if (shift == 24 || key >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&bins[key >> shift & 255u], 1);
            }
            __syncthreads();
            if (tid == 0) {
                uint32_t left = still;
                int b = 255;
                while (b > 0 && (uint32_t)bins[b] < left) left -= (uint32_t)bins[b--];
                found[0] = prefix | (uint32_t)b << shift;
                found[1] = left;
            }
            __syncthreads();
        }
        threshold = found[0];
        ties = (int)found[1];
    }
    int above = 0, equal = 0;                                  // of all slots before the step's
    for (int i0 = 0; i0 < old && wanted > 0; i0 += kSelectThreads) {
        const int i = i0 + tid;
        const uint32_t key = i < old ? key_at(c, s, head, i) : 0u;
        const bool is_above = i < old && key > threshold, is_equal = i < old && key == threshold;
        const uint64_t ma = __ballot(is_above), me = __ballot(is_equal), below = ((uint64_t)1 << lane) - 1;
        __syncthreads();                                       // (the counts of the step before are read)
        if (lane == 0) { counts[0][wave] = __popcll(ma); counts[1][wave] = __popcll(me); }
        __syncthreads();
        int a = above + __popcll(ma & below), e = equal + __popcll(me & below);
        for (int w = 0; w < kSelectThreads / 64; ++w) {
            if (w < wave) { a += counts[0][w]; e += counts[1][w]; }
            above += counts[0][w];
            equal += counts[1][w];
        }
        if (is_above || (is_equal && e < ties)) out[a + min(e, ties)] = i;
    }
    for (int i = tid; i < recent; i += kSelectThreads) out[wanted + i] = old + i;
}

// Second step: the kept tokens' codes, words and weights, 16 lanes a token of a head.
template <int DP>
__global__ __launch_bounds__(256) void cache_move_kernel(cache_args c, cache_args to, int budget, const int32_t* kept)
{
    constexpr int E = DP / 16;
    const int64_t item = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    const int r = threadIdx.x & 15;
    if (item >= (int64_t)c.num_seqs * c.kv_heads * budget) return;
    const int64_t group = item / budget;
    const int j = (int)(item - group * budget), s = (int)(group / c.kv_heads), head = (int)(group - (int64_t)s * c.kv_heads);
    const int slot = kept[item];
    if (slot < 0 || slot >= c.max_length) return;
    const int page = slot / c.page_tokens, at = slot - page * c.page_tokens, new_page = j / to.page_tokens, new_at = j - new_page * to.page_tokens;
    const int64_t id = page_of(c, s, page), new_id = page_of(to, s, new_page);
    if (new_id < 0) return;
    unsigned char* const dst = to.pages + (new_id * c.kv_heads + head) * c.page_bytes;
    const unsigned char* const src = c.pages + (max(id, (int64_t)0) * c.kv_heads + head) * c.page_bytes;
    uint32_t k[(E + 7) / 8] = {}, v[(E + 7) / 8] = {};         // (a page that is not there reads as zeros)
    if (id >= 0) {
        load_codes<DP>(src + key_offset<DP>(at, r), k);
        load_codes<DP>(src + value_offset<DP>(c.page_tokens, at, r), v);
    }
    store_codes<DP>(dst + key_offset<DP>(new_at, r), k);
    store_codes<DP>(dst + value_offset<DP>(c.page_tokens, new_at, r), v);
    if (r < 2)
        *reinterpret_cast<uint32_t*>(dst + word_offset<DP>(c.page_tokens, new_at, r)) =
            id < 0 ? 0u : *reinterpret_cast<const uint32_t*>(src + word_offset<DP>(c.page_tokens, at, r));
    if (r == 2)
        to.weight[(new_id * c.kv_heads + head) * c.page_tokens + new_at] =
            id < 0 ? 0.f : c.weight[(id * c.kv_heads + head) * c.page_tokens + at];
}

#define BY_HEAD_DIM(KERNEL, ...)                                                              \
    switch (padded_head_dim(c.head_dim)) {                                                    \
        case 64: KERNEL(64, __VA_ARGS__); break;                                              \
        case 128: KERNEL(128, __VA_ARGS__); break;                                            \
        default: KERNEL(256, __VA_ARGS__);                                                    \
    }
dim3 groups_of_16(int64_t items) { return dim3((uint32_t)((items + 15) / 16)); }
}  // namespace

hipError_t launch_cache_append(const cache_args& c, int32_t dtype, const void* k, int64_t ldk, const void* v, int64_t ldv, hipStream_t stream)
{
    const dim3 grid = groups_of_16((int64_t)c.num_tokens * c.kv_heads);
    const bool aligned = rows_aligned(k, ldk, v, ldv, c.head_dim, dtype);
#define APPEND(DP, T) LORA_LAUNCH(LORA_K_CACHE_APPEND, (cache_append_kernel<T, DP>), grid, dim3(256), 0, stream, c, static_cast<const T*>(k), ldk, static_cast<const T*>(v), ldv, aligned)
    if (dtype == LORA_F32) { BY_HEAD_DIM(APPEND, float) }
    else { BY_HEAD_DIM(APPEND, bf16_t) }
    return hipGetLastError();
}

hipError_t launch_cache_read(const cache_args& c, int32_t dtype, void* k, int64_t ldk, void* v, int64_t ldv, hipStream_t stream)
{
    const dim3 grid = groups_of_16((int64_t)c.num_tokens * c.kv_heads);
    const bool aligned = rows_aligned(k, ldk, v, ldv, c.head_dim, dtype);
#define READ(DP, T) LORA_LAUNCH(LORA_K_CACHE_READ, (cache_read_kernel<T, DP>), grid, dim3(256), 0, stream, c, static_cast<T*>(k), ldk, static_cast<T*>(v), ldv, aligned)
    if (dtype == LORA_F32) { BY_HEAD_DIM(READ, float) }
    else { BY_HEAD_DIM(READ, bf16_t) }
    return hipGetLastError();
}

hipError_t launch_cache_evict(const cache_args& c, const cache_args& to, int32_t* target_length, int32_t budget, int32_t recent, int32_t* kept,
                              hipStream_t stream)
{
    LORA_LAUNCH(LORA_K_CACHE_SELECT, cache_select_kernel, dim3((uint32_t)(c.num_seqs * c.kv_heads)), dim3(kSelectThreads), 0, stream, c, target_length, budget,
                recent, kept);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || budget == 0) return e;
    const dim3 grid = groups_of_16((int64_t)c.num_seqs * c.kv_heads * budget);
#define MOVE(DP, UNUSED) LORA_LAUNCH(LORA_K_CACHE_MOVE, (cache_move_kernel<DP>), grid, dim3(256), 0, stream, c, to, budget, kept)
    BY_HEAD_DIM(MOVE, )
    return hipGetLastError();
}
