// Attention of new tokens over a cache of 4-bit keys and values.
//
// With a token's value = code * step + zero (keys and values alike, one step and one zero per token and head),
//     q . k_t     = step_t (q . code_t) + zero_t sum(q)
//     sum p_t v_t = sum (p_t step_t) code_t + sum p_t zero_t
// so the matrix cores work on the codes and the scales act on scores and softmax weights, never on elements.  A code becomes
// bf16 by two instructions a pair: (word shifted & 0x00780078) | 0x41804180 is 16 + code twice.  The sums are those of code - 7.5,
// about which the codes lie evenly, and zero + 7.5 step stands in for zero: the score's sum starts at -23.5 sum(q), and
// 23.5 sum(p step), as the matrix cores see it (one more product with ones), is taken off behind the second sum.  So the rounding
// of p step to bf16 meets codes of no common offset (with it: 4.5e-3 of the result instead of 2.3e-3, the output's own rounding,
// 1.7e-3, included).  fp32 queries and weights go in three bf16 terms (24 bits), and codes are converted without the 16.
//
// A wavefront takes 32 tokens of a head at a time, keys as rows of S^T = K Q^T (two products of 16 tokens), so that a lane ends
// with 8 tokens of one query row: exactly what the second product O^T = V^T P^T wants as its second operand.  No token crosses a
// lane; maxima do, over the 4 lanes of a row.  The pages are laid out so that every load is 16 bytes a lane and an operand as
// it is.  The wavefronts of a workgroup (four or eight) take turns at the blocks of 32 and meet in LDS at the end; long contexts
// are split over workgroups as well, which a second launch joins.
//
// Bound by memory: 256 requests of 1024 tokens, 32 heads of 128, 225 us, 5.0 TB/s (vector units busy in 80 % of the cycles).
// The codes come straight to LDS, a ring of blocks for each wavefront: with registers as their target 343 us against 247 at the
// time, as the compiler then has too few left to ask ahead (a ring of three at 128 dims costs a workgroup a compute unit: 280).
// Few requests are bound by the chain length -> page -> codes: 8 of 700 tokens 11.1 us.  Four tokens over 131072, 32 heads on 8,
// with accumulated weights: 39 us here, the scores written out for them (67 MB beside 147) included, 20 in the launch that
// reads them back.  Over chosen pages there are a few blocks a wavefront, and the chain has the list in front of it: 32 of 64 tokens for 32
// requests 19.4 to 20 us (71 MB; 13.2 at the rate of a copy), 16 for 8 requests 13.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "cache_format.h"
#include "launch.h"
#include "mfma_tile.h"

namespace {

// scaled to base 2 behind the subtraction: scores up to the end of 32 bits stay in range
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }

// the two constants of a conversion: one instruction takes at most one scalar register, so the mask lives in a vector register
struct code_bits {
    uint32_t mask, sixteen;
    __device__ __forceinline__ code_bits()
    {
        mask = 0x00780078u;
        sixteen = 0x41804180u;
        asm volatile("" : "+v"(mask));
        asm volatile("" : "+s"(sixteen));
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t w) const { return (w & mask) | sixteen; }
};

// 8 codes (low nibble first) as the operand pairs (i, i + 4)
template <bool EXACT>
__device__ __forceinline__ op16 key_operand(uint32_t w, const code_bits& bits)
{
    op16 o;
    if constexpr (EXACT) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = __float_as_uint((float)(w >> (4 * i) & 15u)), hi = __float_as_uint((float)(w >> (4 * i + 16) & 15u));
            u[i] = lo >> 16 | (hi & 0xffff0000u);
        }
        o.u = uint4{u[0], u[1], u[2], u[3]};
    } else
        o.u = uint4{bits(w << 3), bits(w >> 1), bits(w >> 5), bits(w >> 9)};
    return o;
}

// nibble n (0 or 1) of the bytes in bits 0..7 and 16..23
template <bool EXACT>
__device__ __forceinline__ uint32_t code_pair(uint32_t w, int n, const code_bits& bits)
{
    if constexpr (EXACT) {
        const uint32_t lo = __float_as_uint((float)(w >> (4 * n) & 15u)), hi = __float_as_uint((float)(w >> (4 * n + 16) & 15u));
        return lo >> 16 | (hi & 0xffff0000u);
    }
    return bits(n == 0 ? w << 3 : w >> 1);
}

// A block of 32 tokens in LDS: what each lane wants of it as keys, in rows of 16 bytes a lane (DP 64: as the page has them), then
// as values, then the words of its keys and of its values
template <int DP>
struct block_lds {
    static constexpr int LOADS = DP / 64;                      // of 1 KB, keys and values each
    static constexpr int VALUES = LOADS * 1024, WORDS = 2 * VALUES, BYTES = WORDS + 256, COUNT = 2 * LOADS + 1;
};

__device__ __forceinline__ void get16(const char* p, uint32_t* w)
{
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
}

__device__ __forceinline__ void load4_to_lds(const char* base, uint32_t off, uint32_t lds_base)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(base), "s"(lds_base) : "memory");
}

// this lane's offsets in a page, from the block's own
template <int DP>
struct block_offsets {
    uint32_t key[block_lds<DP>::LOADS], value, word;
    __device__ __forceinline__ block_offsets(int page_tokens, int lane)
    {
        const int r = lane & 15, g = lane >> 4;
#pragma unroll
        for (int i = 0; i < block_lds<DP>::LOADS; ++i)         // DP 128: a product's rows each; 256: their halves
            key[i] = DP == 64 ? 16 * lane : (8 * (r >> 2) + (r & 3) + 4 * (i / (DP / 128))) * (DP / 2) + g * (DP / 8) + i % (DP / 128) * 16;
        value = DP == 64 ? 16 * lane : (g * 16 + r) * (DP / 4);
        word = 4 * (lane < 32 ? lane : page_tokens + lane - 32);
    }
};

// `at`: the block's first place in its page
template <int DP>
__device__ __forceinline__ void fetch_block(const unsigned char* page, int page_tokens, int at, const block_offsets<DP>& off, uint32_t lds)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const char* const p = reinterpret_cast<const char*>(page);
#pragma unroll
    for (int i = 0; i < block_lds<DP>::LOADS; ++i) load16_to_lds(p + at * (DP / 2), off.key[i], lds + i * 1024);
#pragma unroll
    for (int i = 0; i < block_lds<DP>::LOADS; ++i)
        load16_to_lds(p + page_tokens * (DP / 2) + (at >> 5) * (DP * 16) + 16 * i, off.value, lds + block_lds<DP>::VALUES + i * 1024);
    load4_to_lds(p + page_tokens * DP + at * 4, off.word, lds + block_lds<DP>::WORDS);
#endif
}

// operand of the values: row r of the product is dim (DP/16) r + n, its 8 tokens in the registers' order
template <int DP, bool EXACT>
__device__ __forceinline__ op16 value_operand(const uint32_t* v, int n, const code_bits& bits)
{
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {                              // tokens 2i and 2i + 1
        if constexpr (DP == 64) {                              // (two tokens to a word, 4 codes each)
            u[i] = EXACT ? code_pair<EXACT>(v[i] >> (4 * n), 0, bits) : bits(n == 0 ? v[i] << 3 : v[i] >> (4 * n - 3));
        } else {
            constexpr int W = DP / 128;                        // words a token
            const uint32_t a = v[2 * i * W + (n >> 3)], b = v[(2 * i + 1) * W + (n >> 3)];
            const int byte = (n & 7) >> 1;
            const uint32_t w = __builtin_amdgcn_perm(b, a, 0x0c040c00u + byte * 0x00010001u);
            u[i] = code_pair<EXACT>(w, n & 1, bits);
        }
    }
    op16 o;
    o.u = uint4{u[0], u[1], u[2], u[3]};
    return o;
}

// x[0..7] in TERMS bf16 terms
template <int TERMS>
__device__ __forceinline__ void terms_of(const float* x, op16* t)
{
    if constexpr (TERMS == 1) {
        t[0].u = uint4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
        return;
    }
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
    for (int n = 0; n < TERMS; ++n) {
        uint32_t h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[i] = f32_to_bf16(rest[i]);
            rest[i] -= bf16_to_f32((bf16_t)h[i]);
        }
        t[n].u = uint4{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
    }
}

// the greatest of the four lanes of a query row
__device__ __forceinline__ float max_of_rows(float x)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
#endif
    return x;
}

// Dims d0 .. d0 + 7 of a query in key_operand's order; what is past the D that there are comes from among them.  No branch over the
// lanes, so that all loads are on their way together.
template <typename T>
__device__ __forceinline__ void load_query(const T* p, int d0, int D, bool aligned, float* x)
{
    if (!aligned) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = elem<T>::load(p + min(d0 + (i >> 1) + 4 * (i & 1), D - 1));
    } else if constexpr (sizeof(T) == 2) {
        const uint4 u = ld16(p + min(d0, D - 8));
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = (i >> 1) + 4 * (i & 1);
            x[i] = __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
        }
    } else {
        const float4 a = *reinterpret_cast<const float4*>(p + min(d0, D - 4)), b = *reinterpret_cast<const float4*>(p + min(d0 + 4, D - 4));
        x[0] = a.x; x[1] = b.x; x[2] = a.y; x[3] = b.y; x[4] = a.z; x[5] = b.z; x[6] = a.w; x[7] = b.w;
    }
}

// CHOSEN: a token at a time, over the pages that it is given; its blocks are counted along that list, and `number`ed by where they are
template <typename T, int DP, int CT, bool KEEP, int WAVES, bool CHOSEN>
__global__ __launch_bounds__(64 * WAVES, DP > 128 ? 1 : sizeof(T) == 2 && CT == 1 ? 4 : 2) void cache_attention_kernel(cache_attention_args a)
{
    constexpr bool EXACT = sizeof(T) == 4;
    constexpr int TERMS = EXACT ? 3 : 1, NS = DP / 32, NB = DP / 16;
    constexpr float OFFSET = EXACT ? 7.5f : 23.5f;         // of what the matrix cores see, from code - 7.5
    constexpr int RING = DP == 64 ? 3 : 2, RING_BYTES = WAVES * RING * block_lds<DP>::BYTES, RED_BYTES = WAVES * 16 * (DP + 4) * 4;
    __shared__ __align__(16) char lds[RING_BYTES > RED_BYTES ? RING_BYTES : RED_BYTES];
    float (*const red)[16][DP + 4] = reinterpret_cast<float (*)[16][DP + 4]>(lds);           // (when the rings are done with)
    __shared__ float red_m[WAVES][16], red_l[WAVES][16];
    __shared__ int again;
    const cache_args& c = a.c;
    int id = blockIdx.x;
    const int head = id % c.kv_heads;
    id /= c.kv_heads;
    const int rt = id % a.row_tiles;
    id /= a.row_tiles;
    const int split = id % a.splits, seq = CHOSEN ? id / a.splits / c.max_new : id / a.splits;
    cache_rows rows = rows_of(c, seq);
    int held = length_of(c, seq);
    if constexpr (CHOSEN) {                                    // (as a sequence of its own, whose last token it is)
        const int i = id / a.splits % c.max_new;
        if (i >= rows.count) return;
        held = max(0, held - rows.count + i + 1);
        rows = cache_rows{rows.first + i, 1};
    }
    const int length = held;
    const int R = min(rows.count, c.max_new) * a.group, row0 = rt * (16 * CT);      // query rows: token major, then the group's heads
    if (row0 >= R) return;
    // what a query row sees: slots below seen(row)
    auto seen = [&](int row) { return max(0, length - rows.count + row / a.group + 1); };
    const int least = seen(row0), most = seen(min(R, row0 + 16 * CT) - 1);
    const int t0 = split * a.split_tokens, t1 = min(CHOSEN ? a.budget * c.page_tokens : most, t0 + a.split_tokens);

    op16 q[CT][NS][TERMS];
    float qsum[CT], start[CT];
    int limit[CT];
    // Once, but for numbers near the end of 32 bits, which the sums are past (weights go up to 2^8, codes to 31): where a query is so
    // large, all are taken 2^-14 times; where the output is not finite, the blocks are gone through once more with all weights
    // 2^-48 times (a mean does not depend on that).
    float scale = a.scale, down = 1.f, lower = 0.f;
    bool careful = false;
    const bool aligned = ((reinterpret_cast<uintptr_t>(a.q) | (uintptr_t)((a.ldq | c.head_dim) * (int64_t)sizeof(T))) & 15) == 0;       // queries to 16 bytes
    if (threadIdx.x == 0) again = 0;
#pragma unroll 1
    for (;;) {
    float largest = 0.f;
    int tid = threadIdx.x, D = c.head_dim, group = a.group;
    asm volatile("" : "+v"(tid));                              // (opaque, so that nothing made of them is kept for another pass)
    asm volatile("" : "+s"(D), "+s"(group));
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int row = row0 + 16 * ct + r;
        const bool valid = row < R;
        const T* const p = static_cast<const T*>(a.q) + (int64_t)(rows.first + (valid ? row / group : 0)) * a.ldq +
                           (int64_t)(head * group + (valid ? row % group : 0)) * D;
        limit[ct] = valid ? max(0, length - rows.count + row / group + 1) : 0;
        float sum = 0.f;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            float x[8];
            const int d0 = (DP / 4) * g + 8 * s;
            load_query(p, d0, D, aligned, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int d = d0 + (i >> 1) + 4 * (i & 1);
                x[i] = valid && d < D ? x[i] * down : 0.f;
                sum += x[i];
                largest = fmaxf(largest, fabsf(x[i]));
            }
            terms_of<TERMS>(x, q[ct][s]);
        }
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        qsum[ct] = sum * scale;
        start[ct] = -OFFSET * sum;
    }

    if (__builtin_expect(down == 1.f && __ballot(largest > 0x1p114f) != 0, 0)) {
        down = 0x1p-14f;
        scale *= 0x1p14f;
        continue;
    }
    floatx4 acc[CT][NB], ones[CT];
    float m[CT], ref[CT], l[CT], z[CT];                        // l, z: of this lane's tokens only
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        m[ct] = -INFINITY;
        ref[ct] = l[ct] = z[ct] = 0.f;
        ones[ct] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[ct][n] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    op16 one;
    one.u = uint4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};

    const int blocks_a_page = c.page_tokens >> 5, last = (t1 + 31) >> 5;
    typedef const __attribute__((address_space(4))) int32_t* constants;         // (nothing writes the table while the kernel runs)
    const constants table = (constants)(uintptr_t)(c.page_table + (int64_t)seq * c.table_stride);
    const constants chosen = (constants)(uintptr_t)(a.chosen + ((int64_t)rows.first * c.kv_heads + head) * a.budget);
    int number = 0;                                            // of the block that was asked for last
    auto page_at = [&](int b) -> const unsigned char* {        // null: not there
        int n = b / blocks_a_page;
        number = b;
        if constexpr (CHOSEN) {
            const int place = b - n * blocks_a_page;
            n = chosen[n];
            if (n < 0 || n >= (length + c.page_tokens - 1) / c.page_tokens) return nullptr;
            number = n * blocks_a_page + place;
            if (32 * number >= length) return nullptr;
        }
        const int64_t p = table[n];
        return p < 0 || p >= c.num_pages ? nullptr : c.pages + (p * c.kv_heads + head) * c.page_bytes;
    };
    const code_bits bits;
    auto keep_scores = [&](int ct, int tok, const float* x) {
        const int row = row0 + 16 * ct + r;
        if (row >= R) return;
        float* const p = a.scores + ((int64_t)(rows.first + row / group) * a.num_heads + head * group + row % group) * a.score_stride + tok;
        *reinterpret_cast<float4*>(p) = float4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<float4*>(p + 4) = float4{x[4], x[5], x[6], x[7]};
    };
    auto compute = [&](int b, const char* block, auto masked_) {
        constexpr bool masked = decltype(masked_)::value;      // some row does not see all of the block
        typedef block_lds<DP> L;
        float x[CT][8];
        uint32_t kw[8];
        get16(block + L::WORDS + 32 * g, kw);
        get16(block + L::WORDS + 32 * g + 16, kw + 4);
#pragma unroll
        for (int h = 0; h < 2; ++h) {                          // tokens 8g + 4h + i
            uint32_t k[DP / 32];
            if constexpr (DP == 64) {
                const uint2 u = *reinterpret_cast<const uint2*>(block + (8 * (r >> 2) + (r & 3) + 4 * h) * 32 + 8 * g);
                k[0] = u.x; k[1] = u.y;
            } else
#pragma unroll
                for (int i = 0; i < DP / 128; ++i) get16(block + (h * (DP / 128) + i) * 1024 + 16 * lane, k + 4 * i);
            floatx4 s[CT];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) s[ct] = floatx4{start[ct], start[ct], start[ct], start[ct]};
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                const op16 ko = key_operand<EXACT>(k[n], bits);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) s[ct] = mfma(ko, q[ct][n][t], s[ct]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t w = kw[4 * h + i];
                const float step = __uint_as_float(w << 16), middle = __uint_as_float(w & 0xffff0000u) + 7.5f * step;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) x[ct][4 * h + i] = step * scale * s[ct][i] + middle * qsum[ct];
            }
        }
        const int tok = 32 * b + 8 * g;
        if constexpr (masked)
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
                    if (tok + i >= limit[ct]) x[ct][i] = -INFINITY;
        if constexpr (KEEP)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) keep_scores(ct, tok, x[ct]);
        // the running maximum, raised only where a score is 5.5 above it (weights then stay below 2^8)
        float mx[CT];
        bool raise = false;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            mx[ct] = x[ct][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) mx[ct] = fmaxf(mx[ct], x[ct][i]);
            mx[ct] = max_of_rows(mx[ct]);
            raise |= mx[ct] > m[ct] + 5.5f;
        }
        if (__ballot(raise)) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const float mn = fmaxf(m[ct], mx[ct]), alpha = mn == -INFINITY ? 1.f : exp_of(m[ct] - mn);
                m[ct] = mn;
                ref[ct] = mn == -INFINITY ? 0.f : mn;
                l[ct] *= alpha;
                z[ct] *= alpha;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    ones[ct][i] *= alpha;
#pragma unroll
                    for (int n = 0; n < NB; ++n) acc[ct][n][i] *= alpha;
                }
            }
        }
        op16 p[CT][TERMS];
        float w[CT][8];
        uint32_t vw[8];
        get16(block + L::WORDS + 128 + 32 * g, vw);
        get16(block + L::WORDS + 128 + 32 * g + 16, vw + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float step = __uint_as_float(vw[i] << 16), middle = __uint_as_float(vw[i] & 0xffff0000u) + 7.5f * step;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const bool there = !masked || tok + i < limit[ct];
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(x[ct][i] - ref[ct], 1.44269504088896340736f, lower));
                l[ct] += e;
                w[ct][i] = there ? e * step : 0.f;             // (what is not seen may hold anything)
                z[ct] += there ? e * middle : 0.f;
            }
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            terms_of<TERMS>(w[ct], p[ct]);
#pragma unroll
            for (int t = 0; t < TERMS; ++t) ones[ct] = mfma(one, p[ct][t], ones[ct]);
        }
        uint32_t v[DP / 16];                                   // 8 tokens x DP/16 codes
#pragma unroll
        for (int i = 0; i < DP / 64; ++i) get16(block + L::VALUES + i * 1024 + 16 * lane, v + 4 * i);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            const op16 vo = value_operand<DP, EXACT>(v, n, bits);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int t = 0; t < TERMS; ++t) acc[ct][n] = mfma(vo, p[ct][t], acc[ct][n]);
        }
    };
    auto absent = [&](int b) {
        if constexpr (KEEP) {                                  // (a slot that is not there is not seen)
            const float none[8] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) keep_scores(ct, 32 * b + 8 * g, none);
        }
    };
    // the wavefront's first block from b on whose page is there: its page and place, or null and b >= last
    int b = (t0 >> 5) + wave, at = 0;
    auto find = [&]() -> const unsigned char* {
        for (; b < last; b += WAVES) {
            const unsigned char* const p = page_at(b);
            if (p) {
                at = b % blocks_a_page * 32;
                return p;
            }
            absent(b);
        }
        return nullptr;
    };
    // A ring of RING blocks a wavefront: RING - 1 on their way while one is computed with.  Nobody else touches it, so there is no
    // barrier; loads return in order, so when no more are out than the later blocks', this one's have landed.
    const block_offsets<DP> off(c.page_tokens, lane);
    char* const ring = lds + wave * (RING * block_lds<DP>::BYTES);
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane(lds_address(ring));
    const int full = CHOSEN ? least >> 5 : min(last, least >> 5);      // blocks that every row sees
    int queue[RING], slot = 0;                                 // numbers of blocks in their order, or NONE
    constexpr int NONE = 0x7fffffff;
    auto ask = [&](int place) {                                // the next block into a place of the ring
        const unsigned char* const page = find();
        const int found = page ? number : NONE;
        if (page) fetch_block<DP>(page, c.page_tokens, at, off, ring_at + place * block_lds<DP>::BYTES);
        b += WAVES;
        return found;
    };
#pragma unroll
    for (int i = 0; i < RING - 1; ++i) queue[i] = ask(i);
    auto turn = [&](auto masked) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (the block before this one is read: its place is free)
        queue[RING - 1] = ask(slot == 0 ? RING - 1 : slot - 1);
        if (queue[RING - 1] != NONE) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((RING - 1) * block_lds<DP>::COUNT) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        compute(queue[0], ring + slot * block_lds<DP>::BYTES, masked);
#pragma unroll
        for (int i = 0; i < RING - 1; ++i) queue[i] = queue[i + 1];
        slot = slot == RING - 1 ? 0 : slot + 1;
    };
    if constexpr (CHOSEN) {                                    // (in the order of the list, which need not be the blocks'; as a branch in one
#pragma unroll 1                                               // loop both spill: 25.0 in place of 18.6 us, at their least, for 32 sequences' 32 pages, 32 heads on 8)
        while (queue[0] != NONE) {
#pragma unroll 1
            while (queue[0] < full) turn(std::false_type{});
            if (queue[0] != NONE) turn(std::true_type{});
        }
    } else {
        while (queue[0] < full) turn(std::false_type{});
#pragma unroll 1
        while (queue[0] != NONE) turn(std::true_type{});
    }

    bool wild = false;
    // the wavefronts' sums meet, column tile by column tile
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        l[ct] += __shfl_xor(l[ct], 16, 64);
        l[ct] += __shfl_xor(l[ct], 32, 64);
        z[ct] += __shfl_xor(z[ct], 16, 64);
        z[ct] += __shfl_xor(z[ct], 32, 64);
        __syncthreads();
        if (g == 0) red_m[wave][r] = m[ct];
        __syncthreads();
        float top = red_m[0][r];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, red_m[w][r]);
        const float f = m[ct] == -INFINITY ? 0.f : exp_of(ref[ct] - top);
        const float add = z[ct] - OFFSET * ones[ct][0];
        // a wavefront that saw nothing has summed nothing
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < NB; n += 4)
                *reinterpret_cast<float4*>(&red[wave][r][NB * (4 * g + i) + n]) =
                    float4{f * (acc[ct][n][i] + add), f * (acc[ct][n + 1][i] + add), f * (acc[ct][n + 2][i] + add), f * (acc[ct][n + 3][i] + add)};
        if (g == 0) red_l[wave][r] = f * l[ct];
        __syncthreads();
        constexpr int LANES = 4 * WAVES;                       // threads a query row
        const int col = tid / LANES, row = row0 + 16 * ct + col;
        if (row < R) {
            const int64_t out_row = (int64_t)(rows.first + row / group) * a.num_heads + head * group + row % group;
            float sum = 0.f, most_of = -INFINITY;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                sum += red_l[w][col];
                most_of = fmaxf(most_of, red_m[w][col]);
            }
            if (a.stats && tid % LANES == 0) a.stats[out_row * a.splits + split] = float2{most_of, careful ? sum * 0x1p48f : sum};
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            T* const out = static_cast<T*>(a.o) + (int64_t)(rows.first + row / group) * a.ldo + (int64_t)(head * group + row % group) * D;
            for (int d = tid % LANES; d < D; d += LANES) {
                float o = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) o += red[w][col][d];
                o *= inv;
                wild |= !(fabsf(o) < INFINITY);
                if (a.partial) a.partial[(out_row * a.splits + split) * D + d] = o;
                else elem<T>::store(out + d, o);
            }
        }
    }
    if (careful) return;
    if (wild) again = 1;
    __syncthreads();
    if (!again) return;
    careful = true;
    lower = -48.f;
    }
}

// What is left when all splits are done, in one launch: the first `rows` workgroups join the splits of a query row each, the others
// add up accumulated weights, for which they join the statistics themselves (one token over 8 caches of 2000, 32 heads on 8: 21.6 us
// in all with two launches, 18.9 with one).  Bound by the scores that it reads, 67 MB in 20 us for four tokens over 131072.
constexpr int kFinishThreads = LORA_CACHE_FINISH_THREADS, kFinishWaves = kFinishThreads / 64, kWeightSlots = 4 * kFinishThreads;

// a row's splits: the wavefronts take turns at them
template <typename T>
__device__ __forceinline__ void join_row(const cache_attention_args& a, int64_t row)
{
    __shared__ float red[kFinishWaves][LORA_MAX_HEAD_DIM];
    const cache_args& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, D = c.head_dim;
    const int head = (int)(row % a.num_heads);
    const int64_t at = row / a.num_heads;
    const int seq = (int)(at / c.max_new), i = (int)(at % c.max_new);
    const cache_rows rows = rows_of(c, seq);
    if (i >= rows.count) return;
    const int64_t out_row = (int64_t)(rows.first + i) * a.num_heads + head;
    const float2* const st = a.stats + out_row * a.splits;
    // a split's part of the row's sum, by every wavefront for itself; its output is a mean already, which no weight takes out of range
    float top = -INFINITY, sum = 0.f;
    for (int s = lane; s < a.splits; s += 64) top = fmaxf(top, st[s].x);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    auto part = [&](float2 e) { return e.y == 0.f ? 0.f : exp_of(e.x - top) * e.y; };      // (nothing seen: its maximum is -inf, perhaps all are; NaN goes on)
    for (int s = lane; s < a.splits; s += 64) sum += part(st[s]);
    sum = wave_sum(sum);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    float o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = wave; s < a.splits; s += kFinishWaves) {
        const float* const p = a.partial + (out_row * a.splits + s) * D;
        const float f = part(st[s]) * inv;
#pragma unroll
        for (int n = 0; n < 4; ++n)
            if (lane + 64 * n < D) o[n] += f * p[lane + 64 * n];
    }
#pragma unroll
    for (int n = 0; n < 4; ++n)
        if (lane + 64 * n < D) red[wave][lane + 64 * n] = o[n];
    __syncthreads();
    if (tid >= D) return;
    float all = 0.f;
#pragma unroll
    for (int w = 0; w < kFinishWaves; ++w) all += red[w][tid];
    elem<T>::store(static_cast<T*>(a.o) + (int64_t)(rows.first + i) * a.ldo + (int64_t)head * D + tid, all);
}

// Accumulated weights: a thread four slots of one sequence and kv head, over all query rows, whose scores the attention left behind
__device__ __forceinline__ void add_weights(const cache_attention_args& a, int id, int chunks)
{
    constexpr int MOST = 256;
    // Of that many rows at a time: maximum and 1 / sum (0, 0 where nothing is seen).  Apart: in maximum + log(sum) a large maximum
    // takes the sum's bits.
    __shared__ float2 stat[MOST];
    const cache_args& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int chunk = id % chunks;
    id /= chunks;
    const int head = id % c.kv_heads, seq = id / c.kv_heads;
    const cache_rows rows = rows_of(c, seq);
    const int length = length_of(c, seq), R = min(rows.count, c.max_new) * a.group;
    if (R == 0 || (int64_t)chunk * kWeightSlots >= length) return;
    auto row_at = [&](int row) { return (int64_t)(rows.first + row / a.group) * a.num_heads + head * a.group + row % a.group; };
    const int share = a.splits >= 64 ? 6 : 32 - __builtin_clz(max(a.splits, 1) * 2 - 1) - 1, lanes = 1 << share;      // 2^share lanes a row
    const int slot = chunk * kWeightSlots + 4 * tid;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int r0 = 0; r0 < R; r0 += MOST) {
        const int n = min(MOST, R - r0);
        __syncthreads();
        for (int j0 = wave << (6 - share); j0 < n; j0 += kFinishWaves << (6 - share)) {
            const int j = j0 + (lane >> share);
            const float2* const st = a.stats + row_at(r0 + min(j, n - 1)) * a.splits;
            float top = -INFINITY, all = 0.f;
            for (int s = lane & (lanes - 1); s < a.splits; s += lanes) top = fmaxf(top, st[s].x);
            for (int off = lanes >> 1; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
            for (int s = lane & (lanes - 1); s < a.splits; s += lanes) all += st[s].y == 0.f ? 0.f : st[s].y * exp_of(st[s].x - top);
            for (int off = lanes >> 1; off > 0; off >>= 1) all += __shfl_xor(all, off, 64);
            if (j < n && (lane & (lanes - 1)) == 0) stat[j] = all == 0.f ? float2{0.f, 0.f} : float2{top, 1.f / all};
        }
        __syncthreads();
        if (slot >= length) continue;
#pragma unroll 4
        for (int j = 0; j < n; ++j) {
            const int row = r0 + j, sees = length - rows.count + row / a.group + 1 - slot;       // of the four, the first so many
            const float2 e = stat[j];
            const float4 x = *reinterpret_cast<const float4*>(a.scores + row_at(row) * a.score_stride + slot);       // (not written where it sees nothing)
            sum[0] += sees > 0 ? exp_of(x.x - e.x) * e.y : 0.f;
            sum[1] += sees > 1 ? exp_of(x.y - e.x) * e.y : 0.f;
            sum[2] += sees > 2 ? exp_of(x.z - e.x) * e.y : 0.f;
            sum[3] += sees > 3 ? exp_of(x.w - e.x) * e.y : 0.f;
        }
    }
    if (slot >= length) return;
    const int page = slot / c.page_tokens;                     // (of all four: pages are multiples of 32)
    const int64_t p = page_of(c, seq, page);
    if (p < 0) return;
    float* const w = c.weight + (p * c.kv_heads + head) * c.page_tokens + slot - page * c.page_tokens;
    for (int e = 0; e < min(4, length - slot); ++e) w[e] = a.decay == 0.f ? sum[e] : a.decay * w[e] + sum[e];
}

template <typename T>
__global__ __launch_bounds__(kFinishThreads) void cache_finish_kernel(cache_attention_args a, int rows, int chunks)
{
    const int id = blockIdx.x;
    if (id < rows) join_row<T>(a, id);
    else add_weights(a, id - rows, chunks);
}

template <typename T, int DP, int CT, int WAVES>
void launch_shape(const cache_attention_args& a, hipStream_t stream)
{
    const dim3 grid((uint32_t)((int64_t)a.c.num_seqs * a.c.kv_heads * a.splits * a.row_tiles)), block(64 * WAVES);
    if (a.chosen) {
        const dim3 tokens((uint32_t)((int64_t)a.c.num_seqs * a.c.max_new * a.c.kv_heads * a.splits * a.row_tiles));
        LORA_LAUNCH(LORA_K_CACHE_ATTENTION_CHOSEN, (cache_attention_kernel<T, DP, CT, false, WAVES, true>), tokens, block, 0, stream, a);
    } else if (a.scores) LORA_LAUNCH(LORA_K_CACHE_ATTENTION, (cache_attention_kernel<T, DP, CT, true, WAVES, false>), grid, block, 0, stream, a);
    else LORA_LAUNCH(LORA_K_CACHE_ATTENTION, (cache_attention_kernel<T, DP, CT, false, WAVES, false>), grid, block, 0, stream, a);
}

template <typename T, int DP>
void launch_main(const cache_attention_args& a, hipStream_t stream)
{
    if constexpr (cache_tile_rows(sizeof(T) == 4, DP) == 32)
        if ((int64_t)a.group * (a.chosen ? 1 : a.c.max_new) > 16) return launch_shape<T, DP, 2, 4>(a, stream);
    if constexpr (DP <= 128)
        if (a.waves == 8) return launch_shape<T, DP, 1, 8>(a, stream);
    launch_shape<T, DP, 1, 4>(a, stream);
}

template <typename T>
hipError_t launch_all(const cache_attention_args& a, hipStream_t stream)
{
    switch (padded_head_dim(a.c.head_dim)) {
        case 64: launch_main<T, 64>(a, stream); break;
        case 128: launch_main<T, 128>(a, stream); break;
        default: launch_main<T, 256>(a, stream);
    }
    hipError_t e = hipGetLastError();
    const int64_t rows = a.splits > 1 ? (int64_t)a.c.num_seqs * a.c.max_new * a.num_heads : 0;
    const int chunks = a.scores ? (a.c.max_length + kWeightSlots - 1) / kWeightSlots : 0;
    const int64_t last = rows + (int64_t)a.c.num_seqs * a.c.kv_heads * chunks;
    if (e == hipSuccess && last > 0) {
        LORA_LAUNCH(LORA_K_CACHE_FINISH, (cache_finish_kernel<T>), dim3((uint32_t)last), dim3(kFinishThreads), 0, stream, a, (int)rows, chunks);
        e = hipGetLastError();
    }
    return e;
}
}  // namespace

hipError_t launch_cache_attention(const cache_attention_args& a, int32_t dtype, hipStream_t stream)
{
    return dtype == LORA_F32 ? launch_all<float>(a, stream) : launch_all<bf16_t>(a, stream);
}
