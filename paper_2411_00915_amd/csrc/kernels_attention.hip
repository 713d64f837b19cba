// Attention of a batch of prompts.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "device_util.h"
#include "kernels_attention.h"
#include "launch.h"
#include "mfma_tile.h"

// ---------------------------------------------------------------------------
// A workgroup takes up to 128 queries of one head, 32 a wavefront; keys and values come in tiles of BK tokens, one tile ahead of
// the products: straight to LDS where rows and heads are ALIGNED to 16 bytes, else element by element through registers.
//
//     S^T = K Q^T     keys are the rows of the product, so that a lane ends with 16 (of 32) keys of one query, and maximum and
//                     sum of the softmax meet in two lanes only
//     O^T = V^T P^T   the same registers, rounded to bf16, are the second operand as they are; V is read across (transposing
//                     LDS reads), tokens in the order that the first product left them in
//
// bf16: 32 x 32 x 16 products; fp32: 32 x 32 x 2 of exact products.  The softmax runs to base 2 (its factor goes with the
// scale, in 32 bits) against a maximum that is raised only where a weight would pass 2^8, and the weights' sum is that of the
// weights before they are rounded.
//
// What bounds it, bf16: matrix cores and the softmax's vector instructions, which run beside each other only in part.  Two prompts
// of 8192 tokens, 40 heads of 128: 1.35 ms, 1.02 PFLOP/s, matrix cores busy in 53 % of the cycles, vector units in 48 %, no bank
// conflicts.  Four of 1024 tokens, 32 heads: 52 us, 0.66 PFLOP/s: the workgroups' order leaves places empty at the end.  fp32, a
// product of which takes 64 cycles: four of 1024 tokens, 16 heads of 64, 139 us, 62 TFLOP/s, matrix cores busy in 38 %: all
// workgroups have a place at once, and those with the most keys take as long as the whole.  Rows that are not ALIGNED: 4096
// tokens, 32 heads of 128, 127 us against 64.
// bf16 weights are rounded to bf16 because the matrix cores take both operands in one type; outputs are then 2.1e-3 from 64-bit
// arithmetic (normwise), 1.6e-3 of which are the output's own rounding.
// Why so: 32 queries are a product's width, and four wavefronts share what is in LDS; of 64 keys a tile there are half the barriers
// and maxima (32: 1436 against 1315 us at the time), and heads past 128 have room for 32.  Few queries leave wavefronts without work: the
// plan gives those other heads of the same keys, or, where the chip is not full anyway, KS of them share the tile's keys and add up
// in the end (32 heads of 128 on 8, 8 x 20 queries behind 1000 keys: 20.6 -> 15.9 us; of 256 dims 41 -> 43: not there).
namespace {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short shortx4;

// What of rows x width bytes lies from `base` on, for loads of 16 bytes a lane straight to LDS; reads behind `bytes` give zeros
struct tile_source {
    u32x4 rsrc;
    __device__ __forceinline__ void set(const char* base, int64_t bytes)
    {
        const uint64_t b = reinterpret_cast<uint64_t>(base);
        rsrc[0] = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b);
        rsrc[1] = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32) & 0xffff);
        rsrc[2] = (uint32_t)__builtin_amdgcn_readfirstlane((int)min(max(bytes, (int64_t)0), (int64_t)0x7fffffff));
        rsrc[3] = 0x00020000u;
    }
    __device__ __forceinline__ void load(uint32_t offset, uint32_t lds) const
    {
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(rsrc), "s"(lds) : "memory");
#endif
    }
};

// places of 16-byte chunks in a row of LDS, so that the lanes of a read meet different banks
template <typename T, int DP>
__device__ __forceinline__ int key_place(int c, int row)
{
    constexpr int CH = DP * (int)sizeof(T) / 16;
    if constexpr (CH == 12) return (c + (row >> 2 & 3)) % 12;
    else if constexpr (CH == 8) return c ^ (row >> 1 & 7);
    else return c ^ (row & 15);
}
template <typename T, int DP>
__device__ __forceinline__ int key_chunk(int place, int row)      // the other way round
{
    if constexpr (DP * (int)sizeof(T) / 16 == 12) return (place + 12 - (row >> 2 & 3)) % 12;
    else return key_place<T, DP>(place, row);
}
template <typename T, int DP>
__device__ __forceinline__ int value_place(int c, int row)        // its own inverse
{
    constexpr int CH = DP * (int)sizeof(T) / 16;
    if constexpr (sizeof(T) == 4) return c ^ (row >> 2 & 1) << 3;
    else if constexpr (CH == 12) return c;
    else if constexpr (CH == 8) return c ^ (row >> 1 & 1) << 2;
    else return c ^ (row & 3) << 2;
}

// 16 bytes of elements, of which there are n
template <typename T>
__device__ __forceinline__ uint4 load_elements(const T* p, int n)
{
    constexpr int E = 16 / (int)sizeof(T);
    uint32_t u[4] = {};
    auto take = [&](int i) {
        if constexpr (sizeof(T) == 4) u[i] = __float_as_uint(p[i]);
        else u[i / 2] |= (uint32_t)p[i] << 16 * (i & 1);
    };
    if (n >= E)
#pragma unroll
        for (int i = 0; i < E; ++i) take(i);
    else
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i < n) take(i);
    return uint4{u[0], u[1], u[2], u[3]};
}

// two bf16, infinities and NaN as 0
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t u)
{
    return ((u & 0x7f80u) == 0x7f80u ? 0u : u & 0xffffu) | ((u & 0x7f800000u) == 0x7f800000u ? 0u : u & 0xffff0000u);
}

// the greater of the two lanes of a query
__device__ __forceinline__ float max_of_halves(float x)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
#else
    return x;
#endif
}

template <typename T, int DP, int BK, bool ALIGNED, int KS>
__global__ __launch_bounds__(256, DP <= 128 && KS == 1 ? 2 : 1) void attention_tiled_kernel(attention_args a)
{
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int ROW = DP * (int)sizeof(T), CH = ROW / 16;         // bytes and chunks of a token
    constexpr int LOADS = BK * CH / 256;                           // of a wavefront, for one tile of keys
    constexpr int NB = DP / 32, SB = BK / 32 / KS, PART = SB * 32;      // KS wavefronts share a tile's keys, PART of them each
    constexpr int QR = F32 ? DP / 2 : DP / 16;                      // fp32: a register per two dims; bf16: 8 dims a lane and product
    __shared__ __align__(1024) char lds[2][2][BK * ROW];            // buffer, keys / values
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
    const attention_tile t = a.items[blockIdx.x];
    if (t.heads == 0) return;
    const int part = KS == 1 ? 0 : wave % KS, team = wave / KS;
    const int waves = 4 / KS / t.heads, head = t.head + team / waves, row0 = team % waves * 32;      // this wavefront's head, and its first query
    const int D = a.head_dim;
    const char* const kb = static_cast<const char*>(a.k) + ((int64_t)t.kv_row0 * a.ldk + (int64_t)(t.head / a.group) * D) * (int)sizeof(T);
    const char* const vb = static_cast<const char*>(a.v) + ((int64_t)t.kv_row0 * a.ldv + (int64_t)(t.head / a.group) * D) * (int)sizeof(T);
    const int64_t kpitch = a.ldk * (int)sizeof(T), vpitch = a.ldv * (int)sizeof(T);
    const int tiles = (t.max_kv + BK - 1) / BK;

    // this lane's chunks of a tile: what is past head_dim is past every row, and comes as zeros
    uint32_t k_off[LOADS], v_off[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int p = (wave * LOADS + i) * 64 + lane, row = p / CH, place = p % CH;
        const int kc = key_chunk<T, DP>(place, row), vc = value_place<T, DP>(place, row);
        k_off[i] = kc * (16 / (int)sizeof(T)) < D ? (uint32_t)(row * kpitch + kc * 16) : 0x80000000u;
        v_off[i] = vc * (16 / (int)sizeof(T)) < D ? (uint32_t)(row * vpitch + vc * 16) : 0x80000000u;
    }
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(lds)) + wave * (LOADS * 1024);
    auto fetch = [&](int n) {
        if constexpr (!ALIGNED) {
#pragma unroll 2
            for (int i = 0; i < LOADS; ++i) {
                const int p = (wave * LOADS + i) * 64 + lane, row = p / CH, place = p % CH;
                const int kd = key_chunk<T, DP>(place, row) * (16 / (int)sizeof(T)), vd = value_place<T, DP>(place, row) * (16 / (int)sizeof(T));
                const bool there = n * BK + row < t.num_kv;
                const int64_t token = (int64_t)n * BK + (there ? row : 0);
                const uint4 k = load_elements(reinterpret_cast<const T*>(kb) + token * a.ldk + kd, there ? D - kd : 0);
                const uint4 v = load_elements(reinterpret_cast<const T*>(vb) + token * a.ldv + vd, there ? D - vd : 0);
                *reinterpret_cast<uint4*>(lds[n & 1][0] + p * 16) = k;
                *reinterpret_cast<uint4*>(lds[n & 1][1] + p * 16) = v;
            }
            return;
        }
        const int64_t left = (int64_t)t.num_kv - (int64_t)n * BK;          // rows; the last ends with its head
        tile_source s;
        s.set(kb + (int64_t)n * BK * kpitch, (left - 1) * kpitch + (int64_t)D * (int)sizeof(T));
#pragma unroll
        for (int i = 0; i < LOADS; ++i) s.load(k_off[i], lds0 + (n & 1) * (2 * BK * ROW) + i * 1024);
        s.set(vb + (int64_t)n * BK * vpitch, (left - 1) * vpitch + (int64_t)D * (int)sizeof(T));
#pragma unroll
        for (int i = 0; i < LOADS; ++i) s.load(v_off[i], lds0 + (n & 1) * (2 * BK * ROW) + BK * ROW + i * 1024);
    };

    if (tiles > 0) fetch(0);

    // queries; a negative scale turns their sign
    const int row = row0 + col;
    const bool valid = row < t.rows;
    const T* const qp = static_cast<const T*>(a.q) + (int64_t)(t.q_row0 + (valid ? row : 0)) * a.ldq + (int64_t)head * D;
    float qf[F32 ? QR : 1];
    op16 qb[F32 ? 1 : QR];
    if constexpr (F32) {
#pragma unroll
        for (int c = 0; c < QR / 4; ++c) {
            const int d = 8 * c + 4 * half;
            const uint4 x = !ALIGNED ? load_elements(qp + d, valid ? D - d : 0) : valid && d < D ? *reinterpret_cast<const uint4*>(qp + d) : uint4{0, 0, 0, 0};
            qf[4 * c] = __uint_as_float(x.x); qf[4 * c + 1] = __uint_as_float(x.y); qf[4 * c + 2] = __uint_as_float(x.z); qf[4 * c + 3] = __uint_as_float(x.w);
        }
        if (a.scale < 0.f)
#pragma unroll
            for (int i = 0; i < QR; ++i) qf[i] = -qf[i];
    } else {
        const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
        for (int s = 0; s < QR; ++s) {
            const int d = 16 * s + 8 * half;
            const uint4 u = !ALIGNED ? load_elements(qp + d, valid ? D - d : 0) : valid && d < D ? ld16(reinterpret_cast<const bf16_t*>(qp) + d) : uint4{0, 0, 0, 0};
            qb[s].u = uint4{u.x ^ sign, u.y ^ sign, u.z ^ sign, u.w ^ sign};
        }
    }
    const float c2 = fmaxf(fabsf(a.scale) * 1.44269504088896340736f, 1.40129846e-45f);      // (0 would make NaN of -inf, what is not seen)
    const int limit = valid ? max(0, min(t.num_kv, t.ahead + row + 1)) : 0;
    // of the wavefront's queries, what the first and the last see
    const int least = max(0, min(t.num_kv, t.ahead + row0 + 1));
    const int most = row0 < t.rows ? max(0, min(t.num_kv, t.ahead + min(t.rows, row0 + 32))) : 0;

    floatx16 acc[NB];
    float l = 0.f;
    // A weight of 0 does not hide infinities and NaN of a value from the product, scores near the end of 32 bits are past it
    // when scaled to base 2, and so are sums of values near it, with weights of up to 2^8.  Where the result holds infinities
    // or NaN, or a query that sees keys has no weight, the workgroup goes through its tiles once more: such values are taken
    // out of the products where some query does not see the token, scores are scaled behind the subtraction of their
    // maximum, and all of a query's weights together are at most 1/2.
    auto pass = [&](auto careful_) {
    constexpr bool careful = decltype(careful_)::value;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[n][i] = 0.f;
    float m = -INFINITY, ref = 0.f;
    l = 0.f;
    if (careful && tiles > 0) fetch(0);
    for (int n = 0; n < tiles; ++n) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();                                       // the tile is there, and nobody reads the other buffer any more
        if (n + 1 < tiles) fetch(n + 1);
        const int token0 = n * BK + part * PART;
        if (token0 >= most) continue;
        const char* const keys = lds[n & 1][0] + part * (PART * ROW);
        const char* const values = lds[n & 1][1] + part * (PART * ROW);
        floatx16 x[SB];
#pragma unroll
        for (int b = 0; b < SB; ++b) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[b][i] = 0.f;
            const int r = 32 * b + col;
            if constexpr (F32) {
#pragma unroll
                for (int c = 0; c < QR / 4; ++c) {
                    const float4 k = *reinterpret_cast<const float4*>(keys + r * ROW + key_place<T, DP>(2 * c + half, r) * 16);
                    x[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(k.x, qf[4 * c], x[b], 0, 0, 0);
                    x[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(k.y, qf[4 * c + 1], x[b], 0, 0, 0);
                    x[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(k.z, qf[4 * c + 2], x[b], 0, 0, 0);
                    x[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(k.w, qf[4 * c + 3], x[b], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int s = 0; s < QR; ++s) {
                    op16 k;
                    k.u = *reinterpret_cast<const uint4*>(keys + r * ROW + key_place<T, DP>(2 * s + half, r) * 16);
                    x[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.v, qb[s].v, x[b], 0, 0, 0);
                }
            }
        }
        const bool masked = token0 + PART > least;
        if (masked) {
            int first = limit - token0 - 4 * half;
            asm volatile("" : "+v"(first));                    // (a branch, not selects in every tile)
#pragma unroll
            for (int b = 0; b < SB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * b + 8 * (i >> 2) + (i & 3) >= first) x[b][i] = -INFINITY;
        }
        float mx = x[0][0];
#pragma unroll
        for (int b = 0; b < SB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, x[b][i]);
        mx = max_of_halves(mx) * (careful ? 1.f : c2);
        if (__ballot(mx > (careful ? m : m + 8.f))) {
            const float top = fmaxf(m, mx), alpha = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - top) * (careful ? c2 : 1.f));
            m = top;
            ref = top == -INFINITY ? 0.f : top;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] *= alpha;
        }
        float share = 1.f;
        if constexpr (careful) {                               // a power of 2 of at most 1 / (2 tiles BK), made anew so that no register is kept for it
            int count = tiles;
            asm volatile("" : "+s"(count));
            share = __uint_as_float((uint32_t)(94 + __builtin_clz(count) - __builtin_ctz(BK)) << 23);
        }
#pragma unroll
        for (int b = 0; b < SB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[b][i] = __builtin_amdgcn_exp2f(careful ? (x[b][i] - ref) * c2 : x[b][i] * c2 - ref) * share;
                l += x[b][i];
            }
        // values: fp32 one dim a lane, bf16 four tokens of a dim by a transposing read (of 16 lanes, lane i points at 4 dims of
        // token i/4 and gets dim i of the four tokens)
        auto value_f32 = [&](int token, int d) { return *reinterpret_cast<const float*>(values + token * ROW + value_place<T, DP>(d >> 2, token) * 16 + (d & 3) * 4); };
        auto value_bf16 = [&](int b, int s, int d, int lane) {  // tokens 32 b + 16 s + 4 half + (0..3) and 8 on
            union { shortx4 h[2]; op16 o; } u;
#if defined(__HIP_DEVICE_COMPILE__)
            const int c = 4 * d + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int token = 32 * b + 16 * s + 8 * e + 4 * (lane >> 5) + (lane >> 2 & 3);
                u.h[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) shortx4*)(values + token * ROW + value_place<T, DP>(c, token) * 16 + (lane & 1) * 8));
            }
#endif
            return u.o;
        };
        const bool wild = careful && masked;
        if constexpr (F32) {
#pragma unroll
            for (int b = 0; b < SB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
#pragma unroll
                    for (int d = 0; d < NB; ++d) {
                        float v = value_f32(32 * b + 8 * (i >> 2) + 4 * half + (i & 3), 32 * d + col);
                        if (wild) v = fabsf(v) < INFINITY ? v : 0.f;
                        acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, x[b][i], acc[d], 0, 0, 0);
                    }
        } else {
            op16 p[SB][2];
#pragma unroll
            for (int b = 0; b < SB; ++b)
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    p[b][s].u = uint4{pack_bf16(x[b][8 * s], x[b][8 * s + 1]), pack_bf16(x[b][8 * s + 2], x[b][8 * s + 3]),
                                      pack_bf16(x[b][8 * s + 4], x[b][8 * s + 5]), pack_bf16(x[b][8 * s + 6], x[b][8 * s + 7])};
            if (!wild)
#pragma unroll
                for (int b = 0; b < SB; ++b)
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int d = 0; d < NB; ++d) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value_bf16(b, s, d, lane).v, p[b][s].v, acc[d], 0, 0, 0);
            else {
                int here = lane;                               // (opaque, so that no address of this rare path is kept for it)
                asm volatile("" : "+v"(here));
#pragma unroll
                for (int b = 0; b < SB; ++b)
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int d = 0; d < NB; ++d) {
                            op16 v = value_bf16(b, s, d, here);
                            v.u = uint4{finite_or_zero(v.u.x), finite_or_zero(v.u.y), finite_or_zero(v.u.z), finite_or_zero(v.u.w)};
                            acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.v, p[b][s].v, acc[d], 0, 0, 0);
                            __builtin_amdgcn_sched_barrier(0);
                        }
            }
        }
        if (wild) {
            // the products above are over the finite values; what the others make of a dim of a query is found token by token
            int there = half;
            asm volatile("" : "+v"(there));
#pragma unroll 1
            for (int j = 0; j < PART; ++j) {
                const bool sees = token0 + j < limit;
#pragma unroll
                for (int d = 0; d < NB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int at = 32 * d + 8 * (i >> 2) + 4 * there + (i & 3);
                        const float v = elem<T>::load(reinterpret_cast<const T*>(values + j * ROW + value_place<T, DP>(at * (int)sizeof(T) / 16, j) * 16) +
                                                      at % (16 / (int)sizeof(T)));
                        acc[d][i] += sees && !(fabsf(v) < INFINITY) ? v : 0.f;
                        asm volatile("" : "+v"(there));
                    }
            }
        }
    }

    l += __shfl_xor(l, 32, 64);
    if constexpr (KS > 1) {                                    // the first of the wavefronts gets the others' sums
        static_assert(4 / KS * ((KS - 1) * NB * 16 + 2 * KS) * 256 <= sizeof(lds), "they pass through the tiles' space");
        float* const space = reinterpret_cast<float*>(lds) + team * ((KS - 1) * NB * 16 + 2 * KS) * 64 + lane;
        float* const stats = space + (KS - 1) * NB * 16 * 64;
        __syncthreads();
        stats[2 * part * 64] = m;
        __syncthreads();
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < KS; ++w) top = fmaxf(top, stats[2 * w * 64]);
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * (careful ? c2 : 1.f));
        l *= f;
#pragma unroll
        for (int d = 0; d < NB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] *= f;
        if (part > 0) {
            stats[(2 * part + 1) * 64] = l;
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) space[((part - 1) * NB * 16 + d * 16 + i) * 64] = acc[d][i];
        }
        __syncthreads();
        if (part == 0)
#pragma unroll
            for (int w = 1; w < KS; ++w) {
                l += stats[(2 * w + 1) * 64];
#pragma unroll
                for (int d = 0; d < NB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[d][i] += space[((w - 1) * NB * 16 + d * 16 + i) * 64];
            }
    }
    };
    pass(std::false_type{});
    float sum = l;                                             // (not finite where one of them is not, or they are past its range)
#pragma unroll
    for (int d = 0; d < NB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += fabsf(acc[d][i]);
    if (__syncthreads_or(part == 0 && (!(sum < INFINITY) || (l == 0.f && limit > 0)))) pass(std::true_type{});
    if (part > 0) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* const out = static_cast<T*>(a.o) + (int64_t)(t.q_row0 + (valid ? row : 0)) * a.ldo + (int64_t)head * D;
#pragma unroll
    for (int d = 0; d < NB; ++d)
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int at = 32 * d + 2 * i + 4 * half;
                if constexpr (!ALIGNED) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (valid && at + e < D) out[at + e] = acc[d][i + e] * inv;
                } else if (valid && at < D)
                    *reinterpret_cast<float4*>(out + at) = float4{acc[d][i] * inv, acc[d][i + 1] * inv, acc[d][i + 2] * inv, acc[d][i + 3] * inv};
            }
        } else {
#if defined(__HIP_DEVICE_COMPILE__)
            // 4 dims of a query in each half of the wavefront: two such pairs change places to stores of 8 dims a lane
#pragma unroll
            for (int i = 0; i < 16; i += 8) {
                uint32_t u[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] = pack_bf16(acc[d][i + 2 * e] * inv, acc[d][i + 2 * e + 1] * inv);
                const auto x = __builtin_amdgcn_permlane32_swap(u[0], u[2], false, false), y = __builtin_amdgcn_permlane32_swap(u[1], u[3], false, false);
                const int at = 32 * d + 2 * i + 8 * half;
                if constexpr (!ALIGNED) {
                    const uint32_t w[4] = {x[0], y[0], x[1], y[1]};
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (valid && at + e < D) out[at + e] = (bf16_t)(w[e / 2] >> 16 * (e & 1));
                } else if (valid && at < D)
                    *reinterpret_cast<uint4*>(out + at) = uint4{x[0], y[0], x[1], y[1]};
            }
#endif
        }
}
}  // namespace

hipError_t launch_attention(const attention_args& a, int32_t dtype, hipStream_t stream)
{
    const int64_t es = dtype == LORA_F32 ? 4 : 2;
    const uintptr_t all = reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v) | reinterpret_cast<uintptr_t>(a.o) |
                          (uintptr_t)((a.ldq | a.ldk | a.ldv | a.ldo | a.head_dim) * es);
    const attention_instance n = choose_attention(dtype, a.head_dim, a.most_rows, (all & 15) == 0, std::max(a.ldk, a.ldv) * es);
    const dim3 grid((uint32_t)a.num_items);
#define INSTANCE(ID, T, DP, BK, ALIGNED, KS)                                                                                                \
    if (n.dims == DP && n.keys == BK && n.sharing == KS && (bool)n.aligned == ALIGNED) {                                                    \
        LORA_LAUNCH(ID, (attention_tiled_kernel<T, DP, BK, ALIGNED, KS>), grid, dim3(256), 0, stream, a);                                   \
        return hipGetLastError();                                                                                                           \
    }
#define TILED(T, DP, BK)                                                                                                                    \
    INSTANCE(LORA_K_ATTENTION_TILED, T, DP, BK, true, 1)                                                                                    \
    INSTANCE(LORA_K_ATTENTION_UNALIGNED, T, DP, BK, false, 1)
#define SHARED(T, DP, BK, KS) INSTANCE(LORA_K_ATTENTION_SHARED, T, DP, BK, true, KS)
    if (dtype == LORA_F32) {
        SHARED(float, 64, 128, 4)
        SHARED(float, 128, 64, 2)
        TILED(float, 64, 32)
        TILED(float, 128, 32)
        TILED(float, 256, 32)
    } else {
        SHARED(bf16_t, 64, 128, 4)
        SHARED(bf16_t, 96, 128, 4)
        SHARED(bf16_t, 128, 128, 4)
        SHARED(bf16_t, 128, 128, 2)
        TILED(bf16_t, 64, 64)
        TILED(bf16_t, 96, 64)
        TILED(bf16_t, 128, 64)
        TILED(bf16_t, 256, 32)
    }
    return hipErrorInvalidValue;                               // (not reached: these are all that there are)
}
