// Beam search's selection: the best continuations of a request's beams over the vocabulary (include/lora_abi.h, BEAMS).
//
// One pass over the logits.  A row's best num_out are enough, and of any part of a row its own best num_out: a wavefront keeps its part in
// registers, adds up exp(logit - its largest), and finds its best by a bound, the num_out-th largest of its lanes' largest logits:
// what is not below it are a few more than num_out, which are put in order by counting.  A second launch joins the parts: a row's log sum, and the
// request's best of all that is left.
//
// A row's candidates are in the logits' own order whatever is subtracted, but those of different beams meet within 1e-7 of each other
// now and then, so the sums are 64 bits, and an exponential's argument has its rounding carried on (exp2 of the product's upper part,
// times 1 + its lower part): what is left of an error is the hardware's exp2, one step of 32 bits, at random.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "device_util.h"
#include "kernels_sequences.h"
#include "launch.h"

namespace {

constexpr int kWaves = BEAM_THREADS / 64, kMost = LORA_MAX_BEAMS;
constexpr int kHeld = 256;                     // candidates of a wavefront that are put in order by counting

__device__ __forceinline__ int lanes_before(uint64_t mask, int n)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, (uint32_t)n));
#else
    return n;
#endif
}

// whole numbers in the order of the numbers that they stand for (no NaN); -0 is +0
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t order_of(double x)
{
    const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ double number_of(uint64_t u) { return __longlong_as_double((long long)(u >> 63 ? u & 0x7fffffffffffffffull : ~u)); }

// what the wavefront's lanes have put in LDS is there for its other lanes
__device__ __forceinline__ void wave_sync()
{
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#endif
}

template <typename N>
__device__ __forceinline__ N wave_max(N x)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const N y = __shfl_xor(x, off, 64);
        x = y > x ? y : x;
    }
    return x;
}

// exp(d), d <= 0
__device__ __forceinline__ float exp_of(float d)
{
    constexpr float LOG2E = 1.44269504088896340736f, LOG2E_LOW = 1.92596299112661746887e-8f, LN2 = 0.69314718055994530942f;
    d = fmaxf(d, -200.f);                      // (-inf among them)
    const float hi = d * LOG2E, lo = __builtin_fmaf(d, LOG2E, -hi) + d * LOG2E_LOW;
    const float e = __builtin_amdgcn_exp2f(hi);
    return __builtin_fmaf(e, lo * LN2, e);
}

// eight tokens from `token` on; -inf behind the row's end
template <typename T>
__device__ __forceinline__ void load8(const T* row, int token, int vocab, float* x)
{
    struct __attribute__((packed, aligned(sizeof(T)))) eight { T v[8]; };
    if (token + 8 <= vocab) {
        const eight u = *reinterpret_cast<const eight*>(row + token);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if constexpr (sizeof(T) == 2) x[i] = bf16_to_f32(u.v[i]);
            else x[i] = u.v[i];
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = token + i < vocab ? elem<T>::load(row + token + i) : -INFINITY;
}

// Is (x, i) before (y, j): the greater logit, of equal ones the lower token
__device__ __forceinline__ bool before(float x, int i, float y, int j) { return x > y || (x == y && i < j); }

template <typename T, int V>
__global__ __launch_bounds__(BEAM_THREADS) void beam_rows_kernel(beam_args a)
{
    __shared__ beam_entry held[kWaves][kHeld];
    __shared__ beam_entry best[kWaves][kMost];
    __shared__ beam_sum sums[kWaves];
    const int split = blockIdx.x % a.splits, row = blockIdx.x / a.splits, M = a.num_out;
    if (a.last_token && a.end_token >= 0 && a.last_token[row] == a.end_token) return;         // (beam_join_kernel does not look at it)
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T* const logits = static_cast<const T*>(a.logits) + (int64_t)row * a.ld;
    const int start = split * (BEAM_THREADS * V) + wave * (64 * V) + 8 * lane;         // of the lane's first eight; the next are 512 on
    auto token_of = [&](int i) { return start + i / 8 * 512 + i % 8; };
    float x[V];
#pragma unroll
    for (int i = 0; i < V; i += 8) load8(logits, token_of(i), a.vocab, x + i);
    float top = x[0];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        top = fmaxf(top, x[i]);
        bad |= !(x[i] < INFINITY);
    }
    // the bound: as many lanes as wanted have a logit that is not below it (its upper 16 bits are enough: all that is not below is looked at)
    const uint32_t mine = order_of(top) >> 16;
    uint32_t bound = 0;
#pragma unroll
    for (int bit = 15; bit >= 0; --bit) {
        const uint32_t t = bound | 1u << bit;
        if (__popcll(__ballot(mine >= t)) >= M) bound = t;
    }
    top = wave_max(top);
    bad = __ballot(bad) != 0;
    const float ref = fabsf(top) < INFINITY ? top : 0.f;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i) sum += (double)exp_of(x[i] - ref);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (lane == 0) sums[wave] = beam_sum{sum, ref, bad};
    // what is not below it (and is a number that can be chosen)
    const uint32_t least = bound << 16;
    int count = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const bool is = order_of(x[i]) >= least && x[i] > -INFINITY;
        const uint64_t mask = __ballot(is);
        if (mask == 0) continue;
        const int at = lanes_before(mask, count);
        if (is && at < kHeld) held[wave][at] = beam_entry{x[i], token_of(i)};
        count += __popcll(mask);
    }
    if (lane < M) best[wave][lane] = beam_entry{-INFINITY, -1};
    wave_sync();
    if (count <= kHeld) {
        for (int i = lane; i < count; i += 64) {
            const beam_entry e = held[wave][i];
            int rank = 0;
            for (int j = 0; j < count; ++j) {
                const beam_entry o = held[wave][j];
                rank += before(o.logit, o.token, e.logit, e.token);
            }
            if (rank < M) best[wave][rank] = e;
        }
    } else {
        // more equal ones than that: one after the other
        float past = INFINITY;
        int past_token = -1;
        for (int n = 0; n < M; ++n) {
            float most = -INFINITY;
            int token = 0x7fffffff;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (before(past, past_token, x[i], token_of(i)) && before(x[i], token_of(i), most, token)) {
                    most = x[i];
                    token = token_of(i);
                }
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) {
                const float y = __shfl_xor(most, off, 64);
                const int j = __shfl_xor(token, off, 64);
                if (before(y, j, most, token)) {
                    most = y;
                    token = j;
                }
            }
            if (!(most > -INFINITY)) break;
            if (lane == 0) best[wave][n] = beam_entry{most, token};
            past = most;
            past_token = token;
        }
    }
    __syncthreads();
    // the workgroup's best, of the wavefronts'
    beam_entry* const out = a.entries + ((int64_t)row * a.splits + split) * M;
    if (tid < kWaves * M) {
        const int w = tid / M;
        const beam_entry e = best[w][tid - w * M];
        int rank = 0, there = 0;
        for (int v = 0; v < kWaves; ++v)
            for (int j = 0; j < M; ++j) {
                const beam_entry o = best[v][j];
                if (o.token < 0) break;
                ++there;
                rank += before(o.logit, o.token, e.logit, e.token);
            }
        if (e.token >= 0 && rank < M) out[rank] = e;
        if (tid < M && tid >= there) out[tid] = beam_entry{-INFINITY, -1};
    }
    if (tid == 0) {
        beam_sum s = sums[0];
        for (int w = 1; w < kWaves; ++w) {
            const beam_sum o = sums[w];
            if (o.bad || !(o.sum > 0.0) || !(s.sum > 0.0)) {   // (-inf alone has no place on the scale)
                if (o.sum > 0.0) {
                    s.sum = o.sum;
                    s.top = o.top;
                }
                s.bad |= o.bad;
                continue;
            }
            const float ref_all = fmaxf(s.top, o.top);
            s.sum = s.sum * exp((double)(s.top) - ref_all) + o.sum * exp((double)o.top - ref_all);
            s.top = ref_all;
        }
        a.sums[(int64_t)row * a.splits + split] = s;
    }
}

// ---------------------------------------------------------------------------
// A workgroup a request.  Candidates in tiles of a thread each; a wavefront puts its own in order by counting and keeps num_out of them,
// which are put in order with the best so far.  A candidate: what it is worth, then what breaks ties, both greater is better, 0: none.
constexpr int kJoinThreads = BEAM_JOIN_THREADS, kJoinWaves = kJoinThreads / 64;
struct __align__(16) candidate {
    uint64_t worth, tie;       // tie: 63 - beam, the logit's order, 2^24 - 1 - token
};
__device__ __forceinline__ bool better(const candidate& x, const candidate& y) { return x.worth > y.worth || (x.worth == y.worth && x.tie > y.tie); }

__global__ __launch_bounds__(kJoinThreads) void beam_join_kernel(beam_args a)
{
    __shared__ candidate pool[(kJoinWaves + 1) * kMost];       // the wavefronts' best, behind them the best so far
    __shared__ candidate own[kJoinWaves][64];
    __shared__ double worth[kMost], lse[kMost];
    __shared__ int state[kMost];                               // 0: no continuation, 1: from its logits, 2: has ended
    const int group = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, M = a.num_out, B = a.beams;
    const int64_t row0 = (int64_t)group * B;
    for (int b = wave; b < B; b += kJoinWaves) {
        const int64_t row = row0 + b;
        const float score = a.score[row];
        const bool ended = a.last_token && a.end_token >= 0 && a.last_token[row] == a.end_token;
        double sum = 0.0;
        float top = -INFINITY;
        int bad = 0;
        if (!ended) {
            const beam_sum* const s = a.sums + row * a.splits;
            for (int i = lane; i < a.splits; i += 64) {
                if (s[i].sum > 0.0) top = fmaxf(top, s[i].top);
                bad |= s[i].bad;
            }
            top = wave_max(top);
            for (int i = lane; i < a.splits; i += 64)
                if (s[i].sum > 0.0) sum += s[i].sum * exp((double)s[i].top - (double)top);
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
            bad = __ballot(bad != 0) != 0;
        }
        if (lane == 0) {
            const bool scored = fabsf(score) < INFINITY;
            worth[b] = (double)score;
            lse[b] = sum > 0.0 ? (double)top + log(sum) : 0.0;
            state[b] = !scored ? 0 : ended ? 2 : sum > 0.0 && !bad ? 1 : 0;
        }
    }
    if (tid < M) pool[kJoinWaves * M + tid] = candidate{0, 0};
    __syncthreads();
    const int64_t each = (int64_t)a.splits * M, all = each * B;
    for (int64_t base = 0; base < all; base += kJoinThreads) {
        const int64_t at = base + tid;
        candidate c{0, 0};
        if (at < all) {
            const int b = (int)(at / each), st = state[b];
            const uint64_t tie = (uint64_t)(63 - b) << 56;
            if (st == 1) {
                const beam_entry e = a.entries[row0 * each + at];
                if (e.token >= 0) {
                    const double w = worth[b] + ((double)e.logit - lse[b]);
                    c = candidate{order_of(w), tie | (uint64_t)order_of(e.logit) << 24 | (uint32_t)(0xffffff - e.token)};
                }
            } else if (st == 2 && at == b * each)
                c = candidate{order_of(worth[b]), tie | (uint32_t)(0xffffff - a.end_token)};
        }
        // (as long as there is one among them that is better than the last of the best so far)
        const candidate worst = pool[kJoinWaves * M + M - 1];
        if (!__syncthreads_or(better(c, worst))) continue;
        own[wave][lane] = c;
        if (lane < M) pool[wave * M + lane] = candidate{0, 0};
        wave_sync();
        int rank = 0;
        for (int j = 0; j < 64; ++j) rank += better(own[wave][j], c);
        if (c.worth != 0 && rank < M) pool[wave * M + rank] = c;
        __syncthreads();
        const int count = (kJoinWaves + 1) * M;                // at most 576: a thread one or two
        candidate mine[2] = {{0, 0}, {0, 0}};
        int place[2] = {M, M};
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int i = tid + n * kJoinThreads;
            if (i >= count) continue;
            mine[n] = pool[i];
            if (mine[n].worth == 0) continue;
            place[n] = 0;
            for (int w = 0; w <= kJoinWaves; ++w)
                for (int j = 0; j < M; ++j) {
                    if (!better(pool[w * M + j], mine[n])) break;             // (in order)
                    ++place[n];
                }
        }
        __syncthreads();
        if (tid < M) pool[kJoinWaves * M + tid] = candidate{0, 0};
        __syncthreads();
#pragma unroll
        for (int n = 0; n < 2; ++n)
            if (place[n] < M) pool[kJoinWaves * M + place[n]] = mine[n];
        __syncthreads();
    }
    if (tid >= M) return;
    const candidate c = pool[kJoinWaves * M + tid];
    const int64_t out = (int64_t)group * M + tid;
    a.out_score[out] = c.worth == 0 ? -INFINITY : (float)number_of(c.worth);
    a.out_parent[out] = c.worth == 0 ? -1 : (int32_t)(row0 + 63 - (int)(c.tie >> 56));
    a.out_token[out] = c.worth == 0 ? -1 : 0xffffff - (int)(c.tie & 0xffffff);
}

template <typename T>
void launch_rows(const beam_args& a, hipStream_t stream)
{
    const dim3 grid((uint32_t)((int64_t)a.num_groups * a.beams * a.splits));
    if (a.chunk == BEAM_THREADS * BEAM_FEW) LORA_LAUNCH(LORA_K_BEAM_ROWS, (beam_rows_kernel<T, BEAM_FEW>), grid, dim3(BEAM_THREADS), 0, stream, a);
    else LORA_LAUNCH(LORA_K_BEAM_ROWS, (beam_rows_kernel<T, BEAM_MANY>), grid, dim3(BEAM_THREADS), 0, stream, a);
}
}  // namespace

hipError_t launch_beam_select(const beam_args& a, int32_t dtype, hipStream_t stream)
{
    if (dtype == LORA_F32) launch_rows<float>(a, stream);
    else launch_rows<bf16_t>(a, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    LORA_LAUNCH(LORA_K_BEAM_JOIN, beam_join_kernel, dim3((uint32_t)a.num_groups), dim3(kJoinThreads), 0, stream, a);
    return hipGetLastError();
}
