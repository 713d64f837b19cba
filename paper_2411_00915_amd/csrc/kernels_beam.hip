// Beam search's selection: the best continuations of a request's beams over the vocabulary (include/lora_abi.h, BEAMS).
//
// One pass over the logits.  A row's best num_out are enough, and of any part of a row its own best num_out.  A workgroup goes through its
// part a unit of 4096 tokens at a time, 16 a lane in registers, the next unit's loads on their way.  It keeps a bound that num_out tokens
// are known not to be below: at first the num_out-th largest of the lanes' largest logits (16 ballots find it), later of the candidates.
// What is not below the bound goes to LDS, in the mean 41 of a wavefront's 16384 tokens for 16 candidates; everything else is in the sum
// of exponentials and nowhere else: four instructions a token (fused multiply-add, exp2, sum, half a maximum) and one that takes it out of its
// word.  Equal logits by the hundred, which no bound parts, have a path of their own: the num_out-th largest of a unit bit by bit, and
// the first of those that are equal to it.  A second launch joins the parts: a row's log sum, and the request's best of what is left, again
// by a bound over all threads and by counting.
//
// A row's candidates are in the logits' own order whatever is subtracted, but those of different beams meet within 1e-7 of each other
// now and then.  So the candidates' exponentials, which are the largest, are 64 bits, and so are the sums; the others are the hardware's
// exp2 of a product with log2(e) that is rounded once, eight of them added in 32 bits.  With u = 2^-24, g the reference less the logit: g u by the
// product's rounding, 0.224 g u by that of log2(e), 2 u by exp2, 7 u by the sum; the weighted mean of g is at most log(vocab) (the weights'
// entropy), so a log sum is off by (9 + 1.225 log(vocab)) u at most, 1.4e-6 for 131072 tokens.  Measured: 3e-8 for normal logits, where these
// even out, 6e-7 for one logit above 131071 equal ones, which are all rounded alike (that with the rounding of the score).  Without the
// product's roundings (their sum beside the exponentials', six instructions more a logit) 64 requests of 8 beams take 53 us in place of 46.6.
//
// 64 requests of 8 beams over 131072 tokens, 16 candidates: 40.8 us and 7.6, 134 MB at 3.3 TB/s (vector instructions busy in 50 %; 37.1 while wavefronts
// read each other's bounds whenever they liked; a bound that does not rise 320); four beams over 32000: 8.0 and 7.0,
// the chain load -> bound -> exponentials -> candidates -> join.
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

// V tokens of a lane, 16 bytes of them in a row, the next 1024 bytes on, as they lie in memory
template <typename T, int V>
struct lane_words {
    static constexpr int EACH = 16 / sizeof(T), LOADS = V / EACH;
    uint32_t w[4 * LOADS];
    // (offsets of 32 bits from the row: one register, and the row's in scalar ones)
    __device__ __forceinline__ void load(const T* row, uint32_t token)
    {
        struct __attribute__((packed, aligned(sizeof(T)))) words { uint32_t w[4]; };
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const words u = *reinterpret_cast<const words*>(reinterpret_cast<const char*>(row) + (token * (uint32_t)sizeof(T) + 1024u * i));
#pragma unroll
            for (int e = 0; e < 4; ++e) w[4 * i + e] = u.w[e];
        }
    }
    __device__ __forceinline__ float operator()(int i) const
    {
        if constexpr (sizeof(T) == 2) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else return __uint_as_float(w[i]);
    }
};

// Is (x, i) before (y, j): the greater logit, of equal ones the lower token
__device__ __forceinline__ bool before(float x, int i, float y, int j) { return x > y || (x == y && i < j); }

// the greatest number of BITS bits that no fewer than `wanted` lanes reach; 0 where there are too few
template <int BITS>
__device__ __forceinline__ uint32_t reached(uint32_t mine, int wanted)
{
    uint32_t bound = 0;
#pragma unroll
    for (int bit = BITS - 1; bit >= 0; --bit) {
        const uint32_t t = bound | 1u << bit;
        if (__popcll(__ballot(mine >= t)) >= wanted) bound = t;
    }
    return bound;
}

// A wavefront's candidates in LDS, and the exponentials of all else
constexpr float LOG2E = 1.44269504088896340736f;
struct wave_state {
    beam_entry* held;          // [kHeld]; the first `summed` are in `sum` already
    int count, summed;
    float bound;               // what is below it is no candidate
    double sum;                // of exp(logit - ref), this lane's part
    double ref;                // about the bound, or above it
    // exp(x - ref) is exp2(x LOG2E - less_of), as ref is less_of / LOG2E; but past 1e9, where less_of is too coarse, exp2((x - less_of) LOG2E)
    float less_of;
    bool far;
    template <bool FAR>
    __device__ __forceinline__ float fast(float x) const
    {
        return __builtin_amdgcn_exp2f(FAR ? (x - less_of) * LOG2E : __builtin_fmaf(x, LOG2E, -less_of));
    }
};

__device__ __forceinline__ void raise_ref(wave_state& s, float to)
{
    const bool far = !(fabsf(to) < 1e9f);
    const float less_of = far ? to : to * LOG2E;
    const double ref = far ? (double)to : (double)less_of / (double)LOG2E;
    if (ref > s.ref) {
        s.sum = s.sum == 0.0 ? 0.0 : s.sum * exp(s.ref - ref);
        s.ref = ref;
        s.less_of = less_of;
        s.far = far;
    }
}

// Those of the candidates that are not in the sum into it
__device__ __forceinline__ void add_held(wave_state& s, int lane)
{
    float top = -INFINITY;
    for (int i = s.summed + lane; i < s.count; i += 64) top = fmaxf(top, s.held[i].logit);
    top = wave_max(top);
    if (fabsf(top) < INFINITY) raise_ref(s, top);
    for (int i = s.summed + lane; i < s.count; i += 64) s.sum += exp((double)s.held[i].logit - s.ref);
    s.summed = s.count;
}

// numbers from their order
__device__ __forceinline__ float number_of(uint32_t u) { return __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~u); }

// (NaN and +inf raise nothing)
__device__ __forceinline__ void raise_bound(wave_state& s, float to)
{
    if (to > s.bound && to < INFINITY) {
        s.bound = to;
        raise_ref(s, to);
    }
}

// above a number; what is below the bound is then not above it, so that it is the reference of the exponentials (also of the largest
// finite number, above which there is no bound)
__device__ __forceinline__ void raise_above(wave_state& s, float last)
{
    const float to = number_of(order_of(last) + 1);
    if (to > s.bound && to < INFINITY) s.bound = to;
    if (last < INFINITY) raise_ref(s, last);
}

// LDS is full: the best num_out of the candidates are kept.  What comes later has higher tokens, so it has to be above the last of them.
__device__ __forceinline__ void keep_best(wave_state& s, int M, int lane)
{
    wave_sync();
    add_held(s, lane);
    beam_entry mine[kHeld / 64];
    int rank[kHeld / 64];
#pragma unroll
    for (int n = 0; n < kHeld / 64; ++n) {
        mine[n] = s.held[min(n * 64 + lane, s.count - 1)];
        rank[n] = n * 64 + lane < s.count ? 0 : M;
    }
    for (int j = 0; j < s.count; ++j) {
        const beam_entry o = s.held[j];
#pragma unroll
        for (int n = 0; n < kHeld / 64; ++n) rank[n] += before(o.logit, o.token, mine[n].logit, mine[n].token);
    }
    wave_sync();
#pragma unroll
    for (int n = 0; n < kHeld / 64; ++n)
        if (rank[n] < M) s.held[rank[n]] = mine[n];
    wave_sync();
    if (s.count >= M) raise_above(s, s.held[M - 1].logit);
    s.count = s.summed = min(s.count, M);
}

// The same of four numbers a lane
__device__ __forceinline__ uint32_t reached_of_four(const uint32_t* mine, int wanted)
{
    uint32_t bound = 0;
#pragma unroll 1
    for (int bit = 15; bit >= 0; --bit) {
        const uint32_t t = bound | 1u << bit;
        int count = 0;
#pragma unroll
        for (int n = 0; n < kHeld / 64; ++n) count += __popcll(__ballot(mine[n] >= t));
        if (count >= wanted) bound = t;
    }
    return bound;
}

// Raises the bound by the candidates: num_out of them are not below it.  Returns the upper 16 bits of what it found, and what the wavefront's
// share of num_out are not below in *share, which only rises.
__device__ __forceinline__ uint32_t raise_by_held(wave_state& s, int M, int lane, uint32_t* share)
{
    wave_sync();
    const int part = (M + kWaves - 1) / kWaves;
    uint32_t few, least;
    if (s.count <= 64) {
        const uint32_t mine = lane < s.count ? order_of(s.held[lane].logit) >> 16 : 0u;
        few = reached<16>(mine, part);
        least = reached<16>(mine, M);
    } else {
        uint32_t mine[kHeld / 64];
#pragma unroll
        for (int n = 0; n < kHeld / 64; ++n) mine[n] = n * 64 + lane < s.count ? order_of(s.held[n * 64 + lane].logit) >> 16 : 0u;
        few = reached_of_four(mine, part);
        least = reached_of_four(mine, M);
    }
    *share = max(*share, few);
    raise_bound(s, number_of(least << 16));
    return least;
}

// The least of the wavefronts' shares: num_out of the workgroup's candidates are not below it.  Behind a barrier, so that what a row's sum is
// made of does not depend on who was first; slots[2], in turns, so that one barrier an exchange is enough.
__device__ __forceinline__ uint32_t exchange(uint32_t (*slots)[kWaves], int turn, uint32_t share, int wave, int lane)
{
    uint32_t* const slot = slots[turn & 1];
    if (lane == 0) slot[wave] = share;
    __syncthreads();
    uint32_t all = slot[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) all = min(all, slot[w]);
    return all;
}

template <typename T, int V>
__global__ __launch_bounds__(BEAM_THREADS, 4) void beam_rows_kernel(beam_args a)
{
    __shared__ beam_entry held[kWaves][kHeld];
    __shared__ double sums[kWaves];
    __shared__ double refs[kWaves];
    __shared__ uint32_t slots[2][kWaves], shares[kWaves];
    __shared__ int counts[kWaves];
    constexpr int UNIT = BEAM_THREADS * V, PART = 64 * V, EACH = lane_words<T, V>::EACH;
    const int split = blockIdx.x % a.splits, row = blockIdx.x / a.splits, M = a.num_out;
    const bool ends = a.last_token && a.end_token >= 0;
    const int last = ends ? a.last_token[row] : 0;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const T* const logits = static_cast<const T*>(a.logits) + (int64_t)row * a.ld;
    wave_state s{held[wave], 0, 0, -3.402823466e+38f, 0.0, -INFINITY, -3.402823466e+38f, true};      // (-inf is not chosen; NaN: the row is not)
    const int begin = split * a.chunk, end = min(begin + a.chunk, a.vocab);
    // The lane's first token of a unit.  A part that the row's end cuts is loaded from so far before its place, and what it has in common
    // with the part before it is masked.
    auto start_of = [&](int unit) { return max(min(unit + wave * PART, a.vocab - PART), 0) + EACH * lane; };
    int look = 16;                                                 // candidates at which they are looked at for a better bound
    int turn = 0, done = 0;                                        // exchanges and units so far
    uint32_t share = 0;                                            // what the wavefront's share of num_out are not below
    lane_words<T, V> next;
    if (V != BEAM_FEW || a.vocab >= PART) next.load(logits, start_of(begin));      // (on their way together with the last token)
    if (ends && last == a.end_token) return;                       // (beam_join_kernel does not look at it)
#pragma unroll 1
    for (int unit = begin; unit < end; unit += UNIT) {
        const int start = start_of(unit), first = unit + wave * PART;
        auto token_of = [&](int i) { return start + i / EACH * (64 * EACH) + i % EACH; };
        float x[V];
        if (V != BEAM_FEW || a.vocab >= PART) {                    // (divide_beams: rows of many units have a part)
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = next(i);
            if (unit + UNIT < end) next.load(logits, start_of(unit + UNIT));
            if (first + PART > a.vocab)
#pragma unroll
                for (int i = 0; i < V; ++i) x[i] = token_of(i) >= first ? x[i] : -INFINITY;
        } else {                                                   // (no branch over the lanes, so that all loads are on their way together)
#pragma unroll
            for (int i = 0; i < V; ++i)
                x[i] = elem<T>::load(reinterpret_cast<const T*>(reinterpret_cast<const char*>(logits) + (uint32_t)min(token_of(i), a.vocab - 1) * (uint32_t)sizeof(T)));
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = token_of(i) < a.vocab && token_of(i) >= first ? x[i] : -INFINITY;
        }
        float top = x[0];
#pragma unroll
        for (int i = 1; i < V; ++i) top = fmaxf(top, x[i]);
        // Bounds (the upper 16 bits do: all that is not below is looked at).  Of the first tokens two, of which the greater is taken: in
        // every wavefront its share of num_out lanes have a logit that is not below the first, in this one num_out lanes one that is
        // not below the second.  The second is what there is where another wavefront's part is masked or behind the row's end,
        // and again where the first tokens were.
        if (unit == begin) {
            const uint32_t mine = order_of(top) >> 16, least = reached<16>(mine, M);
            share = reached<16>(mine, (M + kWaves - 1) / kWaves);
            raise_bound(s, number_of(max(least, exchange(slots, turn++, share, wave, lane)) << 16));
        } else if (__popcll(__ballot(top >= s.bound)) > M)
            raise_bound(s, number_of(reached<16>(order_of(top) >> 16, M) << 16));
        // what is not below the bound goes to LDS, and is as good as masked here
        const uint64_t lanes = __ballot(top >= s.bound);
        if (lanes != 0) {
            int hits = __popcll(lanes) * V;                        // at most
            if (s.count + hits > kHeld) {
                hits = 0;
#pragma unroll
                for (int i = 0; i < V; ++i) hits += __popcll(__ballot(x[i] >= s.bound));
                if (s.count + hits > kHeld && s.count > kHeld - kMost) keep_best(s, M, lane);
            }
            if (s.count + hits <= kHeld) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const bool is = x[i] >= s.bound;
                    const uint64_t mask = __ballot(is);
                    if (mask != 0) {
                        if (is) s.held[lanes_before(mask, s.count)] = beam_entry{x[i], token_of(i)};
                        s.count += __popcll(mask);
                        x[i] = is ? -INFINITY : x[i];
                    }
                }
                if (s.count >= look) {
                    raise_by_held(s, M, lane, &share);
                    look = s.count + max(8, M / 2);
                }
            } else {
                // More than LDS holds (many equal ones): the best num_out of these tokens alone.  All above the num_out-th largest number, and
                // of those that are equal to it the first few; no later token that is equal to it will do.  (There are more than num_out.)
                uint32_t limit = 0;
#pragma unroll 1
                for (int bit = 31; bit >= 0; --bit) {
                    const float next = number_of(limit | 1u << bit);
                    int count = 0;
#pragma unroll
                    for (int i = 0; i < V; ++i) count += __popcll(__ballot(x[i] >= next));
                    if (count >= M) limit |= 1u << bit;
                }
                const float last = number_of(limit);
                int left = M;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const bool is = x[i] > last;
                    const uint64_t mask = __ballot(is);
                    if (is) s.held[lanes_before(mask, s.count)] = beam_entry{x[i], token_of(i)};
                    s.count += __popcll(mask);
                    left -= __popcll(mask);
                    x[i] = is ? -INFINITY : x[i];
                }
#pragma unroll
                for (int i = 0; i < V; i += EACH) {                // tokens go up along a lane's EACH, then along the lanes
                    int place = 0, all = 0;
#pragma unroll
                    for (int e = i; e < i + EACH; ++e) {
                        const uint64_t mask = __ballot(x[e] == last);
                        place = lanes_before(mask, place);
                        all += __popcll(mask);
                    }
#pragma unroll
                    for (int e = i; e < i + EACH; ++e)
                        if (x[e] == last) {
                            if (place < left) {
                                s.held[s.count + place] = beam_entry{x[e], token_of(e)};
                                x[e] = -INFINITY;
                            }
                            ++place;
                        }
                    const int taken = min(all, left);
                    s.count += taken;
                    left -= taken;
                }
                raise_above(s, last);
            }
        }
        // the exponentials of all else: eight in 32 bits, their sums in 64 (NaN is among these, and makes the sum NaN)
        auto add = [&](auto far_) {
#pragma unroll
            for (int i = 0; i < V; i += 8) {
                float part = 0.f;
#pragma unroll
                for (int e = i; e < i + 8; ++e) part += s.fast<decltype(far_)::value>(x[e]);
                s.sum += (double)part;
            }
        };
        if (__builtin_expect(__builtin_amdgcn_readfirstlane(s.far), 0)) add(std::true_type{});
        else add(std::false_type{});
        // Of shuffled logits as many are above the bound in the first units as in as many again.  (64 requests of 8 beams over 131072 tokens 46.6 us in
        // all, with the shares found anew here 48.1, with no exchange behind the first unit 47.6, for 64 candidates 68, 71 and 94)
        ++done;
        if ((done & (done - 1)) == 0 && unit + UNIT < end) raise_bound(s, number_of(exchange(slots, turn++, share, wave, lane) << 16));
    }
    wave_sync();
    add_held(s, lane);
    uint32_t limit = s.count > 0 ? raise_by_held(s, M, lane, &share) : 0u;
    double sum = s.sum;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (lane == 0) {
        sums[wave] = sum;
        refs[wave] = s.ref;
        shares[wave] = share;
    }
    __syncthreads();
    // What is left of the candidates, now that all wavefronts' bounds are there, to the front; then the workgroup's best in order
    uint32_t least_share = shares[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) least_share = min(least_share, shares[w]);
    limit = max(limit, least_share) << 16;                         // (not the bound, which may be above what is kept of equal ones)
    int kept = 0;
    for (int n = 0; n < s.count; n += 64) {                        // (what is moved goes no further back than it was)
        const beam_entry e = s.held[min(n + lane, s.count - 1)];
        const bool is = n + lane < s.count && order_of(e.logit) >= limit;
        const uint64_t mask = __ballot(is);
        wave_sync();
        if (is) s.held[lanes_before(mask, kept)] = e;
        kept += __popcll(mask);
        wave_sync();
    }
    s.count = kept;
    if (lane == 0) counts[wave] = s.count;
    __syncthreads();
    beam_entry* const out = a.entries + ((int64_t)row * a.splits + split) * M;
    int all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) all += counts[w];
    for (int n = tid; n < all; n += BEAM_THREADS) {
        int w = 0, at = n;
        while (at >= counts[w]) at -= counts[w++];
        const beam_entry e = held[w][at];
        int rank = 0;
        for (int v = 0; v < kWaves; ++v) {
            const int there = __builtin_amdgcn_readfirstlane(counts[v]);
            int j = 0;
            for (; j + 8 <= there; j += 8) {                       // (eight on their way together)
                beam_entry o[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = held[v][j + k];
#pragma unroll
                for (int k = 0; k < 8; ++k) rank += before(o[k].logit, o[k].token, e.logit, e.token);
            }
            for (; j < there; ++j) {
                const beam_entry o = held[v][j];
                rank += before(o.logit, o.token, e.logit, e.token);
            }
        }
        if (rank < M) out[rank] = e;
    }
    if (tid < M && tid >= all) out[tid] = beam_entry{-INFINITY, -1};
    if (wave == kWaves - 1) {
        // the sums on one scale; one of nothing but -inf has no place on it
        const double part = lane < kWaves ? sums[lane] : 0.0;
        const bool some = part != 0.0;
        const double ref = some ? refs[lane & (kWaves - 1)] : -INFINITY, scale = wave_max(ref);
        double of_all = some ? part * exp(ref - scale) : 0.0;
#pragma unroll
        for (int off = kWaves / 2; off > 0; off >>= 1) of_all += __shfl_xor(of_all, off, 64);
        if (lane == 0) a.sums[(int64_t)row * a.splits + split] = beam_sum{of_all, scale};
    }
}

// ---------------------------------------------------------------------------
// A workgroup a request.  Again a bound first, by what every thread's best candidate is worth, and what is not below it put in order
// by counting.  A candidate: what it is worth, then what breaks ties, both greater is better, 0: none.
constexpr int kJoinThreads = BEAM_JOIN_THREADS, kJoinWaves = kJoinThreads / 64, kJoinHeld = 1024;
struct __align__(16) candidate {
    uint64_t worth, tie;       // tie: 63 - beam, the logit's order, 2^24 - 1 - token
};
__device__ __forceinline__ bool better(const candidate& x, const candidate& y) { return x.worth > y.worth || (x.worth == y.worth && x.tie > y.tie); }

// the upper bits of what it is worth, rounded to 32 bits: in the same order, but for equal ones
__device__ __forceinline__ uint32_t about(const candidate& c) { return c.worth == 0 ? 0u : order_of((float)number_of(c.worth)) >> 12; }

__global__ __launch_bounds__(kJoinThreads) void beam_join_kernel(beam_args a)
{
    __shared__ candidate pool[kJoinHeld];
    __shared__ candidate best[kMost];
    __shared__ double worth[kMost], lse[kMost];
    __shared__ int state[kMost];                               // 0: no continuation, 1: from its logits, 2: has ended
    __shared__ uint32_t bounds[kJoinThreads];
    __shared__ int counter;
    const int group = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, M = a.num_out, B = a.beams;
    const int64_t row0 = (int64_t)group * B;
    const int64_t all = (int64_t)a.splits * M * B;
    if (tid == 0) counter = 0;
    if (tid < M) best[tid] = candidate{0, 0};
    // All that a row has, on its way together (of a beam that has ended, what was in the workspace: it is not used).
    constexpr int KEPT = 4;                                    // of a thread's candidates, in registers
    beam_entry near[KEPT];
#pragma unroll
    for (int i = 0; i < KEPT; ++i) near[i] = a.entries[row0 * a.splits * M + min((int64_t)(i * kJoinThreads + tid), all - 1)];
    for (int b = wave; b < B; b += kJoinWaves) {
        const int64_t row = row0 + b;
        const float score = a.score[row];
        const bool ends = a.last_token && a.end_token >= 0;
        const int last = ends ? a.last_token[row] : 0;
        const beam_sum* const s = a.sums + row * a.splits;
        const beam_sum own = s[min(lane, a.splits - 1)];
        const bool ended = ends && last == a.end_token;
        double sum = 0.0, ref = -INFINITY;
        if (!ended) {
            ref = own.ref;                                     // (-inf where there is nothing)
            for (int i = lane + 64; i < a.splits; i += 64) ref = fmax(ref, s[i].ref);
            ref = wave_max(ref);
            if (lane < a.splits && own.sum != 0.0) sum = own.sum * exp(own.ref - ref);
            for (int i = lane + 64; i < a.splits; i += 64)
                if (s[i].sum != 0.0) sum += s[i].sum * exp(s[i].ref - ref);
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
        }
        if (lane == 0) {
            const bool scored = fabsf(score) < INFINITY;
            worth[b] = (double)score;
            lse[b] = sum > 0.0 ? ref + log(sum) : 0.0;
            state[b] = !scored ? 0 : ended ? 2 : sum > 0.0 && sum < INFINITY ? 1 : 0;
        }
    }
    __syncthreads();
    const int each = a.splits * M;                             // of a beam (2^24 tokens in pieces of 2048, 64 each: 2^19)
    auto made_of = [&](int64_t n, const beam_entry& e) {       // candidate n < all
        const int b = (int)((uint32_t)n / (uint32_t)each), st = state[b];
        const uint64_t tie = (uint64_t)(63 - b) << 56;
        candidate c{0, 0};
        if (st == 1) {
            if (e.token >= 0)
                c = candidate{order_of(worth[b] + ((double)e.logit - lse[b])), tie | (uint64_t)order_of(e.logit) << 24 | (uint32_t)(0xffffff - e.token)};
        } else if (st == 2 && n == (int64_t)b * each)
            c = candidate{order_of(worth[b]), tie | (uint32_t)(0xffffff - a.end_token)};
        return c;
    };
    auto at = [&](int64_t n) { return made_of(n, a.entries[row0 * each + n]); };
    candidate kept[KEPT];
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
        const int64_t n = i * kJoinThreads + tid;
        kept[i] = n < all ? made_of(n, near[i]) : candidate{0, 0};
        mine = max(mine, about(kept[i]));
    }
    for (int64_t n = KEPT * kJoinThreads + tid; n < all; n += kJoinThreads) mine = max(mine, about(at(n)));
    bounds[tid] = mine;
    __syncthreads();
    uint32_t bound = 0, theirs[kJoinWaves];                    // the greatest number that num_out threads reach; 0: there are fewer
#pragma unroll
    for (int w = 0; w < kJoinWaves; ++w) theirs[w] = bounds[w * 64 + lane];
#pragma unroll 1
    for (int bit = 19; bit >= 0; --bit) {
        const uint32_t t = bound | 1u << bit;
        int reached = 0;
#pragma unroll
        for (int w = 0; w < kJoinWaves; ++w) reached += __popcll(__ballot(theirs[w] >= t));
        if (reached >= M) bound = t;
    }
    auto collect = [&](const candidate& c) {
        const bool is = c.worth != 0 && about(c) >= bound;
        const uint64_t mask = __ballot(is);
        if (mask == 0) return;
        int first = 0;
        if (lane == 0) first = atomicAdd(&counter, __popcll(mask));
        first = __builtin_amdgcn_readfirstlane(first);
        const int place = lanes_before(mask, first);
        if (is && place < kJoinHeld) pool[place] = c;          // (their order here does not matter: no two are equal)
    };
#pragma unroll
    for (int i = 0; i < KEPT; ++i) collect(kept[i]);
    for (int64_t base = KEPT * kJoinThreads; base < all; base += kJoinThreads) collect(base + tid < all ? at(base + tid) : candidate{0, 0});
    __syncthreads();
    const int count = __builtin_amdgcn_readfirstlane(counter);
    if (count <= kJoinHeld) {
#pragma unroll
        for (int i = 0; i < kJoinHeld / kJoinThreads; ++i) {
            const int n = i * kJoinThreads + tid;
            if (n >= count) break;
            const candidate c = pool[n];
            int rank = 0;
            int j = 0;
            for (; j + 8 <= count; j += 8) {                       // (eight on their way together)
                candidate o[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = pool[j + k];
#pragma unroll
                for (int k = 0; k < 8; ++k) rank += better(o[k], c);
            }
            for (; j < count; ++j) rank += better(pool[j], c);
            if (rank < M) best[rank] = c;
        }
    } else {
        // More: a tile of a thread each at a time, what is better than the last of the best so far put in order with them
        for (int64_t base = 0; base < all; base += kJoinThreads) {
            __syncthreads();
            candidate c = base + tid < all ? at(base + tid) : candidate{0, 0};
            if (!better(c, best[M - 1])) c = candidate{0, 0};
            if (!__syncthreads_or(c.worth != 0)) continue;
            pool[tid] = c;
            if (tid < M) pool[kJoinThreads + tid] = best[tid];
            __syncthreads();
            const candidate old = tid < M ? best[tid] : candidate{0, 0};
            int rank = 0, rank_old = 0;
            for (int j = 0; j < kJoinThreads + M; ++j) {
                const candidate o = pool[j];
                rank += better(o, c);
                rank_old += better(o, old);
            }
            __syncthreads();
            if (c.worth != 0 && rank < M) best[rank] = c;
            if (old.worth != 0 && rank_old < M) best[rank_old] = old;
        }
    }
    __syncthreads();
    if (tid >= M) return;
    const candidate c = best[tid];
    const int64_t out = (int64_t)group * M + tid;
    a.out_score[out] = c.worth == 0 ? -INFINITY : (float)number_of(c.worth);
    a.out_parent[out] = c.worth == 0 ? -1 : (int32_t)(row0 + 63 - (int)(c.tie >> 56));
    a.out_token[out] = c.worth == 0 ? -1 : 0xffffff - (int)(c.tie & 0xffffff);
}

template <typename T>
void launch_rows(const beam_args& a, hipStream_t stream)
{
    const dim3 grid((uint32_t)((int64_t)a.num_groups * a.beams * a.splits));
    if (a.unit == BEAM_THREADS * BEAM_FEW) LORA_LAUNCH(LORA_K_BEAM_ROWS, (beam_rows_kernel<T, BEAM_FEW>), grid, dim3(BEAM_THREADS), 0, stream, a);
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
