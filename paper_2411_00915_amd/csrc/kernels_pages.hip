// Pages given out and taken back on the device, and sequences that become others' (include/lora_abi.h, PAGES).
//
// A call is a few thousand whole numbers, so it is bound by its chain of dependent trips to memory: wanted length -> table ->
// users of the page written next -> free pages -> table -> slots.  Where the tables are small, one workgroup does all of it with barriers
// between the steps, and a thread its sequence's tokens where none has more than four (16 requests a token each: 4.7 us, of which 0.9 a prefix
// over the workgroup; 128 prompts, 8192 tokens: 13.4 us, 14.5 with a lane's tokens one behind the other and divisions by the page's size).
// Else pages are given back by one launch, a second looks for shared pages and for the free ones of every 4096, one workgroup decides, and a
// fourth launch writes tables and slots down (4096 requests, 287000 new tokens: 3.0, 4.2, 11.0 and 9.6 us; more than 4096 are 16 a thread, which it
// holds in scratch memory, 238 registers of them: 53 us for 8192, 89 for 16384; with one workgroup that looks for the free
// pages too, 52 in place of 11 and 4).
// What the atomics do (counts of users, the greatest of the keys of those that share a page) does not depend on their order.
#include <hip/hip_runtime.h>

#include <climits>
#include <type_traits>

#include "device_util.h"
#include "kernels_sequences.h"
#include "launch.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kList = 8192;                    // free pages that are kept in LDS
constexpr int kFew = 4;                        // tokens of a sequence that its thread writes down by itself (no more than a page has)
constexpr int kChunk = PAGES_CHUNK;            // entries or tokens of a sequence that a wavefront writes down

// how many lanes before this one are in the mask, on top of n
__device__ __forceinline__ int lanes_before(uint64_t mask, int n)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, (uint32_t)n));
#else
    return n;
#endif
}

// the page that a place is in (pages are mostly powers of two), and pages that hold so many tokens (at most 2^30)
__device__ __forceinline__ int page_number(const pages_args& p, int at)
{
    return (p.page_tokens & (p.page_tokens - 1)) == 0 ? at >> __builtin_ctz(p.page_tokens) : at / p.page_tokens;
}
__device__ __forceinline__ int pages_of(const pages_args& p, int tokens) { return page_number(p, tokens + p.page_tokens - 1); }
// of the tokens in the page of the last: 0 where it is full
__device__ __forceinline__ int tokens_inside(const pages_args& p, int tokens) { return tokens - page_number(p, tokens) * p.page_tokens; }
__device__ __forceinline__ int length_at(const pages_args& p, int s) { return min(max(p.length[s], 0), p.max_length); }
__device__ __forceinline__ bool known(const pages_args& p, int page) { return page >= 0 && page < p.num_pages; }

// a lane's number and those of the lanes before it
__device__ __forceinline__ int sum_upto(int n) { return wave_sum_upto(n); }
__device__ __forceinline__ int64_t sum_upto(int64_t n)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int64_t below = __shfl_up(n, off, 64);
        if (lane >= off) n += below;
    }
    return n;
}

// exclusive prefix of a thread's number over the workgroup, and the sum
template <typename N>
__device__ __forceinline__ N prefix(N n, N* sums, N* total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const N upto = sum_upto(n);
    __syncthreads();                           // (sums of the call before have been read)
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    N before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const N x = sums[w];
        before += w < wave ? x : 0;
        all += x;
    }
    *total = all;
    return before + upto - n;
}

// entry e of sequence s (between its old and its new end) is given back
__device__ __forceinline__ void give_back(const pages_args& p, int s, int e)
{
    int32_t* const entry = p.page_table + (int64_t)s * p.table_stride + e;
    const int page = *entry;
    if (known(p, page)) atomicSub(p.users + page, 1);
    *entry = -1;
}

// The users of a lane's pages, LOADS times four in a row, 256 on
struct __attribute__((packed, aligned(4))) four { int32_t x[4]; };
template <int LOADS>
__device__ __forceinline__ void load_users(const pages_args& p, int64_t mine, four* u)
{
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int64_t at = mine + 256 * i;
        if (at + 4 <= p.num_pages) u[i] = *reinterpret_cast<const four*>(p.users + at);
        else
#pragma unroll
            for (int c = 0; c < 4; ++c) u[i].x[c] = at + c < p.num_pages ? p.users[at + c] : 1;
    }
}

// The first `most` free pages in order, by one workgroup: how many there are of them.  list[i] is written for i < that.  u: the users of
// the first pages, where nothing has changed them (fresh)
constexpr int kFreeLoads = 4, kFreeWave = kFreeLoads * 256;    // pages of a wavefront at a time
__device__ __forceinline__ int64_t find_free(const pages_args& p, int64_t most, int32_t* list, int* sums, four* u, bool fresh)
{
    constexpr int LOADS = kFreeLoads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t found = 0;
    for (int64_t base = 0; base < p.num_pages && found < most; base += kWaves * kFreeWave) {
        const int64_t mine = base + wave * kFreeWave + 4 * lane;
        if (base > 0 || !fresh) load_users<LOADS>(p, mine, u);
        int before[LOADS], count = 0;                          // of the lanes below, and of the loads before
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            before[i] = count;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint64_t mask = __ballot(u[i].x[c] == 0);
                before[i] = lanes_before(mask, before[i]);
                count += __popcll(mask);
            }
        }
        __syncthreads();
        if (lane == 0) sums[wave] = count;
        __syncthreads();
        int64_t first = found;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            first += w < wave ? sums[w] : 0;
            found += sums[w];
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            int64_t rank = first + before[i];
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (u[i].x[c] == 0) {
                    if (rank < most) list[rank] = (int32_t)(mine + 256 * i + c);
                    ++rank;
                }
        }
    }
    return found < most ? found : most;
}

// the free page of that number, when part_first is where each part's begin: of the part it is in, the one of that place
__device__ __forceinline__ int free_page(const resize_args& a, int number)
{
    int lo = 0, hi = free_parts(a.p.num_pages);
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        (a.part_first[mid] <= number ? lo : hi) = mid;
    }
    return a.list[(int64_t)lo * FREE_PART + number - a.part_first[lo]];
}

// a new token's sequence, position and slot (row < num_tokens)
__device__ __forceinline__ void write_token(const resize_args& a, int row, int s, int position, int page)
{
    if (a.token_seq) a.token_seq[row] = s;
    if (a.token_position) a.token_position[row] = position;
    if (a.token_slot) a.token_slot[row] = known(a.p, page) ? (int64_t)page * a.p.page_tokens + tokens_inside(a.p, position) : -1;
}

// What a sequence has and wants, and the page that it would write next where that holds tokens already and has other users (else -1)
struct wish {
    int from, to, last;
    bool fits;                                 // the wanted length is one
    int page;                                  // that it would write next, if that holds tokens already
    int users;                                 // of that page
};
__device__ __forceinline__ wish wish_of(const resize_args& a, int s)
{
    const int wanted = a.wanted[s], from = length_at(a.p, s);
    const bool fits = wanted >= 0 && wanted <= a.p.max_length;
    return wish{from, fits ? wanted : from, -1, fits, -1, 0};
}
__device__ __forceinline__ void look_at_page(const pages_args& p, int s, wish& w)
{
    if (w.to <= w.from || tokens_inside(p, w.from) == 0) return;
    w.page = p.page_table[(int64_t)s * p.table_stride + page_number(p, w.from)];
    if (!known(p, w.page)) return;
    w.users = p.users[w.page];
    if (w.users > 1) w.last = w.page;
}

// One workgroup decides: a thread R sequences in a row.  ALL: R is 1, and nothing is left to other launches.  Else the launch before has
// left wishes where the grants go, and of each part of the pool the number of free pages.
template <int R, bool ALL>
__global__ __launch_bounds__(kThreads) void pages_decide_kernel(resize_args a)
{
    __shared__ int64_t sums_[kWaves];
    __shared__ int counts[kWaves];
    __shared__ int32_t near[ALL ? kList : 1];
    __shared__ page_grant grants[ALL ? kThreads : 1];
    const pages_args& p = a.p;
    const int tid = threadIdx.x, S = p.num_seqs, s0 = tid * R;
    wish w[R];
    bool shorter = false, some = false;
    four users[ALL ? kFreeLoads : 1];          // (asked for before it is known that they are wanted)
    if constexpr (ALL) load_users<kFreeLoads>(p, (int64_t)(tid >> 6) * kFreeWave + 4 * (tid & 63), users);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        w[r] = wish{0, 0, -1, false, -1, 0};
        if (s0 + r >= S) continue;
        if constexpr (ALL) w[r] = wish_of(a, s0 + r);
        else {
            const page_grant g = a.grants[s0 + r];
            w[r] = wish{g.from, g.to, g.first, g.row != 0, -1, 0};
        }
        shorter |= w[r].to < w[r].from;
    }
    if constexpr (ALL) {
        grants[tid] = page_grant{w[0].from, w[0].to, 0, 0};
        shorter = __syncthreads_or(shorter);
        if (shorter) {
            const int entries = S * p.table_stride;
            for (int e = tid; e < entries; e += kThreads) {
                const int s = e / p.table_stride, i = e - s * p.table_stride;
                const page_grant g = grants[s];
                if (g.to < g.from && i >= pages_of(p, g.to) && i < pages_of(p, g.from)) give_back(p, s, i);
            }
            __syncthreads();
        }
        if (tid < S) look_at_page(p, tid, w[0]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) some |= w[r].last >= 0;
    some = __syncthreads_or(some);
    // all of them leave the page; where nobody stays, the one with the most tokens in it keeps it
    auto key_of = [&](int r) { return -1 - (tokens_inside(p, w[r].from) * LORA_PAGES_MAX_SEQS + s0 + r); };
    if constexpr (ALL) {
        if (some) {
            // They meet in LDS, by page (half the places stay empty, so that every search ends); users never go down to 0 here, so what has
            // been asked for of the free pages stays right.
            constexpr int PLACES = 2 * kThreads;
            int* const pages = near, *const leave = near + PLACES, *const keeper = near + 2 * PLACES;
            static_assert(3 * PLACES <= kList, "");
            for (int i = tid; i < PLACES; i += kThreads) {
                pages[i] = -1;
                leave[i] = 0;
                keeper[i] = 0;
            }
            __syncthreads();
            const int page = w[0].last;
            int at = (int)((uint32_t)page * 0x9e3779b1u >> 21);
            if (page >= 0) {
                for (;;) {
                    const int there = atomicCAS(pages + at, -1, page);
                    if (there == -1 || there == page) break;
                    at = at + 1 & PLACES - 1;
                }
                atomicAdd(leave + at, 1);
                atomicMin(keeper + at, key_of(0));
            }
            __syncthreads();
            if (page >= 0) {
                const int gone = leave[at];
                if (w[0].users <= gone && keeper[at] == key_of(0)) {
                    if (w[0].users < gone) atomicAdd(p.users + page, gone - w[0].users);        // (fewer than name it: it is the one now)
                    w[0].last = -1;
                } else
                    atomicSub(p.users + page, 1);
            }
            __syncthreads();                                   // (the list of free pages is in the same place)
        }
    } else if (some) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (w[r].last >= 0) atomicSub(p.users + w[r].last, 1);
        __syncthreads();
        // (read from the caches' common level: other wavefronts' atomics are there)
        auto users_of = [&](int r) { return __hip_atomic_load(p.users + w[r].last, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (w[r].last >= 0 && users_of(r) <= 0) atomicMin(p.users + w[r].last, key_of(r));
        __syncthreads();
        uint32_t keeps = 0;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (w[r].last >= 0 && users_of(r) == key_of(r)) keeps |= 1u << r;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (keeps >> r & 1) {
                atomicExch(p.users + w[r].last, 1);
                w[r].last = -1;
            }
        __syncthreads();
    }
    // what each needs, and what all before it need.  (Of ALL's tables sums stay below 2^31.)
    using sum_t = std::conditional_t<ALL, int, int64_t>;
    sum_t* const sums = reinterpret_cast<sum_t*>(sums_);
    auto need_of = [&](int r) { return w[r].to > w[r].from ? pages_of(p, w[r].to) - pages_of(p, w[r].from) + (w[r].last >= 0) : 0; };
    sum_t mine = 0, total;
#pragma unroll
    for (int r = 0; r < R; ++r) mine += need_of(r);
    sum_t upto = prefix<sum_t>(mine, sums, &total);
    int32_t* const list = ALL && total > kList ? a.list : near;
    int64_t found = 0;
    if constexpr (ALL) {
        if (total > 0) {
#if defined(__HIP_DEVICE_COMPILE__)
            if (shorter) __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");              // (users have been changed by atomics, in the caches' common level)
#endif
            found = find_free(p, total, list, counts, users, !shorter);
            __syncthreads();
        }
    } else {
        if (total > 0) {
            // where each part's free pages begin among all
            const int parts = free_parts(p.num_pages);
            for (int base = 0; base < parts; base += kThreads) {
                const int i = base + tid;
                int all;
                const int before = prefix<int>(i < parts ? a.part_first[i] : 0, counts, &all);
                if (i < parts) a.part_first[i] = (int)found + before;
                found += all;
            }
        }
        __syncthreads();
    }
    // who is served
    int64_t tokens = 0;
    int first[R];
    uint32_t served = 0;
    bool more = false;                                         // than a thread writes down by itself, while others wait
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int need = need_of(r);
        first[r] = (int)min((int64_t)upto, (int64_t)INT_MAX);  // (past INT_MAX: not served)
        upto += need;
        if (need == 0 || upto <= found) {
            served |= 1u << r;
            tokens += max(0, w[r].to - w[r].from);
            more |= w[r].to - w[r].from > kFew;
        }
    }
    sum_t rows;
    int row;
    if constexpr (ALL) {
        more = __syncthreads_or(more);
        row = prefix<int>((int)tokens, sums, &rows);
    } else
        row = (int)prefix<int64_t>(tokens, sums, &rows);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int s = s0 + r;
        if (s >= S) continue;
        const bool is = served >> r & 1, copy = w[r].last >= 0 && is;
        const int to = is ? w[r].to : w[r].from;
        int target = -1;
        if (copy) {
            target = ALL ? list[first[r]] : free_page(a, first[r]);
            p.users[target] = 1;
            p.page_table[(int64_t)s * p.table_stride + page_number(p, w[r].from)] = target;
        } else if (w[r].last >= 0)
            atomicAdd(p.users + w[r].last, 1);                 // it stays
        a.copies[2 * (int64_t)s] = copy ? w[r].last : -1;
        a.copies[2 * (int64_t)s + 1] = target;
        if (a.granted) a.granted[s] = is && w[r].fits;
        const int after = row + max(0, to - w[r].from);
        if (a.indptr) {
            a.indptr[s] = row;
            if (s == S - 1) a.indptr[S] = after;
        }
        if (is && w[r].fits) p.length[s] = to;
        if constexpr (ALL) {
            if (!more) {
                // few tokens: at most one new page, and nothing that another thread has to know
                const int have = pages_of(p, w[0].from), fresh = pages_of(p, to) > have ? list[first[0] + copy] : -1;
                if (fresh >= 0) {
                    p.users[fresh] = 1;
                    p.page_table[(int64_t)s * p.table_stride + have] = fresh;
                }
                for (int i = row; i < min(after, a.num_tokens); ++i) {
                    const int position = w[0].from + i - row;
                    write_token(a, i, s, position, page_number(p, position) >= have ? fresh : copy ? target : w[0].page);
                }
            }
        }
        const page_grant g{w[r].from, to, first[r] | (copy ? INT_MIN : 0), row};
        if constexpr (ALL) grants[tid] = g;
        else a.grants[s] = g;
        row = after;
    }
    if constexpr (ALL) {
        if (!more) return;
        __syncthreads();
        // new entries: the sequence of each new page, by halves
        const int given = (int)(total < found ? total : found), widest = S > 1 ? 1 << (31 - __builtin_clz(S - 1)) : 0;
        for (int n = tid; n < given; n += kThreads) {
            int s = 0;                                         // the last sequence whose pages start at or before n
            for (int step = widest; step > 0; step >>= 1)
                if (s + step < S && (grants[s + step].first & INT_MAX) <= n) s += step;
            const page_grant g = grants[s];
            const int i = n - (g.first & INT_MAX) - (g.first < 0), e = pages_of(p, g.from) + i;
            if (i < 0 || g.to <= g.from || e >= pages_of(p, g.to)) continue;           // (a copy; pages that would not have been enough)
            p.page_table[(int64_t)s * p.table_stride + e] = list[n];
            p.users[list[n]] = 1;
        }
        __syncthreads();
        const int most = (int)(rows < a.num_tokens ? rows : a.num_tokens);
        if (!a.token_seq && !a.token_position && !a.token_slot) return;
        constexpr int TOGETHER = 4;
        for (int n0 = tid; n0 < most; n0 += TOGETHER * kThreads) {
            int s[TOGETHER], page[TOGETHER], position[TOGETHER];
#pragma unroll
            for (int k = 0; k < TOGETHER; ++k) s[k] = 0;
            for (int step = widest; step > 0; step >>= 1)
#pragma unroll
                for (int k = 0; k < TOGETHER; ++k) {           // (searches side by side)
                    const int next = s[k] + step;
                    if (next < S && grants[next].row <= n0 + k * kThreads) s[k] = next;
                }
#pragma unroll
            for (int k = 0; k < TOGETHER; ++k) position[k] = min(grants[s[k]].from + n0 + k * kThreads - grants[s[k]].row, p.max_length - 1);
#pragma unroll
            for (int k = 0; k < TOGETHER; ++k) page[k] = p.page_table[(int64_t)s[k] * p.table_stride + page_number(p, position[k])];
#pragma unroll
            for (int k = 0; k < TOGETHER; ++k)
                if (n0 + k * kThreads < most) write_token(a, n0 + k * kThreads, s[k], position[k], page[k]);
        }
    }
}

// No sequences: the end of their tokens
__global__ void pages_none_kernel(int32_t* indptr) { indptr[0] = 0; }

// Before the launch that decides: a wavefront a sequence and so many of its entries
__global__ __launch_bounds__(256) void pages_give_back_kernel(resize_args a, int chunks)
{
    const pages_args& p = a.p;
    const int id = blockIdx.x * 4 + (threadIdx.x >> 6), s = id / chunks, lane = threadIdx.x & 63;
    if (s >= p.num_seqs) return;
    const int wanted = a.wanted[s], from = length_at(p, s);
    if (wanted < 0 || wanted >= from) return;
    const int first = pages_of(p, wanted) + id % chunks * kChunk, end = min(pages_of(p, from), first + kChunk);
    for (int e = first + lane; e < end; e += 64) give_back(p, s, e);
}

// Then every sequence's wish, and of every part of the pool the free pages in order, to the part's place in the list, and how many there are
__global__ __launch_bounds__(256) void pages_look_kernel(resize_args a)
{
    __shared__ int sums[4];
    const pages_args& p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t id = (int64_t)blockIdx.x * 256 + tid;
    if (id < p.num_seqs) {
        wish w = wish_of(a, (int)id);
        look_at_page(p, (int)id, w);
        a.grants[id] = page_grant{w.from, w.to, w.last, w.fits};
    }
    const int64_t base = (int64_t)blockIdx.x * FREE_PART;
    if (base >= p.num_pages) return;
    constexpr int LOADS = FREE_PART / 1024;
    const int64_t mine = base + wave * (LOADS * 256) + 4 * lane;
    four u[LOADS];
    load_users<LOADS>(p, mine, u);
    int before[LOADS], count = 0;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        before[i] = count;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint64_t mask = __ballot(u[i].x[c] == 0);
            before[i] = lanes_before(mask, before[i]);
            count += __popcll(mask);
        }
    }
    if (lane == 0) sums[wave] = count;
    __syncthreads();
    int first = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        first += w < wave ? sums[w] : 0;
        all += sums[w];
    }
    int32_t* const list = a.list + base;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        int rank = first + before[i];
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (u[i].x[c] == 0) list[rank++] = (int32_t)(mine + 256 * i + c);
    }
    if (tid == 0) a.part_first[blockIdx.x] = all;
}

// Behind it: a wavefront a sequence and so many of its new entries and tokens.  A token's page is taken from where its entry comes from:
// another wavefront may not have written the entry yet.
__global__ __launch_bounds__(256) void pages_write_kernel(resize_args a, int chunks)
{
    const pages_args& p = a.p;
    const int id = blockIdx.x * 4 + (threadIdx.x >> 6), s = id / chunks, chunk = id % chunks, lane = threadIdx.x & 63;
    if (s >= p.num_seqs) return;
    const page_grant g = a.grants[s];
    if (g.to <= g.from) return;
    const int have = pages_of(p, g.from), want = pages_of(p, g.to), first = (g.first & INT_MAX) + (g.first < 0);
    int32_t* const table = p.page_table + (int64_t)s * p.table_stride;
    for (int e = have + chunk * kChunk + lane; e < min(want, have + (chunk + 1) * kChunk); e += 64) {
        const int page = free_page(a, first + e - have);
        table[e] = page;
        p.users[page] = 1;
    }
    const int begin = chunk * kChunk, end = min(min(g.to - g.from, begin + kChunk), a.num_tokens - g.row);
    if ((!a.token_seq && !a.token_position && !a.token_slot) || begin >= end) return;
    // the pages that these tokens are in, a lane one (1024 tokens lie in 33 at most)
    const int first_number = page_number(p, g.from + begin), mine = first_number + lane;
    const int held = mine >= want ? -1 : mine < have ? table[mine] : free_page(a, first + mine - have);
    for (int i = begin + lane; i < begin + (end - begin + 63) / 64 * 64; i += 64) {
        const int position = g.from + i, page = __shfl(held, page_number(p, position) - first_number, 64);
        if (i < end) write_token(a, g.row + i, s, position, page);
    }
}

// ---------------------------------------------------------------------------
// Sequences that become others'.  An entry of a new row is that of its parent's, or -1 behind it; users count what changes.  In one
// workgroup the new rows wait in registers until all old ones have been read, else in the workspace between two launches.
struct fork_entry {
    int now, before;           // page that the entry names and named, -1: none; now -2: it stays as it is
};

__device__ __forceinline__ fork_entry fork_of(const pages_args& p, const int32_t* parent, int s, int e)
{
    const int from = parent[s];
    if (from == s) return fork_entry{-2, -1};
    const bool there = from >= 0 && from < p.num_seqs && e < pages_of(p, length_at(p, from));
    fork_entry f;
    f.now = there ? p.page_table[(int64_t)from * p.table_stride + e] : -1;
    f.before = e < pages_of(p, length_at(p, s)) ? p.page_table[(int64_t)s * p.table_stride + e] : -1;
    if (f.now == -2) f.now = -1;
    return f;
}

__device__ __forceinline__ void write_fork(const pages_args& p, int s, int e, const fork_entry& f)
{
    if (f.now == -2) return;
    p.page_table[(int64_t)s * p.table_stride + e] = f.now;
    if (f.now == f.before) return;
    if (known(p, f.now)) atomicAdd(p.users + f.now, 1);
    if (known(p, f.before)) atomicSub(p.users + f.before, 1);
}

__device__ __forceinline__ int fork_length(const pages_args& p, const int32_t* parent, int s)
{
    const int from = parent[s];
    return from >= 0 && from < p.num_seqs ? length_at(p, from) : 0;
}

constexpr int kForkEntries = 4;                // of a thread, where one workgroup does

template <int E>
__global__ __launch_bounds__(kThreads) void pages_fork_kernel(pages_args p, const int32_t* parent)
{
    const int tid = threadIdx.x, entries = p.num_seqs * p.table_stride;
    fork_entry f[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int at = i * kThreads + tid;
        f[i] = at < entries ? fork_of(p, parent, at / p.table_stride, at % p.table_stride) : fork_entry{-2, -1};
    }
    const int length = tid < p.num_seqs ? fork_length(p, parent, tid) : 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int at = i * kThreads + tid;
        if (at < entries) write_fork(p, at / p.table_stride, at % p.table_stride, f[i]);
    }
    if (tid < p.num_seqs && parent[tid] != tid) p.length[tid] = length;
}

// the two launches; the workspace: new rows, new lengths, old lengths
__global__ __launch_bounds__(256) void pages_fork_read_kernel(pages_args p, const int32_t* parent, int32_t* space)
{
    const int64_t entries = (int64_t)p.num_seqs * p.table_stride, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at < entries) space[at] = fork_of(p, parent, (int)(at / p.table_stride), (int)(at % p.table_stride)).now;
    if (at < p.num_seqs) {
        space[entries + at] = fork_length(p, parent, (int)at);
        space[entries + p.num_seqs + at] = length_at(p, (int)at);
    }
}

__global__ __launch_bounds__(256) void pages_fork_write_kernel(pages_args p, const int32_t* parent, const int32_t* space)
{
    const int64_t entries = (int64_t)p.num_seqs * p.table_stride, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at < entries) {
        const int s = (int)(at / p.table_stride), e = (int)(at % p.table_stride);
        fork_entry f;
        f.now = space[at];
        f.before = e < pages_of(p, space[entries + p.num_seqs + s]) ? p.page_table[at] : -1;
        write_fork(p, s, e, f);
    }
    if (at < p.num_seqs && parent[at] != at) p.length[at] = space[entries + at];
}
}  // namespace

hipError_t launch_pages_resize(const resize_args& a, hipStream_t stream)
{
    const pages_args& p = a.p;
    static_assert(kThreads == 1024, "");                       // (one_workgroup_resizes)
    if (one_workgroup_resizes(p.num_seqs, p.table_stride, a.num_tokens)) {
        LORA_LAUNCH(LORA_K_PAGES_DECIDE, (pages_decide_kernel<1, true>), dim3(1), dim3(kThreads), 0, stream, a);
        return hipGetLastError();
    }
    const int entries = (int)entry_chunks(p.table_stride), looks = free_parts(p.num_pages) > (p.num_seqs + 255) / 256 ? free_parts(p.num_pages) : (p.num_seqs + 255) / 256;
    auto blocks = [&](int64_t chunks) { return dim3((uint32_t)((p.num_seqs * chunks + 3) / 4)); };
    LORA_LAUNCH(LORA_K_PAGES_GIVE_BACK, pages_give_back_kernel, blocks(entries), dim3(256), 0, stream, a, entries);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    LORA_LAUNCH(LORA_K_PAGES_LOOK, pages_look_kernel, dim3((uint32_t)looks), dim3(256), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.num_seqs <= kThreads) LORA_LAUNCH(LORA_K_PAGES_DECIDE, (pages_decide_kernel<1, false>), dim3(1), dim3(kThreads), 0, stream, a);
    else if (p.num_seqs <= 4 * kThreads) LORA_LAUNCH(LORA_K_PAGES_DECIDE, (pages_decide_kernel<4, false>), dim3(1), dim3(kThreads), 0, stream, a);
    else LORA_LAUNCH(LORA_K_PAGES_DECIDE, (pages_decide_kernel<16, false>), dim3(1), dim3(kThreads), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int chunks = (int)write_chunks(p.table_stride, p.max_length, a.num_tokens, a.token_seq || a.token_position || a.token_slot);
    LORA_LAUNCH(LORA_K_PAGES_WRITE, pages_write_kernel, blocks(chunks), dim3(256), 0, stream, a, chunks);
    return hipGetLastError();
}

hipError_t launch_pages_none(int32_t* indptr, hipStream_t stream)
{
    LORA_LAUNCH(LORA_K_PAGES_DECIDE, pages_none_kernel, dim3(1), dim3(1), 0, stream, indptr);
    return hipGetLastError();
}

hipError_t launch_pages_fork(const pages_args& p, const int32_t* parent, int32_t* workspace, hipStream_t stream)
{
    const int64_t entries = (int64_t)p.num_seqs * p.table_stride, most = entries > p.num_seqs ? entries : p.num_seqs;
    if (p.num_seqs <= kThreads && entries <= kForkEntries * kThreads) {
        if (entries <= kThreads) LORA_LAUNCH(LORA_K_PAGES_FORK, pages_fork_kernel<1>, dim3(1), dim3(kThreads), 0, stream, p, parent);
        else LORA_LAUNCH(LORA_K_PAGES_FORK, pages_fork_kernel<kForkEntries>, dim3(1), dim3(kThreads), 0, stream, p, parent);
        return hipGetLastError();
    }
    const dim3 grid((uint32_t)((most + 255) / 256));
    LORA_LAUNCH(LORA_K_PAGES_FORK, pages_fork_read_kernel, grid, dim3(256), 0, stream, p, parent, workspace);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    LORA_LAUNCH(LORA_K_PAGES_FORK, pages_fork_write_kernel, grid, dim3(256), 0, stream, p, parent, workspace);
    return hipGetLastError();
}
