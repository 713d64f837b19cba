// Pages given out and taken back on the device, and sequences that become others' (include/lora_abi.h, PAGES).
//
// A call is a few thousand whole numbers, so it is bound by its chain of dependent trips to memory: wanted length -> table ->
// users of the page written next -> free pages -> table -> slots.  Where the tables are small, one workgroup does all of it with barriers between
// the steps; else pages are given back by one launch, one workgroup decides, and a third launch writes tables and slots down.
// What the atomics do (counts of users, the greatest of the keys of those that share a page) does not depend on their order.
#include <hip/hip_runtime.h>

#include <climits>

#include "device_util.h"
#include "kernels_sequences.h"
#include "launch.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kList = 8192;                    // free pages that are kept in LDS
constexpr int kChunk = 1024;                   // entries or tokens of a sequence that a wavefront writes down

// how many lanes before this one are in the mask, on top of n
__device__ __forceinline__ int lanes_before(uint64_t mask, int n)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, (uint32_t)n));
#else
    return n;
#endif
}

__device__ __forceinline__ int pages_of(const pages_args& p, int tokens) { return (int)(((int64_t)tokens + p.page_tokens - 1) / p.page_tokens); }
__device__ __forceinline__ int length_at(const pages_args& p, int s) { return min(max(p.length[s], 0), p.max_length); }
__device__ __forceinline__ bool known(const pages_args& p, int page) { return page >= 0 && page < p.num_pages; }

// exclusive prefix of a thread's number over the workgroup, and the sum
template <typename N>
__device__ __forceinline__ N prefix(N n, N* sums, N* total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    N upto = n;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const N below = __shfl_up(upto, off, 64);
        if (lane >= off) upto += below;
    }
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

// The first `most` free pages in order, by one workgroup: how many there are of them.  list[i] is written for i < that.
__device__ __forceinline__ int64_t find_free(const pages_args& p, int64_t most, int32_t* list, int* sums)
{
    struct __attribute__((packed, aligned(4))) four { int32_t x[4]; };
    constexpr int LOADS = 4, WAVE = LOADS * 256;               // pages of a wavefront at a time
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t found = 0;
    for (int64_t base = 0; base < p.num_pages && found < most; base += kWaves * WAVE) {
        const int64_t mine = base + wave * WAVE + 4 * lane;
        four u[LOADS];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int64_t at = mine + 256 * i;
            if (at + 4 <= p.num_pages) u[i] = *reinterpret_cast<const four*>(p.users + at);
            else
#pragma unroll
                for (int c = 0; c < 4; ++c) u[i].x[c] = at + c < p.num_pages ? p.users[at + c] : 1;
        }
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

// a new token's sequence, position and slot
__device__ __forceinline__ void write_token(const resize_args& a, int row, int s, int position)
{
    if (row >= a.num_tokens) return;
    if (a.token_seq) a.token_seq[row] = s;
    if (a.token_position) a.token_position[row] = position;
    if (a.token_slot) {
        const int number = position / a.p.page_tokens, page = a.p.page_table[(int64_t)s * a.p.table_stride + number];
        a.token_slot[row] = known(a.p, page) ? (int64_t)page * a.p.page_tokens + position - number * a.p.page_tokens : -1;
    }
}

// One workgroup decides: a thread R sequences, thread by thread in each thousand.  ALL: R is 1, and nothing is left to another launch.
template <int R, bool ALL>
__global__ __launch_bounds__(kThreads) void pages_decide_kernel(resize_args a)
{
    __shared__ int64_t sums[kWaves];
    __shared__ int counts[kWaves];
    __shared__ int32_t near[ALL ? kList : 1];
    __shared__ page_grant grants[ALL ? kThreads : 1];
    const pages_args& p = a.p;
    const int tid = threadIdx.x, S = p.num_seqs, P = p.page_tokens;
    int from[R], to[R], last[R];               // last: the page that holds the next token's place already, if it has other users
    bool fits[R];                              // the wanted length is one
    bool shorter = false;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int s = r * kThreads + tid;
        from[r] = to[r] = 0;
        fits[r] = false;
        last[r] = -1;
        if (s >= S) continue;
        const int wanted = a.wanted[s];
        from[r] = length_at(p, s);
        fits[r] = wanted >= 0 && wanted <= p.max_length;
        to[r] = fits[r] ? wanted : from[r];
        shorter |= to[r] < from[r];
    }
    if constexpr (ALL) {
        grants[tid] = page_grant{from[0], to[0], 0, 0};
        if (__syncthreads_or(shorter)) {
            const int entries = S * p.table_stride;
            for (int e = tid; e < entries; e += kThreads) {
                const int s = e / p.table_stride, i = e - s * p.table_stride;
                const page_grant g = grants[s];
                if (g.to < g.from && i >= pages_of(p, g.to) && i < pages_of(p, g.from)) give_back(p, s, i);
            }
            __syncthreads();
        }
    }
    // who shares the page that it would write
    bool some = false;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int s = r * kThreads + tid;
        if (to[r] <= from[r] || from[r] % P == 0) continue;
        const int page = p.page_table[(int64_t)s * p.table_stride + from[r] / P];
        if (known(p, page) && p.users[page] > 1) {
            last[r] = page;
            some = true;
        }
    }
    if (__syncthreads_or(some)) {
        // all of them leave it; where nobody stays, the one with the most tokens in it keeps it
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (last[r] >= 0) atomicSub(p.users + last[r], 1);
        __syncthreads();
        int key[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            key[r] = -1 - (from[r] % P * LORA_PAGES_MAX_SEQS + r * kThreads + tid);
            // (from the caches' common level: other wavefronts' atomics are there)
            if (last[r] >= 0 && __hip_atomic_load(p.users + last[r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) <= 0) atomicMin(p.users + last[r], key[r]);
        }
        __syncthreads();
        bool keeps[R];
#pragma unroll
        for (int r = 0; r < R; ++r) keeps[r] = last[r] >= 0 && __hip_atomic_load(p.users + last[r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == key[r];
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (keeps[r]) {
                atomicExch(p.users + last[r], 1);
                last[r] = -1;
            }
        __syncthreads();
    }
    // what each needs, and what all before it need
    int64_t upto[R], total = 0;
    int need[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        need[r] = to[r] > from[r] ? pages_of(p, to[r]) - pages_of(p, from[r]) + (last[r] >= 0) : 0;
        int64_t all;
        upto[r] = total + prefix<int64_t>(need[r], sums, &all) + need[r];
        total += all;
    }
    int32_t* const list = ALL && total <= kList ? near : a.list;
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");         // (users have been changed by atomics, in the caches' common level)
#endif
    const int64_t found = total > 0 ? find_free(p, total, list, counts) : 0;
    __syncthreads();
    // who is served
    int64_t rows = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int s = r * kThreads + tid;
        const bool served = need[r] == 0 || upto[r] <= found;
        if (!served) to[r] = from[r];
        int64_t all;
        const int64_t row = rows + prefix<int64_t>(max(0, to[r] - from[r]), sums, &all);
        rows += all;
        if (s >= S) continue;
        const int first = (int)min(upto[r] - need[r], (int64_t)INT_MAX);       // (past INT_MAX: not served)
        const bool copy = last[r] >= 0 && served;
        int target = -1;
        if (copy) {
            target = list[first];
            atomicExch(p.users + target, 1);
            p.page_table[(int64_t)s * p.table_stride + from[r] / P] = target;
        } else if (last[r] >= 0)
            atomicAdd(p.users + last[r], 1);   // it stays
        a.copies[2 * (int64_t)s] = copy ? last[r] : -1;
        a.copies[2 * (int64_t)s + 1] = target;
        if (a.granted) a.granted[s] = served && fits[r];
        if (a.indptr) {
            a.indptr[s] = (int32_t)row;
            if (s == S - 1) a.indptr[S] = (int32_t)row + max(0, to[r] - from[r]);
        }
        if (served && fits[r]) p.length[s] = to[r];
        const page_grant g{from[r], to[r], first | (copy ? INT_MIN : 0), (int32_t)row};
        if constexpr (ALL) grants[tid] = g;
        else a.grants[s] = g;
    }
    if constexpr (ALL) {
        __syncthreads();
        // new entries: the sequence of each new page, by halves
        const int given = (int)(total < found ? total : found);
        auto search = [&](int n, auto start) { // the last sequence that starts at or before n
            int lo = 0, hi = S;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                (start(mid) <= n ? lo : hi) = mid;
            }
            return lo;
        };
        for (int n = tid; n < given; n += kThreads) {
            const int s = search(n, [&](int i) { return grants[i].first & INT_MAX; });
            const page_grant g = grants[s];
            const int i = n - (g.first & INT_MAX) - (g.first < 0), e = pages_of(p, g.from) + i;
            if (i < 0 || g.to <= g.from || e >= pages_of(p, g.to)) continue;           // (a copy; pages that would not have been enough)
            p.page_table[(int64_t)s * p.table_stride + e] = list[n];
            atomicExch(p.users + list[n], 1);
        }
        __syncthreads();
        const int most = (int)(rows < a.num_tokens ? rows : a.num_tokens);
        if (a.token_seq || a.token_position || a.token_slot)
            for (int n = tid; n < most; n += kThreads) {
                const int s = search(n, [&](int i) { return grants[i].row; });
                write_token(a, n, s, grants[s].from + n - grants[s].row);
            }
    }
}

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

// Behind it: a wavefront a sequence and so many of its new entries and tokens.  A token's page is taken from where its entry comes from:
// another wavefront may not have written the entry yet.
__global__ __launch_bounds__(256) void pages_write_kernel(resize_args a, int chunks)
{
    const pages_args& p = a.p;
    const int id = blockIdx.x * 4 + (threadIdx.x >> 6), s = id / chunks, chunk = id % chunks, lane = threadIdx.x & 63;
    if (s >= p.num_seqs) return;
    const page_grant g = a.grants[s];
    if (g.to <= g.from) return;
    const int have = pages_of(p, g.from), want = pages_of(p, g.to), P = p.page_tokens;
    const int32_t* const list = a.list + (g.first & INT_MAX) + (g.first < 0);
    int32_t* const table = p.page_table + (int64_t)s * p.table_stride;
    for (int e = have + chunk * kChunk + lane; e < min(want, have + (chunk + 1) * kChunk); e += 64) {
        const int page = list[e - have];
        table[e] = page;
        p.users[page] = 1;
    }
    if (!a.token_seq && !a.token_position && !a.token_slot) return;
    const int end = min(g.to - g.from, (chunk + 1) * kChunk);
    for (int i = chunk * kChunk + lane; i < end; i += 64) {
        const int row = g.row + i, position = g.from + i, number = position / P;
        if (row >= a.num_tokens) break;
        if (a.token_seq) a.token_seq[row] = s;
        if (a.token_position) a.token_position[row] = position;
        if (a.token_slot) {
            const int page = number < have ? table[number] : list[number - have];
            a.token_slot[row] = known(p, page) ? (int64_t)page * P + position - number * P : -1;
        }
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

constexpr int kForkEntries = 32, kForkLengths = LORA_PAGES_MAX_SEQS / kThreads;

__global__ __launch_bounds__(kThreads) void pages_fork_kernel(pages_args p, const int32_t* parent)
{
    const int tid = threadIdx.x, entries = p.num_seqs * p.table_stride;
    fork_entry f[kForkEntries];
    int length[kForkLengths];
#pragma unroll
    for (int i = 0; i < kForkEntries; ++i) {
        f[i] = fork_entry{-2, -1};
        const int at = i * kThreads + tid;
        if (at < entries) f[i] = fork_of(p, parent, at / p.table_stride, at % p.table_stride);
    }
#pragma unroll
    for (int i = 0; i < kForkLengths; ++i) {
        const int s = i * kThreads + tid;
        length[i] = s < p.num_seqs ? fork_length(p, parent, s) : 0;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kForkEntries; ++i) {
        const int at = i * kThreads + tid;
        if (at < entries) write_fork(p, at / p.table_stride, at % p.table_stride, f[i]);
    }
#pragma unroll
    for (int i = 0; i < kForkLengths; ++i) {
        const int s = i * kThreads + tid;
        if (s < p.num_seqs && parent[s] != s) p.length[s] = length[i];
    }
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
    // One workgroup for all of it: 1024 sequences, and as many entries and tokens as it writes in the time of another launch
    if (p.num_seqs <= kThreads && (int64_t)p.num_seqs * p.table_stride <= 32 * kThreads && a.num_tokens <= 16 * kThreads) {
        LORA_LAUNCH(LORA_K_PAGES_DECIDE, (pages_decide_kernel<1, true>), dim3(1), dim3(kThreads), 0, stream, a);
        return hipGetLastError();
    }
    const int entries = (p.table_stride + kChunk - 1) / kChunk;
    auto blocks = [&](int64_t chunks) { return dim3((uint32_t)((p.num_seqs * chunks + 3) / 4)); };
    LORA_LAUNCH(LORA_K_PAGES_GIVE_BACK, pages_give_back_kernel, blocks(entries), dim3(256), 0, stream, a, entries);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.num_seqs <= kThreads) LORA_LAUNCH(LORA_K_PAGES_DECIDE, (pages_decide_kernel<1, false>), dim3(1), dim3(kThreads), 0, stream, a);
    else if (p.num_seqs <= 4 * kThreads) LORA_LAUNCH(LORA_K_PAGES_DECIDE, (pages_decide_kernel<4, false>), dim3(1), dim3(kThreads), 0, stream, a);
    else LORA_LAUNCH(LORA_K_PAGES_DECIDE, (pages_decide_kernel<16, false>), dim3(1), dim3(kThreads), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const bool tokens = a.token_seq || a.token_position || a.token_slot;
    const int rows = tokens ? (int)(((int64_t)(a.num_tokens < p.max_length ? a.num_tokens : p.max_length) + kChunk - 1) / kChunk) : 0, chunks = rows > entries ? rows : entries;
    LORA_LAUNCH(LORA_K_PAGES_WRITE, pages_write_kernel, blocks(chunks), dim3(256), 0, stream, a, chunks);
    return hipGetLastError();
}

hipError_t launch_pages_fork(const pages_args& p, const int32_t* parent, int32_t* workspace, hipStream_t stream)
{
    const int64_t entries = (int64_t)p.num_seqs * p.table_stride, most = entries > p.num_seqs ? entries : p.num_seqs;
    if (entries <= kForkEntries * kThreads) {
        LORA_LAUNCH(LORA_K_PAGES_FORK, pages_fork_kernel, dim3(1), dim3(kThreads), 0, stream, p, parent);
        return hipGetLastError();
    }
    const dim3 grid((uint32_t)((most + 255) / 256));
    LORA_LAUNCH(LORA_K_PAGES_FORK, pages_fork_read_kernel, grid, dim3(256), 0, stream, p, parent, workspace);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    LORA_LAUNCH(LORA_K_PAGES_FORK, pages_fork_write_kernel, grid, dim3(256), 0, stream, p, parent, workspace);
    return hipGetLastError();
}
