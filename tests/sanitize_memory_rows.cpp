// Whether rows in memory have bytes in common (tests/test_attention_sanitizers.py), against a count of the bytes
#include <cstdio>
#include <cstdlib>
#include <random>

#include "../paper_2411_00915_amd/csrc/attention_internal.h"

int main()
{
    std::mt19937 rng(12);
    auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
    long found = 0, decided = 0;
    for (int round = 0; round < 400000; ++round) {
        const int wa = pick(1, 9), wb = pick(1, 9), pa = wa + (pick(0, 2) ? pick(0, 12) : 0), pb = pick(0, 2) ? std::max(pa, wb) : wb + pick(0, 12);
        const int na = pick(0, 6), nb = pick(0, 6), a0 = pick(100, 200), b0 = a0 + pick(-70, 70);
        bool bytes[400] = {}, common = false;
        for (int i = 0; i < na; ++i)
            for (int d = 0; d < wa; ++d) bytes[a0 + i * pa + d] = true;
        for (int i = 0; i < nb; ++i)
            for (int d = 0; d < wb; ++d) common |= bytes[b0 + i * pb + d];
        const memory_rows a(reinterpret_cast<const void*>((uintptr_t)a0), na, na == 1 ? 0 : pa, wa, 1), b(reinterpret_cast<const void*>((uintptr_t)b0), nb, pb, wb, 1);
        const bool looked_at = pa == pb || a.one_piece() || b.one_piece(), got = share_bytes(a, b);
        if (got != share_bytes(b, a) || (looked_at ? got != common : got && !common)) {
            std::fprintf(stderr, "%d x %d every %d from %d, %d x %d every %d from %d: %d\n", na, wa, pa, a0, nb, wb, pb, b0, got);
            return 1;
        }
        found += common;
        decided += looked_at;
    }
    const int64_t far = (int64_t)1 << 46;                  // addresses and pitches as large as there are
    const memory_rows q(reinterpret_cast<const void*>((uintptr_t)far), (int64_t)1 << 30, (int64_t)1 << 30, 4096, 4), o(reinterpret_cast<const void*>((uintptr_t)(far + 16384)), 1 << 20, (int64_t)1 << 30, 4096, 4);
    if (share_bytes(q, o) || !share_bytes(q, q)) return 1;
    std::printf("sanitize_memory_rows: ok (%ld of %ld share)\n", found, decided);
    return found < 50000;
}
