// Whether two arrays of rows share memory (csrc/msao_cache.h, rows_meet) against all pairs of
// rows. Used by tests/test_cache_limits_cpu.py.
#include <cstdio>
#include <cstdlib>
#include <random>

#include "msao_cache.h"

using namespace msao;

static bool meet(int64_t a, int64_t sa, int64_t b, int64_t sb, int64_t bytes, int64_t n)
{
    for (int64_t i = 0; i < n; ++i)
        for (int64_t j = 0; j < n; ++j)
            if (std::llabs((a + i * sa) - (b + j * sb)) < bytes) return true;
    return false;
}

int main()
{
    std::mt19937_64 rng(1);
    int bad = 0, both[2] = {0, 0};
    auto to = [](int64_t v) { return (const void*)(uintptr_t)v; };
    for (int i = 0; i < 300000; ++i) {
        const int64_t bytes = 16 * (1 + rng() % 5), n = rng() % 6, sa = bytes + 16 * (rng() % 8);
        const int64_t a = 4096 + 16 * (rng() % 60), b = 4096 + 16 * (rng() % 60);
        const bool want = meet(a, sa, b, sa, bytes, n);
        ++both[want];
        if (rows_meet(to(a), sa, to(b), sa, bytes, n) != want) ++bad;
        // at other distances: never where nothing is shared
        const int64_t sb = bytes + 16 * (rng() % 8);
        const bool got = rows_meet(to(a), sa, to(b), sb, bytes, n);
        if (got && !meet(a, sa, b, sb, bytes, n)) ++bad;
        if (n > 0 && std::llabs(a - b) < bytes && !got) ++bad;
    }
    // far apart and at the ends of the address space
    const int64_t far = (int64_t)1 << 46;
    if (rows_meet(to(16), 64, to(far), 64, 64, 1000) || rows_meet(to(far), 64, to(16), 64, 64, 1000)) ++bad;
    if (!rows_meet(to(16), 64, to(16 + 64 * ((int64_t)1 << 30)), 64, 64, ((int64_t)1 << 30) + 1)) ++bad;
    if (both[0] < 1000 || both[1] < 1000) ++bad;
    printf("%d wrong\n", bad);
    return bad ? 1 : 0;
}
