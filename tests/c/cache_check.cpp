// The paged cache's indexing (csrc/msao_cache.h) on the CPU: rows, lengths and pages
// of any arrays stay in bounds, and the parts of a row cover its tokens once each.
// Used by tests/test_cache_cpu.py.
#include <climits>
#include <cstdio>
#include <random>
#include <vector>

#include "msao_cache.h"

using namespace msao;

static int bad = 0;
#define CHECK(x) do { if (!(x)) { if (++bad < 10) printf("FAIL line %d: %s\n", __LINE__, #x); } } while (0)

int main()
{
    std::mt19937_64 rng(1);
    // parts
    for (int per : {32, 128, 256, 1024, 1 << 29})
        for (int seen : {-5, 0, 1, 31, 32, 33, 127, 128, 129, 300, 4097, 131072, 1 << 29}) {
            const int n = parts_of(seen, per);
            if (seen <= 0) {
                CHECK(n == 0);
                continue;
            }
            CHECK((int64_t)n * per >= seen && (int64_t)(n - 1) * per < seen);
        }
    // quotients by multiplication
    for (int n : {1, 2, 3, 5, 6, 7, 8, 12, 14, 28, 48, 71, 255, 256, 257, 65535, 65537, (1 << 30) - 1, (1 << 30) + 1, INT_MAX - 1, INT_MAX}) {
        const Group g = make_group(n);
        for (int64_t k = 0; k < 3000; ++k)
            for (int64_t r : {k, INT_MAX - k, k * n, k * n - 1, INT_MAX / n * (int64_t)n - k, (int64_t)(rng() & INT_MAX)})
                if (r >= 0 && r <= INT_MAX) CHECK(g.of((int)r) == (int)r / n);
    }
    // what the last row of a group sees
    for (int i = 0; i < 100000; ++i) {
        const int length = (int)(rng() % 300), n = (int)(rng() % 300), group = 1 + (int)(rng() % 8);
        if (n == 0) continue;
        const int row = (int)(rng() % (uint64_t)(n * group));
        const int s = group_sees(length, n, make_group(group), row, true);
        CHECK(s >= 0 && s <= length);
        int count = 0;
        for (int j = 0; j < length; ++j) count += j <= length - n + row / group;
        CHECK(s == count);
        CHECK(group_sees(length, n, make_group(group), row, false) == length);
    }
    // arrays of anything
    const int strange[] = {INT_MIN, INT_MIN + 1, -17, -1, 0, 1, 5, 31, 32, 33, 1000, INT_MAX - 1, INT_MAX};
    for (int i = 0; i < 200000; ++i) {
        CacheDev c{};
        c.page_shift = 4 + (int)(rng() % 4);
        c.per_seq = (int)(rng() % 4);
        c.n_pages = (int)(rng() % 40);
        c.n_seqs = 3;
        c.table_stride = c.per_seq + (int)(rng() % 3);
        std::vector<int32_t> pages((size_t)(3 * c.table_stride) + 1), length(3), start(4);
        for (auto& p : pages) p = strange[rng() % 13];
        for (auto& l : length) l = strange[rng() % 13];
        for (auto& s : start) s = strange[rng() % 13];
        c.pages = pages.data();
        c.length = length.data();
        ChunkDev ch{start.data(), (int)(rng() % 50), 3};
        for (int s = 0; s < 3; ++s) {
            const int L = seq_length(c, s);
            CHECK(L >= 0 && L <= capacity(c));
            const Rows r = seq_rows(ch, s);
            CHECK(r.begin >= 0 && r.n >= 0 && (int64_t)r.begin + r.n <= ch.n_rows);
            if (start[s] >= 0 && start[s + 1] >= start[s] && start[s + 1] <= ch.n_rows)
                CHECK(r.begin == start[s] && r.n == start[s + 1] - start[s]);
            for (int col = 0; col < c.per_seq; ++col) {
                const int p = page_at(c, s, col), named = pages[(size_t)(s * c.table_stride + col)];
                CHECK(p >= -1 && p < c.n_pages);
                CHECK(named >= 0 && named < c.n_pages ? p == named : p == -1);
            }
        }
    }
    printf(bad ? "%d checks failed\n" : "all indexes as expected\n", bad);
    return bad ? 1 : 0;
}
