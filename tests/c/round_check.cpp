// Indexing that the kernels of a speculative round share with the host, against plain loops:
// which item an offset falls into, columns of lengths, which tokens a sequence has from its
// group (arrays out of order and out of range among them). Prints the first difference.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "msao_cache.h"

using namespace msao;

static unsigned long long state = 12345;
static int rnd(int n)
{
    state = state * 6364136223846793005ull + 1442695040888963407ull;
    return (int)((state >> 33) % (unsigned)n);
}

#define CHECK(x)                                                \
    do {                                                        \
        if (!(x)) {                                             \
            std::printf("line %d: %s\n", __LINE__, #x);         \
            return 1;                                           \
        }                                                       \
    } while (0)

int main()
{
    for (int trial = 0; trial < 2000; ++trial) {
        const int n = 1 + rnd(40);
        std::vector<int> extent(n), offset(n);
        int total = 0;
        for (int i = 0; i < n; ++i) {
            extent[i] = rnd(3) ? 0 : rnd(5);
            offset[i] = total;
            total += extent[i];
        }
        for (int i = 0, at = 0; i < n; ++i)
            for (int e = 0; e < extent[i]; ++e, ++at)
                CHECK(item_of(n, at, [&](int q) { return offset[q]; }) == i);
    }
    ResizeArgs r{};
    for (r.page_shift = 4; r.page_shift <= 16; ++r.page_shift)
        for (int n : {0, 1, 15, 16, 17, 65535, 65536, 65537, 1 << 29})
            for (int held : {0, 1, 5, 1 << 25}) {
                const long long page = 1ll << r.page_shift, c = (n + page - 1) / page;
                CHECK(columns_of(r, n, held) == (c > held ? c : held));
            }
    for (int trial = 0; trial < 20000; ++trial) {
        const int seqs = 1 + rnd(9), groups = 1 + rnd(4), rows = rnd(30), wild = rnd(3) == 0;
        std::vector<int> start(seqs + 1), group(groups + 1), tokens(groups), lengths(seqs);
        for (int i = 0, at = 0; i <= seqs; ++i) start[i] = wild ? rnd(60) - 15 : (at += i ? rnd(4) : 0);
        for (int i = 0, at = 0; i <= groups; ++i) group[i] = wild ? rnd(20) - 5 : (at += rnd(4));
        for (int& t : tokens) t = rnd(300) - 20;
        for (int& n : lengths) n = rnd(500) - 20;
        const ChunkDev ch{start.data(), rows, rnd(6)};
        PrefixDev pre{};
        pre.group = group.data();
        pre.tokens = tokens.data();
        pre.length = lengths.data();
        pre.n_groups = groups;
        pre.n_seqs = seqs;
        pre.max_tokens = rnd(300);
        pre.max_rows = rnd(40);
        const int cap = 16 * rnd(30);
        for (int g = 0; g < groups; ++g) {
            const GroupRows gr = group_rows(pre, ch, g);
            CHECK(0 <= gr.first && gr.first <= gr.end && gr.end <= seqs && 0 <= gr.begin && gr.n >= 0 && gr.begin + gr.n <= rows);
            const int t = group_tokens(pre, cap, g);
            CHECK(t >= 0 && t % 16 == 0 && t <= cap && t <= pre.max_tokens && (t == 0 || (t <= tokens[g] && tokens[g] < t + 16)));
            CHECK(t == 0 || (gr.first < seqs && t <= lengths[gr.first]));
        }
        for (int s = 0; s < seqs; ++s)
            for (int g = -1; g <= groups; ++g) {
                const Rows own = seq_rows(ch, s);
                const int length = rnd(cap + 1), causal = rnd(2);
                const int t = prefix_of(pre, ch, cap, s, g, own, length, causal);
                if (t == 0) continue;
                // every row that the call computes is one of the rows that the prefix is computed for, and sees all of it
                const GroupRows gr = group_rows(pre, ch, g);
                const int n = own.n < ch.max_new ? own.n : ch.max_new, done = gr.n < pre.max_rows ? gr.n : pre.max_rows;
                CHECK(g >= 0 && g < groups && s >= gr.first && s < gr.end && t == group_tokens(pre, cap, g));
                for (int i = 0; i < n; ++i) {
                    CHECK(own.begin + i >= gr.begin && own.begin + i < gr.begin + done);
                    CHECK(t - 1 <= (causal ? length - own.n + i : length - 1));
                }
            }
    }
    std::puts("ok");
    return 0;
}
