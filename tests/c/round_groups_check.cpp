// Which workgroups of attention with shared prefixes write the parts of which rows, by the indexing that the
// kernels share with the host: no two groups write those of one row, whatever the groups' array holds, and what
// a sequence takes from its group is written for all its rows. Prints the first difference.
#include <cstdio>
#include <vector>

#include "msao_cache.h"

using namespace msao;

static unsigned long long state = 54321;
static int rnd(int n)
{
    state = state * 6364136223846793005ull + 1442695040888963407ull;
    return (int)((state >> 33) % (unsigned)n);
}

#define CHECK(x)                                                            \
    do {                                                                    \
        if (!(x)) {                                                         \
            std::printf("line %d: %s; groups", __LINE__, #x);               \
            for (int g : group) std::printf(" %d", g);                      \
            std::printf("\n");                                              \
            return 1;                                                       \
        }                                                                   \
    } while (0)

int main()
{
    long shared_rows = 0, shared_lists = 0;
    for (int trial = 0; trial < 60000; ++trial) {
        const int seqs = 1 + rnd(9), groups = 1 + rnd(5), kind = rnd(3), rows = 64;
        std::vector<int> start(seqs + 1), group(groups + 1), tokens(groups), lengths(seqs);
        for (int i = 0, at = 0; i <= seqs; ++i) start[i] = at += i ? rnd(4) : 0;
        for (int i = 0, at = rnd(4) - 2; i <= groups; ++i) group[i] = kind ? rnd(seqs + 4) - 2 : (at += rnd(4));
        if (trial == 0) group = {0, 6, 2, 8, 1, 8}, tokens.resize(5);
        for (int& t : tokens) t = 16 * rnd(8);
        for (int& n : lengths) n = 40 + rnd(200);
        const ChunkDev ch{start.data(), rows, 1 + rnd(4)};
        PrefixDev pre{};
        pre.group = group.data();
        pre.tokens = tokens.data();
        pre.length = lengths.data();
        pre.n_groups = (int)tokens.size();
        pre.n_seqs = seqs;
        pre.max_tokens = 128;
        pre.max_rows = rnd(40);
        const int cap = 256;
        // (a wavefront's lanes each look at some of the list)
        bool ascend = true, by_lanes = true;
        for (int g = 0; g < pre.n_groups; ++g) ascend = ascend && group[g] <= group[g + 1];
        for (int lane = 0; lane < 64; ++lane) by_lanes = groups_ascend(pre, lane, 64) && by_lanes;
        CHECK(by_lanes == ascend && groups_ascend(pre, 0, 1) == ascend);
        std::vector<int> owner(rows, -1);
        for (int g = 0; g < pre.n_groups; ++g) {
            const GroupRows gr = group_rows(pre, ch, g);
            if (!by_lanes || group_tokens(pre, cap, g) == 0) continue;
            for (int r = gr.begin; r < gr.begin + (gr.n < pre.max_rows ? gr.n : pre.max_rows); ++r) {
                CHECK(owner[r] < 0);
                owner[r] = g;
                ++shared_rows;
            }
        }
        shared_lists += by_lanes;
        for (int s = 0; s < seqs; ++s) {
            int g = -1;  // the last one that begins at s or before it
            for (int i = 0; i < pre.n_groups; ++i) g += group[i] <= s;
            const Rows own = seq_rows(ch, s);
            if (!by_lanes || prefix_of(pre, ch, cap, s, g, own, lengths[s], true) == 0) continue;
            for (int i = 0; i < (own.n < ch.max_new ? own.n : ch.max_new); ++i) CHECK(owner[own.begin + i] == g);
        }
    }
    if (shared_rows < 10000 || shared_lists < 10000) return std::puts("few cases share"), 1;
    std::puts("ok");
    return 0;
}
