// Places of a verification's distributions, at the most rows that a chunk counts.
#include <cstdio>
#include <initializer_list>

#include "msao_sample.h"

using namespace msao;

int main()
{
    const int64_t most = INT32_MAX;
    for (int64_t rows : {(int64_t)1, (int64_t)7, ((int64_t)1 << 30) - 1, (int64_t)1 << 30, ((int64_t)1 << 30) + 1, most})
        for (int64_t r : {(int64_t)0, rows / 2, rows - 1})
            for (int which : {0, 1}) {
                const ChunkDev ch{nullptr, (int32_t)rows, 1};
                if (dist_at(ch, which, (int)r) == (which ? rows : 0) + r) continue;
                std::printf("rows %lld, row %lld, which %d: %lld\n", (long long)rows, (long long)r, which, (long long)dist_at(ch, which, (int)r));
                return 1;
            }
    std::puts("ok");
    return 0;
}
