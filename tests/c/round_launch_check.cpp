// Launches of the kernels with a workgroup a row: fewer than 2^32 threads each, every workgroup in one of them, in order.
#include <cstdio>
#include <initializer_list>

#include "msao_sample.h"

using namespace msao;

#define CHECK(x)                                                                       \
    do {                                                                               \
        if (!(x)) return std::printf("line %d: %s (%lld of %d)\n", __LINE__, #x, (long long)n, threads), 1; \
    } while (0)

int main()
{
    for (int threads : {64, kScanThreads, kRowThreads})
        for (int64_t n : {(int64_t)0, (int64_t)1, (int64_t)4194303, (int64_t)4194304, (int64_t)4194305, (int64_t)16777215, (int64_t)33554430,
                          (int64_t)1 << 26}) {
            int64_t next = 0;
            int launches = 0;
            CHECK(in_launches(n, threads, [&](int64_t first, int64_t some) {
                      if (first != next || some < 1 || some * threads >= (int64_t)1 << 32) return 7;
                      next += some;
                      ++launches;
                      return 0;
                  }) == 0);
            CHECK(next == n);
            CHECK(launches == 0 || (launches - 1) * ((((int64_t)1 << 32) - 1) / threads) < n);  // no more of them than it takes
            int calls = 0;
            CHECK(n == 0 || in_launches(n, threads, [&](int64_t, int64_t) { return ++calls, 5; }) == 5);
            CHECK(calls == (n ? 1 : 0));
        }
    std::puts("ok");
    return 0;
}
