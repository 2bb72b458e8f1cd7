// Launches of the join of an attention's parts, on the host: those of a call take each row once, in whole workgroups of adjacent rows, with
// fewer than 2^32 threads.  Prints the first violation and returns 1.
#include "ska_cache_plan.h"

#include <algorithm>
#include <cstdio>

int main()
{
    long several = 0;
    for (int d : {32, 64, 128})
        for (int parts : {2, 3, 4, 7, 8, 9, 16, 100, 512}) {
            const CaJoin join(parts, d);
            if (join.slices > parts || join.per < 1 || join.per * join.slices * (d / 4) != CaJoin::THREADS) return std::printf("d = %d, %d parts: %d slices, %ld rows\n", d, parts, join.slices, join.per), 1;
            for (long rows : {1L, 31L, 1000L, (1L << 25) - 1, 1L << 25, (1L << 26) - 1, 1L << 26, (1L << 26) + 1, 1L << 27, (1L << 28) + 5, 1L << 29}) {
                long next = 0;
                int launches = 0;
                for (long first = 0; first < rows; first += join.most(), ++launches) {
                    const long n = std::min(rows - first, join.most()), threads = (n + join.per - 1) / join.per * CaJoin::THREADS;
                    // (a launch but the last ends with a whole workgroup, which takes no row of the next)
                    if (first != next || threads >= 1L << 32 || (first + n < rows && n % join.per)) return std::printf("d = %d, %d parts, %ld rows: %ld threads at row %ld\n", d, parts, rows, threads, first), 1;
                    next = first + n;
                }
                if (next != rows) return std::printf("d = %d, %d parts: %ld of %ld rows\n", d, parts, next, rows), 1;
                several += launches > 1;
            }
        }
    std::printf("%ld calls of several launches\n", several);
    return several > 0 ? 0 : 1;
}
