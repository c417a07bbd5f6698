// The grids that a catch-up of the last pages is launched on (split_rule.h) against counting them.  Exit code 0: all hold.
#include <cstdint>
#include <cstdio>

#include "split_rule.h"

int main()
{
    for (int ppg : {1, 2, 3, 16, 64, 256})
        for (int pages : {1, 2, 15, 64, 65, 300, 1000}) {
            const int grids = (pages + ppg - 1) / ppg;
            for (int recent : {1, 2, 3, 16, 17, 63, 64, 65, 66, 299, 300, 1000, 1001, INT32_MAX - 256, INT32_MAX - 63, INT32_MAX - 1, INT32_MAX}) {
                int most = 0;                         // over all lengths: from the grid of the first recent page to the last page's
                for (int p = 1; p <= pages; ++p) {
                    const int first = p > recent ? p - recent : 0;
                    const int n = (p - 1) / ppg - first / ppg + 1;
                    if (n > most) most = n;
                }
                const int64_t got = chess::recent_grids(recent, ppg, grids);
                if (got < most || got > grids || got < 1 || (recent >= pages && got != grids)) {
                    std::printf("%d pages of a grid, %d pages, the last %d: %lld grids, %d are touched\n", ppg, pages, recent, (long long)got, most);
                    return 1;
                }
            }
        }
    std::printf("ok\n");
    return 0;
}
