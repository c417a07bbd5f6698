// The tiles of a line (split_rule.h, attention over 8-bit pages of many sequences) are counted in 32 bits: no line where there can be more.  Exit code 0: all hold.
#include <cstdint>
#include <cstdio>

#include "split_rule.h"

using namespace chess;

int main()
{
    int lines = 0, rows = 0;
    for (int n_cu : {64, 256, 304})
        for (int heads : {1, 2, 8, 32})
            for (int group : {1, 4, 16})
                for (int tile_pages : {2, 4})
                    for (int batch : {2, 13, 52, 64, 200, 1000, 4096, 60000})
                        for (int64_t tiles : {33LL, 1000LL, 35791LL, 524287LL, 524288LL, 524289LL, 10737418LL, 33554431LL, 33554432LL, 1LL << 28}) {
                            const SplitLimits c{n_cu, 3 * n_cu, 256, heads, group, tile_pages, 0, 4};
                            const int64_t pages = tiles * tile_pages;
                            if (pages > INT32_MAX) continue;
                            const SplitShape s = choose_quant_splits(c, batch, pages, false);
                            const bool line = s.n_slots > 0 && s.waves == 4;
                            if (line && batch * tiles > INT32_MAX) {
                                std::printf("a line of %lld tiles: cu %d heads %d batch %d\n", (long long)(batch * tiles), n_cu, heads, batch);
                                return 1;
                            }
                            if (batch * tiles > INT32_MAX && s.n_slots == 0 && (s.n_splits != 1 || s.waves != 4)) { std::printf("not a workgroup a row\n"); return 1; }
                            lines += line;
                            rows += !line && batch * tiles > INT32_MAX;
                        }
    std::printf(lines > 0 && rows > 0 ? "ok\n" : "no such shape was tried\n");
    return 0;
}
