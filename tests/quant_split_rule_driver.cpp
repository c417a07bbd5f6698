// Runs the split rule of attention over 8-bit pages (split_rule.h) over the range of shapes.  Exit code 0: all hold.
#include <cstdio>

#include "split_rule.h"

using namespace chess;

int main()
{
    for (int n_cu : {1, 64, 256, 304})
        for (int blocks : {1, 2, 3, 8})
            for (int heads : {1, 2, 4, 8, 16, 300})
                for (int group : {1, 2, 4, 5, 7, 16})
                    for (int tile_pages : {2, 4})
                        for (int batch = 1; batch <= 1500; batch = batch < 20 ? batch + 1 : batch * 9 / 8)
                            for (int64_t pages = 1; pages <= 1 << 17; pages = pages < 24 ? pages + 1 : pages * 5 / 4)
                                for (bool listed : {false, true}) {
                                    const SplitLimits c{n_cu, blocks * n_cu, 256, heads, group, tile_pages, 0, 4};
                                    const SplitShape s = choose_quant_splits(c, batch, pages, listed);
                                    const int64_t pairs = (int64_t)batch * heads, tiles = cdiv(pages, tile_pages), ns = s.n_splits;
                                    // partial rows: of a line, a share may hold the end of a sequence and the beginning of another
                                    const int64_t used = s.n_slots == 0 ? pairs * ns : (int64_t)s.n_slots * heads + (s.waves == 4 ? pairs : 0);
                                    const char* bad = nullptr;
                                    if (ns < 1 || ns > 256 || ns * group > 1024) bad = "split count";
                                    else if ((ns > 1 || s.n_slots > 0) && used > partial_rows(n_cu, pairs)) bad = "partials outgrow the workspace";
                                    else if (s.waves != 4 && s.waves != 8) bad = "waves";
                                    else if (s.n_slots > 0 && (listed || batch < 2)) bad = "dealt slots";
                                    else if (s.n_slots > 0 && s.waves == 8 && (s.n_slots < batch || s.n_slots * heads > n_cu)) bad = "slots dealt by length";
                                    else if (s.n_slots > 0 && s.waves == 4 && s.n_slots * heads > blocks * n_cu) bad = "shares of a line";
                                    else if (!listed && batch == 1 && (s.waves != 8 || s.n_slots != 0 || ns > tiles || (ns > 1 && pairs * ns > n_cu))) bad = "one sequence";
                                    if (bad != nullptr) {
                                        std::printf("%s: cu %d blocks %d heads %d G %d tile pages %d batch %d pages %lld listed %d -> ns %d waves %d slots %d\n",
                                                    bad, n_cu, blocks, heads, group, tile_pages, batch, (long long)pages, listed, s.n_splits, s.waves, s.n_slots);
                                        return 1;
                                    }
                                }
    // a forced count of splits is what it says; every page takes eight waves then, a list four unless eight are asked for
    for (int waves : {1, 4, 8})
        for (bool listed : {false, true}) {
            const SplitLimits c{256, 768, 256, 8, 4, 2, 3, waves};
            const SplitShape s = choose_quant_splits(c, 4, 100, listed);
            if (s.n_splits != 3 || s.n_slots != 0 || s.waves != (!listed || waves == 8 ? 8 : 4)) { std::printf("forced shape\n"); return 1; }
        }
    std::printf("ok\n");
    return 0;
}
