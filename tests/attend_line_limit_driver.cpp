// Attention of few new tokens a sequence lays a batch's tiles in a line that is counted in 32 bits: no such line where there can be more, shares rounded up
// included.  The line is dealt as the kernel deals it, in 64 bits.  Exit code 0: all hold.
#include <cstdint>
#include <cstdio>

#include "split_rule.h"

using namespace chess;

int main()
{
    int64_t lines = 0, others = 0, longest = 0;
    for (int64_t slots : {1, 8, 32, 128, 256, 304})
        for (int64_t batch : {1, 2, 13, 31, 32, 33, 64, 200, 1000, 4095, 4096})
            for (int64_t tiles : {0LL, 1LL, 33LL, 1000LL, 35791LL, 524272LL, 524287LL, 524288LL, 524289LL, 10737418LL, 33554431LL, 33554432LL, 67108863LL})
                for (int64_t rows : {1, 5, 64, 65}) {
                    if (!few_rows(rows, batch, tiles, slots)) {
                        // only for a reason: many rows, or a line that comes close to 32 bits
                        if (rows <= 64 && batch * tiles < INT32_MAX - 16 * slots - batch) { std::printf("no line: slots %lld batch %lld tiles %lld\n", (long long)slots, (long long)batch, (long long)tiles); return 1; }
                        others += rows <= 64;
                        continue;
                    }
                    if (rows > 64) { std::printf("%lld rows are few\n", (long long)rows); return 1; }
                    const int64_t each = tiles > 1 ? tiles : 1, total = batch * each;      // (a sequence has one at least)
                    int64_t share = (total + slots - 1) / slots;
                    if (share < 4) share = 4;
                    int64_t end = slots * share;
                    if (batch <= slots && batch <= 64)
                        for (int64_t more = 0; more <= 12; more += 4) {
                            const int64_t shares = batch * ((each + share + more - 1) / (share + more));
                            const int64_t past = each + share + more - 1;
                            if (past > UINT32_MAX) { std::printf("shares of a sequence\n"); return 1; }
                            if (shares <= slots) {
                                end = slots * (share + more);
                                break;
                            }
                        }
                    if (total > INT32_MAX || end > INT32_MAX) { std::printf("a line of %lld, shares to %lld: slots %lld batch %lld tiles %lld\n", (long long)total, (long long)end, (long long)slots, (long long)batch, (long long)tiles); return 1; }
                    if (total > longest) longest = total;
                    ++lines;
                }
    std::printf(lines > 0 && others > 0 && longest > (1LL << 30) ? "ok\n" : "no such shape was tried\n");
    return 0;
}
