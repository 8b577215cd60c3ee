// The LDS of few new tokens: parts that follow each other without meeting, vectors of 16 bytes where they have to be.
#include <cstdio>
#include <initializer_list>

#include "st3_block_few.h"

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s (D %d, waves %d, columns %d)\n", __LINE__, #x, D, waves, cols); return 1; } } while (0)

template <int D>
static int check() {
    for (int waves : {4, 8, 12})
        for (int cols = 1; cols <= (waves == 12 ? 16 : 32); ++cols) {
            const st3::FewLds<D> at(waves, cols);
            CHECK(at.maxima >= waves * 64 * D / 4 && at.maxima >= waves * cols * (D + 4));      // blocks of 64 rows of codes; outputs
            CHECK(at.maxima % 4 == 0);
            CHECK(at.sums >= at.maxima + waves * cols && at.heads >= at.sums + waves * cols && at.heads % 2 == 0);      // (read as pairs)
            CHECK(at.staged >= at.heads + 2 * cols);
            CHECK(at.staged % 4 == 0);
            for (int stage : {0, 64, 1280}) CHECK(at.bytes(cols, stage) == 4u * (unsigned)(at.staged + cols * stage));
            CHECK(at.bytes(cols, 0) <= 160u << 10);
        }
    return 0;
}

int main() {
    if (check<64>() || check<128>()) return 1;
    std::printf("ok\n");
    return 0;
}
