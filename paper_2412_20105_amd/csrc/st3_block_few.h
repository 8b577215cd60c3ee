// Where a workgroup's LDS holds what in the attention of few new tokens: one layout for the kernel and for the launcher that sizes it.
#pragma once

#include <cstddef>

#include "st3.h"

namespace st3 {

// Offsets in floats.  From 0 on the waves' blocks of keys, and where those were their outputs [waves][cols][D + 4]; behind them the waves' maxima and sums
// [2][waves][cols], a row's maximum and one over its sum [cols][2], and the logits [cols][stage], which are written and read 16 bytes at a time (stage: a
// multiple of 4): they begin at a multiple of 4, whatever `cols` is.
template <int D>
struct FewLds {
    int maxima, sums, heads, staged;
    constexpr FewLds(int waves, int cols)
        : maxima(waves * (ST3_BLOCK_TOKENS * D / 4 > cols * (D + 4) ? ST3_BLOCK_TOKENS * D / 4 : cols * (D + 4))),
          sums(maxima + waves * cols), heads(sums + waves * cols), staged((heads + 2 * cols + 3) / 4 * 4) {}
    constexpr size_t bytes(int cols, long long stage) const { return sizeof(float) * ((size_t)staged + (size_t)cols * (size_t)stage); }
};

}  // namespace st3
