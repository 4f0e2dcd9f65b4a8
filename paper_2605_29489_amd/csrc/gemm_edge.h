// Which K tiles of a product are read in whole chunks, without a look at the
// operand's end.  Plain C++: host code alone asks, once a launch.
#pragma once

#include <cstdint>

namespace mp {

// K tiles of bk rows, from the first on, whose chunks of v elements all lie
// inside an operand of P rows of `cols` elements, ld apart.  A row's last chunk
// passes its columns by up to v - 1 elements, which belong to the rows behind
// it, and the last K tile has none behind it.  Nor are its rows enough for the
// tile before it where they are few and short: the last of 64 rows of one bf16
// reads 7 elements more, and one row behind it holds one.  ld >= cols, so that
// less than v rows can be concerned, fewer than a K tile has.
inline int64_t whole_k_tiles(int64_t P, int64_t cols, int64_t ld, int v, int bk)
{
    if (P == 0)
        return 0;
    const int64_t last = (P - 1) / bk, left = P - last * bk;  // the last K tile, its rows
    const int64_t past = (cols + v - 1) / v * v - cols;
    return last > 0 && past > left * ld ? last - 1 : last;
}

}  // namespace mp
