// What one launch holds, host only.
#pragma once

#include <stdint.h>

namespace som {

// A dimension of a grid counts its threads in 32 bits.
inline bool grid_holds(int64_t blocks, int64_t threads) {
    return blocks <= ((int64_t)UINT32_MAX) / threads;
}

// The most rows of `units` units that one launch takes, with `per` units, which need not be
// of one row, to a workgroup of `threads`; 1 at least.
inline int64_t rows_at_once(int64_t units, int64_t per, int64_t threads) {
    const int64_t rows = (int64_t)UINT32_MAX / threads * per / units;
    return rows > 1 ? rows : 1;
}

}  // namespace som
