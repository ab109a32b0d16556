// Host rules of the frame matrix product's launch, which need no device.
#pragma once

#include "rf_internal.h"

namespace rf {

// Rows of the largest tile.
constexpr int64_t kLinearTileRows = 256;

// Rows of x that lie between two rows of one tile besides those that the product has there: where
// rows are read at full positions, those of the frames that are not listed. Frames j < i of the list
// meet in a tile when the frames between them and a row of each fit into it, so neighbours always may.
inline int64_t linear_gap(const RowFrames &f, int32_t M, int64_t N) {
    int64_t widest = 0;
    for (int32_t i = 1, j = 0; i < M; ++i) {
        while ((i - j - 1) * N + 2 > kLinearTileRows) ++j;
        const int64_t gap = (f.in(i) - f.in(j) - (i - j)) * N;
        widest = gap > widest ? gap : widest;
    }
    return widest;
}

// Rows of x in one tile may lie 2 GB apart: their offsets from the tile's first row then do not fit
// the 31 bits of a buffer resource's range.
inline bool linear_far(const RowFrames &f, int32_t M, int64_t N, int64_t row_bytes) {
    return static_cast<double>(linear_gap(f, M, N) + kLinearTileRows + 1) * static_cast<double>(row_bytes) >= 2147483647.0;
}

}  // namespace rf
