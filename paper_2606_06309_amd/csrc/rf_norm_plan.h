// Host rules of the group norm's launches, which need no device.
#pragma once

#include "rf_internal.h"

namespace rf {

constexpr int kNormThreads = 256;

// A frame's rows are cut into `parts` runs of rows and its channels into `slices` of `cols` 16-byte
// columns, a workgroup each; a workgroup's threads cover `cols` columns and `lines` rows at a time.
struct NormPlan {
    int32_t vec;            // channels of a 16-byte column
    int32_t cols, slices, lines;
    int32_t parts;          // runs of a frame's rows
    int64_t per_part;       // rows of a run
    int32_t local;          // groups that a slice meets at most
    int64_t entries;        // partial sums: [M][parts][slices][local]
    int64_t ws_bytes;       // they, then mean and 1 / deviation of each group
};

inline NormPlan norm_plan(int32_t M, int64_t N, int32_t C, int32_t groups, int32_t together, int32_t dtype, int32_t cus) {
    NormPlan p{};
    auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    p.vec = dtype == RF_F32 ? 4 : 8;
    const int64_t columns = C / p.vec;
    p.slices = static_cast<int32_t>(up(columns, kNormThreads));
    p.cols = static_cast<int32_t>(up(columns, p.slices));
    p.slices = static_cast<int32_t>(up(columns, p.cols));
    p.lines = kNormThreads / p.cols;
    // eight workgroups to a compute unit, of eight rows a thread at least
    const int64_t want = up(8LL * cus, static_cast<int64_t>(M) * p.slices), most = up(N, 8LL * p.lines);
    const int64_t parts = want < most ? want : most;
    p.per_part = up(N, parts);
    p.parts = static_cast<int32_t>(up(N, p.per_part));
    const int64_t local = (static_cast<int64_t>(p.cols) * p.vec - 2) / (C / groups) + 2;
    p.local = static_cast<int32_t>(local < groups ? local : groups);
    p.entries = static_cast<int64_t>(M) * p.parts * p.slices * p.local;
    p.ws_bytes = (p.entries + static_cast<int64_t>(M / together) * groups) * 8;
    return p;
}

}  // namespace rf
