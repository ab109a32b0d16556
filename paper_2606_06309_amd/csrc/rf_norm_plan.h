// Host rules of the group norm's launches, which need no device.
#pragma once

#include "rf_internal.h"

namespace rf {

constexpr int kNormThreads = 256;

// i / n for 0 <= i < 8192 and n <= 8192, given `share` = 1 / n: (i + 1/2) / n is 1 / (2 n) from a whole number at
// least, which is more than the product's rounding, (i + 1/2) / n * 2^-23.
__host__ __device__ inline int32_t divide(int32_t i, float share) {
    return static_cast<int32_t>((static_cast<float>(i) + 0.5f) * share);
}

// Rows of a thread in a chunk.
constexpr int kNormRows = 8;

// Rows of a part: every parts-th chunk of a frame, the last of which may be short. (Whole numbers below 2^24:
// frames have four parts to a compute unit, and no memory holds 2^34 rows.)
struct NormParts {
    int32_t more;           // parts with one whole chunk more than the others; the next has the last rows
    float each, chunk, last;
    __host__ __device__ float rows(int32_t part) const { return each + (part < more ? chunk : part == more ? last : 0.0f); }
};

// Two forms.
//  * slices: a workgroup has whole groups' columns of all rows that share their statistics, few
//    enough to stay in its LDS: one launch, x read once.
//  * parts: chunks of a frame's rows go to `parts` workgroups in turn, and its channels in `slices` of
//    `cols` 16-byte columns to workgroups of their own, for the statistics; a second launch goes over
//    x again.
// A workgroup's threads cover `cols` columns and `lines` rows at a time.
struct NormPlan {
    int32_t vec;            // channels of a 16-byte column
    int32_t block, hold;    // slices: threads of a workgroup, rows of a thread; parts: 0
    int32_t cols, slices, lines;
    int32_t parts;          // of a frame's rows
    NormParts runs;
    int32_t row_parts;      // those of the second launch
    int32_t local;          // groups that a slice meets at most
    int32_t x_past, y_past; // the second launch reads x, writes y past the caches
    int32_t few_parts;      // a group's parts are joined by the workgroups that use them
    int64_t sums;           // partial sums: [M][parts][slices][local]
    int64_t entries;        // of 8 bytes: they and, of fp32, their and the groups' means' rests (4 bytes each); an even number
    int64_t ws_bytes;       // these, then the groups' mean and 1 / deviation
};

// Where the workgroups of the second launch join the parts of the groups that they use, instead of a launch
// between: parts of a group and groups of a workgroup up to these (22.0 us for a norm of 11 parts into 8 bits and
// its product, 24.7 with the launch between; 19.4 with 65 parts, and 18.5; from 11 to 65 it was not measured where it
// turns), and workgroups to a compute unit: 20.4 us
// at 64 x 300 rows x 512 channels, five of them, 46.0 at 64 x 900 x 512, 14, where the launch between makes it 21.9
// and 47.2; 63.0 at 200 x 160 x 1,280, 31, and 61.3 with it. (Rows in 8 bits never have more than seven.)
constexpr int kNormFewParts = 16, kNormFewGroups = 64, kNormFewWorkgroups = 16;
// Workgroups of the second launch to a compute unit. They are short, as many as have four rows to a
// thread: 200 us for a norm of 409 MB, 203 with 16 to a compute unit, 211 with 8.
constexpr int64_t kRowRounds = 64;
// Bytes of y from which it goes past the caches: 66 us at 128 MB, 83 through them (157 and 152 with the product
// that reads it next), 200 and 240 at 409; smaller ones stay there for that product (75 and 72 us at 42 MB). The times at
// 128 MB are of two inputs in turn; where more take turns, 73 us for the 66.
constexpr double kNormCached = 96e6;
// Bytes of x from which the second launch reads it past the caches; smaller ones it finds there in part, going the
// other way than the first (which always leaves behind what it read): with a product of as many channels between,
// 10 x 3,120 x 640 takes 71.5 us a layer, 75 if both read past them, 21 x 1,560 x 1,536 into 8 bits and on, with
// residual, 163 and 181. 410 MB: 641 us a layer with the first only leaving x behind, 653 with both, 653 with neither.
constexpr double kNormHeld = 256e6;

// Workgroups of slices: threads, and rows of a thread that it holds at most (16 bytes each, in LDS with 32
// or 16 more bytes of a thread, of 160 KB); groups of a slice.
struct NormBlock {
    int32_t threads, hold;
};
constexpr NormBlock kNormBlocks[2] = {{512, 4}, {1024, 7}};
constexpr int kNormSliceGroups = 512;

// Whether `cols` columns of `rows` rows fit a workgroup; of the smallest that they do.
inline bool norm_slice(NormPlan *p, int64_t columns, int64_t cols, int64_t rows, int64_t per_group) {
    if (cols * p->vec / per_group > kNormSliceGroups) return false;
    for (const NormBlock &b : kNormBlocks) {
        const int64_t lines = b.threads / cols;
        if (lines < 1 || (rows + lines - 1) / lines > b.hold) continue;
        p->block = b.threads;
        p->cols = static_cast<int32_t>(cols);
        p->lines = static_cast<int32_t>(lines);
        p->hold = static_cast<int32_t>((rows + lines - 1) / lines);
        p->slices = static_cast<int32_t>(columns / cols);
        return true;
    }
    return false;
}

inline NormPlan norm_plan(int32_t M, int64_t N, int32_t C, int32_t groups, int32_t together, bool rows8, int32_t dtype,
                          int32_t cus) {
    NormPlan p{};
    auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    p.vec = dtype == RF_F32 ? 4 : 8;
    const int64_t columns = C / p.vec;
    if (!rows8) {
        // whole groups in whole columns: the least, and from there on rows of 64 bytes and no more
        // workgroups than a round. All of one round (two workgroups of 512 to a compute unit, one of
        // 1,024): 16 us at 6 x 700 rows x 1,280 channels, 192 of the latter, where parts take 19, but 46 and
        // 33 at 21 x 700 x 1,280, 24.5 and 22.5 at 33 x 400 x 640.
        int64_t unit = C / groups;
        while (unit % p.vec != 0) unit += C / groups;
        unit /= p.vec;
        const int64_t segments = M / together, rows = together * N;
        bool fits = norm_slice(&p, columns, unit, rows, C / groups);
        for (int64_t cols = unit + unit; fits && cols <= columns; cols += unit) {
            if (p.cols * 16 >= 64 && segments * p.slices <= 2LL * cus) break;
            if (columns % cols == 0 && !norm_slice(&p, columns, cols, rows, C / groups)) break;
        }
        if (fits && segments * p.slices <= static_cast<int64_t>(cus) * (p.block == kNormBlocks[0].threads ? 2 : 1)) return p;
        p.block = 0;
    }
    p.slices = static_cast<int32_t>(up(columns, kNormThreads));
    p.cols = static_cast<int32_t>(up(columns, p.slices));
    p.slices = static_cast<int32_t>(up(columns, p.cols));
    p.lines = kNormThreads / p.cols;
    // four workgroups to a compute unit, of eight rows a thread at least
    const int64_t want = up(4LL * cus, static_cast<int64_t>(M) * p.slices), most = up(N, kNormRows * p.lines);
    const int64_t parts = want < most ? want : most;
    p.parts = static_cast<int32_t>(parts < 65535 ? parts : 65535);
    const int64_t chunk = kNormRows * p.lines, whole = N / chunk;
    p.runs.more = static_cast<int32_t>(whole % p.parts);
    p.runs.each = static_cast<float>(whole / p.parts * chunk);
    p.runs.chunk = static_cast<float>(chunk);
    p.runs.last = static_cast<float>(N - whole * chunk);
    int64_t row_want = up(kRowRounds * cus, static_cast<int64_t>(M) * p.slices), row_most = up(N, 4 * p.lines);
    if (rows8) {
        // whole rows of 16, 64 or 256 threads, which have to fetch what they are normalised with first:
        // as many workgroups as a compute unit holds
        const int32_t eights = (C + (C <= 2048 ? 511 : 2047)) / (C <= 2048 ? 512 : 2048);   // of channels, a thread
        row_want = up((eights == 1 ? 6 : eights == 2 ? 4 : eights == 3 ? 3 : 2) * static_cast<int64_t>(cus), M);
        row_most = up(N, C <= 128 ? 16 : C <= 2048 ? 4 : 1);
    }
    const int64_t row_parts = row_want < row_most ? row_want : row_most;
    p.row_parts = static_cast<int32_t>(row_parts < 65535 ? row_parts : 65535);   // (an axis of a grid)
    const int64_t local = (static_cast<int64_t>(p.cols) * p.vec - 2) / (C / groups) + 2;
    p.local = static_cast<int32_t>(local < groups ? local : groups);
    const double bytes = static_cast<double>(M) * static_cast<double>(N) * C * (16 / p.vec);
    p.y_past = bytes > kNormCached;
    p.x_past = bytes > kNormHeld;
    p.few_parts = p.parts * together <= kNormFewParts && (rows8 ? groups : p.local) <= kNormFewGroups &&
                  (rows8 || static_cast<int64_t>(p.row_parts) * M * p.slices <= static_cast<int64_t>(kNormFewWorkgroups) * cus);
    const int64_t totals = static_cast<int64_t>(M / together) * groups;
    p.sums = static_cast<int64_t>(M) * p.parts * p.slices * p.local;
    p.entries = up(p.sums + (dtype == RF_F32 ? up(p.sums + totals, 2) : 0), 2) * 2;
    p.ws_bytes = (p.entries + totals) * 8;
    return p;
}

}  // namespace rf
