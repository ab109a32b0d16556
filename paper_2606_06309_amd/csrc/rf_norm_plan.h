// Host rules of the group norm's launches, which need no device.
#pragma once

#include "rf_internal.h"

namespace rf {

constexpr int kNormThreads = 256;

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
    int32_t row_parts;      // those of the second launch
    int32_t local;          // groups that a slice meets at most
    int32_t stream;         // y is written past the caches
    int64_t entries;        // partial sums: [M][parts][slices][local], an even number
    int64_t ws_bytes;       // they, then what each frame's channels are normalised with, three numbers each
};

// Rows of a thread in a chunk.
constexpr int kNormRows = 8;
// Workgroups of the second launch to a compute unit. They are short, as many as have four rows to a
// thread: 130 us at 409 MB, 141 with 16 to a compute unit, 142 with 4.
constexpr int64_t kRowRounds = 64;
// Bytes of y from which it goes past the caches: 219 us at 409 MB, 246 through them; smaller ones
// stay there for the product that reads them.
constexpr double kNormCached = 96e6;
__host__ __device__ inline int64_t part_rows(int64_t N, int64_t chunk, int64_t parts, int64_t part) {
    const int64_t whole = N / chunk, turn = whole / parts, over = whole - turn * parts;
    return (turn + (part < over)) * chunk + (part == over ? N - whole * chunk : 0);
}

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
        // workgroups than four rounds
        int64_t unit = C / groups;
        while (unit % p.vec != 0) unit += C / groups;
        unit /= p.vec;
        const int64_t segments = M / together, rows = together * N;
        bool fits = norm_slice(&p, columns, unit, rows, C / groups);
        for (int64_t cols = unit + unit; fits && cols <= columns; cols += unit) {
            if (p.cols * 16 >= 64 && segments * p.slices <= 4LL * cus) break;
            if (columns % cols == 0 && !norm_slice(&p, columns, cols, rows, C / groups)) break;
        }
        if (fits) return p;
    }
    p.slices = static_cast<int32_t>(up(columns, kNormThreads));
    p.cols = static_cast<int32_t>(up(columns, p.slices));
    p.slices = static_cast<int32_t>(up(columns, p.cols));
    p.lines = kNormThreads / p.cols;
    // four workgroups to a compute unit, of eight rows a thread at least
    const int64_t want = up(4LL * cus, static_cast<int64_t>(M) * p.slices), most = up(N, kNormRows * p.lines);
    p.parts = static_cast<int32_t>(want < most ? want : most);
    int64_t row_want = up(kRowRounds * cus, static_cast<int64_t>(M) * p.slices), row_most = up(N, 4 * p.lines);
    if (rows8) {
        // whole rows of 16, 64 or 256 threads, which have to fetch what they are normalised with first:
        // as many workgroups as a compute unit holds
        const int32_t eights = (C + (C <= 2048 ? 511 : 2047)) / (C <= 2048 ? 512 : 2048);   // of channels, a thread
        row_want = up((eights == 1 ? 6 : eights == 2 ? 4 : eights == 3 ? 3 : 2) * static_cast<int64_t>(cus), M);
        row_most = up(N, C <= 128 ? 16 : C <= 2048 ? 4 : 1);
    }
    p.row_parts = static_cast<int32_t>(row_want < row_most ? row_want : row_most);
    const int64_t local = (static_cast<int64_t>(p.cols) * p.vec - 2) / (C / groups) + 2;
    p.local = static_cast<int32_t>(local < groups ? local : groups);
    p.stream = static_cast<double>(M) * static_cast<double>(N) * C * (16 / p.vec) > kNormCached;
    p.entries = (static_cast<int64_t>(M) * p.parts * p.slices * p.local + 1) / 2 * 2;
    p.ws_bytes = p.entries * 8 + static_cast<int64_t>(M) * C * 12;
    return p;
}

}  // namespace rf
