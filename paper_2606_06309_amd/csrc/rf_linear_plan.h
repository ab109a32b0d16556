// Host rules of the frame matrix product's launch, which need no device, and the sizes that the
// kernels share with them.
#pragma once

#include <math.h>

#include "rf_internal.h"

namespace rf {

// Bytes of a row that a step takes; rows of the largest tile; waves of a workgroup where rows are few.
constexpr int kLinearStep = 128;
constexpr int64_t kLinearTileRows = 256;
constexpr int kLinearFewWaves = 8;

// Rows of x that lie between two rows of one tile besides those that the product has there: where
// rows are read at full positions, those of the frames that are not listed. Frames j < i of the list
// meet in a tile when the last row of one and the first of the other do (each tile of every form lies
// in one of the largest), so neighbours may unless it divides their rows.
inline int64_t linear_gap(const RowFrames &f, int32_t M, int64_t N) {
    int64_t widest = 0;
    for (int32_t i = 1, j = 0; i < M; ++i) {
        while (((j + 1) * N - 1) / kLinearTileRows < i * N / kLinearTileRows) ++j;   // (ends at j = i)
        const int64_t gap = (f.in(i) - f.in(j) - (i - j)) * N;
        widest = gap > widest ? gap : widest;
    }
    return widest;
}

// Rows of x in one tile may lie 2 GB apart: their offsets from the tile's first row then do not fit
// the 31 bits of a buffer resource's range, and only the 128 x 128 form has 64-bit ones (two frames of
// 3,600 rows x 20,480 x 5,120 bf16, 2.8 GB apart: 1,840 us, where the same rows side by side take 1,480).
inline bool linear_far(const RowFrames &f, int32_t M, int64_t N, int64_t row_bytes) {
    return static_cast<double>(linear_gap(f, M, N) + kLinearTileRows + 1) * static_cast<double>(row_bytes) >= 2147483647.0;
}

// The kernels' forms: up to 16, 32 or 64 rows straight to registers; up to 32 or 64 (bf16) rows of a
// large W, and tiles of 64 x 128, 128 x 128 or (bf16) 256 x 256 (rows x features), through LDS.
enum LinearForm { kFew16, kFew32, kFew64, kStream32, kStream64, kTile64, kTile128, kTile256, kLinearForms };
struct LinearPlan {
    LinearForm form;
    int64_t row_tiles, col_tiles;
    int32_t steps, per_part, parts;
};

// A launch of this many workgroups (a multiple of the XCDs, 64 at most, of them) has fewer than 2^32
// threads.
inline bool linear_fits(int64_t groups, int64_t threads) { return (groups + 63) * threads <= 0xffffffffLL; }

// Whether tiles of 128 x 128, the form that every product may take, can be launched.
inline bool linear_whole_fits(int64_t rows, int64_t n_out) {
    return linear_fits(((rows + 127) / 128) * ((n_out + 127) / 128), 256);
}

// far: rows of a tile may lie 2 GB apart (only the smaller tile's kernel takes them).
inline LinearPlan linear_plan(int64_t rows, int32_t K, int32_t n_out, int32_t dtype, int32_t cus, bool far, bool may_split) {
    LinearPlan p{};
    const int64_t bytes = static_cast<int64_t>(K) * (dtype == RF_F32 ? 4 : 2);
    auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    if (rows <= 64 && !far) {
        // Straight to registers, through LDS in tiles of 256 features, or (33 rows on) as
        // products of more rows: by the bytes of W from which the latter are faster. us of a
        // product, registers / LDS, bf16: 16 rows x 4,096 x 4,096 10.6 / 11.5, 8 x 5,120 x 5,120
        // 19.2 / 16.2, 16 x 20,480 x 5,120 73 / 41; 17 x 1,536 x 1,536 8.3 / 8.3, 17 x 1,536 x
        // 6,144 12.3 / 9.7; fp32: 16 x 4,096 x 4,096 18.5 / 18.8, 8 x 5,120 x 5,120 33 / 29, 17 x
        // 1,536 x 6,144 24.7 / 14.8. Registers / tiles of 64 x 128, bf16: 64 x 1,536 x 1,024 9.3 /
        // 10.0, 64 x 1,536 x 1,536 11.4 / 10.9; fp32: 64 x 1,024 x 1,536 11.1 / 14.4, 64 x 1,536 x
        // 1,536 - / 15.7. LDS, 256 features / tiles of 64 x 128, 64 rows: 1,536 x 1,536 13.2 / 10.9,
        // 4,096 x 4,096 18.5 / 16.2, 10,240 x 5,120 36 / 29, 20,480 x 5,120 61 / 73; 24 rows: 1,536 x
        // 6,144 12.5 / 12.0, in fp32 17 / 21.
        const double w_mb = static_cast<double>(n_out) * static_cast<double>(bytes) * 1e-6;
        const bool few = w_mb < (dtype == RF_F32 ? 2 : 1) * (rows <= 16 ? 40 : rows <= 32 ? 8 : 4);
        const bool stream = !few && (rows <= 32 || (dtype == RF_BF16 && w_mb >= 150));
        if (stream) {
            p.form = rows <= 32 ? kStream32 : kStream64;
            p.row_tiles = 1;
            p.col_tiles = up(n_out, 256);
            p.steps = static_cast<int32_t>(up(bytes, kLinearStep));
            // two workgroups to a compute unit, of six steps at least
            const int64_t want = 2 * cus / p.col_tiles, most = p.steps / 6;
            p.parts = static_cast<int32_t>(!may_split ? 1 : want < most ? want : most);
            if (p.parts < 1) p.parts = 1;
            p.per_part = static_cast<int32_t>(up(p.steps, p.parts));
            p.parts = static_cast<int32_t>(up(p.steps, p.per_part));
            return p;
        }
        if (few) {
            p.form = rows <= 16 ? kFew16 : rows <= 32 ? kFew32 : kFew64;
            p.row_tiles = 1;
            p.col_tiles = up(n_out, rows > 16 && rows <= 32 ? 32 : 16);
            p.steps = static_cast<int32_t>(up(bytes, 64));
            // a wave takes four pieces at least; two workgroups to a compute unit
            const int64_t want = up(2 * cus, p.col_tiles), most = up(p.steps, 4 * kLinearFewWaves);
            p.parts = static_cast<int32_t>(!may_split || p.col_tiles >= cus ? 1 : want < most ? want : most);
            p.per_part = static_cast<int32_t>(up(up(p.steps, p.parts), 4) * 4);
            p.parts = static_cast<int32_t>(up(p.steps, p.per_part));
            return p;
        }
    }
    // Tiles of 64 x 128, 128 x 128 or in bf16 256 x 256 (rows x features) and parts of the reduction,
    // by the time in us that they come to, counted in rounds of the device: a round has a
    // fixed part and its steps, which take the longer the more workgroups share a compute
    // unit; a split adds the second kernel and its parts, written and read again. The
    // counts are fitted to products of 70 to 21,600 rows, 8 to 20,480 inputs and 256 to
    // 6,144 features, whose weights come from beyond the L2s, as from one layer to the
    // next: a workgroup alone on a compute unit then takes 0.53 us for a step of the
    // smallest tile where it takes 0.38 with the weights at hand. (Unsplit / split so: 512 x
    // 1,536 x 1,536 18.6 / 16.0, 1,000 x 6,144 x 1,536 58 / 35, 2,000 x 6,144 x 1,536 72 / 54;
    // fp32 1,500 x 4,096 x 320 84 / 53.) us, 64 x 128 / 128 x 128 / 256 x 256 (* split), bf16, weights
    // at hand: 512 x 1,536 x 1,536 11.6 / 17.5 / 41; 500 x 8,960 x 1,536 29.5* / 29.8* / 36*; 3,600 x 1,536 x 1,536 27 / 26 /
    // 41; 9,360 x 1,536 x 1,536 64 / 53 / 47; fp32: 512 x 1,536 x 1,536 31* / 41* / 74*; 7,800 x
    // 1,536 x 1,536 279 / 353 / 363; 9,360 x 1,536 x 6,144 - / 1,247 / 1,438 (the largest form is never
    // the best in fp32: two rounds of 128 x 128 take less than one of its rounds).
    struct Form {
        LinearForm form;
        int64_t rows, cols;
        int32_t most;        // workgroups to a compute unit
        double round;
        double step[3];      // with one, two, three workgroups to a compute unit
    };
    static const Form forms[2][3] = {{{kTile64, 64, 128, 3, 3.0, {0.53, 0.68, 1.0}},
                                      {kTile128, 128, 128, 2, 4.0, {0.80, 0.95, 0.95}},
                                      {kTile256, 256, 256, 1, 8.0, {1.55, 1.55, 1.55}}},
                                     {{kTile64, 64, 128, 3, 3.0, {1.1, 1.95, 2.93}},
                                      {kTile128, 128, 128, 2, 4.0, {2.4, 3.65, 3.65}}}};
    const int n_forms = dtype == RF_F32 ? 2 : 3;
    constexpr int64_t kLeastSteps = 4, kMostParts = 16;
    constexpr double kJoin = 3.0;
    const double join_mb = dtype == RF_F32 ? 0.6 : 0.45;
    p.steps = static_cast<int32_t>(up(bytes, kLinearStep));
    double best = 0.0;
    for (int i = 0; i < n_forms; ++i) {
        const Form &f = forms[dtype == RF_F32][i];
        if (far && f.form != kTile128) continue;
        const int64_t row_tiles = up(rows, f.rows), col_tiles = up(n_out, f.cols);
        for (int64_t parts = 1; parts <= kMostParts; ++parts) {
            if (parts > 1 && (!may_split || p.steps / parts < kLeastSteps)) break;
            const int64_t per = up(p.steps, parts), tiles = row_tiles * col_tiles * parts;
            if (parts > 1 && up(p.steps, per) != parts) continue;
            if (!linear_fits(tiles, f.form == kTile256 ? 512 : 256)) break;
            const int64_t share = up(tiles, cus) < f.most ? up(tiles, cus) : f.most;
            const double full = static_cast<double>(tiles) / static_cast<double>(cus * share);
            // (workgroups of the smallest tile follow each other closely enough to fill a broken round)
            const double rounds = f.form == kTile64 ? (full > 0.8 ? full + 0.2 : 1.0) : ceil(full);
            double t = rounds * (f.round + static_cast<double>(per) * f.step[share - 1]);
            if (parts > 1)
                t += kJoin + join_mb * 4e-6 * static_cast<double>(parts) * static_cast<double>(rows) * n_out;
            if (best == 0.0 || t < best) {
                best = t;
                p.form = f.form;
                p.row_tiles = row_tiles;
                p.col_tiles = col_tiles;
                p.parts = static_cast<int32_t>(parts);
                p.per_part = static_cast<int32_t>(per);
            }
        }
    }
    return p;
}

}  // namespace rf
