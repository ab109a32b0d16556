/* Host rules of the frame matrix product's launch against plain walks over rows. Prints "ok <checks>"; exits 1 at the
   first mismatch. */
#include <cmath>
#include <cstdio>
#include <random>
#include <vector>

#include "rf_linear_plan.h"

static int checks;
#define CHECK(cond)                                                                     \
    do {                                                                                \
        ++checks;                                                                       \
        if (!(cond)) return std::printf("line %d: %s\n", __LINE__, #cond), 1;           \
    } while (0)

static rf::RowFrames list(const std::vector<int> &ids, bool full) {
    rf::RowFrames f{};
    for (size_t i = 0; i < ids.size(); ++i) f.frame[i] = static_cast<uint8_t>(ids[i]);
    f.in_full = full;
    return f;
}

// The widest distance in x, in rows, of two rows that a tile of 256 rows of the product holds: its
// first and last one, as positions grow.
static int64_t widest(const std::vector<int> &ids, int64_t N, bool full) {
    const int64_t rows = static_cast<int64_t>(ids.size()) * N;
    auto at = [&](int64_t r) { return full ? ids[r / N] * N + r % N : r; };
    int64_t most = 0;
    for (int64_t r = 0; r < rows; r += 256) {
        const int64_t last = r + 255 < rows ? r + 255 : rows - 1;
        most = at(last) - at(r) > most ? at(last) - at(r) : most;
    }
    return most;
}

static int meeting(const std::vector<int> &ids, int64_t N) {
    const int32_t M = static_cast<int32_t>(ids.size());
    for (const bool full : {false, true}) {
        const rf::RowFrames f = list(ids, full);
        const int64_t gap = rf::linear_gap(f, M, N), far = widest(ids, N, full);
        CHECK(gap <= far && far <= gap + 255);   // (no tile is wider, and one is as wide)
        CHECK(full || gap == 0);
        // 32-bit offsets exactly where the widest tile's fit, for rows of 16 bytes to just below 8 MB
        for (int64_t row = 16; row < (1 << 23); row = row * 3 + 16) {
            CHECK(rf::linear_far(f, M, N, row) || (far + 1) * row <= 2147483647);
            CHECK(!rf::linear_far(f, M, N, row) || (far + 258) * row >= 2147483647);
        }
    }
    return 0;
}

static int frames_that_meet() {
    const int64_t sizes[] = {1, 2, 37, 84, 85, 86, 127, 128, 129, 200, 253, 254, 255, 256, 257, 300, 511, 512, 1024, 1560, 3600};
    std::mt19937 rng(7);
    for (const int64_t N : sizes) {
        for (const std::vector<int> &ids : {std::vector<int>{0}, {255}, {0, 1}, {0, 255}, {0, 20}, {0, 1, 255}, {0, 254, 255},
                                            {0, 127, 255}, {3, 4, 5, 200, 201, 255}})
            if (meeting(ids, N)) return 1;
        for (int i = 0; i < 40; ++i) {
            std::vector<int> ids;
            const int keep = 1 + static_cast<int>(rng() % 100);
            for (int t = 0; t < 256; ++t)
                if (static_cast<int>(rng() % 100) < keep) ids.push_back(t);
            if (!ids.empty() && meeting(ids, N)) return 1;
        }
    }
    // keyframes of a 720p video and a wide feed-forward's rows: 3,600 rows of 40,960 bytes, 19 frames apart
    CHECK(rf::linear_far(list({0, 20}, true), 2, 3600, 40960));
    CHECK(!rf::linear_far(list({0, 20}, false), 2, 3600, 40960));
    // frames of whole tiles never meet in one
    CHECK(!rf::linear_far(list({0, 20}, true), 2, 4096, 40960));
    return 0;
}

// A plan covers its product, and every form is some product's best in each type that has it.
static int forms_in_use() {
    std::mt19937_64 rng(3);
    auto upto = [&](double most) { return static_cast<int64_t>(std::exp(std::uniform_real_distribution<>(0, std::log(most))(rng))); };
    int64_t seen[2][2][rf::kLinearForms] = {};
    for (int i = 0; i < 200000; ++i) {
        const int dtype = i & 1 ? RF_F32 : RF_BF16;
        const int64_t rows = i % 3 ? upto(100000) : upto(64), K = 8 * upto(4000), n = 8 * upto(4000);
        const bool far = i % 5 == 0, ws = i % 4 != 0;
        const rf::LinearPlan p = rf::linear_plan(rows, static_cast<int32_t>(K), static_cast<int32_t>(n), dtype, 256, far, ws);
        CHECK(p.form >= 0 && p.form < rf::kLinearForms);
        CHECK(!far || p.form == rf::kTile128);
        CHECK(dtype == RF_BF16 || (p.form != rf::kStream64 && p.form != rf::kTile256));
        const int64_t tile_rows[] = {16, 32, 64, 32, 64, 64, 128, 256}, tile_cols[] = {16, 32, 16, 256, 256, 128, 128, 256};
        CHECK(p.row_tiles == (rows + tile_rows[p.form] - 1) / tile_rows[p.form]);
        CHECK(p.col_tiles == (n + tile_cols[p.form] - 1) / tile_cols[p.form]);
        const int64_t step = p.form <= rf::kFew64 ? 64 : rf::kLinearStep, bytes = K * (dtype == RF_F32 ? 4 : 2);
        CHECK(p.steps == (bytes + step - 1) / step);
        CHECK(p.parts >= 1 && (ws || p.parts == 1));
        // every part has a step, and the last one ends the reduction
        CHECK(static_cast<int64_t>(p.parts) * p.per_part >= p.steps && static_cast<int64_t>(p.parts - 1) * p.per_part < p.steps);
        ++seen[dtype][p.parts > 1][p.form];
    }
    for (int form = 0; form < rf::kLinearForms; ++form) {
        CHECK(seen[RF_BF16][0][form] + seen[RF_BF16][1][form] > 0);
        if (form != rf::kStream64 && form != rf::kTile256) CHECK(seen[RF_F32][0][form] + seen[RF_F32][1][form] > 0);
    }
    return 0;
}

// What is not refused can be launched: threads of the launch, and of the join's, below 2^32.
static int launches_fit() {
    std::mt19937_64 rng(5);
    auto upto = [&](double most) { return static_cast<int64_t>(std::exp(std::uniform_real_distribution<>(0, std::log(most))(rng))); };
    int near = 0, refused = 0;
    for (int i = 0; i < 300000; ++i) {
        const int dtype = i & 1 ? RF_F32 : RF_BF16;
        const int64_t rows = i % 3 ? 1 + static_cast<int64_t>(rng() % 2147483647) : upto(2147483647.0);
        const int64_t K = 8 * upto(200000), n = i % 4 ? 8 * upto(16) : 8 * upto(268435455);
        const int cus = i % 5 ? 256 : 1 + static_cast<int>(upto(RF_MAX_COMPUTE_UNITS - 1)), xcds = i % 7 ? 8 : 1 + static_cast<int>(rng() % 64);
        if (!rf::linear_whole_fits(rows, n)) {
            ++refused;
            continue;
        }
        const rf::LinearPlan p = rf::linear_plan(rows, static_cast<int32_t>(K), static_cast<int32_t>(n), dtype, cus, i % 11 == 0, i % 2);
        const int64_t tiles = p.row_tiles * p.col_tiles, rounded = p.form <= rf::kFew64 ? tiles : (tiles + xcds - 1) / xcds * xcds;
        const int64_t threads = rounded * p.parts * (p.form <= rf::kFew64 || p.form == rf::kTile256 ? 512 : 256);
        CHECK(tiles > 0 && threads <= 0xffffffffLL);
        CHECK(p.parts == 1 || (rows * (n / 4) + 255) / 256 * 256 <= 0xffffffffLL);
        near += threads > (1LL << 30);
    }
    CHECK(near > 100 && refused > 100);
    return 0;
}

int main() {
    if (frames_that_meet() || forms_in_use() || launches_fit()) return 1;
    std::printf("ok %d\n", checks);
    return 0;
}
