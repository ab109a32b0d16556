/* Host rules of the group norm's launches against plain walks over rows and channels, and of products of 8-bit integers.
   Prints "ok <checks>"; exits 1 at the first mismatch. */
#include <cmath>
#include <cstdio>
#include <random>

#include "rf_linear_plan.h"
#include "rf_norm_plan.h"

static long checks;
#define CHECK(cond)                                                                     \
    do {                                                                                \
        ++checks;                                                                       \
        if (!(cond)) return std::printf("line %d: %s\n", __LINE__, #cond), 1;           \
    } while (0)

static int check(int32_t M, int64_t N, int32_t C, int32_t G, int32_t together, bool rows8, int32_t dtype, int32_t cus,
                 int *slices, int *few) {
    const rf::NormPlan p = rf::norm_plan(M, N, C, G, together, rows8, dtype, cus);
    const int64_t vec = dtype == RF_F32 ? 4 : 8, columns = C / vec, per = C / G;
    CHECK(p.vec == vec);
    CHECK(p.cols >= 1 && p.lines >= 1 && p.slices >= 1);
    // every column has a slice, and no slice is empty
    CHECK(static_cast<int64_t>(p.slices) * p.cols >= columns && static_cast<int64_t>(p.slices - 1) * p.cols < columns);
    if (p.block > 0) {
        ++*slices;
        CHECK(!rows8 && p.ws_bytes == 0);
        // whole groups, all rows, what LDS holds
        CHECK(static_cast<int64_t>(p.cols) * p.slices == columns && p.cols * vec % per == 0);
        CHECK(p.cols * p.lines <= p.block && static_cast<int64_t>(p.hold) * p.lines >= together * N);
        CHECK(static_cast<int64_t>(p.hold - 1) * p.lines < together * N);
        const int64_t some = p.block * 4, groups = 2 * rf::kNormSliceGroups * 4;
        int64_t hold = 0;
        for (const rf::NormBlock &b : rf::kNormBlocks)
            if (b.threads == p.block) hold = b.hold;
        CHECK(p.hold <= hold && hold * p.block * 16 + p.block * vec * 4 + some + groups <= 160 * 1024);
        CHECK(p.cols * vec / per <= rf::kNormSliceGroups);
        CHECK(static_cast<int64_t>(M / together) * p.slices <= 2LL * cus);
        return 0;
    }
    CHECK(p.cols * p.lines <= rf::kNormThreads && p.parts >= 1 && p.parts <= 65535 && p.row_parts >= 1 && p.row_parts <= 65535);
    // parts: the chunks of a frame in turn
    const int64_t chunk = static_cast<int64_t>(rf::kNormRows) * p.lines;
    int64_t all = 0;
    if (N <= 200000) {
        for (int32_t part = 0; part < p.parts; ++part) {
            int64_t rows = 0;
            for (int64_t at = part * chunk; at < N; at += p.parts * chunk) rows += at + chunk <= N ? chunk : N - at;
            CHECK(static_cast<float>(rows) == p.runs.rows(part));
            CHECK(rows > 0);
            all += rows;
        }
        CHECK(all == N);
    }
    // groups that a slice meets
    for (int32_t s = 0; s < p.slices; ++s) {
        const int64_t c0 = static_cast<int64_t>(s) * p.cols * vec, c1 = c0 + p.cols * vec < C ? c0 + p.cols * vec : C;
        CHECK((c1 - 1) / per - c0 / per + 1 <= p.local);
    }
    CHECK(p.entries % 2 == 0 && p.entries >= static_cast<int64_t>(M) * p.parts * p.slices * p.local);
    CHECK(p.ws_bytes == p.entries * 8 + static_cast<int64_t>(M / together) * G * 8);
    if (p.few_parts) {
        ++*few;
        CHECK(p.parts * together <= rf::kNormFewParts && (rows8 ? G : p.local) <= rf::kNormFewGroups);
        CHECK(rows8 || (p.row_parts * static_cast<int64_t>(M) * p.slices <= rf::kNormFewWorkgroups * static_cast<int64_t>(cus) && !p.y_past));
    }
    // launches of fewer than 2^32 threads
    const double threads = 256.0 * M * p.slices;
    CHECK(threads * p.parts < 4294967296.0 && threads * p.row_parts < 4294967296.0 && 64.0 * G * (M / together) < 4294967296.0);
    return 0;
}

// A plan covers its product, by a form that 8-bit integers have, each of which is some product's best.
static int products() {
    std::mt19937_64 rng(11);
    auto upto = [&](double most) { return static_cast<int64_t>(std::exp(std::uniform_real_distribution<>(0, std::log(most))(rng))); };
    int64_t seen[rf::kLinearForms] = {}, split = 0;
    for (int i = 0; i < 100000; ++i) {
        const int64_t rows = i % 3 ? upto(100000) : upto(64), K = 16 * upto(4096), n = 4 * upto(8000);
        const bool far = i % 5 == 0, ws = i % 4 != 0;
        const rf::LinearPlan p = rf::linear_plan(rows, static_cast<int32_t>(K), static_cast<int32_t>(n), rf::kI8, 256, far, ws);
        CHECK(p.form >= 0 && p.form < rf::kLinearForms && p.form != rf::kStream32 && p.form != rf::kStream64);
        CHECK(!far || p.form == rf::kTile128);
        const int64_t tile_rows[] = {16, 32, 64, 32, 64, 64, 128, 256}, tile_cols[] = {16, 32, 16, 256, 256, 128, 128, 256};
        CHECK(p.row_tiles == (rows + tile_rows[p.form] - 1) / tile_rows[p.form]);
        CHECK(p.col_tiles == (n + tile_cols[p.form] - 1) / tile_cols[p.form]);
        const int64_t step = p.form <= rf::kFew64 ? 64 : rf::kLinearStep;
        CHECK(p.steps == (K + step - 1) / step && p.parts >= 1 && (ws || p.parts == 1));
        CHECK(static_cast<int64_t>(p.parts) * p.per_part >= p.steps && static_cast<int64_t>(p.parts - 1) * p.per_part < p.steps);
        ++seen[p.form];
        split += p.parts > 1;
    }
    for (int form = 0; form < rf::kLinearForms; ++form)
        CHECK(form == rf::kStream32 || form == rf::kStream64 || seen[form] > 0);
    CHECK(split > 0);
    return 0;
}

int main() {
    if (products()) return 1;
    for (int32_t n = 1; n <= 8192; ++n) {
        const float share = 1.0f / static_cast<float>(n);
        for (int32_t i = 0; i < 8192; ++i)
            if (rf::divide(i, share) != i / n) return std::printf("%d / %d\n", i, n), 1;
        ++checks;
        if (n <= 1024)      // (of columns of four and eight, as the kernels make them)
            for (const int32_t v : {4, 8})
                for (int32_t i = 0; i < 8192; ++i)
                    if (rf::divide(i, share * (1.0f / static_cast<float>(v))) != i / (n * v)) return std::printf("%d / %d %d\n", i, n, v), 1;
    }
    int slices = 0, few = 0, bad = 0;
    std::mt19937 rng(7);
    auto upto = [&](double most) { return static_cast<int64_t>(std::exp(std::uniform_real_distribution<double>(0, std::log(most))(rng))); };
    for (int i = 0; i < 20000 && !bad; ++i) {
        const int32_t dtype = i % 2 ? RF_F32 : RF_BF16;
        const bool rows8 = i % 3 == 0;
        const int32_t unit = rows8 ? 16 : dtype == RF_F32 ? 4 : 8, C = unit * static_cast<int32_t>(upto(8192.0 / unit));
        int32_t G = static_cast<int32_t>(upto(C));
        while (C % G != 0) --G;
        const int32_t M = static_cast<int32_t>(upto(257)), together = i % 5 ? 1 : M;
        const int64_t N = upto(i % 7 ? 5000 : 2147483647.0 / M);
        const int32_t cus = i % 4 == 0 ? 1 + static_cast<int32_t>(upto(304)) : 256;
        bad = check(M, N, C, G, together, rows8, dtype, cus, &slices, &few);
        if (bad) std::printf("M=%d N=%lld C=%d G=%d together=%d rows8=%d dtype=%d cus=%d\n", M, static_cast<long long>(N), C, G, together, rows8, dtype, cus);
    }
    if (bad) return 1;
    if (slices < 500 || few < 200) return std::printf("slices %d few %d\n", slices, few), 1;
    std::printf("ok %ld\n", checks);
    return 0;
}
