/* Host rules of a cross attention's launch: whatever is not refused can be launched. Prints "ok <checks>"; exits 1 at
   the first mismatch. */
#include <cmath>
#include <cstdio>
#include <random>

#include "rf_cross_plan.h"

static int checks;
#define CHECK(cond)                                                                     \
    do {                                                                                \
        ++checks;                                                                       \
        if (!(cond)) return std::printf("line %d: %s\n", __LINE__, #cond), 1;           \
    } while (0)

// The threads of the launch that a plan stands for, on a device of `xcds` parts.
static int64_t threads(const rf::CrossPlan &p, int head_dim, int dtype, bool mask, int cus, int xcds) {
    if (!p.few && dtype == RF_BF16) {   // walkers
        const int64_t most = static_cast<int64_t>(rf::cross_tile_waves(head_dim, mask)) * cus;
        return ((p.tiles < most ? p.tiles : most) + xcds - 1) / xcds * xcds * 256;
    }
    const int64_t groups = (p.tiles + xcds - 1) / xcds * xcds * p.parts;
    return groups * 64 * (p.few ? rf::cross_few_waves(head_dim, dtype) : rf::kCrossTileRows / 32);
}

static int launches_fit() {
    std::mt19937_64 rng(11);
    auto upto = [&](double most) { return static_cast<int64_t>(std::exp(std::uniform_real_distribution<>(0, std::log(most))(rng))); };
    int near = 0, refused = 0;
    for (int i = 0; i < 400000; ++i) {
        const int64_t Lq = i % 3 == 0 ? 1 + i % 40 : upto(1 << 28), kv = upto(128), group = i % 2 ? 1 : upto(64);
        const int64_t most = (int64_t{1} << 24) / ((Lq + 31) / 32 * kv * group);
        if (most < 1) continue;
        const int64_t B = i % 2 ? most - static_cast<int64_t>(rng() % 3) : upto(most);   // up to the documented limit
        if (B < 1) continue;
        for (const int dtype : {RF_BF16, RF_F32})
            for (const int head_dim : {64, 128}) {
                const int64_t Lk = upto(1 << 30);
                const bool mask = rng() & 1, ws = rng() & 1;
                const int cus = i % 5 ? 256 : 1 + static_cast<int>(upto(RF_MAX_COMPUTE_UNITS - 1));
                const int xcds = i % 7 ? 8 : 1 + static_cast<int>(rng() % 64);
                if (!rf::cross_whole_fits(B, group * Lq, kv, dtype)) {
                    CHECK(dtype == RF_F32 && (group * Lq + 127) / 128 * B * kv > (1 << 24) - 64);
                    ++refused;
                    continue;
                }
                const rf::CrossPlan p = rf::cross_plan(B, group * Lq, kv, Lk, head_dim, dtype, mask, ws, cus);
                CHECK(p.parts >= 1 && p.parts <= rf::kCrossMaxParts && (p.parts == 1 || p.few));
                CHECK(p.tiles == (group * Lq + (p.few ? 31 : 127)) / (p.few ? 32 : 128) * B * kv);
                const int64_t n = threads(p, head_dim, dtype, mask, cus, xcds);
                CHECK(n <= 0xffffffffLL);
                CHECK(p.parts == 1 || p.tiles * 32 * 256 <= 0xffffffffLL);   // the join
                near += n > (1LL << 30);
            }
    }
    CHECK(near > 100 && refused > 100);
    return 0;
}

int main() {
    if (launches_fit()) return 1;
    std::printf("ok %d\n", checks);
    return 0;
}
