/* The group norm's workspace holds what its launches put there, one after the other: partial sums of 8 bytes, of fp32 rows the rests
   of their means and of the groups' (4 bytes each), the groups' mean and 1 / deviation. Prints "ok <checks>"; exits 1 at the first
   mismatch. */
#include <cmath>
#include <cstdio>
#include <random>

#include "rf_norm_plan.h"

int main() {
    std::mt19937 rng(17);
    auto upto = [&](double most) { return static_cast<int64_t>(std::exp(std::uniform_real_distribution<double>(0, std::log(most))(rng))); };
    long checks = 0, parts = 0;
    for (int i = 0; i < 100000; ++i) {
        const int32_t dtype = i % 2 ? RF_F32 : RF_BF16;
        const bool rows8 = i % 3 == 0;
        const int32_t unit = rows8 ? 16 : dtype == RF_F32 ? 4 : 8, C = unit * static_cast<int32_t>(upto(8192.0 / unit));
        int32_t G = static_cast<int32_t>(upto(C));
        while (C % G != 0) --G;
        const int32_t M = static_cast<int32_t>(upto(257)), together = i % 5 ? 1 : M;
        const int64_t N = upto(i % 7 ? 5000 : 2147483647.0 / M);
        const int32_t cus = i % 4 == 0 ? 1 + static_cast<int32_t>(upto(304)) : 256;
        const rf::NormPlan p = rf::norm_plan(M, N, C, G, together, rows8, dtype, cus);
        ++checks;
        if (p.block > 0) {
            if (p.ws_bytes != 0) return std::printf("a workspace of %lld bytes for one launch\n", static_cast<long long>(p.ws_bytes)), 1;
            continue;
        }
        ++parts;
        const int64_t totals = static_cast<int64_t>(M / together) * G, rests = dtype == RF_F32 ? (p.sums + totals) * 4 : 0;
        if (p.sums != static_cast<int64_t>(M) * p.parts * p.slices * p.local || p.sums * 8 + rests > p.entries * 8 ||
            p.entries * 8 % 16 != 0 || p.entries * 8 + totals * 8 > p.ws_bytes)
            return std::printf("M=%d N=%lld C=%d G=%d together=%d rows8=%d dtype=%d cus=%d\n", M, static_cast<long long>(N), C, G, together,
                               rows8, dtype, cus), 1;
    }
    if (parts < 10000) return std::printf("%ld plans of parts\n", parts), 1;
    std::printf("ok %ld\n", checks);
    return 0;
}
