/* Every form that a matrix product is planned in is one that its operands' type has, whatever the sizes, the device and
   the workspace: a launch of another would leave y unwritten. Prints "ok <checks>"; exits 1 at the first mismatch. */
#include <cmath>
#include <cstdio>
#include <random>

#include "rf_linear_plan.h"

int main() {
    long checks = 0;
    std::mt19937_64 rng(13);
    auto upto = [&](double most) { return static_cast<int64_t>(std::exp(std::uniform_real_distribution<>(0, std::log(most))(rng))); };
    long seen[3][rf::kLinearForms] = {};
    for (int i = 0; i < 300000; ++i) {
        const int32_t in = i % 3;      // RF_BF16, RF_F32, kI8
        const int64_t rows = i % 2 ? upto(100000) : upto(64), K = 16 * upto(4096), n = 8 * upto(i % 5 ? 4000 : 200000);
        const int32_t cus = i % 7 ? 256 : static_cast<int32_t>(upto(RF_MAX_COMPUTE_UNITS));
        const rf::LinearPlan p = rf::linear_plan(rows, static_cast<int32_t>(K), static_cast<int32_t>(n), in, cus, i % 11 == 0, i % 4 != 0);
        if (!rf::linear_has(p.form, in) || p.row_tiles < 1 || p.col_tiles < 1)
            return std::printf("form %d of type %d: %lld x %lld x %lld, %d units\n", p.form, in, static_cast<long long>(rows),
                               static_cast<long long>(K), static_cast<long long>(n), cus), 1;
        ++seen[in][p.form];
        ++checks;
    }
    // and what a type has is planned for some product of it
    for (int32_t in = 0; in < 3; ++in)
        for (int32_t form = 0; form < rf::kLinearForms; ++form) {
            if (rf::linear_has(form, in) != (seen[in][form] > 0)) return std::printf("form %d of type %d, %ld products\n", form, in, seen[in][form]), 1;
            ++checks;
        }
    if (rf::linear_has(rf::kLinearForms, RF_BF16) || rf::linear_has(-1, rf::kI8)) return std::printf("no form\n"), 1;
    std::printf("ok %ld\n", checks);
    return 0;
}
