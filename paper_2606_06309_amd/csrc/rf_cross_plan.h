// How a cross attention's launch is cut: host rules, which need no device, and the sizes that the
// kernels share with them.
#pragma once

#include "rf_internal.h"

namespace rf {

// Both types' tiles: rows of a workgroup where rows are many, and where they are few.
constexpr int kCrossTileRows = 128;
constexpr int kCrossFewRows = 32;
// bf16: keys of a tile where rows are many, and where they are few; workgroups to a compute unit.
constexpr int kCrossTileKeys = 64;
constexpr int cross_few_keys(int head_dim) { return head_dim == 64 ? 64 : 32; }
constexpr int cross_tile_waves(int head_dim, bool mask) { return head_dim == 64 && !mask ? 3 : 2; }
// Waves of a workgroup where rows are few.
constexpr int cross_few_waves(int head_dim, int dtype) { return dtype == RF_F32 && head_dim == 128 ? 4 : 8; }
// Parts that a key axis is split into at most.
constexpr int kCrossMaxParts = 64;

// A launch has fewer than 2^32 threads along an axis (of workgroups a multiple of the XCDs, 64 at most).
constexpr bool cross_fits(int64_t tiles, int64_t parts, int64_t threads) {
    return (tiles + 63) * parts * threads <= 0xffffffffLL;
}

// Whether the form of many rows can be launched, the one that is left where the other cannot:
// in bf16 always (as many workgroups as are resident walk its tiles).
inline bool cross_whole_fits(int32_t B, int64_t rows, int32_t kv_heads, int32_t dtype) {
    const int64_t tiles = (rows + kCrossTileRows - 1) / kCrossTileRows * B * kv_heads;
    return dtype != RF_F32 || cross_fits(tiles, 1, 2 * kCrossTileRows);
}

// How a launch is cut: tiles of 128 rows, or of 32 with the keys shared out and
// `parts` workgroups to a tile.
//
// The choice goes by the forms' times in us, counted in rounds of the device: a round
// has a fixed part and the tiles of keys that a workgroup (of the few-row form: its
// busiest wave) walks; a split has the join. Tiles of keys cost more where more
// workgroups share a compute unit, and a round that few of them share counts for as
// much less. Counts and measured times, us (tile / few):
//   1,560 x 512 keys, 12 heads x 128: 14 / 25     9,360 x 77, 12 x 128: 21 / 66
//   2 x 500 x 1,000, 8 x 128: 22 / 12             300 x 5,000, 8 x 128: 83 / 20 (3 parts)
//   128 x 20,000, 8 x 64: 224 / 21 (8 parts)      3 x 1,581 x 334, 5 x 64: 10 / 17
// and in fp32 1,560 x 512, 12 x 128: 76 / 72; 512 x 512, 12 x 64: 41 / 15;
// 4,680 x 512, 12 x 128: 140 / 166; 6,400 x 512, 12 x 64: 114 / 137.
struct CrossPlan {
    bool few;
    int32_t parts;
    int64_t tiles;
};

struct CrossCost {
    double tile[3];            // a tile of keys with one, two, three workgroups to a compute unit
    double few;                // a wave's tile of keys in the few-row form
    int32_t keys, few_keys;    // keys of a tile
    int32_t few_waves;
};
// us of a round whatever its keys, in either form, and of the join.
constexpr double kCrossRound = 4.0, kCrossFewRound = 4.5, kCrossJoin = 4.0;

inline CrossPlan cross_plan(int32_t B, int64_t rows, int32_t kv_heads, int32_t Lk, int32_t head_dim, int32_t dtype,
                            bool mask, bool may_split, int32_t cus) {
    static const CrossCost costs[2][2] = {
        {{{0.7, 1.06, 1.44}, 1.9, kCrossTileKeys, cross_few_keys(64), cross_few_waves(64, RF_BF16)},
         {{1.0, 1.9, 1.9}, 1.9, kCrossTileKeys, cross_few_keys(128), cross_few_waves(128, RF_BF16)}},
        {{{2.4, 4.8, 4.8}, 4.5, 32, 32, cross_few_waves(64, RF_F32)},
         {{4.5, 9.0, 9.0}, 4.9, 32, 32, cross_few_waves(128, RF_F32)}}};
    const CrossCost &c = costs[dtype == RF_F32][head_dim == 128];
    auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    const int64_t heads = static_cast<int64_t>(B) * kv_heads;
    const int64_t whole = up(rows, kCrossTileRows) * heads, few = up(rows, kCrossFewRows) * heads;
    const int64_t most = dtype == RF_F32 ? 2 : cross_tile_waves(head_dim, mask);   // workgroups to a compute unit
    const int64_t share = up(whole, cus) < most ? up(whole, cus) : most;
    const double t_whole = static_cast<double>(up(whole, cus)) / static_cast<double>(share) *
                           (kCrossRound + static_cast<double>(up(Lk, c.keys)) * c.tile[share - 1]);
    CrossPlan p{false, 1, whole};
    double best = 0.95 * t_whole;   // (the few-row form reads keys four times as often)
    const int64_t key_tiles = up(Lk, c.few_keys);
    for (int64_t parts = 1; parts <= kCrossMaxParts; ++parts) {
        if (!cross_fits(few, parts, 64 * c.few_waves)) break;
        if (parts > 1 && (!may_split || parts * c.few_waves > key_tiles || few * (parts - 1) >= 2 * cus)) break;
        const double t = static_cast<double>(up(few * parts, cus)) *
                             (kCrossFewRound + static_cast<double>(up(key_tiles, parts * c.few_waves)) * c.few) +
                         (parts > 1 ? kCrossJoin : 0.0);
        if (t < best) {
            best = t;
            p = CrossPlan{true, static_cast<int32_t>(parts), few};
        }
    }
    return p;
}

}  // namespace rf
