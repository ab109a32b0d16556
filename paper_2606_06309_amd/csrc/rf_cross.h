// What the kernels of cross attention share: the launch arguments, the query
// rows of a tile, a sequence's keys, and the join of a split key axis.
//
// The query heads that read one key head are walked as one list of rows: row r
// of key head hk is query r % Lq of head hk * group + r / Lq. A tile of rows thus
// holds several heads where queries are few.
#pragma once

#include "rf_cross_plan.h"
#include "rf_device.h"

namespace rf {

struct CrossKArgs {
    const void *q, *k, *v;
    void *out;
    const int32_t *kv_lengths;
    const uint8_t *key_mask;
    int64_t qs[3], ks[3], vs[3], os[3];   // {batch, token, head} in elements
    uint32_t rows;           // query rows of a key head: group * Lq
    int32_t B, Lq, Lk, group;
    int32_t q_tiles;         // tiles of rows of a (sequence, key head)
    int32_t tiles;           // of the launch
    int32_t per_xcd, xcds;   // workgroup id i runs on XCD i % xcds
    int32_t parts;           // of the key axis (1: not split)
    int32_t walkers;         // many rows: workgroups of the launch, each with a run of tiles
    float scale_log2;        // log2(e) / sqrt(d)
    float *ws_o;             // [tile * parts + part][32][D] unnormalised O
    float *ws_ml;            // [tile * parts + part][32][2] reference and row sum
};

// A tile: its sequence, key head and first row. Tiles are counted by key head, then
// rows, then sequence: sequences may differ much in length (a prompt's and an empty
// one's, in guidance), and this way neighbours share out the long ones. Consecutive
// workgroup ids go round-robin to the XCDs, so each XCD gets a contiguous range of
// tiles whose workgroups read the same heads' keys and values through that XCD's L2.
struct CrossTile {
    int32_t tile, b, hk;
    uint32_t row0;
};
template <int kRows>
__device__ __forceinline__ CrossTile cross_tile_at(const CrossKArgs &a, int32_t tile) {
    CrossTile t;
    t.tile = tile;
    const int32_t r = tile / a.B;
    t.b = tile - r * a.B;
    t.hk = r / a.q_tiles;
    t.row0 = static_cast<uint32_t>(r - t.hk * a.q_tiles) * kRows;
    return t;
}
template <int kRows>
__device__ __forceinline__ bool cross_tile(const CrossKArgs &a, int bid, CrossTile &t) {
    const int32_t tile = (bid % a.xcds) * a.per_xcd + bid / a.xcds;
    if (tile >= a.tiles) return false;
    t = cross_tile_at<kRows>(a, tile);
    return true;
}

// Element offset of query row r's first element in a tensor of these strides.
__device__ __forceinline__ int64_t row_offset(const CrossKArgs &a, const int64_t (&s)[3], const CrossTile &t,
                                              uint32_t r) {
    const uint32_t g = a.group == 1 ? 0 : r / static_cast<uint32_t>(a.Lq);
    return t.b * s[0] + static_cast<int64_t>(r - g * a.Lq) * s[1] + (t.hk * a.group + static_cast<int64_t>(g)) * s[2];
}

// A sequence's length as it stands, and as it counts.
__device__ __forceinline__ int32_t given_count(const CrossKArgs &a, int b) {
    return a.kv_lengths ? a.kv_lengths[b] : a.Lk;
}
__device__ __forceinline__ int32_t key_count(const CrossKArgs &a, int32_t given) {
    const int32_t n = __builtin_amdgcn_readfirstlane(given);
    return n < 0 ? 0 : n < a.Lk ? n : a.Lk;
}

// A masked launch's valid keys among keys key0 .. key0 + 63 (n: the sequence's length).
__device__ __forceinline__ uint64_t key_bits(const CrossKArgs &a, int b, int32_t key0, int32_t n, int lane) {
    bool ok = key0 + lane < n;
    if (ok) ok = a.key_mask[static_cast<int64_t>(b) * a.Lk + key0 + lane] != 0;
    return __builtin_amdgcn_ballot_w64(ok);
}

// An offset past every buffer resource: a load from it gives zero.
constexpr int kNowhere = 0x7fffffff - 15;

hipError_t launch_cross_f32(const CrossKArgs &a, int32_t head_dim, bool few, uint32_t grid, hipStream_t stream);

}  // namespace rf
