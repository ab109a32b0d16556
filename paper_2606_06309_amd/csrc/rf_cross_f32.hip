// Attention to an encoder's states of another length for gfx950, fp32 throughout
// on the fp32 matrix instructions; the method and the layouts are those of the
// bf16 kernels in rf_cross.hip, with these differences:
//
//  * v_mfma_f32_32x32x2_f32 takes one fp32 per lane of either operand, so a
//    16-byte LDS read of a K row feeds four of them; the accumulators of
//    S^T = K Q^T are, step by step, the B operand of O^T = V^T P^T, whose row i
//    may stand for any dimension: lane i takes dimensions i D/32 .. + D/32 - 1, one
//    wide LDS read of a V row.
//  * The reference is the exact running maximum, subtracted before the scale, so the
//    largest score gives exactly 1 however large it is.
//  * A tile is 32 keys, 16 KB (head dimension 128) or 8 KB (64) of K and of V.
//
// What bounds it: on long walks the fp32 matrix instructions (64 cycles each), busy 79 % of the
// cycles at 8,000 x 4,000 keys, 12 heads x 64 (798 us, 123 TFLOP/s); one 16-byte LDS read
// feeds four, and the vector and LDS pipes are at 15 % and 5 %. Over a prompt they are busy less,
// as workgroups do not share out evenly: 6,400 x 512, 12 x 64 (109 us, 92 TFLOP/s, 55 %) is 600 of
// them on 512 places, and the last 88 take a quarter of the time alone; 2 x 5,000 x 1,000, 8 x 64:
// 208 us, 98, 63 %. Small calls are bound by the launch and one walk of a tile: 192 x 77, 2 x 64: 8.4 us.
#include "rf_cross.h"

namespace rf {
namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

constexpr float kInf = __builtin_huge_valf();
constexpr int kKeys = 32;   // of a tile

template <int D>
struct Tile {
    static constexpr int kRow = 4 * D;
    static constexpr int kSlots = kRow / 16;
    static constexpr int kBytes = kKeys * kRow;
    static constexpr int kRowsPerLoad = 1024 / kRow;
    static constexpr int kLoads = kBytes / 1024;
};

template <int D>
struct Wave {
    static constexpr int kDb = D / 32;
    f32x4_t qf[D / 8];
    f32x16_t o[kDb];
    float m, l;   // running maximum of the raw scores; this lane's part of the row sum
};

template <int D>
__device__ __forceinline__ void start(const CrossKArgs &a, const CrossTile &t, uint32_t row, int grp, Wave<D> &w) {
    if (row < a.rows) {
        const float *qp = static_cast<const float *>(a.q) + row_offset(a, a.qs, t, row) + grp * 4;
#pragma unroll
        for (int c = 0; c < D / 8; ++c) w.qf[c] = *reinterpret_cast<const f32x4_t *>(qp + c * 8);
    } else {
#pragma unroll
        for (int c = 0; c < D / 8; ++c) w.qf[c] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
#pragma unroll
    for (int db = 0; db < Wave<D>::kDb; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) w.o[db][r] = 0.0f;
    w.m = -kInf;
    w.l = 0.0f;
}

// Loads i0 .. i0 + kN - 1 of a tile into LDS (1 KB each); K's 16-byte slots permuted by key % 16.
template <int D, bool kMask, bool kKey, int kN>
__device__ __forceinline__ void issue(const float *head, int64_t stride, int32_t key0, int32_t left, uint64_t bits,
                                      uint8_t *dst, int i0, int lane) {
    using L = Tile<D>;
    const int64_t span = ((static_cast<int64_t>(left) - 1) * stride + D) * 4;
    const int32_t rec = __builtin_amdgcn_readfirstlane(static_cast<int32_t>(span < kNowhere ? span : kNowhere));
    const __amdgpu_buffer_rsrc_t r =
        __builtin_amdgcn_make_buffer_rsrc(uniform_ptr(head + key0 * stride), 0, rec, kBufferWord3);
    const int sub = lane / L::kSlots, slot = lane % L::kSlots;
    const int step = static_cast<int>(L::kRowsPerLoad * stride * 4), at0 = static_cast<int>(sub * stride * 4);
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        const int key = (i0 + i) * L::kRowsPerLoad + sub;
        int at = at0 + (i0 + i) * step + (kKey ? slot ^ (key & 15) : slot) * 16;
        if constexpr (kMask) {
            if (!((bits >> key) & 1)) at = kNowhere;
        }
        load_lds16(r, (lds_void_t *)(dst + (i0 + i) * 1024), at);
    }
}

template <int D>
__device__ __forceinline__ f32x16_t scores(const uint8_t *kb, int col, int grp, const f32x4_t (&qf)[D / 8]) {
    const uint8_t *row = kb + col * (4 * D);
    const int base = (grp ^ (col & 15)) * 16;
    f32x16_t s = {};
#pragma unroll
    for (int c = 0; c < D / 8; ++c) {
        const f32x4_t kf = *reinterpret_cast<const f32x4_t *>(row + (base ^ (c * 32)));
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qf[c][e], s, 0, 0, 0);
    }
    return s;
}

template <int D>
__device__ __forceinline__ void softmax(Wave<D> &w, f32x16_t &s, uint32_t word, int grp, float sl2) {
    if (word != 0xffffffffu) {
        const uint32_t mine = word >> (4 * grp);
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (!((mine >> ((r / 4) * 8 + r % 4)) & 1u)) s[r] = -kInf;
    }
    float mx = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
    mx = fmaxf(w.m, halves_max(mx));
    // rows whose maximum stays keep O and l as they are (their factor is exactly 1)
    if (__builtin_amdgcn_ballot_w64(mx > w.m) != 0) {
        const float corr = mx > w.m ? fast_exp2((w.m - mx) * sl2) : 1.0f;   // 0 from -inf on
        w.l *= corr;
#pragma unroll
        for (int db = 0; db < Wave<D>::kDb; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) w.o[db][r] *= corr;
        w.m = mx;
    }
    const float ref = mx == -kInf ? 0.0f : mx;   // no score above -inf so far: every probability is 0
    float sum[4];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        s[r] = fast_exp2((s[r] - ref) * sl2);
        sum[r / 4] = r % 4 == 0 ? s[r] : sum[r / 4] + s[r];
    }
    w.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

template <int D>
__device__ __forceinline__ void values(Wave<D> &w, const uint8_t *vb, const f32x16_t &p, int col, int grp) {
    constexpr int kDb = D / 32;
    typedef float vread_t __attribute__((ext_vector_type(kDb)));
    const uint8_t *lane0 = vb + grp * 4 * (4 * D) + col * (4 * kDb);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const vread_t v = *reinterpret_cast<const vread_t *>(lane0 + ((r / 4) * 8 + r % 4) * (4 * D));
#pragma unroll
        for (int db = 0; db < kDb; ++db) w.o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[db], p[r], w.o[db], 0, 0, 0);
    }
}

// A tile's valid keys.
template <bool kMask>
__device__ __forceinline__ uint64_t tile_keys(const CrossKArgs &a, int b, int32_t key0, int32_t n, int lane) {
    if constexpr (kMask) return key_bits(a, b, key0, n, lane) & 0xffffffffull;
    const int32_t left = n - key0;
    return left >= kKeys ? 0xffffffffull : left <= 0 ? 0ull : (1ull << left) - 1;
}

// Many rows: 4 waves, 128 rows, shared double-buffered tiles.
constexpr int kTileWaves = kCrossTileRows / 32;

template <int D, bool kMask>
__global__ __launch_bounds__(64 * kTileWaves) __attribute__((amdgpu_waves_per_eu(2)))
void cross_f32_tile_kernel(const CrossKArgs a) {
    using L = Tile<D>;
    constexpr int kN = L::kLoads / kTileWaves;
    __shared__ __attribute__((aligned(1024))) uint8_t kb[2][L::kBytes];
    __shared__ __attribute__((aligned(1024))) uint8_t vb[2][L::kBytes];
    CrossTile t;
    if (!cross_tile<kCrossTileRows>(a, blockIdx.x, t)) return;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, grp = lane >> 5;
    const uint32_t row = t.row0 + wave * 32 + col;
    const int32_t n = key_count(a, given_count(a, t.b));
    const float *kh = static_cast<const float *>(a.k) + t.b * a.ks[0] + t.hk * a.ks[2];
    const float *vh = static_cast<const float *>(a.v) + t.b * a.vs[0] + t.hk * a.vs[2];
    auto load = [&](int32_t i, uint64_t bits, int buf) {
        issue<D, kMask, true, kN>(kh, a.ks[1], i * kKeys, n - i * kKeys, bits, kb[buf], wave * kN, lane);
        issue<D, kMask, false, kN>(vh, a.vs[1], i * kKeys, n - i * kKeys, bits, vb[buf], wave * kN, lane);
    };
    Wave<D> w;
    const int32_t tiles = static_cast<int32_t>((static_cast<int64_t>(n) + kKeys - 1) / kKeys);
    auto tile_bits = [&](int32_t i) { return tile_keys<kMask>(a, t.b, i * kKeys, n, lane); };
    uint64_t cur = 0, nxt = 0;
    if (tiles > 0) {
        cur = tile_bits(0);
        load(0, cur, 0);
        nxt = tile_bits(1);
    }
    start<D>(a, t, row, grp, w);
    for (int32_t i = 0; i < tiles; ++i) {
        wait_loads<0>();   // this wave's loads have reached LDS
        __syncthreads();   // and everybody's; the other buffer is read
        uint64_t next = 0;
        if (i + 1 < tiles) {
            load(i + 1, nxt, (i + 1) & 1);
            next = tile_bits(i + 2);
        }
        if (!kMask || cur != 0) {
            f32x16_t s = scores<D>(kb[i & 1], col, grp, w.qf);
            softmax<D>(w, s, static_cast<uint32_t>(cur), grp, a.scale_log2);
            values<D>(w, vb[i & 1], s, col, grp);
        }
        cur = nxt;
        nxt = next;
    }
    if (row >= a.rows) return;
    const float l = halves_sum(w.l), inv = l == 0.0f ? 0.0f : 1.0f / l;
    constexpr int kDb = D / 32;
    typedef float vread_t __attribute__((ext_vector_type(kDb)));
    float *op = static_cast<float *>(a.out) + row_offset(a, a.os, t, row);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        vread_t x;
#pragma unroll
        for (int db = 0; db < kDb; ++db) x[db] = w.o[db][r] * inv;
        *reinterpret_cast<vread_t *>(op + ((r / 4) * 8 + grp * 4 + r % 4) * kDb) = x;
    }
}

// Few rows: 32 rows, the keys of a part shared out among the waves, merged through LDS.
template <int D> constexpr int kWaves = cross_few_waves(D, RF_F32);

template <int D, bool kMask>
__global__ __launch_bounds__(64 * kWaves<D>) __attribute__((amdgpu_waves_per_eu(kWaves<D> / 4)))
void cross_f32_few_kernel(const CrossKArgs a) {
    using L = Tile<D>;
    constexpr int kW = kWaves<D>, kDb = D / 32, kN = L::kLoads;
    typedef float vread_t __attribute__((ext_vector_type(kDb)));
    __shared__ __attribute__((aligned(1024))) uint8_t ks[kW * L::kBytes];
    __shared__ __attribute__((aligned(1024))) uint8_t vs[kW * L::kBytes];
    __shared__ float ml[kW][kCrossFewRows][2];
    const int part = blockIdx.x % a.parts;
    CrossTile t;
    if (!cross_tile<kCrossFewRows>(a, blockIdx.x / a.parts, t)) return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, grp = lane >> 5;
    const int32_t n = key_count(a, given_count(a, t.b));
    const float *kh = static_cast<const float *>(a.k) + t.b * a.ks[0] + t.hk * a.ks[2];
    const float *vh = static_cast<const float *>(a.v) + t.b * a.vs[0] + t.hk * a.vs[2];
    uint8_t *kb = ks + wave * L::kBytes, *vb = vs + wave * L::kBytes;
    const int64_t tiles = (static_cast<int64_t>(n) + kKeys - 1) / kKeys;
    const int64_t first = part * kW + wave, step = static_cast<int64_t>(a.parts) * kW;
    auto tile_bits = [&](int64_t i) { return tile_keys<kMask>(a, t.b, static_cast<int32_t>(i) * kKeys, n, lane); };
    Wave<D> w;
    uint64_t cur = 0;
    if (first < tiles) {
        const int32_t key0 = static_cast<int32_t>(first) * kKeys;
        cur = tile_bits(first);
        issue<D, kMask, true, kN>(kh, a.ks[1], key0, n - key0, cur, kb, 0, lane);
        issue<D, kMask, false, kN>(vh, a.vs[1], key0, n - key0, cur, vb, 0, lane);
    }
    start<D>(a, t, t.row0 + col, grp, w);
    if (first < tiles) {
        wait_loads<0>();
        for (int64_t i = first; i < tiles; i += step) {
            // (past the last tile it is fetched again and not used: with the loads on every
            // path the waits below can be counted)
            const int64_t next = i + step < tiles ? i + step : i;
            const int32_t key0 = static_cast<int32_t>(next) * kKeys;
            const uint64_t nxt = tile_bits(next);
            wait_loads<kN>();       // K is there; V may still be in flight
            f32x16_t s = scores<D>(kb, col, grp, w.qf);
            wait_lds_reads();       // K is read: its buffer is free
            issue<D, kMask, true, kN>(kh, a.ks[1], key0, n - key0, nxt, kb, 0, lane);
            softmax<D>(w, s, static_cast<uint32_t>(cur), grp, a.scale_log2);
            wait_loads<kN>();       // V is there; the next K may still be in flight
            values<D>(w, vb, s, col, grp);
            wait_lds_reads();
            issue<D, kMask, false, kN>(vh, a.vs[1], key0, n - key0, nxt, vb, 0, lane);
            cur = nxt;
        }
        wait_loads<0>();   // nothing lands in the buffers any more
    }

    // ---- merge: every wave's O rows into its own K buffer, units permuted by row % 16 ----
    const float l = halves_sum(w.l);
    if (grp == 0) {
        ml[wave][col][0] = w.m;
        ml[wave][col][1] = l;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        vread_t x;
#pragma unroll
        for (int db = 0; db < kDb; ++db) x[db] = w.o[db][r];
        const int unit = ((r / 4) * 8 + grp * 4 + r % 4) ^ (col & 15);
        *reinterpret_cast<vread_t *>(kb + col * L::kRow + unit * (4 * kDb)) = x;
    }
    __syncthreads();
    for (int u = tid; u < kCrossFewRows * 32; u += 64 * kW) {
        const int r = u / 32, unit = u % 32;
        const uint32_t row = t.row0 + r;
        if (row >= a.rows) break;
        float m = ml[0][r][0];
#pragma unroll
        for (int p = 1; p < kW; ++p) m = fmaxf(m, ml[p][r][0]);
        const float ref = m == -kInf ? 0.0f : m;
        float lsum = 0.0f;
        vread_t x = {};
#pragma unroll
        for (int p = 0; p < kW; ++p) {
            const float wgt = fast_exp2((ml[p][r][0] - ref) * a.scale_log2);
            lsum = fmaf(wgt, ml[p][r][1], lsum);
            const vread_t y =
                *reinterpret_cast<const vread_t *>(ks + p * L::kBytes + r * L::kRow + (unit ^ (r & 15)) * (4 * kDb));
#pragma unroll
            for (int db = 0; db < kDb; ++db) x[db] = fmaf(wgt, y[db], x[db]);
        }
        if (a.parts > 1) {
            const int64_t slot = (static_cast<int64_t>(t.tile) * a.parts + part) * kCrossFewRows + r;
            if (unit == 0) *reinterpret_cast<f32x2_t *>(a.ws_ml + slot * 2) = f32x2_t{m, lsum};
            *reinterpret_cast<vread_t *>(a.ws_o + slot * D + unit * kDb) = x;
            continue;
        }
        const float inv = lsum == 0.0f ? 0.0f : 1.0f / lsum;
#pragma unroll
        for (int db = 0; db < kDb; ++db) x[db] *= inv;
        *reinterpret_cast<vread_t *>(static_cast<float *>(a.out) + row_offset(a, a.os, t, row) + unit * kDb) = x;
    }
}

template <int D>
void run(const CrossKArgs &a, bool few, bool mask, dim3 grid, hipStream_t stream) {
    if (few && mask) hipLaunchKernelGGL((cross_f32_few_kernel<D, true>), grid, dim3(64 * kWaves<D>), 0, stream, a);
    else if (few) hipLaunchKernelGGL((cross_f32_few_kernel<D, false>), grid, dim3(64 * kWaves<D>), 0, stream, a);
    else if (mask) hipLaunchKernelGGL((cross_f32_tile_kernel<D, true>), grid, dim3(64 * kTileWaves), 0, stream, a);
    else hipLaunchKernelGGL((cross_f32_tile_kernel<D, false>), grid, dim3(64 * kTileWaves), 0, stream, a);
}

}  // namespace

hipError_t launch_cross_f32(const CrossKArgs &a, int32_t head_dim, bool few, uint32_t grid, hipStream_t stream) {
    if (head_dim == 128) run<128>(a, few, a.key_mask != nullptr, dim3(grid), stream);
    else run<64>(a, few, a.key_mask != nullptr, dim3(grid), stream);
    return hipGetLastError();
}

}  // namespace rf
