// Attention to an encoder's states of another length for gfx950, bf16 (the fp32
// kernels are in rf_cross_f32.hip).
//
// The method is that of keyframe-query attention, one pass over the keys with
// a running softmax; what differs is that keys are few (a prompt) and rows many,
// or rows few (a caption's next word) and keys many, that a sequence has a length
// and a mask of its own, and that tensors come with strides.
//
//  * Scores are computed transposed, S^T = K Q^T (v_mfma_f32_32x32x16_bf16): K
//    rows from LDS are the A operand, a wave's 32 query rows, in registers, the B
//    operand. A lane then holds 16 of 32 scores of ONE row (lane l and l ^ 32
//    share row l % 32), and those, rounded to bf16, are the B operand of
//    O^T = V^T P^T as they stand. V^T operands are transposing LDS reads of the
//    natural [key][dim] tile.
//  * K and V tiles go from memory straight into LDS. The buffer resource of a tile
//    ends at its last key within the sequence's length; a masked key's lanes load
//    from past the resource. Either way the row reads as zero, so what the memory
//    holds there (NaN, infinities) has no effect, and its score becomes -inf.
//  * Softmax in the log2 domain against a reference that is a past row maximum,
//    replaced when a row's probabilities of a tile sum to more than 256 (the sum
//    bounds each of them). A walk's first tile takes its own maximum. Probabilities
//    are rounded to bf16 for the second product: its operands are bf16 on the matrix
//    cores, and as sums of two bf16 they would double it. The row sum, in fp32, adds the
//    rounded ones, so their errors (2^-8 of each at most) are weighted alike: results are
//    off by 2.3e-3 of their norm, where fp32 probabilities rounded at the end give 1.7e-3.
//
// What bounds them, and what they measure:
//  * Many rows, many keys (8,000 x 4,000, 12 heads x 128: 185 us, 1,060 TFLOP/s): issue of
//    the matrix instructions and the softmax's vector instructions, as in self attention.
//  * Many rows, a prompt (21,600 x 512, 40 heads x 128: 262 to 276 us by card, 820 to 864
//    TFLOP/s; at heads of 64 157 us): the same, and each 128 rows' queries and results, 64 KB, which the
//    other workgroup of the compute unit covers in part. Tiles of 32 keys with three
//    workgroups to a compute unit at 128 (279 us where this had 267), the next queries
//    held in registers (313) or touched ahead (288), a wait that leaves them out (no
//    change) did not cover more.
//  * Short prompts (2 x 9,360 rows, 12 heads x 128, 116 MB: 37 to 42 us): memory, q in and out,
//    little of it under the matrix work (busy 19 %).
//  * One token over 20,280 keys, 4 key heads x 128: 17 us, 5.0 TB/s of K and V, and 4 of
//    the join.
#include "rf_cross.h"

namespace rf {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4_t;

constexpr float kInf = __builtin_huge_valf();
constexpr float kRebaseBound = 256.0f;

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    const bf16x2_t v = {static_cast<__bf16>(lo), static_cast<__bf16>(hi)};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ bf16x8_t as_bf16x8(u32x4_t w) { return __builtin_bit_cast(bf16x8_t, w); }
__device__ __forceinline__ float add_bf16x2(uint32_t word, float acc) {
    const bf16x2_t one = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, word), one, acc, false);
}

// An LDS tile's rows are 2 D bytes without padding (a wave's load fills 1 KB of
// them in order). The 16-byte slots of a row are permuted by the key so that the
// 16 lanes of a K read, and the 32 of a transposing V read, meet different banks.
template <int D>
struct Tile {
    static constexpr int kRow = 2 * D;
    static constexpr int kSlots = kRow / 16;
    static constexpr int kRowsPerWin = 256 / kRow;
    static constexpr int kRowsPerLoad = 1024 / kRow;
    __host__ __device__ static constexpr int kswz(int key) { return (key / kRowsPerWin) % kSlots; }
    __host__ __device__ static constexpr int vswz(int key) { return 4 * ((key / kRowsPerWin) % (kSlots / 4)); }
};

// One wave's 32 query rows, their running softmax and O^T.
template <int D>
struct Wave {
    u32x4_t qf[D / 16];
    f32x16_t o[D / 32];
    float m;      // reference: a past maximum of the raw scores, -inf before the first
    float mref;   // m in the log2 domain, rounded; what probabilities are taken against
    float l;      // this lane's part of the row sum
};

// Query fragments: the B operand of S^T = K Q^T. Rows past the last read the last one
// (nothing is stored for them).
template <int D>
__device__ __forceinline__ void load_queries(const CrossKArgs &a, const CrossTile &t, uint32_t row, int grp,
                                             u32x4_t (&qf)[D / 16]) {
    const uint16_t *qp = static_cast<const uint16_t *>(a.q) +
                         row_offset(a, a.qs, t, row < a.rows ? row : a.rows - 1) + grp * 8;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) qf[kk] = *reinterpret_cast<const u32x4_t *>(qp + kk * 16);
}

template <int D>
__device__ __forceinline__ void clear(Wave<D> &w) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) w.o[db][r] = 0.0f;
    w.m = w.mref = -kInf;
    w.l = 0.0f;
}

// LDS offsets of a lane's K fragments (block 0) and of its V^T operand halves.
template <int D>
struct Fragments {
    int k[D / 16], v[D / 32];
    __device__ __forceinline__ explicit Fragments(int lane) {
        using L = Tile<D>;
        const int col = lane & 31, grp = lane >> 5;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) k[kk] = col * L::kRow + (((2 * kk) ^ grp ^ L::kswz(col)) * 16);
        const int g16 = (lane >> 4) & 1, j = lane & 15;
        const int rr = grp * 4 + j / 4;
#pragma unroll
        for (int db = 0; db < D / 32; ++db) v[db] = rr * L::kRow + (((2 * db + g16) ^ (L::vswz(rr) / 2)) * 32) + 8 * (j % 4);
    }
};

// S^T of kNB blocks of 32 keys; fragments are read four ahead of the matrix core.
template <int D, int kNB>
__device__ __forceinline__ void scores(const uint8_t *kb, const Fragments<D> &f, const u32x4_t (&qf)[D / 16],
                                       f32x16_t (&s)[kNB]) {
    constexpr int kSteps = D / 16, kNF = kNB * kSteps, kLead = 4;
    u32x4_t ring[kLead];
    auto rd = [&](int i) {
        return *reinterpret_cast<const u32x4_t *>(kb + f.k[i % kSteps] + (i / kSteps) * 32 * Tile<D>::kRow);
    };
#pragma unroll
    for (int i = 0; i < kLead; ++i) ring[i] = rd(i);
#pragma unroll
    for (int i = 0; i < kNF; ++i) {
        const int b = i / kSteps, kk = i % kSteps;
        const f32x16_t c = kk == 0 ? f32x16_t{} : s[b];
        s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(ring[i % kLead]), as_bf16x8(qf[kk]), c, 0, 0, 0);
        if (i + kLead < kNF) ring[i % kLead] = rd(i + kLead);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, kLead, 0);
#pragma unroll
    for (int i = 0; i < kNF - kLead; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, kLead, 0);
}

// O^T += V^T P^T of kNB blocks; operands are read three ahead.
template <int D, int kNB>
__device__ __forceinline__ void values(const uint8_t *vb, const Fragments<D> &f, const u32x4_t (&pw)[2 * kNB],
                                       f32x16_t (&o)[D / 32]) {
    constexpr int kNF = 2 * kNB * (D / 32), kLead = 3, kRow = Tile<D>::kRow;
    u32x4_t ring[kLead];
    auto rd = [&](int i) {
        const uint8_t *p = vb + f.v[i % (D / 32)] + (i / (D / 32)) * 16 * kRow;
        const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t *)p);
        const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t *)(p + 8 * kRow));
        return __builtin_shufflevector(__builtin_bit_cast(u32x2_t, lo), __builtin_bit_cast(u32x2_t, hi), 0, 1, 2, 3);
    };
#pragma unroll
    for (int i = 0; i < kLead; ++i) ring[i] = rd(i);
#pragma unroll
    for (int i = 0; i < kNF; ++i) {
        const int c = i / (D / 32), db = i % (D / 32);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(ring[i % kLead]), as_bf16x8(pw[c]), o[db], 0, 0, 0);
        if (i + kLead < kNF) ring[i % kLead] = rd(i + kLead);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 2 * kLead, 0);
#pragma unroll
    for (int i = 0; i < kNF - kLead; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, kLead, 0);
}

// A reference so large that the rounding of its log2 form (2^-24 of it) would
// show in a probability: then (s - m) * scale is formed instead.
constexpr float kFarReference = 4096.0f;

// Scores of keys that are not valid become -inf. `bits`: the tile's valid keys.
template <int kNB>
__device__ __forceinline__ void mask_scores(f32x16_t (&s)[kNB], uint64_t bits, int grp) {
    static_assert(kNB <= 2, "a tile's keys fit a word");
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
        const uint32_t word = static_cast<uint32_t>(bits >> (32 * b));
        const uint32_t mine = word >> (4 * grp);   // accumulator r holds key (r/4)*8 + grp*4 + r%4
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (!((mine >> ((r / 4) * 8 + r % 4)) & 1u)) s[b][r] = -kInf;
    }
}

// Probabilities of kNB blocks of 32 keys, packed as the B operand of the second
// product, and the running softmax.
template <int D, int kNB>
__device__ __forceinline__ void softmax(Wave<D> &w, f32x16_t (&s)[kNB], float sl2, bool first, u32x4_t (&pw)[2 * kNB]) {
    auto probs = [&](float m, float mref) {
        // four partial sums, of the rounded values that the matrix cores take
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        const bool far = __builtin_amdgcn_ballot_w64(fabsf(mref) > kFarReference && fabsf(mref) < kInf) != 0;
        auto body = [&](auto arg) {
#pragma unroll
            for (int b = 0; b < kNB; ++b)
#pragma unroll
                for (int r = 0; r < 16; r += 2) {
                    const uint32_t word = pack_bf16x2(fast_exp2(arg(s[b][r])), fast_exp2(arg(s[b][r + 1])));
                    sum[(r / 2) % 4] = add_bf16x2(word, sum[(r / 2) % 4]);
                    pw[b * 2 + r / 8][(r % 8) / 2] = word;
                }
        };
        if (far) {
            const bool mine = fabsf(mref) > kFarReference;
            body([&](float x) { return mine ? (x - m) * sl2 : fmaf(x, sl2, -mref); });
        } else {
            body([&](float x) { return fmaf(x, sl2, -mref); });
        }
        return (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };
    float ls = 0.0f;
    bool need = first;
    if (!first) {
        // (before any score is met mref is -inf: the sum is then inf or NaN)
        ls = probs(w.m, w.mref);
        need = !(halves_sum(ls) <= kRebaseBound);
    }
    if (need) {   // both lanes of a row take it
        float mx = -kInf;
#pragma unroll
        for (int b = 0; b < kNB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[b][r]);
        const float m = fmaxf(w.m, halves_max(mx)), mref = m * sl2;
        const bool far = fabsf(w.mref) > kFarReference || fabsf(mref) > kFarReference;
        const float corr = w.m == -kInf ? 0.0f : fast_exp2(far ? (w.m - m) * sl2 : w.mref - mref);
        w.m = m;
        w.mref = mref;
        w.l *= corr;
        if (!first) {
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) w.o[db][r] *= corr;
        }
        // rows without any score above -inf so far: against 0 every probability is 0
        ls = probs(m == -kInf ? 0.0f : m, m == -kInf ? 0.0f : mref);
    }
    w.l += ls;
}

// This wave's global->LDS loads i0 .. i0 + kN - 1 of a tile (each fills 1 KB). `key`: the
// tile's first key; `left`: the sequence's keys from there on, at which the resource ends.
// bits: the valid keys, taken for masked launches only.
template <int D, bool kMask, int kBc, int kN>
__device__ __forceinline__ void issue(const uint16_t *key, int64_t stride, int32_t left, uint64_t bits,
                                      uint8_t *dst, int i0, const int (&go)[kN], int lane) {
    // (a tile spans less than 2^31 bytes)
    const int32_t rec = __builtin_amdgcn_readfirstlane(
        left >= kBc ? kNowhere : (left - 1) * static_cast<int32_t>(stride) * 2 + 2 * D);
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(uniform_ptr(key), 0, rec, kBufferWord3);
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        int at = go[i];
        if constexpr (kMask) {
            const int k = (i0 + i) * Tile<D>::kRowsPerLoad + lane / Tile<D>::kSlots;
            if (!((bits >> k) & 1)) at = kNowhere;
        }
        load_lds16(r, (lds_void_t *)(dst + (i0 + i) * 1024), at);
    }
}

template <int D, bool kKey, int kN>
__device__ __forceinline__ void load_offsets(int64_t stride, int i0, int lane, int (&go)[kN]) {
    using L = Tile<D>;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        const int key = (i0 + i) * L::kRowsPerLoad + lane / L::kSlots, slot = lane % L::kSlots;
        go[i] = static_cast<int>(key * stride * 2) + (slot ^ (kKey ? L::kswz(key) : L::vswz(key))) * 16;
    }
}

// ---------------------------------------------------------------------------
// Many rows: a workgroup of 4 waves owns 128 rows of one key head at a time; its
// waves share double-buffered tiles of 64 keys (64 KB of LDS at head dimension 128, 32
// at 64), one barrier a tile; two workgroups to a compute unit, three at 64 without mask.
// A prompt is a few tiles long, so the time between two tiles of rows counts: a
// workgroup walks a run of tiles of rows, and under the last tile of keys of one
// the first keys and values of the next are on their way, its queries from where the
// last scores are done.
// ---------------------------------------------------------------------------

constexpr int kTileWaves = kCrossTileRows / 32;

template <int D, bool kMask>
__global__ __launch_bounds__(64 * kTileWaves) __attribute__((amdgpu_waves_per_eu(cross_tile_waves(D, kMask))))
void cross_tile_kernel(const CrossKArgs a) {
    constexpr int kBc = kCrossTileKeys, kNB = kBc / 32, kTileBytes = kBc * Tile<D>::kRow;
    constexpr int kN = kTileBytes / 1024 / kTileWaves;
    // [K, V][buffer]
    __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * kTileBytes];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, grp = lane >> 5;
    int32_t tile, end;
    {
        // An XCD's walkers have neighbouring runs, alike to one tile; the first ones, which go to
        // a compute unit each, have the longer (fewer walkers, of runs alike, where tiles do not
        // share out evenly: 224 against 188 us at 8,000 x 4,000 keys, 12 heads x 128, 82 against
        // 75 at 2 x 9,360 x 512).
        const int32_t x = blockIdx.x % a.xcds, w = blockIdx.x / a.xcds, per = a.walkers / a.xcds;
        const int32_t x0 = static_cast<int32_t>(static_cast<int64_t>(x) * a.tiles / a.xcds);
        const int32_t n = static_cast<int32_t>(static_cast<int64_t>(x + 1) * a.tiles / a.xcds) - x0;
        const int32_t each = n / per, more = n - each * per;
        tile = x0 + w * each + (w < more ? w : more);
        end = tile + each + (w < more);
    }
    if (tile >= end) return;
    int kgo[kN], vgo[kN];
    load_offsets<D, true, kN>(a.ks[1], wave * kN, lane, kgo);
    load_offsets<D, false, kN>(a.vs[1], wave * kN, lane, vgo);
    // a sequence's keys from one on: the first of a tile
    struct Keys {
        const uint16_t *k, *v;
        int32_t key, left;
        uint64_t bits;   // masked launches: the tile's valid keys
    };
    auto keys_of = [&](const CrossTile &t, int32_t given) {
        Keys r;
        r.k = static_cast<const uint16_t *>(a.k) + t.b * a.ks[0] + t.hk * a.ks[2];
        r.v = static_cast<const uint16_t *>(a.v) + t.b * a.vs[0] + t.hk * a.vs[2];
        r.key = 0;
        r.left = key_count(a, given);
        return r;
    };
    auto load = [&](Keys &s, const CrossTile &t, int buf) {
        if constexpr (kMask) s.bits = key_bits(a, t.b, s.key, s.key + s.left, lane);
        uint8_t *kd = lds + buf * kTileBytes, *vd = lds + (2 + buf) * kTileBytes;
        issue<D, kMask, kBc, kN>(s.k, a.ks[1], s.left, s.bits, kd, wave * kN, kgo, lane);
        issue<D, kMask, kBc, kN>(s.v, a.vs[1], s.left, s.bits, vd, wave * kN, vgo, lane);
    };
    auto tile_done = [&]() {
        wait_loads<0>();   // this wave's loads have reached LDS
        __syncthreads();
    };
    const Fragments<D> f(lane);
    CrossTile t = cross_tile_at<kCrossTileRows>(a, tile);
    Keys cur = keys_of(t, given_count(a, t.b));
    Wave<D> w;
    int buf = 0;
    load_queries<D>(a, t, t.row0 + wave * 32 + col, grp, w.qf);
    if (cur.left > 0) load(cur, t, 0);
    tile_done();
    for (; tile < end; ++tile) {
        clear<D>(w);
        bool first = true;
        CrossTile tn = t;
        if (tile + 1 < end) tn = cross_tile_at<kCrossTileRows>(a, tile + 1);
        const int32_t given = given_count(a, tn.b);   // (asked for early, waited for below)
        // whole tiles of keys, each under the loads of the next one
        while (cur.left > kBc) {
            Keys next = cur;
            next.k += kBc * a.ks[1];
            next.v += kBc * a.vs[1];
            next.key += kBc;
            next.left -= kBc;
            load(next, t, buf ^ 1);
            if (!kMask || first || cur.bits != 0) {
                f32x16_t s[kNB];
                scores<D, kNB>(lds + buf * kTileBytes, f, w.qf, s);
                if constexpr (kMask) mask_scores<kNB>(s, cur.bits, grp);
                u32x4_t pw[2 * kNB];
                softmax<D, kNB>(w, s, a.scale_log2, first, pw);
                values<D, kNB>(lds + (2 + buf) * kTileBytes, f, pw, w.o);
            }
            first = false;
            cur = next;
            buf ^= 1;
            tile_done();
        }
        // the last one, whole or not (or none), under those of the next tile of rows, whose
        // queries follow as soon as this one's have met their last keys
        Keys next = cur;
        if (tile + 1 < end) {
            next = keys_of(tn, given);
            if (next.left > 0) load(next, tn, buf ^ 1);
        }
        auto turn = [&]() {
            if (tile + 1 < end) load_queries<D>(a, tn, tn.row0 + wave * 32 + col, grp, w.qf);
        };
        if (cur.left > 0) {
            f32x16_t s[kNB];
            scores<D, kNB>(lds + buf * kTileBytes, f, w.qf, s);
            turn();
            if constexpr (!kMask) cur.bits = cur.left >= kBc ? ~0ull : (1ull << cur.left) - 1;
            if (kMask || cur.left < kBc) mask_scores<kNB>(s, cur.bits, grp);
            u32x4_t pw[2 * kNB];
            softmax<D, kNB>(w, s, a.scale_log2, first, pw);
            values<D, kNB>(lds + (2 + buf) * kTileBytes, f, pw, w.o);
        } else {
            turn();
        }
        buf ^= 1;
        tile_done();
        // The result goes through this wave's part of the buffer just freed (the part that
        // only its own loads fill next) and leaves in whole rows. (Past the caches it would be
        // gone sooner, 21.9 -> 17.9 us at 9,360 x 77, 12 heads x 128, but the projection that reads
        // it next would wait for it: 73.9 -> 78.0 for the two, 151 -> 160 at 2 x 9,360 x 512.)
        // (What follows from the lane is formed here, not held in registers through the loop.)
        using L = Tile<D>;
        int ln = lane;
        asm volatile("" : "+v"(ln));
        const int cl = ln & 31, gp = ln >> 5;
        uint8_t *part[2] = {lds + (buf ^ 1) * kTileBytes + wave * kN * 1024,
                            lds + (2 + (buf ^ 1)) * kTileBytes + wave * kN * 1024};
        static_assert(kN * 1024 == 16 * L::kRow, "16 rows to each");
        const float l = halves_sum(w.l), inv = l == 0.0f ? 0.0f : 1.0f / l;
        uint8_t *to = (cl < 16 ? part[0] : part[1]) + (cl & 15) * L::kRow;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int g4 = 0; g4 < 4; g4 += 2) {
                // accumulator r holds dimension db*32 + (r/4)*8 + grp*4 + r%4: two groups of four,
                // and the half-waves trade one each, so that a lane has eight neighbours
                uint32_t lo[2], hi[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int r = g4 * 4 + 2 * x;
                    lo[x] = pack_bf16x2(w.o[db][r] * inv, w.o[db][r + 1] * inv);
                    hi[x] = pack_bf16x2(w.o[db][r + 4] * inv, w.o[db][r + 5] * inv);
                    const auto sw = __builtin_amdgcn_permlane32_swap(lo[x], hi[x], false, false);
                    lo[x] = sw[0];
                    hi[x] = sw[1];
                }
                *reinterpret_cast<u32x4_t *>(to + (((db * 4 + g4 + gp) ^ L::kswz(cl)) * 16)) =
                    u32x4_t{lo[0], lo[1], hi[0], hi[1]};
            }
        wait_lds_reads();
#pragma unroll
        for (int i = 0; i < 32 / L::kRowsPerLoad; ++i) {
            const int r = i * L::kRowsPerLoad + ln / L::kSlots, slot = ln % L::kSlots;
            const u32x4_t x = *reinterpret_cast<const u32x4_t *>(part[i * L::kRowsPerLoad / 16] + (r & 15) * L::kRow +
                                                                 ((slot ^ L::kswz(r)) * 16));
            const uint32_t row = t.row0 + wave * 32 + r;
            uint16_t *op = static_cast<uint16_t *>(a.out) + row_offset(a, a.os, t, row < a.rows ? row : 0) + slot * 8;
            if (row < a.rows) *reinterpret_cast<u32x4_t *>(op) = x;
        }
        wait_lds_reads();
        t = tn;
        cur = next;
    }
}

// ---------------------------------------------------------------------------
// Few rows: a workgroup owns 32 rows and a part of the key axis, which its 8
// waves share out (wave w of part p takes tiles 8 p + w, 8 p + w + 8 parts, ...),
// each streaming tiles into LDS of its own, without barriers; the waves' results
// are merged through LDS, the parts' by the join kernel.
// ---------------------------------------------------------------------------

constexpr int kFewWaves = cross_few_waves(64, RF_BF16);
static_assert(kFewWaves == cross_few_waves(128, RF_BF16), "one for both");

template <int D, bool kMask>
__global__ __launch_bounds__(64 * kFewWaves) __attribute__((amdgpu_waves_per_eu(2)))
void cross_few_kernel(const CrossKArgs a) {
    constexpr int kBc = cross_few_keys(D), kNB = kBc / 32, kTileBytes = kBc * Tile<D>::kRow, kN = kTileBytes / 1024;
    __shared__ __attribute__((aligned(1024))) uint8_t ks[kFewWaves * kTileBytes];
    __shared__ __attribute__((aligned(1024))) uint8_t vs[kFewWaves * kTileBytes];
    __shared__ float ml[kFewWaves][kCrossFewRows][2];
    const int part = blockIdx.x % a.parts;
    CrossTile t;
    if (!cross_tile<kCrossFewRows>(a, blockIdx.x / a.parts, t)) return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, grp = lane >> 5;
    const int32_t n = key_count(a, given_count(a, t.b));
    const uint16_t *kh = static_cast<const uint16_t *>(a.k) + t.b * a.ks[0] + t.hk * a.ks[2];
    const uint16_t *vh = static_cast<const uint16_t *>(a.v) + t.b * a.vs[0] + t.hk * a.vs[2];
    uint8_t *kb = ks + wave * kTileBytes, *vb = vs + wave * kTileBytes;
    int kgo[kN], vgo[kN];
    load_offsets<D, true, kN>(a.ks[1], 0, lane, kgo);
    load_offsets<D, false, kN>(a.vs[1], 0, lane, vgo);
    const Fragments<D> f(lane);
    const int64_t tiles = (static_cast<int64_t>(n) + kBc - 1) / kBc;
    const int64_t first = part * kFewWaves + wave, step = static_cast<int64_t>(a.parts) * kFewWaves;
    uint64_t cur = 0, nxt;
    auto tile_bits = [&](int32_t key0) -> uint64_t {
        if constexpr (kMask) return key_bits(a, t.b, key0, n, lane);
        else return n - key0 >= 64 ? ~0ull : (1ull << (n - key0)) - 1;
    };
    auto load = [&](bool key, int32_t key0, uint64_t bits) {
        if (key) issue<D, kMask, kBc, kN>(kh + key0 * a.ks[1], a.ks[1], n - key0, bits, kb, 0, kgo, lane);
        else issue<D, kMask, kBc, kN>(vh + key0 * a.vs[1], a.vs[1], n - key0, bits, vb, 0, vgo, lane);
    };
    Wave<D> w;
    if (first < tiles) {
        const int32_t key0 = static_cast<int32_t>(first) * kBc;
        cur = tile_bits(key0);
        load(true, key0, cur);
        load(false, key0, cur);
    }
    load_queries<D>(a, t, t.row0 + col, grp, w.qf);
    clear<D>(w);
    if (first < tiles) {
        wait_loads<0>();
        for (int64_t i = first; i < tiles; i += step) {
            // (past the last tile it is fetched again and not used: with the loads on every
            // path the waits below can be counted)
            const int64_t next = i + step < tiles ? i + step : i;
            const int32_t key0 = static_cast<int32_t>(next) * kBc;
            nxt = tile_bits(key0);
            wait_loads<kN>();       // K is there; V may still be in flight
            f32x16_t s[kNB];
            scores<D, kNB>(kb, f, w.qf, s);
            wait_lds_reads();       // K is read: its buffer is free
            load(true, key0, nxt);
            if (kMask || n - static_cast<int32_t>(i) * kBc < kBc) mask_scores<kNB>(s, cur, grp);
            u32x4_t pw[2 * kNB];
            softmax<D, kNB>(w, s, a.scale_log2, i == first, pw);
            wait_loads<kN>();       // V is there; the next K may still be in flight
            values<D, kNB>(vb, f, pw, w.o);
            wait_lds_reads();
            load(false, key0, nxt);
            cur = nxt;
        }
        wait_loads<0>();   // nothing lands in the buffers any more
    }

    // ---- merge: dimensions 0..63 of a wave's O rows go into its own K buffer, 64..127
    // into its V buffer, 256 bytes a row, their 16-byte units permuted by row % 16 ----
    const float l = halves_sum(w.l);
    if (grp == 0) {
        ml[wave][col][0] = w.m;
        ml[wave][col][1] = l;
    }
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4) {
            const int unit = ((db % 2) * 8 + g4 * 2 + grp) ^ (col & 15);
            *reinterpret_cast<f32x4_t *>((db < 2 ? kb : vb) + col * 256 + unit * 16) =
                f32x4_t{w.o[db][g4 * 4], w.o[db][g4 * 4 + 1], w.o[db][g4 * 4 + 2], w.o[db][g4 * 4 + 3]};
        }
    __syncthreads();
    const int r = tid / 16, unit = tid % 16;   // 512 threads: 32 rows x 16 units
    const uint32_t row = t.row0 + r;
    if (row >= a.rows) return;
    float m = ml[0][r][0];
#pragma unroll
    for (int p = 1; p < kFewWaves; ++p) m = fmaxf(m, ml[p][r][0]);
    const float ref = m == -kInf ? 0.0f : m;
    float wgt[kFewWaves], lsum = 0.0f;
#pragma unroll
    for (int p = 0; p < kFewWaves; ++p) {
        wgt[p] = fast_exp2((ml[p][r][0] - ref) * a.scale_log2);
        lsum = fmaf(wgt[p], ml[p][r][1], lsum);
    }
    const int64_t slot = (static_cast<int64_t>(t.tile) * a.parts + part) * kCrossFewRows + r;
    const float inv = a.parts > 1 ? 1.0f : lsum == 0.0f ? 0.0f : 1.0f / lsum;
    if (a.parts > 1 && unit == 0) *reinterpret_cast<f32x2_t *>(a.ws_ml + slot * 2) = f32x2_t{m, lsum};
    uint16_t *op = static_cast<uint16_t *>(a.out) + row_offset(a, a.os, t, row) + unit * 4;
#pragma unroll
    for (int half = 0; half < D / 64; ++half) {
        f32x4_t x = {};
#pragma unroll
        for (int p = 0; p < kFewWaves; ++p) {
            const f32x4_t y = *reinterpret_cast<const f32x4_t *>((half == 0 ? ks : vs) + p * kTileBytes + r * 256 +
                                                                 (unit ^ (r & 15)) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = fmaf(wgt[p], y[e], x[e]);
        }
        if (a.parts > 1) {
            *reinterpret_cast<f32x4_t *>(a.ws_o + slot * D + half * 64 + unit * 4) = x;
        } else {
            const u32x2_t y = {pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv)};
            *reinterpret_cast<u32x2_t *>(op + half * 64) = y;
        }
    }
}

// ---------------------------------------------------------------------------
// Join of a split key axis: for each row the parts' references m_p (raw scores),
// sums l_p and unnormalised outputs O_p give, with w_p = 2^((m_p - max m) scale),
// sum w_p O_p / sum w_p l_p. A workgroup owns a row: thread (p, c) takes four
// dimensions of parts p, p + 256 / (D/4), ..., all loaded before their weights are
// known; its sums meet in LDS in a fixed order.
// ---------------------------------------------------------------------------

template <int D, typename E>
__global__ __launch_bounds__(256) void cross_join_kernel(const CrossKArgs a) {
    constexpr int kCols = D / 4, kGroups = 256 / kCols, kEach = (kCrossMaxParts + kGroups - 1) / kGroups;
    __shared__ float ml[kCrossMaxParts][2];
    __shared__ __attribute__((aligned(16))) float sums[kGroups][D];
    const CrossTile t = cross_tile_at<kCrossFewRows>(a, blockIdx.x / kCrossFewRows);
    const int r = blockIdx.x % kCrossFewRows, tid = threadIdx.x;
    if (t.row0 + r >= a.rows) return;
    const int64_t slot0 = static_cast<int64_t>(t.tile) * a.parts * kCrossFewRows + r;
    const int g = tid / kCols, c = tid % kCols;
    f32x4_t x[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int p = g + i * kGroups;
        x[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        if (p < a.parts)
            x[i] = *reinterpret_cast<const f32x4_t *>(a.ws_o + (slot0 + static_cast<int64_t>(p) * kCrossFewRows) * D + c * 4);
    }
    if (tid < a.parts) {
        const f32x2_t y = *reinterpret_cast<const f32x2_t *>(a.ws_ml + (slot0 + static_cast<int64_t>(tid) * kCrossFewRows) * 2);
        ml[tid][0] = y[0];
        ml[tid][1] = y[1];
    }
    __syncthreads();
    float m = ml[0][0];
    for (int p = 1; p < a.parts; ++p) m = fmaxf(m, ml[p][0]);
    const float ref = m == -kInf ? 0.0f : m;
    float l = 0.0f;
    for (int p = 0; p < a.parts; ++p) l = fmaf(fast_exp2((ml[p][0] - ref) * a.scale_log2), ml[p][1], l);
    f32x4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int p = g + i * kGroups;
        if (p >= a.parts) break;
        const float wgt = fast_exp2((ml[p][0] - ref) * a.scale_log2);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(wgt, x[i][e], o[e]);
    }
    *reinterpret_cast<f32x4_t *>(&sums[g][c * 4]) = o;
    __syncthreads();
    if (tid >= D / 2) return;
    float v[2] = {0.0f, 0.0f};
#pragma unroll
    for (int p = 0; p < kGroups; ++p) {
        v[0] += sums[p][2 * tid];
        v[1] += sums[p][2 * tid + 1];
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    E *op = static_cast<E *>(a.out) + row_offset(a, a.os, t, t.row0 + r) + 2 * tid;
    if constexpr (sizeof(E) == 4) *reinterpret_cast<f32x2_t *>(op) = f32x2_t{v[0] * inv, v[1] * inv};
    else *reinterpret_cast<uint32_t *>(op) = pack_bf16x2(v[0] * inv, v[1] * inv);
}

}  // namespace

int64_t cross_workspace(int32_t B, int32_t Lq, int32_t Lk, int32_t heads, int32_t kv_heads, int32_t head_dim,
                        int32_t dtype, int32_t cus) {
    int64_t bytes = 0;   // (masked or not: room for either)
    for (const bool mask : {false, true}) {
        const CrossPlan c = cross_plan(B, static_cast<int64_t>(heads / kv_heads) * Lq, kv_heads, Lk, head_dim, dtype,
                                       mask, true, cus);
        const int64_t need = c.parts > 1 ? c.tiles * c.parts * kCrossFewRows * (static_cast<int64_t>(head_dim) * 4 + 8) : 0;
        bytes = need > bytes ? need : bytes;
    }
    return bytes;
}

hipError_t launch_cross(const CrossParams &p, hipStream_t stream) {
    const int32_t xcds = p.geo.xcds;
    if (p.geo.cus < 1 || xcds < 1 || xcds > 64) return hipErrorInvalidValue;
    CrossKArgs a{};
    a.q = p.q;
    a.k = p.k;
    a.v = p.v;
    a.out = p.out;
    a.kv_lengths = p.kv_lengths;
    a.key_mask = p.key_mask;
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = p.qs[i];
        a.ks[i] = p.ks[i];
        a.vs[i] = p.vs[i];
        a.os[i] = p.os[i];
    }
    a.Lq = p.Lq;
    a.Lk = p.Lk;
    a.B = p.B;
    a.group = p.heads / p.kv_heads;
    a.rows = static_cast<uint32_t>(a.group) * static_cast<uint32_t>(p.Lq);   // (2^29 at most: the tiles' limit)
    a.scale_log2 = static_cast<float>(1.4426950408889634 / sqrt(static_cast<double>(p.head_dim)));
    a.xcds = xcds;
    const CrossPlan c = cross_plan(p.B, a.rows, p.kv_heads, p.Lk, p.head_dim, p.dtype, p.key_mask != nullptr,
                                   p.ws != nullptr, p.geo.cus);
    a.parts = c.parts;
    const int64_t rows = c.few ? kCrossFewRows : kCrossTileRows;
    if (c.tiles > 0x7fffffffLL / 64) return hipErrorInvalidConfiguration;
    a.q_tiles = static_cast<int32_t>((a.rows + rows - 1) / rows);
    a.tiles = static_cast<int32_t>(c.tiles);
    a.per_xcd = (a.tiles + xcds - 1) / xcds;
    int64_t grid = static_cast<int64_t>(a.per_xcd) * xcds * c.parts;
    if (!c.few && p.dtype == RF_BF16) {
        // as many walkers as are resident, or one to a tile, in whole XCDs
        const int64_t resident = cross_tile_waves(p.head_dim, p.key_mask != nullptr) * static_cast<int64_t>(p.geo.cus);
        const int64_t want = a.tiles < resident ? a.tiles : resident;
        grid = (want + xcds - 1) / xcds * xcds;
        a.walkers = static_cast<int32_t>(grid);
    }
    if (grid > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    if (c.parts > 1) {
        a.ws_o = static_cast<float *>(p.ws);
        a.ws_ml = a.ws_o + c.tiles * c.parts * kCrossFewRows * p.head_dim;
    }
    const dim3 g(static_cast<uint32_t>(grid)), block(64 * (c.few ? kFewWaves : kTileWaves));
    const bool mask = p.key_mask != nullptr;
    if (p.dtype == RF_F32) {
        const hipError_t e = launch_cross_f32(a, p.head_dim, c.few, static_cast<uint32_t>(grid), stream);
        if (e != hipSuccess) return e;
    } else if (p.head_dim == 128) {
        if (c.few && mask) hipLaunchKernelGGL((cross_few_kernel<128, true>), g, block, 0, stream, a);
        else if (c.few) hipLaunchKernelGGL((cross_few_kernel<128, false>), g, block, 0, stream, a);
        else if (mask) hipLaunchKernelGGL((cross_tile_kernel<128, true>), g, block, 0, stream, a);
        else hipLaunchKernelGGL((cross_tile_kernel<128, false>), g, block, 0, stream, a);
    } else {
        if (c.few && mask) hipLaunchKernelGGL((cross_few_kernel<64, true>), g, block, 0, stream, a);
        else if (c.few) hipLaunchKernelGGL((cross_few_kernel<64, false>), g, block, 0, stream, a);
        else if (mask) hipLaunchKernelGGL((cross_tile_kernel<64, true>), g, block, 0, stream, a);
        else hipLaunchKernelGGL((cross_tile_kernel<64, false>), g, block, 0, stream, a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || c.parts == 1) return e;
    const dim3 jg(static_cast<uint32_t>(c.tiles * kCrossFewRows));
    if (p.dtype == RF_F32 && p.head_dim == 128)
        hipLaunchKernelGGL((cross_join_kernel<128, float>), jg, dim3(256), 0, stream, a);
    else if (p.dtype == RF_F32) hipLaunchKernelGGL((cross_join_kernel<64, float>), jg, dim3(256), 0, stream, a);
    else if (p.head_dim == 128) hipLaunchKernelGGL((cross_join_kernel<128, uint16_t>), jg, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((cross_join_kernel<64, uint16_t>), jg, dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace rf
