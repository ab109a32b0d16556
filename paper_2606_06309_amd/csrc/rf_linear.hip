// Matrix product with bias, activation, gate and residual in its epilogue for
// gfx950: y = residual + gate * act(x W^T + bias), on the rows of listed frames.
//
// x and W both hold their reduction index contiguously, so a 16-byte piece of a
// row of either is a lane's operand of a matrix instruction as it stands. Both
// types work in the same bytes: a step is 128 bytes of every row, 64 bf16 or 32
// fp32, and a pair of 16-byte pieces feeds one 32x32x16 bf16 instruction or four
// 32x32x2 fp32 ones (whose two half-waves then hold reduction indices that are four
// apart; both operands agree on it, and a sum's order is free).
//
// W's rows are the A operand, x's rows the B operand: a lane then holds one row
// of y and runs of four features.
//
//  * linear_tile_kernel: a workgroup owns kBM rows x kBN features, 8 or 4 waves of
//    32 kRB x 64: (bf16) 256 x 256, 128 x 128 and 64 x 128, and 32 x 256 and (bf16) 64 x
//    256 where rows are few and W large. Steps go from memory straight into LDS,
//    double-buffered, one barrier a step. Rows of 128 bytes are stored without
//    padding, their eight 16-byte slots permuted by (row / 2) % 8, so the 16 lanes of
//    a read pass meet 16 different slots of the 256-byte bank window.
//  * linear_few_kernel: up to 64 rows of a small W, where reading W is all that
//    costs: a workgroup owns 16 or 32 features, its 8 waves share out the reduction
//    index, operands go straight to registers, and the waves' sums meet in LDS.
//  * A reduction index may also be split over workgroups, whose fp32 parts go to the
//    workspace; linear_join_kernel adds them in order and runs the epilogue.
//
// What bounds them, and what they measure:
//  * Large bf16 products (21,600 x 20,480 x 5,120 with gate and residual: 3.79 to 3.94 ms by
//    card, 1,150 to 1,197 TFLOP/s): matrix instructions are busy 64 to 66 % of the cycles. Per step a
//    256 x 256 tile reads 192 KB of LDS while 64 KB of loads are written into it; the
//    same loop without the loads runs at 1,570. Four waves of 128 x 128 (1,225 TFLOP/s
//    where this had 1,323), a ring of four half steps (1,218) and loads between the
//    matrix instructions (1,248) were slower.
//  * One round of tiles (9,360 x 1,536 x 1,536: 45 us, 47 with rows read at full positions, 52
//    to 54 with gate and residual): 24
//    steps of 1.55 us, the first loads and the epilogue's memory time.
//  * fp32 (7,800 x 1,536 x 1,536: 280 us, 131 TFLOP/s): the matrix instructions, busy 82 %.
//  * Few rows (6 x 1,536 x 9,216: 10.0 us, 2.9 TB/s): 576 workgroups in two rounds and a
//    quarter, each with loads that wait for one another and the waves' sums. A library's
//    product without epilogue takes 6.5: this is not the least that it can take.
#include "rf_device.h"
#include "rf_linear_plan.h"

namespace rf {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kStep = kLinearStep;

struct LinearKArgs {
    const uint8_t *x, *w;
    const void *bias, *gate, *residual;
    void *y;
    float *ws;                 // parts > 1: [part][rows][n_out]
    int64_t row_bytes;         // of x and W
    uint32_t rows, N;          // N: rows per frame
    int32_t n_out;
    int32_t steps;             // of the whole reduction
    int32_t steps_per_part, parts;
    int32_t row_tiles, col_tiles, tiles, per_xcd, xcds;
    int32_t activation, gate_rows;
    int32_t stream;            // 256-row tiles: y goes past the caches
    RowFrames frames;
};

// What lanes past the end of a row load.
__device__ const u32x4_t kZeros = {0u, 0u, 0u, 0u};

// 16 bytes per lane from memory straight into LDS: lane l's bytes land at dst + 16 l.
// (Kept out of the kernel templates: the host pass drops the launch stub of a
// template that names this builtin.)
__device__ __forceinline__ void global_lds16(const uint8_t *p, uint8_t *dst) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)p, (lds_void_t *)dst, 16, 0, 0);
}

// The same from a buffer resource; an offset of -1 reads as zero.
__device__ __forceinline__ void buffer_lds16(__amdgpu_buffer_rsrc_t r, uint8_t *dst, int voffset, int soffset) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t *)dst, 16, voffset, soffset, 0, 0);
}

__device__ __forceinline__ u32x4_t buffer_load16(__amdgpu_buffer_rsrc_t r, int voffset, int soffset) {
    return __builtin_amdgcn_raw_buffer_load_b128(r, voffset, soffset, 0);
}

template <typename E>
__device__ __forceinline__ f32x16_t mma32(u32x4_t a, u32x4_t b, f32x16_t c) {
    if constexpr (sizeof(E) == 2) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b),
                                                       c, 0, 0, 0);
    } else {
        const f32x4_t fa = __builtin_bit_cast(f32x4_t, a), fb = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[e], fb[e], c, 0, 0, 0);
        return c;
    }
}
template <typename E>
__device__ __forceinline__ f32x4_t mma16(u32x4_t a, u32x4_t b, f32x4_t c) {
    if constexpr (sizeof(E) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b),
                                                       c, 0, 0, 0);
    } else {
        const f32x4_t fa = __builtin_bit_cast(f32x4_t, a), fb = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[e], fb[e], c, 0, 0, 0);
        return c;
    }
}

// kN (4 or 8) consecutive elements, widened / rounded once to nearest even.
template <typename E, int kN>
__device__ __forceinline__ void load_n(const void *p, int64_t at, float (&v)[kN]) {
    if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < kN; i += 4) {
            const f32x4_t x = *reinterpret_cast<const f32x4_t *>(static_cast<const float *>(p) + at + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i + e] = x[e];
        }
    } else {
        typedef uint32_t raw_t __attribute__((ext_vector_type(kN / 2)));
        const raw_t x = *reinterpret_cast<const raw_t *>(static_cast<const uint16_t *>(p) + at);
#pragma unroll
        for (int e = 0; e < kN / 2; ++e) {
            v[2 * e] = __uint_as_float(x[e] << 16);
            v[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u);
        }
    }
}
template <typename E, int kN>
__device__ __forceinline__ void store_n(void *p, int64_t at, const float (&v)[kN]) {
    if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < kN; i += 4)
            *reinterpret_cast<f32x4_t *>(static_cast<float *>(p) + at + i) = f32x4_t{v[i], v[i + 1], v[i + 2], v[i + 3]};
    } else {
        typedef uint32_t raw_t __attribute__((ext_vector_type(kN / 2)));
        raw_t x;
#pragma unroll
        for (int e = 0; e < kN / 2; ++e) {
            const bf16x2_t b = {static_cast<__bf16>(v[2 * e]), static_cast<__bf16>(v[2 * e + 1])};
            x[e] = __builtin_bit_cast(uint32_t, b);
        }
        *reinterpret_cast<raw_t *>(static_cast<uint16_t *>(p) + at) = x;
    }
}

// The same past the caches: for results, which are written once and as whole lines.
template <typename E>
__device__ __forceinline__ void stream_8(void *p, int64_t at, const float (&v)[8]) {
    if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < 8; i += 4)
            __builtin_nontemporal_store((f32x4_t{v[i], v[i + 1], v[i + 2], v[i + 3]}),
                                        reinterpret_cast<f32x4_t *>(static_cast<float *>(p) + at + i));
    } else {
        u32x4_t x;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bf16x2_t b = {static_cast<__bf16>(v[2 * e]), static_cast<__bf16>(v[2 * e + 1])};
            x[e] = __builtin_bit_cast(uint32_t, b);
        }
        __builtin_nontemporal_store(x, reinterpret_cast<u32x4_t *>(static_cast<uint16_t *>(p) + at));
    }
}

// x / (1 + 2^t): both sigmoid forms. 2^t = inf gives 0. (The reciprocal is the hardware's, off by one
// last place of fp32; a divide would be ten instructions, and 2^t is off by as much.)
__device__ __forceinline__ float gated(float x, float t) {
    return x * __builtin_amdgcn_rcpf(1.0f + fast_exp2(t));
}
template <int kN>
__device__ __forceinline__ void activate(int kind, float (&v)[kN]) {
    constexpr float kLog2e = 1.4426950408889634f;
    if (kind == RF_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < kN; ++e) v[e] = 0.5f * v[e] * (1.0f + erff(v[e] * 0.70710678118654752f));
    } else if (kind == RF_ACT_GELU_TANH) {
        // x/2 (1 + tanh u) = x / (1 + e^(-2u))
#pragma unroll
        for (int e = 0; e < kN; ++e)
            v[e] = gated(v[e], (-2.0f * 0.79788456080286536f * kLog2e) * (v[e] + 0.044715f * (v[e] * v[e] * v[e])));
    } else {
#pragma unroll
        for (int e = 0; e < kN; ++e) v[e] = gated(v[e], -kLog2e * v[e]);
    }
}

__device__ __forceinline__ void widen8(u32x4_t x, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(x[e] << 16);
        v[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u);
    }
}

// Bias and gate of kN neighbouring features c.., in fp32 as everything between the
// products' sums and the result's one rounding.
template <int kN>
struct Epilogue {
    float bias[kN], gate[kN];
    // frame: whose gate (-1: gate_of will say)
    template <typename E>
    __device__ __forceinline__ void load(const LinearKArgs &a, int c, int frame) {
        if (a.bias) load_n<E, kN>(a.bias, c, bias);
        if (frame >= 0) gate_of<E>(a, c, frame);
    }
    template <typename E>
    __device__ __forceinline__ void gate_of(const LinearKArgs &a, int c, int frame) {
        if (a.gate) load_n<E, kN>(a.gate, a.gate_rows ? static_cast<int64_t>(frame) * a.n_out + c : c, gate);
    }
    __device__ __forceinline__ void apply(const LinearKArgs &a, float (&v)[kN]) const {
        if (a.bias) {
#pragma unroll
            for (int e = 0; e < kN; ++e) v[e] += bias[e];
        }
        if (a.activation != RF_ACT_NONE) activate(a.activation, v);
        if (a.gate) {
#pragma unroll
            for (int e = 0; e < kN; ++e) v[e] *= gate[e];
        }
    }
};

// The epilogue of kN neighbouring features c.. of product row r: what it takes from
// memory, early, and the rest.
template <typename E, int kN>
struct Finish {
    Epilogue<kN> ep;
    float residual[kN];
    int64_t dst;
    int frame, out;
    // (the frames' loads and what depends on them apart: loads return in order, so a wait
    // for a frame is one for all loads before it)
    __device__ __forceinline__ void frames(const LinearKArgs &a, uint32_t r) {
        const uint32_t m = r / a.N;
        frame = a.frames.frame[m];
        out = a.frames.out(m);
    }
    __device__ __forceinline__ void load(const LinearKArgs &a, uint32_t r, int c) {
        dst = (static_cast<int64_t>(out) * a.N + r % a.N) * a.n_out;
        ep.template load<E>(a, c, frame);
        if (a.residual) load_n<E, kN>(a.residual, dst + c, residual);
    }
    __device__ __forceinline__ void store(const LinearKArgs &a, int c, float (&v)[kN]) const {
        ep.apply(a, v);
        if (a.residual) {
#pragma unroll
            for (int e = 0; e < kN; ++e) v[e] += residual[e];
        }
        store_n<E, kN>(a.y, dst + c, v);
    }
};
template <typename E, int kN>
__device__ __forceinline__ void finish(const LinearKArgs &a, uint32_t r, int c, float (&v)[kN]) {
    Finish<E, kN> f;
    f.frames(a, r);
    f.load(a, r, c);
    f.store(a, c, v);
}

// Product row r's (clamped to the last one) first byte in x.
__device__ __forceinline__ const uint8_t *x_row(const LinearKArgs &a, uint32_t r) {
    if (r >= a.rows) r = a.rows - 1;
    const uint32_t m = r / a.N;
    return a.x + (static_cast<int64_t>(a.frames.in(m)) * a.N + (r - m * a.N)) * a.row_bytes;
}
__device__ __forceinline__ const uint8_t *w_row(const LinearKArgs &a, int c) {
    return a.w + static_cast<int64_t>(c < a.n_out ? c : a.n_out - 1) * a.row_bytes;
}

// Workgroup id -> tile. Ids go round-robin to the XCDs: each takes a contiguous
// range of tiles, walked in bands of eight row tiles, so the workgroups that share
// an L2 at a time form a block of both operands.
constexpr int kBand = 8;
__device__ __forceinline__ bool tile_of(const LinearKArgs &a, int bid, int &rt, int &ct) {
    const int tile = (bid % a.xcds) * a.per_xcd + bid / a.xcds;
    if (tile >= a.tiles) return false;
    const int band = tile / (kBand * a.col_tiles), first = band * kBand;
    const int height = a.row_tiles - first < kBand ? a.row_tiles - first : kBand;
    const int in = tile - band * kBand * a.col_tiles;
    ct = in / height;
    rt = first + in - ct * height;
    return true;
}

// kRB blocks of 32 rows to a wave, kWR x kWC waves of (32 kRB rows x 64 features).
// kFar: rows of x may lie further than 2 GB from the tile's first (64-bit addresses).
template <typename E, int kRB, int kWR, int kWC, bool kFar>
__global__ __launch_bounds__(64 * kWR * kWC) __attribute__((amdgpu_waves_per_eu(2)))
void linear_tile_kernel(const LinearKArgs a) {
    constexpr int kWaves = kWR * kWC, kBM = 32 * kRB * kWR, kBN = 64 * kWC;
    constexpr int kXLoads = kBM / 8 / kWaves, kWLoads = kBN / 8 / kWaves;   // 8 rows each
    constexpr int kXBuf = kBM * kStep, kWBuf = kBN * kStep;
    // [W, even step][W, odd][x, even][x, odd]
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * (kXBuf + kWBuf)];
    static_assert((kXBuf & (kXBuf - 1)) == 0 && (kWBuf & (kWBuf - 1)) == 0 && kXBuf <= kWBuf,
                  "a step's parity is one bit of an LDS offset");
    int rt, ct;
    const int part = blockIdx.x % a.parts;
    if (!tile_of(a, blockIdx.x / a.parts, rt, ct)) return;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, grp = lane >> 5;
    const int wr = wave / kWC, wc = wave % kWC;

    // A load fills 8 rows: this lane's are row lane / 8 and the piece whose slot is lane % 8;
    // (row / 2) % 8 of row 8 i + sub is sub / 2, and 4 more where i is odd.
    const int sub = lane / 8, piece = (lane % 8) ^ (sub / 2);
    const uint32_t row0 = static_cast<uint32_t>(rt) * kBM;
    const int32_t rb = static_cast<int32_t>(a.row_bytes);
    const __amdgpu_buffer_rsrc_t wres = __builtin_amdgcn_make_buffer_rsrc(
        uniform_ptr(w_row(a, ct * kBN)), 0, 0x7fffffff, kBufferWord3);
    int32_t wo[kWLoads];
#pragma unroll
    for (int i = 0; i < kWLoads; ++i) {
        const int at = wave * kWLoads + i, c = at * 8 + sub, most = a.n_out - 1 - ct * kBN;
        wo[i] = (c < most ? c : most) * rb + 16 * (piece ^ ((at % 2) * 4));
    }
    // Loads of a step, W's and x's, into the buffers of its parity. The reduction's last
    // step may be short: from then on lanes past the row's end load zeros.
    const int32_t tail = rb % kStep;
    auto issue_w = [&](int step, int odd) {
        const int32_t at0 = step * kStep;
        if (tail != 0 && at0 + kStep > rb) {
#pragma unroll
            for (int i = 0; i < kWLoads; ++i)
                if (16 * (piece ^ (((wave * kWLoads + i) % 2) * 4)) >= tail) wo[i] = -1;
        }
        uint8_t *wd = lds + odd * kWBuf + wave * kWLoads * 1024;
#pragma unroll
        for (int i = 0; i < kWLoads; ++i) buffer_lds16(wres, wd + i * 1024, wo[i], at0);
    };
    const int s0 = part * a.steps_per_part;
    const int s1 = s0 + a.steps_per_part < a.steps ? s0 + a.steps_per_part : a.steps;
    issue_w(s0, 0);   // W does not wait for where x's rows are
    const uint8_t *const x0 = static_cast<const uint8_t *>(uniform_ptr(x_row(a, row0)));
    const __amdgpu_buffer_rsrc_t xres =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(x0), 0, 0x7fffffff, kBufferWord3);
    [[maybe_unused]] const uint8_t *xp[kXLoads];
    [[maybe_unused]] int32_t xo[kXLoads];
#pragma unroll
    for (int i = 0; i < kXLoads; ++i) {
        const int at = wave * kXLoads + i;
        const uint8_t *p = x_row(a, row0 + at * 8 + sub) + 16 * (piece ^ ((at % 2) * 4));
        if constexpr (kFar) xp[i] = p;
        else xo[i] = static_cast<int32_t>(p - x0);
    }
    auto issue_x = [&](int step, int odd) {
        const int32_t at0 = step * kStep;
        if (tail != 0 && at0 + kStep > rb) {
#pragma unroll
            for (int i = 0; i < kXLoads; ++i)
                if (16 * (piece ^ (((wave * kXLoads + i) % 2) * 4)) >= tail) {
                    if constexpr (kFar) xp[i] = reinterpret_cast<const uint8_t *>(&kZeros) - at0;
                    else xo[i] = -1;
                }
        }
        uint8_t *xd = lds + 2 * kWBuf + odd * kXBuf + wave * kXLoads * 1024;
#pragma unroll
        for (int i = 0; i < kXLoads; ++i) {
            if constexpr (kFar) global_lds16(xp[i] + at0, xd + i * 1024);
            else buffer_lds16(xres, xd + i * 1024, xo[i], at0);
        }
    };
    issue_x(s0, 0);
    auto issue = [&](int step, int odd) {
        issue_x(step, odd);
        issue_w(step, odd);
    };

    f32x16_t acc[2][kRB];
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int b = 0; b < kRB; ++b) acc[f][b] = f32x16_t{};
    // this lane's pieces 2 kk + grp of its row in each block
    int xat[4], wat[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
        const int at = ((2 * kk + grp) ^ ((col / 2) % 8)) * 16;
        xat[kk] = 2 * kWBuf + (wr * kRB * 32 + col) * kStep + at;
        wat[kk] = (wc * 64 + col) * kStep + at;
    }
    // Four pairs of pieces to a step; the next pair's operands are read while this one's
    // multiply, across the steps' border too: at the last pair a wave waits for its loads
    // of the next step and its reads of this one, meets the others (so the next step is
    // whole and this one's buffer free), sends for the step after the next and reads on.
    u32x4_t wf[2][2], xf[2][kRB];
    auto read = [&](int kk) {
#pragma unroll
        for (int f = 0; f < 2; ++f) wf[kk % 2][f] = *reinterpret_cast<const u32x4_t *>(lds + wat[kk] + f * 32 * kStep);
#pragma unroll
        for (int b = 0; b < kRB; ++b) xf[kk % 2][b] = *reinterpret_cast<const u32x4_t *>(lds + xat[kk] + b * 32 * kStep);
    };
    constexpr int kReads = 2 + kRB, kMma = 2 * kRB * (sizeof(E) == 2 ? 1 : 4);
    auto multiply = [&](int kk) {
#pragma unroll
        for (int b = 0; b < kRB; ++b)
#pragma unroll
            for (int f = 0; f < 2; ++f) acc[f][b] = mma32<E>(wf[kk % 2][f], xf[kk % 2][b], acc[f][b]);
    };
    // The order that the compiler keeps: one read after every kMma / kReads matrix
    // instructions (left alone it reads a pair's operands right before they multiply).
    auto interleaved = [&]() {
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, kMma / kReads, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, kMma - kMma / kReads * kReads, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    // The residual's rows come into LDS ahead of the epilogue, 32 rows x 64 features of a
    // wave at a time, 4 KB, block b in one of two places (bf16; in fp32 the products outlast
    // their latency). The buffers of the last step but one are free under the last step: the
    // first two blocks go there then, the others as their places get free. Loaded where they
    // are added, one row after the other, they cost 23 us of 69 at 9,360 x 1,536 x 1,536; a
    // block ahead within the epilogue 2 us more than so.
    constexpr bool kStage = sizeof(E) == 2;
    const bool stage = kStage && a.residual && a.parts == 1;
    const int free_odd = (s1 - s0) & 1;
    constexpr int kBlocks = kWaves * 4096;
    static_assert(kBlocks <= kWBuf && (kRB == 1 || kBlocks <= kXBuf || 2 * kBlocks <= kWBuf), "they fit");
    const int c = ct * kBN + wc * 64 + (lane % 8) * 8;
    // (a row past the last, or features past the last, load those)
    const int cs = c < a.n_out ? c : a.n_out - 8;
    auto block = [&](int b) {
        constexpr bool kBoth = 2 * kBlocks <= kWBuf;   // in W's buffer; else one in W's, one in x's
        const int at = b % 2 == 0 ? free_odd * kWBuf
                       : kBoth    ? free_odd * kWBuf + kBlocks
                                  : 2 * kWBuf + free_odd * kXBuf;
        return lds + at + wave * 4096;
    };
    auto residual = [&](int b) {
        uint8_t *to = block(b);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t r = row0 + (wr * kRB + b) * 32 + i * 8 + sub;
            if (r >= a.rows) r = a.rows - 1;
            const uint32_t m = r / a.N;
            const int64_t dst = static_cast<int64_t>(a.frames.out(m)) * a.N + (r - m * a.N);
            global_lds16(static_cast<const uint8_t *>(a.residual) + (dst * a.n_out + cs) * 2, to + i * 1024);
        }
    };
    auto residuals = [&]() {
        residual(0);
        if constexpr (kRB > 1) residual(1);
    };
    wait_loads<0>();
    __syncthreads();
    if (s0 + 1 < s1) issue(s0 + 1, 1);
    else if (stage) residuals();
    read(0);
    for (int s = s0; s < s1; ++s) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kk = 0; kk < 3; ++kk) {
            read(kk + 1);
            multiply(kk);
            interleaved();
        }
        wait_loads<0>();
        wait_lds_reads();
        __syncthreads();
        if (s + 2 < s1) issue(s + 2, (s - s0) & 1);
        else if (s + 2 == s1 && stage) residuals();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            xat[kk] ^= kXBuf;
            wat[kk] ^= kWBuf;
        }
        read(0);   // (after the last step: what is there, and not used)
        multiply(3);
        interleaved();
        // (without a use here the reads would sink to the next step's first multiplication)
#pragma unroll
        for (int f = 0; f < 2; ++f) asm volatile("" : "+v"(wf[0][f]));
#pragma unroll
        for (int b = 0; b < kRB; ++b) asm volatile("" : "+v"(xf[0][b]));
    }
    wait_lds_reads();
    __syncthreads();

    // ---- epilogue: 32 rows x 64 features at a time through 8 KB of the wave's own, 256
    // bytes a row, 16-byte units permuted by row % 16; a lane then has 8 neighbouring
    // features of a row, and eight lanes whole lines of y. 256-row tiles, taken where y is
    // large, send it past the caches if it is no wider than x: 50 -> 45 us at 9,360 x 1,536 x
    // 1,536 without residual, 1,977 -> 1,896 at 21,600 x 5,120 x 5,120 and a product that reads
    // it next; wider ones so, a feed-forward's, 1,536 to 6,144 and back: 323 -> 340; 128-row tiles
    // so, the two at 3,600 x 1,536 x 1,536: 54 -> 56. ----
    // bias and gate of this lane's features, where all the tile's rows have one gate
    const uint32_t last = row0 + kBM - 1 < a.rows ? row0 + kBM - 1 : a.rows - 1;
    const bool one_gate = !a.gate_rows || row0 / a.N == last / a.N;
    Epilogue<8> ep;
    if (a.parts == 1 && c + 8 <= a.n_out) ep.template load<E>(a, c, one_gate ? a.frames.frame[row0 / a.N] : -1);
    // (8 KB of a wave, in the buffers of the last step, and in 64-row tiles all of x's)
    uint8_t *mine = lds + (wave < kWC ? (free_odd ^ 1) * kWBuf + wave * 8192
                                      : 2 * kWBuf + (kRB == 1 ? 0 : (free_odd ^ 1) * kXBuf) + (wave - kWC) * 8192);
#pragma unroll
    for (int b = 0; b < kRB; ++b) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4) {
                const int unit = (f * 8 + g4 * 2 + grp) ^ (col & 15);
                *reinterpret_cast<f32x4_t *>(mine + col * 256 + unit * 16) =
                    f32x4_t{acc[f][b][g4 * 4], acc[f][b][g4 * 4 + 1], acc[f][b][g4 * 4 + 2], acc[f][b][g4 * 4 + 3]};
            }
        wait_lds_reads();   // (a wave's LDS accesses run in order; this orders the compiler's)
        if (stage) {
            // (block b's loads are older than the stores of the block before, four of them
            // if any row of this block is stored, and the next block's loads)
            if (b == 0) wait_loads<0>();
            else if (b + 1 < kRB) wait_loads<8>();
            else wait_loads<4>();
        }
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
            const int lr = i * 8 + sub;
            const uint32_t r = row0 + (wr * kRB + b) * 32 + lr;
            float v[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4_t x =
                    *reinterpret_cast<const f32x4_t *>(mine + lr * 256 + ((((lane % 8) * 2 + h) ^ (lr & 15)) * 16));
#pragma unroll
                for (int e = 0; e < 4; ++e) v[h * 4 + e] = x[e];
            }
            if (r >= a.rows || c >= a.n_out) continue;
            // (fp32 may end in the middle of eight features)
            if (sizeof(E) == 4 && c + 8 > a.n_out) {
                float lo[4] = {v[0], v[1], v[2], v[3]};
                if (a.parts > 1) store_n<float, 4>(a.ws, (static_cast<int64_t>(part) * a.rows + r) * a.n_out + c, lo);
                else finish<E, 4>(a, r, c, lo);
                continue;
            }
            if (a.parts > 1) {
                store_n<float, 8>(a.ws, (static_cast<int64_t>(part) * a.rows + r) * a.n_out + c, v);
                continue;
            }
            const uint32_t m = r / a.N;
            const int64_t dst = static_cast<int64_t>(a.frames.out(m)) * a.N + (r - m * a.N);
            if (!one_gate) ep.template gate_of<E>(a, c, a.frames.frame[m]);
            ep.apply(a, v);
            if (a.residual) {
                float t[8];
                if constexpr (kStage) widen8(*reinterpret_cast<const u32x4_t *>(block(b) + i * 1024 + lane * 16), t);
                else load_n<E, 8>(a.residual, dst * a.n_out + c, t);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += t[e];
            }
            if (kRB == 4 && a.stream) {
                asm volatile("" ::: "memory");   // (without these two the compiler makes one store of both)
                stream_8<E>(a.y, dst * a.n_out + c, v);
                asm volatile("" ::: "memory");
            } else {
                store_n<E, 8>(a.y, dst * a.n_out + c, v);
            }
        }
        wait_lds_reads();
        if (stage && b + 2 < kRB) residual(b + 2);
    }
}

constexpr int kFewWaves = kLinearFewWaves;

// kR blocks of 16 rows, kF blocks of 16 features. The reduction goes in pieces of 64
// bytes (16 bytes a lane, four lanes to a row). The waves of a part take two at a time
// in turn, 1 KB of a row in all, and have the next two in flight while two multiply (four
// at a time: 11.0 against 10.0 us at 6 x 1,536 x 9,216, 9.1 against 7.7 at 8 x 3,000 x 2,000).
template <typename E, int kR, int kF>
__global__ __launch_bounds__(64 * kFewWaves) void linear_few_kernel(const LinearKArgs a) {
    __shared__ __attribute__((aligned(16))) float sums[kFewWaves][16 * kR][16 * kF];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int part = blockIdx.x % a.parts, tile = blockIdx.x / a.parts;
    const int rt = tile / a.col_tiles, c0 = (tile - rt * a.col_tiles) * (16 * kF);
    const uint32_t r0 = static_cast<uint32_t>(rt) * (16 * kR);
    const int l16 = lane & 15, grp = lane >> 4;
    // (steps here are pieces of 64 bytes)
    constexpr int kAhead = 2, kRound = kAhead * kFewWaves;
    const int s0 = part * a.steps_per_part + wave * kAhead;
    const int s1 = (part + 1) * a.steps_per_part < a.steps ? (part + 1) * a.steps_per_part : a.steps;
    const int32_t rb = static_cast<int32_t>(a.row_bytes), end = rb - grp * 16;
    const __amdgpu_buffer_rsrc_t wres = __builtin_amdgcn_make_buffer_rsrc(
        uniform_ptr(w_row(a, c0)), 0, 0x7fffffff, kBufferWord3);
    int32_t wo[kF], xo[kR];
#pragma unroll
    for (int f = 0; f < kF; ++f) {
        const int c = f * 16 + l16, most = a.n_out - 1 - c0;
        wo[f] = (c < most ? c : most) * rb + grp * 16;
    }
    f32x4_t acc[kF][kR];
#pragma unroll
    for (int f = 0; f < kF; ++f)
#pragma unroll
        for (int b = 0; b < kR; ++b) acc[f][b] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    struct Batch {
        u32x4_t w[kAhead][kF], x[kAhead][kR];
    };
    // (lanes past the end read zeros: a load under a condition would be waited for at once)
    auto place = [&](int s, int i) { return s + i < s1 ? (s + i) * 64 : 0x7fffff00; };
    auto load_w = [&](int s, Batch &t) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int32_t at = place(s, i);
#pragma unroll
            for (int f = 0; f < kF; ++f) t.w[i][f] = buffer_load16(wres, at >= end ? -1 : wo[f], at);
        }
    };
    // where x's and y's rows are is asked for first, W next, which does not wait for it
    uint32_t xr[kR];
    int32_t xf[kR];
#pragma unroll
    for (int b = 0; b < kR; ++b) {
        const uint32_t r = r0 + b * 16 + l16;
        xr[b] = r < a.rows ? r : a.rows - 1;
        xf[b] = a.frames.in(xr[b] / a.N);
    }
    const int32_t f0 = a.frames.in(r0 / a.N);
    // this thread's four results and what the epilogue takes from memory for them
    static_assert(16 * kR * 4 * kF <= 64 * kFewWaves, "a thread finishes one run of four features");
    const int lr = tid / (4 * kF), q = tid % (4 * kF), c = c0 + q * 4;
    const uint32_t r = r0 + lr;
    const bool mine = tid < 16 * kR * 4 * kF && r < a.rows && c < a.n_out;
    Finish<E, 4> fin;
    if (mine) fin.frames(a, r);
    Batch even, odd;
    load_w(s0, even);
    auto row_at = [&](int32_t frame, uint32_t row) {
        return (static_cast<int64_t>(frame) * a.N + row % a.N) * a.row_bytes;
    };
    const int64_t x0 = row_at(f0, r0);
    const __amdgpu_buffer_rsrc_t xres =
        __builtin_amdgcn_make_buffer_rsrc(uniform_ptr(a.x + x0), 0, 0x7fffffff, kBufferWord3);
#pragma unroll
    for (int b = 0; b < kR; ++b)
        // (lanes of rows past the last read zeros: no line is fetched for them)
        xo[b] = r0 + b * 16 + l16 < a.rows ? static_cast<int32_t>(row_at(xf[b], xr[b]) - x0) + grp * 16 : -1;
    auto load_x = [&](int s, Batch &t) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int32_t at = place(s, i);
#pragma unroll
            for (int b = 0; b < kR; ++b) t.x[i][b] = buffer_load16(xres, at >= end ? -1 : xo[b], at);
        }
    };
    load_x(s0, even);
    if (mine && a.parts == 1) fin.load(a, r, c);
    auto multiply = [&](const Batch &t) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int f = 0; f < kF; ++f)
#pragma unroll
                for (int b = 0; b < kR; ++b) acc[f][b] = mma16<E>(t.w[i][f], t.x[i][b], acc[f][b]);
    };
    for (int s = s0; s < s1; s += 2 * kRound) {
        load_w(s + kRound, odd);
        load_x(s + kRound, odd);
        multiply(even);
        load_w(s + 2 * kRound, even);
        load_x(s + 2 * kRound, even);
        multiply(odd);
    }
    // lane: row l16 of a block, features 4 grp .. 4 grp + 3
#pragma unroll
    for (int f = 0; f < kF; ++f)
#pragma unroll
        for (int b = 0; b < kR; ++b)
            *reinterpret_cast<f32x4_t *>(&sums[wave][b * 16 + l16][f * 16 + grp * 4]) = acc[f][b];
    __syncthreads();
    if (!mine) return;
    f32x4_t x = *reinterpret_cast<const f32x4_t *>(&sums[0][lr][q * 4]);
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) {
        const f32x4_t y = *reinterpret_cast<const f32x4_t *>(&sums[w][lr][q * 4]);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += y[e];
    }
    float v[4] = {x[0], x[1], x[2], x[3]};
    if (a.parts > 1) store_n<float, 4>(a.ws, (static_cast<int64_t>(part) * a.rows + r) * a.n_out + c, v);
    else fin.store(a, c, v);
}

template <typename E>
__global__ __launch_bounds__(256) void linear_join_kernel(const LinearKArgs a) {
    const int64_t per_row = a.n_out / 4, id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (id >= per_row * a.rows) return;
    const uint32_t r = static_cast<uint32_t>(id / per_row);
    const int c = static_cast<int>(id - r * per_row) * 4;
    Finish<E, 4> fin;
    fin.frames(a, r);
    fin.load(a, r, c);
    f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
    const float *p = a.ws + static_cast<int64_t>(r) * a.n_out + c;
    const int64_t step = static_cast<int64_t>(a.rows) * a.n_out;
#pragma unroll 8
    for (int i = 0; i < a.parts; ++i) {
        const f32x4_t y = *reinterpret_cast<const f32x4_t *>(p + i * step);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += y[e];
    }
    float v[4] = {x[0], x[1], x[2], x[3]};
    fin.store(a, c, v);
}

template <typename E>
void run(const LinearPlan &p, const LinearKArgs &a, bool far, dim3 grid, hipStream_t stream) {
    switch (p.form) {
        case kFew16: hipLaunchKernelGGL((linear_few_kernel<E, 1, 1>), grid, dim3(512), 0, stream, a); break;
        case kFew32: hipLaunchKernelGGL((linear_few_kernel<E, 2, 2>), grid, dim3(512), 0, stream, a); break;
        case kFew64: hipLaunchKernelGGL((linear_few_kernel<E, 4, 1>), grid, dim3(512), 0, stream, a); break;
        case kStream32: hipLaunchKernelGGL((linear_tile_kernel<E, 1, 1, 4, false>), grid, dim3(256), 0, stream, a); break;
        case kStream64:   // (bf16 only)
            if constexpr (sizeof(E) == 2)
                hipLaunchKernelGGL((linear_tile_kernel<E, 2, 1, 4, false>), grid, dim3(256), 0, stream, a);
            break;
        case kTile64: hipLaunchKernelGGL((linear_tile_kernel<E, 1, 2, 2, false>), grid, dim3(256), 0, stream, a); break;
        case kTile128:
            if (far) hipLaunchKernelGGL((linear_tile_kernel<E, 2, 2, 2, true>), grid, dim3(256), 0, stream, a);
            else hipLaunchKernelGGL((linear_tile_kernel<E, 2, 2, 2, false>), grid, dim3(256), 0, stream, a);
            break;
        case kTile256:    // (bf16 only)
            if constexpr (sizeof(E) == 2)
                hipLaunchKernelGGL((linear_tile_kernel<E, 4, 2, 4, false>), grid, dim3(512), 0, stream, a);
            break;
        case kLinearForms: break;
    }
}

}  // namespace

int64_t linear_workspace(int64_t rows, int32_t K, int32_t n_out, int32_t dtype, int32_t cus) {
    // (far or not is the frame list's: room for either)
    int64_t bytes = 0;
    for (const bool far : {false, true}) {
        const LinearPlan p = linear_plan(rows, K, n_out, dtype, cus, far, true);
        const int64_t need = p.parts > 1 ? p.parts * rows * n_out * 4 : 0;
        bytes = need > bytes ? need : bytes;
    }
    return bytes;
}

hipError_t launch_linear(const LinearParams &p, hipStream_t stream) {
    const int32_t xcds = p.geo.xcds;
    if (p.geo.cus < 1 || xcds < 1 || xcds > 64) return hipErrorInvalidValue;
    const int64_t rows = p.M * p.N;
    const int64_t row_bytes = static_cast<int64_t>(p.K) * (p.dtype == RF_F32 ? 4 : 2);
    const bool far = linear_far(p.frames, p.M, p.N, row_bytes);
    const LinearPlan plan = linear_plan(rows, p.K, p.n_out, p.dtype, p.geo.cus, far, p.ws != nullptr);
    LinearKArgs a{};
    a.x = static_cast<const uint8_t *>(p.x);
    a.w = static_cast<const uint8_t *>(p.weight);
    a.bias = p.bias;
    a.gate = p.gate;
    a.residual = p.residual;
    a.y = p.y;
    a.ws = static_cast<float *>(p.ws);
    a.row_bytes = row_bytes;
    a.rows = static_cast<uint32_t>(rows);
    a.N = static_cast<uint32_t>(p.N);
    a.n_out = p.n_out;
    a.steps = plan.steps;
    a.steps_per_part = plan.per_part;
    a.parts = plan.parts;
    a.activation = p.activation;
    a.gate_rows = p.gate_rows;
    a.stream = p.n_out <= p.K;
    a.frames = p.frames;
    const int64_t tiles = plan.row_tiles * plan.col_tiles;
    if (tiles > 0x7fffffffLL / 64) return hipErrorInvalidConfiguration;
    a.row_tiles = static_cast<int32_t>(plan.row_tiles);
    a.col_tiles = static_cast<int32_t>(plan.col_tiles);
    a.tiles = static_cast<int32_t>(tiles);
    a.xcds = xcds;
    a.per_xcd = (a.tiles + xcds - 1) / xcds;
    const bool few = plan.form <= kFew64;
    const int64_t grid = (few ? tiles : static_cast<int64_t>(a.per_xcd) * xcds) * plan.parts;
    if (grid > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    const dim3 g(static_cast<uint32_t>(grid));
    if (p.dtype == RF_F32) run<float>(plan, a, far, g, stream);
    else run<uint16_t>(plan, a, far, g, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.parts == 1) return e;
    const int64_t blocks = (rows * (p.n_out / 4) + 255) / 256;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    const dim3 jg(static_cast<uint32_t>(blocks));
    if (p.dtype == RF_F32) hipLaunchKernelGGL(linear_join_kernel<float>, jg, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL(linear_join_kernel<uint16_t>, jg, dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace rf
