// Rotary positions over time, height and width for gfx950.
//
// Pair p of a head's leading R dimensions turns by phi = position * turns[p]
// (in turns), position being origin + step * index on the pair's axis: frame,
// row or column of the token. The rows of the listed frames come compact or at
// their places among all frames and go to either, so the rotation doubles as
// the frame gather or scatter.
//
// What bounds it: every element is read and written once (memory). A thread
// owns 8 neighbouring dimensions of a token (4 pairs; with halves, 8 + 8) and
// walks heads of q and k with them, four at a time, so a sine and cosine serve
// all its heads and four loads are in flight.
// 21 frames of 30 x 52, 12 + 12 heads x 128, bf16: 72.5 us, 5.55 TB/s (a large copy 4.9
// to 5.2); 6 of them, views of a fused projection, to their positions: 24 us, 4.8 TB/s. With
// halves 74.5 and 22.6 us; fp32, either way, 170 us (4.7 TB/s) and 50 to 51 (4.5).
// Lanes interleaved over heads, 1 KB contiguous to a load, took 86.8 us where this took 73.3.
// Angles are formed in double, reduced to half a turn there and only then
// rounded: at position 2^20 an fp32 angle would be off by 0.06.
#include "rf_internal.h"

namespace rf {
namespace {

// One wave a workgroup (5.5 TB/s at 21 frames of 30 x 52, 12 + 12 heads x 128, against
// 5.2 of 256 threads), and loads and stores that do not stay in the caches (against
// 5.1): each element is met once here.
constexpr int kThreads = 64;
// Workgroups that fill the device (32 to each of 256 compute units).
constexpr int64_t kFill = 8192;

struct RotaryKArgs {
    RotaryParams p;
    uint32_t N;                // tokens per frame
    uint32_t units;            // threads per token
    uint32_t rot_units;        // of them, those that own turning dimensions
    int32_t heads_per_thread;  // of q's and k's heads, one after the other
};
static_assert(sizeof(RotaryKArgs) <= 4096, "kernel arguments exceed 4 KB");

template <typename E>
struct Vec8;   // 8 elements as loaded
template <>
struct Vec8<uint16_t> {
    typedef uint32_t raw_t __attribute__((ext_vector_type(4)));
    raw_t w;
    __device__ __forceinline__ float get(int e) const {
        return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    }
    // one rounding to nearest even of each pair of results
    __device__ __forceinline__ void set2(int e, float lo, float hi) {
        typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
        const bf16x2_t v = {static_cast<__bf16>(lo), static_cast<__bf16>(hi)};
        w[e / 2] = __builtin_bit_cast(uint32_t, v);
    }
};
template <>
struct Vec8<float> {
    typedef float raw_t __attribute__((ext_vector_type(4)));
    raw_t w[2];
    __device__ __forceinline__ float get(int e) const { return w[e / 4][e % 4]; }
    __device__ __forceinline__ void set2(int e, float lo, float hi) {
        w[e / 4][e % 4] = lo;
        w[e / 4][e % 4 + 1] = hi;
    }
};

__device__ __forceinline__ Vec8<uint16_t> load8(const uint16_t *p) {
    Vec8<uint16_t> v;
    v.w = __builtin_nontemporal_load(reinterpret_cast<const Vec8<uint16_t>::raw_t *>(p));
    return v;
}
__device__ __forceinline__ Vec8<float> load8(const float *p) {
    Vec8<float> v;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        v.w[i] = __builtin_nontemporal_load(reinterpret_cast<const Vec8<float>::raw_t *>(p) + i);
    return v;
}
__device__ __forceinline__ void store8(uint16_t *p, const Vec8<uint16_t> &v) {
    __builtin_nontemporal_store(v.w, reinterpret_cast<Vec8<uint16_t>::raw_t *>(p));
}
__device__ __forceinline__ void store8(float *p, const Vec8<float> &v) {
#pragma unroll
    for (int i = 0; i < 2; ++i) __builtin_nontemporal_store(v.w[i], reinterpret_cast<Vec8<float>::raw_t *>(p) + i);
}

// One head's 8 (with halves 8 + 8) elements of a thread.
template <typename E, bool kHalves>
struct Piece {
    Vec8<E> v, w;
    E *to;
};

template <typename E, bool kHalves>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryKArgs a) {
    const RotaryParams &p = a.p;
    const uint32_t m = blockIdx.z;
    // (a frame has at most 2^26 tokens of 32 threads)
    const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
    const uint32_t n = id / a.units, unit = id - n * a.units;
    if (n >= a.N) return;
    const uint32_t y = n / static_cast<uint32_t>(p.W), x = n - y * static_cast<uint32_t>(p.W);
    const bool turns = unit < a.rot_units;
    // halves: unit u < rot_units owns dimensions 8u.. and R/2 + 8u..; later units 8 dimensions past R
    const int at = kHalves && !turns ? 2 * p.pairs + 8 * (unit - a.rot_units) : 8 * unit;

    const int64_t src = static_cast<int64_t>(p.frames.in(m)) * a.N + n;
    const int64_t dst = static_cast<int64_t>(p.frames.out(m)) * a.N + n;
    const int total = p.heads[0] + p.heads[1];
    const int h0 = blockIdx.y * a.heads_per_thread;
    const int h1 = h0 + a.heads_per_thread < total ? h0 + a.heads_per_thread : total;
    auto load = [&](int h) {
        const int t = h < p.heads[0] ? 0 : 1;
        const int64_t col = static_cast<int64_t>(h - (t ? p.heads[0] : 0)) * p.head_dim + at;
        const E *from = static_cast<const E *>(p.x[t]) + src * p.x_stride[t] + col;
        Piece<E, kHalves> r;
        r.to = static_cast<E *>(p.y[t]) + dst * p.y_stride[t] + col;
        r.v = load8(from);
        if (kHalves && turns) r.w = load8(from + p.pairs);
        return r;
    };
    constexpr int kAhead = 4;
    Piece<E, kHalves> r[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (h0 + i < h1) r[i] = load(h0 + i);

    constexpr int kP = kHalves ? 8 : 4;   // pairs
    float c[kP], s[kP];
#pragma unroll
    for (int i = 0; i < kP; ++i) {
        const int pair = kP * unit + i;
        c[i] = 1.0f;
        s[i] = 0.0f;
        if (pair < p.pairs) {
            const int axis = pair < p.pair_end[0] ? 0 : pair < p.pair_end[1] ? 1 : 2;
            const double index = axis == 0 ? p.frames.frame[m] : axis == 1 ? y : x;
            const double t = fma(p.step[axis], index, p.origin[axis]) * p.turns[pair];
            sincospif(static_cast<float>(2.0 * (t - rint(t))), &s[i], &c[i]);
        }
    }
    auto turn = [&](Piece<E, kHalves> &q) {
        if (turns && kHalves) {
            const Vec8<E> v = q.v, w = q.w;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const float a0 = v.get(i), a1 = v.get(i + 1), b0 = w.get(i), b1 = w.get(i + 1);
                q.v.set2(i, fmaf(a0, c[i], -(b0 * s[i])), fmaf(a1, c[i + 1], -(b1 * s[i + 1])));
                q.w.set2(i, fmaf(a0, s[i], b0 * c[i]), fmaf(a1, s[i + 1], b1 * c[i + 1]));
            }
            store8(q.to + p.pairs, q.w);
        } else if (turns) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // (a pair past R passes as it is, infinities and NaN too)
                if (kP * static_cast<int>(unit) + i >= p.pairs) continue;
                const float a0 = q.v.get(2 * i), b0 = q.v.get(2 * i + 1);
                q.v.set2(2 * i, fmaf(a0, c[i], -(b0 * s[i])), fmaf(a0, s[i], b0 * c[i]));
            }
        }
        store8(q.to, q.v);
    };
    for (int h = h0; h < h1; h += kAhead) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (h + i < h1) turn(r[i]);
        if (h + kAhead >= h1) break;
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (h + kAhead + i < h1) r[i] = load(h + kAhead + i);
    }
}

template <typename E, bool kHalves>
hipError_t launch(const RotaryKArgs &a, dim3 grid, hipStream_t stream) {
    hipLaunchKernelGGL((rotary_kernel<E, kHalves>), grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryParams &p, hipStream_t stream) {
    RotaryKArgs a{};
    a.p = p;
    const int64_t N = static_cast<int64_t>(p.H) * p.W;
    // (halves: R/2 is a multiple of 8; else the unit that holds the last pair may pass some dimensions on)
    a.rot_units = p.halves ? p.pairs / 8 : (p.pairs + 3) / 4;
    a.units = p.halves ? a.rot_units + (p.head_dim - 2 * p.pairs) / 8 : p.head_dim / 8;
    const int64_t blocks = (N * a.units + kThreads - 1) / kThreads;
    // (a launch has fewer than 2^32 threads along an axis: each frame is one step of the third)
    if (N * a.units > 0x7fffffffLL + 1) return hipErrorInvalidConfiguration;
    a.N = static_cast<uint32_t>(N);
    const int heads = p.heads[0] + p.heads[1];
    // a thread takes all heads of its token, or fewer where tokens do not fill the device
    const int64_t most = (heads + 3) / 4, want = kFill / (blocks * p.M) + 1;
    const int64_t groups = want < most ? want : most;
    a.heads_per_thread = static_cast<int32_t>((heads + groups - 1) / groups);
    const dim3 grid(static_cast<uint32_t>(blocks),
                    static_cast<uint32_t>((heads + a.heads_per_thread - 1) / a.heads_per_thread),
                    static_cast<uint32_t>(p.M));
    if (p.dtype == RF_F32) return p.halves ? launch<float, true>(a, grid, stream) : launch<float, false>(a, grid, stream);
    return p.halves ? launch<uint16_t, true>(a, grid, stream) : launch<uint16_t, false>(a, grid, stream);
}

}  // namespace rf
