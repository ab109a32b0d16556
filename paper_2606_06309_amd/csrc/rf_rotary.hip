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
// walks heads of q and k with them, so a sine and cosine serve all its heads.
// Angles are formed in double, reduced to half a turn there and only then
// rounded: at position 2^20 an fp32 angle would be off by 0.06.
#include "rf_internal.h"

namespace rf {
namespace {

constexpr int kThreads = 256;

struct RotaryKArgs {
    RotaryParams p;
    int64_t N;
    int64_t threads;           // rows * units
    int32_t units;             // threads per token
    int32_t rot_units;         // of them, those that own turning dimensions
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
    typedef float raw_t __attribute__((ext_vector_type(8)));
    raw_t w;
    __device__ __forceinline__ float get(int e) const { return w[e]; }
    __device__ __forceinline__ void set2(int e, float lo, float hi) {
        w[e] = lo;
        w[e + 1] = hi;
    }
};

template <typename E>
__device__ __forceinline__ Vec8<E> load8(const E *p) {
    Vec8<E> v;
    typedef typename Vec8<E>::raw_t aligned_t __attribute__((aligned(16)));
    v.w = *reinterpret_cast<const aligned_t *>(p);
    return v;
}
template <typename E>
__device__ __forceinline__ void store8(E *p, const Vec8<E> &v) {
    typedef typename Vec8<E>::raw_t aligned_t __attribute__((aligned(16)));
    *reinterpret_cast<aligned_t *>(p) = v.w;
}

template <typename E, bool kHalves>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryKArgs a) {
    const RotaryParams &p = a.p;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (id >= a.threads) return;
    const int64_t row = id / a.units;
    const int unit = static_cast<int>(id - row * a.units);
    const int m = static_cast<int>(row / a.N);
    const int64_t n = row - m * a.N;
    const int y = static_cast<int>(n / p.W), x = static_cast<int>(n - static_cast<int64_t>(y) * p.W);
    const bool turns = unit < a.rot_units;
    // halves: unit u < rot_units owns dimensions 8u.. and R/2 + 8u..; later units 8 dimensions past R
    const int at = kHalves && !turns ? 2 * p.pairs + 8 * (unit - a.rot_units) : 8 * unit;

    constexpr int kP = kHalves ? 8 : 4;   // pairs
    float c[kP], s[kP];
    if (turns) {
#pragma unroll
        for (int i = 0; i < kP; ++i) {
            const int pair = (kHalves ? 8 : 4) * unit + i;
            c[i] = 1.0f;
            s[i] = 0.0f;
            if (pair < p.pairs) {
                const int axis = pair < p.pair_end[0] ? 0 : pair < p.pair_end[1] ? 1 : 2;
                const double index = axis == 0 ? p.frame[m] : axis == 1 ? y : x;
                const double t = fma(p.step[axis], index, p.origin[axis]) * p.turns[pair];
                sincospif(static_cast<float>(2.0 * (t - rint(t))), &s[i], &c[i]);
            }
        }
    }
    const int64_t src = static_cast<int64_t>(p.src_frame[m]) * a.N + n;
    const int64_t dst = static_cast<int64_t>(p.dst_frame[m]) * a.N + n;
    const int h0 = blockIdx.y * a.heads_per_thread;
    const int total = p.heads[0] + p.heads[1];
    const int h1 = h0 + a.heads_per_thread < total ? h0 + a.heads_per_thread : total;
    for (int h = h0; h < h1; ++h) {
        const int t = h < p.heads[0] ? 0 : 1;
        const int64_t col = static_cast<int64_t>(h - (t ? p.heads[0] : 0)) * p.head_dim + at;
        const E *xp = static_cast<const E *>(p.x[t]) + src * p.x_stride[t] + col;
        E *yp = static_cast<E *>(p.y[t]) + dst * p.y_stride[t] + col;
        Vec8<E> v = load8(xp);
        if (turns && kHalves) {
            Vec8<E> w = load8(xp + p.pairs);
            const Vec8<E> v0 = v, w0 = w;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const float a0 = v0.get(i), a1 = v0.get(i + 1), b0 = w0.get(i), b1 = w0.get(i + 1);
                v.set2(i, fmaf(a0, c[i], -(b0 * s[i])), fmaf(a1, c[i + 1], -(b1 * s[i + 1])));
                w.set2(i, fmaf(a0, s[i], b0 * c[i]), fmaf(a1, s[i + 1], b1 * c[i + 1]));
            }
            store8(yp + p.pairs, w);
        } else if (turns) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // (a pair past R passes as it is, infinities and NaN too)
                if (4 * unit + i >= p.pairs) continue;
                const float a0 = v.get(2 * i), b0 = v.get(2 * i + 1);
                v.set2(2 * i, fmaf(a0, c[i], -(b0 * s[i])), fmaf(a0, s[i], b0 * c[i]));
            }
        }
        store8(yp, v);
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
    a.N = static_cast<int64_t>(p.H) * p.W;
    // (halves: R/2 is a multiple of 8; else the unit that holds the last pair may pass some dimensions on)
    a.rot_units = p.halves ? p.pairs / 8 : (p.pairs + 3) / 4;
    a.units = p.halves ? a.rot_units + (p.head_dim - 2 * p.pairs) / 8 : p.head_dim / 8;
    a.threads = p.M * a.N * a.units;
    a.heads_per_thread = p.heads[0] + p.heads[1];
    const int64_t blocks = (a.threads + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    const dim3 grid(static_cast<uint32_t>(blocks), 1);
    if (p.dtype == RF_F32) return p.halves ? launch<float, true>(a, grid, stream) : launch<float, false>(a, grid, stream);
    return p.halves ? launch<uint16_t, true>(a, grid, stream) : launch<uint16_t, false>(a, grid, stream);
}

}  // namespace rf
