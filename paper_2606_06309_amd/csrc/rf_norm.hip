// Group norm with an activation, channels last, and rows in 8 bits, for gfx950.
//
//   y = act((x - mean) / sqrt(var + eps) * weight + bias),   mean, var over rows x channels of a group
//   scale = max |x| / 127,  q = x * (127 / max |x|) to the nearest integer
//
//  * norm_stats_kernel: a workgroup has a run of a frame's rows and up to 256 16-byte columns;
//    a thread keeps its column's channels and walks rows, eight at a time: their mean and
//    squared deviations from it, joined to those so far (a sum of squares about another
//    point than the mean would lose what small deviations around a large mean are). The
//    threads' rows, then the channels of each group, meet in LDS.
//  * norm_total_kernel: a wave joins the parts of a group, in a fixed order.
//  * norm_rows_kernel: x again, to y; norm_rows8_kernel: whole rows at a time, to 8 bits.
//  * quantize_kernel: rows of x to 8 bits.
#include "rf_norm_plan.h"
#include "rf_rows.h"

namespace rf {
namespace {

constexpr int kThreads = kNormThreads;
constexpr int kAhead = 8;      // rows of a thread in flight

struct NormKArgs {
    const uint8_t *x;
    uint8_t *y;
    float *y_scale;
    const void *weight, *bias;
    float2 *partial;               // [M][parts][slices][local]: mean, sum of squared deviations
    float2 *total;                 // [M / together][groups]: mean, 1 / sqrt(var + eps)
    int64_t N, per_part;
    int64_t x_stride, y_stride;    // bytes
    double eps;
    int32_t M, C, groups, together, per_group;
    int32_t cols, slices, lines, parts, local;
    int32_t activation, affine_rows;
    RowFrames frames;
};

// n values of mean `mean` and squared deviations `m2`, joined by n_b more: the means' distance adds
// n n_b / (n + n_b) of its square.
__device__ __forceinline__ void join(float n, float &mean, float &m2, float n_b, float mean_b, float m2_b, float share_b) {
    const float d = mean_b - mean;
    mean = fmaf(d, share_b, mean);
    m2 += fmaf(d * d, n * share_b, m2_b);
}

template <typename E>
__device__ __forceinline__ void widen(u32x4_t x, float (&v)[16 / sizeof(E)]) {
    if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(x[e]);
    } else {
        widen8(x, v);
    }
}

template <typename E>
__global__ __launch_bounds__(kThreads) void norm_stats_kernel(const NormKArgs a) {
    constexpr int kV = 16 / sizeof(E);
    __shared__ float s_mean[kV][kThreads], s_m2[kV][kThreads], s_n[kThreads];
    const int tid = threadIdx.x;
    int id = blockIdx.x;
    const int slice = id % a.slices;
    id /= a.slices;
    const int part = id % a.parts, m = id / a.parts;
    const int line = tid / a.cols, col = tid - line * a.cols, column = slice * a.cols + col;
    const bool active = line < a.lines && column * kV < a.C;
    const int64_t r0 = part * a.per_part, r1 = r0 + a.per_part < a.N ? r0 + a.per_part : a.N;
    float n = 0.0f, mean[kV], m2[kV];
#pragma unroll
    for (int e = 0; e < kV; ++e) mean[e] = m2[e] = 0.0f;
    if (active) {
        const uint8_t *p = a.x + (a.frames.in(m) * a.N + r0 + line) * a.x_stride + column * 16;
        const int64_t step = a.lines * a.x_stride;
        int64_t left = r1 - r0 > line ? (r1 - r0 - line + a.lines - 1) / a.lines : 0;   // rows of this thread
        for (; left >= kAhead; left -= kAhead, p += kAhead * step) {
            u32x4_t raw[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) raw[i] = *reinterpret_cast<const u32x4_t *>(p + i * step);
            float v[kAhead][kV];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) widen<E>(raw[i], v[i]);
            const float share = kAhead / (n + kAhead);
#pragma unroll
            for (int e = 0; e < kV; ++e) {
                float s = 0.0f, q = 0.0f;
#pragma unroll
                for (int i = 0; i < kAhead; ++i) s += v[i][e];
                s *= 1.0f / kAhead;
#pragma unroll
                for (int i = 0; i < kAhead; ++i) q = fmaf(v[i][e] - s, v[i][e] - s, q);
                join(n, mean[e], m2[e], kAhead, s, q, share);
            }
            n += kAhead;
        }
        for (; left > 0; --left, p += step) {
            float v[kV];
            widen<E>(*reinterpret_cast<const u32x4_t *>(p), v);
            const float share = 1.0f / (n + 1.0f);
#pragma unroll
            for (int e = 0; e < kV; ++e) join(n, mean[e], m2[e], 1.0f, v[e], 0.0f, share);
            n += 1.0f;
        }
    }
    s_n[tid] = n;
#pragma unroll
    for (int e = 0; e < kV; ++e) {
        s_mean[e][tid] = mean[e];
        s_m2[e][tid] = m2[e];
    }
    // lines of a column, in halves
    for (int width = a.lines; width > 1;) {
        const int half = (width + 1) / 2;
        __syncthreads();
        if (line + half < width) {
            const int other = tid + half * a.cols;
            const float n_b = s_n[other];
            if (n_b > 0.0f) {
                const float share = n_b / (n + n_b);
#pragma unroll
                for (int e = 0; e < kV; ++e) {
                    join(n, mean[e], m2[e], n_b, s_mean[e][other], s_m2[e][other], share);
                    s_mean[e][tid] = mean[e];
                    s_m2[e][tid] = m2[e];
                }
                n += n_b;
                s_n[tid] = n;
            }
        }
        width = half;
    }
    __syncthreads();
    // the channels of a group, all of as many rows: lanes share out its channels of this slice
    const int c0 = slice * a.cols * kV, c1 = c0 + a.cols * kV < a.C ? c0 + a.cols * kV : a.C;
    const int g0 = c0 / a.per_group, n_local = (c1 - 1) / a.per_group - g0 + 1;
    int lanes = 1;
    while (lanes < 64 && 2 * lanes * n_local <= kThreads) lanes *= 2;
    const int lane = tid % lanes;
    const float rows = static_cast<float>(r1 - r0);
    for (int l = tid / lanes; l < n_local; l += kThreads / lanes) {
        const int first = (g0 + l) * a.per_group, behind = first + a.per_group;
        const int lo = (first > c0 ? first : c0) - c0, hi = (behind < c1 ? behind : c1) - c0;
        float s = 0.0f, q = 0.0f;
        for (int c = lo + lane; c < hi; c += lanes) s += s_mean[c % kV][c / kV];
        for (int d = lanes / 2; d > 0; d /= 2) s += __shfl_xor(s, d);
        s /= static_cast<float>(hi - lo);
        for (int c = lo + lane; c < hi; c += lanes) {
            const float d = s_mean[c % kV][c / kV] - s;
            q += fmaf(rows * d, d, s_m2[c % kV][c / kV]);
        }
        for (int d = lanes / 2; d > 0; d /= 2) q += __shfl_xor(q, d);
        if (lane == 0)
            a.partial[((static_cast<int64_t>(m) * a.parts + part) * a.slices + slice) * a.local + l] = make_float2(s, q);
    }
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) x += __shfl_xor(x, d);
    return x;
}

// A wave joins a group's parts, in 64 bits: their means first, then the deviations about it.
template <typename E>
__global__ __launch_bounds__(kThreads) void norm_total_kernel(const NormKArgs a) {
    constexpr int kV = 16 / sizeof(E);
    const int lane = threadIdx.x & 63;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + threadIdx.x / 64;
    const int seg = static_cast<int>(id / a.groups), g = static_cast<int>(id - static_cast<int64_t>(seg) * a.groups);
    if (seg * a.together >= a.M) return;
    const int width = a.cols * kV;
    const int s0 = g * a.per_group / width, s1 = ((g + 1) * a.per_group - 1) / width;
    const int runs = a.together * a.parts;
    double mean = 0.0, m2 = 0.0;
    const double all = static_cast<double>(a.together) * static_cast<double>(a.N) * a.per_group;
    for (int pass = 0; pass < 2; ++pass) {
        double sum = 0.0;
        for (int s = s0; s <= s1; ++s) {
            const int c0 = s * width, first = g * a.per_group;
            const int lo = first > c0 ? first : c0;
            int hi = first + a.per_group < c0 + width ? first + a.per_group : c0 + width;
            const int l = g - c0 / a.per_group;
            for (int i = lane; i < runs; i += 64) {
                const int part = i % a.parts;
                const int64_t r0 = part * a.per_part, r1 = r0 + a.per_part < a.N ? r0 + a.per_part : a.N;
                const double n = static_cast<double>(r1 - r0) * (hi - lo);
                const float2 v = a.partial[((static_cast<int64_t>(seg) * runs + i) * a.slices + s) * a.local + l];
                if (pass == 0) {
                    sum += n * v.x;
                } else {
                    const double d = v.x - mean;
                    sum += v.y + n * d * d;
                }
            }
        }
        sum = wave_sum(sum);
        if (pass == 0) mean = sum / all;
        else m2 = sum / all;
    }
    if (lane == 0) a.total[id] = make_float2(static_cast<float>(mean), static_cast<float>(1.0 / sqrt(m2 + a.eps)));
}

// What channel c of listed frame m is normalised with: (x - mean) * mul + add.
struct Affine {
    float mean, mul, add;
};
template <typename E>
__device__ __forceinline__ float element(const void *p, int64_t at) {
    if constexpr (sizeof(E) == 4) return static_cast<const float *>(p)[at];
    else return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t *>(p)[at]) << 16);
}
template <typename E>
__device__ __forceinline__ Affine affine_of(const NormKArgs &a, int m, int c) {
    const float2 t = a.total[static_cast<int64_t>(m / a.together) * a.groups + c / a.per_group];
    const int64_t at = (a.affine_rows ? static_cast<int64_t>(a.frames.frame[m]) * a.C : 0) + c;
    return {t.x, a.weight ? t.y * element<E>(a.weight, at) : t.y, a.bias ? element<E>(a.bias, at) : 0.0f};
}

template <typename E>
__global__ __launch_bounds__(kThreads) void norm_rows_kernel(const NormKArgs a) {
    constexpr int kV = 16 / sizeof(E);
    const int tid = threadIdx.x;
    int id = blockIdx.x;
    const int slice = id % a.slices;
    id /= a.slices;
    const int part = id % a.parts, m = id / a.parts;
    const int line = tid / a.cols, col = tid - line * a.cols, column = slice * a.cols + col;
    if (line >= a.lines || column * kV >= a.C) return;
    const int64_t r0 = part * a.per_part, r1 = r0 + a.per_part < a.N ? r0 + a.per_part : a.N;
    Affine f[kV];
#pragma unroll
    for (int e = 0; e < kV; ++e) f[e] = affine_of<E>(a, m, column * kV + e);
    // (y may be x: no row is read again)
    const uint8_t *p = a.x + (a.frames.in(m) * a.N) * a.x_stride + column * 16;
    uint8_t *q = a.y + (a.frames.out(m) * a.N) * a.y_stride + column * 16;
    constexpr int kRows = 4;
    for (int64_t r = r0 + line; r < r1; r += kRows * a.lines) {
        u32x4_t raw[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int64_t at = r + i * a.lines;
            raw[i] = *reinterpret_cast<const u32x4_t *>(p + (at < r1 ? at : r) * a.x_stride);
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int64_t at = r + i * a.lines;
            if (at >= r1) break;
            float v[kV];
            widen<E>(raw[i], v);
#pragma unroll
            for (int e = 0; e < kV; ++e) v[e] = fmaf(v[e] - f[e].mean, f[e].mul, f[e].add);
            if (a.activation != RF_ACT_NONE) activate(a.activation, v);
            store_n<E, kV>(q + at * a.y_stride, 0, v);
        }
    }
}

// The largest of kLanes neighbouring lanes' values (kLanes > 64: of all of the workgroup's kLanes
// threads, through LDS; `turn` takes two places in turn, so that one barrier does).
template <int kLanes>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v, uint32_t (*places)[kLanes / 64 > 0 ? kLanes / 64 : 1], int turn) {
#pragma unroll
    for (int d = 1; d < (kLanes < 64 ? kLanes : 64); d *= 2) {
        const uint32_t o = __shfl_xor(v, d);
        v = v > o ? v : o;
    }
    if constexpr (kLanes > 64) {
        if ((threadIdx.x & 63) == 0) places[turn & 1][threadIdx.x / 64] = v;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kLanes / 64; ++w) {
            const uint32_t o = places[turn & 1][w];
            v = v > o ? v : o;
        }
    }
    return v;
}

// kLanes threads to a row, kPer columns to a thread, lane after lane; kC: most channels.
template <typename E, int kLanes, int kPer, int kC>
__global__ __launch_bounds__(kThreads) void norm_rows8_kernel(const NormKArgs a) {
    constexpr int kV = 16 / sizeof(E), kRows = kThreads / kLanes;
    __shared__ __attribute__((aligned(16))) float s_mean[kC], s_mul[kC], s_add[kC];
    __shared__ uint32_t places[2][kLanes / 64 > 0 ? kLanes / 64 : 1];
    const int tid = threadIdx.x;
    const int part = blockIdx.x % a.parts, m = blockIdx.x / a.parts;
    for (int c = tid; c < a.C; c += kThreads) {
        const Affine f = affine_of<E>(a, m, c);
        s_mean[c] = f.mean;
        s_mul[c] = f.mul;
        s_add[c] = f.add;
    }
    __syncthreads();
    const int lane = tid % kLanes, line = tid / kLanes, columns = a.C / kV;
    const int64_t r0 = part * a.per_part, r1 = r0 + a.per_part < a.N ? r0 + a.per_part : a.N;
    const uint8_t *x = a.x + (a.frames.in(m) * a.N) * a.x_stride;
    uint8_t *y = a.y + (a.frames.out(m) * a.N) * a.C;
    float *scales = a.y_scale + a.frames.out(m) * a.N;
    int turn = 0;
    for (int64_t first = r0; first < r1; first += kRows, ++turn) {
        const int64_t r = first + line < r1 ? first + line : r1 - 1;
        u32x4_t raw[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int col = lane + i * kLanes;
            raw[i] = *reinterpret_cast<const u32x4_t *>(x + r * a.x_stride + (col < columns ? col : columns - 1) * 16);
        }
        float v[kPer][kV];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int col = lane + i * kLanes, c = (col < columns ? col : columns - 1) * kV;
            widen<E>(raw[i], v[i]);
#pragma unroll
            for (int e = 0; e < kV; ++e) v[i][e] = fmaf(v[i][e] - s_mean[c + e], s_mul[c + e], s_add[c + e]);
            if (a.activation != RF_ACT_NONE) activate(a.activation, v[i]);
#pragma unroll
            for (int e = 0; e < kV; ++e) {
                const uint32_t bits = __float_as_uint(v[i][e]) & 0x7fffffffu;
                top = top > bits ? top : bits;
            }
        }
        const RowScale s(lanes_max<kLanes>(top, places, turn));
        if (first + line >= r1) continue;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int col = lane + i * kLanes;
            if (col >= columns) break;
            uint32_t *to = reinterpret_cast<uint32_t *>(y + r * a.C + col * kV);
            if constexpr (kV == 8) *reinterpret_cast<u32x2_t *>(to) = u32x2_t{round4(v[i], s.inverse), round4(v[i] + 4, s.inverse)};
            else *to = round4(v[i], s.inverse);
        }
        if (lane == 0) scales[r] = s.scale;
    }
}

struct QuantizeKArgs {
    const uint8_t *x;
    uint8_t *q;
    float *scale;
    int64_t x_stride;      // bytes
    int64_t rows, N;
    int32_t K;
    RowFrames frames;
};

// kLanes threads to a row, up to kPer columns to a thread, which stay in registers as they came.
template <typename E, int kLanes, int kPer>
__global__ __launch_bounds__(kLanes > kThreads ? kLanes : kThreads) void quantize_kernel(const QuantizeKArgs a) {
    constexpr int kV = 16 / sizeof(E), kBlock = kLanes > kThreads ? kLanes : kThreads, kRows = kBlock / kLanes;
    __shared__ uint32_t places[2][kLanes / 64 > 0 ? kLanes / 64 : 1];
    const int tid = threadIdx.x;
    const int lane = tid % kLanes, line = tid / kLanes, columns = a.K / kV;
    int turn = 0;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * kRows; first < a.rows;
         first += static_cast<int64_t>(gridDim.x) * kRows, ++turn) {
        const int64_t row = first + line < a.rows ? first + line : a.rows - 1;
        const uint32_t m = static_cast<uint32_t>(row) / static_cast<uint32_t>(a.N);
        const int64_t in = row - m * a.N;
        const uint8_t *x = a.x + (a.frames.in(m) * a.N + in) * a.x_stride;
        u32x4_t raw[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int col = lane + i * kLanes;
            raw[i] = *reinterpret_cast<const u32x4_t *>(x + (col < columns ? col : columns - 1) * 16);
        }
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t b = raw[i][e];
                if constexpr (sizeof(E) == 4) {
                    top = top > (b & 0x7fffffffu) ? top : b & 0x7fffffffu;
                } else {
                    top = top > ((b << 16) & 0x7fffffffu) ? top : (b << 16) & 0x7fffffffu;
                    top = top > (b & 0x7fff0000u) ? top : b & 0x7fff0000u;
                }
            }
        const RowScale s(lanes_max<kLanes>(top, places, turn));
        if (first + line >= a.rows) continue;
        const int64_t out = a.frames.out(m) * a.N + in;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int col = lane + i * kLanes;
            if (col >= columns) break;
            float v[kV];
            widen<E>(raw[i], v);
            uint32_t *to = reinterpret_cast<uint32_t *>(a.q + out * a.K + col * kV);
            if constexpr (kV == 8) *reinterpret_cast<u32x2_t *>(to) = u32x2_t{round4(v, s.inverse), round4(v + 4, s.inverse)};
            else *to = round4(v, s.inverse);
        }
        if (lane == 0) a.scale[out] = s.scale;
    }
}

template <typename E>
void rows8(const NormKArgs &a, dim3 grid, hipStream_t stream) {
    const int columns = a.C / (16 / static_cast<int>(sizeof(E)));
    constexpr int kLong = sizeof(E) == 2 ? 4 : 8;      // 32 channels of a thread
    if (columns <= 16) hipLaunchKernelGGL((norm_rows8_kernel<E, 16, 1, 128>), grid, dim3(kThreads), 0, stream, a);
    else if (columns <= 64) hipLaunchKernelGGL((norm_rows8_kernel<E, 64, 1, 512>), grid, dim3(kThreads), 0, stream, a);
    else if (columns <= 64 * kLong) hipLaunchKernelGGL((norm_rows8_kernel<E, 64, kLong, 2048>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((norm_rows8_kernel<E, 256, kLong, RF_NORM_CHANNELS>), grid, dim3(kThreads), 0, stream, a);
}

template <typename E>
hipError_t run_norm(const NormKArgs &a, hipStream_t stream) {
    const int64_t blocks = static_cast<int64_t>(a.M) * a.parts * a.slices;
    const int64_t totals = (static_cast<int64_t>(a.M / a.together) * a.groups + kThreads / 64 - 1) / (kThreads / 64);
    if (blocks > 0xffffff || totals > 0xffffff) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(norm_stats_kernel<E>, dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(norm_total_kernel<E>, dim3(static_cast<uint32_t>(totals)), dim3(kThreads), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.y_scale) rows8<E>(a, dim3(static_cast<uint32_t>(a.M) * a.parts), stream);
    else hipLaunchKernelGGL(norm_rows_kernel<E>, dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

template <typename E>
hipError_t run_quantize(const QuantizeKArgs &a, hipStream_t stream) {
    const int64_t columns = a.K / (16 / static_cast<int>(sizeof(E)));
    auto grid = [&](int per_block) {
        const int64_t n = (a.rows + per_block - 1) / per_block;
        return dim3(static_cast<uint32_t>(n < (1 << 20) ? n : 1 << 20));
    };
    if (columns <= 8) hipLaunchKernelGGL((quantize_kernel<E, 8, 1>), grid(32), dim3(256), 0, stream, a);
    else if (columns <= 64) hipLaunchKernelGGL((quantize_kernel<E, 64, 1>), grid(4), dim3(256), 0, stream, a);
    else if (columns <= 256) hipLaunchKernelGGL((quantize_kernel<E, 64, 4>), grid(4), dim3(256), 0, stream, a);
    else if (columns <= 1024) hipLaunchKernelGGL((quantize_kernel<E, 256, 4>), grid(1), dim3(256), 0, stream, a);
    else if (columns <= 4096) hipLaunchKernelGGL((quantize_kernel<E, 256, 16>), grid(1), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((quantize_kernel<E, 1024, 16>), grid(1), dim3(1024), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

int64_t norm_workspace(int32_t M, int64_t N, int32_t C, int32_t groups, int32_t together, bool, int32_t dtype,
                       int32_t cus) {
    return norm_plan(M, N, C, groups, together, dtype, cus).ws_bytes;
}

hipError_t launch_norm(const NormParams &p, hipStream_t stream) {
    if (p.geo.cus < 1) return hipErrorInvalidValue;
    const NormPlan plan = norm_plan(p.M, p.N, p.C, p.groups, p.together, p.dtype, p.geo.cus);
    const int64_t esize = p.dtype == RF_F32 ? 4 : 2;
    NormKArgs a{};
    a.x = static_cast<const uint8_t *>(p.x);
    a.y = static_cast<uint8_t *>(p.y);
    a.y_scale = p.y_scale;
    a.weight = p.weight;
    a.bias = p.bias;
    a.partial = static_cast<float2 *>(p.ws);
    a.total = a.partial + plan.entries;
    a.N = p.N;
    a.per_part = plan.per_part;
    a.x_stride = p.x_stride * esize;
    a.y_stride = p.y_scale ? p.y_stride : p.y_stride * esize;
    a.eps = p.eps;
    a.M = p.M;
    a.C = p.C;
    a.groups = p.groups;
    a.together = p.together;
    a.per_group = p.C / p.groups;
    a.cols = plan.cols;
    a.slices = plan.slices;
    a.lines = plan.lines;
    a.parts = plan.parts;
    a.local = plan.local;
    a.activation = p.activation;
    a.affine_rows = p.affine_rows;
    a.frames = p.frames;
    return p.dtype == RF_F32 ? run_norm<float>(a, stream) : run_norm<uint16_t>(a, stream);
}

hipError_t launch_quantize(const QuantizeParams &p, hipStream_t stream) {
    QuantizeKArgs a{};
    a.x = static_cast<const uint8_t *>(p.x);
    a.q = reinterpret_cast<uint8_t *>(p.q);
    a.scale = p.scale;
    a.x_stride = p.x_stride * (p.dtype == RF_F32 ? 4 : 2);
    a.rows = p.M * p.N;
    a.N = p.N;
    a.K = p.K;
    a.frames = p.frames;
    return p.dtype == RF_F32 ? run_quantize<float>(a, stream) : run_quantize<uint16_t>(a, stream);
}

}  // namespace rf
