// Group norm with an activation, channels last, and rows in 8 bits, for gfx950.
//
//   y = act((x - mean) / sqrt(var + eps) * weight + bias),   mean, var over rows x channels of a group
//   scale = max |x| / 127,  q = x * (127 / max |x|) to the nearest integer
//
//  * norm_slice_kernel: where all rows that share statistics fit, a few groups' channels of them, a
//    workgroup's LDS: x is read once, in one launch.
//  * norm_stats_kernel: else a workgroup has every parts-th chunk of a frame's rows and up to 256 16-byte
//    columns; a thread keeps its column's channels and walks rows, eight at a time: their mean and
//    squared deviations from it, joined to those so far (a sum of squares about another
//    point than the mean would lose what small deviations around a large mean are). The
//    threads' rows, then the channels of each group, meet in LDS.
//    A mean of fp32 rows is two numbers everywhere, itself and the rest that its rounding left, so that deviations
//    are as exact as the rows are, and values that do not deviate come out as 0 (summed and held in one number, 192 rows x 16
//    channels of 10,000.3 normalise to 0.29 with eps 1e-5). Sums of bf16 rows have the bits to spare.
//  * norm_total_kernel: a wave joins the parts of a group; where these are few, each workgroup of the
//    next kernel does so itself.
//  * norm_rows_kernel: x again, to y; norm_rows8_kernel: whole rows at a time, to 8 bits.
//  * quantize_kernel: rows of x to 8 bits. (fp32 rows of more than 16,384 features, 16 columns to each of 1,024
//    threads, leave 18 of a lane's registers in memory: 148 us at 5,120 x 20,480, 3.6 TB/s, where 5,120 x 16,384
//    takes 82, 5.1 TB/s.)
//
// What bounds them, and what they measure (bf16 but for the first):
//  * Slices: what one launch takes, its loads, two sums through LDS and its stores one after the other:
//    6.7 us at 3 x 64 rows x 128 channels of fp32, 9.3 at 3 x 527 x 320.
//  * Short launches (6 x 1,560 rows x 640 channels, 12 MB: 7, 3 and 8 us, 18.2 together): their starts and ends
//    and the parts' way from one to the next; 12 MB in and out take 4 us at the rate of a large copy.
//  * Large ones: memory, x read twice as it does not fit the chip: 5 x 24,960 rows x 512 channels, 128 MB in and
//    out, 66 to 73 us (the second time it is in the caches behind the L2s in part), 409 MB 200, 6.1 TB/s.
//  * Rows to 8 bits: memory, with about ten vector instructions an element beside three bytes: 21,600 x 20,480,
//    227 us, 5.9 TB/s, vector instructions busy 63 % of the cycles.
#include "rf_norm_plan.h"
#include "rf_rows.h"

namespace rf {
namespace {

constexpr int kThreads = kNormThreads;
struct NormKArgs {
    const uint8_t *x;
    uint8_t *y;
    float *y_scale;
    const void *weight, *bias;
    float2 *partial;               // [M][parts][slices][local]: mean, sum of squared deviations
    float2 *total;                 // [M / together][groups]: mean, 1 / deviation
    float *partial_rest, *total_rest;   // of fp32 rows: what the means' rounding left
    int64_t N;
    int64_t x_stride, y_stride;    // bytes
    double eps;
    int32_t M, C, groups, together, per_group;
    int32_t cols, slices, lines, hold, parts, row_parts, local;
    float per_col, group_share;    // 1 / cols, 1 / per_group
    NormParts runs;
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

// A column of x; kPast: past the caches.
template <bool kPast>
__device__ __forceinline__ u32x4_t load_x(const uint8_t *p) {
    if constexpr (kPast) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p));
    else return *reinterpret_cast<const u32x4_t *>(p);
}

// The same of means in two numbers, mean + rest.
__device__ __forceinline__ void join(float n, float &mean, float &rest, float &m2, float n_b, float mean_b, float rest_b,
                                     float m2_b, float share_b) {
    const float far = mean_b - mean, near = rest_b - rest, d = far + near, step = far * share_b, sum = mean + step;
    rest = fmaf(near, share_b, rest) + (step - (sum - mean));
    mean = sum;
    m2 += fmaf(d * d, n * share_b, m2_b);
}

template <typename E>
__global__ __launch_bounds__(kThreads) void norm_stats_kernel(const NormKArgs a) {
    constexpr int kV = 16 / sizeof(E);
    constexpr bool kRest = sizeof(E) == 4;
    // (a channel's columns a bank on from the one's before: neighbouring channels are read together)
    __shared__ float s_mean[kV][kThreads + 1], s_m2[kV][kThreads + 1], s_n[kThreads];
    __shared__ float s_rest[kRest ? kV : 1][kRest ? kThreads + 1 : 1];
    const int tid = threadIdx.x, slice = blockIdx.x, part = blockIdx.y, m = blockIdx.z;
    const int line = divide(tid, a.per_col), col = tid - line * a.cols, column = slice * a.cols + col;
    const bool active = line < a.lines && column * kV < a.C;
    const int chunk = a.lines * kNormRows;
    float n = 0.0f, mean[kV], m2[kV];
    [[maybe_unused]] float rest[kV];
#pragma unroll
    for (int e = 0; e < kV; ++e) mean[e] = m2[e] = rest[e] = 0.0f;
    if (active) {
        const uint8_t *const x = a.x + a.frames.in(m) * a.N * a.x_stride + column * 16;
        const int64_t step = a.lines * a.x_stride;
        for (int64_t first = static_cast<int64_t>(part) * chunk; first < a.N; first += static_cast<int64_t>(a.parts) * chunk) {
            const uint8_t *p = x + (first + line) * a.x_stride;
            if (first + chunk <= a.N) {
                u32x4_t raw[kNormRows];
#pragma unroll
                for (int i = 0; i < kNormRows; ++i) raw[i] = load_x<false>(p + i * step);
                float v[kNormRows][kV];
#pragma unroll
                for (int i = 0; i < kNormRows; ++i) widen<E>(raw[i], v[i]);
                const float share = kNormRows / (n + kNormRows);
#pragma unroll
                for (int e = 0; e < kV; ++e) {
                    float s = 0.0f, q = 0.0f;
#pragma unroll
                    for (int i = 0; i < kNormRows; ++i) s += v[i][e];
                    s *= 1.0f / kNormRows;
                    if constexpr (kRest) {
                        // (deviations about a mean that is off by their mean, which their squares are then too many by)
                        float off = 0.0f;
#pragma unroll
                        for (int i = 0; i < kNormRows; ++i) {
                            off += v[i][e] - s;
                            q = fmaf(v[i][e] - s, v[i][e] - s, q);
                        }
                        q = fmaf(off * (-1.0f / kNormRows), off, q);
                        join(n, mean[e], rest[e], m2[e], kNormRows, s, off * (1.0f / kNormRows), q, share);
                    } else {
#pragma unroll
                        for (int i = 0; i < kNormRows; ++i) q = fmaf(v[i][e] - s, v[i][e] - s, q);
                        join(n, mean[e], m2[e], kNormRows, s, q, share);
                    }
                }
                n += kNormRows;
            } else {      // the frame's last rows, one by one (but in flight together)
                u32x4_t raw[kNormRows];
#pragma unroll
                for (int i = 0; i < kNormRows; ++i) {
                    const int64_t r = first + line + i * a.lines;
                    raw[i] = load_x<false>(x + (r < a.N ? r : a.N - 1) * a.x_stride);
                }
#pragma unroll
                for (int i = 0; i < kNormRows; ++i) {
                    if (first + line + i * a.lines >= a.N) continue;
                    float v[kV];
                    widen<E>(raw[i], v);
                    const float share = 1.0f / (n + 1.0f);
#pragma unroll
                    for (int e = 0; e < kV; ++e) {
                        if constexpr (kRest) join(n, mean[e], rest[e], m2[e], 1.0f, v[e], 0.0f, 0.0f, share);
                        else join(n, mean[e], m2[e], 1.0f, v[e], 0.0f, share);
                    }
                    n += 1.0f;
                }
            }
        }
    }
    s_n[tid] = n;
#pragma unroll
    for (int e = 0; e < kV; ++e) {
        s_mean[e][tid] = mean[e];
        s_m2[e][tid] = m2[e];
        if constexpr (kRest) s_rest[e][tid] = rest[e];
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
                    if constexpr (kRest) {
                        join(n, mean[e], rest[e], m2[e], n_b, s_mean[e][other], s_rest[e][other], s_m2[e][other], share);
                        s_rest[e][tid] = rest[e];
                    } else {
                        join(n, mean[e], m2[e], n_b, s_mean[e][other], s_m2[e][other], share);
                    }
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
    const int g0 = divide(c0, a.group_share), n_local = divide(c1 - 1, a.group_share) - g0 + 1;
    int lanes = 1;
    while (lanes < 64 && 2 * lanes * n_local <= kThreads) lanes *= 2;
    const int lane = tid % lanes;
    const float rows = a.runs.rows(part);
    for (int l = tid / lanes; l < n_local; l += kThreads / lanes) {
        const int first = (g0 + l) * a.per_group, behind = first + a.per_group;
        const int lo = (first > c0 ? first : c0) - c0, hi = (behind < c1 ? behind : c1) - c0;
        float s = 0.0f, q = 0.0f;
        [[maybe_unused]] float left = 0.0f;
        if constexpr (kRest) {
            double sum = 0.0;
            for (int c = lo + lane; c < hi; c += lanes)
                sum += static_cast<double>(s_mean[c % kV][c / kV]) + static_cast<double>(s_rest[c % kV][c / kV]);
            for (int d = lanes / 2; d > 0; d /= 2) sum += __shfl_xor(sum, d);
            sum /= static_cast<double>(hi - lo);
            s = static_cast<float>(sum);
            left = static_cast<float>(sum - static_cast<double>(s));
        } else {
            for (int c = lo + lane; c < hi; c += lanes) s += s_mean[c % kV][c / kV];
            for (int d = lanes / 2; d > 0; d /= 2) s += __shfl_xor(s, d);
            s /= static_cast<float>(hi - lo);
        }
        for (int c = lo + lane; c < hi; c += lanes) {
            float d = s_mean[c % kV][c / kV] - s;
            if constexpr (kRest) d += s_rest[c % kV][c / kV] - left;
            q += fmaf(rows * d, d, s_m2[c % kV][c / kV]);
        }
        for (int d = lanes / 2; d > 0; d /= 2) q += __shfl_xor(q, d);
        if (lane == 0) {
            const int64_t at = ((static_cast<int64_t>(m) * a.parts + part) * a.slices + slice) * a.local + l;
            a.partial[at] = make_float2(s, q);
            if constexpr (kRest) a.partial_rest[at] = left;
        }
    }
}

// Mean and 1 / deviation of n_groups groups from g0 on, of the frames of a segment, by kBlock threads (of fp32 rows
// what the mean's rounding left besides): lanes together join a group's parts, in 64 bits and one order: sums of the
// parts' means and their squares about the first part's (64 bits lose nothing there that 32 had).
template <typename E, int kBlock>
__device__ __forceinline__ void totals(const NormKArgs &a, int seg, int g0, int n_groups, float2 *to, float *rest_to) {
    constexpr int kV = 16 / sizeof(E);
    constexpr bool kRest = sizeof(E) == 4;
    int lanes = 1;
    while (lanes < 64 && 2 * lanes * n_groups <= kBlock) lanes *= 2;
    const int lane = threadIdx.x % lanes, width = a.cols * kV, runs = a.together * a.parts;
    const int64_t step = static_cast<int64_t>(a.slices) * a.local;
    const double all = static_cast<double>(a.together) * static_cast<double>(a.N) * a.per_group;
    for (int l = threadIdx.x / lanes; l < n_groups; l += kBlock / lanes) {
        const int first = (g0 + l) * a.per_group, behind = first + a.per_group, s0 = divide(first, a.per_col * (1.0f / kV));
        double pivot = 0.0, sum = 0.0, square = 0.0;
        for (int s = s0; s * width < behind; ++s) {
            const int c0 = s * width, lo = first > c0 ? first : c0, hi = behind < c0 + width ? behind : c0 + width;
            const int64_t from = (static_cast<int64_t>(seg) * runs * a.slices + s) * a.local + (g0 + l - divide(c0, a.group_share));
            const float2 *p = a.partial + from;
            if (s == s0) pivot = p->x;
            int part = lane;
            while (part >= a.parts) part -= a.parts;
#pragma unroll 8
            for (int i = lane; i < runs; i += lanes) {
                const float2 v = p[i * step];
                const double n = a.runs.rows(part) * static_cast<float>(hi - lo);
                double d = v.x - pivot;
                if constexpr (kRest) d += static_cast<double>(a.partial_rest[from + i * step]);
                sum += n * d;
                square += n * d * d + v.y;
                part += lanes;
                while (part >= a.parts) part -= a.parts;
            }
        }
        for (int d = lanes / 2; d > 0; d /= 2) {
            sum += __shfl_xor(sum, d);
            square += __shfl_xor(square, d);
        }
        const double m = sum / all, var = square / all - m * m;
        if (lane == 0) {
            const float mean = static_cast<float>(pivot + m);
            to[l] = make_float2(mean, static_cast<float>(rsqrt((var < 0.0 ? 0.0 : var) + a.eps)));
            if constexpr (kRest) rest_to[l] = static_cast<float>(pivot - static_cast<double>(mean) + m);
        }
    }
}

// A wave to a group.
template <typename E>
__global__ __launch_bounds__(64) void norm_total_kernel(const NormKArgs a) {
    const int g = blockIdx.x, seg = blockIdx.y;
    const int64_t at = static_cast<int64_t>(seg) * a.groups + g;
    totals<E, 64>(a, seg, g, 1, a.total + at, a.total_rest + at);
}

// What kV channels from c on of listed frame m are normalised with, (x - mean) * mul + add; total and rests: of the
// groups from g0 on.
template <typename E>
__device__ __forceinline__ void affine_at(const NormKArgs &a, int m, int c, const float2 *total, const float *rests, int g0,
                                          float (&mean)[16 / sizeof(E)], float (&mul)[16 / sizeof(E)],
                                          float (&add)[16 / sizeof(E)]) {
    constexpr int kV = 16 / sizeof(E);
    constexpr bool kRest = sizeof(E) == 4;
    [[maybe_unused]] float rest[kV];
    const int64_t at = (a.affine_rows ? static_cast<int64_t>(frame_at(a.frames, m)) * a.C : 0) + c;
#pragma unroll
    for (int e = 0; e < kV; ++e) {
        mul[e] = 1.0f;
        add[e] = 0.0f;
    }
    if (a.weight) load_n<E, kV>(a.weight, at, mul);
    if (a.bias) load_n<E, kV>(a.bias, at, add);
    if (2 * a.per_group >= kV) {      // (three groups at most: 200 us at 4 x 399,360 x 128, 32 groups, 202 with a load a channel)
        const int first = divide(c, a.group_share), last = divide(c + kV - 1, a.group_share);
        const float2 t = total[first - g0], t2 = total[(first < last ? first + 1 : last) - g0], t3 = total[last - g0];
        const int border = (first + 1) * a.per_group - c, border2 = border + a.per_group;
#pragma unroll
        for (int e = 0; e < kV; ++e) {
            mean[e] = e < border ? t.x : e < border2 ? t2.x : t3.x;
            mul[e] *= e < border ? t.y : e < border2 ? t2.y : t3.y;
        }
        if constexpr (kRest) {
            const float r = rests[first - g0], r2 = rests[(first < last ? first + 1 : last) - g0], r3 = rests[last - g0];
#pragma unroll
            for (int e = 0; e < kV; ++e) rest[e] = e < border ? r : e < border2 ? r2 : r3;
        }
    } else {
        float2 t[kV];
#pragma unroll
        for (int e = 0; e < kV; ++e) {
            t[e] = total[divide(c + e, a.group_share) - g0];
            if constexpr (kRest) rest[e] = rests[divide(c + e, a.group_share) - g0];
        }
#pragma unroll
        for (int e = 0; e < kV; ++e) {
            mean[e] = t[e].x;
            mul[e] *= t[e].y;
        }
    }
    if constexpr (kRest) {
#pragma unroll
        for (int e = 0; e < kV; ++e) add[e] = fmaf(-rest[e], mul[e], add[e]);
    }
}

// A workgroup's threads hold kV channels each, `cols` threads to a line, `lines` lines: done(group of the
// slice, sum of its values) for every group, by one thread. Channels first, a thread to a channel and
// as many of them as there are threads to share out its lines, then a group's channels, lanes
// together. `lines * cols * kV` floats of `all` and kBlock of `some` are its own.
template <int kV, int kBlock, typename Done>
__device__ __forceinline__ void group_sums(const float (&v)[kV], int line, int cols, int lines, int per_group, int n_groups,
                                           int shares, float channel_share, float *all, float *some, Done done) {
    const int tid = threadIdx.x, channels = cols * kV;
    if (line < lines) {
#pragma unroll
        for (int e = 0; e < kV; e += 4)
            *reinterpret_cast<f32x4_t *>(all + tid * kV + e) = f32x4_t{v[e], v[e + 1], v[e + 2], v[e + 3]};
    }
    __syncthreads();
    for (int t = tid; t < channels * shares; t += kBlock) {
        const int share = divide(t, channel_share), c = t - share * channels;
        float s = 0.0f;
#pragma unroll 4
        for (int l = share; l < lines; l += shares) s += all[l * channels + c];
        if (shares == 1) all[c] = s;      // (line 0's place of this channel, which no other thread reads)
        else some[c * shares + share] = s;
    }
    __syncthreads();
    const float *from = shares == 1 ? all : some;
    int lanes = 1;
    while (lanes < 64 && 2 * lanes * n_groups <= kBlock) lanes *= 2;
    for (int g = tid / lanes; g < n_groups; g += kBlock / lanes) {
        float s = 0.0f;
#pragma unroll 4
        for (int i = tid % lanes; i < per_group * shares; i += lanes) s += from[g * per_group * shares + i];
        for (int d = lanes / 2; d > 0; d /= 2) s += __shfl_xor(s, d);
        if (tid % lanes == 0) done(g, s);
    }
    __syncthreads();
}

// A value that stays as it is: what was made of it before is not kept for what follows (else the
// compiler holds bf16 values widened, at twice the registers, or spills them).
__device__ __forceinline__ void pin(u32x4_t &x) { asm volatile("" : "+v"(x)); }

// Whole groups' columns of all rows that share their statistics, up to kHold rows of a thread, straight
// from memory into LDS, where they stay: the mean, then the squared deviations from it, then the
// results. (Held in registers they need loops unrolled to their end, 77 KB of code that a short launch
// waits for: 10.3 us at 3 x 527 rows x 320 channels.)
template <typename E, int kHold, int kBlock>
__global__ __launch_bounds__(kBlock) void norm_slice_kernel(const NormKArgs a) {
    constexpr int kV = 16 / sizeof(E);
    __shared__ __attribute__((aligned(1024))) uint8_t held[kHold * kBlock * 16];
    constexpr bool kRest = sizeof(E) == 4;
    __shared__ __attribute__((aligned(16))) float all[kBlock * kV], some[kBlock], mean[kNormSliceGroups],
        inverse[kNormSliceGroups], rest[kRest ? kNormSliceGroups : 1];
    const int tid = threadIdx.x;
    const int slice = blockIdx.x, seg = blockIdx.y;
    const int line = divide(tid, a.per_col), col = tid - line * a.cols, column = slice * a.cols + col;
    const uint32_t N = static_cast<uint32_t>(a.N), rows = N * static_cast<uint32_t>(a.together);
    // This thread's i-th row, i < a.hold: line + i lines, in frame f of the segment; the last may be past
    // the end, then the last row is loaded (as by the threads behind the last line, whose sums nobody reads).
    auto row_of = [&](int i, uint32_t &f) {
        uint32_t r = line + i * a.lines;
        r = r < rows ? r : rows - 1;
        f = a.together > 1 ? r / N : 0;
        return r - f * N;
    };
    uint8_t *const to = held + __builtin_amdgcn_readfirstlane(tid / 64) * 1024;
#pragma unroll 1
    for (int i = 0; i < a.hold; ++i) {
        uint32_t f;
        const uint32_t r = row_of(i, f);
        global_lds16(a.x + (a.frames.in(seg * a.together + f) * a.N + r) * a.x_stride + column * 16, to + i * (kBlock * 16));
    }
    int local[kV];
#pragma unroll
    for (int e = 0; e < kV; ++e) local[e] = divide(col * kV + e, a.group_share);
    float weight[kV], bias[kV];
#pragma unroll
    for (int e = 0; e < kV; ++e) {
        weight[e] = 1.0f;
        bias[e] = 0.0f;
    }
    auto affine = [&](int m) {
        const int64_t at = (a.affine_rows ? static_cast<int64_t>(a.frames.frame[m]) * a.C : 0) + column * kV;
        if (a.weight) load_n<E, kV>(a.weight, at, weight);
        if (a.bias) load_n<E, kV>(a.bias, at, bias);
    };
    const bool each = a.affine_rows && a.together > 1;   // (then a row's frame has its own)
    if (!each) affine(seg * a.together);
    const int mine = line + (a.hold - 1) * a.lines < static_cast<int>(rows) ? a.hold : a.hold - 1;
    // threads to a channel of group_sums
    const int channels = a.cols * kV, n_groups = divide(channels, a.group_share);
    const float channel_share = a.per_col * (1.0f / kV);
    const int shares = channels < kBlock ? divide(kBlock, channel_share) : 1;
    const double share = 1.0 / (static_cast<double>(rows) * a.per_group);
    auto row = [&](int i, float (&v)[kV]) {
        widen<E>(*reinterpret_cast<const u32x4_t *>(held + (i * kBlock + tid) * 16), v);
    };
    wait_loads<0>();   // (a thread reads its own rows only)
    float s[kV], mu[kV];
    // fp32 values are summed as what they are above their group's first one in the segment's first row
    [[maybe_unused]] float above[kV];
    auto first_of = [&](int g) {
        const int c = g * a.per_group;
        return *reinterpret_cast<const float *>(held + c / kV * 16 + c % kV * 4);
    };
    if constexpr (kRest) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kV; ++e) above[e] = first_of(local[e]);
    }
#pragma unroll
    for (int e = 0; e < kV; ++e) s[e] = 0.0f;
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
        float v[kV];
        row(i, v);
#pragma unroll
        for (int e = 0; e < kV; ++e) s[e] += kRest ? v[e] - above[e] : v[e];
    }
    group_sums<kV, kBlock>(s, line, a.cols, a.lines, a.per_group, n_groups, shares, channel_share, all, some,
                           [&](int g, float sum) {
                               if constexpr (kRest) {
                                   const double m = static_cast<double>(first_of(g)) + sum * share;
                                   mean[g] = static_cast<float>(m);
                                   rest[g] = static_cast<float>(m - static_cast<double>(mean[g]));
                               } else {
                                   mean[g] = static_cast<float>(sum * share);
                               }
                           });
#pragma unroll
    for (int e = 0; e < kV; ++e) {
        mu[e] = mean[local[e]];
        s[e] = 0.0f;
    }
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
        float v[kV];
        row(i, v);
#pragma unroll
        for (int e = 0; e < kV; ++e) s[e] = fmaf(v[e] - mu[e], v[e] - mu[e], s[e]);
    }
    group_sums<kV, kBlock>(s, line, a.cols, a.lines, a.per_group, n_groups, shares, channel_share, all, some,
                           [&](int g, float sum) {
                               double var = sum * share;
                               if constexpr (kRest) {      // (of deviations from the mean without its rest)
                                   var -= static_cast<double>(rest[g]) * static_cast<double>(rest[g]);
                                   var = var < 0.0 ? 0.0 : var;
                               }
                               inverse[g] = static_cast<float>(rsqrt(var + a.eps));
                           });
    if (line >= a.lines) return;
    float mul[kV], add[kV];
    auto factors = [&]() {
#pragma unroll
        for (int e = 0; e < kV; ++e) {
            mul[e] = inverse[local[e]] * weight[e];
            add[e] = kRest ? fmaf(-rest[kRest ? local[e] : 0], mul[e], bias[e]) : bias[e];
        }
    };
    with_activation(a.activation, [&](auto act) {
        factors();
#pragma unroll 1
        for (int i = 0; i < mine; ++i) {
            uint32_t f;
            const uint32_t r = row_of(i, f);
            const int m = seg * a.together + static_cast<int>(f);
            if (each) {
                affine(m);
                factors();
            }
            float v[kV];
            row(i, v);
#pragma unroll
            for (int e = 0; e < kV; ++e) v[e] = fmaf(v[e] - mu[e], mul[e], add[e]);
            if constexpr (act.kind != RF_ACT_NONE) activate_fitted(act.kind, v);
            store_n<E, kV>(a.y + (a.frames.out(m) * a.N + r) * a.y_stride + column * 16, 0, v);
        }
    });
}

// A column's results past the caches.
template <typename E, int kN>
__device__ __forceinline__ void stream_n(void *p, const float (&v)[kN]) {
    if constexpr (kN == 8) stream_8<E>(p, 0, v);
    else __builtin_nontemporal_store((f32x4_t{v[0], v[1], v[2], v[3]}), static_cast<f32x4_t *>(p));
}

template <typename E, bool kStream, bool kPast, bool kOwn>
__global__ __launch_bounds__(kThreads) void norm_rows_kernel(const NormKArgs a) {
    constexpr int kV = 16 / sizeof(E);
    const int tid = threadIdx.x, slice = blockIdx.x, part = blockIdx.y, m = blockIdx.z;
    const int line = divide(tid, a.per_col), col = tid - line * a.cols, column = slice * a.cols + col;
    __shared__ float2 own[kOwn ? kNormFewGroups : 1];
    __shared__ float own_rest[kOwn && sizeof(E) == 4 ? kNormFewGroups : 1];
    const int64_t segment = static_cast<int64_t>(m / a.together) * a.groups;
    const float2 *total = a.total + segment;
    const float *rests = a.total_rest + segment;
    int g0 = 0;
    if constexpr (kOwn) {
        const int c0 = slice * a.cols * kV, c1 = c0 + a.cols * kV < a.C ? c0 + a.cols * kV : a.C;
        g0 = divide(c0, a.group_share);
        totals<E, kThreads>(a, m / a.together, g0, divide(c1 - 1, a.group_share) - g0 + 1, own, own_rest);
        total = own;
        rests = own_rest;
        __syncthreads();
    }
    if (line >= a.lines || column * kV >= a.C) return;
    float mean[kV], mul[kV], add[kV];
    affine_at<E>(a, m, column * kV, total, rests, g0, mean, mul, add);
    // (y may be x: no row is read again)
    const uint8_t *p = a.x + (a.frames.in(m) * a.N) * a.x_stride + column * 16;
    uint8_t *q = a.y + (a.frames.out(m) * a.N) * a.y_stride + column * 16;
    // From the frame's last rows to its first, the other way than the statistics' kernel went: what
    // that read last is in the caches still.
    constexpr int kRows = 4;
    const int chunk = kRows * a.lines;
    const int64_t chunks = (a.N + chunk - 1) / chunk;
    with_activation(a.activation, [&](auto act) {
        for (int64_t at = chunks - 1 - part; at >= 0; at -= a.row_parts) {
            const int64_t r = at * chunk + line;
            u32x4_t raw[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int64_t k = r + i * a.lines;
                raw[i] = load_x<kPast>(p + (k < a.N ? k : a.N - 1) * a.x_stride);
            }
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int64_t k = r + i * a.lines;
                if (k >= a.N) break;
                float v[kV];
                widen<E>(raw[i], v);
#pragma unroll
                for (int e = 0; e < kV; ++e) v[e] = fmaf(v[e] - mean[e], mul[e], add[e]);
                if constexpr (act.kind != RF_ACT_NONE) activate_fitted(act.kind, v);
                if constexpr (kStream) stream_n<E, kV>(q + k * a.y_stride, v);
                else store_n<E, kV>(q + k * a.y_stride, 0, v);
            }
        }
    });
}

// The larger of each lane's value and that of the lane kDpp names (0 where there is none).
template <int kDpp, int kRows>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    const uint32_t o = __builtin_amdgcn_update_dpp(0, v, kDpp, kRows, 0xf, false);
    return v > o ? v : o;
}
// The largest of kLanes neighbouring lanes' values (kLanes > 64: of all of the workgroup's kLanes
// threads, through LDS; `turn` takes two places in turn, so that one barrier does).
template <int kLanes>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v, uint32_t (*places)[kLanes / 64 > 0 ? kLanes / 64 : 1], int turn) {
    if constexpr (kLanes < 64) {
#pragma unroll
        for (int d = 1; d < kLanes; d *= 2) {
            const uint32_t o = __shfl_xor(v, d);
            v = v > o ? v : o;
        }
    } else {
        // rows of 16 lanes to their last lane, that to the next rows', lane 63 has all
        v = dpp_max<0x111, 0xf>(v);      // row_shr 1, 2, 4, 8
        v = dpp_max<0x112, 0xf>(v);
        v = dpp_max<0x114, 0xf>(v);
        v = dpp_max<0x118, 0xf>(v);
        v = dpp_max<0x142, 0xa>(v);      // row_bcast 15 into rows 1 and 3
        v = dpp_max<0x143, 0xc>(v);      // row_bcast 31 into rows 2 and 3
        v = __builtin_amdgcn_readlane(v, 63);
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

// kLanes threads to a row, kPer columns to a thread, lane after lane. What they are normalised with stays
// in registers; so does the row until its scale is known.
template <typename E, int kLanes, int kPer, bool kPast, bool kOwn>
__global__ __launch_bounds__(kThreads) void norm_rows8_kernel(const NormKArgs a) {
    constexpr int kV = 16 / sizeof(E), kRows = kThreads / kLanes;
    __shared__ uint32_t places[2][kLanes / 64 > 0 ? kLanes / 64 : 1];
    const int tid = threadIdx.x;
    const int part = blockIdx.x, m = blockIdx.y;
    const int lane = tid % kLanes, line = tid / kLanes, columns = a.C / kV;
    const uint8_t *x = a.x + (a.frames.in(m) * a.N) * a.x_stride;
    uint8_t *y = a.y + (a.frames.out(m) * a.N) * a.C;
    float *scales = a.y_scale + a.frames.out(m) * a.N;
    // (columns past the last are the last once more)
    float mean[kPer][kV], mul[kPer][kV], add[kPer][kV];
    __shared__ float2 own[kOwn ? kNormFewGroups : 1];
    __shared__ float own_rest[kOwn && sizeof(E) == 4 ? kNormFewGroups : 1];
    const int64_t segment = static_cast<int64_t>(m / a.together) * a.groups;
    const float2 *total = a.total + segment;
    const float *rests = a.total_rest + segment;
    if constexpr (kOwn) {
        totals<E, kThreads>(a, m / a.together, 0, a.groups, own, own_rest);
        total = own;
        rests = own_rest;
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int col = lane + i * kLanes;
        affine_at<E>(a, m, (col < columns ? col : columns - 1) * kV, total, rests, 0, mean[i], mul[i], add[i]);
    }
    with_activation(a.activation, [&](auto act) {
        int turn = 0;
        const int64_t rounds = (a.N + kRows - 1) / kRows;
        // (a row ahead: the next one's columns are on their way while this one's are rounded)
        u32x4_t next[kPer];
        auto ahead = [&](int64_t at) {
            const int64_t r = at * kRows + line;
            const uint8_t *p = x + (at < 0 ? 0 : r < a.N ? r : a.N - 1) * a.x_stride;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int col = lane + i * kLanes;
                next[i] = load_x<kPast>(p + (col < columns ? col : columns - 1) * 16);
            }
        };
        ahead(rounds - 1 - part);
        for (int64_t at = rounds - 1 - part; at >= 0; at -= a.row_parts, ++turn) {
            const int64_t first = at * kRows, r = first + line < a.N ? first + line : a.N - 1;
            u32x4_t raw[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) raw[i] = next[i];
            ahead(at - a.row_parts);
            float v[kPer][kV];
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                widen<E>(raw[i], v[i]);
#pragma unroll
                for (int e = 0; e < kV; ++e) v[i][e] = fmaf(v[i][e] - mean[i][e], mul[i][e], add[i][e]);
                if constexpr (act.kind != RF_ACT_NONE) activate_fitted(act.kind, v[i]);
#pragma unroll
                for (int e = 0; e < kV; ++e) {
                    const uint32_t bits = __float_as_uint(v[i][e]) & 0x7fffffffu;
                    top = top > bits ? top : bits;
                }
            }
            const RowScale s(lanes_max<kLanes>(top, places, turn));
            if (first + line >= a.N) continue;
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
    });
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

// kLanes threads to a row, up to kPer columns to a thread, which stay in registers as they came (but for 18 of the
// widest fp32 form's).
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
#pragma unroll
        for (int i = 0; i < kPer; ++i) pin(raw[i]);
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

template <typename E, bool kPast, bool kOwn>
void rows8(const NormKArgs &a, dim3 grid, hipStream_t stream) {
    // eights of channels to a thread
    constexpr int kEight = sizeof(E) / 2;
    auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a); };
    if (a.C <= 128) run(norm_rows8_kernel<E, 16, kEight, kPast, kOwn>);
    else if (a.C <= 512) run(norm_rows8_kernel<E, 64, kEight, kPast, kOwn>);
    else if (a.C <= 1024) run(norm_rows8_kernel<E, 64, 2 * kEight, kPast, kOwn>);
    else if (a.C <= 1536) run(norm_rows8_kernel<E, 64, 3 * kEight, kPast, kOwn>);
    else if (a.C <= 2048) run(norm_rows8_kernel<E, 64, 4 * kEight, kPast, kOwn>);
    else if (a.C <= 4096) run(norm_rows8_kernel<E, 256, 2 * kEight, kPast, kOwn>);
    else if (a.C <= 6144) run(norm_rows8_kernel<E, 256, 3 * kEight, kPast, kOwn>);
    else run(norm_rows8_kernel<E, 256, 4 * kEight, kPast, kOwn>);
}

template <typename E>
hipError_t run_slices(const NormPlan &p, const NormKArgs &a, hipStream_t stream) {
    const dim3 grid(a.slices, a.M / a.together);
    if (p.block == kNormBlocks[0].threads)
        hipLaunchKernelGGL((norm_slice_kernel<E, kNormBlocks[0].hold, kNormBlocks[0].threads>), grid, dim3(p.block), 0, stream, a);
    else
        hipLaunchKernelGGL((norm_slice_kernel<E, kNormBlocks[1].hold, kNormBlocks[1].threads>), grid, dim3(p.block), 0, stream, a);
    return hipGetLastError();
}

template <typename E>
hipError_t run_norm(const NormPlan &p, const NormKArgs &a, hipStream_t stream) {
    hipLaunchKernelGGL(norm_stats_kernel<E>, dim3(a.slices, a.parts, a.M), dim3(kThreads), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (!p.few_parts) {
        hipLaunchKernelGGL(norm_total_kernel<E>, dim3(a.groups, a.M / a.together), dim3(64), 0, stream, a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 grid8(a.row_parts, a.M), grid(a.slices, a.row_parts, a.M);
    auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a); };
    if (a.y_scale && p.x_past) p.few_parts ? rows8<E, true, true>(a, grid8, stream) : rows8<E, true, false>(a, grid8, stream);
    else if (a.y_scale) p.few_parts ? rows8<E, false, true>(a, grid8, stream) : rows8<E, false, false>(a, grid8, stream);
    else if (p.few_parts) run(norm_rows_kernel<E, false, false, true>);
    else if (p.x_past) run(norm_rows_kernel<E, true, true, false>);
    else if (p.y_past) run(norm_rows_kernel<E, true, false, false>);
    else run(norm_rows_kernel<E, false, false, false>);
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
    else hipLaunchKernelGGL((quantize_kernel<E, 1024, sizeof(E) == 2 ? 8 : 16>), grid(1), dim3(1024), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

int64_t norm_workspace(int32_t M, int64_t N, int32_t C, int32_t groups, int32_t together, bool rows8, int32_t dtype,
                       int32_t cus) {
    return norm_plan(M, N, C, groups, together, rows8, dtype, cus).ws_bytes;
}

hipError_t launch_norm(const NormParams &p, hipStream_t stream) {
    if (p.geo.cus < 1) return hipErrorInvalidValue;
    const NormPlan plan = norm_plan(p.M, p.N, p.C, p.groups, p.together, p.y_scale != nullptr, p.dtype, p.geo.cus);
    const int64_t esize = p.dtype == RF_F32 ? 4 : 2;
    NormKArgs a{};
    a.x = static_cast<const uint8_t *>(p.x);
    a.y = static_cast<uint8_t *>(p.y);
    a.y_scale = p.y_scale;
    a.weight = p.weight;
    a.bias = p.bias;
    a.partial = static_cast<float2 *>(p.ws);
    a.total = a.partial + plan.entries;
    a.partial_rest = reinterpret_cast<float *>(a.partial + plan.sums);
    a.total_rest = a.partial_rest + plan.sums;
    a.N = p.N;
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
    a.hold = plan.hold;
    a.row_parts = plan.row_parts;
    a.local = plan.local;
    a.per_col = 1.0f / static_cast<float>(plan.cols);
    a.group_share = 1.0f / static_cast<float>(a.per_group);
    a.runs = plan.runs;
    a.activation = p.activation;
    a.affine_rows = p.affine_rows;
    a.frames = p.frames;
    if (plan.block > 0) return p.dtype == RF_F32 ? run_slices<float>(plan, a, stream) : run_slices<uint16_t>(plan, a, stream);
    return p.dtype == RF_F32 ? run_norm<float>(plan, a, stream) : run_norm<uint16_t>(plan, a, stream);
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
