// Matrix product with bias, activation, gate and residual in its epilogue for
// gfx950: y = residual + gate * act(x W^T + bias), on the rows of listed frames.
//
// A workgroup of 256 threads owns 64 x 64 outputs; 16 reduction steps at a
// time go through LDS, a thread owns 4 x 4 outputs.
#include "rf_internal.h"

namespace rf {
namespace {

template <typename E>
__device__ __forceinline__ float widen(E x);
template <>
__device__ __forceinline__ float widen<float>(float x) { return x; }
template <>
__device__ __forceinline__ float widen<uint16_t>(uint16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }

__device__ __forceinline__ void put(float *p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t *p, float x) {
    *p = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
}

__device__ __forceinline__ float activate(int kind, float x) {
    switch (kind) {
        case RF_ACT_GELU: return 0.5f * x * (1.0f + erff(x * 0.70710678f));
        case RF_ACT_GELU_TANH: return 0.5f * x * (1.0f + tanhf(0.79788456f * (x + 0.044715f * x * x * x)));
        case RF_ACT_SILU: return x / (1.0f + expf(-x));
        default: return x;
    }
}

template <typename E>
__global__ __launch_bounds__(256) void linear_kernel(const LinearParams p) {
    __shared__ float xs[16][65], ws[16][65];
    const int64_t rows = p.M * p.N;
    const int64_t r0 = static_cast<int64_t>(blockIdx.y) * 64;
    const int c0 = blockIdx.x * 64;
    const int tid = threadIdx.x, tr = tid / 16, tc = tid % 16;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < p.K; k0 += 16) {
        for (int i = tid; i < 64 * 16; i += 256) {
            const int kk = i % 16, rr = i / 16;
            const int64_t r = r0 + rr;
            float x = 0.0f, w = 0.0f;
            if (r < rows && k0 + kk < p.K) {
                const int64_t m = r / p.N;
                x = widen(static_cast<const E *>(p.x)[(p.src_frame[m] * p.N + (r - m * p.N)) * p.K + k0 + kk]);
            }
            if (c0 + rr < p.n_out && k0 + kk < p.K)
                w = widen(static_cast<const E *>(p.weight)[static_cast<int64_t>(c0 + rr) * p.K + k0 + kk]);
            xs[kk][rr] = x;
            ws[kk][rr] = w;
        }
        __syncthreads();
        for (int kk = 0; kk < 16; ++kk)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = fmaf(xs[kk][tr + 16 * i], ws[kk][tc + 16 * j], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i) {
        const int64_t r = r0 + tr + 16 * i;
        if (r >= rows) continue;
        const int64_t m = r / p.N, dst = p.dst_frame[m] * p.N + (r - m * p.N);
        for (int j = 0; j < 4; ++j) {
            const int c = c0 + tc + 16 * j;
            if (c >= p.n_out) continue;
            float x = acc[i][j];
            if (p.bias) x += widen(static_cast<const E *>(p.bias)[c]);
            x = activate(p.activation, x);
            if (p.gate)
                x *= widen(static_cast<const E *>(p.gate)[static_cast<int64_t>(p.gate_rows ? p.frame[m] : 0) * p.n_out + c]);
            if (p.residual) x += widen(static_cast<const E *>(p.residual)[dst * p.n_out + c]);
            put(static_cast<E *>(p.y) + dst * p.n_out + c, x);
        }
    }
}

}  // namespace

int64_t linear_workspace(int64_t, int32_t, int32_t, int32_t, int32_t) { return 0; }

hipError_t launch_linear(const LinearParams &p, hipStream_t stream) {
    const int64_t by = (p.M * p.N + 63) / 64;
    if (by > 65535) return hipErrorInvalidConfiguration;
    const dim3 grid(static_cast<uint32_t>((p.n_out + 63) / 64), static_cast<uint32_t>(by));
    if (p.dtype == RF_F32) hipLaunchKernelGGL(linear_kernel<float>, grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL(linear_kernel<uint16_t>, grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace rf
