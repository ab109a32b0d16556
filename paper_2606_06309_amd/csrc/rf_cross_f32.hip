// Attention to an encoder's states of another length for gfx950.
//
// One wave per (sequence, head, query): lane l scores keys l, l + 64, ..., the
// running maximum and sum of the softmax are the wave's, and lane l owns every
// 64th dimension of the output.
#include "rf_cross.h"

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

template <typename E, int D>
__global__ __launch_bounds__(256) void cross_kernel(const CrossParams p) {
    __shared__ float qs[4][D];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 4 + wave;
    const int b = blockIdx.z, h = blockIdx.y, hk = h / (p.heads / p.kv_heads);
    const bool live = i < p.Lq;
    const E *q = static_cast<const E *>(p.q) + b * p.qs[0] + i * p.qs[1] + h * p.qs[2];
    if (live)
        for (int d = lane; d < D; d += 64) qs[wave][d] = widen(q[d]);
    __syncthreads();
    if (!live) return;
    const E *k = static_cast<const E *>(p.k) + b * p.ks[0] + hk * p.ks[2];
    const E *v = static_cast<const E *>(p.v) + b * p.vs[0] + hk * p.vs[2];
    int n = p.Lk;
    if (p.kv_lengths) n = p.kv_lengths[b] < 0 ? 0 : p.kv_lengths[b] < p.Lk ? p.kv_lengths[b] : p.Lk;
    const uint8_t *mask = p.key_mask ? p.key_mask + static_cast<int64_t>(b) * p.Lk : nullptr;
    const float scale = static_cast<float>(1.0 / sqrt(static_cast<double>(D)));
    float m = -__builtin_huge_valf(), l = 0.0f, o[D / 64] = {};
    bool any = false;
    for (int j0 = 0; j0 < n; j0 += 64) {
        const int j = j0 + lane;
        const bool ok = j < n && (!mask || mask[j]);
        const uint64_t valid = __ballot(ok);
        if (valid == 0) continue;
        any = true;
        float s = -__builtin_huge_valf();
        if (ok) {
            s = 0.0f;
            for (int d = 0; d < D; ++d) s = fmaf(qs[wave][d], widen(k[j * p.ks[1] + d]), s);
            s *= scale;
        }
        float mx = s;
        for (int x = 32; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor(mx, x));
        mx = fmaxf(m, mx);
        const float ref = mx == -__builtin_huge_valf() ? 0.0f : mx;
        const float corr = m == -__builtin_huge_valf() ? 0.0f : expf(m - ref);
        const float e = ok ? expf(s - ref) : 0.0f;
        float sum = e;
        for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x);
        l = l * corr + sum;
        for (int c = 0; c < D / 64; ++c) o[c] *= corr;
        for (int t = 0; t < 64; ++t) {
            if (!((valid >> t) & 1)) continue;
            const float pt = __shfl(e, t);
            for (int c = 0; c < D / 64; ++c) o[c] = fmaf(pt, widen(v[(j0 + t) * p.vs[1] + lane + 64 * c]), o[c]);
        }
        m = mx;
    }
    E *out = static_cast<E *>(p.out) + b * p.os[0] + i * p.os[1] + h * p.os[2];
    for (int c = 0; c < D / 64; ++c) put(out + lane + 64 * c, any ? o[c] / l : 0.0f);
}

}  // namespace

hipError_t launch_cross_f32(const CrossParams &p, const CrossKArgs &, hipStream_t stream) {
    const int64_t blocks = (static_cast<int64_t>(p.Lq) + 3) / 4;
    if (blocks > 0x7fffffffLL || p.heads > 65535 || p.B > 65535) return hipErrorInvalidConfiguration;
    const dim3 grid(static_cast<uint32_t>(blocks), p.heads, p.B);
    if (p.head_dim == 128) hipLaunchKernelGGL((cross_kernel<float, 128>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((cross_kernel<float, 64>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace rf
