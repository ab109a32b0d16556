// Elements of rows as the block operators' kernels load, store, activate and round them.
#pragma once

#include "rf_device.h"

namespace rf {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// 16 bytes per lane from memory straight into LDS: lane l's bytes land at dst + 16 l.
// (Kept out of the kernel templates: the host pass drops the launch stub of a
// template that names this builtin.)
__device__ __forceinline__ void global_lds16(const uint8_t *p, uint8_t *dst) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)p, (lds_void_t *)dst, 16, 0, 0);
}

// Frame m of the list, m the same for all lanes: a scalar load of the four bytes that it is among.
__device__ __forceinline__ int frame_at(const RowFrames &f, int m) {
    const uint32_t four = reinterpret_cast<const uint32_t *>(f.frame)[static_cast<uint32_t>(m) / 4];
    return static_cast<int>((four >> (8 * (m % 4))) & 255);
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

// gelu by the erf of a fit of its own, for the group norm and the 8-bit products (the device's erff costs
// 110 instructions, four fifths of their epilogue: 6 us of 22 at 1,581 x 1,360 x 1,004). erfc(x) =
// t e^(P(t) - x^2) with t = 1 / (1 + 0.4 x) for x >= 0, P of degree 8 fitted to ln(erfc(x) e^(x^2) / t)
// by exchange of extrema: off by 9e-8 of erfc at most in 64 bits. With x = |z| / sqrt 2, z times half of it is gelu
// below 0, and z less that above; the base is 2 and the half is in the constant. In fp32, where the exponent's
// roundings grow with z^2, results are off by 6e-7 of themselves for |z| < 1, 1e-6 down to -3, 2e-6 to -6, 4e-6 to -9 and 8e-6
// beyond, above 1 by 1.3e-7 (measured; z (1 + erf) / 2 in fp32 by 3e-7, 1.2e-5, and below -5.5 it is 0).
template <int kN>
__device__ __forceinline__ void gelu_fitted(float (&v)[kN]) {
    constexpr float p[9] = {-3.1477283157f, 1.4446996621f, 0.5797163299f, 0.4226135587f, -0.6163823429f, 1.4100290353f, -2.1181933443f, 1.3223464084f, -0.2971011160f};
#pragma unroll
    for (int e = 0; e < kN; ++e) {
        const float z = v[e], t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.2828427125f, 1.0f));
        float s = p[8];
#pragma unroll
        for (int i = 7; i >= 0; --i) s = fmaf(s, t, p[i]);
        const float half = t * fast_exp2(fmaf(z * z, -0.7213475204f, s));
        v[e] = z * (z < 0.0f ? half : 1.0f - half);
    }
}
template <int kN>
__device__ __forceinline__ void activate_fitted(int kind, float (&v)[kN]) {
    if (kind == RF_ACT_GELU) gelu_fitted(v);
    else activate(kind, v);
}

// run(k), k.kind being the activation as a constant: a loop of rows then holds the code of one.
template <int kKind>
struct Activation {
    static constexpr int kind = kKind;
};
template <typename Run>
__device__ __forceinline__ void with_activation(int kind, Run run) {
    if (kind == RF_ACT_NONE) run(Activation<RF_ACT_NONE>{});
    else if (kind == RF_ACT_GELU) run(Activation<RF_ACT_GELU>{});
    else if (kind == RF_ACT_GELU_TANH) run(Activation<RF_ACT_GELU_TANH>{});
    else run(Activation<RF_ACT_SILU>{});
}

__device__ __forceinline__ void widen8(u32x4_t x, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(x[e] << 16);
        v[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u);
    }
}

// A row in 8 bits. Magnitudes are compared as the bits of |x|: those of infinities and NaN are above
// all others', so a row that holds one is seen by its largest.
constexpr uint32_t kInfBits = 0x7f800000u, kTinyBits = (127u - 100u) << 23;   // of 2^-100
struct RowScale {
    float scale, inverse;
    __device__ __forceinline__ explicit RowScale(uint32_t top) {
        const float a = __uint_as_float(top);
        const bool none = top < kTinyBits || top >= kInfBits;   // no finite magnitude to go by: q is 0
        scale = top >= kInfBits ? __uint_as_float(0x7fc00000u) : none ? 0.0f : a / 127.0f;
        inverse = none ? 0.0f : 127.0f / a;
    }
};
// Four of a row's values as 8-bit integers: to the nearest, ties to even, by adding 1.5 * 2^23, whose
// last bits are then those of the sum's integer part (the product is rounded by itself first, as the
// definition says: no fused multiply-add). Values whose row has inverse 0 may be infinite or NaN.
__device__ __forceinline__ uint32_t round4(const float *v, float inverse) {
#pragma clang fp contract(off)
    uint32_t b[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float p = v[e] * inverse;
        b[e] = __float_as_uint(p + 12582912.0f);
    }
    const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
    return inverse == 0.0f ? 0u : lo | hi;
}

}  // namespace rf
