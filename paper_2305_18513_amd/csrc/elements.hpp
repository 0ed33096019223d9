// Elements of a 16-byte vector in fp32 and back, and GELU: shared by the quantiser and the gated activations.
#pragma once

#include "common.hpp"

namespace slimfit {
namespace {

template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int V = 4;
    using raw = f32x4;
    __device__ static void unpack(const raw &r, float (&f)[4]) { f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w; }
    __device__ static raw pack(const float (&f)[4]) { return raw{f[0], f[1], f[2], f[3]}; }
    __device__ static float load1(const float *p) { return *p; }
    __device__ static void store1(float *p, float v) { *p = v; }
};
template <> struct Vec<uint16_t> {   // bf16 bit patterns
    static constexpr int V = 8;
    using raw = u32x4;
    __device__ static void unpack(const raw &r, float (&f)[8])
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __builtin_bit_cast(float, w[i] << 16);
            f[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xFFFF0000u);
        }
    }
    __device__ static raw pack(const float (&f)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = bf16_narrow2(f[2 * i], f[2 * i + 1]);
        return raw{w[0], w[1], w[2], w[3]};
    }
    __device__ static float load1(const uint16_t *p) { return bf16_widen(*p); }
    __device__ static void store1(uint16_t *p, float v) { *p = (uint16_t)bf16_narrow(v); }
};

// Exact (erf) GELU and its derivative in fp32.
// 1 + erf(x / sqrt 2) is built from erfc(t), t = |x| / sqrt 2:  2 - erfc(t) for
// x >= 0 and erfc(t) itself for x < 0, which also keeps the left tail free of
// cancellation.  erfc(t) = exp(-t * Q(t)) with Q(t) = -ln(erfc t) / t, a smooth
// function (Q(0) = 2 / sqrt pi) replaced by a degree-8 polynomial fitted to it
// on [0, 4.2] (weighted least squares at Chebyshev nodes, weight erfc(t) * t);
// beyond 4.2 erfc is below 3e-9 and t is clamped (`far`; up to 6 the polynomial
// goes on falling, to 8e-15 for erfc's 2e-17, and then rises).  In fp32 with fused
// multiply-adds and the hardware exp2 the absolute error of erfc stays under
// 1.5e-7 (checked against fp64 on 3 M points), one branch-free path of about 16
// instructions where the library erff takes two divergent ones of about 40.
__device__ __forceinline__ float erfc_nonneg(float t, float far)
{
    t = fminf(t, far);
    float q = -8.094536919e-06f;
    q = fmaf(q, t, 1.064909658e-04f);
    q = fmaf(q, t, -5.896771888e-04f);
    q = fmaf(q, t, 1.580125120e-03f);
    q = fmaf(q, t, -6.248015670e-05f);
    q = fmaf(q, t, -1.921485045e-02f);
    q = fmaf(q, t, 1.027984564e-01f);
    q = fmaf(q, t, 6.366162197e-01f);
    q = fmaf(q, t, 1.128379327e+00f);
    return __builtin_amdgcn_exp2f(-(q * t) * 1.44269504088896340736f);
}
__device__ __forceinline__ float twice_normal_cdf(float x, float far = 4.2f)        // 1 + erf(x / sqrt 2)
{
    const float e = erfc_nonneg(fabsf(x) * 0.70710678118654752440f, far);
    return x >= 0.0f ? 2.0f - e : e;
}
__device__ __forceinline__ float gelu_f32(float x) { return (0.5f * x) * twice_normal_cdf(x); }
__device__ __forceinline__ float gelu_slope_f32(float x)
{
    const float pdf = __builtin_amdgcn_exp2f(((-0.5f * x) * x) * 1.44269504088896340736f) * 0.39894228040143267794f;
    return 0.5f * twice_normal_cdf(x) + x * pdf;
}

}  // namespace
}  // namespace slimfit
