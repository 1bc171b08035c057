// Capped scores in log2 units, two at a time where they are far below the cap.
#pragma once
#include "umma.cuh"

namespace stc {

// Two raw products capped, in log2 units, where they stay below 0.35 of the cap: x scale (1 + u P(u)) with u the square of
// x scale / cap, P of three terms by weighted least squares at Chebyshev nodes (relative error 4.3e-8 of tanh).
constexpr float kCapSmall = 0.35f, kCap1 = -0.33332642912864685f, kCap2 = 0.13299374282360077f, kCap3 = -0.049123503267765045f;
__device__ __forceinline__ float2 cap_small(float2 x, float cap_in, float scale_log2) {
    const float2 z = mul2(x, both(cap_in)), u = mul2(z, z);
    float2 p = fma2(both(kCap3 * scale_log2), u, both(kCap2 * scale_log2));
    p = fma2(p, u, both(kCap1 * scale_log2));
    p = fma2(p, u, both(scale_log2));
    return mul2(x, p);
}
__device__ __forceinline__ float cap_any(float x, float cap_in, float cap_log2) {
    const float z = x * cap_in, lo = tanh_small(z), hi = tanh_large(z);
    return cap_log2 * (fabsf(z) <= kTanhSmall ? lo : hi);
}
// Cap the N scores of a row: far below the cap (the usual case; the warp votes once per tile instead of branching per
// score), and of any size.
template <int N>
__device__ __forceinline__ void cap_scores_low(uint32_t (&r)[N], float cap_in, float scale_log2) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float2 y = cap_small(make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), cap_in, scale_log2);
        r[i] = __float_as_uint(y.x);
        r[i + 1] = __float_as_uint(y.y);
    }
}
template <int N>
__device__ __forceinline__ void cap_scores_any(uint32_t (&r)[N], float cap_in, float cap_log2) {
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = __float_as_uint(cap_any(__uint_as_float(r[i]), cap_in, cap_log2));
}
template <int N>
__device__ __forceinline__ float magnitude(const uint32_t (&r)[N]) {
    float b[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; i += 2)
        b[(i >> 1) & 3] = fmaxf(fmaxf(b[(i >> 1) & 3], fabsf(__uint_as_float(r[i]))), fabsf(__uint_as_float(r[i + 1])));
    return fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3]));
}

}  // namespace stc
