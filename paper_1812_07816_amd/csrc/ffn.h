// What the kernels of the gated feed-forward block share.
#pragma once
#include "mi3d_internal.h"
#include "rows_common.h"

namespace mi3d {

// act(g) and act'(g); silu: g s(g) with the logistic s, gelu: g Phi(g) with the normal distribution's Phi.  fp32: the library's functions.
// bf16: the hardware's exponential and reciprocal, and erfc(z) = e^(-z^2) t P(t), t = 1 / (1 + 0.41 z), z = |g| / sqrt 2, whose
// exponential is that of the derivative as well.  P, of six coefficients, was fitted to erfc by linear programming on 0 <= z <= 9.6 (beyond, e^(-z^2)
// is below the least normal number) so that neither the error (1e-7) nor its ratio to erfc (2e-4, a twentieth of half a step of
// bf16) is large: the tail below zero holds to its end, at the time of the five terms of a fit to the error alone, which is 1 % off at
// g = -8 (data gradient of 16384 x 1024 x 4096 466 and 465 us, forward pass of 27648 x 320 x 1280 118 and 118).
template <typename T, int ACT>
__device__ __forceinline__ void activation(float g, float& a, float& d) {
    if constexpr (ACT == MI3D_ACT_SILU) {
        const float s = sizeof(T) == 2 ? __builtin_amdgcn_rcpf(1.f + __expf(-g)) : 1.f / (1.f + expf(-g));
        a = g * s;
        d = fmaf(a, 1.f - s, s);
    } else {
        const float e = sizeof(T) == 2 ? __expf(-0.5f * g * g) : expf(-0.5f * g * g);      // e^(-z^2), z = |g| / sqrt 2
        float c;
        if (sizeof(T) == 2) {
            const float t = __builtin_amdgcn_rcpf(fmaf(0.41f * 0.70710678f, fabsf(g), 1.f));
            const float P = fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, -0.178960204f, 0.574866056f), -0.192743808f), 0.362556666f), 0.200580105f), 0.233701095f);
            const float q = 0.5f * e * t * P;
            c = g < 0.f ? q : 1.f - q;
        } else {
            c = 0.5f * erfcf(g * -0.70710678f);      // (1 + erf cancels below zero: 4 % off at g = -5, 0 from -5.6 on)
        }
        a = g * c;
        d = fmaf(g * 0.39894228f, e, c);
    }
}
template <typename T, int ACT>
__device__ __forceinline__ float activation(float g) {
    float a, d;
    activation<T, ACT>(g, a, d);
    return a;
}

// The forward products of few rows, or of small matrices.  gated: w holds 2 N rows, out = act(g) * u (and [g | u] where gu is not
// null); otherwise N rows and out = x w^T.  K and N are multiples of 8.  few_rows_us: what its model expects it to take (very long:
// too many rows).
double few_rows_us(bool bf16, long long rows, long long K, long long N);
int few_rows_product(bool bf16, bool gated, const void* x, const void* w, long long rows, int K, int N, int act, void* out, void* gu, hipStream_t s);

}  // namespace mi3d
