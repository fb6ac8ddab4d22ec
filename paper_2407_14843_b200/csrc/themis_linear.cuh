// Activations and their slopes.
#pragma once

#include "themis_numeric.cuh"
#include "themis_forecast_internal.h"

namespace themis {

// Normal distribution function by Abramowitz and Stegun 7.1.26 (erf(x) = 1 - (a1 t + .. + a5 t^5) e^-x^2,
// t = 1 / (1 + p x), within 1.5e-7): one exponential, which the density needs as well.  gelu(v) is within
// 4.3e-7 for v in -13..8.  Relative to itself, below 0: 7e-7 down to -1, 5e-5 to -3, 5e-4 to -4, 2e-3 to -5, 4e-3 to
// -6, 1e-2 to -8; 0.5 v (1 + erf) in 32 bits is within 2e-7, 1e-5, 5e-4, 5e-2 and from -6 on off by all of it.
// Half a unit in the last place is 2e-3 to 4e-3 in bf16, 2.4e-4 to 4.9e-4 in fp16.
__device__ __forceinline__ float normal_cdf(float v, float &gauss)
{
    const float t = reciprocal(fmaf(0.3275911f * 0.70710678f, fabsf(v), 1.0f));
    gauss = ex2(-0.5f * kLog2e * v * v);
    float s = fmaf(1.061405429f, t, -1.453152027f);
    s = fmaf(s, t, 1.421413741f);
    s = fmaf(s, t, -0.284496736f);
    s = fmaf(s, t, 0.254829592f);
    const float tail = 0.5f * s * t * gauss;         // beyond |v|
    return v < 0.0f ? tail : 1.0f - tail;
}

__device__ __forceinline__ float activate(float v, int act)
{
    float gauss;
    switch (act) {
        case THEMIS_ACT_RELU: return v < 0.0f ? 0.0f : v;      // NaN stays NaN
        case THEMIS_ACT_SILU: return silu(v);
        case THEMIS_ACT_GELU: return v * normal_cdf(v, gauss);
        default: return v;
    }
}

// d act(v) / dv; relu's is 0 at 0
__device__ __forceinline__ float act_slope(float v, int act)
{
    float gauss;
    switch (act) {
        case THEMIS_ACT_RELU: return v > 0.0f ? 1.0f : 0.0f;
        case THEMIS_ACT_SILU: return silu_slope(v, sigmoid(v));
        case THEMIS_ACT_GELU: {
            const float cdf = normal_cdf(v, gauss);
            return fmaf(v * 0.39894228f, gauss, cdf);
        }
        default: return 1.0f;
    }
}

inline size_t align256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace themis
