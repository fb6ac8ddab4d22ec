// Types, paired 32-bit arithmetic and functions of the forecasting kernels.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <float.h>
#include <stdint.h>

namespace themis {

// --- types ---------------------------------------------------------------------------------
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// --- two neighbouring values of a row -----------------------------------------------------------
template <typename T> struct PairOf { typedef uint32_t type; };
template <> struct PairOf<float> { typedef uint2 type; };
template <typename T> using Pair = typename PairOf<T>::type;

template <typename T> __device__ __forceinline__ Pair<T> zero_pair();
template <> __device__ __forceinline__ uint2 zero_pair<float>() { return make_uint2(0, 0); }
template <> __device__ __forceinline__ uint32_t zero_pair<__nv_bfloat16>() { return 0; }
template <> __device__ __forceinline__ uint32_t zero_pair<__half>() { return 0; }

__device__ __forceinline__ uint32_t bits_of(__nv_bfloat16 v) { return __bfloat16_as_ushort(v); }
__device__ __forceinline__ uint32_t bits_of(__half v) { return __half_as_ushort(v); }

// whether a row of pairs from `first` on can be read with one access each, row after row
template <typename T> __device__ __forceinline__ bool pairs_ok(const T *first, int64_t stride, bool two)
{
    return two && ((uintptr_t)first & (2 * sizeof(T) - 1)) == 0 && (stride & 1) == 0;
}
// two neighbouring 16-bit values, or one twice (!two)
template <typename T> __device__ __forceinline__ uint32_t load_two(const T *p, bool two)
{
    return bits_of(p[0]) | bits_of(p[two ? 1 : 0]) << 16;
}

template <typename T> struct Unpack;
template <> struct Unpack<float> {
    __device__ __forceinline__ static void run(uint2 v, float (&f)[2])
    {
        f[0] = __uint_as_float(v.x);
        f[1] = __uint_as_float(v.y);
    }
};
template <> struct Unpack<__nv_bfloat16> {
    __device__ __forceinline__ static void run(uint32_t v, float (&f)[2])
    {
        f[0] = __uint_as_float(v << 16);
        f[1] = __uint_as_float(v & 0xffff0000u);
    }
};
template <> struct Unpack<__half> {
    __device__ __forceinline__ static void run(uint32_t v, float (&f)[2])
    {
        const float2 r = __half22float2(*reinterpret_cast<const __half2 *>(&v));
        f[0] = r.x;
        f[1] = r.y;
    }
};

__device__ __forceinline__ void store_pair(float *p, const float (&v)[2], bool pair, bool two)
{
    if (pair) {
        *reinterpret_cast<float2 *>(p) = make_float2(v[0], v[1]);
    } else {
        p[0] = v[0];
        if (two) p[1] = v[1];
    }
}
__device__ __forceinline__ void store_pair(__nv_bfloat16 *p, const float (&v)[2], bool pair, bool two)
{
    if (pair) {
        *reinterpret_cast<__nv_bfloat162 *>(p) = __floats2bfloat162_rn(v[0], v[1]);
    } else {
        p[0] = __float2bfloat16_rn(v[0]);
        if (two) p[1] = __float2bfloat16_rn(v[1]);
    }
}
__device__ __forceinline__ void store_pair(__half *p, const float (&v)[2], bool pair, bool two)
{
    if (pair) {
        *reinterpret_cast<__half2 *>(p) = __floats2half2_rn(v[0], v[1]);
    } else {
        p[0] = __float2half_rn(v[0]);
        if (two) p[1] = __float2half_rn(v[1]);
    }
}

// --- two 32-bit floats in one 64-bit register (one issue slot for two multiply-adds) ----------
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float lo, float hi)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float &lo, float &hi)
{
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// --- functions -----------------------------------------------------------------------------
constexpr float kLog2e = 1.4426950408889634f;

// 2^v by the special-function unit (relative error below 2^-22; 0 below -126).
__device__ __forceinline__ float ex2(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ f32x2 ex2_pair(f32x2 v)
{
    float lo, hi;
    unpack2(v, lo, hi);
    return pack2(ex2(lo), ex2(hi));
}

// exp(s A) from A log2(e).  ex2.approx is low by 0.5e-8 to 5e-8 on average (measured over exponents from
// -0.0002 to -20), and a factor close to 1 that is applied a thousand times adds that up, so the exponent
// is raised by kExpShift in the multiply-add that forms it: -0.7e-8 to +0.4e-8 on average for exponents
// of 0.0002 to 0.02 and within 1.5e-8 up to 1.  exp(0) stays 1.
constexpr float kExpShift = 1.3e-8f;
// A log2(e), kept finite (NaN stays): a time that does not exist has a step of 0 and its factor has to be 1 for
// the lowest A and for -inf too, where 0 times an infinity would be no number.
__device__ __forceinline__ float log2_rate(float a)
{
    float v = a * kLog2e;
    asm("max.NaN.f32 %0, %0, %1;\n\tmin.NaN.f32 %0, %0, %2;" : "+f"(v) : "f"(-FLT_MAX), "f"(FLT_MAX));
    return v;
}
__device__ __forceinline__ float decay(float s, float a2) { return ex2(fmaf(s, a2, kExpShift)); }
__device__ __forceinline__ f32x2 decay2(f32x2 s, f32x2 a2) { return ex2_pair(fma2(s, a2, pack2(kExpShift, kExpShift))); }

__device__ __forceinline__ float reciprocal(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// The exponent's product is rounded: e^-v is off by |v| 2^-24, which the sum with 1 hides unless v
// is far below 0, where the function itself vanishes.
__device__ __forceinline__ float sigmoid(float v) { return reciprocal(1.0f + ex2(-kLog2e * v)); }
// v = -inf would give inf / inf in a quotient; the product with a zero is NaN, as the formula's is
__device__ __forceinline__ float silu(float v) { return v * sigmoid(v); }
// d silu(v) / dv for s = sigmoid(v)
__device__ __forceinline__ float silu_slope(float v, float s) { return s * fmaf(v, 1.0f - s, 1.0f); }

// log(1 + e^v) = max(v, 0) + log1p(e), e = e^-|v| in (0, 1].  With w = e / (2 + e) <= 1/3,
// log1p(e) = 2 artanh(w) = w P(w^2): no cancellation for small e, where log(1 + e) would lose the
// low bits.  P is the degree-4 polynomial of least relative error on [0, 1/9] (Remez exchange; 8e-9).
// The exponent's product is rounded, which leaves a relative error of |v| 2^-24.
__device__ __forceinline__ float softplus(float v)
{
    const float e = ex2(-kLog2e * fabsf(v));
    const float w = e * reciprocal(2.0f + e), q = w * w;
    float s = 0x1.208bd0p-2f;
    s = fmaf(s, q, 0x1.1e510ap-2f);
    s = fmaf(s, q, 0x1.99dae6p-2f);
    s = fmaf(s, q, 0x1.5554e0p-1f);
    s = fmaf(s, q, 2.0f);
    return fmaf(s, w, fmaxf(v, 0.0f));
}

}  // namespace themis
