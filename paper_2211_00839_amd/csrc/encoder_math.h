// Element types, activations and the 8-bit block format of the feature encoder's kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

namespace enc {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int MX_BLOCK = 32;     // elements that share a scale

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__bf16 v) { return (float)v; }

// Vectors of 16 bytes that need no alignment beyond their element's: global loads and stores of this architecture take any
// address, and rows of odd lengths are as common as padded ones.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(1)));
typedef unsigned u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
template <typename T> struct Any;
template <> struct Any<float> { typedef f32x4_any type; };
template <> struct Any<__bf16> { typedef bf16x8_any type; };

// 8 consecutive elements of a row as fp32; `count` of them exist, the others come out as 0.
template <typename T>
__device__ __forceinline__ void load8(const T *__restrict__ p, int count, float (&v)[8])
{
    if (count >= 8) {
        if constexpr (sizeof(T) == 4) {
            const f32x4 a = reinterpret_cast<const f32x4_any *>(p)[0], b = reinterpret_cast<const f32x4_any *>(p)[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = a[i];
                v[4 + i] = b[i];
            }
        } else {
            const bf16x8 a = *reinterpret_cast<const bf16x8_any *>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < count ? to_f32(p[i]) : 0.f;
}

template <typename T>
__device__ __forceinline__ void store8(T *__restrict__ p, int count, const float (&v)[8])
{
    if (count >= 8) {
        if constexpr (sizeof(T) == 4) {
            reinterpret_cast<f32x4_any *>(p)[0] = f32x4{v[0], v[1], v[2], v[3]};
            reinterpret_cast<f32x4_any *>(p)[1] = f32x4{v[4], v[5], v[6], v[7]};
        } else {
            bf16x8 a;
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = (__bf16)v[i];
            *reinterpret_cast<bf16x8_any *>(p) = a;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) p[i] = (T)v[i];
}

// e^x to about an ulp: 2^(x log2 e) with the product's rounding error given back.  x is held within -104 (0) .. 88.7
// (3.3e38) first, so that no infinity meets its own negative below; a NaN comes out as a number, which no caller lets
// through (each multiplies by the NaN itself).
__device__ __forceinline__ float exp_f32(float x)
{
    const float c = __builtin_amdgcn_fmed3f(x, -104.f, 88.7f);
    const float t = c * 1.44269504f;
    const float lost = fmaf(c, 1.44269504f, -t) + c * 1.92596299e-8f;    // log2 e = 1.44269504 + 1.926e-8
    return fmaf(__builtin_amdgcn_exp2f(t), lost * 0.693147181f, __builtin_amdgcn_exp2f(t));
}

// 1 / (1 + e^-z); 0 from where it is below the normal numbers on (so that silu of -infinity is the formula's NaN).
__device__ __forceinline__ float logistic(float z) { return z < -87.f ? 0.f : __builtin_amdgcn_rcpf(1.f + exp_f32(-z)); }

// Phi(z) and the density's e^(-z^2/2), which it is made of: erfc(x) = (a1 t + .. + a5 t^5) e^(-x^2) with
// t = 1 / (1 + p x), x = |z| / sqrt 2, off by at most 1.5e-7 (Abramowitz and Stegun, 7.1.26); Phi to half of that.  No
// branch, where a library's erf has two; an epilogue of gelu is as long as its instructions.
__device__ __forceinline__ float normal_cdf(float z, float *bell)
{
    const float e = exp_f32(-0.5f * z * z);
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.3275911f * 0.707106781f, 1.f));
    float q = fmaf(t, 1.061405429f, -1.453152027f);
    q = fmaf(t, q, 1.421413741f);
    q = fmaf(t, q, -0.284496736f);
    q = fmaf(t, q, 0.254829592f);
    const float tail = 0.5f * t * q * e;
    *bell = e;
    return z < 0.f ? tail : 1.f - tail;
}

// act(z): 0 none, 1 relu, 2 silu, 3 gelu (rcd_act)
template <int ACT> __device__ __forceinline__ float activate_as(float z)
{
    if (ACT == 0) return z;
    if (ACT == 1) return z < 0.f ? 0.f : z;        // (a NaN stays one)
    if (ACT == 2) return z * logistic(z);
    float bell;
    return z * normal_cdf(z, &bell);
}
__device__ __forceinline__ float activate(float z, int act)
{
    return act == 0 ? activate_as<0>(z) : act == 1 ? activate_as<1>(z) : act == 2 ? activate_as<2>(z) : activate_as<3>(z);
}

// act(z) and act'(z)
template <int ACT> __device__ __forceinline__ void activate_both_as(float z, float *value, float *slope)
{
    if (ACT == 0) {
        *value = z;
        *slope = 1.f;
    } else if (ACT == 1) {
        *value = z < 0.f ? 0.f : z;
        *slope = z > 0.f ? 1.f : 0.f;
    } else if (ACT == 2) {
        const float s = logistic(z);
        *value = z * s;
        *slope = s * fmaf(z, 1.f - s, 1.f);
    } else {
        float bell;
        const float cdf = normal_cdf(z, &bell);
        *value = z * cdf;
        *slope = fmaf(z, 0.398942280f * bell, cdf);
    }
}

// Calls go(act as a constant): the choice once for many elements.
template <typename Go> __device__ __forceinline__ void with_act(int act, Go go)
{
    if (act == 0) go(std::integral_constant<int, 0>{});
    else if (act == 1) go(std::integral_constant<int, 1>{});
    else if (act == 2) go(std::integral_constant<int, 2>{});
    else go(std::integral_constant<int, 3>{});
}

// The block exponent e: the least power of two with amax <= 448 * 2^e, not below 2^-127.  448 = 1.75 * 2^8.
__device__ __forceinline__ int mx_exponent(float amax)
{
    const unsigned bits = __builtin_bit_cast(unsigned, amax);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, -127);            // (zero and denormals: the exponent field is 0)
}
__device__ __forceinline__ float pow2(int e) { return __builtin_bit_cast(float, (unsigned)(e + 127) << 23); }   // -126 .. 127

// Four values, already divided by their scale, as e4m3 bytes; what is not finite becomes NaN (0x7f).
__device__ __forceinline__ unsigned to_e4m3x4(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    const float v[4] = {a, b, c, d};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (!(fabsf(v[i]) <= 448.f)) w = (w & ~(0xff << (8 * i))) | (0x7f << (8 * i));
    return (unsigned)w;
}

// 2^(s - 127) of a scale byte; 255 is NaN.
__device__ __forceinline__ float mx_scale(int s)
{
    return __builtin_bit_cast(float, s == 255 ? 0x7fc00000u : s == 0 ? 0x00400000u : (unsigned)s << 23);
}

// Eight e4m3 bytes times their scale as bf16: exact, a value has four significant bits (below 2^-126 bf16 has fewer).
__device__ __forceinline__ bf16x8 widen8(unsigned lo, unsigned hi, float scale)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    bf16x8 r;
    const unsigned w[2] = {lo, hi};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
        r[4 * i] = (__bf16)(a[0] * scale);
        r[4 * i + 1] = (__bf16)(a[1] * scale);
        r[4 * i + 2] = (__bf16)(b[0] * scale);
        r[4 * i + 3] = (__bf16)(b[1] * scale);
    }
    return r;
}

} // namespace enc
