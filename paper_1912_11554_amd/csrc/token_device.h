// Device helpers of the token-model kernels: element types, activations, the
// parts of an fp32 value.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/nuts_token.h"

namespace nuts {
namespace token {

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// 16 bytes at any alignment of their elements (one memory instruction).
typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(2), may_alias));
__device__ __forceinline__ v4u load16(const void* p) { return *(const v4u_any*)p; }
__device__ __forceinline__ void store16(void* p, v4u v) { *(v4u_any*)p = v; }
// PAST: past the caches, for outputs that do not fit them.
template <bool PAST>
__device__ __forceinline__ void store16(void* p, v4u v)
{
    if constexpr (PAST) __builtin_nontemporal_store(v, (v4u_any*)p);
    else store16(p, v);
}

// The elements of 16 bytes.
template <typename T>
__device__ __forceinline__ void unpack(v4u raw, float (&v)[16 / sizeof(T)])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(raw[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(raw[i] << 16);
            v[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
        }
    }
}
template <typename T>
__device__ __forceinline__ v4u pack(const float (&v)[16 / sizeof(T)])
{
    v4u raw;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = __float_as_uint(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const v2bf t = {(__bf16)v[2 * i], (__bf16)v[2 * i + 1]};
            raw[i] = __builtin_bit_cast(uint32_t, t);
        }
    }
    return raw;
}

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__bf16 x) { return (float)x; }
template <typename T>
__device__ __forceinline__ T from_f32(float x)
{
    return (T)x;  // rounds to nearest even
}

// Orders the lanes' LDS accesses before it against those after it.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Element i of an array of either type.
__device__ __forceinline__ float load_as_f32(const void* p, int dtype, int64_t i)
{
    return dtype == NUTS_BF16 ? (float)((const __bf16*)p)[i] : ((const float*)p)[i];
}
__device__ __forceinline__ void store_f32(void* p, int dtype, int64_t i, float v)
{
    if (dtype == NUTS_BF16) ((__bf16*)p)[i] = (__bf16)v;
    else ((float*)p)[i] = v;
}

// exp(x + rest), |rest| far below |x|, as 2^t: what rounding takes off t = x log2(e)
// goes into a factor 1 + d ln 2.  Left to itself that rounding is a relative error of
// |x| 2^-24.
__device__ __forceinline__ float exp_f32(float x, float rest = 0.0f)
{
    constexpr float log2e = 0x1.715476p+0f, log2e_low = 0x1.4ae0cp-26f, ln2 = 0x1.62e43p-1f;  // log2(e), in two parts
    const float t = x * log2e;
    const float d = fmaf(x, log2e_low, fmaf(rest, log2e, fmaf(x, log2e, -t)));
    const float e = __builtin_amdgcn_exp2f(t);
    return fabsf(t) < 126.0f ? fmaf(e, d * ln2, e) : e;  // (past that e may be 0, an infinity or NaN)
}

// act(z).  The logistic function with the reciprocal of the fp32 units: exp(-z)
// overflows to infinity below z = -88, whose reciprocal is the limit 0; z =
// -infinity gives silu 0, its limit.
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.0f + exp_f32(-z)); }

__device__ __forceinline__ float activate(float z, int act)
{
    switch (act) {
    case NUTS_ACT_RELU: return z > 0.0f ? z : (z != z ? z : 0.0f);
    case NUTS_ACT_SIGMOID: return logistic(z);
    case NUTS_ACT_SILU: return z == -__builtin_inff() ? 0.0f : z * logistic(z);
    case NUTS_ACT_GELU: return z == -__builtin_inff() ? 0.0f : 0.5f * z * erfcf(-z * 0.70710678118654752f);
    default: return z;
    }
}

// p = logistic(z) and p (1 - p).  1 - p is logistic(-z) and taken as such: near p = 1
// the difference has few digits, or none.
__device__ __forceinline__ void logistic_slope(float z, float* p, float* pq)
{
    const float e = exp_f32(-fabsf(z)), d = __builtin_amdgcn_rcpf(1.0f + e);
    *p = z < 0.0f ? e * d : d;
    *pq = e * d * d;
}

// act(z) and act'(z).
__device__ __forceinline__ void activate_slope(float z, int act, float* a, float* slope)
{
    switch (act) {
    case NUTS_ACT_RELU:
        *a = activate(z, act);
        *slope = z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
        break;
    case NUTS_ACT_SIGMOID: {
        logistic_slope(z, a, slope);
        break;
    }
    case NUTS_ACT_SILU: {
        // an infinite z takes the limits: 0 and 0, or z and 1
        float p, pq;
        logistic_slope(z, &p, &pq);
        *a = z == -__builtin_inff() ? 0.0f : z * p;
        *slope = p + (fabsf(z) == __builtin_inff() ? 0.0f : z * pq);
        break;
    }
    case NUTS_ACT_GELU: {
        const float cdf = 0.5f * erfcf(-z * 0.70710678118654752f);
        const float square = z * z;
        const float pdf = 0.39894228040143268f * exp_f32(-0.5f * square, -0.5f * fmaf(z, z, -square));
        *a = z == -__builtin_inff() ? 0.0f : z * cdf;
        *slope = cdf + (fabsf(z) == __builtin_inff() ? 0.0f : z * pdf);
        break;
    }
    default:
        *a = z;
        *slope = 1.0f;
    }
}

// The three bf16 parts of fp32 values, cut off rather than rounded: eight of the
// 24 bits each, so the parts hold the value exactly (down to bf16's least
// magnitude, 2^-133) and no finite value leaves the range.  An infinity's other
// parts are NaN, which the products' corrections drop.  A NaN is made quiet first: a
// signalling one may have all of its set bits in the half that is cut off, where the
// first part would be an infinity.  out[p]: part p of two values, the first in the
// low half.
__device__ __forceinline__ void parts3(float x, float y, uint32_t (&out)[3])
{
    x = __builtin_canonicalizef(x);
    y = __builtin_canonicalizef(y);
#pragma unroll
    for (int p = 0; p < 3; ++p) {
        const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
        out[p] = __builtin_amdgcn_perm(b, a, 0x07060302);
        x -= __uint_as_float(a & 0xffff0000u);
        y -= __uint_as_float(b & 0xffff0000u);
    }
}

}  // namespace token
}  // namespace nuts
