// Activations and their derivatives on 32-bit floats, and the conversions of 16-bit types.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/distsim.h"

namespace distsim {

// ---- pairs of 32-bit floats in one 64-bit register: one instruction for both halves (f32x2) ----

typedef unsigned long long Pair;

__device__ __forceinline__ Pair make_pair2(float a, float b)
{
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 halves(Pair v)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ Pair both(float a) { return make_pair2(a, a); }
__device__ __forceinline__ Pair add2(Pair a, Pair b)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b)
{
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float total(Pair v)
{
    const float2 f = halves(v);
    return f.x + f.y;
}

// 2^v and 1 / v, to two units of 32 bits.
__device__ __forceinline__ float fast_exp2(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float fast_reciprocal(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// ---- activations -------------------------------------------------------------------------------

// 1 / (1 + exp(-v))
__device__ __forceinline__ Pair logistic(Pair v)
{
    const float2 u = halves(mul2(v, both(-1.4426950408889634f)));
    const float2 w = halves(add2(make_pair2(fast_exp2(u.x), fast_exp2(u.y)), both(1.f)));
    return make_pair2(fast_reciprocal(w.x), fast_reciprocal(w.y));
}

// The smaller one; not a number if either is not.
__device__ __forceinline__ float min_or_nan(float a, float b)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// The normal distribution function's tail at -|z|, negated, with |z| (cut to 10000: its tail is zero, and
// infinity would make their product no number) and exp(-z^2 / 2).  The tail is exp(-z^2 / 2) times a
// function that falls slowly, as t times a polynomial in t = 1 / (1 + 0.3 |z|) (the form of Hastings,
// "Approximations for Digital Computers", 1955), fitted here over 0 <= |z| <= 14.5 by least squares of the
// relative error, reweighted towards the largest (1.6e-7).  So both tails keep their digits: off by 2.4e-7
// absolutely, and of itself by 6e-7 down to -2, 2e-6 down to -6, 8e-6 down to -13 (the exponential's argument
// is rounded), where it is below the smallest 32-bit number.
// It costs an exponential more than 1/2 + z P(z^2) / Q(z^2), which is exact to 3.3e-7 absolutely only (4 %
// off at -4.5): 8192 x 1024 -> 4096 with its argument kept 80.9 against 78.2 us, in turn.
__device__ __forceinline__ Pair normal_tail(Pair z, Pair &size, Pair &bell)
{
    const float2 f = halves(z);
    size = make_pair2(min_or_nan(fabsf(f.x), 1e4f), min_or_nan(fabsf(f.y), 1e4f));
    const float2 d = halves(fma2(size, both(0.3f), both(1.f)));
    const float2 e = halves(mul2(mul2(z, z), both(-0.72134752044448170f)));              // -z^2 / 2 in powers of two
    const Pair t = make_pair2(fast_reciprocal(d.x), fast_reciprocal(d.y));
    bell = make_pair2(fast_exp2(e.x), fast_exp2(e.y));
    Pair p = fma2(t, both(-0.03542425483465195f), both(0.15616053342819214f));
    p = fma2(p, t, both(-0.20456023514270782f));
    p = fma2(p, t, both(0.05203711614012718f));
    p = fma2(p, t, both(-0.12769336998462677f));
    p = fma2(p, t, both(-0.10017548501491547f));
    p = fma2(p, t, both(-0.12071221321821213f));
    p = fma2(p, t, both(-0.11963200569152832f));
    return mul2(mul2(p, t), bell);
}
// z Phi(z) = max(z, 0) - |z| Phi(-|z|)
__device__ __forceinline__ Pair times_cdf(Pair z, Pair size, Pair tail)
{
    const float2 f = halves(z);
    return fma2(size, tail, make_pair2(fmaxf(f.x, 0.f), fmaxf(f.y, 0.f)));
}

__device__ __forceinline__ float relu(float z) { return z > 0.f ? z : (z != z ? z : 0.f); }

template <int ACT>
__device__ __forceinline__ Pair activation(Pair z)
{
    if (ACT == DISTSIM_ACT_RELU) {
        const float2 f = halves(z);
        return make_pair2(relu(f.x), relu(f.y));
    }
    if (ACT == DISTSIM_ACT_GELU) {
        Pair size, bell;
        const Pair tail = normal_tail(z, size, bell);
        return times_cdf(z, size, tail);
    }
    if (ACT == DISTSIM_ACT_GELU_TANH)                                // (1 + tanh v) / 2 = logistic(2 v)
        return mul2(z, logistic(mul2(z, fma2(both(0.0713548162726f), mul2(z, z), both(1.59576912160573f)))));
    if (ACT == DISTSIM_ACT_SILU) return mul2(z, logistic(z));
    return z;
}

// act(z) and act'(z)
template <int ACT>
__device__ __forceinline__ void activation_both(Pair z, Pair &value, Pair &slope)
{
    if (ACT == DISTSIM_ACT_RELU) {
        const float2 f = halves(z);
        value = make_pair2(relu(f.x), relu(f.y));
        slope = make_pair2(f.x > 0.f ? 1.f : 0.f, f.y > 0.f ? 1.f : 0.f);
    } else if (ACT == DISTSIM_ACT_GELU) {
        Pair size, bell;
        const Pair tail = normal_tail(z, size, bell);
        const float2 f = halves(z), below = halves(mul2(tail, both(-1.f))), above = halves(add2(tail, both(1.f)));
        value = times_cdf(z, size, tail);
        slope = fma2(mul2(z, both(0.39894228040143268f)), bell, make_pair2(f.x < 0.f ? below.x : above.x, f.y < 0.f ? below.y : above.y));
    } else if (ACT == DISTSIM_ACT_GELU_TANH) {
        const Pair z2 = mul2(z, z);
        const Pair s = logistic(mul2(z, fma2(both(0.0713548162726f), z2, both(1.59576912160573f))));
        value = mul2(z, s);
        // from |z| = 100 on s is 0 or 1 and the first factor zero: z^2 stays finite
        const float2 f = halves(z2);
        const Pair cut = make_pair2(fminf(f.x, 1e4f), fminf(f.y, 1e4f));
        slope = fma2(fma2(value, mul2(s, both(-1.f)), value), fma2(both(0.2140644488178f), cut, both(1.59576912160573f)), s);
    } else if (ACT == DISTSIM_ACT_SILU) {
        const Pair s = logistic(z);
        value = mul2(z, s);
        slope = add2(fma2(value, mul2(s, both(-1.f)), value), s);
    } else {
        value = z;
        slope = both(1.f);
    }
}

// Runs f with the activation as a compile-time constant.
template <class F>
__device__ __forceinline__ void with_activation(int act, F &&f)
{
    switch (act) {
    case DISTSIM_ACT_RELU: f(std::integral_constant<int, DISTSIM_ACT_RELU>()); break;
    case DISTSIM_ACT_GELU: f(std::integral_constant<int, DISTSIM_ACT_GELU>()); break;
    case DISTSIM_ACT_GELU_TANH: f(std::integral_constant<int, DISTSIM_ACT_GELU_TANH>()); break;
    case DISTSIM_ACT_SILU: f(std::integral_constant<int, DISTSIM_ACT_SILU>()); break;
    default: f(std::integral_constant<int, DISTSIM_ACT_NONE>()); break;
    }
}

template <class T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float(float v) { return v; }
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_float(__half v) { return __half2float(v); }

template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float(float v) { return __float2half_rn(v); }

// Two neighbouring values in one word, the first in the low half.
template <class T> __device__ __forceinline__ uint32_t pack_pair(float a, float b);
template <> __device__ __forceinline__ uint32_t pack_pair<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <> __device__ __forceinline__ uint32_t pack_pair<__half>(float a, float b)
{
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <class T>
__device__ __forceinline__ uint32_t pack(Pair v)
{
    const float2 f = halves(v);
    return pack_pair<T>(f.x, f.y);
}
template <class T> __device__ __forceinline__ float2 unpack_pair(uint32_t w);
template <> __device__ __forceinline__ float2 unpack_pair<__nv_bfloat16>(uint32_t w)
{
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <> __device__ __forceinline__ float2 unpack_pair<__half>(uint32_t w)
{
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}

template <class T>
__device__ __forceinline__ Pair unpack(uint32_t w)
{
    const float2 f = unpack_pair<T>(w);
    return make_pair2(f.x, f.y);
}

}  // namespace distsim
