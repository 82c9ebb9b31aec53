// Gates of a gated layer, y = act(g) * u: the function and its slope.
#ifndef PF_TC_GATED_CUH_
#define PF_TC_GATED_CUH_
#include "pf.h"
#include "pf_f32x2.cuh"

namespace pf {

// 1 / (1 + e^-x) and 1 less that, each to its own precision: with t = e^-|x|, which never overflows, they are 1 / (1 + t) and t / (1 + t).
// kExact: by expf and a division; else by the hardware's approximations (each off by 2^-22 or less, of results that are rounded by 2^-9).
template <bool kExact>
__device__ __forceinline__ void sigmoids(float x, float* up, float* down) {
    float t, d;
    if constexpr (kExact) {
        t = expf(-fabsf(x));
        d = 1.f / (1.f + t);
    } else {
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(-1.44269504f * fabsf(x)));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(1.f + t));
    }
    const float e = t * d;
    *up = x < 0.f ? e : d;
    *down = x < 0.f ? d : e;
    if (x != x) *up = *down = x;
}
// 1 / (1 + e^-x) alone.
__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + expf(-x)); }

// The tanh form of the Gaussian unit is g * sigmoid(x) with x = sqrt(8 / pi) (g + 0.044715 g^3).
constexpr float kGelu1 = 1.5957691216f, kGelu3 = 0.0713548163f;      // sqrt(8 / pi), and 0.044715 of it

template <int kAct>
__device__ __forceinline__ float gate(float g) {
    if constexpr (kAct == PF_GATE_RELU) return g > 0.f || g != g ? g : 0.f;
    if constexpr (kAct == PF_GATE_SIGMOID) return sigmoid(g);
    if constexpr (kAct == PF_GATE_GELU) return g * sigmoid(g * fmaf(kGelu3, g * g, kGelu1));
    return g * sigmoid(g);
}
// act(g) and act'(g).
template <int kAct, bool kExact>
__device__ __forceinline__ void gate_slope(float g, float* value, float* slope) {
    if constexpr (kAct == PF_GATE_RELU) {
        *value = g > 0.f || g != g ? g : 0.f;
        *slope = g > 0.f ? 1.f : 0.f;
    } else {
        const bool gelu = kAct == PF_GATE_GELU;
        float up, down;
        sigmoids<kExact>(gelu ? g * fmaf(kGelu3, g * g, kGelu1) : g, &up, &down);
        if constexpr (kAct == PF_GATE_SIGMOID) {
            *value = up;
            *slope = up * down;
        } else {
            *value = g * up;
            const float steep = gelu ? fmaf(3.f * kGelu3, g * g, kGelu1) : 1.f, both = up * down;
            // (far out up * down is 0, and what it stands beside may be infinite)
            *slope = both == 0.f ? up : fmaf(both, g * steep, up);
        }
    }
}
// 1 / (1 + 2^x) of two, approximately.  Special functions are an eighth as fast as products, and two for an element bounded the gate (forward, 16384 x 4096 over 64:
// 50.7 us, so 48.7), so the reciprocal is Newton's method: taken from exponent and mantissa at once it is within 0.051, and a step of third order and one of
// second leave 2^-23.  Subnormal numbers are taken as 0, so that from 2^126.5 on, where 2^x is held, the result is 0.
__device__ __forceinline__ F2 fma2_ftz(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.ftz.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ F2 logistic2(F2 x) {
    const float2 v = split(x);
    float a, b;
    asm("{\n .reg .f32 t;\n min.NaN.f32 t, %1, %2;\n ex2.approx.ftz.f32 %0, t;\n}" : "=f"(a) : "f"(v.x), "f"(126.5f));
    asm("{\n .reg .f32 t;\n min.NaN.f32 t, %1, %2;\n ex2.approx.ftz.f32 %0, t;\n}" : "=f"(b) : "f"(v.y), "f"(126.5f));
    const F2 one = f2(1.f, 1.f), minus = f2(-1.f, -1.f), d = fma2(f2(a, b), minus, minus);      // -(1 + 2^x)
    const float2 dv = split(d);
    constexpr uint32_t kTwice = 0x7ef31000u + 0x80000000u;
    const F2 r0 = f2(__uint_as_float(kTwice - __float_as_uint(dv.x)), __uint_as_float(kTwice - __float_as_uint(dv.y)));
    const F2 e0 = fma2_ftz(d, r0, one), r1 = fma2_ftz(r0, fma2(e0, e0, e0), r0);
    return fma2_ftz(r1, fma2_ftz(d, r1, one), r1);
}
// act(g) u of two, approximately: the gate's own value first, as g u may overflow where act(g) is nothing.
template <int kAct>
__device__ __forceinline__ F2 gated2(F2 g, F2 u) {
    constexpr float kLog2e = 1.44269504f;
    if constexpr (kAct == PF_GATE_RELU) {
        const float2 v = split(g);
        return mul2(f2(gate<kAct>(v.x), gate<kAct>(v.y)), u);
    } else if constexpr (kAct == PF_GATE_SIGMOID) {
        return mul2(logistic2(mul2(g, f2(-kLog2e, -kLog2e))), u);
    } else if constexpr (kAct == PF_GATE_GELU) {
        const F2 steep = fma2(mul2(g, g), f2(-kLog2e * kGelu3, -kLog2e * kGelu3), f2(-kLog2e * kGelu1, -kLog2e * kGelu1));
        return mul2(mul2(g, logistic2(mul2(g, steep))), u);
    } else {
        return mul2(mul2(g, logistic2(mul2(g, f2(-kLog2e, -kLog2e)))), u);
    }
}
// dY act'(g) u (in this order) and dY act(g) of two, approximately.  With s = sigmoid(x): 1 - s is off by 2^-24, which beside slopes near 1 is nothing; the sigmoid's own slope
// takes the form that keeps it.
template <int kAct>
__device__ __forceinline__ void gated_grad2(F2 g, F2 u, F2 dy, F2* dg, F2* du) {
    constexpr float kLog2e = 1.44269504f;
    const F2 one = f2(1.f, 1.f);
    if constexpr (kAct == PF_GATE_RELU || kAct == PF_GATE_SIGMOID) {
        const float2 v = split(g);
        float a, b, sa, sb;
        gate_slope<kAct, false>(v.x, &a, &sa);
        gate_slope<kAct, false>(v.y, &b, &sb);
        *dg = mul2(mul2(dy, f2(sa, sb)), u);
        *du = mul2(dy, f2(a, b));
    } else if constexpr (kAct == PF_GATE_GELU) {
        const F2 steep = fma2(mul2(g, g), f2(-kLog2e * kGelu3, -kLog2e * kGelu3), f2(-kLog2e * kGelu1, -kLog2e * kGelu1));
        const F2 s = logistic2(mul2(g, steep)), h = mul2(g, s);
        // g (x)' s (1 - s), the first factor within what s (1 - s) leaves of it (nothing from |g| = 11 on)
        const float2 v = split(g);
        const F2 near = f2(fminf(fmaxf(v.x, -40.f), 40.f), fminf(fmaxf(v.y, -40.f), 40.f));
        const F2 w = mul2(near, fma2(mul2(near, near), f2(3.f * kGelu3, 3.f * kGelu3), f2(kGelu1, kGelu1)));
        const F2 slope = fma2(mul2(w, s), fma2(s, negated(one), one), s);
        *dg = mul2(mul2(dy, slope), u);
        *du = mul2(dy, h);
    } else {
        const F2 s = logistic2(mul2(g, f2(-kLog2e, -kLog2e))), h = mul2(g, s);
        const F2 slope = fma2(h, fma2(s, negated(one), one), s);
        *dg = mul2(mul2(dy, slope), u);
        *du = mul2(dy, h);
    }
}

}  // namespace pf
#endif
