// AdamW over a list of tensors: the step that follows the exchange of the flat gradient buffer, in one launch for up to 448 tensors.
//
//   g = grad_scale * grad          m <- beta1 m + (1 - beta1) g          v <- beta2 v + (1 - beta2) g^2
//   p <- p - lr (weight_decay p + (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps))
//
// All arithmetic is in fp32.  The products and sums of m and v are rounded one by one, so that the states (and which way the
// 8-bit ones are rounded) are the same whatever evaluates the formulas; the update of p uses fused multiply-adds and the
// approximate square root and quotient (a few 2^-23 of an update, which is itself small against p).
//
// Bound by memory: every element is read and written once (28 bytes with bf16 gradients, fp32 masters and fp32 states; 10 with bf16
// parameters and 8-bit states).
//
// States in 8 bits: blocks of 256 elements, from the tensor's first; m as e4m3, v as e5m2, each times a power of two per block that
// puts the block's largest value into [128, 256) and [2^14, 2^15): one binade is left for rounding up.  Scaling by a power of two is
// exact, so a value is rounded once.  It is rounded up with the probability of what is cut off (16 random bits from the seed and the
// element's place): with 1 - beta2 below half a step of the format, rounding to nearest would leave v where it is for
// ever.  Values below the smallest normal number of the format (2^-14 and 2^-29 of the largest value's binade) become zero in
// m; in v they become that number, so that a denominator never vanishes.  Elements whose gradients stay below 2^-12 of their block's largest pay for that
// with most of their update (steady gradients, 300 steps, beta 0.9 and 0.98: 0.67 of it at 2^-12 to 2^-13, 0.1 below, 0.02 below 2^-16; 1.01 above).
// What is not finite is stored as NaN and leaves its neighbours alone.
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <cmath>

#include "pf_f32x2.cuh"
#include "pf_internal.h"

namespace pf {
namespace {

constexpr int kAdamThreads = 256, kAdamWarps = kAdamThreads / 32;
constexpr int kAdamVec = 8;                    // elements of a thread at a time
constexpr int kAdamDeep = 2;                   // such pieces in flight
constexpr int kAdamPiece = kAdamThreads * kAdamVec;      // elements of a block at a time; it takes AdamTable::steps of them, at most kAdamDeep
constexpr int kStateBlock = 256;               // elements that share a scale: one piece of a warp
constexpr int kNoVectors = -1;                 // AdamTable::head of a tensor whose arrays never come to 16-byte boundaries together

constexpr int kAdamStarts = 64;

enum ParamKind : int { P_F32 = 0, P_BF16 = 1, P_MASTER = 2 };      // P_MASTER: bf16 parameters that follow fp32 masters

// The tensors of a launch; the table travels in the kernel's parameters.
template <int kMost>
struct AdamTable {
    void* p[kMost];
    float* master[kMost];
    const void* g[kMost];
    void* m[kMost];
    void* v[kMost];
    float* m_scale[kMost];
    float* v_scale[kMost];
    int64_t n[kMost];
    int chunk_prefix[kMost + 1];
    signed char head[kMost];      // elements in front of the first one at which every array is at a 16-byte boundary
    int first, count;             // place of tensor 0 in the caller's list
    int steps;
    unsigned short start[kAdamStarts];      // the tensor of chunk i << start_shift
    int start_shift;
};

// p <- p - lr (wd p + (m r1) / (sqrt(v r2) + eps)), r = 1 / (1 - beta^t), is p - pace (decay p + m / (sqrt(v) + eps / sqrt(r2))) with
// pace = lr r1 / sqrt(r2).
struct AdamHyper {
    float b1, c1, b2, c2, eps, wd;
    float pace, decay, floor, grad_scale;      // floor = eps / sqrt(r2), at least 2^-63
    uint32_t seed;
    const pf_adamw_scalars* scalars;           // replace the last row and the seed
    template <typename R>
    __host__ __device__ void settle(R lr, R correction1, R correction2, float scale, uint32_t bits) {
        const R root = sqrt(correction2), speed = root / correction1;
        pace = static_cast<float>(lr * speed);
        decay = pace != 0.f ? static_cast<float>(wd / speed) : 0.f;
        floor = static_cast<float>(eps * root);
        floor = floor > 0x1p-63f ? floor : 0x1p-63f;
        grad_scale = scale;
        seed = bits;
    }
};

// (Operands below the normal numbers count as zero: the floor is at least 2^-63, the root of the smallest normal number.)
__device__ __forceinline__ float sqrt_fast(float x) {
    float y;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ F2 both(float x) { return f2(x, x); }

// The hyperparameters as pairs of fp32 numbers.
struct AdamPairs {
    F2 b1, c1, b2, c2, floor, decay, minus_pace, grad_scale;
    __device__ __forceinline__ explicit AdamPairs(const AdamHyper& h)
        : b1(both(h.b1)), c1(both(h.c1)), b2(both(h.b2)), c2(both(h.c2)), floor(both(h.floor)), decay(both(h.decay)), minus_pace(both(-h.pace)),
          grad_scale(both(h.grad_scale)) {}
};
// m and v of two elements after the step; b1m = beta1 times a power of two where m is in units of that (and b2v).
__device__ __forceinline__ void moments(const AdamPairs& h, F2 grad, F2 b1m, F2 b2v, F2& m, F2& v) {
    // (A product that is a fused multiply-add with zero is rounded by itself: one that is added as it is gets fused with the sum in the end.)
    const F2 zero = both(0.f), g = mul2(grad, h.grad_scale);
    m = add2(fma2(m, b1m, zero), fma2(g, h.c1, zero));
    v = add2(fma2(v, b2v, zero), fma2(mul2(g, g), h.c2, zero));
}
__device__ __forceinline__ F2 stepped(const AdamPairs& h, F2 p, F2 m, F2 v) {
    const float2 w = split(v);
    const float2 d = split(add2(f2(sqrt_fast(w.x), sqrt_fast(w.y)), h.floor));
    return fma2(h.minus_pace, fma2(h.decay, p, mul2(m, f2(rcp_fast(d.x), rcp_fast(d.y)))), p);
}

__device__ __forceinline__ float bf16_to_f32(unsigned short raw) { return __uint_as_float(static_cast<unsigned>(raw) << 16); }
__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned*>(&t);
}
// Eight elements at a 16-byte boundary, as they lie in memory.
template <typename T> struct Eight;
template <> struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4); }
    __device__ __forceinline__ void get(F2 (&x)[4]) const { x[0] = f2(a.x, a.y); x[1] = f2(a.z, a.w); x[2] = f2(b.x, b.y); x[3] = f2(b.z, b.w); }
    static __device__ __forceinline__ void store(float* p, const F2 (&x)[4]) {
        const float2 c = split(x[0]), d = split(x[1]), e = split(x[2]), f = split(x[3]);
        *reinterpret_cast<float4*>(p) = make_float4(c.x, c.y, d.x, d.y);
        *reinterpret_cast<float4*>(p + 4) = make_float4(e.x, e.y, f.x, f.y);
    }
};
template <> struct Eight<__nv_bfloat16> {
    uint4 a;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void get(F2 (&x)[4]) const {
        const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = f2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const F2 (&x)[4]) {
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = split(x[i]);
            w[i] = pack_bf16(f.x, f.y);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return bf16_to_f32(*reinterpret_cast<const unsigned short*>(p)); }
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

template <int kParam> struct ParamType { using T = __nv_bfloat16; };
template <> struct ParamType<P_F32> { using T = float; };

// What a step reads of the parameters, and the arrays of one tensor.
template <int kParam> struct ReadType { using T = typename ParamType<kParam>::T; };
template <> struct ReadType<P_MASTER> { using T = float; };
template <int kParam, typename G>
struct Arrays {
    using R = typename ReadType<kParam>::T;
    typename ParamType<kParam>::T* p;
    float* master;
    const G* g;
    __device__ __forceinline__ const R* read() const {
        if constexpr (kParam == P_MASTER) return master; else return p;
    }
    __device__ __forceinline__ void store8p(int64_t i, const F2 (&x)[4]) const {
        if constexpr (kParam == P_MASTER) Eight<float>::store(master + i, x);
        Eight<typename ParamType<kParam>::T>::store(p + i, x);
    }
    __device__ __forceinline__ void store1p(int64_t i, float x) const {
        if constexpr (kParam == P_MASTER) master[i] = x;
        store1(p + i, x);
    }
};

template <int kMost>
__device__ __forceinline__ int tensor_of(const AdamTable<kMost>& tb, int chunk) {
    int t = tb.start[chunk >> tb.start_shift];
    while (tb.chunk_prefix[t + 1] <= chunk) ++t;
    return t;
}
// The hyperparameters of this launch, once the kernel before has completed.
__device__ __forceinline__ AdamHyper resolved(AdamHyper h) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (h.scalars) {
        const pf_adamw_scalars& o = *h.scalars;
        h.settle<float>(o.lr, o.correction1, o.correction2, o.grad_scale, o.seed);
    }
    return h;
}

// fp32 states.  A tensor's arrays often start at the same odd element of flat buffers: up to seven elements in front and behind are
// taken one by one, the rest in pieces of eight at 16-byte boundaries.
template <int kMost, int kParam, typename G>
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(const __grid_constant__ AdamTable<kMost> tb, const AdamHyper hyper) {
    const int chunk = blockIdx.x, t = tensor_of(tb, chunk), local = chunk - tb.chunk_prefix[t];
    const AdamHyper h = resolved(hyper);
    using P = typename ParamType<kParam>::T;
    const Arrays<kParam, G> a{static_cast<P*>(tb.p[t]), tb.master[t], static_cast<const G*>(tb.g[t])};
    float* const ms = static_cast<float*>(tb.m[t]);
    float* const vs = static_cast<float*>(tb.v[t]);
    const int64_t n = tb.n[t];
    const AdamPairs hp(h);
    auto single = [&](int64_t i) {
        F2 m = f2(ms[i], 0.f), v = f2(vs[i], 0.f);
        const F2 p = f2(load1(a.read() + i), 0.f);
        moments(hp, f2(load1(a.g + i), 0.f), hp.b1, hp.b2, m, v);
        ms[i] = split(m).x;
        vs[i] = split(v).x;
        a.store1p(i, split(stepped(hp, p, m, v)).x);
    };
    const int head = tb.head[t];
    if (head == kNoVectors) {
        const int64_t beg = static_cast<int64_t>(local) * tb.steps * kAdamPiece, end = min(n, beg + tb.steps * kAdamPiece);
#pragma unroll 4
        for (int64_t i = beg + threadIdx.x; i < end; i += kAdamThreads) single(i);
        return;
    }
    const int64_t vectors = n > head ? (n - head) / kAdamVec : 0;
    if (local == 0) {
        if (static_cast<int>(threadIdx.x) < head && threadIdx.x < n) single(threadIdx.x);
        const int64_t i = head + vectors * kAdamVec + threadIdx.x;
        if (i < n) single(i);
    }
    const int64_t mine = static_cast<int64_t>(local) * tb.steps * kAdamThreads, last = min(vectors, mine + tb.steps * kAdamThreads);
    for (int64_t k = mine + threadIdx.x; k < last; k += kAdamDeep * kAdamThreads) {
        Eight<G> g[kAdamDeep];
        Eight<float> m[kAdamDeep], v[kAdamDeep];
        Eight<typename Arrays<kParam, G>::R> p[kAdamDeep];
#pragma unroll
        for (int u = 0; u < kAdamDeep; ++u) {
            const int64_t i = head + (k + u * kAdamThreads) * kAdamVec;
            if (k + u * kAdamThreads < last) { g[u].load(a.g + i); m[u].load(ms + i); v[u].load(vs + i); p[u].load(a.read() + i); }
        }
#pragma unroll
        for (int u = 0; u < kAdamDeep; ++u) {
            const int64_t i = head + (k + u * kAdamThreads) * kAdamVec;
            if (k + u * kAdamThreads >= last) break;
            F2 fg[4], fm[4], fv[4], fp[4];
            g[u].get(fg);
            m[u].get(fm);
            v[u].get(fv);
            p[u].get(fp);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                moments(hp, fg[e], hp.b1, hp.b2, fm[e], fv[e]);
                fp[e] = stepped(hp, fp[e], fm[e], fv[e]);
            }
            Eight<float>::store(ms + i, fm);
            Eight<float>::store(vs + i, fv);
            a.store8p(i, fp);
        }
    }
}

// ------------------------------------------------------------------------------ 8-bit states
// 32 random bits for an element: a key for the tensor and the seed, then two rounds of multiply and fold.
__device__ __forceinline__ uint32_t tensor_key(uint32_t seed, int tensor) { return seed + static_cast<uint32_t>(tensor + 1) * 0x9E3779B9u; }
constexpr uint32_t kFirstRound = 0xA3D95FA7u, kSecondRound = 0xC8B1F265u, kBeyond32 = 0x9C2F1D35u;
// `x`: (the element's place ^ key) * kFirstRound.  Returns the bits before the last fold, whose upper half is v's and whose halves together are m's.
__device__ __forceinline__ uint32_t random_bits(uint32_t x) { return (x ^ (x >> 15)) * kSecondRound; }

// The two formats: kCut fp32 mantissa bits that are cut off, kTop the binade of a block's largest value, kLeast the least exponent
// field of a scale (so that fp32 numbers below the normal ones are below the format's as well).
struct E4M3 { static constexpr int kCut = 20, kTop = 7, kLeast = 8; };
struct E5M2 { static constexpr int kCut = 21, kTop = 14, kLeast = 16; };

// The exponent field of a block's scale, as in fp32.
template <typename F>
__device__ __forceinline__ int scale_field(uint32_t largest) {
    const int e = static_cast<int>(largest >> 23) - F::kTop;
    return e > F::kLeast ? e : F::kLeast;
}
// A value with 16 random bits added below the cut and the rest cut off: rounded to the format's digits, the sign with them.
template <typename F>
__device__ __forceinline__ uint32_t rounded(uint32_t bits, uint32_t random16) {
    return (bits + random16 * (1u << (F::kCut - 16))) & ~((1u << F::kCut) - 1u);
}

template <__nv_fp8_interpretation_t kFormat>
__device__ __forceinline__ void decode4(uint32_t four, F2* x) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(four >> (16 * i)), kFormat);
        const float2 f = __half22float2(__half2(h));
        x[i] = f2(f.x, f.y);
    }
}
template <__nv_fp8_interpretation_t kFormat>
__device__ __forceinline__ uint32_t encode4(F2 a, F2 b) {
    return static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(split(a), __NV_SATFINITE, kFormat)) |
           static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(split(b), __NV_SATFINITE, kFormat)) << 16;
}
// The larger magnitude, NaN if either is.
__device__ __forceinline__ float larger(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
}

// A block of 256 elements of a warp: lane l has elements 8 l .. 8 l + 7 (kVectors), or l, l + 32, ... of which `left` exist.
template <int kParam, typename G, bool kVectors>
struct StateBlock {
    using A = Arrays<kParam, G>;
    Eight<G> g;
    Eight<typename A::R> p;
    F2 g1[kVectors ? 1 : 4], p1[kVectors ? 1 : 4];
    uint32_t m[2], v[2];
    float m_scale, v_scale;

    static __device__ __forceinline__ int place(int lane, int e) { return kVectors ? lane * 8 + e : e * 32 + lane; }
    __device__ __forceinline__ void load(const A& a, const uint8_t* mc, const uint8_t* vc, const float* msc, const float* vsc, int64_t beg, int left,
                                         int lane) {
        m_scale = msc[beg / kStateBlock];
        v_scale = vsc[beg / kStateBlock];
        if constexpr (kVectors) {
            const int64_t i = beg + lane * 8;
            g.load(a.g + i);
            p.load(a.read() + i);
            const uint2 x = *reinterpret_cast<const uint2*>(mc + i), y = *reinterpret_cast<const uint2*>(vc + i);
            m[0] = x.x; m[1] = x.y; v[0] = y.x; v[1] = y.y;
        } else {
            m[0] = m[1] = v[0] = v[1] = 0;
            float gg[8], pp[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t i = beg + place(lane, e);
                const bool there = place(lane, e) < left;
                gg[e] = there ? load1(a.g + i) : 0.f;
                pp[e] = there ? load1(a.read() + i) : 0.f;
                m[e / 4] |= (there ? static_cast<uint32_t>(mc[i]) : 0u) << (8 * (e % 4));
                v[e / 4] |= (there ? static_cast<uint32_t>(vc[i]) : 0u) << (8 * (e % 4));
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) { g1[e] = f2(gg[2 * e], gg[2 * e + 1]); p1[e] = f2(pp[2 * e], pp[2 * e + 1]); }
        }
    }
    // `scales`: where the block leaves its two scales.
    __device__ __forceinline__ void step(const AdamPairs& h, const A& a, uint8_t* mc, uint8_t* vc, float2& scales, int64_t beg, int left, int lane,
                                         uint32_t key) {
        F2 fg[4], fp[4], fm[4], fv[4];
        if constexpr (kVectors) {
            g.get(fg);
            p.get(fp);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) { fg[e] = g1[e]; fp[e] = p1[e]; }
        }
        decode4<__NV_E4M3>(m[0], fm);
        decode4<__NV_E4M3>(m[1], fm + 2);
        decode4<__NV_E5M2>(v[0], fv);
        decode4<__NV_E5M2>(v[1], fv + 2);
        // (scale and beta in one factor: the scale is a power of two)
        const F2 b1m = mul2(h.b1, both(m_scale)), b2v = mul2(h.b2, both(v_scale));
        float top_m = 0.f, top_v = 0.f;
        uint32_t low_v = 0xffffffffu;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            moments(h, fg[e], b1m, b2v, fm[e], fv[e]);
            fp[e] = stepped(h, fp[e], fm[e], fv[e]);
            if constexpr (!kVectors) {
                const float2 x = split(fm[e]), y = split(fv[e]);
                const bool one = place(lane, 2 * e) < left, two = place(lane, 2 * e + 1) < left;
                fm[e] = f2(one ? x.x : 0.f, two ? x.y : 0.f);
                fv[e] = f2(one ? y.x : 0.f, two ? y.y : 0.f);
            }
            const float2 x = split(fm[e]), y = split(fv[e]);
            top_m = larger(larger(top_m, x.x), x.y);
            top_v = larger(larger(top_v, y.x), y.y);
            low_v = min(min(low_v, __float_as_uint(y.x)), __float_as_uint(y.y));
        }
        if constexpr (kVectors) {
            a.store8p(beg + lane * 8, fp);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 x = split(fp[e / 2]);
                if (place(lane, e) < left) a.store1p(beg + place(lane, e), e % 2 ? x.y : x.x);
            }
        }
        constexpr uint32_t kInf = 0x7f800000u;
        uint32_t most_m = __reduce_max_sync(0xffffffffu, __float_as_uint(top_m)), most_v = __reduce_max_sync(0xffffffffu, __float_as_uint(top_v));
        uint32_t nan_m[2] = {0, 0}, nan_v[2] = {0, 0};
        if (most_m >= kInf || most_v >= kInf) {      // what is not finite is taken as zero, and its codes as NaN in the end
            most_m = most_v = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float2 x = split(fm[e / 2]), y = split(fv[e / 2]);
                float& xe = e % 2 ? x.y : x.x;
                float& ye = e % 2 ? y.y : y.x;
                if ((__float_as_uint(xe) & 0x7fffffffu) >= kInf) { xe = 0.f; nan_m[e / 4] |= 0x7fu << (8 * (e % 4)); }
                if ((__float_as_uint(ye) & 0x7fffffffu) >= kInf) { ye = 0.f; nan_v[e / 4] |= 0x7fu << (8 * (e % 4)); }
                most_m = max(most_m, __float_as_uint(xe) & 0x7fffffffu);
                most_v = max(most_v, __float_as_uint(ye));
                fm[e / 2] = f2(x.x, x.y);
                fv[e / 2] = f2(y.x, y.y);
            }
            most_m = __reduce_max_sync(0xffffffffu, most_m);
            most_v = __reduce_max_sync(0xffffffffu, most_v);
        }
        const int field_m = scale_field<E4M3>(most_m), field_v = scale_field<E5M2>(most_v);
        const F2 over_m = both(__int_as_float((254 - field_m) << 23)), over_v = both(__int_as_float((254 - field_v) << 23));      // 1 / scale
        const uint32_t least_v = static_cast<uint32_t>(field_v - 14) << 23;      // e5m2's smallest normal number, 2^-14
        const F2 down = both(0x1p-120f), up = both(0x1p120f), zero = both(0.f);
        const uint32_t beyond = key + static_cast<uint32_t>(beg >> 32) * kBeyond32;      // (a block lies on one side of 2^32)
        const uint32_t first = ((static_cast<uint32_t>(beg) + static_cast<uint32_t>(lane) * 8) ^ (beyond & ~7u)) * kFirstRound;
        uint32_t zm[8], zv[8];
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const float2 x = split(fm[n / 2]), y = split(fv[n / 2]);
            // (eight places from a multiple of eight on differ from the key in three bits apart from the others, so the product is a sum)
            const uint32_t start = kVectors ? first + ((beyond & 7u) ^ n) * kFirstRound
                                            : ((static_cast<uint32_t>(beg) + static_cast<uint32_t>(place(lane, n))) ^ beyond) * kFirstRound;
            const uint32_t r = random_bits(start), upper = r >> 16;
            zm[n] = rounded<E4M3>(__float_as_uint(n % 2 ? x.y : x.x), (r ^ upper) & 0xffffu);
            zv[n] = rounded<E5M2>(__float_as_uint(n % 2 ? y.y : y.x), upper);
        }
        // (few blocks have a v that small, or none: without one the rounded values need no limit)
        if (__any_sync(0xffffffffu, low_v < least_v)) {
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                const float2 y = split(fv[n / 2]);
                zv[n] = max(zv[n], min(__float_as_uint(n % 2 ? y.y : y.x), 1u) * least_v);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            // m below e4m3's smallest normal number, 2^-6, becomes zero: that is 2^-126 in between (and minus zero plus zero is zero)
            const F2 sm = mul2(f2(__uint_as_float(zm[2 * e]), __uint_as_float(zm[2 * e + 1])), over_m);
            fm[e] = fma2(mul2_flush(sm, down), up, zero);
            fv[e] = mul2(f2(__uint_as_float(zv[2 * e]), __uint_as_float(zv[2 * e + 1])), over_v);
        }
        // (a value of fp32's highest binade that is rounded up is an infinity in between, and 256 or 2^15 as a code)
        if (field_m == 254 - E4M3::kTop || field_v == 254 - E5M2::kTop) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 x = split(fm[e]), y = split(fv[e]);
                fm[e] = f2(fmaxf(fminf(x.x, 256.f), -256.f), fmaxf(fminf(x.y, 256.f), -256.f));
                fv[e] = f2(fminf(y.x, 0x1p15f), fminf(y.y, 0x1p15f));
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            m[i] = encode4<__NV_E4M3>(fm[2 * i], fm[2 * i + 1]) | nan_m[i];
            v[i] = encode4<__NV_E5M2>(fv[2 * i], fv[2 * i + 1]) | nan_v[i];
        }
        if (lane == 0) scales = make_float2(__int_as_float(field_m << 23), __int_as_float(field_v << 23));
        if constexpr (kVectors) {
            const int64_t i = beg + lane * 8;
            *reinterpret_cast<uint2*>(mc + i) = make_uint2(m[0], m[1]);
            *reinterpret_cast<uint2*>(vc + i) = make_uint2(v[0], v[1]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t i = beg + place(lane, e);
                if (place(lane, e) >= left) continue;
                mc[i] = static_cast<uint8_t>(m[e / 4] >> (8 * (e % 4)));
                vc[i] = static_cast<uint8_t>(v[e / 4] >> (8 * (e % 4)));
            }
        }
    }
};

// Pieces of a thread at a time: two where all is in 16 bits and less (26.8 M elements: 51 us, with one 59); parameters read in fp32 have enough under
// way with one (15.1 M with masters: 41.0 us, with two 43.7; 17.3 M of fp32: 45.2 and 46.7).
template <int kParam> constexpr int kAdam8Deep = kParam == P_BF16 ? kAdamDeep : 1;

template <int kMost, int kParam, typename G>
__global__ void __launch_bounds__(kAdamThreads, 4) adamw8_kernel(const __grid_constant__ AdamTable<kMost> tb, const AdamHyper hyper) {
    const int chunk = blockIdx.x, t = tensor_of(tb, chunk), local = chunk - tb.chunk_prefix[t];
    const AdamHyper h = resolved(hyper);
    const AdamPairs hp(h);
    using P = typename ParamType<kParam>::T;
    const Arrays<kParam, G> a{static_cast<P*>(tb.p[t]), tb.master[t], static_cast<const G*>(tb.g[t])};
    uint8_t* const mc = static_cast<uint8_t*>(tb.m[t]);
    uint8_t* const vc = static_cast<uint8_t*>(tb.v[t]);
    const int64_t n = tb.n[t];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t key = tensor_key(h.seed, tb.first + t);
    float* const msc = tb.m_scale[t];
    float* const vsc = tb.v_scale[t];
    const int64_t beg = static_cast<int64_t>(local) * tb.steps * kAdamPiece + warp * kStateBlock;
    // The scales of a block's pieces are stored together in the end: one by one they are parts of 32-byte sectors that other warps still read, which
    // kept those waiting (26.8 M elements: 57 us, 93 with half of the loads in flight; 53 without the stores).
    constexpr int kDeep = kAdam8Deep<kParam>;
    __shared__ float2 scales[kDeep][kAdamWarps];
    if (tb.head[t] == 0 && beg + (tb.steps - 1) * kAdamPiece + kStateBlock <= n) {      // whole blocks, all on the way at once
        StateBlock<kParam, G, true> b[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; ++u)
            if (u < tb.steps) b[u].load(a, mc, vc, msc, vsc, beg + u * kAdamPiece, kStateBlock, lane);
#pragma unroll
        for (int u = 0; u < kDeep; ++u)
            if (u < tb.steps) b[u].step(hp, a, mc, vc, scales[u][warp], beg + u * kAdamPiece, kStateBlock, lane, key);
    } else {
#pragma unroll 1
        for (int u = 0; u < tb.steps; ++u) {
            const int64_t at = beg + u * kAdamPiece;
            if (at >= n) break;
            const int left = n - at < kStateBlock ? static_cast<int>(n - at) : kStateBlock;
            StateBlock<kParam, G, false> b;
            b.load(a, mc, vc, msc, vsc, at, left, lane);
            b.step(hp, a, mc, vc, scales[u][warp], at, left, lane, key);
        }
    }
    __syncthreads();
    const int64_t first = static_cast<int64_t>(local) * tb.steps * kAdamWarps, i = first + lane;
    if (warp < 2 && lane < tb.steps * kAdamWarps && i * kStateBlock < n) {
        const float2 x = scales[lane / kAdamWarps][lane % kAdamWarps];
        if (warp == 0) msc[i] = x.x; else vsc[i] = x.y;
    }
}

// ------------------------------------------------------------------------------ launches
struct AdamList {
    void* const* p;
    float* const* master;
    const void* const* g;
    void* const* m;
    void* const* v;
    float* const* m_scale;
    float* const* v_scale;
    const int64_t* n;
    int count, param_dtype, grad_dtype;
    bool state8;
};

// Elements in front of the first one at which every array of tensor i is at its boundary.
int head_of(const AdamList& l, int i) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(l.p[i]), w = l.master ? reinterpret_cast<uintptr_t>(l.master[i]) : 0, g = reinterpret_cast<uintptr_t>(l.g[i]);
    const uintptr_t m = reinterpret_cast<uintptr_t>(l.m[i]), v = reinterpret_cast<uintptr_t>(l.v[i]);
    const size_t sp = dtype_size(l.param_dtype), sg = dtype_size(l.grad_dtype);
    if (l.state8) return ((p | w | g) & 15) == 0 && ((m | v) & 7) == 0 ? 0 : kNoVectors;
    for (size_t h = 0; h < kAdamVec; ++h)
        if ((((p + h * sp) | (l.master ? w + h * 4 : 0) | (g + h * sg) | (m + h * 4) | (v + h * 4)) & 15) == 0) return static_cast<int>(h);
    return kNoVectors;
}

constexpr int kAdamFill = 8;      // blocks of an SM, those that wait for their turn among them
template <int kMost, int kParam, typename G>
cudaError_t adamw_by(const AdamList& l, const AdamHyper& h, cudaStream_t stream) {
    int64_t pieces = 0;
    for (int i = 0; i < l.count; ++i) pieces += ceil_div(l.n[i], kAdamPiece);
    // a block takes several pieces where enough blocks are left for every SM
    const int64_t fill = static_cast<int64_t>(num_sms()) * kAdamFill;
    const int deep = l.state8 ? kAdam8Deep<kParam> : kAdamDeep, steps = pieces >= deep * fill ? deep : 1;
    int i = 0;
    while (i < l.count) {
        AdamTable<kMost> tb;
        tb.count = 0;
        tb.first = i;
        tb.chunk_prefix[0] = 0;
        tb.steps = steps;
        for (; i < l.count && i - tb.first < kMost; ++i) {      // (empty tensors keep their place)
            const int64_t chunks = ceil_div(l.n[i], static_cast<int64_t>(steps) * kAdamPiece);
            if (tb.chunk_prefix[tb.count] + chunks > 0x7fffffff) break;
            const int c = tb.count++;
            tb.p[c] = l.p[i];
            tb.master[c] = l.master ? l.master[i] : nullptr;
            tb.g[c] = l.g[i];
            tb.m[c] = l.m[i];
            tb.v[c] = l.v[i];
            tb.m_scale[c] = l.state8 ? l.m_scale[i] : nullptr;
            tb.v_scale[c] = l.state8 ? l.v_scale[i] : nullptr;
            tb.n[c] = l.n[i];
            tb.head[c] = static_cast<signed char>(head_of(l, i));
            tb.chunk_prefix[c + 1] = tb.chunk_prefix[c] + static_cast<int>(chunks);
        }
        if (tb.count == 0) return cudaErrorInvalidValue;
        const int blocks = tb.chunk_prefix[tb.count];
        if (blocks == 0) continue;
        tb.start_shift = 0;
        while ((blocks - 1) >> tb.start_shift >= kAdamStarts) ++tb.start_shift;
        for (int c = 0, t = 0; c < blocks; c += 1 << tb.start_shift) {
            while (tb.chunk_prefix[t + 1] <= c) ++t;
            tb.start[c >> tb.start_shift] = static_cast<unsigned short>(t);
            if (c > 0x7fffffff - (1 << tb.start_shift)) break;
        }
        const auto kernel = l.state8 ? adamw8_kernel<kMost, kParam, G> : adamw_kernel<kMost, kParam, G>;
        const cudaError_t e = launch_beside(kernel, dim3(static_cast<unsigned>(blocks)), kAdamThreads, 0, 1, stream, tb, h);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}
template <int kParam, typename G>
cudaError_t adamw_sized(const AdamList& l, const AdamHyper& h, cudaStream_t stream) {
    // (short lists have tables of their own, as in pf_pack.cu: a launch copies all of it, 31 KB for 448 tensors)
    if (l.count <= 16) return adamw_by<16, kParam, G>(l, h, stream);
    if (l.count <= 64) return adamw_by<64, kParam, G>(l, h, stream);
    if (l.count <= 192) return adamw_by<192, kParam, G>(l, h, stream);
    return adamw_by<448, kParam, G>(l, h, stream);
}
template <int kParam>
cudaError_t adamw_graded(const AdamList& l, const AdamHyper& h, cudaStream_t stream) {
    if (l.grad_dtype == PF_BF16) return adamw_sized<kParam, __nv_bfloat16>(l, h, stream);
    return adamw_sized<kParam, float>(l, h, stream);
}

}  // namespace
}  // namespace pf

using namespace pf;

extern "C" int pf_adamw_step(void* const* params, float* const* masters, const void* const* grads, void* const* m, void* const* v,
                             float* const* m_scales, float* const* v_scales, const int64_t* numels, int count, int param_dtype,
                             int grad_dtype, int state, const pf_adamw* hyper, const pf_adamw_scalars* scalars, void* cuda_stream) {
    if (!valid_dtype(param_dtype) || !valid_dtype(grad_dtype) || (state != PF_STATE_F32 && state != PF_STATE_8BIT)) return PF_ERR_INVALID_ARG;
    if (count < 0 || !hyper || (masters && param_dtype != PF_BF16)) return PF_ERR_INVALID_ARG;
    const pf_adamw& o = *hyper;
    const bool state8 = state == PF_STATE_8BIT;
    if (!(o.beta1 >= 0 && o.beta1 < 1) || !(o.beta2 >= 0 && o.beta2 < 1) || !(o.eps >= 0) || !std::isfinite(o.eps) || !std::isfinite(o.weight_decay))
        return PF_ERR_INVALID_ARG;
    if (!scalars && (!std::isfinite(o.lr) || o.step < 1 || !std::isfinite(o.grad_scale))) return PF_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(scalars) % 4 != 0) return PF_ERR_INVALID_ARG;
    if (count > 0 && (!params || !grads || !m || !v || !numels || (state8 && (!m_scales || !v_scales)))) return PF_ERR_INVALID_ARG;
    const auto f32 = [](const void* p) { return p && elem_aligned(p, PF_F32); };
    for (int i = 0; i < count; ++i) {
        if (numels[i] < 0) return PF_ERR_INVALID_ARG;
        if (numels[i] == 0) continue;
        if (!params[i] || !elem_aligned(params[i], param_dtype) || !grads[i] || !elem_aligned(grads[i], grad_dtype)) return PF_ERR_INVALID_ARG;
        if (masters && !f32(masters[i])) return PF_ERR_INVALID_ARG;
        if (state8 ? !m[i] || !v[i] || !f32(m_scales[i]) || !f32(v_scales[i]) : !f32(m[i]) || !f32(v[i])) return PF_ERR_INVALID_ARG;
        if (numels[i] > (1LL << 42)) return PF_ERR_UNSUPPORTED;
    }
    AdamHyper h = {};
    h.b1 = static_cast<float>(o.beta1);
    h.c1 = static_cast<float>(1.0 - o.beta1);
    h.b2 = static_cast<float>(o.beta2);
    h.c2 = static_cast<float>(1.0 - o.beta2);
    h.eps = static_cast<float>(o.eps);
    h.wd = static_cast<float>(o.weight_decay);
    h.scalars = scalars;
    if (!scalars) {
        const double t = static_cast<double>(o.step);
        h.settle<double>(o.lr, 1.0 - std::pow(o.beta1, t), 1.0 - std::pow(o.beta2, t), o.grad_scale, o.seed);
    }
    const AdamList l{params, masters, grads, m, v, m_scales, v_scales, numels, count, param_dtype, grad_dtype, state8};
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (param_dtype == PF_F32) PF_CUDA(adamw_graded<P_F32>(l, h, stream));
    else if (masters) PF_CUDA(adamw_graded<P_MASTER>(l, h, stream));
    else PF_CUDA(adamw_graded<P_BF16>(l, h, stream));
    return PF_OK;
}
