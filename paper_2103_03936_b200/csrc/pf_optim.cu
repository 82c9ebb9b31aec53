// AdamW over a list of tensors: the step that follows the exchange of the flat gradient buffer, in one launch for up to 256 tensors.
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
// m; in v they become that number, so that a denominator never vanishes.  What is not finite is stored as NaN and leaves its neighbours alone.
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <cmath>

#include "pf_internal.h"

namespace pf {
namespace {

constexpr int kAdamThreads = 256, kAdamWarps = kAdamThreads / 32;
constexpr int kAdamVec = 8;                    // elements of a thread at a time
constexpr int kAdamDeep = 2;                   // such pieces in flight
constexpr int kAdamChunk = kAdamThreads * kAdamVec * kAdamDeep;
constexpr int kStateBlock = 256;               // elements that share a scale: one piece of a warp
constexpr int kNoVectors = -1;                 // AdamTable::head of a tensor whose arrays never come to 16-byte boundaries together

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
};

struct AdamHyper {
    float b1, c1, b2, c2, eps, wd;
    float lr, r1, r2, grad_scale;      // r1 = 1 / (1 - beta1^t), r2 likewise
    uint32_t seed;
    const pf_adamw_scalars* scalars;   // replace lr, r1, r2, grad_scale and seed
};

__device__ __forceinline__ float sqrt_fast(float x) {
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ void moments(const AdamHyper& h, float grad, float& m, float& v) {
    const float g = __fmul_rn(grad, h.grad_scale);
    m = __fadd_rn(__fmul_rn(m, h.b1), __fmul_rn(g, h.c1));
    v = __fadd_rn(__fmul_rn(v, h.b2), __fmul_rn(__fmul_rn(g, g), h.c2));
}
__device__ __forceinline__ float stepped(const AdamHyper& h, float p, float m, float v) {
    const float u = __fdividef(m * h.r1, sqrt_fast(v * h.r2) + h.eps);
    return fmaf(-h.lr, fmaf(h.wd, p, u), p);
}

__device__ __forceinline__ float bf16_to_f32(unsigned short raw) { return __uint_as_float(static_cast<unsigned>(raw) << 16); }
__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned*>(&t);
}
// Eight elements at a 16-byte boundary (bf16) or two (fp32).
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&x)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return bf16_to_f32(*reinterpret_cast<const unsigned short*>(p)); }
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

template <int kParam> struct ParamType { using T = __nv_bfloat16; };
template <> struct ParamType<P_F32> { using T = float; };

// The arrays of one tensor.
template <int kParam, typename G>
struct Arrays {
    typename ParamType<kParam>::T* p;
    float* master;
    const G* g;
    __device__ __forceinline__ void load8p(int64_t i, float (&x)[8]) const {
        if constexpr (kParam == P_MASTER) load8(master + i, x); else load8(p + i, x);
    }
    __device__ __forceinline__ void store8p(int64_t i, const float (&x)[8]) const {
        if constexpr (kParam == P_MASTER) store8(master + i, x);
        store8(p + i, x);
    }
    __device__ __forceinline__ float load1p(int64_t i) const {
        if constexpr (kParam == P_MASTER) return master[i]; else return load1(p + i);
    }
    __device__ __forceinline__ void store1p(int64_t i, float x) const {
        if constexpr (kParam == P_MASTER) master[i] = x;
        store1(p + i, x);
    }
};

template <int kMost>
__device__ __forceinline__ int tensor_of(const AdamTable<kMost>& tb, int chunk) {
    int lo = 0, hi = tb.count;      // chunk_prefix[lo] <= chunk < chunk_prefix[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (tb.chunk_prefix[mid] <= chunk) lo = mid; else hi = mid;
    }
    return lo;
}
// The hyperparameters of this launch, once the kernel before has completed.
__device__ __forceinline__ AdamHyper resolved(AdamHyper h) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (h.scalars) {
        h.lr = h.scalars->lr;
        h.r1 = 1.f / h.scalars->correction1;
        h.r2 = 1.f / h.scalars->correction2;
        h.grad_scale = h.scalars->grad_scale;
        h.seed = h.scalars->seed;
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
    auto single = [&](int64_t i) {
        float m = ms[i], v = vs[i];
        const float p = a.load1p(i);
        moments(h, load1(a.g + i), m, v);
        ms[i] = m;
        vs[i] = v;
        a.store1p(i, stepped(h, p, m, v));
    };
    const int head = tb.head[t];
    if (head == kNoVectors) {
        const int64_t beg = static_cast<int64_t>(local) * kAdamChunk, end = beg + kAdamChunk < n ? beg + kAdamChunk : n;
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
    const int64_t first = static_cast<int64_t>(local) * (kAdamThreads * kAdamDeep) + threadIdx.x;
    float g[kAdamDeep][8], m[kAdamDeep][8], v[kAdamDeep][8], p[kAdamDeep][8];
#pragma unroll
    for (int u = 0; u < kAdamDeep; ++u) {
        const int64_t k = first + u * kAdamThreads, i = head + k * kAdamVec;
        if (k < vectors) { load8(a.g + i, g[u]); load8(ms + i, m[u]); load8(vs + i, v[u]); a.load8p(i, p[u]); }
    }
#pragma unroll
    for (int u = 0; u < kAdamDeep; ++u) {
        const int64_t k = first + u * kAdamThreads, i = head + k * kAdamVec;
        if (k >= vectors) break;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            moments(h, g[u][e], m[u][e], v[u][e]);
            p[u][e] = stepped(h, p[u][e], m[u][e], v[u][e]);
        }
        store8(ms + i, m[u]);
        store8(vs + i, v[u]);
        a.store8p(i, p[u]);
    }
}

// ------------------------------------------------------------------------------ 8-bit states
// 32 random bits for an element: a key for the tensor and the seed, then two rounds of multiply and fold.
__device__ __forceinline__ uint32_t tensor_key(uint32_t seed, int tensor) { return seed + static_cast<uint32_t>(tensor + 1) * 0x9E3779B9u; }
__device__ __forceinline__ uint32_t random_bits(uint32_t key, uint32_t index) {
    uint32_t x = (index ^ key) * 0xA3D95FA7u;
    x ^= x >> 15;
    x *= 0xC8B1F265u;
    return x ^ (x >> 16);
}

// The two formats: kCut fp32 mantissa bits that are cut off, kBias the exponent bias, kTop the binade of a block's largest value,
// kLeast the least exponent field of a scale (so that fp32 numbers below the normal ones are below the format's as well).
struct E4M3 { static constexpr int kCut = 20, kBias = 7, kTop = 7, kLeast = 8; };
struct E5M2 { static constexpr int kCut = 21, kBias = 15, kTop = 14, kLeast = 16; };

template <typename F>
__device__ __forceinline__ int scale_field(uint32_t largest) {
    const int e = static_cast<int>(largest >> 23) - F::kTop;
    return e > F::kLeast ? e : F::kLeast;
}
// The code of a value's magnitude: its bits with the exponent moved by the scale, random bits added below the cut, the rest taken.
template <typename F, bool kKeep>
__device__ __forceinline__ uint32_t coded(uint32_t magnitude, uint32_t random16, int field) {
    const int s = static_cast<int>(magnitude + (random16 << (F::kCut - 16)) - (static_cast<uint32_t>(field - F::kBias) << 23));
    constexpr int kNormal = 1 << 23;
    if (s < kNormal) return kKeep && magnitude != 0 ? static_cast<uint32_t>(kNormal >> F::kCut) : 0u;
    return static_cast<uint32_t>(s) >> F::kCut;
}

template <__nv_fp8_interpretation_t kFormat>
__device__ __forceinline__ void decode4(uint32_t four, float scale, float* x) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(four >> (16 * i)), kFormat);
        const float2 f = __half22float2(__half2(h));
        x[2 * i] = f.x * scale;
        x[2 * i + 1] = f.y * scale;
    }
}

// A block of 256 elements of a warp: lane l has elements 8 l .. 8 l + 7 (kVectors), or l, l + 32, ... of which `left` exist.
template <int kParam, typename G, bool kVectors>
struct StateBlock {
    float g[8], p[8];
    uint32_t m[2], v[2];
    float m_scale, v_scale;

    static __device__ __forceinline__ int place(int lane, int e) { return kVectors ? lane * 8 + e : e * 32 + lane; }
    __device__ __forceinline__ void load(const Arrays<kParam, G>& a, const uint8_t* mc, const uint8_t* vc, const float* msc, const float* vsc,
                                         int64_t beg, int left, int lane) {
        m_scale = msc[beg / kStateBlock];
        v_scale = vsc[beg / kStateBlock];
        if constexpr (kVectors) {
            const int64_t i = beg + lane * 8;
            load8(a.g + i, g);
            a.load8p(i, p);
            const uint2 x = *reinterpret_cast<const uint2*>(mc + i), y = *reinterpret_cast<const uint2*>(vc + i);
            m[0] = x.x; m[1] = x.y; v[0] = y.x; v[1] = y.y;
        } else {
            m[0] = m[1] = v[0] = v[1] = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t i = beg + place(lane, e);
                const bool there = place(lane, e) < left;
                g[e] = there ? load1(a.g + i) : 0.f;
                p[e] = there ? a.load1p(i) : 0.f;
                m[e / 4] |= (there ? static_cast<uint32_t>(mc[i]) : 0u) << (8 * (e % 4));
                v[e / 4] |= (there ? static_cast<uint32_t>(vc[i]) : 0u) << (8 * (e % 4));
            }
        }
    }
    __device__ __forceinline__ void step(const AdamHyper& h, const Arrays<kParam, G>& a, uint8_t* mc, uint8_t* vc, float* msc, float* vsc, int64_t beg,
                                         int left, int lane, uint32_t key) {
        float fm[8], fv[8];
        decode4<__NV_E4M3>(m[0], m_scale, fm);
        decode4<__NV_E4M3>(m[1], m_scale, fm + 4);
        decode4<__NV_E5M2>(v[0], v_scale, fv);
        decode4<__NV_E5M2>(v[1], v_scale, fv + 4);
        uint32_t most_m = 0, most_v = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            moments(h, g[e], fm[e], fv[e]);
            p[e] = stepped(h, p[e], fm[e], fv[e]);
            if (!kVectors && place(lane, e) >= left) fm[e] = fv[e] = 0.f;
            most_m = max(most_m, __float_as_uint(fm[e]) & 0x7fffffffu);
            most_v = max(most_v, __float_as_uint(fv[e]) & 0x7fffffffu);
        }
        most_m = __reduce_max_sync(0xffffffffu, most_m);
        most_v = __reduce_max_sync(0xffffffffu, most_v);
        constexpr uint32_t kInf = 0x7f800000u;
        const bool finite = most_m < kInf && most_v < kInf;
        if (!finite) {      // the largest of the finite ones
            most_m = most_v = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t x = __float_as_uint(fm[e]) & 0x7fffffffu, y = __float_as_uint(fv[e]) & 0x7fffffffu;
                if (x < kInf) most_m = max(most_m, x);
                if (y < kInf) most_v = max(most_v, y);
            }
            most_m = __reduce_max_sync(0xffffffffu, most_m);
            most_v = __reduce_max_sync(0xffffffffu, most_v);
        }
        const int field_m = scale_field<E4M3>(most_m), field_v = scale_field<E5M2>(most_v);
        m[0] = m[1] = v[0] = v[1] = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int64_t i = beg + place(lane, e);
            const uint32_t r = random_bits(key + static_cast<uint32_t>(i >> 32) * 0x9C2F1D35u, static_cast<uint32_t>(i));
            const uint32_t x = __float_as_uint(fm[e]), size = x & 0x7fffffffu, y = __float_as_uint(fv[e]) & 0x7fffffffu;
            uint32_t cm = coded<E4M3, false>(size, r & 0xffffu, field_m), cv = coded<E5M2, true>(y, r >> 16, field_v);
            if (cm != 0) cm |= (x >> 24) & 0x80u;
            if (!finite) {
                if (size >= kInf) cm = 0x7fu;
                if (y >= kInf) cv = 0x7fu;
            }
            m[e / 4] |= cm << (8 * (e % 4));
            v[e / 4] |= cv << (8 * (e % 4));
        }
        if (lane == 0) {
            msc[beg / kStateBlock] = __int_as_float(field_m << 23);
            vsc[beg / kStateBlock] = __int_as_float(field_v << 23);
        }
        if constexpr (kVectors) {
            const int64_t i = beg + lane * 8;
            *reinterpret_cast<uint2*>(mc + i) = make_uint2(m[0], m[1]);
            *reinterpret_cast<uint2*>(vc + i) = make_uint2(v[0], v[1]);
            a.store8p(i, p);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t i = beg + place(lane, e);
                if (place(lane, e) >= left) continue;
                mc[i] = static_cast<uint8_t>(m[e / 4] >> (8 * (e % 4)));
                vc[i] = static_cast<uint8_t>(v[e / 4] >> (8 * (e % 4)));
                a.store1p(i, p[e]);
            }
        }
    }
};

template <int kMost, int kParam, typename G>
__global__ void __launch_bounds__(kAdamThreads) adamw8_kernel(const __grid_constant__ AdamTable<kMost> tb, const AdamHyper hyper) {
    const int chunk = blockIdx.x, t = tensor_of(tb, chunk), local = chunk - tb.chunk_prefix[t];
    const AdamHyper h = resolved(hyper);
    using P = typename ParamType<kParam>::T;
    const Arrays<kParam, G> a{static_cast<P*>(tb.p[t]), tb.master[t], static_cast<const G*>(tb.g[t])};
    uint8_t* const mc = static_cast<uint8_t*>(tb.m[t]);
    uint8_t* const vc = static_cast<uint8_t*>(tb.v[t]);
    const int64_t n = tb.n[t];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t key = tensor_key(h.seed, tb.first + t);
    const int64_t beg = static_cast<int64_t>(local) * kAdamChunk + warp * kStateBlock;
    constexpr int kApart = kAdamWarps * kStateBlock;
    if (tb.head[t] == 0 && beg + (kAdamDeep - 1) * kApart + kStateBlock <= n) {
        StateBlock<kParam, G, true> b[kAdamDeep];
#pragma unroll
        for (int u = 0; u < kAdamDeep; ++u) b[u].load(a, mc, vc, tb.m_scale[t], tb.v_scale[t], beg + u * kApart, kStateBlock, lane);
#pragma unroll
        for (int u = 0; u < kAdamDeep; ++u)
            b[u].step(h, a, mc, vc, tb.m_scale[t], tb.v_scale[t], beg + u * kApart, kStateBlock, lane, key);
        return;
    }
#pragma unroll 1
    for (int u = 0; u < kAdamDeep; ++u) {
        const int64_t at = beg + u * kApart;
        if (at >= n) break;
        const int left = n - at < kStateBlock ? static_cast<int>(n - at) : kStateBlock;
        StateBlock<kParam, G, false> b;
        b.load(a, mc, vc, tb.m_scale[t], tb.v_scale[t], at, left, lane);
        b.step(h, a, mc, vc, tb.m_scale[t], tb.v_scale[t], at, left, lane, key);
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
    struct { const void* p; unsigned size, boundary; } arrays[5] = {
        {l.p[i], static_cast<unsigned>(dtype_size(l.param_dtype)), 16}, {l.master ? l.master[i] : nullptr, 4, 16},
        {l.g[i], static_cast<unsigned>(dtype_size(l.grad_dtype)), 16}, {l.m[i], l.state8 ? 1u : 4u, l.state8 ? 8u : 16u},
        {l.v[i], l.state8 ? 1u : 4u, l.state8 ? 8u : 16u}};
    for (int h = 0; h < (l.state8 ? 1 : kAdamVec); ++h) {
        bool all = true;
        for (const auto& a : arrays)      // (no masters: nothing to align)
            if (a.p) all = all && (reinterpret_cast<uintptr_t>(a.p) + h * a.size) % a.boundary == 0;
        if (all) return h;
    }
    return kNoVectors;
}

template <int kMost, int kParam, typename G>
cudaError_t adamw_by(const AdamList& l, const AdamHyper& h, cudaStream_t stream) {
    int i = 0;
    while (i < l.count) {
        AdamTable<kMost> tb;
        tb.count = 0;
        tb.first = i;
        tb.chunk_prefix[0] = 0;
        for (; i < l.count && i - tb.first < kMost; ++i) {      // (empty tensors keep their place)
            const int64_t chunks = ceil_div(l.n[i], kAdamChunk);
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
        const auto kernel = l.state8 ? adamw8_kernel<kMost, kParam, G> : adamw_kernel<kMost, kParam, G>;
        const cudaError_t e = launch_beside(kernel, dim3(static_cast<unsigned>(blocks)), kAdamThreads, 0, 1, stream, tb, h);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}
template <int kParam, typename G>
cudaError_t adamw_sized(const AdamList& l, const AdamHyper& h, cudaStream_t stream) {
    // (short lists have a table of their own, as in pf_pack.cu: a launch copies all of it)
    if (l.count <= 16) return adamw_by<16, kParam, G>(l, h, stream);
    return adamw_by<256, kParam, G>(l, h, stream);
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
        h.lr = static_cast<float>(o.lr);
        h.r1 = static_cast<float>(1.0 / (1.0 - std::pow(o.beta1, static_cast<double>(o.step))));
        h.r2 = static_cast<float>(1.0 / (1.0 - std::pow(o.beta2, static_cast<double>(o.step))));
        h.grad_scale = o.grad_scale;
        h.seed = o.seed;
    }
    const AdamList l{params, masters, grads, m, v, m_scales, v_scales, numels, count, param_dtype, grad_dtype, state8};
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (param_dtype == PF_F32) PF_CUDA(adamw_graded<P_F32>(l, h, stream));
    else if (masters) PF_CUDA(adamw_graded<P_MASTER>(l, h, stream));
    else PF_CUDA(adamw_graded<P_BF16>(l, h, stream));
    return PF_OK;
}
