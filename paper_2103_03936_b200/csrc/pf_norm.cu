// A residual's addition and the root-mean-square norm that follows, forward (rows in the inputs' type, in 8 bits with scales, or both) and
// backward.
//
// For a row of `width` elements: h = x + residual, y = n w with n = h r, r = 1 / sqrt(mean(h^2) + eps).  In 8 bits: for each block of elements
// s = max |y| / 448 and codes y / s as e4m3 floats.  Backward, for the gradients g of y and d of h: s = g w, dx = d + r (s - n mean(s n)),
// dw = sum of g n over the rows; r is computed again.
//
// Bound by memory: every row is read and written once, and stays in registers between its sum of squares and its output.  A lane has
// sixteen elements in units of 16 bytes, a row is as many lanes as that takes (four for 64 elements, 32 warps for 16384), and short rows
// share a warp or a block.  Blocks stay and walk over rows: the sums for dw are in registers, and a thread's next row is on its way into its own places of shared
// memory while the present one is computed.
#include <algorithm>
#include <type_traits>

#include "pf_internal.h"
#include "pf_rows.cuh"

namespace pf {
namespace {

constexpr int kLaneElems = 16;                         // of a lane, in units of 16 bytes
template <typename T> constexpr int kUnits = kLaneElems / Unit<T>::kN;
constexpr int kNormWarpElems = kLaneElems * 32;
constexpr int kNormMaxWarps = 32, kNormMaxWidth = kNormMaxWarps * kNormWarpElems;

struct NormParams {
    const void* x;              // backward: h
    const void* residual;       // backward: dh
    const void* w;
    const void* dy;             // backward
    void* h;                    // backward: dx
    void* y;
    uint8_t* y8;
    float* scales;
    float* partial;             // backward: a row of sums for dw for each block, or null
    int64_t ldx, ldr, lddy, ldh, ldy, ldy8;
    int64_t tokens;
    int width, lanes, warps, rows;     // (lanes of a warp and) warps to a row, rows to a block
    int block, blocks;          // elements to a scale (0: the row), scales of a row
    float eps, least;           // (least: see far_off)
};

__device__ __forceinline__ float max_or_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
struct Add {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return max_or_nan(a, b); }
};
// What the lanes of a row have, together.  (All threads of the block take part.)  `places`: a number for each warp, another set for each use.
template <typename Op>
__device__ __forceinline__ float in_warp(float v, int lanes, Op op) {
#pragma unroll
    for (int o = 16; o > 0; o /= 2)
        if (o < lanes) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
template <typename Op>
__device__ __forceinline__ float of_warps(const float* places, int warps, int row, Op op) {      // a lane's (a warp at most: the same order in every one)
    const int lane = threadIdx.x & 31;
    const float v = places[row * warps + (lane < warps ? lane : 0)];
    return lane < warps ? v : op(0.f, 0.f);
}
template <typename Op>
__device__ __forceinline__ float over_row(float v, float* places, int lanes, int warps, int warp, int row, Op op) {
    v = in_warp(v, lanes, op);
    if (warps == 1) return v;
    if ((threadIdx.x & 31) == 0) places[warp] = v;
    __syncthreads();
    return in_warp(of_warps(places, warps, row, op), 32, op);
}

// A row's squares may leave fp32 where the row does not: above 2^64, and (where eps is no more than that) below 2^-63.  Rows whose sum of squares (a warp's part of it) is not
// between `least` and kMostSquares are multiplied by a power of two and summed again; eps by its square.  *far: whether a row of those that share barriers, or a warp, needs that.
constexpr float kMostSquares = 0x1p100f, kLeastSquares = 0x1p-60f;
__device__ __forceinline__ float squares_over_row(float v, float* places, int lanes, int warps, int warp, int row, float least, bool* far) {
    if (warps == 1) {
        v = over_row(v, places, lanes, 1, warp, row, Add());
        *far = __any_sync(0xffffffffu, !(v <= kMostSquares && v >= least));
        return v;
    }
    const int lane = threadIdx.x & 31;
    v = in_warp(v, 32, Add());
    if (lane == 0) places[warp] = v;
    __syncthreads();
    const float any = places[min(lane, static_cast<int>(blockDim.x >> 5) - 1)];
    v = of_warps(places, warps, row, Add());
    *far = __any_sync(0xffffffffu, !(any <= kMostSquares && any >= least));
    return in_warp(v, 32, Add());
}
__device__ __forceinline__ float factor_of(float sum, float least) { return !(sum <= kMostSquares) ? 0x1p-76f : sum < least ? 0x1p90f : 1.f; }
// ... the second time, in which only rows with an infinity or a NaN have no finite sum: these are NaN throughout.
__device__ __forceinline__ float finite_or_nan(float sum) { return sum <= 3.4e38f ? sum : __int_as_float(0x7fffffff); }

// Four numbers as e4m3 codes, largest finite one at most.
__device__ __forceinline__ unsigned codes_of(F2 a, F2 b, F2 inverse) {
    unsigned short lo, hi;
    const float2 x = split(mul2(a, inverse)), y = split(mul2(b, inverse));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x.y), "f"(x.x));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(y.y), "f"(y.x));
    return lo | static_cast<unsigned>(hi) << 16;
}

// This thread's units of a row: elements at[u] .. at[u] + n[u] - 1.
template <typename T>
struct NormShare {
    int at[kUnits<T>], n[kUnits<T>];
    __device__ __forceinline__ NormShare(int first, int lanes, int width) {      // (lanes of the row)
#pragma unroll
        for (int u = 0; u < kUnits<T>; ++u) {
            at[u] = Unit<T>::kN * (first + u * lanes);
            n[u] = max(0, min(Unit<T>::kN, width - at[u]));
        }
    }
};

// Rows that a thread keeps on the way into its own places of shared memory: `kStages` rows of `kInputs` matrices, 16 bytes a unit, one thread beside the
// other.  With two stages what a row needs was asked for a row ago; nothing is exchanged between threads, and what a row's later passes need is read from there again
// (in registers it took 80 and spilled: 16384 x 4096 backward 211 us, so 105).
template <typename T, int kPiece, int kInputs, int kStages>
struct NormRing {
    static constexpr int kPlaces = kStages * kInputs * kUnits<T>;
    static constexpr size_t bytes(int threads) { return static_cast<size_t>(kPlaces) * 16 * threads; }
    unsigned char* mine;
    uint32_t apart;
    int ahead, now;      // stages to fill and to read
    __device__ __forceinline__ void init(unsigned char* smem) {
        mine = smem + threadIdx.x * 16;
        apart = blockDim.x * 16;
        ahead = now = 0;
        // (what of a row's last unit does not exist stays zero, and of a row behind the last what was there, which is finite or of no consequence)
        for (int i = 0; i < kPlaces; ++i) *reinterpret_cast<uint4*>(mine + i * apart) = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void ask(int input, const T* row, const NormShare<T>& s) {
#pragma unroll
        for (int u = 0; u < kUnits<T>; ++u) fetch_unit<T, kPiece>(mine + ((ahead * kInputs + input) * kUnits<T> + u) * apart, row + s.at[u], s.n[u]);
    }
    __device__ __forceinline__ void asked() {
        asm volatile("cp.async.commit_group;" ::: "memory");
        ahead = ahead == kStages - 1 ? 0 : ahead + 1;
    }
    __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory"); }
    __device__ __forceinline__ void get(int input, int u, F2 (&x)[Unit<T>::kN / 2]) const {
        Unit<T>::get(*reinterpret_cast<const uint4*>(mine + ((now * kInputs + input) * kUnits<T> + u) * apart), x);
    }
    __device__ __forceinline__ void put(int input, int u, const F2 (&x)[Unit<T>::kN / 2]) {
        *reinterpret_cast<uint4*>(mine + ((now * kInputs + input) * kUnits<T> + u) * apart) = Unit<T>::pack(x);
    }
    __device__ __forceinline__ void done() { now = now == kStages - 1 ? 0 : now + 1; }
};
// Stages of a ring.  Rows of more than 8192 fp32 elements have no room for two.
template <typename T, int kThreads> constexpr int kNormStages = kThreads > 512 && sizeof(T) == 4 ? 1 : 2;
// Blocks that an SM holds, for want of registers.
template <bool kBwd, int kThreads> constexpr int kNormBlocks = kThreads > 512 ? 1 : (kBwd ? 3 : 4) * 256 / kThreads;

// kThreads: of a block at most (256 up to rows of 4096 elements, 512 up to 8192, 1024).  kEightBit: also codes and scales.
template <typename T, int kPiece, bool kEightBit, int kThreads>
__global__ void __launch_bounds__(kThreads, kNormBlocks<false, kThreads>) norm_kernel(const NormParams p) {
    constexpr int kN = Unit<T>::kN, kStages = kNormStages<T, kThreads>;
    extern __shared__ __align__(16) unsigned char norm_smem[];
    __shared__ float places[2][3][kNormMaxWarps];      // sums, largest numbers and sums of rows that are far off, of alternate rows
    const int warp = threadIdx.x >> 5, of_warp = kThreads > 256 ? 32 : p.lanes, lanes = of_warp * p.warps;
    const int row = kThreads > 256 ? 0 : threadIdx.x / static_cast<unsigned>(lanes);
    const NormShare<T> share(threadIdx.x - row * lanes, lanes, p.width);
    NormRing<T, kPiece, 2, kStages> ring;
    ring.init(norm_smem);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int64_t step = static_cast<int64_t>(gridDim.x) * p.rows;
    int64_t t = static_cast<int64_t>(blockIdx.x) * p.rows + row;
    auto ask = [&](int64_t token) {
        if (token < p.tokens) {
            ring.ask(0, static_cast<const T*>(p.x) + token * p.ldx, share);
            if (p.residual) ring.ask(1, static_cast<const T*>(p.residual) + token * p.ldr, share);
        }
        ring.asked();
    };
    if constexpr (kStages > 1) ask(t);
    const T* const w = static_cast<const T*>(p.w);
    const float inv_width = 1.f / static_cast<float>(p.width);
    int turn = 0;
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * p.rows; t0 < p.tokens; t0 += step, t += step, turn ^= 1) {
        const bool live = t < p.tokens;
        ask(t + (kStages - 1) * step);
        ring.wait();
        F2 h[kUnits<T>][kN / 2];
        F2 sum2 = f2(0.f, 0.f);
#pragma unroll
        for (int u = 0; u < kUnits<T>; ++u) {
            ring.get(0, u, h[u]);
            if (p.residual) {
                F2 b[kN / 2];
                ring.get(1, u, b);
#pragma unroll
                for (int i = 0; i < kN / 2; ++i) h[u][i] = add2(h[u][i], b[i]);
            }
#pragma unroll
            for (int i = 0; i < kN / 2; ++i) sum2 = fma2(h[u][i], h[u][i], sum2);
        }
        ring.done();
        if (p.h && live) {
            T* const ph = static_cast<T*>(p.h) + t * p.ldh;
#pragma unroll
            for (int u = 0; u < kUnits<T>; ++u) store_unit<T, kPiece>(ph + share.at[u], share.n[u], h[u]);
        }
        uint4 weight[kUnits<T>];      // (on the way while the row's sum is made: 5001 x 2048 to 8 bits 19.0 us behind it, 15.8 so)
        if (w) {
#pragma unroll
            for (int u = 0; u < kUnits<T>; ++u) weight[u] = load_unit<T, kPiece>(w + share.at[u], share.n[u]);
        }
        const float2 sums = split(sum2);
        bool far;
        float sum = squares_over_row(sums.x + sums.y, places[turn][0], of_warp, p.warps, warp, row, p.least, &far), eps = p.eps;
        if (far) {
            const float f = factor_of(sum, p.least);
            sum2 = f2(0.f, 0.f);
#pragma unroll
            for (int u = 0; u < kUnits<T>; ++u)
#pragma unroll
                for (int i = 0; i < kN / 2; ++i) {
                    h[u][i] = mul2(h[u][i], f2(f, f));
                    sum2 = fma2(h[u][i], h[u][i], sum2);
                }
            const float2 again = split(sum2);
            sum = finite_or_nan(over_row(again.x + again.y, places[turn][2], of_warp, p.warps, warp, row, Add()));
            eps = eps * f * f;
        }
        const float rms = rsqrtf(fmaf(sum, inv_width, eps));
        const F2 scale2 = f2(rms, rms);
#pragma unroll
        for (int u = 0; u < kUnits<T>; ++u) {
#pragma unroll
            for (int i = 0; i < kN / 2; ++i) h[u][i] = mul2(h[u][i], scale2);
            if (w) {
                F2 b[kN / 2];
                Unit<T>::get(weight[u], b);
#pragma unroll
                for (int i = 0; i < kN / 2; ++i) h[u][i] = mul2(h[u][i], b[i]);
            }
        }
        if (p.y && live) {
            T* const py = static_cast<T*>(p.y) + t * p.ldy;
#pragma unroll
            for (int u = 0; u < kUnits<T>; ++u) store_unit<T, kPiece>(py + share.at[u], share.n[u], h[u]);
        }
        if constexpr (kEightBit) {
            float most[kUnits<T>];
#pragma unroll
            for (int u = 0; u < kUnits<T>; ++u) {
                most[u] = 0.f;
#pragma unroll
                for (int i = 0; i < kN / 2; ++i) {
                    const float2 v = split(h[u][i]);
                    if constexpr (kPiece == 16) {
                        most[u] = max_or_nan(most[u], max_or_nan(fabsf(v.x), fabsf(v.y)));
                    } else {      // (what is behind the row's end is 0, or NaN where the row is)
                        most[u] = 2 * i < share.n[u] ? max_or_nan(most[u], fabsf(v.x)) : most[u];
                        most[u] = 2 * i + 1 < share.n[u] ? max_or_nan(most[u], fabsf(v.y)) : most[u];
                    }
                }
                if (kPiece == 16 && share.n[u] == 0) most[u] = 0.f;
            }
            if (p.block == 0) {
                float all = most[0];
#pragma unroll
                for (int u = 1; u < kUnits<T>; ++u) all = max_or_nan(all, most[u]);
                all = over_row(all, places[turn][1], of_warp, p.warps, warp, row, Max());
#pragma unroll
                for (int u = 0; u < kUnits<T>; ++u) most[u] = all;
            } else {
#pragma unroll
                for (int o = 64 / kN; o > 0; o /= 2) {      // lanes of a block: block / kN
                    if (2 * o * kN > p.block) continue;
#pragma unroll
                    for (int u = 0; u < kUnits<T>; ++u) most[u] = max_or_nan(most[u], __shfl_xor_sync(0xffffffffu, most[u], o));
                }
            }
#pragma unroll
            for (int u = 0; u < kUnits<T>; ++u) {
                if (!live || share.n[u] == 0) continue;
                // (a scale below the normal numbers has no inverse: such a block, unless it is all zeros, has the smallest normal number)
                const bool small = most[u] < 448.f * 0x1p-126f;
                const float scale = !small ? most[u] * (1.f / 448.f) : most[u] > 0.f ? 0x1p-126f : 0.f;
                const float inverse = !small ? __fdividef(448.f * 0x1p-8f, most[u] * 0x1p-8f) : 0x1p126f;      // (its divisors end at 2^126)
                unsigned codes[kN / 4];
#pragma unroll
                for (int i = 0; i < kN / 4; ++i) codes[i] = codes_of(h[u][2 * i], h[u][2 * i + 1], f2(inverse, inverse));
                uint8_t* const out = p.y8 + t * p.ldy8 + share.at[u];
                if (share.n[u] == kN && (reinterpret_cast<uintptr_t>(out) & (kN - 1)) == 0) {
                    if constexpr (kN == 8) *reinterpret_cast<uint2*>(out) = make_uint2(codes[0], codes[kN / 4 - 1]);
                    else *reinterpret_cast<unsigned*>(out) = codes[0];
                } else {
#pragma unroll
                    for (int i = 0; i < kN; ++i)
                        if (i < share.n[u]) out[i] = static_cast<uint8_t>(codes[i / 4] >> (8 * (i & 3)));
                }
                const int block = p.block == 0 ? 0 : p.block == 32 ? share.at[u] >> 5 : share.at[u] >> 7;
                if (p.block == 0 ? share.at[u] == 0 : (share.at[u] & (p.block - 1)) == 0) p.scales[t * p.blocks + block] = scale;
            }
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

template <typename T, int kPiece, int kThreads>
__global__ void __launch_bounds__(kThreads, kNormBlocks<true, kThreads>) norm_bwd_kernel(const NormParams p) {
    constexpr int kN = Unit<T>::kN, kStages = kNormStages<T, kThreads>;
    extern __shared__ __align__(16) unsigned char norm_smem[];      // the ring, then sums for dw of the rows of a block
    __shared__ float places[2][4][kNormMaxWarps];      // both sums, and those of rows that are far off, of alternate rows
    const int warp = threadIdx.x >> 5, of_warp = kThreads > 256 ? 32 : p.lanes, lanes = of_warp * p.warps;
    const int row = kThreads > 256 ? 0 : threadIdx.x / static_cast<unsigned>(lanes);
    const NormShare<T> share(threadIdx.x - row * lanes, lanes, p.width);
    NormRing<T, kPiece, 3, kStages> ring;
    ring.init(norm_smem);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int64_t step = static_cast<int64_t>(gridDim.x) * p.rows;
    int64_t t = static_cast<int64_t>(blockIdx.x) * p.rows + row;
    auto ask = [&](int64_t token) {
        if (token < p.tokens) {
            ring.ask(0, static_cast<const T*>(p.x) + token * p.ldx, share);
            ring.ask(1, static_cast<const T*>(p.dy) + token * p.lddy, share);
            if (p.residual) ring.ask(2, static_cast<const T*>(p.residual) + token * p.ldr, share);
        }
        ring.asked();
    };
    if constexpr (kStages > 1) ask(t);
    const T* const w = static_cast<const T*>(p.w);
    F2 dw[kUnits<T>][kN / 2];
#pragma unroll
    for (int u = 0; u < kUnits<T>; ++u)
#pragma unroll
        for (int i = 0; i < kN / 2; ++i) dw[u][i] = f2(0.f, 0.f);
    const float inv_width = 1.f / static_cast<float>(p.width);
    int turn = 0;
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * p.rows; t0 < p.tokens; t0 += step, t += step, turn ^= 1) {
        const bool live = t < p.tokens;
        ask(t + (kStages - 1) * step);
        ring.wait();
        F2 sum2 = f2(0.f, 0.f), dot2 = f2(0.f, 0.f);      // of h^2 and of h s
        auto add_up = [&](auto again, float f) {
#pragma unroll
            for (int u = 0; u < kUnits<T>; ++u) {
                F2 h[kN / 2], s[kN / 2];
                ring.get(0, u, h);
                ring.get(1, u, s);
                if (w) {
                    F2 b[kN / 2];
                    Unit<T>::get(load_unit<T, kPiece>(w + share.at[u], share.n[u]), b);
#pragma unroll
                    for (int i = 0; i < kN / 2; ++i) s[i] = mul2(s[i], b[i]);
                }
                if constexpr (decltype(again)::value) {      // (a power of two: exact, but for what is nothing beside the row's largest)
#pragma unroll
                    for (int i = 0; i < kN / 2; ++i) h[i] = mul2(h[i], f2(f, f));
                    ring.put(0, u, h);
                }
#pragma unroll
                for (int i = 0; i < kN / 2; ++i) {
                    sum2 = fma2(h[i], h[i], sum2);
                    dot2 = fma2(h[i], s[i], dot2);
                }
            }
        };
        add_up(std::false_type(), 1.f);
        const float2 sums = split(sum2), dots = split(dot2);
        bool far;
        float sum = squares_over_row(sums.x + sums.y, places[turn][0], of_warp, p.warps, warp, row, p.least, &far), f = 1.f;
        float rms = rsqrtf(fmaf(sum, inv_width, p.eps));
        float dot = over_row(dots.x + dots.y, places[turn][1], of_warp, p.warps, warp, row, Add());
        if (far) {      // (h is f h from here on)
            f = factor_of(sum, p.least);
            sum2 = dot2 = f2(0.f, 0.f);
            add_up(std::true_type(), f);
            const float2 sums2 = split(sum2), dots2 = split(dot2);
            sum = finite_or_nan(over_row(sums2.x + sums2.y, places[turn][2], of_warp, p.warps, warp, row, Add()));
            dot = over_row(dots2.x + dots2.y, places[turn][3], of_warp, p.warps, warp, row, Add());
            rms = rsqrtf(fmaf(sum, inv_width, p.eps * f * f));
        }
        const float mean = dot * rms * inv_width;      // of s n, as n = h r
        if (live) {
            const F2 rr = f2(rms, rms), mm = f2(-mean, -mean), rx = f2(rms * f, rms * f);
            T* const out = static_cast<T*>(p.h) + t * p.ldh;
#pragma unroll
            for (int u = 0; u < kUnits<T>; ++u) {
                F2 h[kN / 2], s[kN / 2], b[kN / 2];
                ring.get(0, u, h);
                ring.get(1, u, s);
                if (w) Unit<T>::get(load_unit<T, kPiece>(w + share.at[u], share.n[u]), b);
#pragma unroll
                for (int i = 0; i < kN / 2; ++i) {
                    h[i] = mul2(h[i], rr);
                    dw[u][i] = fma2(s[i], h[i], dw[u][i]);
                    if (w) s[i] = mul2(s[i], b[i]);
                    h[i] = mul2(rx, fma2(h[i], mm, s[i]));
                }
                if (p.residual) {
                    ring.get(2, u, b);
#pragma unroll
                    for (int i = 0; i < kN / 2; ++i) h[i] = add2(h[i], b[i]);
                }
                store_unit<T, kPiece>(out + share.at[u], share.n[u], h);
            }
        }
        ring.done();
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (!p.partial) return;
    float* const sums = reinterpret_cast<float*>(norm_smem);
    float* const mine = p.rows > 1 ? sums + row * lanes * kLaneElems : p.partial + static_cast<int64_t>(blockIdx.x) * p.width;
    __syncthreads();      // (all have read their places)
    const bool whole = p.rows > 1 || p.width % 4 == 0;
#pragma unroll
    for (int u = 0; u < kUnits<T>; ++u)
#pragma unroll
        for (int i = 0; i < kN; i += 4) {
            const float2 a = split(dw[u][i / 2]), b = split(dw[u][i / 2 + 1]);
            float* const to = mine + share.at[u] + i;
            if (i + 4 <= share.n[u] && whole) {
                *reinterpret_cast<float4*>(to) = make_float4(a.x, a.y, b.x, b.y);
            } else {
                if (i < share.n[u]) to[0] = a.x;
                if (i + 1 < share.n[u]) to[1] = a.y;
                if (i + 2 < share.n[u]) to[2] = b.x;
                if (i + 3 < share.n[u]) to[3] = b.y;
            }
        }
    if (p.rows == 1) return;
    __syncthreads();
    for (int i = threadIdx.x; i < p.width; i += blockDim.x) {
        float sum = 0.f;
        for (int k = 0; k < p.rows; ++k) sum += sums[k * lanes * kLaneElems + i];
        p.partial[static_cast<int64_t>(blockIdx.x) * p.width + i] = sum;
    }
}

// dw from the blocks' sums: a block has 8 columns (a sector of memory for each row), its threads every 128th row each, added up in order.
struct NormSums {
    const float* partial;
    void* dw;
    int blocks, width;
    int accumulate;
};
constexpr int kSumCols = 8, kSumRows = 128;
template <typename T>
__global__ void __launch_bounds__(kSumCols * kSumRows) norm_weight_kernel(const NormSums p) {
    __shared__ float red[kSumRows][kSumCols + 1];
    const int c = threadIdx.x % kSumCols, k = threadIdx.x / kSumCols, col = blockIdx.x * kSumCols + c;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    float sum = 0.f;
    if (col < p.width) {
#pragma unroll 4
        for (int b = k; b < p.blocks; b += kSumRows) sum += p.partial[static_cast<int64_t>(b) * p.width + col];
    }
    red[k][c] = sum;
    __syncthreads();
    // a warp's lanes every fourth row each
    if (threadIdx.x >= 4 * kSumCols) return;
    sum = 0.f;
#pragma unroll 8
    for (int i = k; i < kSumRows; i += 4) sum += red[i][c];
    sum += __shfl_xor_sync(0xffffffffu, sum, 8);
    sum += __shfl_xor_sync(0xffffffffu, sum, 16);
    if (k != 0 || col >= p.width) return;
    T* const out = static_cast<T*>(p.dw) + col;
    if (p.accumulate) sum += static_cast<float>(*out);
    *out = static_cast<T>(sum);
}

struct NormPlan {
    int lanes, warps, rows, threads;
    int64_t groups;      // of rows
};
// Rows of up to 256 elements share a warp (200000 x 64 bf16 forward 64 us with a warp each); the lanes of a block of 8-bit codes are neighbours in one unit.
NormPlan norm_plan(int64_t tokens, int64_t width, int block, int dtype) {
    NormPlan pl;
    pl.warps = static_cast<int>(ceil_div(width, kNormWarpElems));
    pl.lanes = 4;
    while (pl.lanes < 32 && (pl.lanes * kLaneElems < width || pl.lanes * 16 / static_cast<int>(dtype_size(dtype)) < block)) pl.lanes *= 2;
    pl.rows = std::max(1, 256 / (32 * pl.warps)) * (32 / pl.lanes);
    pl.threads = pl.warps * pl.rows * pl.lanes;
    pl.groups = ceil_div(tokens, pl.rows);
    return pl;
}
// Blocks of a backward at most: as many of its threads as an SM holds registers for.  (The workspace has a row of sums for each.)
int64_t norm_bwd_blocks(const NormPlan& pl) {
    return std::min<int64_t>(pl.groups, static_cast<int64_t>(num_sms()) * std::max(1, kNormBlocks<true, 256> * 256 / pl.threads));
}

// A kernel and the bytes of its ring.
struct NormKernel {
    void (*run)(NormParams);
    size_t ring;
    int blocks, threads;      // that an SM holds of its largest blocks, and their threads
    std::atomic<uint64_t>* done;
};
constexpr int64_t kNormSmem = 228 * 1024;      // of an SM
template <typename T, int kPiece, int kThreads>
NormKernel norm_with(bool bwd, bool eight, int threads) {
    static std::atomic<uint64_t> done[3];
    if (bwd) return {norm_bwd_kernel<T, kPiece, kThreads>, NormRing<T, kPiece, 3, kNormStages<T, kThreads>>::bytes(threads), kNormBlocks<true, kThreads>, kThreads, done};
    return {eight ? norm_kernel<T, kPiece, true, kThreads> : norm_kernel<T, kPiece, false, kThreads>, NormRing<T, kPiece, 2, kNormStages<T, kThreads>>::bytes(threads),
            kNormBlocks<false, kThreads>, kThreads, done + (eight ? 1 : 2)};
}
template <typename T, int kPiece>
NormKernel norm_of(bool bwd, bool eight, int threads) {
    return threads <= 256 ? norm_with<T, kPiece, 256>(bwd, eight, threads) : threads <= 512 ? norm_with<T, kPiece, 512>(bwd, eight, threads)
           : norm_with<T, kPiece, 1024>(bwd, eight, threads);
}
// `piece` as in pf_rows.cuh
NormKernel pick_norm(int dtype, int piece, bool bwd, bool eight, int threads) {
    using B = __nv_bfloat16;
    if (dtype == PF_BF16)
        return piece == 16 ? norm_of<B, 16>(bwd, eight, threads) : piece == 8 ? norm_of<B, 8>(bwd, eight, threads) : piece == 4 ? norm_of<B, 4>(bwd, eight, threads)
               : norm_of<B, 2>(bwd, eight, threads);
    return piece == 16 ? norm_of<float, 16>(bwd, eight, threads) : piece == 8 ? norm_of<float, 8>(bwd, eight, threads) : norm_of<float, 4>(bwd, eight, threads);
}
// `more`: shared memory that is needed beside the ring, behind it in time.  *blocks: how many there are, `most` at most
cudaError_t norm_launch(const NormKernel& k, const NormPlan& pl, size_t more, const NormParams& p, cudaStream_t stream, int64_t most, int* blocks) {
    const size_t smem = std::max(k.ring, more);
    const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(k.run), 200 * 1024, *k.done);      // (1024 threads' bf16 ring: 192 KB)
    if (e != cudaSuccess) return e;
    const int64_t room = std::max<int64_t>(1, std::min<int64_t>(k.blocks * k.threads / pl.threads, kNormSmem / static_cast<int64_t>(smem + 2048)));
    *blocks = static_cast<int>(std::min<int64_t>(most, num_sms() * room));
    return launch_beside(k.run, dim3(static_cast<unsigned>(*blocks)), pl.threads, smem, 1, stream, p);
}

bool rows_ok(const void* p, int64_t ld, int64_t width, int dtype) { return p && ld >= width && elem_aligned(p, dtype); }
// What the row's address and pitch leave of the bytes that accesses may have.
uint64_t alignment(const void* p, int64_t ld, int dtype) {
    return p ? reinterpret_cast<uintptr_t>(p) | static_cast<uint64_t>(ld) * dtype_size(dtype) : 0;
}
int piece_of(uint64_t all) {
    all |= 16;
    return static_cast<int>(all & (~all + 1));
}
int validate_norm(int64_t tokens, int64_t width, double eps, int dtype, const void* w) {
    if (!valid_dtype(dtype) || tokens < 0 || width < 1 || !(eps >= 0.0) || !(eps <= 3.0e38) || !elem_aligned(w, dtype)) return PF_ERR_INVALID_ARG;
    if (width > kNormMaxWidth || tokens > (1LL << 40)) return PF_ERR_UNSUPPORTED;
    return PF_OK;
}

}  // namespace
}  // namespace pf

using namespace pf;

extern "C" {

int pf_add_rms_norm_fwd(const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* w, void* h, int64_t ldh, void* y, int64_t ldy,
                        void* y8, int64_t ldy8, float* scales, int block, int64_t tokens, int64_t width, double eps, int dtype, void* cuda_stream) {
    const int st = validate_norm(tokens, width, eps, dtype, w);
    if (st != PF_OK || tokens == 0) return st;
    if ((!h && !y && !y8) || (y8 == nullptr) != (scales == nullptr)) return PF_ERR_INVALID_ARG;
    if (y8 && ((block != 0 && block != 32 && block != 128) || ldy8 < width || reinterpret_cast<uintptr_t>(scales) % 4 != 0)) return PF_ERR_INVALID_ARG;
    if (!rows_ok(x, ldx, width, dtype) || (residual && !rows_ok(residual, ldr, width, dtype)) || (h && !rows_ok(h, ldh, width, dtype)) ||
        (y && !rows_ok(y, ldy, width, dtype)))
        return PF_ERR_INVALID_ARG;
    const NormPlan pl = norm_plan(tokens, width, y8 ? block : 0, dtype);
    int blocks;
    NormParams p = {};
    p.x = x; p.ldx = ldx; p.residual = residual; p.ldr = ldr; p.w = w;
    p.h = h; p.ldh = ldh; p.y = y; p.ldy = ldy;
    p.y8 = static_cast<uint8_t*>(y8); p.ldy8 = ldy8; p.scales = scales; p.block = block;
    p.blocks = block ? static_cast<int>(ceil_div(width, block)) : 1;
    p.tokens = tokens; p.width = static_cast<int>(width); p.lanes = pl.lanes; p.warps = pl.warps; p.rows = pl.rows;
    p.eps = static_cast<float>(eps);
    p.least = p.eps < 1e-18f ? kLeastSquares : 0.f;
    const int piece = piece_of(alignment(x, ldx, dtype) | alignment(residual, ldr, dtype) | alignment(h, ldh, dtype) | alignment(y, ldy, dtype) |
                               alignment(w, 0, dtype) | static_cast<uint64_t>(width) * dtype_size(dtype));
    PF_CUDA(norm_launch(pick_norm(dtype, piece, false, y8 != nullptr, pl.threads), pl, 0, p, static_cast<cudaStream_t>(cuda_stream), pl.groups, &blocks));
    return PF_OK;
}

size_t pf_add_rms_norm_bwd_workspace(int64_t tokens, int64_t width) {
    if (tokens <= 0 || width < 1 || width > kNormMaxWidth || tokens > (1LL << 40)) return 0;
    return align_up(sizeof(float) * static_cast<size_t>(width) * norm_bwd_blocks(norm_plan(tokens, width, 0, PF_F32)), 256);
}

int pf_add_rms_norm_bwd(const void* h, int64_t ldh, const void* w, const void* dy, int64_t lddy, const void* dh, int64_t lddh, void* dx, int64_t lddx,
                        void* dw, int64_t tokens, int64_t width, double eps, int dtype, unsigned flags, void* workspace, size_t workspace_bytes,
                        void* cuda_stream) {
    const int st = validate_norm(tokens, width, eps, dtype, w);
    if (st != PF_OK) return st;
    if (flags & ~static_cast<unsigned>(PF_GRAD_ACCUMULATE | PF_GRAD_F32)) return PF_ERR_INVALID_ARG;
    const int wtype = flags & PF_GRAD_F32 ? PF_F32 : dtype;
    if (!elem_aligned(dw, wtype)) return PF_ERR_INVALID_ARG;
    if (tokens > 0 && (!rows_ok(h, ldh, width, dtype) || !rows_ok(dy, lddy, width, dtype) || !rows_ok(dx, lddx, width, dtype) ||
                       (dh && !rows_ok(dh, lddh, width, dtype))))
        return PF_ERR_INVALID_ARG;
    const int wst = check_ws(workspace, workspace_bytes, dw ? pf_add_rms_norm_bwd_workspace(tokens, width) : 0);
    if (wst != PF_OK) return wst;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (tokens == 0) {
        if (dw && !(flags & PF_GRAD_ACCUMULATE)) PF_CUDA(cudaMemsetAsync(dw, 0, width * dtype_size(wtype), stream));
        return PF_OK;
    }
    const NormPlan pl = norm_plan(tokens, width, 0, dtype);
    int blocks;
    NormParams p = {};
    p.x = h; p.ldx = ldh; p.residual = dh; p.ldr = lddh; p.w = w; p.dy = dy; p.lddy = lddy; p.h = dx; p.ldh = lddx;
    p.partial = dw ? static_cast<float*>(workspace) : nullptr;
    p.tokens = tokens; p.width = static_cast<int>(width); p.lanes = pl.lanes; p.warps = pl.warps; p.rows = pl.rows;
    p.eps = static_cast<float>(eps);
    p.least = p.eps < 1e-18f ? kLeastSquares : 0.f;
    const int piece = piece_of(alignment(h, ldh, dtype) | alignment(dh, lddh, dtype) | alignment(dy, lddy, dtype) | alignment(dx, lddx, dtype) |
                               alignment(w, 0, dtype) | static_cast<uint64_t>(width) * dtype_size(dtype));
    const size_t sums = dw && pl.rows > 1 ? sizeof(float) * pl.threads * kLaneElems : 0;      // (16 KB at most)
    PF_CUDA(norm_launch(pick_norm(dtype, piece, true, false, pl.threads), pl, sums, p, stream, norm_bwd_blocks(pl), &blocks));
    if (!dw) return PF_OK;
    const NormSums s = {p.partial, dw, blocks, p.width, flags & PF_GRAD_ACCUMULATE ? 1 : 0};
    const auto add = wtype == PF_BF16 ? norm_weight_kernel<__nv_bfloat16> : norm_weight_kernel<float>;
    PF_CUDA(launch_beside(add, dim3(static_cast<unsigned>(ceil_div(width, kSumCols))), kSumCols * kSumRows, 0, 1, stream, s));
    return PF_OK;
}

}  // extern "C"
