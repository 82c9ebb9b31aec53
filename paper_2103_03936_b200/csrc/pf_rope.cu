// Norm and position rotation of the queries and keys of an attention layer, for each head, forward and backward.
//
// For a row x of `dim` elements (one head of one token at position t), n = x r with r = 1 / sqrt(mean(x^2) + eps), z = n w; the
// first `rot` elements of z are pairs (a, b) turned by the angle t f_i of their pair:
//   (a, b) -> (a cos - b sin, b cos + a sin)
// Backward, for the upstream gradient g: e = g turned back, dw = sum e n, s = e w, dx = r (s - n mean(s n)); r is recomputed.
//
// Bound by memory: a row is read and written once (backward: two read, one written).  A row's pair elements lie rot / 2 apart
// (PF_ROPE_HALVES) or side by side (PF_ROPE_PAIRS); a lane takes one 16-byte piece of each half, so that both elements of a pair are
// in one lane under either style, and a row is 2 to 32 lanes.  A warp takes several heads of a token, so that the angles (product
// and reduction to a turn in pairs of fp64, sine and cosine in fp32) are computed once for all of them and stay in registers.
#include <algorithm>
#include <cmath>

#include "pf_internal.h"

namespace pf {
namespace {

constexpr int kRopeThreads = 256, kRopeWarps = kRopeThreads / 32;
constexpr int kMaxDim = 1024;
constexpr int kMaxPairs = 256;      // of the rows that the vector kernels take
constexpr int kAnyThreads = 128, kAnyWarps = kAnyThreads / 32;

// Queries or keys.
struct RopeSide {
    const void* x;
    const void* w;
    const void* g;          // backward: upstream gradient
    void* out;              // forward: the rotated rows; backward: dx
    float* partial;         // backward: one row of sums for dw per block, or null
    int64_t ldx, sx, ldg, sg, ldo, so;
    int heads, heads_per_unit, units_per_token, blocks;
};
struct RopeParams {
    RopeSide side[2];
    const int64_t* positions;
    const float* inv_freq;
    int64_t tokens;
    int dim, rot;
    float eps;
};

// Cosine and sine of the angle position * f, position up to 2^53.  Product and turns are pairs of fp64 numbers (the second what rounding the first
// left out), so that what remains of them after the whole turns is good to fp32 at any position; it is rounded only then.
__device__ __forceinline__ float2 turn_of(int64_t position, float f) {
    constexpr double kTurn = 0.15915494309189535, kTurnRest = -9.839338337591243e-18;      // 1 / (2 pi)
    const double t = static_cast<double>(position), a = t * static_cast<double>(f), a_rest = fma(t, static_cast<double>(f), -a);
    const double turns = a * kTurn, rest = fma(a, kTurn, -turns) + fma(a, kTurnRest, a_rest * kTurn);
    float s, c;
    sincospif(2.f * static_cast<float>((turns - rint(turns)) + rest), &s, &c);
    return make_float2(c, s);
}

template <typename T> struct Piece;      // 16 bytes
template <> struct Piece<float> {
    static constexpr int kN = 4;
    float4 raw;
    __device__ __forceinline__ void load(const float* p) { raw = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void get(float* x) const { x[0] = raw.x; x[1] = raw.y; x[2] = raw.z; x[3] = raw.w; }
    static __device__ __forceinline__ void store(float* p, const float* x) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }
};
template <> struct Piece<__nv_bfloat16> {
    static constexpr int kN = 8;
    uint4 raw;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { raw = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void get(float* x) const {
        const unsigned w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* x) {
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 t = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const unsigned*>(&t);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
__device__ __forceinline__ float get1(const float* p) { return *p; }
__device__ __forceinline__ float get1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put1(float* p, float x) { *p = x; }
__device__ __forceinline__ void put1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// Turns a lane's pairs in place: a[] and b[] are its two pieces, cs its pairs in order (sine negated: turns back).
template <int kN, bool kPairs>
__device__ __forceinline__ void turn(float (&a)[kN], float (&b)[kN], const float2 (&cs)[kN], float sign) {
    if constexpr (kPairs) {
#pragma unroll
        for (int i = 0; i < kN / 2; ++i) {
            const float c0 = cs[i].x, s0 = sign * cs[i].y, c1 = cs[kN / 2 + i].x, s1 = sign * cs[kN / 2 + i].y;
            const float a0 = a[2 * i], a1 = a[2 * i + 1], b0 = b[2 * i], b1 = b[2 * i + 1];
            a[2 * i] = a0 * c0 - a1 * s0;
            a[2 * i + 1] = a1 * c0 + a0 * s0;
            b[2 * i] = b0 * c1 - b1 * s1;
            b[2 * i + 1] = b1 * c1 + b0 * s1;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const float c = cs[i].x, s = sign * cs[i].y, x = a[i], y = b[i];
            a[i] = x * c - y * s;
            b[i] = y * c + x * s;
        }
    }
}

template <int kLanes>
__device__ __forceinline__ float sum_lanes(float x) {
#pragma unroll
    for (int o = kLanes / 2; o > 0; o /= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// The rows that a warp takes one after the other: kRows heads at a time of the units of (token, some of its heads) that are its share.
struct RopeWalk {
    int64_t token;
    int part, h, end;      // the unit's place among its token's, the next head, the first behind the unit
    __device__ __forceinline__ bool valid(const RopeParams& p) const { return token < p.tokens; }
    __device__ __forceinline__ void enter(const RopeSide& s) {
        h = part * s.heads_per_unit;
        end = min(h + s.heads_per_unit, s.heads);
    }
    __device__ __forceinline__ void start(const RopeSide& s, int64_t unit) {
        token = unit / s.units_per_token;
        part = static_cast<int>(unit - token * s.units_per_token);
        enter(s);
    }
    // The next unit is step_tokens tokens and step_parts parts on.
    __device__ __forceinline__ void next_unit(const RopeSide& s, int64_t step_tokens, int step_parts) {
        token += step_tokens;
        part += step_parts;
        if (part >= s.units_per_token) { part -= s.units_per_token; ++token; }
        enter(s);
    }
};

__device__ __forceinline__ void fetch16(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

// kLanes lanes to a row (the power of two from the row's pieces / 2 on), 32 / kLanes rows of a warp at a time.  Each lane keeps the
// pieces of its next kStages - 1 rows on the way into its own places of shared memory, across units: what a warp waits for was asked for rows
// ago, and nothing is exchanged between lanes but the sums.
template <bool kBwd> constexpr int kRopeStages = kBwd ? 4 : 6;
template <bool kBwd> constexpr int kRopePieces = kBwd ? 4 : 2;      // 16-byte pieces of a lane for a row: two of x, two of the gradient
template <bool kBwd> constexpr int kRopeRing = kRopeWarps * kRopeStages<kBwd> * kRopePieces<kBwd> * 32 * 16;

template <typename T, int kLanes, bool kPairs, bool kBwd>
__global__ void __launch_bounds__(kRopeThreads, kBwd ? 2 : 3) rope_kernel(const RopeParams p) {
    constexpr int kN = Piece<T>::kN, kRows = 32 / kLanes, kStages = kRopeStages<kBwd>, kPieces = kRopePieces<kBwd>;
    extern __shared__ __align__(16) unsigned char rope_smem[];      // the lanes' pieces, then each warp's angles
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool key = static_cast<int>(blockIdx.x) >= p.side[0].blocks;
    const RopeSide& s = p.side[key ? 1 : 0];
    const int block = static_cast<int>(blockIdx.x) - (key ? p.side[0].blocks : 0);
    // this lane's pieces: the first ones of a row cover the pairs, the others what is not turned
    const int l = lane % kLanes, row = lane / kLanes, half = p.rot / 2;
    const bool there = 2 * kN * l < p.dim, turned = kN * l < half;
    const int ia = turned ? kN * l : p.rot + kN * l - half, ib = ia + (turned ? half : (p.dim - p.rot) / 2);
    unsigned char* const ring = rope_smem + (warp * kStages * kPieces * 32 + lane) * 16;
    const uint32_t ring_at = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
    float2* const angles = reinterpret_cast<float2*>(rope_smem + kRopeRing<kBwd>) + warp * half;
    const int64_t step = static_cast<int64_t>(s.blocks) * kRopeWarps, step_tokens = step / s.units_per_token;
    const int step_parts = static_cast<int>(step - step_tokens * s.units_per_token);
    RopeWalk ahead, at;      // rows to ask for, rows to compute
    ahead.start(s, static_cast<int64_t>(block) * kRopeWarps + warp);
    at = ahead;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const T* const xs = static_cast<const T*>(s.x);
    const T* const gs = static_cast<const T*>(s.g);
    auto ask = [&](int stage) {
        if (ahead.valid(p)) {
            const int64_t head = ahead.h + row;
            if (there && head < ahead.end) {
                const uint32_t to = ring_at + stage * (kPieces * 32 * 16);
                const T* const x = xs + ahead.token * s.ldx + head * s.sx;
                fetch16(to, x + ia);
                fetch16(to + 512, x + ib);
                if constexpr (kBwd) {
                    const T* const g = gs + ahead.token * s.ldg + head * s.sg;
                    fetch16(to + 1024, g + ia);
                    fetch16(to + 1536, g + ib);
                }
            }
            ahead.h += kRows;
            if (ahead.h >= ahead.end) ahead.next_unit(s, step_tokens, step_parts);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) ask(i);
    auto position_of = [&](const RopeWalk& w) { return !w.valid(p) ? 0 : p.positions ? p.positions[w.token] : w.token; };
    int64_t position = position_of(at);
    float wa[kN], wb[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) wa[i] = wb[i] = 1.f;
    if (s.w && there) {
        Piece<T> t;
        t.load(static_cast<const T*>(s.w) + ia);
        t.get(wa);
        t.load(static_cast<const T*>(s.w) + ib);
        t.get(wb);
    }
    float dwa[kN], dwb[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) dwa[i] = dwb[i] = 0.f;
    const float inv_dim = 1.f / static_cast<float>(p.dim);
    int stage = 0;
    while (at.valid(p)) {
        __syncwarp();
        for (int i = lane; i < half; i += 32) angles[i] = turn_of(position, p.inv_freq[i]);
        __syncwarp();
        float2 cs[kN];
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int pair = kPairs ? (i < kN / 2 ? ia / 2 + i : ib / 2 + i - kN / 2) : ia + i;
            cs[i] = turned ? angles[pair] : make_float2(1.f, 0.f);
        }
        RopeWalk next = at;
        next.next_unit(s, step_tokens, step_parts);
        position = position_of(next);
        T* const out = static_cast<T*>(s.out) + at.token * s.ldo;
        for (; at.h < at.end; at.h += kRows) {
            __syncwarp();
            ask(stage == 0 ? kStages - 1 : stage - 1);      // the place that the row before has left
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
            const unsigned char* const in = ring + stage * (kPieces * 32 * 16);
            stage = stage == kStages - 1 ? 0 : stage + 1;
            const int64_t head = at.h + row;
            const bool live = head < at.end, on = there && live;
            float a[kN], b[kN];
            Piece<T> xa, xb;
            xa.raw = {};
            xb.raw = {};
            if (on) {
                xa.load(reinterpret_cast<const T*>(in));
                xb.load(reinterpret_cast<const T*>(in + 512));
            }
            xa.get(a);
            xb.get(b);
            float sq = 0.f;
#pragma unroll
            for (int i = 0; i < kN; ++i) sq = fmaf(a[i], a[i], fmaf(b[i], b[i], sq));
            sq = sum_lanes<kLanes>(sq);
            // (a row behind the last head adds nothing to dw, whatever eps is)
            const float r = live ? rsqrtf(fmaf(sq, inv_dim, p.eps)) : 0.f;
            if constexpr (!kBwd) {
#pragma unroll
                for (int i = 0; i < kN; ++i) { a[i] *= r * wa[i]; b[i] *= r * wb[i]; }
                turn<kN, kPairs>(a, b, cs, 1.f);
            } else {
                Piece<T> ga, gb;
                ga.raw = {};
                gb.raw = {};
                if (on) {
                    ga.load(reinterpret_cast<const T*>(in + 1024));
                    gb.load(reinterpret_cast<const T*>(in + 1536));
                }
                float ea[kN], eb[kN], dot = 0.f;
                ga.get(ea);
                gb.get(eb);
                turn<kN, kPairs>(ea, eb, cs, -1.f);
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    a[i] *= r;
                    b[i] *= r;
                    dwa[i] = fmaf(ea[i], a[i], dwa[i]);
                    dwb[i] = fmaf(eb[i], b[i], dwb[i]);
                    ea[i] *= wa[i];
                    eb[i] *= wb[i];
                    dot = fmaf(ea[i], a[i], fmaf(eb[i], b[i], dot));
                }
                dot = sum_lanes<kLanes>(dot) * inv_dim;
#pragma unroll
                for (int i = 0; i < kN; ++i) { a[i] = r * (ea[i] - a[i] * dot); b[i] = r * (eb[i] - b[i] * dot); }
            }
            if (on) {
                T* const o = out + head * s.so;
                Piece<T>::store(o + ia, a);
                Piece<T>::store(o + ib, b);
            }
        }
        at = next;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if constexpr (kBwd) {
        if (!s.partial) return;
        // rows of a warp, then warps in order
        float* const red = reinterpret_cast<float*>(rope_smem);      // (16 KB of the pieces' places at most)
        static_assert(kRopeWarps * 2 * kN * kLanes * 4 <= kRopeRing<kBwd>, "");
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kN; ++i) {
#pragma unroll
            for (int o = kLanes; o < 32; o *= 2) {
                dwa[i] += __shfl_xor_sync(0xffffffffu, dwa[i], o);
                dwb[i] += __shfl_xor_sync(0xffffffffu, dwb[i], o);
            }
            if (row == 0) {
                red[(warp * 2 * kN + i) * kLanes + l] = dwa[i];
                red[(warp * 2 * kN + kN + i) * kLanes + l] = dwb[i];
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * kN * kLanes; c += kRopeThreads) {
            const int cl = c % kLanes, i = c / kLanes;
            if (2 * kN * cl >= p.dim) continue;
            float sum = 0.f;
            for (int w = 0; w < kRopeWarps; ++w) sum += red[(w * 2 * kN + i) * kLanes + cl];
            const bool t = kN * cl < half;
            const int a0 = t ? kN * cl : p.rot + kN * cl - half, b0 = a0 + (t ? half : (p.dim - p.rot) / 2);
            s.partial[static_cast<int64_t>(block) * p.dim + (i < kN ? a0 + i : b0 + i - kN)] = sum;
        }
    }
}

// Rows of any width, pitch and alignment: a warp to a row, element after element, the other element of a pair read again.
template <typename T, bool kPairs, bool kBwd>
__global__ void __launch_bounds__(kAnyThreads) rope_any_kernel(const RopeParams p) {
    extern __shared__ float any_smem[];      // per warp: angles of a token, then (backward) sums for dw
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool key = static_cast<int>(blockIdx.x) >= p.side[0].blocks;
    const RopeSide& s = p.side[key ? 1 : 0];
    const int block = static_cast<int>(blockIdx.x) - (key ? p.side[0].blocks : 0);
    const int half = p.rot / 2;
    float2* const cs = reinterpret_cast<float2*>(any_smem) + warp * half;
    float* const dw = any_smem + kAnyWarps * p.rot + warp * p.dim;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (kBwd)
        for (int i = lane; i < p.dim; i += 32) dw[i] = 0.f;
    const T* const w = static_cast<const T*>(s.w);
    auto weight = [&](int i) { return w ? get1(w + i) : 1.f; };
    const float inv_dim = 1.f / static_cast<float>(p.dim);
    const int64_t units = p.tokens * s.units_per_token;
    for (int64_t unit = static_cast<int64_t>(block) * kAnyWarps + warp; unit < units; unit += static_cast<int64_t>(s.blocks) * kAnyWarps) {
        const int64_t token = unit / s.units_per_token;
        const int head0 = static_cast<int>(unit % s.units_per_token) * s.heads_per_unit;
        const int head1 = min(head0 + s.heads_per_unit, s.heads);
        const int64_t position = p.positions ? p.positions[token] : token;
        __syncwarp();
        for (int i = lane; i < half; i += 32) cs[i] = turn_of(position, p.inv_freq[i]);
        __syncwarp();
        for (int64_t head = head0; head < head1; ++head) {
            const T* const x = static_cast<const T*>(s.x) + token * s.ldx + head * s.sx;
            const T* const g = static_cast<const T*>(s.g) + token * s.ldg + head * s.sg;
            T* const out = static_cast<T*>(s.out) + token * s.ldo + head * s.so;
            // element i of `row` turned by the angle of its pair
            auto turned = [&](const T* row, int i, float scale, bool weighted, float sign) {
                const float z = get1(row + i) * scale * (weighted ? weight(i) : 1.f);
                if (i >= p.rot) return z;
                const bool second = kPairs ? i & 1 : i >= half;
                const int j = kPairs ? i ^ 1 : second ? i - half : i + half;
                const float2 c = cs[kPairs ? i / 2 : second ? j : i];
                const float other = get1(row + j) * scale * (weighted ? weight(j) : 1.f);
                return z * c.x + (second ? other : -other) * sign * c.y;
            };
            float sq = 0.f;
            for (int i = lane; i < p.dim; i += 32) { const float v = get1(x + i); sq = fmaf(v, v, sq); }
            const float r = rsqrtf(fmaf(sum_lanes<32>(sq), inv_dim, p.eps));
            if constexpr (!kBwd) {
                for (int i = lane; i < p.dim; i += 32) put1(out + i, turned(x, i, r, true, 1.f));
            } else {
                float dot = 0.f;
                for (int i = lane; i < p.dim; i += 32) {
                    const float e = turned(g, i, 1.f, false, -1.f), n = get1(x + i) * r;
                    dw[i] = fmaf(e, n, dw[i]);
                    dot = fmaf(e * weight(i), n, dot);
                }
                dot = sum_lanes<32>(dot) * inv_dim;
                for (int i = lane; i < p.dim; i += 32)
                    put1(out + i, r * (turned(g, i, 1.f, false, -1.f) * weight(i) - get1(x + i) * r * dot));
            }
        }
    }
    if constexpr (kBwd) {
        if (!s.partial) return;
        __syncthreads();
        for (int c = threadIdx.x; c < p.dim; c += kAnyThreads) {
            float sum = 0.f;
            for (int v = 0; v < kAnyWarps; ++v) sum += any_smem[kAnyWarps * p.rot + v * p.dim + c];
            s.partial[static_cast<int64_t>(block) * p.dim + c] = sum;
        }
    }
}

// dw of both sides: the sums of the blocks, added in block order by eight warps to 32 columns (warp v takes blocks v, v + 8, ...).
struct WeightSums {
    const float* partial[2];
    void* out[2];
    int blocks[2];
    int dim, accumulate;
};
template <typename T>
__global__ void __launch_bounds__(256) rope_weight_kernel(const WeightSums p) {
    const int side = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = static_cast<int>(blockIdx.x) * 32 + lane;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    T* const out = static_cast<T*>(p.out[side]);
    if (!out) return;
    float sum = 0.f;
    if (col < p.dim)
#pragma unroll 8
        for (int b = warp; b < p.blocks[side]; b += 8) sum += p.partial[side][static_cast<int64_t>(b) * p.dim + col];
    __shared__ float red[8][32];
    red[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && col < p.dim) {
#pragma unroll
        for (int v = 1; v < 8; ++v) sum += red[v][lane];
        put1(out + col, p.accumulate ? get1(out + col) + sum : sum);
    }
}

// ------------------------------------------------------------------------------ host side
struct RowsView {
    const void* p;
    int64_t ld, s;
};
// Rows [tokens, heads, dim] that do not overlap: heads inside a token's pitch or tokens inside a head's.
bool rows_apart(const RowsView& v, int64_t tokens, int heads, int dim) {
    if (tokens <= 1 && heads <= 1) return true;
    if (tokens <= 1) return v.s >= dim;
    if (heads <= 1) return v.ld >= dim;
    return (v.s >= dim && v.ld >= v.s * (heads - 1) + dim) || (v.ld >= dim && v.s >= v.ld * (tokens - 1) + dim);
}
bool rows_valid(const RowsView& v, int64_t tokens, int heads, int dim, int dtype) {
    return v.p && elem_aligned(v.p, dtype) && v.ld >= 0 && v.s >= 0 && v.ld < (1LL << 40) && v.s < (1LL << 40) && rows_apart(v, tokens, heads, dim);
}
bool rows_in_pieces(const RowsView& v, int dtype) {
    const int64_t n = 16 / static_cast<int64_t>(dtype_size(dtype));
    return reinterpret_cast<uintptr_t>(v.p) % 16 == 0 && v.ld % n == 0 && v.s % n == 0;
}

// How the rows of a call are divided: both kernels walk units of (token, some of its heads).
struct RopePlan {
    bool pieces;
    int lanes, warps;            // lanes of a row, warps of a block
    int blocks[2], heads_per_unit[2], units_per_token[2];
};
// Blocks of an SM: what its shared memory holds of the vector kernels (64 and 80 KB each with the most angles), and as many of the others.
constexpr int rope_blocks_per_sm(bool bwd) { return bwd ? 2 : 3; }
RopePlan rope_plan(int64_t tokens, const int (&heads)[2], int dim, int rot, int dtype, bool pieces, bool bwd) {
    RopePlan pl = {};
    const int n = 16 / static_cast<int>(dtype_size(dtype));
    pl.pieces = pieces && dim % (2 * n) == 0 && rot % (2 * n) == 0 && dim / (2 * n) <= 32 && rot / 2 <= kMaxPairs;
    pl.lanes = 32;
    if (pl.pieces)
        for (pl.lanes = 2; pl.lanes < dim / (2 * n);) pl.lanes *= 2;
    pl.warps = pl.pieces ? kRopeWarps : kAnyWarps;
    const int rows = pl.pieces ? 32 / pl.lanes : 1, all = heads[0] + heads[1];
    const int64_t most = static_cast<int64_t>(num_sms()) * rope_blocks_per_sm(bwd) * (pl.pieces ? 1 : 2);
    for (int i = 0; i < 2; ++i) {
        if (heads[i] == 0) continue;
        // all heads of a token in one unit, unless that leaves warps without any
        const int64_t wanted = ceil_div(most * pl.warps, tokens);
        const int per_warp = static_cast<int>(ceil_div(heads[i], rows));
        const int units = static_cast<int>(std::min<int64_t>(per_warp, std::max<int64_t>(1, wanted * heads[i] / all)));
        pl.heads_per_unit[i] = static_cast<int>(ceil_div(per_warp, units)) * rows;
        pl.units_per_token[i] = static_cast<int>(ceil_div(heads[i], pl.heads_per_unit[i]));
        const int64_t share = std::max<int64_t>(1, most * heads[i] / all);
        pl.blocks[i] = static_cast<int>(std::min<int64_t>(share, ceil_div(tokens * pl.units_per_token[i], pl.warps)));
    }
    return pl;
}

template <typename T, int kLanes, bool kPairs, bool kBwd>
cudaError_t rope_styled(const RopeParams& p, int blocks, cudaStream_t stream) {
    static std::atomic<uint64_t> allowed{0};
    const auto kernel = rope_kernel<T, kLanes, kPairs, kBwd>;
    const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(kernel), kRopeRing<kBwd> + kRopeWarps * kMaxPairs * sizeof(float2), allowed);
    if (e != cudaSuccess) return e;
    return launch_beside(kernel, dim3(static_cast<unsigned>(blocks)), kRopeThreads, kRopeRing<kBwd> + kRopeWarps * (p.rot / 2) * sizeof(float2), 1, stream, p);
}
template <typename T, int kLanes, bool kBwd>
cudaError_t rope_pieces(const RopeParams& p, bool pairs, int blocks, cudaStream_t stream) {
    return pairs ? rope_styled<T, kLanes, true, kBwd>(p, blocks, stream) : rope_styled<T, kLanes, false, kBwd>(p, blocks, stream);
}
template <typename T, bool kBwd>
cudaError_t rope_launch(const RopeParams& p, const RopePlan& pl, bool pairs, cudaStream_t stream) {
    const int blocks = pl.blocks[0] + pl.blocks[1];
    if (!pl.pieces) {
        const size_t smem = sizeof(float) * kAnyWarps * (p.rot + (kBwd ? p.dim : 0));      // at most 32 KB
        const auto kernel = pairs ? rope_any_kernel<T, true, kBwd> : rope_any_kernel<T, false, kBwd>;
        return launch_beside(kernel, dim3(static_cast<unsigned>(blocks)), kAnyThreads, smem, 1, stream, p);
    }
    switch (pl.lanes) {
        case 2: return rope_pieces<T, 2, kBwd>(p, pairs, blocks, stream);
        case 4: return rope_pieces<T, 4, kBwd>(p, pairs, blocks, stream);
        case 8: return rope_pieces<T, 8, kBwd>(p, pairs, blocks, stream);
        case 16: return rope_pieces<T, 16, kBwd>(p, pairs, blocks, stream);
        default: return rope_pieces<T, 32, kBwd>(p, pairs, blocks, stream);
    }
}

int validate_rope(const RowsView (&x)[2], const void* const (&w)[2], const int64_t* positions, const float* inv_freq, const RowsView (&out)[2],
                  int64_t tokens, const int (&heads)[2], int dim, int rot, int style, double eps, int dtype) {
    if (!valid_dtype(dtype) || tokens < 0 || heads[0] < 0 || heads[1] < 0 || (heads[0] == 0 && heads[1] == 0) || dim < 1) return PF_ERR_INVALID_ARG;
    if (rot < 0 || rot > dim || rot % 2 != 0 || (style != PF_ROPE_HALVES && style != PF_ROPE_PAIRS)) return PF_ERR_INVALID_ARG;
    if (!(eps >= 0) || !std::isfinite(eps) || (rot > 0 && (!inv_freq || !elem_aligned(inv_freq, PF_F32)))) return PF_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(positions) % 8 != 0) return PF_ERR_INVALID_ARG;
    for (int i = 0; i < 2; ++i) {
        if (w[i] && !elem_aligned(w[i], dtype)) return PF_ERR_INVALID_ARG;
        if (heads[i] > 0 && tokens > 0 && (!rows_valid(x[i], tokens, heads[i], dim, dtype) || !rows_valid(out[i], tokens, heads[i], dim, dtype)))
            return PF_ERR_INVALID_ARG;
    }
    if (dim > kMaxDim || tokens > (1LL << 31) || heads[0] > (1 << 16) || heads[1] > (1 << 16)) return PF_ERR_UNSUPPORTED;
    return PF_OK;
}

}  // namespace
}  // namespace pf

using namespace pf;

extern "C" {

int pf_qk_norm_rope_fwd(const void* q, int64_t ldq, int64_t sq, const void* k, int64_t ldk, int64_t sk, const void* wq, const void* wk,
                        const int64_t* positions, const float* inv_freq, void* q_out, int64_t ldqo, int64_t sqo, void* k_out, int64_t ldko,
                        int64_t sko, int64_t tokens, int q_heads, int k_heads, int dim, int rot_dim, int style, double eps, int dtype,
                        void* cuda_stream) {
    const RowsView x[2] = {{q, ldq, sq}, {k, ldk, sk}}, out[2] = {{q_out, ldqo, sqo}, {k_out, ldko, sko}};
    const void* const w[2] = {wq, wk};
    const int heads[2] = {q_heads, k_heads};
    const int st = validate_rope(x, w, positions, inv_freq, out, tokens, heads, dim, rot_dim, style, eps, dtype);
    if (st != PF_OK || tokens == 0) return st;
    bool pieces = true;
    for (int i = 0; i < 2; ++i)
        if (heads[i] > 0)
            pieces = pieces && rows_in_pieces(x[i], dtype) && rows_in_pieces(out[i], dtype) && reinterpret_cast<uintptr_t>(w[i]) % 16 == 0;
    const RopePlan pl = rope_plan(tokens, heads, dim, rot_dim, dtype, pieces, false);
    RopeParams p = {};
    p.positions = positions;
    p.inv_freq = inv_freq;
    p.tokens = tokens;
    p.dim = dim;
    p.rot = rot_dim;
    p.eps = static_cast<float>(eps);
    for (int i = 0; i < 2; ++i)
        p.side[i] = RopeSide{x[i].p, w[i], nullptr, const_cast<void*>(out[i].p), nullptr, x[i].ld, x[i].s, 0, 0, out[i].ld, out[i].s, heads[i],
                             pl.heads_per_unit[i], pl.units_per_token[i], pl.blocks[i]};
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool pairs = style == PF_ROPE_PAIRS;
    PF_CUDA((dtype == PF_BF16 ? rope_launch<__nv_bfloat16, false>(p, pl, pairs, stream) : rope_launch<float, false>(p, pl, pairs, stream)));
    return PF_OK;
}

size_t pf_qk_norm_rope_bwd_workspace(int64_t tokens, int q_heads, int k_heads, int dim) {
    if (tokens <= 0 || q_heads < 0 || k_heads < 0 || dim < 1) return 0;
    // a row of sums for each block, of which there are at most so many on either side
    return align_up(sizeof(float) * dim * (static_cast<size_t>(num_sms()) * 2 * rope_blocks_per_sm(true) + 2), 256);
}

int pf_qk_norm_rope_bwd(const void* q, int64_t ldq, int64_t sq, const void* k, int64_t ldk, int64_t sk, const void* wq, const void* wk,
                        const int64_t* positions, const float* inv_freq, const void* dq_out, int64_t lddqo, int64_t sdqo, const void* dk_out,
                        int64_t lddko, int64_t sdko, void* dq, int64_t lddq, int64_t sdq, void* dk, int64_t lddk, int64_t sdk, void* dwq, void* dwk,
                        int64_t tokens, int q_heads, int k_heads, int dim, int rot_dim, int style, double eps, int dtype, unsigned flags,
                        void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const RowsView x[2] = {{q, ldq, sq}, {k, ldk, sk}}, g[2] = {{dq_out, lddqo, sdqo}, {dk_out, lddko, sdko}}, out[2] = {{dq, lddq, sdq}, {dk, lddk, sdk}};
    const void* const w[2] = {wq, wk};
    void* const dw[2] = {dwq, dwk};
    const int heads[2] = {q_heads, k_heads};
    const int st = validate_rope(x, w, positions, inv_freq, out, tokens, heads, dim, rot_dim, style, eps, dtype);
    if (st != PF_OK) return st;
    if (flags & ~static_cast<unsigned>(PF_GRAD_ACCUMULATE | PF_GRAD_F32)) return PF_ERR_INVALID_ARG;
    const int wtype = flags & PF_GRAD_F32 ? PF_F32 : dtype;
    bool pieces = true, sums = false;
    for (int i = 0; i < 2; ++i) {
        if (dw[i] && (heads[i] == 0 || !elem_aligned(dw[i], wtype))) return PF_ERR_INVALID_ARG;
        sums = sums || dw[i];
        if (heads[i] == 0) continue;
        if (tokens > 0 && !rows_valid(g[i], tokens, heads[i], dim, dtype)) return PF_ERR_INVALID_ARG;
        pieces = pieces && rows_in_pieces(x[i], dtype) && rows_in_pieces(g[i], dtype) && rows_in_pieces(out[i], dtype) &&
                 reinterpret_cast<uintptr_t>(w[i]) % 16 == 0;
    }
    const int wst = check_ws(workspace, workspace_bytes, sums ? pf_qk_norm_rope_bwd_workspace(tokens, q_heads, k_heads, dim) : 0);
    if (wst != PF_OK) return wst;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (tokens == 0) {
        for (int i = 0; i < 2; ++i)
            if (dw[i] && !(flags & PF_GRAD_ACCUMULATE)) PF_CUDA(cudaMemsetAsync(dw[i], 0, dim * dtype_size(wtype), stream));
        return PF_OK;
    }
    const RopePlan pl = rope_plan(tokens, heads, dim, rot_dim, dtype, pieces, true);
    RopeParams p = {};
    p.positions = positions;
    p.inv_freq = inv_freq;
    p.tokens = tokens;
    p.dim = dim;
    p.rot = rot_dim;
    p.eps = static_cast<float>(eps);
    float* const partial = static_cast<float*>(workspace);
    WeightSums ws = {};
    for (int i = 0; i < 2; ++i) {
        float* const part = dw[i] ? partial + static_cast<int64_t>(i ? pl.blocks[0] : 0) * dim : nullptr;
        p.side[i] = RopeSide{x[i].p, w[i], g[i].p, const_cast<void*>(out[i].p), part, x[i].ld, x[i].s, g[i].ld, g[i].s, out[i].ld, out[i].s, heads[i],
                             pl.heads_per_unit[i], pl.units_per_token[i], pl.blocks[i]};
        ws.partial[i] = part;
        ws.out[i] = dw[i];
        ws.blocks[i] = pl.blocks[i];
    }
    const bool pairs = style == PF_ROPE_PAIRS;
    PF_CUDA((dtype == PF_BF16 ? rope_launch<__nv_bfloat16, true>(p, pl, pairs, stream) : rope_launch<float, true>(p, pl, pairs, stream)));
    if (!sums) return PF_OK;
    ws.dim = dim;
    ws.accumulate = flags & PF_GRAD_ACCUMULATE ? 1 : 0;
    const auto add = wtype == PF_BF16 ? rope_weight_kernel<__nv_bfloat16> : rope_weight_kernel<float>;
    PF_CUDA(launch_beside(add, dim3(static_cast<unsigned>(ceil_div(dim, 32)), 2), 256, 0, 1, stream, ws));
    return PF_OK;
}

}  // extern "C"
