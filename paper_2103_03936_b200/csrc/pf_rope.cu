// Norm and position rotation of the queries and keys of an attention layer, for each head, forward and backward.
//
// For a row x of `dim` elements (one head of one token at position t), n = x r with r = 1 / sqrt(mean(x^2) + eps), z = n w; the
// first `rot` elements of z are pairs (a, b) turned by the angle t f_i of their pair:
//   (a, b) -> (a cos - b sin, b cos + a sin)
// Backward, for the upstream gradient g: e = g turned back, dw = sum e n, s = e w, dx = r (s - n mean(s n)); r is recomputed.
//
// Bound by memory: a row is read and written once (backward: two read, one written).  A row's pair elements lie rot / 2 apart
// (PF_ROPE_HALVES) or side by side (PF_ROPE_PAIRS); a lane takes one 16-byte piece of each half, so that both elements of a pair are
// in one lane under either style, and a row is 2 to 32 lanes.  A warp takes several heads of a token, so that the angles (an
// integer product in parts of a turn, sine and cosine in fp32) are computed once for all of them and stay in registers.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "pf_f32x2.cuh"
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
    int step_tokens, step_parts;      // from a warp's unit to its next
    bool across;                      // the rows of a warp are one head's of several tokens (a unit is as many tokens), not several heads' of one
};
struct RopeParams {
    RopeSide side[2];
    const int64_t* positions;
    const float* inv_freq;
    int64_t tokens;
    int dim, rot;
    float eps;
};

// Angles are counted in 2^-64 of a turn, modulo a turn: a position times the turn that one position takes is then an integer product, off by at most
// 2^-65 of a turn for each position (2^-25 at position 2^40), and its upper half is the angle to 2^-32.
//
// The turn of one position, f / (2 pi): f's 24 bits times 1 / (2 pi) in 2^-96, moved by f's exponent and rounded to nearest (f up to 2^31; the whole
// turns fall off the top).  The constant is off by less than half of its last bit, 2^23 of the product's last: nothing beside the rounding until f reaches
// 2^20 (product moved down by 35), a quarter of 2^-64 at 2^31.
// A frequency that is not finite has kNoTurn, which makes its pair NaN (a finite one of just that turn is moved by 2^-64).
constexpr uint64_t kNoTurn = 1ull << 63;
__device__ __forceinline__ uint64_t turn_per_position(float f) {
    constexpr uint32_t k0 = 0x28be60dbu, k1 = 0x9391054au, k2 = 0x7f09d5f4u;      // 2^96 / (2 pi)
    const uint32_t bits = __float_as_uint(f), exponent = (bits >> 23) & 0xffu;
    const uint32_t digits = exponent ? (bits & 0x7fffffu) | 0x800000u : 0u;
    // digits * k: 120 bits, low (32), then high (88)
    const uint64_t p2 = static_cast<uint64_t>(digits) * k2, p1 = static_cast<uint64_t>(digits) * k1 + (p2 >> 32);
    const uint64_t p0 = static_cast<uint64_t>(digits) * k0 + (p1 >> 32);
    const uint64_t low = (p1 << 32) | (p2 & 0xffffffffu);
    // f = digits 2^(exponent - 150), so that the product is in 2^(exponent - 246) of a turn
    const int down = 182 - static_cast<int>(exponent);
    uint64_t turn = 0;
    if (down > 64) turn = down < 128 ? ((p0 >> (down - 65)) + 1) >> 1 : 0;
    else if (down > 0) turn = (down < 64 ? (p0 << (64 - down)) | (low >> down) : p0) + ((low >> (down - 1)) & 1);
    if (turn == kNoTurn) ++turn;
    return exponent == 255 ? kNoTurn : bits >> 31 ? 0 - turn : turn;
}
// Cosine and sine.  kExact: to fp32, the nearest quarter turn taken off as an integer, so that the eighth of a turn that is left has 24 bits of its own.
// Else the hardware's approximations within half a turn, off by 2^-20.4 (2^-21.2 of their own for angles up to pi, which are off by 2^-21.7 as fp32
// numbers): 2^-12 of half a step of a bf16 result as large as its pair (with angles in fp64 and sincospif instead
// the forward of 16384 x 40 heads of 128 took 70 us where it took 66 with these).
template <bool kExact>
__device__ __forceinline__ float2 turn_of(int64_t position, uint64_t each) {
    const uint32_t angle = static_cast<uint32_t>((static_cast<uint64_t>(position) * each) >> 32);
    float s, c;
    if (each == kNoTurn) return make_float2(__int_as_float(0x7fffffff), __int_as_float(0x7fffffff));
    if constexpr (kExact) {
        const uint32_t quarter = (angle + 0x20000000u) >> 30;
        sincospif(static_cast<float>(static_cast<int>(angle - (quarter << 30))) * 0x1p-31f, &s, &c);
        const float x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;
        c = (quarter + 1) & 2 ? -x : x;
        s = quarter & 2 ? -y : y;
    } else {
        const float x = static_cast<float>(static_cast<int>(angle)) * 0x1p-31f * 3.14159265f;
        s = __sinf(x);
        c = __cosf(x);
    }
    return make_float2(c, s);
}

__device__ __forceinline__ float get1(const float* p) { return *p; }
__device__ __forceinline__ float get1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put1(float* p, float x) { *p = x; }
__device__ __forceinline__ void put1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

template <typename T> struct Piece;      // 16 bytes: kN elements, kN / 2 pairs of neighbours
template <> struct Piece<float> {
    static constexpr int kN = 4;
    float4 raw;
    __device__ __forceinline__ void load(const void* p) { raw = *static_cast<const float4*>(p); }
    __device__ __forceinline__ void get(F2* x) const { x[0] = f2(raw.x, raw.y); x[1] = f2(raw.z, raw.w); }
    static __device__ __forceinline__ void store(void* p, const F2* x) {
        const float2 a = split(x[0]), b = split(x[1]);
        *static_cast<float4*>(p) = make_float4(a.x, a.y, b.x, b.y);
    }
};
template <> struct Piece<__nv_bfloat16> {
    static constexpr int kN = 8;
    uint4 raw;
    __device__ __forceinline__ void load(const void* p) { raw = *static_cast<const uint4*>(p); }
    __device__ __forceinline__ void get(F2* x) const {
        const unsigned w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = f2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
    static __device__ __forceinline__ void store(void* p, const F2* x) {
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = split(x[i]);
            const __nv_bfloat162 t = __floats2bfloat162_rn(f.x, f.y);
            w[i] = *reinterpret_cast<const unsigned*>(&t);
        }
        *static_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// A lane's pairs turned in place by the angles of c and s (kBack: back).  kPairs: a pair is two neighbours, those of a[] come first in c and s; else
// a pair is an element of a[] and one of b[].
template <int kN, bool kPairs, bool kBack>
__device__ __forceinline__ void turn(F2 (&a)[kN / 2], F2 (&b)[kN / 2], const F2 (&c)[kN / 2], const F2 (&s)[kN / 2]) {
    if constexpr (kPairs) {
        auto one = [](F2 x, float c1, float s1) {
            const float2 v = split(x);
            return kBack ? f2(v.x * c1 + v.y * s1, v.y * c1 - v.x * s1) : f2(v.x * c1 - v.y * s1, v.y * c1 + v.x * s1);
        };
#pragma unroll
        for (int i = 0; i < kN / 4; ++i) {
            const float2 ca = split(c[i]), sa = split(s[i]), cb = split(c[kN / 4 + i]), sb = split(s[kN / 4 + i]);
            a[2 * i] = one(a[2 * i], ca.x, sa.x);
            a[2 * i + 1] = one(a[2 * i + 1], ca.y, sa.y);
            b[2 * i] = one(b[2 * i], cb.x, sb.x);
            b[2 * i + 1] = one(b[2 * i + 1], cb.y, sb.y);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kN / 2; ++i) {
            const F2 x = a[i], y = b[i];
            a[i] = fma2(kBack ? y : negated(y), s[i], mul2(x, c[i]));
            b[i] = fma2(kBack ? negated(x) : x, s[i], mul2(y, c[i]));
        }
    }
}

template <int kLanes>
__device__ __forceinline__ float sum_lanes(float x) {
#pragma unroll
    for (int o = kLanes / 2; o > 0; o /= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

__device__ __forceinline__ void fetch16(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

// The rows that a warp takes one after the other: some heads at a time of the units of (token, some of its heads) that are its share.
struct RopeWalk {
    int token, part, h, end;      // the unit's place among its token's, the next head, the first behind the unit
    __device__ __forceinline__ void enter(const RopeSide& s) {
        h = part * s.heads_per_unit;
        end = min(h + s.heads_per_unit, s.heads);
    }
    __device__ __forceinline__ void next_unit(const RopeSide& s) {
        token += s.step_tokens;
        part += s.step_parts;
        if (part >= s.units_per_token) { part -= s.units_per_token; ++token; }
        enter(s);
    }
};

// A warp's cosines (and sines): those of a token's pairs, then from a multiple of four on those of eight pairs that are not turned.
__host__ __device__ constexpr int rope_still(int half) { return (half + 3) / 4 * 4; }
__host__ __device__ constexpr int rope_angles(int half) { return rope_still(half) + 8; }

// Which elements of a row a lane has: na from ia on and nb from ib on (kN each, fewer in the last pieces of rows of odd widths), and its pairs.
struct RopeShare {
    int ia, ib, na, nb, pair_a, pair_b;      // pair_b: PF_ROPE_PAIRS only
};
template <int kN, bool kPairs, bool kMasked>
__device__ __forceinline__ RopeShare rope_share(int l, int dim, int rot) {
    const int half = rot / 2;
    RopeShare s;
    if constexpr (!kMasked) {
        // pieces of each half of what is turned, then of each half of what is not
        const bool turned = kN * l < half;
        s.ia = turned ? kN * l : rot + kN * l - half;
        s.ib = s.ia + (turned ? half : (dim - rot) / 2);
        s.na = s.nb = 2 * kN * l < dim ? kN : 0;
        s.pair_a = turned ? (kPairs ? s.ia / 2 : s.ia) : rope_still(half);
        s.pair_b = turned ? s.ib / 2 : rope_still(half);
    } else {
        // as many lanes as what is turned takes; two pieces side by side where pairs are neighbours, and of what is not turned
        const int lanes = kPairs ? (rot + 2 * kN - 1) / (2 * kN) : (half + kN - 1) / kN;
        const bool turned = l < lanes, apart = turned && !kPairs;
        const int end = apart ? half : turned ? rot : dim;
        s.ia = apart ? kN * l : turned ? 2 * kN * l : rot + 2 * kN * (l - lanes);
        s.na = max(0, min(kN, end - s.ia));
        s.ib = s.ia + (apart ? half : kN);
        s.nb = apart ? s.na : max(0, min(kN, end - s.ib));
        s.pair_a = turned ? kN * l : rope_still(half);
        s.pair_b = turned ? kN * l + kN / 2 : rope_still(half);
    }
    return s;
}
// Eight elements of a row of any alignment, of which n exist.  bf16: put together from the aligned words that hold them.
__device__ __forceinline__ void load_some(const float* p, int n, F2 (&x)[4]) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = f2(v[2 * i], v[2 * i + 1]);
}
__device__ __forceinline__ void load_some(const __nv_bfloat16* p, int n, F2 (&x)[4]) {
    const unsigned odd = static_cast<unsigned>(reinterpret_cast<uintptr_t>(p) >> 1) & 1u;
    const unsigned* const low = reinterpret_cast<const unsigned*>(p - odd);
    unsigned w[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = n > 0 && 2 * i - static_cast<int>(odd) < n ? low[i] : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned t = __funnelshift_r(w[i], w[i + 1], odd * 16);
        x[i] = f2(2 * i < n ? __uint_as_float(t << 16) : 0.f, 2 * i + 1 < n ? __uint_as_float(t & 0xffff0000u) : 0.f);
    }
}
__device__ __forceinline__ void store_some(float* p, int n, const F2 (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 v = split(x[i]);
        if (2 * i < n) p[2 * i] = v.x;
        if (2 * i + 1 < n) p[2 * i + 1] = v.y;
    }
}
__device__ __forceinline__ void store_some(__nv_bfloat16* p, int n, const F2 (&x)[4]) {
    __nv_bfloat162 t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 v = split(x[i]);
        t[i] = __floats2bfloat162_rn(v.x, v.y);
    }
    if ((reinterpret_cast<uintptr_t>(p) & 2) == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (2 * i + 1 < n) *reinterpret_cast<__nv_bfloat162*>(p + 2 * i) = t[i];
            else if (2 * i < n) p[2 * i] = t[i].x;
        }
    } else {
        if (n > 0) p[0] = t[0].x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i < 3 && 2 * i + 2 < n) *reinterpret_cast<__nv_bfloat162*>(p + 2 * i + 1) = __nv_bfloat162(t[i].y, t[i < 3 ? i + 1 : 3].x);
            else if (2 * i + 1 < n) p[2 * i + 1] = t[i].y;
        }
    }
}

// kLanes lanes to a row (the power of two from the row's pieces / 2 on), 32 / kLanes rows of a warp at a time.  Each lane keeps the
// pieces of its next kStages - 1 rows on the way into its own places of shared memory, across units: what a warp waits for was asked for rows
// ago, and nothing is exchanged between lanes but the sums and the angles.  Few rows ahead are enough, and more cost time (16384 x 40 heads of 128: forward
// 59.5 us with 3 stages, 62.2 with 5, 62.8 with 8; backward 84 with 2, 92 with 3, 94 with 4).
template <bool kBwd> constexpr int kRopeStages = kBwd ? 2 : 3;
template <bool kBwd> constexpr int kRopePieces = kBwd ? 4 : 2;      // 16-byte pieces of a lane for a row: two of x, two of the gradient
template <bool kBwd> constexpr int kRopeRing = kRopeWarps * kRopeStages<kBwd> * kRopePieces<kBwd> * 32 * 16;
// (kMasked: no places, but room for the sums of dw.)
template <bool kBwd, bool kMasked> constexpr int kRopeBefore = !kMasked ? kRopeRing<kBwd> : kBwd ? 16384 : 0;
// Behind them each warp's cosines, then its sines.

// kMasked: rows of any width and alignment, element loads straight to registers.  kAcross: kernels that know sides with RopeSide::across (apart, for the
// registers that they need: 16384 x 40 heads of 128 backward 79 -> 89 us).
template <typename T, int kLanes, bool kPairs, bool kBwd, bool kMasked, bool kAcross>
__global__ void __launch_bounds__(kRopeThreads, 2) rope_kernel(const RopeParams p) {
    constexpr int kN = kMasked ? 8 : Piece<T>::kN, kRows = 32 / kLanes, kStages = kRopeStages<kBwd>, kPieces = kRopePieces<kBwd>, kStage = kPieces * 32 * 16;
    constexpr bool kExact = sizeof(T) == 4;
    extern __shared__ __align__(16) unsigned char rope_smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool key = static_cast<int>(blockIdx.x) >= p.side[0].blocks;
    const RopeSide& s = p.side[key ? 1 : 0];
    const bool across = kAcross && s.across;
    const int block = static_cast<int>(blockIdx.x) - (key ? p.side[0].blocks : 0);
    const int l = lane % kLanes, row = lane / kLanes, half = p.rot / 2, tokens = static_cast<int>(p.tokens);
    const RopeShare share = rope_share<kN, kPairs, kMasked>(l, p.dim, p.rot);
    const int ia = share.ia, ib = share.ib, pair_a = share.pair_a, pair_b = share.pair_b;
    const bool there = share.na > 0;
    unsigned char* const ring = rope_smem + (warp * kStages * kPieces * 32 + lane) * 16;
    const uint32_t ring_at = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
    float* const cosines = reinterpret_cast<float*>(rope_smem + kRopeBefore<kBwd, kMasked>) + warp * 2 * rope_angles(half);
    float* const sines = cosines + rope_angles(half);
    RopeWalk ahead, at;      // rows to ask for, rows to compute
    {
        const unsigned unit = static_cast<unsigned>(block) * kRopeWarps + warp, per = static_cast<unsigned>(s.units_per_token);
        ahead.token = static_cast<int>(unit / per);
        ahead.part = static_cast<int>(unit - ahead.token * per);
        if (across) ahead.token *= kRows;
        ahead.enter(s);
        at = ahead;
    }
    const int turn_heads = across ? 1 : kRows;      // from a warp's rows to its next
    const T* const x0 = static_cast<const T*>(s.x) + row * (across ? s.ldx : s.sx);
    const T* const g0 = static_cast<const T*>(s.g) + row * (across ? s.ldg : s.sg);
    auto has_row = [&](const RopeWalk& w) { return across ? w.token + row < tokens : w.h + row < w.end; };
    const T* xp = x0 + ahead.token * s.ldx + ahead.h * s.sx;
    const T* gp = g0 + ahead.token * s.ldg + ahead.h * s.sg;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    auto ask = [&](int stage) {
        if constexpr (kMasked) return;
        if (ahead.token < tokens) {
            if (there && has_row(ahead)) {
                const uint32_t to = ring_at + stage * kStage;
                fetch16(to, xp + ia);
                fetch16(to + 512, xp + ib);
                if constexpr (kBwd) {
                    fetch16(to + 1024, gp + ia);
                    fetch16(to + 1536, gp + ib);
                }
            }
            ahead.h += turn_heads;
            if (ahead.h >= ahead.end) {
                ahead.next_unit(s);
                xp = x0 + ahead.token * s.ldx + ahead.h * s.sx;
                if constexpr (kBwd) gp = g0 + ahead.token * s.ldg + ahead.h * s.sg;
            } else {
                xp += turn_heads * s.sx;
                if constexpr (kBwd) gp += turn_heads * s.sg;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) ask(i);
    auto position_of = [&](const RopeWalk& w) -> int64_t {      // (across: of this lane's token)
        const int token = across ? w.token + row : w.token;
        return token >= tokens ? 0 : p.positions ? p.positions[token] : token;
    };
    int64_t position = position_of(at);
    // the turns of this lane's first angles for a position (those of rows of more than 64 pairs are made again for each token)
    constexpr int kKept = 2;
    uint64_t each[kKept];
#pragma unroll
    for (int i = 0; i < kKept; ++i) each[i] = lane + 32 * i < half ? turn_per_position(p.inv_freq[lane + 32 * i]) : 0;
    // (across: those of all pairs for the block)
    uint64_t* const turns = reinterpret_cast<uint64_t*>(rope_smem + kRopeBefore<kBwd, kMasked>);
    if (across) {
        for (int i = threadIdx.x; i < half; i += kRopeThreads) turns[i] = turn_per_position(p.inv_freq[i]);
        __syncthreads();
    } else if (lane < rope_angles(half) - half) {
        cosines[half + lane] = 1.f;
        sines[half + lane] = 0.f;
    }
    F2 wa[kN / 2], wb[kN / 2];
#pragma unroll
    for (int i = 0; i < kN / 2; ++i) wa[i] = wb[i] = f2(1.f, 1.f);
    if (s.w && there) {
        if constexpr (kMasked) {
            load_some(static_cast<const T*>(s.w) + ia, share.na, wa);
            load_some(static_cast<const T*>(s.w) + ib, share.nb, wb);
        } else {
            Piece<T> t;
            t.load(static_cast<const T*>(s.w) + ia);
            t.get(wa);
            t.load(static_cast<const T*>(s.w) + ib);
            t.get(wb);
        }
    }
    F2 dwa[kN / 2], dwb[kN / 2];
#pragma unroll
    for (int i = 0; i < kN / 2; ++i) dwa[i] = dwb[i] = f2(0.f, 0.f);
    const float inv_dim = 1.f / static_cast<float>(p.dim);
    int stage = 0;
    while (at.token < tokens) {
        F2 c[kN / 2], sn[kN / 2];
        if (across) {      // each lane the angles of its own pairs
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                const int pair = !kPairs || i < kN / 2 ? pair_a + i : pair_b + i - kN / 2;
                const float2 v = pair < half ? turn_of<kExact>(position, turns[pair]) : make_float2(1.f, 0.f);
                const float2 cv = split(c[i / 2]), sv = split(sn[i / 2]);
                c[i / 2] = i % 2 ? f2(cv.x, v.x) : f2(v.x, 0.f);
                sn[i / 2] = i % 2 ? f2(sv.x, v.y) : f2(v.y, 0.f);
            }
        } else {
            __syncwarp();
            auto angle = [&](int i, uint64_t turn_each) {
                const float2 v = turn_of<kExact>(position, turn_each);
                cosines[i] = v.x;
                sines[i] = v.y;
            };
#pragma unroll
            for (int i = 0; i < kKept; ++i)
                if (lane + 32 * i < half) angle(lane + 32 * i, each[i]);
            for (int i = lane + 32 * kKept; i < half; i += 32) angle(i, turn_per_position(p.inv_freq[i]));
            __syncwarp();
#pragma unroll
            for (int i = 0; i < kN / 2; ++i) {
                const int at_pair = !kPairs ? pair_a + 2 * i : i < kN / 4 ? pair_a + 2 * i : pair_b + 2 * i - kN / 2;
                c[i] = *reinterpret_cast<const F2*>(cosines + at_pair);
                sn[i] = *reinterpret_cast<const F2*>(sines + at_pair);
            }
        }
        RopeWalk next = at;
        next.next_unit(s);
        position = position_of(next);
        T* out = static_cast<T*>(s.out) + at.token * s.ldo + at.h * s.so + row * (across ? s.ldo : s.so);
        for (; at.h < at.end; at.h += turn_heads, out += turn_heads * s.so) {
            const bool live = has_row(at), on = there && live;
            F2 a[kN / 2], b[kN / 2], ea[kN / 2], eb[kN / 2];      // x, and the upstream gradient
            if constexpr (kMasked) {
                const T* const x = x0 + at.token * s.ldx + at.h * s.sx;
                load_some(x + ia, on ? share.na : 0, a);
                load_some(x + ib, on ? share.nb : 0, b);
                if constexpr (kBwd) {
                    const T* const g = g0 + at.token * s.ldg + at.h * s.sg;
                    load_some(g + ia, on ? share.na : 0, ea);
                    load_some(g + ib, on ? share.nb : 0, eb);
                }
            } else {
                __syncwarp();
                ask(stage == 0 ? kStages - 1 : stage - 1);      // the place that the row before has left
                asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
                const unsigned char* const in = ring + stage * kStage;
                stage = stage == kStages - 1 ? 0 : stage + 1;
                auto get = [&](F2 (&x)[kN / 2], int piece) {
                    Piece<T> t;
                    t.raw = {};
                    if (on) t.load(in + 512 * piece);
                    t.get(x);
                };
                get(a, 0);
                get(b, 1);
                if constexpr (kBwd) {
                    get(ea, 2);
                    get(eb, 3);
                }
            }
            F2 sq2 = mul2(a[0], a[0]);
#pragma unroll
            for (int i = 1; i < kN / 2; ++i) sq2 = fma2(a[i], a[i], sq2);
#pragma unroll
            for (int i = 0; i < kN / 2; ++i) sq2 = fma2(b[i], b[i], sq2);
            const float2 pairs2 = split(sq2);
            const float sq = sum_lanes<kLanes>(pairs2.x + pairs2.y);      // (all lanes take part)
            // (a row behind the last head adds nothing to dw, whatever eps is)
            const float r = live ? rsqrtf(fmaf(sq, inv_dim, p.eps)) : 0.f;
            const F2 rr = f2(r, r);
            if constexpr (!kBwd) {
#pragma unroll
                for (int i = 0; i < kN / 2; ++i) { a[i] = mul2(a[i], mul2(rr, wa[i])); b[i] = mul2(b[i], mul2(rr, wb[i])); }
                turn<kN, kPairs, false>(a, b, c, sn);
            } else {
                turn<kN, kPairs, true>(ea, eb, c, sn);
                F2 dot2 = f2(0.f, 0.f);
#pragma unroll
                for (int i = 0; i < kN / 2; ++i) {
                    a[i] = mul2(a[i], rr);
                    b[i] = mul2(b[i], rr);
                    dwa[i] = fma2(ea[i], a[i], dwa[i]);
                    dwb[i] = fma2(eb[i], b[i], dwb[i]);
                    ea[i] = mul2(ea[i], wa[i]);
                    eb[i] = mul2(eb[i], wb[i]);
                    dot2 = fma2(ea[i], a[i], fma2(eb[i], b[i], dot2));
                }
                const float2 d = split(dot2);
                const float dot = -sum_lanes<kLanes>(d.x + d.y) * inv_dim;
                const F2 dd = f2(dot, dot);
#pragma unroll
                for (int i = 0; i < kN / 2; ++i) { a[i] = mul2(rr, fma2(a[i], dd, ea[i])); b[i] = mul2(rr, fma2(b[i], dd, eb[i])); }
            }
            if constexpr (kMasked) {
                store_some(out + ia, on ? share.na : 0, a);
                store_some(out + ib, on ? share.nb : 0, b);
            } else if (on) {
                Piece<T>::store(out + ia, a);
                Piece<T>::store(out + ib, b);
            }
        }
        at = next;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if constexpr (kBwd) {
        if (!s.partial) return;
        // rows of a warp, then warps in order
        float* const red = reinterpret_cast<float*>(rope_smem);      // (16 KB of the pieces' places at most)
        static_assert(kRopeWarps * 2 * kN * kLanes * 4 <= kRopeBefore<kBwd, kMasked>, "");
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            float da = i % 2 ? split(dwa[i / 2]).y : split(dwa[i / 2]).x, db = i % 2 ? split(dwb[i / 2]).y : split(dwb[i / 2]).x;
#pragma unroll
            for (int o = kLanes; o < 32; o *= 2) {
                da += __shfl_xor_sync(0xffffffffu, da, o);
                db += __shfl_xor_sync(0xffffffffu, db, o);
            }
            if (row == 0) {
                red[(warp * 2 * kN + i) * kLanes + l] = da;
                red[(warp * 2 * kN + kN + i) * kLanes + l] = db;
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * kN * kLanes; i += kRopeThreads) {
            const int e = i / kLanes;
            const RopeShare q = rope_share<kN, kPairs, kMasked>(i % kLanes, p.dim, p.rot);
            if (e < kN ? e >= q.na : e - kN >= q.nb) continue;
            float sum = 0.f;
            for (int w = 0; w < kRopeWarps; ++w) sum += red[(w * 2 * kN + e) * kLanes + i % kLanes];
            s.partial[static_cast<int64_t>(block) * p.dim + (e < kN ? q.ia + e : q.ib + e - kN)] = sum;
        }
    }
}

// Rows that are too wide for a warp's registers: a warp to a row, element after element, the other element of a pair read again.
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
        for (int i = lane; i < half; i += 32) cs[i] = turn_of<true>(position, turn_per_position(p.inv_freq[i]));
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

// dw of both sides: the sums of the blocks, added in block order by 32 warps to 32 columns (warp v takes blocks v, v + 32, ...).
constexpr int kWeightWarps = 32;
struct WeightSums {
    const float* partial[2];
    void* out[2];
    int blocks[2];
    int dim, accumulate;
};
template <typename T>
__global__ void __launch_bounds__(kWeightWarps * 32) rope_weight_kernel(const WeightSums p) {
    const int side = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = static_cast<int>(blockIdx.x) * 32 + lane;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    T* const out = static_cast<T*>(p.out[side]);
    if (!out) return;
    float sum = 0.f;
    if (col < p.dim)
#pragma unroll 8
        for (int b = warp; b < p.blocks[side]; b += kWeightWarps) sum += p.partial[side][static_cast<int64_t>(b) * p.dim + col];
    __shared__ float red[kWeightWarps][32];
    red[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && col < p.dim) {
#pragma unroll
        for (int v = 1; v < kWeightWarps; ++v) sum += red[v][lane];
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
    enum Kind { kAny, kMasked, kPieces } kind;
    int lanes, warps;            // lanes of a row, warps of a block
    int blocks[2], heads_per_unit[2], units_per_token[2], tokens_per_unit[2];
    RopeSide side(int i, RopeSide s) const {
        s.heads_per_unit = heads_per_unit[i];
        s.units_per_token = units_per_token[i];
        s.blocks = blocks[i];
        if (s.heads > 0) {
            s.step_tokens = blocks[i] * warps / units_per_token[i] * tokens_per_unit[i];
            s.step_parts = blocks[i] * warps % units_per_token[i];
            s.across = tokens_per_unit[i] > 1;
        }
        return s;
    }
};
// Blocks of an SM: two of the vector kernels, whose registers (80 for three forward ones) would otherwise spill: 16384 x 40 heads of 128 forward 66 us with
// three, 59.5 with two.  Twice as many of the others.
constexpr int kRopeBlocksPerSm = 2;
RopePlan rope_plan(int64_t tokens, const int (&heads)[2], int dim, int rot, bool pairs, int dtype, bool pieces) {
    RopePlan pl = {};
    const int n = 16 / static_cast<int>(dtype_size(dtype));
    const int half = rot / 2;
    if (pieces && dim % (2 * n) == 0 && rot % (2 * n) == 0 && dim / (2 * n) <= 32 && half <= kMaxPairs) {
        pl.kind = RopePlan::kPieces;
        pl.lanes = dim / (2 * n);
    } else {
        pl.lanes = static_cast<int>((pairs ? ceil_div(rot, 16) : ceil_div(half, 8)) + ceil_div(dim - rot, 16));
        pl.kind = pl.lanes <= 32 && half <= kMaxPairs ? RopePlan::kMasked : RopePlan::kAny;
    }
    const bool any = pl.kind == RopePlan::kAny;
    int lanes = 2;
    while (lanes < pl.lanes && lanes < 32) lanes *= 2;
    pl.lanes = lanes;
    pl.warps = any ? kAnyWarps : kRopeWarps;
    const int rows = any ? 1 : 32 / pl.lanes;
    const int64_t most = static_cast<int64_t>(num_sms()) * kRopeBlocksPerSm * (any ? 2 : 1);
    // A side of few heads fills a warp with one head's rows of several tokens, each with angles of its own (8192 tokens of one head of 64: 8.3 us
    // with idle lanes, 4.0 so).
    double time[2];      // of a side by one warp, in turns of a warp at its rows; what a unit costs besides is kUnit of one (kOwn with own angles)
    constexpr double kUnit = 0.5, kOwn = 1.0;
    for (int i = 0; i < 2; ++i) {
        const bool across = pl.kind == RopePlan::kPieces && pl.lanes < 32 && heads[i] > 0 && heads[i] * 2 <= rows && tokens > 1;
        pl.tokens_per_unit[i] = across ? rows : 1;
        time[i] = heads[i] == 0 ? 0.0 : across ? (heads[i] + kOwn) / rows : ceil_div(heads[i], rows) + kUnit;
    }
    for (int i = 0; i < 2; ++i) {
        if (heads[i] == 0) continue;
        const int64_t share = std::max<int64_t>(1, static_cast<int64_t>(most * time[i] / (time[0] + time[1])));
        const int64_t turns = ceil_div(heads[i], rows);
        pl.heads_per_unit[i] = heads[i];
        // units as large as leave the warps equal shares
        double best = 0;
        for (int64_t units = 1; units <= turns && pl.tokens_per_unit[i] == 1; units *= 2) {
            const int64_t each = ceil_div(turns, units);
            const double t = static_cast<double>(ceil_div(tokens * ceil_div(turns, each), share * pl.warps)) * (each + kUnit);
            if (units > 1 && t > 0.98 * best) continue;
            best = t;
            pl.heads_per_unit[i] = static_cast<int>(each) * rows;
        }
        pl.units_per_token[i] = static_cast<int>(ceil_div(heads[i], pl.heads_per_unit[i]));
        const int64_t units = ceil_div(tokens, pl.tokens_per_unit[i]) * pl.units_per_token[i];
        pl.blocks[i] = static_cast<int>(std::min<int64_t>(share, ceil_div(units, pl.warps)));
    }
    return pl;
}

template <typename T, int kLanes, bool kPairs, bool kBwd, bool kMasked, bool kAcross>
cudaError_t rope_styled(const RopeParams& p, int blocks, cudaStream_t stream) {
    static std::atomic<uint64_t> allowed{0};
    constexpr int kBefore = kRopeBefore<kBwd, kMasked>, kAngle = kRopeWarps * 2 * static_cast<int>(sizeof(float));
    const auto kernel = rope_kernel<T, kLanes, kPairs, kBwd, kMasked, kAcross>;
    const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(kernel), kBefore + kAngle * rope_angles(kMaxPairs), allowed);
    if (e != cudaSuccess) return e;
    return launch_beside(kernel, dim3(static_cast<unsigned>(blocks)), kRopeThreads, kBefore + kAngle * rope_angles(p.rot / 2), 1, stream, p);
}
template <typename T, bool kBwd, bool kMasked, bool kAcross>
cudaError_t rope_by_lanes(const RopeParams& p, int lanes, bool pairs, int blocks, cudaStream_t stream) {
    const auto run = [&](auto n) {
        constexpr int kLanes = decltype(n)::value;
        return pairs ? rope_styled<T, kLanes, true, kBwd, kMasked, kAcross>(p, blocks, stream) : rope_styled<T, kLanes, false, kBwd, kMasked, kAcross>(p, blocks, stream);
    };
    switch (lanes) {
        case 2: return run(std::integral_constant<int, 2>());
        case 4: return run(std::integral_constant<int, 4>());
        case 8: return run(std::integral_constant<int, 8>());
        case 16: return run(std::integral_constant<int, 16>());
        default: return run(std::integral_constant<int, 32>());
    }
}
template <typename T, bool kBwd>
cudaError_t rope_launch(const RopeParams& p, const RopePlan& pl, bool pairs, cudaStream_t stream) {
    const int blocks = pl.blocks[0] + pl.blocks[1];
    const bool across = p.side[0].across || p.side[1].across;
    if (pl.kind == RopePlan::kPieces)
        return across ? rope_by_lanes<T, kBwd, false, true>(p, pl.lanes, pairs, blocks, stream) : rope_by_lanes<T, kBwd, false, false>(p, pl.lanes, pairs, blocks, stream);
    if (pl.kind == RopePlan::kMasked) return rope_by_lanes<T, kBwd, true, false>(p, pl.lanes, pairs, blocks, stream);
    const size_t smem = sizeof(float) * kAnyWarps * (p.rot + (kBwd ? p.dim : 0));      // at most 32 KB
    const auto kernel = pairs ? rope_any_kernel<T, true, kBwd> : rope_any_kernel<T, false, kBwd>;
    return launch_beside(kernel, dim3(static_cast<unsigned>(blocks)), kAnyThreads, smem, 1, stream, p);
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
    if (dim > kMaxDim || tokens > (1LL << 30) || heads[0] > (1 << 16) || heads[1] > (1 << 16)) return PF_ERR_UNSUPPORTED;
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
    const RopePlan pl = rope_plan(tokens, heads, dim, rot_dim, style == PF_ROPE_PAIRS, dtype, pieces);
    RopeParams p = {};
    p.positions = positions;
    p.inv_freq = inv_freq;
    p.tokens = tokens;
    p.dim = dim;
    p.rot = rot_dim;
    p.eps = static_cast<float>(eps);
    for (int i = 0; i < 2; ++i)
        p.side[i] = pl.side(i, RopeSide{x[i].p, w[i], nullptr, const_cast<void*>(out[i].p), nullptr, x[i].ld, x[i].s, 0, 0, out[i].ld, out[i].s, heads[i]});
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool pairs = style == PF_ROPE_PAIRS;
    PF_CUDA((dtype == PF_BF16 ? rope_launch<__nv_bfloat16, false>(p, pl, pairs, stream) : rope_launch<float, false>(p, pl, pairs, stream)));
    return PF_OK;
}

size_t pf_qk_norm_rope_bwd_workspace(int64_t tokens, int q_heads, int k_heads, int dim) {
    if (tokens <= 0 || q_heads < 0 || k_heads < 0 || dim < 1) return 0;
    // a row of sums for each block, of which there are at most so many on either side
    return align_up(sizeof(float) * dim * (static_cast<size_t>(num_sms()) * 2 * kRopeBlocksPerSm + 2), 256);
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
    const RopePlan pl = rope_plan(tokens, heads, dim, rot_dim, style == PF_ROPE_PAIRS, dtype, pieces);
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
        p.side[i] = pl.side(i, RopeSide{x[i].p, w[i], g[i].p, const_cast<void*>(out[i].p), part, x[i].ld, x[i].s, g[i].ld, g[i].s, out[i].ld, out[i].s, heads[i]});
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
    PF_CUDA(launch_beside(add, dim3(static_cast<unsigned>(ceil_div(dim, 32)), 2), kWeightWarps * 32, 0, 1, stream, ws));
    return PF_OK;
}

}  // extern "C"
