// Row operators over a vocabulary's logits: log probabilities of given tokens with entropy and the largest alternatives, the divergence
// from a teacher's largest logits, and the gradients of both.
//
// For a row z of logits and a factor s: M = max z, S = sum exp(s (z - M)), W = sum exp(s (z - M)) s (z - M), so that log p = s (z - M) - log S and the
// entropy is log S - W / S (both parts >= 0: nothing cancels).  Gradients are p (a + b log p), and what the given tokens take away.
//
// Bound by memory, and next to it by issue (about seven instructions for an element, one of them a power of two).  Two kernels:
//   vocab_kernel          a block has a row, or a part of one where it is longer than 64 KB or rows are few: it stays in shared memory between its statistics and its
//                         gradient; the parts of a row are a cluster, whose blocks read one another's M, S and W.  64 KB leave room for three blocks on an SM, one of which
//                         loads while another computes or stores.
//   vocab_stream_kernel   forward of many long rows: three blocks stay on each SM and walk over rows, chunks of which (16 KB) come through a ring, asked for across rows' ends.
// 2048 x 131072 bf16: log probabilities and entropy 93 us (5.8 TB/s), with 20 alternatives 125, gradient 241 (4.5 TB/s); 4096 x 32001: 60 us (4.4 TB/s), with 8 79,
// gradient 99 (5.3 TB/s); divergence from 64 entries, 4096 x 32768: 66 us, gradient 113.
// A thread takes the largest of four pieces of 16 bytes before their powers.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "pf_f32x2.cuh"
#include "pf_internal.h"
#include "pf_tc.h"
#include "pf_tc_prims.cuh"

namespace pf {
namespace {

enum VocabMode { kLogprobsFwd, kLogprobsBwd, kDistillFwd, kDistillBwd };

constexpr int kMaxTop = 128, kMaxTeacher = 256, kMaxParts = 8;
constexpr int kCollected = 512;        // of a block's candidates that are ranked against one another
constexpr int kOwners = 256;           // shares that are gone through again at most
constexpr int64_t kPartBytes = 65536, kPartBytesMost = 200 << 10, kPartBytesLeast = 8192;
constexpr int kDeep = 4, kMaxChunks = 16;      // pieces of a thread in a chunk of the row, one bulk copy; chunks (13 of 256 threads in 200 KB)
// A term e^d d of a logit of -infinity, or of one so far below the largest that d is, has to be 0 and not NaN.  Beside a largest logit between -kFar and kFar, logits below
// -2^100 are taken as that, which leaves d finite at every scale (distances of kFarthest at most).  Elsewhere, and where the gradient times that distance is not finite, exponents
// below kLeast, whose powers are 0, are taken as that (a few instructions more).
constexpr float kFar = 1e30f, kLowest = -0x1p100f, kFarthest = 2.3e30f, kLeast = -200.f;

struct VocabParams {
    const void* logits;
    const int64_t* ids;              // [tokens], or [tokens, k] of the teacher
    const float* dlogprobs;
    const float* dentropy;
    const float* teacher;
    const float* teacher_lse;
    const float* dloss;
    float *logprobs, *entropy, *lse, *top_logprobs, *loss;
    int64_t* top_ids;
    void* dlogits;
    int64_t ld, lddl, tokens;
    int vocab, parts, top, k;
    float scale;
    unsigned int* status;
};

struct alignas(16) Stats {
    float m, s, w;
    float pad;
};
// For finding the largest elements.
struct Largest {
    uint64_t candidates[kCollected];
    uint64_t best[8];
    int warps[8];
    int counts[2][2];      // of alternate uses: candidates, owners
    uint16_t owners[kOwners];
};
// What a row's given tokens, or the teacher's, are.
struct alignas(16) TeacherShared {
    int id[kMaxTeacher];      // (behind the last -1, up to a multiple of four)
    float q[kMaxTeacher], logq[kMaxTeacher], z[kMaxTeacher];
};
// Of vocab_kernel, in front of the pieces of the row.
struct VocabShared {
    uint64_t bars[kMaxChunks];
    float extra[16];                       // elements before the first piece of the row, and behind the last
    Stats warp[9];
    Stats part;
    uint32_t abort;
};
struct VocabTop {
    union {
        Largest largest;
        uint64_t parts[kMaxParts * kMaxTop];      // the parts' largest, behind that in time
    };
    uint64_t list[kMaxTop];                       // this part's, in order
    alignas(16) uint32_t keys[256];               // the threads' largest logits
};
struct VocabNone {};
template <int kMode>
struct VocabRow : VocabShared {
    std::conditional_t<kMode == kLogprobsFwd, VocabTop, std::conditional_t<kMode == kLogprobsBwd, VocabNone, TeacherShared>> own;
};
template <int kMode> constexpr size_t kVocabHead = (sizeof(VocabRow<kMode>) + 15) / 16 * 16;

__device__ __forceinline__ float exp2_of(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Exponents d of two logits less base (kClamp: kLeast at least), and e = 2^d.
template <bool kClamp>
__device__ __forceinline__ F2 powers(F2 x, F2 minus_base, F2 c, F2* d) {
    *d = mul2(add2(x, minus_base), c);
    float2 v = split(*d);
    if constexpr (kClamp) {
        v.x = max_nan(v.x, kLeast);
        v.y = max_nan(v.y, kLeast);
        *d = f2(v.x, v.y);
    }
    return f2(exp2_of(v.x), exp2_of(v.y));
}

// 16 bytes of logits.
template <typename T> struct Logits;
template <> struct Logits<__nv_bfloat16> {
    static constexpr int kN = 8;
    static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
    static __device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
    template <int kDeep>
    static __device__ __forceinline__ float largest(const uint4 (&v)[kDeep]) {      // (NaN only if all are)
        uint32_t m = Logits::kNone;
#pragma unroll
        for (int j = 0; j < kDeep; ++j) m = max_bf16x2(m, max_bf16x2(max_bf16x2(v[j].x, v[j].y), max_bf16x2(v[j].z, v[j].w)));
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    }
    static __device__ __forceinline__ void get(uint4 v, F2 (&x)[4]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = f2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
    static __device__ __forceinline__ uint4 raised(uint4 v) {      // kLowest at least
        return make_uint4(max_nan_bf16x2(v.x, 0xf180f180u), max_nan_bf16x2(v.y, 0xf180f180u), max_nan_bf16x2(v.z, 0xf180f180u), max_nan_bf16x2(v.w, 0xf180f180u));
    }
    static constexpr uint32_t kNone = 0xff80ff80u;      // -infinity
    static __device__ __forceinline__ float element(uint4 v, int i) {
        const uint32_t w = i < 4 ? (i < 2 ? v.x : v.y) : i < 6 ? v.z : v.w;
        return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
    }
    static __device__ __forceinline__ uint4 pack(const F2 (&x)[4]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = split(x[i]);
            const __nv_bfloat162 t = __floats2bfloat162_rn(f.x, f.y);
            w[i] = *reinterpret_cast<const uint32_t*>(&t);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Logits<float> {
    static constexpr int kN = 4;
    static __device__ __forceinline__ float one(const float* p) { return *p; }
    static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
    template <int kDeep>
    static __device__ __forceinline__ float largest(const uint4 (&v)[kDeep]) {
        float m = -INFINITY;
#pragma unroll
        for (int j = 0; j < kDeep; ++j)
            m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(v[j].x), __uint_as_float(v[j].y)), fmaxf(__uint_as_float(v[j].z), __uint_as_float(v[j].w))));
        return m;
    }
    static __device__ __forceinline__ void get(uint4 v, F2 (&x)[2]) {
        x[0] = f2(__uint_as_float(v.x), __uint_as_float(v.y));
        x[1] = f2(__uint_as_float(v.z), __uint_as_float(v.w));
    }
    static __device__ __forceinline__ uint4 raised(uint4 v) {
        auto one = [](uint32_t x) { return __float_as_uint(max_nan(__uint_as_float(x), kLowest)); };
        return make_uint4(one(v.x), one(v.y), one(v.z), one(v.w));
    }
    static constexpr uint32_t kNone = 0xff800000u;
    static __device__ __forceinline__ float element(uint4 v, int i) { return __uint_as_float(i < 2 ? (i < 1 ? v.x : v.y) : i < 3 ? v.z : v.w); }
    static __device__ __forceinline__ uint4 pack(const F2 (&x)[2]) {
        const float2 a = split(x[0]), b = split(x[1]);
        return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
    }
};

// The order of logits as whole numbers: larger ones first, NaN behind all of them (1); 0 is no element.  Behind it, in 64 bits, lower places first.
__device__ __forceinline__ uint32_t order_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);
    return v != v ? 1u : b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) {
    return order == 1u ? __uint_as_float(0x7fffffffu) : __uint_as_float(order >> 31 ? order & 0x7fffffffu : ~order);
}
__device__ __forceinline__ uint64_t key_of(float v, int place) { return static_cast<uint64_t>(order_of(v)) << 32 | static_cast<uint32_t>(~place); }

__device__ __forceinline__ uint32_t smem_at(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ uint32_t of_part(uint32_t at, int part) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(part));
    return r;
}
// (all lanes of a warp at once)
__device__ __forceinline__ void cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// `bytes` of a row to shared memory (16-byte boundaries), counted on a barrier.
__device__ __forceinline__ void bulk_copy(uint32_t to, const void* from, int bytes, uint32_t bar) {
    tc::mbar_expect_tx(bar, static_cast<uint32_t>(bytes));
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}

// Of a block that has given up: until its copies have come (fills first .. last - 1 of a ring, one after the other), or once more the time after which it gives up.
__device__ __noinline__ void wait_for_copies(uint32_t bars, uint32_t first, uint32_t last, uint32_t stages) {
    const long long t0 = clock64();
    for (uint32_t f = first; f < last; ++f)
        while (!tc::mbar_try_wait(bars + 8 * (f % stages), f / stages & 1u))
            if (clock64() - t0 > tc::kWaitCycleLimit) return;
}

// Which elements of a row a part has.
template <typename T>
struct Part {
    int head, pieces, first, count;      // elements before the row's first piece, its pieces, this part's first and their number
    __device__ __forceinline__ Part(const T* row, int vocab, int part, int parts) {
        constexpr int kN = Logits<T>::kN;
        const int off = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        head = min(vocab, off ? kN - off : 0);
        pieces = (vocab - head) / kN;
        const int each = (pieces + parts - 1) / parts;
        first = min(pieces, part * each);
        count = min(pieces, first + each) - first;
    }
};

// Statistics of what a thread has seen of a row.
struct Sums {
    float m;
    F2 s2, w2;
    __device__ __forceinline__ void start() {
        m = -INFINITY;
        s2 = w2 = f2(0.f, 0.f);
    }
    __device__ __forceinline__ void move_to(float most, float c) {      // what there is, by a new largest logit
        if (most > m && m != -INFINITY) {
            const float d = fmaxf((m - most) * c, kLeast), f = exp2_of(d);
            w2 = mul2(f2(f, f), fma2(f2(d, d), s2, w2));
            s2 = mul2(f2(f, f), s2);
        }
        m = most;
    }
    __device__ __forceinline__ void add_one(float z, float c) {
        move_to(fmaxf(m, z), c);
        const float d = max_nan((z - (m == -INFINITY ? 0.f : m)) * c, kLeast), e = exp2_of(d);
        s2 = add2(s2, f2(e, 0.f));
        w2 = add2(w2, f2(e * d, 0.f));
    }
    // kW: w2 as well
    // (the largest of them)
    template <typename T, bool kW, int kDeep>
    __device__ __forceinline__ float add(const uint4 (&v)[kDeep], float c) {
        constexpr int kN = Logits<T>::kN;
        const float most = Logits<T>::largest(v);
        move_to(fmaxf(m, most), c);
        const float base = m == -INFINITY ? 0.f : m;
        const F2 base2 = f2(-base, -base), c2 = f2(c, c);
        auto terms = [&](auto clamp) {
            constexpr bool kClamp = decltype(clamp)::value;
#pragma unroll
            for (int j = 0; j < kDeep; ++j) {
                F2 x[kN / 2];
                Logits<T>::get(kClamp || !kW ? v[j] : Logits<T>::raised(v[j]), x);
#pragma unroll
                for (int e = 0; e < kN / 2; ++e) {
                    F2 d;
                    const F2 y = powers<kClamp>(x[e], base2, c2, &d);
                    s2 = add2(s2, y);
                    if constexpr (kW) w2 = fma2(y, d, w2);
                }
            }
        };
        if (kW ? fabsf(m) <= kFar : m != -INFINITY) terms(std::false_type());
        else terms(std::true_type());
        return most;
    }
};
// Statistics of parts of a row, together.  (A part without a logit above -infinity has only zeros, or NaN.)
__device__ __forceinline__ Stats together(const Stats& a, const Stats& b, float c) {
    Stats r;
    r.m = fmaxf(a.m, b.m);
    const float base = r.m == -INFINITY ? 0.f : r.m;
    const float da = a.m == -INFINITY ? 0.f : fmaxf((a.m - base) * c, kLeast), db = b.m == -INFINITY ? 0.f : fmaxf((b.m - base) * c, kLeast);
    const float fa = exp2_of(da), fb = exp2_of(db);
    r.s = fmaf(a.s, fa, b.s * fb);
    r.w = fmaf(fa, fmaf(da, a.s, a.w), fb * fmaf(db, b.s, b.w));
    r.pad = 0.f;
    return r;
}
__device__ __forceinline__ Stats by(const Stats& a, float base, float c) {
    const float d = a.m == -INFINITY ? 0.f : fmaxf((a.m - base) * c, kLeast), f = exp2_of(d);
    return {base, a.s * f, f * fmaf(d, a.s, a.w), 0.f};
}
__device__ __forceinline__ Stats warp_stats(const Sums& mine, float c) {
    const float2 s = split(mine.s2), w = split(mine.w2);
    float most = mine.m;
#pragma unroll
    for (int o = 16; o > 0; o /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    Stats a = by({mine.m, s.x + s.y, w.x + w.y, 0.f}, most == -INFINITY ? 0.f : most, c);
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
        a.w += __shfl_xor_sync(0xffffffffu, a.w, o);
    }
    a.m = most;
    return a;
}
template <int kWarps>
__device__ __forceinline__ Stats block_stats(const Stats* warps, float c) {      // (a whole warp)
    Stats a = warps[threadIdx.x % kWarps];
    float most = a.m;
#pragma unroll
    for (int o = kWarps / 2; o > 0; o /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    a = by(a, most == -INFINITY ? 0.f : most, c);
#pragma unroll
    for (int o = kWarps / 2; o > 0; o /= 2) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
        a.w += __shfl_xor_sync(0xffffffffu, a.w, o);
    }
    a.m = most;
    return a;
}

// What a row's statistics give.
struct RowResult {
    bool nothing;      // no logit above -infinity
    float log_s, base, entropy, scale;
    __device__ __forceinline__ RowResult(const Stats& all, float scale_) {
        nothing = all.s == 0.f;
        log_s = nothing ? 0.f : logf(all.s);
        base = nothing ? 0.f : all.m;
        entropy = nothing ? 0.f : log_s - 0.69314718f * (all.w / all.s);
        scale = scale_;
    }
    __device__ __forceinline__ float logprob(float z) const {      // (by halves: the two ends of the range are further apart than it is long)
        return nothing ? -INFINITY : 2.f * (scale * (0.5f * z - 0.5f * base)) - log_s;
    }
    __device__ __forceinline__ float lse() const { return nothing ? -INFINITY : fmaf(scale, base, log_s); }
};
// gradient = e (a + b d) with e = 2^d, d = log2(e) scale (z - M), less (distillation) or plus what the given tokens get.
template <bool kB>
struct Gradient {
    float a, b, c, base;
    __device__ __forceinline__ float one(float z) const {
        const float d = max_nan((z - base) * c, kLeast);
        return exp2_of(d) * (kB ? fmaf(b, d, a) : a);
    }
    template <typename T, bool kClamp>
    __device__ __forceinline__ void piece(uint4 raw, F2 (&x)[Logits<T>::kN / 2]) const {
        const F2 a2 = f2(a, a), b2 = f2(b, b), base2 = f2(-base, -base), c2 = f2(c, c);
        Logits<T>::get(kClamp || !kB ? raw : Logits<T>::raised(raw), x);
#pragma unroll
        for (int e = 0; e < Logits<T>::kN / 2; ++e) {
            F2 d;
            const F2 y = powers<kClamp>(x[e], base2, c2, &d);
            x[e] = mul2(y, kB ? fma2(b2, d, a2) : a2);
        }
    }
};
template <typename T>
__device__ __forceinline__ void store_piece(T* to, bool whole, uint4 v) {
    if (whole) {
        *reinterpret_cast<uint4*>(to) = v;
    } else {
#pragma unroll
        for (int e = 0; e < Logits<T>::kN; ++e) Logits<T>::put(to + e, Logits<T>::element(v, e));
    }
}

// The largest elements of a row or part, by kThreads threads.  The largest of each of kKeys shares of the pieces are known (keys: order_of, of bf16 logits its upper half;
// 0: an empty share); the k-th of those is a bound that at least k elements reach, found bit by bit by each warp for itself.  With k up to three quarters of the shares few more
// do (with more the bound is near the least of their largest, and 0 where there are not as many); all are in shares that reach it, which are gone through again, and are ranked
// against one another.  Where too many are equal to the bound, those above it and the first k that equal it are; where that is not enough (too many above it, or NaN among the
// largest) they are found one after the other.
//   piece(i): piece i of `pieces`; element e of it is the row's place0 + i kN + e.   piece_of(share, j): the share's j-th piece, j < each (`pieces` or more: none).
//   beside(j), j < 16: an element outside the pieces, its place in *place, or false.
//   use: 0 and 1 in turn, whose counters are zero.  meet(): a barrier of the kThreads threads.  rank_of(key, rank) is called once for each of the k largest, by some thread.
template <typename T> using ShareKey = std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>;
template <typename T>
__device__ __forceinline__ ShareKey<T> share_key(bool any, float v) { return any ? static_cast<ShareKey<T>>(order_of(v) >> (sizeof(T) == 2 ? 16 : 0)) : ShareKey<T>(0); }
template <typename T>
__device__ __forceinline__ uint32_t largest_of(uint4 keys) {
    if constexpr (sizeof(T) == 4) return max(max(keys.x, keys.y), max(keys.z, keys.w));
    const uint32_t two = __vmaxu2(__vmaxu2(keys.x, keys.y), __vmaxu2(keys.z, keys.w));
    return max(two >> 16, two & 0xffffu);
}
template <typename T, int kKeys, int kThreads, typename Piece, typename PieceOf, typename Beside, typename Meet, typename RankOf>
__device__ __forceinline__ void largest(Largest& sh, int use, const ShareKey<T>* keys, int t, int k, int pieces, int place0, int elements, int each, const Piece& piece,
                                        const PieceOf& piece_of, const Beside& beside, const Meet& meet, const RankOf& rank_of) {
    constexpr int kN = Logits<T>::kN, kBits = sizeof(T) == 2 ? 16 : 32, kShift = 32 - kBits, kWarps = kThreads / 32;
    constexpr bool kEight = kKeys * sizeof(ShareKey<T>) >= 512;      // (each lane 16 bytes of keys at least)
    const int lane = t & 31, warp = t >> 5;
    int &count = sh.counts[use][0], &owners_count = sh.counts[use][1];
    uint32_t bound = 0;
    if (k <= 32) {      // among the largest of 32 groups of shares: a bound that is a little lower and found in a third of the time
        uint32_t most = 0;
        if constexpr (kEight) {
            constexpr int kPieces = kKeys * static_cast<int>(sizeof(ShareKey<T>)) / 16;
#pragma unroll 4
            for (int j = lane; j < kPieces; j += 32) most = max(most, largest_of<T>(reinterpret_cast<const uint4*>(keys)[j]));
        } else {
#pragma unroll
            for (int j = lane; j < kKeys; j += 32) most = max(most, static_cast<uint32_t>(keys[j]));
        }
        // (the bits that all groups have are the bound's)
        const uint32_t same = ~(__reduce_or_sync(0xffffffffu, most) ^ __reduce_and_sync(0xffffffffu, most));
        const int differ = 31 - __clz(~same);      // the first bit that they do not
        if (differ < 31) bound = most >> (differ + 1) << (differ + 1);
#pragma unroll 1
        for (int b = differ; b >= 0; --b) {
            const uint32_t c = bound | (1u << b);
            if (__popc(__ballot_sync(0xffffffffu, most >= c)) >= k) bound = c;
        }
    } else {
        // among 256 groups at most, eight of a lane
        constexpr int kGroups = kKeys > 256 ? 8 : kKeys / 32;
        uint32_t mine[kGroups];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) mine[g] = kKeys > 256 ? largest_of<T>(reinterpret_cast<const uint4*>(keys)[lane + 32 * g]) : static_cast<uint32_t>(keys[lane + 32 * g]);
#pragma unroll 1
        for (int b = kBits - 1; b >= 0; --b) {
            const uint32_t c = bound | (1u << b);
            int n = 0;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) n += mine[g] >= c;
            if (__reduce_add_sync(0xffffffffu, n) >= k) bound = c;
        }
    }
    auto keep = [&](float v, int place) {
        const int at = atomicAdd(&count, 1);
        if (at < kCollected) sh.candidates[at] = key_of(v, place);
    };
    // elements from the order `least` on, into an empty list
    auto collect = [&](uint32_t least, bool empty) {
        if (!empty) {
            meet();
            if (t == 0) count = owners_count = 0;
            meet();
        }
        auto go_through = [&](uint4 w, int at) {
            const uint4 one[1] = {w};
            if (least != 0 && (order_of(Logits<T>::largest(one)) >> kShift) < least) return;
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                const float x = Logits<T>::element(w, e);
                if ((order_of(x) >> kShift) >= least) keep(x, place0 + at * kN + e);
            }
        };
        float v;
        int place;
        if (t < 16 && beside(t, &v, &place) && (order_of(v) >> kShift) >= least) keep(v, place);
        auto owner = [&](uint32_t key, int i) {
            if (key != 0 && key >= least) {
                const int at = atomicAdd(&owners_count, 1);
                if (at < kOwners) sh.owners[at] = static_cast<uint16_t>(i);
            }
        };
        if constexpr (kKeys * sizeof(ShareKey<T>) == kThreads * 16) {      // (16 bytes of keys a thread)
            constexpr int kEach = 16 / sizeof(ShareKey<T>), kWord = kEach / 4;
            const uint4 w = reinterpret_cast<const uint4*>(keys)[t];
            const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < kEach; ++j) owner(kWord == 2 ? (j & 1 ? words[j / 2] >> 16 : words[j / 2] & 0xffffu) : words[j / kWord], t * kEach + j);
        } else {
#pragma unroll
            for (int i = t; i < kKeys; i += kThreads) owner(keys[i], i);
        }
        meet();
        const int owners = owners_count > kOwners ? 0 : owners_count;
        if (owners_count > kOwners && t == 0) count = kCollected + 1;
        // (all threads go through all of their pieces, from memory two at a time)
        const int items = owners * each;
        constexpr int kAhead = kKeys == kThreads ? 1 : 2;
        for (int i0 = t; i0 < items; i0 += kAhead * kThreads) {
            uint4 w[kAhead];
            int at[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int item = i0 + a * kThreads, owner = item / each;
                at[a] = item < items ? piece_of(sh.owners[owner], item - owner * each) : pieces;
                w[a] = make_uint4(0, 0, 0, 0);
                if (at[a] < pieces) w[a] = piece(at[a]);
            }
#pragma unroll
            for (int a = 0; a < kAhead; ++a)
                if (at[a] < pieces) go_through(w[a], at[a]);
        }
        meet();
    };
    collect(bound, true);
    int n = count;
    if (n > kCollected && bound != 0xffffffffu >> kShift) {
        collect(bound + 1, false);
        const int above = count;
        if (above + k <= kCollected) {
            // the first k that equal the bound, in the order of their places: elements before the pieces, pieces, those behind
            int found = 0;      // (the same in all threads)
            auto these = [&](int mine, auto put) {      // the threads' numbers of such elements, in order
                int before = mine;
#pragma unroll
                for (int o = 1; o < 32; o *= 2) {
                    const int v = __shfl_up_sync(0xffffffffu, before, o);
                    if (lane >= o) before += v;
                }
                if (lane == 31) sh.warps[warp] = before;
                meet();
                int total = 0;
                before -= mine;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const int v = sh.warps[w];
                    if (w < warp) before += v;
                    total += v;
                }
                put(found + before);
                found += total;
                meet();
            };
            auto equal = [&](float x) { return (order_of(x) >> kShift) == bound; };
            auto side = [&](bool behind) {
                float v = 0.f;
                int place = 0;
                const bool mine = t < 16 && beside(t, &v, &place) && (place >= place0) == behind && equal(v);
                these(mine, [&](int at) { if (mine && at < k) sh.candidates[above + at] = key_of(v, place); });
            };
            side(false);
            for (int i0 = 0; i0 < pieces && found < k; i0 += kThreads) {
                const int i = i0 + t;
                uint4 v = make_uint4(0, 0, 0, 0);
                uint32_t mask = 0;
                if (i < pieces) {
                    v = piece(i);
#pragma unroll
                    for (int e = 0; e < kN; ++e) mask |= equal(Logits<T>::element(v, e)) ? 1u << e : 0u;
                }
                these(__popc(mask), [&](int at) {
#pragma unroll
                    for (int e = 0; e < kN; ++e)
                        if (mask >> e & 1) {
                            if (at < k) sh.candidates[above + at] = key_of(Logits<T>::element(v, e), place0 + i * kN + e);
                            ++at;
                        }
                });
            }
            if (found < k) side(true);
            n = above + min(found, k);
        }
    }
    if (n <= kCollected && n >= min(k, elements)) {
        for (int i = t; i < n; i += kThreads) {
            const uint64_t key = sh.candidates[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += sh.candidates[j] > key;
            if (rank < k) rank_of(key, rank);
        }
        return;
    }
    uint64_t last = ~0ull;
    for (int r = 0; r < k; ++r) {
        uint64_t best = 0;
        auto next = [&](float v, int place) {
            const uint64_t key = key_of(v, place);
            if (key < last && key > best) best = key;
        };
        float x;
        int place;
        if (t < 16 && beside(t, &x, &place)) next(x, place);
#pragma unroll 2
        for (int i = t; i < pieces; i += kThreads) {
            const uint4 v = piece(i);
#pragma unroll
            for (int e = 0; e < kN; ++e) next(Logits<T>::element(v, e), place0 + i * kN + e);
        }
#pragma unroll
        for (int o = 16; o > 0; o /= 2) {
            const uint64_t other = __shfl_xor_sync(0xffffffffu, best, o);
            best = other > best ? other : best;
        }
        meet();
        if (lane == 0) sh.best[warp] = best;
        meet();
#pragma unroll
        for (int i = 0; i < kWarps; ++i) best = sh.best[i] > best ? sh.best[i] : best;
        if (t == 0 && best != 0) rank_of(best, r);
        last = best;
    }
}

// A lane's entries of a teacher's row: tokens (-1: none) and logits.
struct Entries {
    int id[kMaxTeacher / 32];
    float v[kMaxTeacher / 32];
    __device__ __forceinline__ void load(const VocabParams& p, int64_t r, int lane) {
        const int64_t* const ids = p.ids + r * p.k;
        const float* const teacher = p.teacher + r * p.k;
#pragma unroll
        for (int j = 0; j < kMaxTeacher / 32; ++j)
            if (lane + 32 * j < p.k) {
                const int64_t i = ids[lane + 32 * j];
                id[j] = i >= 0 && i < p.vocab ? static_cast<int>(i) : -1;
                v[j] = teacher[lane + 32 * j];
            }
    }
};
// The teacher's probabilities of a row, by one warp: th, and their sum.
template <typename T>
__device__ __forceinline__ float teacher_of(TeacherShared& th, const VocabParams& p, const Entries& e, int64_t r, const T* row, int lane) {
    float z[kMaxTeacher / 32], most = -INFINITY;
#pragma unroll
    for (int j = 0; j < kMaxTeacher / 32; ++j) {
        z[j] = 0.f;
        if (lane + 32 * j < p.k && e.id[j] >= 0) z[j] = Logits<T>::one(row + e.id[j]);
    }
#pragma unroll
    for (int j = 0; j < kMaxTeacher / 32; ++j)
        if (lane + 32 * j < p.k) {
            const float v = e.id[j] >= 0 ? e.v[j] : -INFINITY;
            th.id[lane + 32 * j] = e.id[j];
            th.logq[lane + 32 * j] = v;
            most = fmaxf(most, v);
        }
    if (lane < (-p.k & 3)) th.id[p.k + lane] = -1;
    // log q = scale (teacher - top) - less, by differences of logits that are near one another
    float top = 0.f, less;
    if (p.teacher_lse) {
        less = p.teacher_lse[r];
    } else {
        top = most;
#pragma unroll
        for (int o = 16; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        float sum = 0.f;      // (a NaN comes through here)
        for (int j = lane; j < p.k; j += 32) sum += th.logq[j] == -INFINITY ? 0.f : expf(p.scale * (th.logq[j] - top));
#pragma unroll
        for (int o = 16; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        less = logf(sum);
    }
    float q_sum = 0.f;
    for (int j = lane; j < p.k; j += 32) {
        const float logq = fmaf(p.scale, th.logq[j] - top, -less), q = th.logq[j] == -INFINITY ? 0.f : expf(logq);
        th.q[j] = q;
        th.logq[j] = logq;
        q_sum += q;
    }
#pragma unroll
    for (int j = 0; j < kMaxTeacher / 32; ++j)
        if (lane + 32 * j < p.k) th.z[lane + 32 * j] = z[j];
#pragma unroll
    for (int o = 16; o > 0; o /= 2) q_sum += __shfl_xor_sync(0xffffffffu, q_sum, o);
    return q_sum;
}
// ... and what they make of the row's loss, by one warp.
__device__ __forceinline__ float loss_of(const TeacherShared& th, const RowResult& res, int k, int lane) {
    float sum = 0.f;
    for (int j = lane; j < k; j += 32) {
        const float q = th.q[j];
        sum += q == 0.f ? 0.f : q * (th.logq[j] - res.logprob(th.z[j]));
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return sum;
}
// Of the entries with token j's id: their probabilities together, and whether j is the first of them.  (Four at a time: nearly always none of them is.)
__device__ __forceinline__ bool first_of_token(const TeacherShared& th, int k, int j, float* q) {
    bool first = true;
    const int id = th.id[j];
    *q = 0.f;
#pragma unroll 4
    for (int l = 0; l < k; l += 4) {
        const int4 v = *reinterpret_cast<const int4*>(th.id + l);
        if (v.x != id && v.y != id && v.z != id && v.w != id) continue;
        const int of[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (of[e] == id) {
                first = first && l + e >= j;
                *q += th.q[l + e];
            }
    }
    return first;
}
template <bool kDistill>
__device__ __forceinline__ Gradient<!kDistill> gradient_of(const VocabParams& p, const Stats& all, const RowResult& res, float c, float upstream, float dentropy, float q_sum,
                                                           float* taken) {
    Gradient<!kDistill> g = {0.f, 0.f, c, res.base};
    *taken = 0.f;
    if (res.nothing) return g;
    *taken = p.scale * upstream;
    if constexpr (kDistill) {
        g.a = *taken * q_sum / all.s;
    } else {
        g.a = -p.scale * (upstream + dentropy * (res.entropy - res.log_s)) / all.s;
        g.b = -p.scale * dentropy * 0.69314718f / all.s;
    }
    return g;
}

// Distillation has a warp more, which looks up the teacher's tokens meanwhile.
template <int kMode, int kThreads> constexpr int kVocabThreads = kThreads + (kMode == kDistillFwd || kMode == kDistillBwd ? 32 : 0);
template <typename T, int kMode, int kThreads>
__global__ void __launch_bounds__(kVocabThreads<kMode, kThreads>) vocab_kernel(const VocabParams p) {
    constexpr int kN = Logits<T>::kN, kChunk = kDeep * kThreads, kWarps = kThreads / 32;
    constexpr bool kDistill = kMode == kDistillFwd || kMode == kDistillBwd, kBwd = kMode == kLogprobsBwd || kMode == kDistillBwd;
    extern __shared__ __align__(16) unsigned char vocab_smem[];
    VocabRow<kMode>& sh = *reinterpret_cast<VocabRow<kMode>*>(vocab_smem);
    unsigned char* const data = vocab_smem + kVocabHead<kMode>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = kDistill && warp == kWarps ? 1 << 28 : static_cast<int>(threadIdx.x);      // (no share of the row)
    const int part = p.parts > 1 ? static_cast<int>(blockIdx.x) % p.parts : 0;
    const int64_t r = blockIdx.x / static_cast<unsigned>(p.parts);
    const T* const row = static_cast<const T*>(p.logits) + r * p.ld;
    const Part<T> pt(row, p.vocab, part, p.parts);
    const int tail0 = pt.head + pt.pieces * kN, place0 = pt.head + pt.first * kN, chunks = (pt.count + kChunk - 1) / kChunk;
    volatile uint32_t* const abort_flag = &sh.abort;
    if (t == 0) {
        for (int i = 0; i < chunks; ++i) tc::mbar_init(smem_at(&sh.bars[i]), 1);
        sh.abort = 0;
        tc::fence_barrier_init();
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (t == 0) {
        const unsigned char* const from = reinterpret_cast<const unsigned char*>(row + place0);
        for (int i = 0; i < chunks; ++i) bulk_copy(smem_at(data) + i * kChunk * 16, from + static_cast<int64_t>(i) * kChunk * 16, min(kChunk, pt.count - i * kChunk) * 16, smem_at(&sh.bars[i]));
    }
    __syncthreads();
    // An element beside the pieces: eight threads' before them (first part), eight threads' behind them (last part).
    const int extra = t < 8 ? t : tail0 + t - 8;
    const bool has_extra = t < 16 && (t < 8 ? part == 0 && t < pt.head : part == p.parts - 1 && extra < p.vocab);
    float beside = -INFINITY;
    if (has_extra) beside = Logits<T>::one(row + extra);
    // The given token, or the teacher's (by the last warp).
    int64_t id = -1;
    float z_id = 0.f, upstream = 0.f, dentropy = 0.f;
    if constexpr (!kDistill) {
        if (p.ids) id = p.ids[r];
        if (id < 0 || id >= p.vocab) id = -1;
        else z_id = Logits<T>::one(row + id);      // (before the barrier behind which a gradient may be written over it)
        if (kBwd && p.dentropy) dentropy = p.dentropy[r];
        if (kBwd && p.dlogprobs && id >= 0) upstream = p.dlogprobs[r];
    } else {
        if (kBwd) upstream = p.dloss[r];
        if (warp == kWarps) {
            Entries entries;
            entries.load(p, r, lane);
            const float q_sum = teacher_of<T>(sh.own, p, entries, r, row, lane);
            if (lane == 0) sh.part.pad = q_sum;
        }
    }

    // statistics
    const float c = p.scale * 1.44269504f;
    Sums sums;
    sums.start();
    for (int ck = 0; ck < (t < kThreads ? chunks : 0); ++ck) {
        tc::mbar_wait(smem_at(&sh.bars[ck]), 0, abort_flag, p.status);
        const int i0 = ck * kChunk + t;
        uint4 v[kDeep];
#pragma unroll
        for (int j = 0; j < kDeep; ++j) {
            v[j] = make_uint4(Logits<T>::kNone, Logits<T>::kNone, Logits<T>::kNone, Logits<T>::kNone);
            if (i0 + j * kThreads < pt.count) v[j] = *reinterpret_cast<const uint4*>(data + (i0 + j * kThreads) * 16);
        }
        sums.template add<T, !kDistill>(v, c);
    }
    const float piece_most = sums.m;
    if (has_extra) sums.add_one(beside, c);
    if (t < 16) sh.extra[t] = beside;
    if constexpr (kMode == kLogprobsFwd) {
        reinterpret_cast<ShareKey<T>*>(sh.own.keys)[t] = share_key<T>(t < pt.count, piece_most);
        for (int i = t; i < p.top; i += kThreads) sh.own.list[i] = 0;
        if (t == 0) sh.own.largest.counts[0][0] = sh.own.largest.counts[0][1] = 0;
    }

    // the block's, then the row's
    Stats all = warp_stats(sums, c);
    if (lane == 0) sh.warp[warp] = all;
    __syncthreads();
    if constexpr (kWarps > 1 || kDistill) all = block_stats<kWarps>(sh.warp, c);
    const float q_sum = kDistill ? sh.part.pad : 0.f;
    if constexpr (kMode == kLogprobsFwd) {
        if (p.top > 0) {
            const int elements = pt.count * kN + (part == 0 ? pt.head : 0) + (part == p.parts - 1 ? p.vocab - tail0 : 0);
            largest<T, kThreads, kThreads>(sh.own.largest, 0, reinterpret_cast<const ShareKey<T>*>(sh.own.keys), t, p.top, pt.count, place0, elements,
                                           (pt.count + kThreads - 1) / kThreads, [&](int i) { return *reinterpret_cast<const uint4*>(data + i * 16); },
                                           [&](int share, int j) { return share + j * kThreads; },
                                           [&](int, float* v, int* place) {
                                               *v = beside;
                                               *place = extra;
                                               return has_extra;
                                           },
                                           [] { __syncthreads(); }, [&](uint64_t key, int rank) { sh.own.list[rank] = key; });
            __syncthreads();
        }
    }
    if (p.parts > 1) {
        if (t == 0) { sh.part.m = all.m; sh.part.s = all.s; sh.part.w = all.w; }
        cluster_arrive();
        cluster_wait();
        const uint32_t at = smem_at(&sh.part);
        auto of = [&](int i) {
            Stats s;
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(s.m), "=f"(s.s), "=f"(s.w), "=f"(s.pad) : "r"(of_part(at, i)) : "memory");
            return s;
        };
        all = of(0);
        for (int i = 1; i < p.parts; ++i) all = together(all, of(i), c);
        if (kMode != kLogprobsFwd) cluster_arrive();      // (ahead of the gradient, for whose stores it would wait)
    }
    const RowResult res(all, p.scale);

    const bool ok = *abort_flag == 0;      // (else this part's copies did not come)
    if (!ok && t == 0) wait_for_copies(smem_at(sh.bars), 0, static_cast<uint32_t>(chunks), kMaxChunks);
    if (part == 0 && ok) {
        if constexpr (!kDistill) {
            if (t == 0) {
                if (p.logprobs) p.logprobs[r] = id >= 0 ? res.logprob(z_id) : 0.f;
                if (p.entropy) p.entropy[r] = res.entropy;
                if (kMode == kLogprobsFwd && p.lse) p.lse[r] = res.lse();
            }
        } else if (p.loss && warp == 0) {
            const float loss = loss_of(sh.own, res, p.k, lane);
            if (lane == 0) p.loss[r] = loss;
        }
        if constexpr (kMode == kLogprobsFwd) {
            const int n = p.parts * p.top;
            if (p.parts > 1 && n > 0) {
                for (int i = t; i < n; i += kThreads) {
                    const int from = i / p.top;
                    const uint32_t at = of_part(smem_at(sh.own.list + (i - from * p.top)), from);
                    uint64_t key;
                    asm volatile("ld.shared::cluster.b64 %0, [%1];" : "=l"(key) : "r"(at) : "memory");
                    sh.own.parts[i] = key;
                }
                __syncthreads();
            }
            const uint64_t* const keys = p.parts > 1 ? sh.own.parts : sh.own.list;
            for (int i = t; i < n; i += kThreads) {
                const uint64_t key = keys[i];
                int rank = i;
                if (p.parts > 1) {
                    rank = 0;
                    for (int j = 0; j < n; ++j) rank += keys[j] > key;
                }
                if (key != 0 && rank < p.top) {
                    if (p.top_logprobs) p.top_logprobs[r * p.top + rank] = res.logprob(value_of(static_cast<uint32_t>(key >> 32)));
                    if (p.top_ids) p.top_ids[r * p.top + rank] = static_cast<uint32_t>(~key);
                }
            }
        }
    }

    if (kBwd && ok) {
        float taken;
        const auto g = gradient_of<kDistill>(p, all, res, c, upstream, dentropy, q_sum, &taken);
        T* const out = static_cast<T*>(p.dlogits) + r * p.lddl;
        T* const pieces = out + place0;
        const bool whole = (reinterpret_cast<uintptr_t>(pieces) & 15) == 0;
        auto write = [&](auto clamp) {
#pragma unroll 2
            for (int i = t; i < pt.count; i += kThreads) {
                F2 x[kN / 2];
                g.template piece<T, decltype(clamp)::value>(*reinterpret_cast<const uint4*>(data + i * 16), x);
                store_piece(pieces + static_cast<int64_t>(i) * kN, whole, Logits<T>::pack(x));
            }
        };
        if (kDistill || (fabsf(res.base) <= kFar && fabsf(g.b) * (kFarthest * c) <= 1e38f)) write(std::false_type());
        else write(std::true_type());
        if (has_extra) Logits<T>::put(out + extra, g.one(beside));
        __syncthreads();      // the given tokens' elements, written anew behind the others
        auto logit = [&](int i, float* z) {      // of this part
            if (i < pt.head || i >= tail0) {
                if (part != (i < pt.head ? 0 : p.parts - 1)) return false;
                *z = sh.extra[i < pt.head ? i : 8 + i - tail0];
                return true;
            }
            const int at = i - place0;
            if (at < 0 || at >= pt.count * kN) return false;
            *z = Logits<T>::one(reinterpret_cast<const T*>(data) + at);
            return true;
        };
        if (!res.nothing) {
            float z;
            if constexpr (kDistill) {
                for (int j = threadIdx.x; j < p.k; j += kThreads + 32) {
                    float q;
                    if (sh.own.id[j] < 0 || !logit(sh.own.id[j], &z) || !first_of_token(sh.own, p.k, j, &q)) continue;
                    Logits<T>::put(out + sh.own.id[j], g.one(z) - taken * q);
                }
            } else if (t == 0 && id >= 0 && logit(static_cast<int>(id), &z)) {
                Logits<T>::put(out + id, g.one(z) + taken);
            }
        }
    }
    if (p.parts > 1) {      // no block leaves while another may read its numbers
        if (kMode == kLogprobsFwd) cluster_arrive();
        cluster_wait();
    }
}

// Eight warps go through rows; one asks for chunks, one looks up a row's given tokens while the row before is in work.  (Sixteen warps, two blocks an SM: 4096 x 32001
// forward 104 us; eight and three: 57.  The largest elements by a warp of their own: 2048 x 131072 with 20 of them 275 us, for want of issue slots.)
constexpr int kStreamThreads = 256, kStreamStages = 4, kStreamBlocks = 3, kStreamChunk = kDeep * kStreamThreads;
// Shares of a row that its largest elements are looked for in: a thread's of each eighth (fp32: quarter) of the chunks.
template <typename T> constexpr int kShares = sizeof(T) == 2 ? 8 : 4;
constexpr int kStreamKeyWords = kStreamThreads * 4;
constexpr int kStreamAll = kStreamThreads + 64;
struct StreamShared {
    uint64_t full[kStreamStages], empty[kStreamStages], given_full[2], given_empty[2], stats_full[2], stats_empty[2];
    Stats warp[2][kStreamThreads / 32];            // of alternate rows, as what follows in twos
    union {
        struct {
            alignas(16) uint32_t keys[kStreamKeyWords];      // [shares of chunks][threads]: read for the last time before the last barrier of a row
            Largest largest;
        };
        TeacherShared th[2];     // (distillation)
    };
    int id[2];
    float z[2];
    uint32_t abort;
};

template <typename T, int kMode>
__global__ void __launch_bounds__(kStreamAll, kStreamBlocks) vocab_stream_kernel(const VocabParams p) {
    constexpr bool kDistill = kMode == kDistillFwd;
    constexpr int kN = Logits<T>::kN, kThreads = kStreamThreads, kStages = kStreamStages, kWarps = kThreads / 32;
    extern __shared__ __align__(16) unsigned char vocab_smem[];
    StreamShared& sh = *reinterpret_cast<StreamShared*>(vocab_smem);
    unsigned char* const data = vocab_smem + (sizeof(StreamShared) + 15) / 16 * 16;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    volatile uint32_t* const abort_flag = &sh.abort;
    const uint32_t full0 = smem_at(sh.full), empty0 = smem_at(sh.empty);
    if (t == 0) {
        for (int s = 0; s < kStages; ++s) {
            tc::mbar_init(full0 + 8 * s, 1);
            tc::mbar_init(empty0 + 8 * s, kWarps);
        }
        for (int b = 0; b < 2; ++b) {
            tc::mbar_init(smem_at(&sh.given_full[b]), 1);
            tc::mbar_init(smem_at(&sh.given_empty[b]), 1);
            tc::mbar_init(smem_at(&sh.stats_full[b]), kWarps);
            tc::mbar_init(smem_at(&sh.stats_empty[b]), 1);
        }
        sh.abort = 0;
        if (!kDistill) sh.largest.counts[0][0] = sh.largest.counts[0][1] = sh.largest.counts[1][0] = sh.largest.counts[1][1] = 0;
        tc::fence_barrier_init();
    }
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    auto meet = [] { asm volatile("bar.sync 1, %0;" ::"n"(kStreamThreads) : "memory"); };
    auto meet_any = [](bool mine) {      // whether any of them says so: the same answer for all
        uint32_t any;
        asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.or.pred q, 1, %2, p;\n selp.u32 %0, 1, 0, q;\n}"
                     : "=r"(any) : "r"(static_cast<uint32_t>(mine)), "n"(kStreamThreads) : "memory");
        return any != 0;
    };
    auto row_of = [&](int64_t r) { return static_cast<const T*>(p.logits) + r * p.ld; };
    const float c = p.scale * 1.44269504f;
    uint32_t b = 0, b_ph = 0;      // which of the two rows
    auto next_row = [&]() {
        b ^= 1u;
        if (b == 0) b_ph ^= 1u;
    };

    if (warp == kWarps) {
        // ---------------------------------------------------------------- chunks
        if (lane == 0) {
            uint32_t s = 0, ph = 1, fills = 0;
            bool ok = true;
            for (int64_t r = blockIdx.x; r < p.tokens && ok; r += gridDim.x) {
                const Part<T> pt(row_of(r), p.vocab, 0, 1);
                const unsigned char* const from = reinterpret_cast<const unsigned char*>(row_of(r) + pt.head);
                const int chunks = (pt.count + kStreamChunk - 1) / kStreamChunk;
                for (int ck = 0; ck < chunks; ++ck) {
                    ok = tc::mbar_wait(empty0 + 8 * s, ph, abort_flag, p.status);
                    if (!ok) break;
                    bulk_copy(smem_at(data) + s * kStreamChunk * 16, from + static_cast<int64_t>(ck) * kStreamChunk * 16, min(kStreamChunk, pt.count - ck * kStreamChunk) * 16,
                              full0 + 8 * s);
                    ++fills;
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
            }
            if (!ok) wait_for_copies(full0, fills > kStages ? fills - kStages : 0, fills, kStages);
        }
        return;
    }
    if (warp == kWarps + 1) {
        // ---------------------------------------------------------------- given tokens
        Entries entries;      // (of the next row: what they refer to is then looked up at once)
        if (kDistill && blockIdx.x < p.tokens) entries.load(p, blockIdx.x, lane);
        for (int64_t r = blockIdx.x; r < p.tokens; r += gridDim.x, next_row()) {
            if (!tc::mbar_wait_warp(smem_at(&sh.given_empty[b]), b_ph ^ 1u, abort_flag, p.status)) break;
            const T* const row = row_of(r);
            if constexpr (kDistill) {
                const Entries now = entries;
                if (r + gridDim.x < p.tokens) entries.load(p, r + gridDim.x, lane);
                teacher_of<T>(sh.th[b], p, now, r, row, lane);
            } else if (lane == 0) {
                const int64_t id = p.ids ? p.ids[r] : -1;
                const bool given = id >= 0 && id < p.vocab;
                sh.id[b] = given ? static_cast<int>(id) : -1;
                sh.z[b] = given ? Logits<T>::one(row + id) : 0.f;
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(smem_at(&sh.given_full[b]));
        }
        return;
    }
    // A row's results, by one warp.
    auto results = [&](int64_t r, const RowResult& res) {
        if constexpr (!kDistill) {
            if (lane == 0) {
                if (p.logprobs) p.logprobs[r] = sh.id[b] >= 0 ? res.logprob(sh.z[b]) : 0.f;
                if (p.entropy) p.entropy[r] = res.entropy;
                if (!kDistill && p.lse) p.lse[r] = res.lse();
            }
        } else if (p.loss) {
            const float loss = loss_of(sh.th[b], res, p.k, lane);
            if (lane == 0) p.loss[r] = loss;
        }
    };
    // -------------------------------------------------------------------- rows
    uint32_t s = 0, ph = 0;      // stage
    bool ok = true;
    auto next_stage = [&]() {      // this one has been read
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(empty0 + 8 * s);
        if (++s == kStages) { s = 0; ph ^= 1u; }
    };
    for (int64_t r = blockIdx.x; r < p.tokens && ok; r += gridDim.x, next_row()) {
        const T* const row = row_of(r);
        const Part<T> pt(row, p.vocab, 0, 1);
        const int tail0 = pt.head + pt.pieces * kN, chunks = (pt.count + kStreamChunk - 1) / kStreamChunk;
        const int extra = t < 8 ? t : tail0 + t - 8;
        const bool has_extra = t < 16 && (t < 8 ? t < pt.head : extra < p.vocab);
        float beside = -INFINITY;
        if (has_extra) beside = Logits<T>::one(row + extra);
        Sums sums;
        sums.start();
        // (the largest of a share of the chunks)
        const bool top = kMode == kLogprobsFwd && p.top > 0;
        const int per = (chunks + kShares<T> - 1) / kShares<T>;
        int share = 0, until = per;
        float share_most = -INFINITY;
        for (int ck = 0; ck < chunks && ok; ++ck) {
            // (a warp gives up as a whole, and no warp but with all others of the block where they meet)
            ok = __all_sync(0xffffffffu, tc::mbar_wait(full0 + 8 * s, ph, abort_flag, p.status)) != 0;
            if (!ok) break;
            const uint4* const in = reinterpret_cast<const uint4*>(data + s * kStreamChunk * 16) + t;
            const int left = pt.count - ck * kStreamChunk - t;
            uint4 v[kDeep];
#pragma unroll
            for (int j = 0; j < kDeep; ++j) {
                v[j] = make_uint4(Logits<T>::kNone, Logits<T>::kNone, Logits<T>::kNone, Logits<T>::kNone);
                if (j * kThreads < left) v[j] = in[j * kThreads];
            }
            next_stage();
            const float most = sums.template add<T, !kDistill>(v, c);
            if (top) {
                share_most = fmaxf(share_most, most);
                if (ck + 1 == until || ck + 1 == chunks) {
                    reinterpret_cast<ShareKey<T>*>(sh.keys)[share * kThreads + t] = share_key<T>(share * per * kStreamChunk + t < pt.count, share_most);
                    ++share;
                    until += per;
                    share_most = -INFINITY;
                }
            }
        }
        if (top)
            for (; share < kShares<T>; ++share) reinterpret_cast<ShareKey<T>*>(sh.keys)[share * kThreads + t] = 0;
        if (has_extra) sums.add_one(beside, c);
        Stats all = warp_stats(sums, c);
        // Where only the first warp goes on with the row, the others leave their statistics (once it has taken those of two rows ago) and go to the next.
        const bool alone = !top;
        if (alone) {
            if (warp != 0) ok = tc::mbar_wait_warp(smem_at(&sh.stats_empty[b]), b_ph ^ 1u, abort_flag, p.status) && ok;
            if (!ok) break;
            if (lane == 0) {
                sh.warp[b][warp] = all;
                tc::mbar_arrive(smem_at(&sh.stats_full[b]));
            }
            if (warp != 0) continue;
            ok = tc::mbar_wait_warp(smem_at(&sh.stats_full[b]), b_ph, abort_flag, p.status) && ok;
            ok = tc::mbar_wait_warp(smem_at(&sh.given_full[b]), b_ph, abort_flag, p.status) && ok;
            if (!ok) break;
            results(r, RowResult(block_stats<kWarps>(sh.warp[b], c), p.scale));
            __syncwarp();
            if (lane == 0) {
                tc::mbar_arrive(smem_at(&sh.given_empty[b]));
                tc::mbar_arrive(smem_at(&sh.stats_empty[b]));
            }
            continue;
        }
        if (lane == 0) sh.warp[b][warp] = all;
        ok = tc::mbar_wait_warp(smem_at(&sh.given_full[b]), b_ph, abort_flag, p.status) && ok;
        if (meet_any(!ok)) break;
        all = block_stats<kWarps>(sh.warp[b], c);
        const RowResult res(all, p.scale);
        if (warp == 0) results(r, res);
        if constexpr (kMode == kLogprobsFwd) {
            const uint4* const pieces = reinterpret_cast<const uint4*>(row + pt.head);
            if (t == 0) sh.largest.counts[b ^ 1u][0] = sh.largest.counts[b ^ 1u][1] = 0;      // (all are done with the row before)
            largest<T, kThreads * kShares<T>, kThreads>(sh.largest, static_cast<int>(b), reinterpret_cast<const ShareKey<T>*>(sh.keys), t, p.top, pt.count, pt.head, p.vocab, per * kDeep,
                                                        [&](int i) { return __ldg(pieces + i); },
                                                        [&](int share_of, int j) { return share_of / kThreads * per * kStreamChunk + share_of % kThreads + j * kThreads; },
                                                        [&](int, float* v, int* place) {
                                                            *v = beside;
                                                            *place = extra;
                                                            return has_extra;
                                                        },
                                                        meet,
                                                        [&](uint64_t key, int rank) {
                                                            if (p.top_logprobs) p.top_logprobs[r * p.top + rank] = res.logprob(value_of(static_cast<uint32_t>(key >> 32)));
                                                            if (p.top_ids) p.top_ids[r * p.top + rank] = static_cast<uint32_t>(~key);
                                                        });
        }
        __syncwarp();
        if (lane == 0 && warp == 0) tc::mbar_arrive(smem_at(&sh.given_empty[b]));
    }
}

struct VocabPlan {
    bool stream;
    int parts, threads;
    size_t part;      // bytes
};
// Forward, rows of more than 64 KB of which every SM has two or more stream (2048 x 131072: 92 us; as parts 147).  Others: parts of at most 64 KB; more of them, of 8 KB at
// least, while rows are too few for the SMs.  Short rows have small blocks, of which an SM holds more.  (All four operators add up rows of parts in the same order.)
// Short rows of which many alternatives are wanted have blocks of more threads than that, for more shares (2048 rows of 4000, 128 alternatives: 128 threads, one after the
// other, 898 us, 256 threads 45; 1000, 64: 32 threads 196, 128 threads 17; but 4000, 65: 22.6 and 31.9), unless all of a row can be ranked or there are fewer pieces than alternatives
// anyway (1000, 128, one after the other: 32 threads 378, 256 threads 508).
bool vocab_plan(int64_t tokens, int64_t vocab, int dtype, int top, VocabPlan* pl) {
    const int64_t bytes = vocab * static_cast<int64_t>(dtype_size(dtype));
    pl->stream = bytes > kPartBytes && tokens >= 2 * num_sms();
    pl->parts = 1;
    while (pl->parts < kMaxParts && ceil_div(bytes, pl->parts) > kPartBytes) pl->parts *= 2;
    while (pl->parts < kMaxParts && tokens * pl->parts < num_sms() && bytes / (2 * pl->parts) >= kPartBytesLeast) pl->parts *= 2;
    const int64_t part = ceil_div(ceil_div(bytes, 16), pl->parts) * 16;
    if (part > kPartBytesMost) return false;
    auto enough = [&](int threads) { return vocab <= kCollected || 4 * top <= 3 * threads || bytes / 16 < top; };
    pl->threads = part <= 2048 && enough(32) ? 32 : part <= 16384 && pl->parts == 1 && enough(128) ? 128 : 256;
    pl->part = static_cast<size_t>(part);
    return true;
}
constexpr size_t kStreamSmem = (sizeof(StreamShared) + 15) / 16 * 16 + static_cast<size_t>(kStreamStages) * kStreamChunk * 16;
static_assert(kStreamBlocks * (kStreamSmem + 1024) <= 228 * 1024, "");

template <typename T, int kMode>
int vocab_launch(const VocabParams& p, const VocabPlan& pl, cudaStream_t stream) {
    static std::atomic<uint64_t> done, stream_done;
    if constexpr (kMode == kLogprobsFwd || kMode == kDistillFwd) {
        if (pl.stream) {
            PF_CUDA(allow_dynamic_smem(reinterpret_cast<const void*>(vocab_stream_kernel<T, kMode>), kStreamSmem, stream_done));
            const int64_t blocks = std::min<int64_t>(p.tokens, kStreamBlocks * num_sms());
            PF_CUDA(launch_beside(vocab_stream_kernel<T, kMode>, dim3(static_cast<unsigned>(blocks)), kStreamAll, kStreamSmem, 1, stream, p));
            return PF_OK;
        }
    }
    void (*kernel)(VocabParams) = pl.threads == 32 ? vocab_kernel<T, kMode, 32> : pl.threads == 128 ? vocab_kernel<T, kMode, 128> : vocab_kernel<T, kMode, 256>;
    if (pl.threads == 256)
        PF_CUDA(allow_dynamic_smem(reinterpret_cast<const void*>(kernel), kVocabHead<kMode> + kPartBytesMost, done));
    PF_CUDA(launch_beside(kernel, dim3(static_cast<unsigned>(p.tokens * pl.parts)), pl.threads + kVocabThreads<kMode, 0>, kVocabHead<kMode> + pl.part, pl.parts, stream, p));
    return PF_OK;
}
template <int kMode>
int vocab_run(VocabParams& p, int64_t tokens, int64_t vocab, int dtype, double scale, cudaStream_t stream) {
    VocabPlan pl;
    if (!vocab_plan(tokens, vocab, dtype, p.top, &pl)) return PF_ERR_UNSUPPORTED;
    p.tokens = tokens;
    p.vocab = static_cast<int>(vocab);
    p.parts = pl.parts;
    p.status = device_status_ptr();
    p.scale = static_cast<float>(scale);
    return dtype == PF_BF16 ? vocab_launch<__nv_bfloat16, kMode>(p, pl, stream) : vocab_launch<float, kMode>(p, pl, stream);
}

template <typename T>
bool aligned_to(const T* p) { return reinterpret_cast<uintptr_t>(p) % sizeof(T) == 0; }
// What all four share.
int validate_vocab(const void* logits, int64_t ld, int64_t tokens, int64_t vocab, double scale, int dtype) {
    if (!valid_dtype(dtype) || tokens < 0 || vocab < 1 || ld < vocab || !(scale >= 1e-6) || !(scale <= 1e6)) return PF_ERR_INVALID_ARG;
    if ((tokens > 0 && !logits) || !elem_aligned(logits, dtype)) return PF_ERR_INVALID_ARG;
    if (tokens > (1LL << 27) || vocab > kMaxParts * kPartBytesMost / static_cast<int64_t>(dtype_size(dtype))) return PF_ERR_UNSUPPORTED;
    return PF_OK;
}
int validate_gradient(const void* dlogits, int64_t lddl, int64_t vocab, int dtype) {
    return !dlogits || lddl < vocab || !elem_aligned(dlogits, dtype) ? PF_ERR_INVALID_ARG : PF_OK;
}
int validate_teacher(const int64_t* ids, const float* teacher, const float* teacher_lse, int k) {
    if (k < 1 || !ids || !teacher || !aligned_to(ids) || !aligned_to(teacher) || !aligned_to(teacher_lse)) return PF_ERR_INVALID_ARG;
    return PF_OK;
}

}  // namespace
}  // namespace pf

using namespace pf;

extern "C" {

int pf_logprobs_fwd(const void* logits, int64_t ld, const int64_t* ids, double scale, float* logprobs, float* entropy, float* lse, int top,
                    float* top_logprobs, int64_t* top_ids, int64_t tokens, int64_t vocab, int dtype, void* cuda_stream) {
    const int st = validate_vocab(logits, ld, tokens, vocab, scale, dtype);
    if (st != PF_OK || tokens == 0) return st;
    if (!aligned_to(ids) || !aligned_to(logprobs) || !aligned_to(entropy) || !aligned_to(lse) || !aligned_to(top_logprobs) || !aligned_to(top_ids))
        return PF_ERR_INVALID_ARG;
    if (top < 0 || top > vocab || (top > 0) != (top_logprobs || top_ids) || (logprobs && !ids) ||
        (!logprobs && !entropy && !lse && top == 0))
        return PF_ERR_INVALID_ARG;
    if (top > kMaxTop) return PF_ERR_UNSUPPORTED;
    VocabParams p = {};
    p.logits = logits; p.ld = ld; p.ids = ids; p.logprobs = logprobs; p.entropy = entropy; p.lse = lse;
    p.top = top; p.top_logprobs = top_logprobs; p.top_ids = top_ids;
    return vocab_run<kLogprobsFwd>(p, tokens, vocab, dtype, scale, static_cast<cudaStream_t>(cuda_stream));
}

int pf_logprobs_bwd(const void* logits, int64_t ld, const int64_t* ids, double scale, const float* dlogprobs, const float* dentropy, void* dlogits,
                    int64_t lddl, float* logprobs, float* entropy, int64_t tokens, int64_t vocab, int dtype, void* cuda_stream) {
    const int st = validate_vocab(logits, ld, tokens, vocab, scale, dtype);
    if (st != PF_OK || tokens == 0) return st;
    if (validate_gradient(dlogits, lddl, vocab, dtype) != PF_OK || !aligned_to(ids) || !aligned_to(dlogprobs) || !aligned_to(dentropy) ||
        !aligned_to(logprobs) || !aligned_to(entropy))
        return PF_ERR_INVALID_ARG;
    if ((!dlogprobs && !dentropy) || ((dlogprobs || logprobs) && !ids)) return PF_ERR_INVALID_ARG;
    VocabParams p = {};
    p.logits = logits; p.ld = ld; p.ids = ids; p.dlogprobs = dlogprobs; p.dentropy = dentropy; p.dlogits = dlogits; p.lddl = lddl;
    p.logprobs = logprobs; p.entropy = entropy;
    return vocab_run<kLogprobsBwd>(p, tokens, vocab, dtype, scale, static_cast<cudaStream_t>(cuda_stream));
}

int pf_distill_fwd(const void* logits, int64_t ld, const int64_t* ids, const float* teacher, const float* teacher_lse, int k, double scale, float* loss,
                   int64_t tokens, int64_t vocab, int dtype, void* cuda_stream) {
    const int st = validate_vocab(logits, ld, tokens, vocab, scale, dtype);
    if (st != PF_OK || tokens == 0) return st;
    if (validate_teacher(ids, teacher, teacher_lse, k) != PF_OK || !loss || !aligned_to(loss)) return PF_ERR_INVALID_ARG;
    if (k > kMaxTeacher) return PF_ERR_UNSUPPORTED;
    VocabParams p = {};
    p.logits = logits; p.ld = ld; p.ids = ids; p.teacher = teacher; p.teacher_lse = teacher_lse; p.k = k; p.loss = loss;
    return vocab_run<kDistillFwd>(p, tokens, vocab, dtype, scale, static_cast<cudaStream_t>(cuda_stream));
}

int pf_distill_bwd(const void* logits, int64_t ld, const int64_t* ids, const float* teacher, const float* teacher_lse, int k, double scale,
                   const float* dloss, void* dlogits, int64_t lddl, float* loss, int64_t tokens, int64_t vocab, int dtype, void* cuda_stream) {
    const int st = validate_vocab(logits, ld, tokens, vocab, scale, dtype);
    if (st != PF_OK || tokens == 0) return st;
    if (validate_teacher(ids, teacher, teacher_lse, k) != PF_OK || validate_gradient(dlogits, lddl, vocab, dtype) != PF_OK ||
        !dloss || !aligned_to(dloss) || !aligned_to(loss))
        return PF_ERR_INVALID_ARG;
    if (k > kMaxTeacher) return PF_ERR_UNSUPPORTED;
    VocabParams p = {};
    p.logits = logits; p.ld = ld; p.ids = ids; p.teacher = teacher; p.teacher_lse = teacher_lse; p.k = k; p.dloss = dloss;
    p.dlogits = dlogits; p.lddl = lddl; p.loss = loss;
    return vocab_run<kDistillBwd>(p, tokens, vocab, dtype, scale, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
