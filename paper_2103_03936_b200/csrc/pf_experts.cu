// Tokens of a layer with experts: sorted by expert into the rows that the grouped layers read, and their results combined again.
//
// `tokens` tokens choose `k` of `experts` experts each: assignment a = token * k + j goes to expert id[a].  An expert's
// assignments keep their order; the r-th of expert e gets row
//   slot = e * capacity + r   (none from r = capacity on),     or, without a capacity,   offset[e] + r
// so that [experts, capacity, width] is a grouped layer's input as it stands.
//   dispatch     xs[slot(t, j)] = x[t], rows without a token 0;           backward  dx[t] = sum_j dxs[slot(t, j)]
//   combine      y[t] = sum_j w[t, j] ys[slot(t, j)];                     backward  dys[slot(t, j)] = w[t, j] dy[t], dw[t, j] = <dy[t], ys[slot(t, j)]>
// Sums run over j in order, in fp32.  Nothing is added by atomics: a row has one token, a token finds its rows by `slots`.
//
// Everything but the sort is bound by memory, and walks tokens: a token's row is read or written once for all of its experts.
#include <algorithm>
#include <initializer_list>

#include "pf_internal.h"

namespace pf {
namespace {

// ------------------------------------------------------------------------------ sort
// Blocks with a contiguous share of the assignments each, each of their warps with a contiguous part of that.  Counting first gives every
// warp the rows before its own (the warps before it in its block, the blocks before it); then a warp walks its assignments in order, 32 at a
// time: lanes that chose the same expert find one another by ballots, the first of them moves the warp's counter.
//
// Up to 32768 assignments: one cluster of up to eight blocks, which read one another's counts from distributed shared memory.  Bound by
// latency: a launch, a trip to memory for the assignments (which stay in registers), the cluster's meeting.  More of them keep eight SMs busy for
// too long, with single stores of sources above all (240 000 to 256 experts: 35 us): then a launch counts and a
// second one sorts, on up to every SM (15.5 us).
constexpr int kSortBlocks = 8;
constexpr int kMostExperts = 2048;
constexpr int64_t kClusterMost = 32768;

struct SortParams {
    int* totals;      // [blocks, experts]: the blocks' counts, where they are no cluster
    const int* ids;
    int* slots;
    int* sources;
    int* counts;
    int* offsets;
    int assignments, experts, capacity, rows;
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ int load_cluster(const int* p, uint32_t rank) {
    uint32_t from;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(from) : "memory");
    return v;
}

// The lanes whose values have the same lowest `bits` bits, a bit at a time (240 000 assignments to 256 experts on eight blocks: 35 us, with
// __match_any_sync 40).
__device__ __forceinline__ unsigned same_value(int value, int bits) {
    unsigned same = 0xffffffffu;
    for (int b = 0; b < bits; ++b) {
        const bool set = (value >> b) & 1;
        const unsigned with = __ballot_sync(0xffffffffu, set);
        same &= set ? with : ~with;
    }
    return same;
}

// The blocks' counts for a sort by more blocks than a cluster has.
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;
__global__ void __launch_bounds__(kSortThreads) count_kernel(const SortParams p) {
    extern __shared__ int sort_smem[];
    for (int e = threadIdx.x; e < p.experts; e += kSortThreads) sort_smem[e] = 0;
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int blocks = static_cast<int>(gridDim.x);
    const int64_t per_block = static_cast<int64_t>((p.assignments + blocks * kSortThreads - 1) / (blocks * kSortThreads)) * kSortThreads;
    const int64_t beg = blockIdx.x * per_block, end = min(beg + per_block, static_cast<int64_t>(p.assignments));
#pragma unroll 4
    for (int64_t a = beg + threadIdx.x; a < end; a += kSortThreads) {
        const int e = p.ids[a];
        if (e >= 0 && e < p.experts) atomicAdd(sort_smem + e, 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.experts; e += kSortThreads) p.totals[static_cast<int64_t>(blockIdx.x) * p.experts + e] = sort_smem[e];
}

// Shared memory: warps x experts counters (which become each warp's next row), then for each expert the block's total, the first row
// and the whole total.
template <bool kCluster>
__global__ void __launch_bounds__(kSortThreads) sort_kernel(const SortParams p) {
    extern __shared__ int sort_smem[];
    const int E = p.experts, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int* const mine = sort_smem + warp * E;
    int* const total = sort_smem + kSortWarps * E;      // (kCluster: of this block; else of the blocks before it)
    int* const first = total + E;
    int* const chosen = first + E;
    __shared__ int scan[kSortWarps];
    const int blocks = kCluster ? static_cast<int>(cluster_size()) : static_cast<int>(gridDim.x);
    const int rank = kCluster ? static_cast<int>(cluster_rank()) : static_cast<int>(blockIdx.x);
    const int per_warp = (p.assignments + blocks * kSortThreads - 1) / (blocks * kSortThreads) * 32;      // (at most 2^30 assignments)
    const int64_t beg64 = static_cast<int64_t>(rank * kSortWarps + warp) * per_warp;
    const int beg = beg64 < p.assignments ? static_cast<int>(beg64) : p.assignments;
    const int end = p.assignments - beg < per_warp ? p.assignments : beg + per_warp;
    for (int e = lane; e < E; e += 32) mine[e] = 0;
    __syncwarp();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const unsigned before = (1u << lane) - 1u;
    const int bits = 33 - __clz(E);      // (-1 differs from every expert in the highest of them; `held` has no other value outside)
    constexpr int kHeld = 8;      // assignments of a lane in registers
    int held[kHeld];
    auto hold = [&](int a0) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int a = a0 + 32 * i + lane;
            held[i] = a < end ? p.ids[a] : -1;
            // (another negative id could have an expert's lowest bits, which are all that the ballots compare)
            if (static_cast<unsigned>(held[i]) >= static_cast<unsigned>(E)) held[i] = -1;
        }
    };
    for (int a0 = beg; a0 < end; a0 += 32 * kHeld) {
        hold(a0);
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (held[i] >= 0) atomicAdd(mine + held[i], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += kSortThreads) {
        int sum = 0;
        for (int w = 0; w < kSortWarps; ++w) {
            const int c = sort_smem[w * E + e];
            sort_smem[w * E + e] = sum;
            sum += c;
        }
        if (kCluster) total[e] = sum;
    }
    if (kCluster) {
        cluster_sync();
    } else {
        // the blocks' counts, of as many at a time as there are threads for
        for (int e = threadIdx.x; e < E; e += kSortThreads) total[e] = chosen[e] = 0;
        __syncthreads();
        const int wide = min(E, kSortThreads), apart = kSortThreads / wide, part = threadIdx.x / wide;
        for (int e = threadIdx.x - part * wide; e < E && part < apart; e += wide) {
            int below = 0, count = 0;
#pragma unroll 8
            for (int b = part; b < blocks; b += apart) {
                const int c = p.totals[static_cast<int64_t>(b) * E + e];
                if (b < rank) below += c;
                count += c;
            }
            if (below) atomicAdd(total + e, below);
            if (count) atomicAdd(chosen + e, count);
        }
        __syncthreads();
    }
    // first rows of the experts: every block adds up the whole
    int carry = 0;
    for (int e0 = 0; e0 < E; e0 += kSortThreads) {
        const int e = e0 + threadIdx.x;
        int count = 0, below = 0;      // of all blocks, of those before this one
        if (e < E && kCluster) {
            int c[kSortBlocks];      // (asked for all at once)
#pragma unroll
            for (int b = 0; b < kSortBlocks; ++b) c[b] = b < blocks ? load_cluster(total + e, b) : 0;
#pragma unroll
            for (int b = 0; b < kSortBlocks; ++b) {
                if (b < rank) below += c[b];
                count += c[b];
            }
        } else if (e < E) {
            below = total[e];
            count = chosen[e];
        }
        int row = e < E ? e * p.capacity : 0;
        if (p.capacity == 0) {
            int x = count;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            __syncthreads();
            if (lane == 31) scan[warp] = x;
            __syncthreads();
            row = carry + x - count;
            for (int w = 0; w < kSortWarps; ++w) {
                if (w < warp) row += scan[w];
                carry += scan[w];
            }
        }
        if (e < E) {
            first[e] = row;
            chosen[e] = count;
            for (int w = 0; w < kSortWarps; ++w) sort_smem[w * E + e] += below;
            if (rank == 0) {
                p.counts[e] = count;
                p.offsets[e] = row;
                if (e == E - 1) p.offsets[E] = p.capacity == 0 ? row + count : E * p.capacity;
            }
        }
    }
    if (kCluster) asm volatile("barrier.cluster.arrive.release;" ::: "memory");      // this block has read the others' totals
    __syncthreads();
    // rows that no assignment takes
    const int thread = rank * kSortThreads + threadIdx.x, threads = blocks * kSortThreads;
    if (p.capacity > 0) {
        for (int r = thread; r < p.rows; r += threads) {
            const int e = r / p.capacity;
            if (r - e * p.capacity >= chosen[e]) p.sources[r] = -1;
        }
    } else {
        for (int r = first[E - 1] + chosen[E - 1] + thread; r < p.rows; r += threads) p.sources[r] = -1;
    }
    for (int a0 = beg; a0 < end; a0 += 32 * kHeld) {
        if (end - beg > 32 * kHeld) hold(a0);
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int a = a0 + 32 * i + lane, e = held[i];
            if (a0 + 32 * i >= end) break;
            const unsigned same = same_value(e, bits);
            int r = 0;
            if (e >= 0) r = mine[e] + __popc(same & before);
            __syncwarp();
            if (e >= 0 && (same & before) == 0) mine[e] += __popc(same);
            __syncwarp();
            if (a < end) {
                const bool in = e >= 0 && (p.capacity == 0 || r < p.capacity);
                const int slot = in ? first[e] + r : -1;
                p.slots[a] = slot;
                if (in) p.sources[slot] = a;
            }
        }
    }
    if (kCluster) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");        // (no block leaves while another reads its totals)
}

// ------------------------------------------------------------------------------ rows
template <int kBytes> struct Raw;
template <> struct Raw<16> { using T = uint4; };
template <> struct Raw<8> { using T = uint2; };
template <> struct Raw<4> { using T = unsigned; };

// A piece of a row: kBytes, kN elements of T.
template <typename T, int kBytes>
struct Part {
    static constexpr int kN = kBytes / static_cast<int>(sizeof(T));
    union {
        typename Raw<kBytes>::T raw;
        unsigned short half[kBytes / 2];
        unsigned word[kBytes / 4];
    };
    __device__ __forceinline__ Part() {}
    __device__ __forceinline__ void get(float (&x)[kN]) const {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(word[i]);
            else x[i] = __uint_as_float(static_cast<unsigned>(half[i]) << 16);
        }
    }
    __device__ __forceinline__ void set(const float (&x)[kN]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < kN; ++i) word[i] = __float_as_uint(x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kBytes / 4; ++i) {
                const __nv_bfloat162 t = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                word[i] = *reinterpret_cast<const unsigned*>(&t);
            }
        }
    }
};

// Rows in pieces of kUnit bytes (16, 8 or 4), at boundaries of which all rows start and end.  kUnit = 2 (bf16, odd widths and pitches): in
// pieces of 16 bytes, those of memory that a row (the one that is written, or the one that `frame` names) lies in: the first starts up to 14
// bytes before the row, the last ends as far behind it.  Such a piece of another row is put together from the aligned words that it
// lies in, of which only those are read that hold a byte of the row; the ends of a row are written element by element.
template <typename T, int kUnit>
struct Rows {
    static constexpr bool kAligned = kUnit != 2;
    static constexpr int kBytes = kAligned ? kUnit : 16;
    using P = Part<T, kBytes>;
    static __device__ __forceinline__ int lead(const char* frame) { return kAligned ? 0 : static_cast<int>(reinterpret_cast<uintptr_t>(frame) & 15); }
    static __device__ __forceinline__ int pieces(const char* frame, int bytes) { return kAligned ? bytes / kBytes : (lead(frame) + bytes + 15) / 16; }
    // Byte of the row at which piece v starts.
    static __device__ __forceinline__ int place(const char* frame, int v) { return v * kBytes - lead(frame); }
    static __device__ __forceinline__ bool whole(int at, int bytes) { return kAligned || (at >= 0 && at + 16 <= bytes); }
    static __device__ __forceinline__ bool inside(int at, int i, int bytes) {
        const int b = at + i * static_cast<int>(sizeof(T));
        return b >= 0 && b < bytes;
    }
    static __device__ __forceinline__ void load(P& d, const char* row, int at, int bytes) {
        if constexpr (kAligned) {
            d.raw = *reinterpret_cast<const decltype(d.raw)*>(row + at);
        } else {
            const char* const p = row + at;
            const int odd = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 2);
            const char* const low = p - odd;
            // (no branch: it would keep the loads of the pieces that differ in it apart)
            const int beg = -at + odd, end = bytes - at + odd;      // the row's bytes, counted from `low`
            unsigned w[5];
#pragma unroll
            for (int i = 0; i < 5; ++i)
                w[i] = 4 * i + 4 > beg && 4 * i < end && (i < 4 || odd) ? *reinterpret_cast<const unsigned*>(low + 4 * i) : 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) d.word[i] = __funnelshift_r(w[i], w[i + 1], odd * 8);
        }
    }
    static __device__ __forceinline__ void store(const P& d, char* row, int at, int bytes) {
        if (whole(at, bytes)) {
            *reinterpret_cast<decltype(P::raw)*>(row + at) = d.raw;
        } else {
#pragma unroll
            for (int i = 0; i < P::kN; ++i)
                if (inside(at, i, bytes)) *reinterpret_cast<unsigned short*>(row + at + 2 * i) = d.half[i];
        }
    }
};

struct RowParams {
    const char* x;            // rows of tokens that are read: x, dy
    char* y;                  // ... that are written: y, dx
    const char* rows_in;      // rows of experts that are read: ys, dxs
    char* rows_out;           // ... that are written: xs, dys
    const int* slots;
    const int* sources;
    const float* weights;     // null: 1
    float* dweights;
    int64_t pitch, in_pitch, out_pitch;      // bytes
    int tokens, k, rows;
    int bytes;                // of a row
    int lanes;                // of a warp to a token: 8, 16 or 32
    int segments;             // blocks that share the rows of a block's tokens (dispatch)
};

constexpr int kRowThreads = 256, kRowWarps = kRowThreads / 32;
constexpr int kWideThreads = 128, kWideWarps = kWideThreads / 32;      // of a block to a token
constexpr int kRowsToClear = 4;      // rows of experts that the lanes of a token look at besides
constexpr int kDispatchDeep = 4;      // pieces of a row that a lane has in hand

// Clears those of four rows that no token has: pieces v0, v0 + step, ... of them.
template <typename T, int kUnit>
__device__ __forceinline__ void clear_rows(const RowParams& p, int64_t item, int v0, int step) {
    const int64_t first = item * kRowsToClear;
    bool empty[kRowsToClear];
#pragma unroll
    for (int r = 0; r < kRowsToClear; ++r) empty[r] = first + r < p.rows && p.sources[first + r] < 0;
    using R = Rows<T, kUnit>;
    typename R::P z;
#pragma unroll
    for (int i = 0; i < R::kBytes / 4; ++i) z.word[i] = 0;
#pragma unroll
    for (int r = 0; r < kRowsToClear; ++r) {
        if (!empty[r]) continue;
        char* const to = p.rows_out + (first + r) * p.out_pitch;
        const int n = R::pieces(to, p.bytes);
        for (int v = v0; v < n; v += step) R::store(z, to, R::place(to, v), p.bytes);
    }
}

// The block's place: its tokens, and its part of their rows.  Dispatch, which reads and writes whole rows, has the parts of a row beside one another,
// so that what is in flight lies together (16384 x 2, 4096 wide: 75 us, 80 with the tokens' first parts together); combine, which gathers, the
// tokens' first parts (58 us against 67).
struct RowPlace {
    int64_t block;
    int segment;
};
template <bool kTogether>
__device__ __forceinline__ RowPlace row_place(const RowParams& p) {
    if constexpr (!kTogether) return {blockIdx.x, static_cast<int>(blockIdx.y)};
    const unsigned b = blockIdx.x, n = static_cast<unsigned>(p.segments), q = n == 1 ? b : b / n;
    return {q, static_cast<int>(b - q * n)};
}

// xs[slot] = x[token], a group of lanes to a token, several to a long row.
template <typename T, int kUnit>
__global__ void __launch_bounds__(kRowThreads) dispatch_kernel(const RowParams p) {
    using R = Rows<T, kUnit>;
    using P = typename R::P;
    constexpr int kDeep = R::kAligned ? kDispatchDeep : 2;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const RowPlace place = row_place<true>(p);
    const int lane = threadIdx.x & (p.lanes - 1), step = p.segments * p.lanes * kDeep;
    const int64_t item = (place.block * kRowThreads + threadIdx.x) / p.lanes;
    if (item < p.tokens) {
        const char* const from = p.x + item * p.pitch;
        const int* const slots = p.slots + item * p.k;
        if constexpr (R::kAligned) {      // read once
            const int n = p.bytes / R::kBytes;
            for (int v0 = place.segment * p.lanes * kDeep + lane; v0 < n; v0 += step) {
                P d[kDeep];
#pragma unroll
                for (int u = 0; u < kDeep; ++u)
                    if (v0 + p.lanes * u < n) R::load(d[u], from, (v0 + p.lanes * u) * R::kBytes, p.bytes);
#pragma unroll 2
                for (int j = 0; j < p.k; ++j) {
                    const int slot = slots[j];
                    if (slot < 0 || slot >= p.rows) continue;
                    char* const to = p.rows_out + slot * p.out_pitch;
#pragma unroll
                    for (int u = 0; u < kDeep; ++u)
                        if (v0 + p.lanes * u < n) R::store(d[u], to, (v0 + p.lanes * u) * R::kBytes, p.bytes);
                }
            }
        } else {                       // each row that is written has its own pieces
            for (int j = 0; j < p.k; ++j) {
                const int slot = slots[j];
                if (slot < 0 || slot >= p.rows) continue;
                char* const to = p.rows_out + slot * p.out_pitch;
                const int n = R::pieces(to, p.bytes);
                for (int v0 = place.segment * p.lanes * kDeep + lane; v0 < n; v0 += step) {
                    P d[kDeep];
#pragma unroll
                    for (int u = 0; u < kDeep; ++u)
                        if (v0 + p.lanes * u < n) R::load(d[u], from, R::place(to, v0 + p.lanes * u), p.bytes);
#pragma unroll
                    for (int u = 0; u < kDeep; ++u)
                        if (v0 + p.lanes * u < n) R::store(d[u], to, R::place(to, v0 + p.lanes * u), p.bytes);
                }
            }
        }
    }
    clear_rows<T, kUnit>(p, item, place.segment * p.lanes + lane, p.segments * p.lanes);
}

// y[token] = sum_j w_j rows_in[slot_j], kGroup experts of a token and kDeep pieces of a lane at a time (two of 16 bytes: 16384 x 2, 4096
// wide: 58 us, with four 69, with one 74; four of 8 or 4 bytes: 8192 x 2, 1002 wide: 16 us, with two 19).
template <typename T, int kUnit, int kGroup, int kDeep>
__global__ void __launch_bounds__(kRowThreads) combine_kernel(const RowParams p) {
    using R = Rows<T, kUnit>;
    using P = typename R::P;
    constexpr int kN = P::kN;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const RowPlace place = row_place<false>(p);
    const int lane = threadIdx.x & (p.lanes - 1);
    const int64_t token = (place.block * kRowThreads + threadIdx.x) / p.lanes;
    if (token >= p.tokens) return;
    char* const y = p.y + token * p.pitch;
    const int n = R::pieces(y, p.bytes);
    for (int v0 = place.segment * p.lanes * kDeep + lane; v0 < n; v0 += static_cast<int>(gridDim.y) * p.lanes * kDeep) {
        float sum[kDeep][kN];
#pragma unroll
        for (int u = 0; u < kDeep; ++u)
#pragma unroll
            for (int i = 0; i < kN; ++i) sum[u][i] = 0.f;
        for (int j0 = 0; j0 < p.k; j0 += kGroup) {
            int slot[kGroup];
            float w[kGroup];
            P d[kGroup][kDeep];
#pragma unroll
            for (int j = 0; j < kGroup; ++j) {
                slot[j] = j0 + j < p.k ? p.slots[token * p.k + j0 + j] : -1;
                if (slot[j] >= p.rows) slot[j] = -1;
                w[j] = p.weights && j0 + j < p.k ? p.weights[token * p.k + j0 + j] : 1.f;
            }
#pragma unroll
            for (int j = 0; j < kGroup; ++j) {
                if (slot[j] < 0) continue;
                const char* const from = p.rows_in + slot[j] * p.in_pitch;
#pragma unroll
                for (int u = 0; u < kDeep; ++u)
                    if (v0 + p.lanes * u < n) R::load(d[j][u], from, R::place(y, v0 + p.lanes * u), p.bytes);
            }
#pragma unroll
            for (int j = 0; j < kGroup; ++j) {
                if (slot[j] < 0) continue;
#pragma unroll
                for (int u = 0; u < kDeep; ++u) {
                    if (v0 + p.lanes * u >= n) continue;
                    float x[kN];
                    d[j][u].get(x);
#pragma unroll
                    for (int i = 0; i < kN; ++i) sum[u][i] = fmaf(w[j], x[i], sum[u][i]);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            if (v0 + p.lanes * u >= n) continue;
            P d;
            d.set(sum[u]);
            R::store(d, y, R::place(y, v0 + p.lanes * u), p.bytes);
        }
    }
}

// dys[slot] = w dy[token], dw = <dy[token], ys[slot]> for kGroup experts of a token at a time (one by one where each row has its own pieces): kWide a block
// to a token, else a group of lanes.
template <typename T, int kUnit, bool kWide, int kGroup>
__global__ void __launch_bounds__(kWide ? kWideThreads : kRowThreads) combine_bwd_kernel(const RowParams p) {
    constexpr int kThreads = kWide ? kWideThreads : kRowThreads;
    using R = Rows<T, kUnit>;
    using P = typename R::P;
    constexpr int kN = P::kN, kDeep = kGroup == 4 ? 1 : 2;
    static_assert(R::kAligned || kGroup == 1, "");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lanes = kWide ? 32 : p.lanes, lane = threadIdx.x & (lanes - 1), warp = threadIdx.x >> 5;
    const int64_t item = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / lanes, token = kWide ? blockIdx.x : item;
    const int start = kWide ? static_cast<int>(threadIdx.x) : lane, step = kWide ? kThreads : lanes;
    __shared__ float red[kWide ? kWideWarps * kGroup : 1];
    if (kWide ? token < p.tokens : __any_sync(0xffffffffu, token < p.tokens)) {      // (all lanes of a warp take part in the sums)
        const bool there = token < p.tokens;
        const char* const dy = p.x + token * p.pitch;
        for (int j0 = 0; j0 < p.k; j0 += kGroup) {
            int slot[kGroup];
            float w[kGroup], dot[kGroup];
#pragma unroll
            for (int j = 0; j < kGroup; ++j) {
                const bool in = there && j0 + j < p.k;
                slot[j] = in ? p.slots[token * p.k + j0 + j] : -1;
                if (slot[j] >= p.rows) slot[j] = -1;
                w[j] = in ? p.weights[token * p.k + j0 + j] : 0.f;
                dot[j] = 0.f;
            }
            // the pieces are those of the row that is written, or read where none is
            const char* frame = dy;
            if (!R::kAligned && slot[0] >= 0) frame = p.rows_out ? p.rows_out + slot[0] * p.out_pitch : p.rows_in + slot[0] * p.in_pitch;
            bool any = false;
#pragma unroll
            for (int j = 0; j < kGroup; ++j) any = any || slot[j] >= 0;
            const int n = any ? R::pieces(frame, p.bytes) : 0;
            for (int v0 = start; v0 < n; v0 += step * kDeep) {
                P d[kDeep], r[kGroup][kDeep];
#pragma unroll
                for (int u = 0; u < kDeep; ++u) {
                    const int v = v0 + u * step;
                    if (v >= n) continue;
                    R::load(d[u], dy, R::place(frame, v), p.bytes);
#pragma unroll
                    for (int j = 0; j < kGroup; ++j)
                        if (slot[j] >= 0) R::load(r[j][u], p.rows_in + slot[j] * p.in_pitch, R::place(frame, v), p.bytes);
                }
#pragma unroll
                for (int u = 0; u < kDeep; ++u) {
                    const int v = v0 + u * step;
                    if (v >= n) continue;
                    const int at = R::place(frame, v);
                    float g[kN];
                    d[u].get(g);
#pragma unroll
                    for (int j = 0; j < kGroup; ++j) {
                        if (slot[j] < 0) continue;
                        float x[kN];
                        r[j][u].get(x);
                        if (!R::whole(at, p.bytes)) {      // what lies beside the row is not part of the sum
#pragma unroll
                            for (int i = 0; i < kN; ++i)
                                if (!R::inside(at, i, p.bytes)) g[i] = x[i] = 0.f;
                        }
#pragma unroll
                        for (int i = 0; i < kN; ++i) {
                            dot[j] = fmaf(g[i], x[i], dot[j]);
                            x[i] = g[i] * w[j];
                        }
                        if (p.rows_out) {
                            r[j][u].set(x);
                            R::store(r[j][u], p.rows_out + slot[j] * p.out_pitch, at, p.bytes);
                        }
                    }
                }
            }
            if (!p.dweights) continue;
#pragma unroll
            for (int j = 0; j < kGroup; ++j)
                for (int o = lanes / 2; o > 0; o /= 2) dot[j] += __shfl_xor_sync(0xffffffffu, dot[j], o);
            if constexpr (kWide) {
                __syncthreads();
                if (lane == 0)
#pragma unroll
                    for (int j = 0; j < kGroup; ++j) red[warp * kGroup + j] = dot[j];
                __syncthreads();
                if (threadIdx.x < kGroup && j0 + static_cast<int>(threadIdx.x) < p.k) {
                    float s = 0.f;
                    for (int u = 0; u < kWideWarps; ++u) s += red[u * kGroup + threadIdx.x];
                    p.dweights[token * p.k + j0 + threadIdx.x] = s;
                }
            } else if (there && lane == 0) {
#pragma unroll
                for (int j = 0; j < kGroup; ++j)
                    if (j0 + j < p.k) p.dweights[token * p.k + j0 + j] = dot[j];
            }
        }
    }
    if (p.rows_out) clear_rows<T, kUnit>(p, item, lane, lanes);
}

// ------------------------------------------------------------------------------ host side
struct Matrix {
    const void* p;
    int64_t ld;
};
bool matrix_valid(const Matrix& m, int64_t rows, int64_t width, int dtype) {
    return rows == 0 || (m.p && elem_aligned(m.p, dtype) && m.ld >= width && m.ld < (1LL << 40));
}
bool list_valid(const void* p, int64_t n) { return n == 0 || (p && reinterpret_cast<uintptr_t>(p) % 4 == 0); }
// The bytes at a multiple of which the rows of all these matrices start and end, 16 at most.
int rows_unit(std::initializer_list<Matrix> all, int64_t width, int dtype) {
    const int64_t s = static_cast<int64_t>(dtype_size(dtype));
    uint64_t bits = static_cast<uint64_t>(width * s) | 16;
    for (const Matrix& m : all)
        if (m.p) bits |= reinterpret_cast<uintptr_t>(m.p) | static_cast<uint64_t>(m.ld * s);
    return static_cast<int>(bits & (~bits + 1));
}
int check_sizes(int64_t tokens, int k, int64_t rows, int64_t width, int dtype) {
    if (!valid_dtype(dtype) || tokens < 0 || k < 1 || rows < 0 || width < 1) return PF_ERR_INVALID_ARG;
    if (k > (1 << 16) || tokens > (1LL << 30) / k || rows > (1LL << 30) || width > (1LL << 28)) return PF_ERR_UNSUPPORTED;
    return PF_OK;
}

int check_assignments(int64_t tokens, int k, int experts, int64_t capacity) {
    if (tokens < 0 || k < 1 || experts < 1 || capacity < 0) return PF_ERR_INVALID_ARG;
    if (k > (1 << 16) || tokens > (1LL << 30) / k || experts > kMostExperts || capacity > (1LL << 30) / experts) return PF_ERR_UNSUPPORTED;
    return PF_OK;
}

// Blocks of a sort: a cluster's (1, 2, 4 or 8), or more of them.
int sort_blocks(int64_t assignments) {
    if (assignments > kClusterMost) return static_cast<int>(std::max<int64_t>(kSortBlocks + 1, std::min<int64_t>(num_sms(), ceil_div(assignments, 4 * kSortThreads))));
    int blocks = 1;
    while (blocks < kSortBlocks && static_cast<int64_t>(blocks) * kSortThreads < assignments) blocks *= 2;
    return blocks;
}

enum RowOp { kDispatch, kCombine, kCombineBwd };
template <typename T, int kUnit>
cudaError_t rows_run(RowOp op, RowParams p, cudaStream_t stream) {
    constexpr bool kAligned = Rows<T, kUnit>::kAligned;
    const int pieces = p.bytes / Rows<T, kUnit>::kBytes + (kAligned ? 0 : 1);
    p.lanes = pieces <= 8 ? 8 : pieces <= 16 ? 16 : 32;
    // (backward of combine) a block to a token where a warp to each would leave most of the machine idle
    const bool wide = op == kCombineBwd && p.tokens < num_sms() * kRowWarps * 2 && pieces > 32;
    const int threads = wide ? kWideThreads : kRowThreads, per_block = threads / p.lanes;
    int64_t blocks = wide ? static_cast<int64_t>(p.tokens) : ceil_div(p.tokens, per_block), segments = 1;
    if (p.rows_out) blocks = std::max(blocks, ceil_div(p.rows, static_cast<int64_t>(kRowsToClear) * per_block));
    if (blocks == 0) return cudaSuccess;
    void (*kernel)(RowParams) = nullptr;
    if (op == kDispatch) {
        kernel = dispatch_kernel<T, kUnit>;
        segments = ceil_div(pieces, 32 * kDispatchDeep);
    } else if (op == kCombine) {
        constexpr int kDeep = Rows<T, kUnit>::kBytes == 16 ? 2 : 4;
        kernel = p.k == 1 ? combine_kernel<T, kUnit, 1, kDeep> : p.k == 2 ? combine_kernel<T, kUnit, 2, kDeep> : combine_kernel<T, kUnit, 4, 2>;
        segments = ceil_div(pieces, 32 * (p.k <= 2 ? kDeep : 2));
    } else if constexpr (kAligned) {
        kernel = wide ? (p.k == 1 ? combine_bwd_kernel<T, kUnit, true, 1> : p.k == 2 ? combine_bwd_kernel<T, kUnit, true, 2> : combine_bwd_kernel<T, kUnit, true, 4>)
                      : (p.k == 1 ? combine_bwd_kernel<T, kUnit, false, 1> : p.k == 2 ? combine_bwd_kernel<T, kUnit, false, 2> : combine_bwd_kernel<T, kUnit, false, 4>);
    } else {
        kernel = wide ? combine_bwd_kernel<T, kUnit, true, 1> : combine_bwd_kernel<T, kUnit, false, 1>;
    }
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
    segments = std::min<int64_t>(segments, op == kDispatch ? 0x7fffffffLL / blocks : 65535);
    p.segments = static_cast<int>(segments);
    const dim3 grid = op == kDispatch ? dim3(static_cast<unsigned>(blocks * segments)) : dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(segments));
    return launch_beside(kernel, grid, threads, 0, 1, stream, p);
}
cudaError_t rows_launch(RowOp op, RowParams p, int unit, int64_t width, int dtype, cudaStream_t stream) {
    p.bytes = static_cast<int>(width * static_cast<int64_t>(dtype_size(dtype)));
    if (dtype == PF_BF16) {
        switch (unit) {
            case 16: return rows_run<__nv_bfloat16, 16>(op, p, stream);
            case 8: return rows_run<__nv_bfloat16, 8>(op, p, stream);
            case 4: return rows_run<__nv_bfloat16, 4>(op, p, stream);
            default: return rows_run<__nv_bfloat16, 2>(op, p, stream);
        }
    }
    switch (unit) {
        case 16: return rows_run<float, 16>(op, p, stream);
        case 8: return rows_run<float, 8>(op, p, stream);
        default: return rows_run<float, 4>(op, p, stream);
    }
}

}  // namespace
}  // namespace pf

using namespace pf;

extern "C" {

int64_t pf_expert_rows(int64_t tokens, int k, int experts, int64_t capacity) {
    if (check_assignments(tokens, k, experts, capacity) != PF_OK) return 0;
    return capacity > 0 ? experts * capacity : tokens * k;
}

size_t pf_expert_sort_workspace(int64_t tokens, int k, int experts) {
    if (check_assignments(tokens, k, experts, 0) != PF_OK) return 0;
    const int blocks = sort_blocks(tokens * k);
    return blocks > kSortBlocks ? align_up(sizeof(int) * static_cast<size_t>(blocks) * experts, 256) : 0;
}

int pf_expert_sort(const int32_t* ids, int64_t tokens, int k, int experts, int64_t capacity, int32_t* slots, int32_t* sources, int32_t* counts,
                   int32_t* offsets, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const int sizes = check_assignments(tokens, k, experts, capacity);
    if (sizes != PF_OK) return sizes;
    const int64_t a = tokens * k, rows = pf_expert_rows(tokens, k, experts, capacity);
    if (!list_valid(ids, a) || !list_valid(slots, a) || !list_valid(sources, rows) || !list_valid(counts, 1) || !list_valid(offsets, 1))
        return PF_ERR_INVALID_ARG;
    const int st = check_ws(workspace, workspace_bytes, pf_expert_sort_workspace(tokens, k, experts));
    if (st != PF_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const SortParams p{static_cast<int*>(workspace), ids, slots, sources, counts, offsets, static_cast<int>(a), experts, static_cast<int>(capacity), static_cast<int>(rows)};
    const int blocks = sort_blocks(a);
    const bool cluster = blocks <= kSortBlocks;
    const auto kernel = cluster ? sort_kernel<true> : sort_kernel<false>;
    const size_t each = sizeof(int) * (kSortWarps + 3);      // of shared memory for an expert: 152 KB for the most of them
    static std::atomic<uint64_t> allowed[2];
    // (48 KB without asking, of which the kernel's own array takes a part)
    if (each * experts > 47 * 1024) PF_CUDA(allow_dynamic_smem(reinterpret_cast<const void*>(kernel), each * kMostExperts, allowed[cluster ? 1 : 0]));
    const dim3 grid(static_cast<unsigned>(blocks));
    if (!cluster) PF_CUDA(launch_beside(count_kernel, grid, kSortThreads, sizeof(int) * experts, 1, stream, p));
    PF_CUDA(launch_beside(kernel, grid, kSortThreads, each * experts, cluster ? blocks : 1, stream, p));
    return PF_OK;
}

int pf_expert_dispatch_fwd(const void* x, int64_t ldx, const int32_t* slots, const int32_t* sources, void* xs, int64_t ldxs, int64_t tokens, int k,
                           int64_t rows, int64_t width, int dtype, void* cuda_stream) {
    const int st = check_sizes(tokens, k, rows, width, dtype);
    if (st != PF_OK) return st;
    if (!matrix_valid({x, ldx}, tokens, width, dtype) || !matrix_valid({xs, ldxs}, rows, width, dtype)) return PF_ERR_INVALID_ARG;
    if (!list_valid(slots, tokens) || !list_valid(sources, rows)) return PF_ERR_INVALID_ARG;
    if (rows == 0) return PF_OK;
    const int64_t s = static_cast<int64_t>(dtype_size(dtype));
    RowParams p = {};
    p.x = static_cast<const char*>(x);
    p.pitch = ldx * s;
    p.rows_out = static_cast<char*>(xs);
    p.out_pitch = ldxs * s;
    p.slots = slots;
    p.sources = sources;
    p.tokens = static_cast<int>(tokens);
    p.k = k;
    p.rows = static_cast<int>(rows);
    PF_CUDA(rows_launch(kDispatch, p, rows_unit({{tokens ? x : nullptr, ldx}, {xs, ldxs}}, width, dtype), width, dtype, static_cast<cudaStream_t>(cuda_stream)));
    return PF_OK;
}

int pf_expert_combine_fwd(const void* ys, int64_t ldys, const int32_t* slots, const float* weights, void* y, int64_t ldy, int64_t tokens, int k,
                          int64_t rows, int64_t width, int dtype, void* cuda_stream) {
    const int st = check_sizes(tokens, k, rows, width, dtype);
    if (st != PF_OK) return st;
    if (!matrix_valid({ys, ldys}, rows, width, dtype) || !matrix_valid({y, ldy}, tokens, width, dtype)) return PF_ERR_INVALID_ARG;
    if (!list_valid(slots, tokens) || reinterpret_cast<uintptr_t>(weights) % 4 != 0) return PF_ERR_INVALID_ARG;
    if (tokens == 0) return PF_OK;
    const int64_t s = static_cast<int64_t>(dtype_size(dtype));
    RowParams p = {};
    p.rows_in = static_cast<const char*>(ys);
    p.in_pitch = ldys * s;
    p.y = static_cast<char*>(y);
    p.pitch = ldy * s;
    p.slots = slots;
    p.weights = weights;
    p.tokens = static_cast<int>(tokens);
    p.k = k;
    p.rows = static_cast<int>(rows);
    PF_CUDA(rows_launch(kCombine, p, rows_unit({{rows ? ys : nullptr, ldys}, {y, ldy}}, width, dtype), width, dtype, static_cast<cudaStream_t>(cuda_stream)));
    return PF_OK;
}

int pf_expert_dispatch_bwd(const void* dxs, int64_t lddxs, const int32_t* slots, void* dx, int64_t lddx, int64_t tokens, int k, int64_t rows,
                           int64_t width, int dtype, void* cuda_stream) {
    return pf_expert_combine_fwd(dxs, lddxs, slots, nullptr, dx, lddx, tokens, k, rows, width, dtype, cuda_stream);
}

int pf_expert_combine_bwd(const void* ys, int64_t ldys, const int32_t* slots, const int32_t* sources, const float* weights, const void* dy,
                          int64_t lddy, void* dys, int64_t lddys, float* dweights, int64_t tokens, int k, int64_t rows, int64_t width, int dtype,
                          void* cuda_stream) {
    const int st = check_sizes(tokens, k, rows, width, dtype);
    if (st != PF_OK) return st;
    if (!dys && !dweights && rows > 0) return PF_ERR_INVALID_ARG;
    if (!matrix_valid({ys, ldys}, rows, width, dtype) || !matrix_valid({dy, lddy}, tokens, width, dtype)) return PF_ERR_INVALID_ARG;
    if (dys && !matrix_valid({dys, lddys}, rows, width, dtype)) return PF_ERR_INVALID_ARG;
    if (!list_valid(slots, tokens) || !list_valid(weights, tokens) || !list_valid(sources, dys ? rows : 0) || reinterpret_cast<uintptr_t>(dweights) % 4 != 0)
        return PF_ERR_INVALID_ARG;
    const int64_t s = static_cast<int64_t>(dtype_size(dtype));
    RowParams p = {};
    p.rows_in = static_cast<const char*>(ys);
    p.in_pitch = ldys * s;
    p.x = static_cast<const char*>(dy);
    p.pitch = lddy * s;
    p.rows_out = rows > 0 ? static_cast<char*>(dys) : nullptr;
    p.out_pitch = lddys * s;
    p.slots = slots;
    p.sources = sources;
    p.weights = weights;
    p.dweights = dweights;
    p.tokens = static_cast<int>(tokens);
    p.k = k;
    p.rows = static_cast<int>(rows);
    PF_CUDA(rows_launch(kCombineBwd, p, rows_unit({{rows ? ys : nullptr, ldys}, {tokens ? dy : nullptr, lddy}, {p.rows_out, lddys}}, width, dtype), width,
                        dtype, static_cast<cudaStream_t>(cuda_stream)));
    return PF_OK;
}

}  // extern "C"
