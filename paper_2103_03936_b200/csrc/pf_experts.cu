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
// One cluster of blocks, each with a contiguous share of the assignments, each of its warps with a contiguous part of that.  Counting
// first gives every warp the rows before its own (the warps before it in its block, the blocks before it through distributed shared
// memory); then a warp walks its assignments in order, 32 at a time: lanes that chose the same expert find one another, the
// first of them moves the warp's counter.  Bound by latency: a launch, one trip to memory for up to 256 assignments of a warp, which stay
// in registers, and the cluster's meeting.
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32, kSortBlocks = 8;
constexpr int kMostExperts = 2048;

struct SortParams {
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

// Shared memory: warps x experts counters (which become each warp's next row), then for each expert the block's total, the first row
// and the whole total.
__global__ void __launch_bounds__(kSortThreads) sort_kernel(const SortParams p) {
    extern __shared__ int sort_smem[];
    const int E = p.experts, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int* const mine = sort_smem + warp * E;
    int* const total = sort_smem + kSortWarps * E;
    int* const first = total + E;
    int* const chosen = first + E;
    __shared__ int scan[kSortWarps];
    const int blocks = static_cast<int>(cluster_size()), rank = static_cast<int>(cluster_rank());
    const int per_warp = (p.assignments + blocks * kSortThreads - 1) / (blocks * kSortThreads) * 32;      // (at most 2^30 assignments)
    const int64_t beg64 = static_cast<int64_t>(rank * kSortWarps + warp) * per_warp;
    const int beg = beg64 < p.assignments ? static_cast<int>(beg64) : p.assignments;
    const int end = p.assignments - beg < per_warp ? p.assignments : beg + per_warp;
    for (int e = lane; e < E; e += 32) mine[e] = 0;
    __syncwarp();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const unsigned before = (1u << lane) - 1u;
    constexpr int kHeld = 8;      // assignments of a lane in registers
    int held[kHeld];
    auto hold = [&](int a0) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int a = a0 + 32 * i + lane;
            held[i] = a < end ? p.ids[a] : -1;
            if (held[i] >= E) held[i] = -1;
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
        total[e] = sum;
    }
    cluster_sync();
    // first rows of the experts: every block adds up the whole
    int carry = 0;
    for (int e0 = 0; e0 < E; e0 += kSortThreads) {
        const int e = e0 + threadIdx.x;
        int count = 0, below = 0;      // of all blocks, of those before this one
        if (e < E) {
            for (int b = 0; b < blocks; ++b) {
                const int c = load_cluster(total + e, b);
                if (b < rank) below += c;
                count += c;
            }
        }
        int row = e * p.capacity;
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
            const unsigned same = __match_any_sync(0xffffffffu, e);
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
    cluster_sync();      // (no block leaves while another reads its totals)
}

// ------------------------------------------------------------------------------ rows
template <int kBytes> struct Raw;
template <> struct Raw<16> { using T = uint4; };
template <> struct Raw<8> { using T = uint2; };
template <> struct Raw<4> { using T = unsigned; };
template <> struct Raw<2> { using T = unsigned short; };

// A piece of a row: kBytes of elements of T.
template <typename T, int kBytes>
struct Part {
    static constexpr int kN = kBytes / static_cast<int>(sizeof(T));
    union {
        typename Raw<kBytes>::T raw;
        unsigned short half[kBytes / 2];
        unsigned word[(kBytes + 3) / 4];
    };
    __device__ __forceinline__ Part() {}
    __device__ __forceinline__ void load(const void* p) { raw = *static_cast<const typename Raw<kBytes>::T*>(p); }
    __device__ __forceinline__ void store(void* p) const { *static_cast<typename Raw<kBytes>::T*>(p) = raw; }
    __device__ __forceinline__ void zero() { raw = typename Raw<kBytes>::T{}; }
    __device__ __forceinline__ void get(float (&x)[kN]) const {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(word[i]);
            else x[i] = __uint_as_float(static_cast<unsigned>(half[i]) << 16);
        }
    }
    __device__ __forceinline__ void set(const float (&x)[kN]) {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            if constexpr (sizeof(T) == 4) word[i] = __float_as_uint(x[i]);
            else {
                const __nv_bfloat16 t = __float2bfloat16_rn(x[i]);
                half[i] = *reinterpret_cast<const unsigned short*>(&t);
            }
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
    int parts;                // pieces of a row
};

constexpr int kRowThreads = 256, kRowWarps = kRowThreads / 32;
constexpr int kRowsToClear = 4;      // rows of experts that a warp looks at beside its token
constexpr int kDispatchDeep = 4, kCombineDeep = 2;      // pieces of a row that a lane has in hand

// Clears those of a warp's rows that no token has, pieces v0, v0 + step, ... of them.
template <typename T, int kBytes>
__device__ __forceinline__ void clear_rows(const RowParams& p, int64_t item, int v0, int step) {
    const int lane = threadIdx.x & 31;
    const int64_t first = item * kRowsToClear;
    if (first >= p.rows) return;
    const int64_t row = first + lane;
    unsigned empty = __ballot_sync(0xffffffffu, lane < kRowsToClear && row < p.rows && p.sources[row] < 0);
    Part<T, kBytes> z;
    z.zero();
    for (; empty; empty &= empty - 1) {
        char* const to = p.rows_out + (first + __ffs(empty) - 1) * p.out_pitch;
        for (int v = v0; v < p.parts; v += step) z.store(to + static_cast<int64_t>(v) * kBytes);
    }
}

// xs[slot] = x[token]: a warp to a token's row, 32 * kDispatchDeep pieces at a time (gridDim.y warps to long ones).
template <typename T, int kBytes>
__global__ void __launch_bounds__(kRowThreads) dispatch_kernel(const RowParams p) {
    constexpr int kDeep = kDispatchDeep;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * kRowWarps + (threadIdx.x >> 5);
    if (item < p.tokens) {
        const char* const from = p.x + item * p.pitch;
        for (int v0 = blockIdx.y * 32 * kDeep + lane; v0 < p.parts; v0 += gridDim.y * 32 * kDeep) {
            Part<T, kBytes> d[kDeep];
#pragma unroll
            for (int u = 0; u < kDeep; ++u)
                if (v0 + 32 * u < p.parts) d[u].load(from + static_cast<int64_t>(v0 + 32 * u) * kBytes);
            for (int j = 0; j < p.k; ++j) {
                const int slot = p.slots[item * p.k + j];
                if (slot < 0 || slot >= p.rows) continue;
                char* const to = p.rows_out + static_cast<int64_t>(slot) * p.out_pitch;
#pragma unroll
                for (int u = 0; u < kDeep; ++u)
                    if (v0 + 32 * u < p.parts) d[u].store(to + static_cast<int64_t>(v0 + 32 * u) * kBytes);
            }
        }
    }
    clear_rows<T, kBytes>(p, item, blockIdx.y * 32 + lane, gridDim.y * 32);
}

// y[token] = sum_j w_j rows_in[slot_j]: a warp to 32 * kCombineDeep pieces of a token's row at a time.
template <typename T, int kBytes>
__global__ void __launch_bounds__(kRowThreads) combine_kernel(const RowParams p) {
    constexpr int kDeep = kCombineDeep, kN = Part<T, kBytes>::kN;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int64_t token = static_cast<int64_t>(blockIdx.x) * kRowWarps + (threadIdx.x >> 5);
    if (token >= p.tokens) return;
    for (int v0 = blockIdx.y * 32 * kDeep + lane; v0 < p.parts; v0 += gridDim.y * 32 * kDeep) {
        float sum[kDeep][kN];
#pragma unroll
        for (int u = 0; u < kDeep; ++u)
#pragma unroll
            for (int i = 0; i < kN; ++i) sum[u][i] = 0.f;
#pragma unroll 2
        for (int j = 0; j < p.k; ++j) {
            const int slot = p.slots[token * p.k + j];
            if (slot < 0 || slot >= p.rows) continue;
            const float w = p.weights ? p.weights[token * p.k + j] : 1.f;
            const char* const from = p.rows_in + static_cast<int64_t>(slot) * p.in_pitch;
            Part<T, kBytes> d[kDeep];
#pragma unroll
            for (int u = 0; u < kDeep; ++u)
                if (v0 + 32 * u < p.parts) d[u].load(from + static_cast<int64_t>(v0 + 32 * u) * kBytes);
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
                if (v0 + 32 * u >= p.parts) continue;
                float x[kN];
                d[u].get(x);
#pragma unroll
                for (int i = 0; i < kN; ++i) sum[u][i] = fmaf(w, x[i], sum[u][i]);
            }
        }
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            if (v0 + 32 * u >= p.parts) continue;
            Part<T, kBytes> d;
            d.set(sum[u]);
            d.store(p.y + token * p.pitch + static_cast<int64_t>(v0 + 32 * u) * kBytes);
        }
    }
}

// dys[slot] = w dy[token], dw = <dy[token], ys[slot]> for kGroup experts of a token at a time: kWide a block to a token, else a warp.
template <typename T, int kBytes, bool kWide, int kGroup>
__global__ void __launch_bounds__(kRowThreads) combine_bwd_kernel(const RowParams p) {
    constexpr int kN = Part<T, kBytes>::kN, kDeep = kGroup == 4 ? 1 : 2;
    constexpr int kStep = kWide ? kRowThreads : 32;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * kRowWarps + warp, token = kWide ? blockIdx.x : item;
    __shared__ float red[kWide ? kRowWarps * kGroup : 1];
    if (token < p.tokens) {
        const char* const dy = p.x + token * p.pitch;
        for (int j0 = 0; j0 < p.k; j0 += kGroup) {
            int slot[kGroup];
            float w[kGroup], dot[kGroup];
#pragma unroll
            for (int j = 0; j < kGroup; ++j) {
                const bool in = j0 + j < p.k;
                slot[j] = in ? p.slots[token * p.k + j0 + j] : -1;
                if (slot[j] >= p.rows) slot[j] = -1;
                w[j] = in ? p.weights[token * p.k + j0 + j] : 0.f;
                dot[j] = 0.f;
            }
            for (int v0 = kWide ? static_cast<int>(threadIdx.x) : lane; v0 < p.parts; v0 += kStep * kDeep) {
                Part<T, kBytes> d[kDeep], r[kGroup][kDeep];
#pragma unroll
                for (int u = 0; u < kDeep; ++u) {
                    const int v = v0 + u * kStep;
                    if (v >= p.parts) continue;
                    d[u].load(dy + static_cast<int64_t>(v) * kBytes);
#pragma unroll
                    for (int j = 0; j < kGroup; ++j)
                        if (slot[j] >= 0) r[j][u].load(p.rows_in + slot[j] * p.in_pitch + static_cast<int64_t>(v) * kBytes);
                }
#pragma unroll
                for (int u = 0; u < kDeep; ++u) {
                    const int v = v0 + u * kStep;
                    if (v >= p.parts) continue;
                    float g[kN];
                    d[u].get(g);
#pragma unroll
                    for (int j = 0; j < kGroup; ++j) {
                        if (slot[j] < 0) continue;
                        float x[kN];
                        r[j][u].get(x);
#pragma unroll
                        for (int i = 0; i < kN; ++i) {
                            dot[j] = fmaf(g[i], x[i], dot[j]);
                            x[i] = g[i] * w[j];
                        }
                        if (p.rows_out) {
                            r[j][u].set(x);
                            r[j][u].store(p.rows_out + slot[j] * p.out_pitch + static_cast<int64_t>(v) * kBytes);
                        }
                    }
                }
            }
            if (!p.dweights) continue;
#pragma unroll
            for (int j = 0; j < kGroup; ++j)
#pragma unroll
                for (int o = 16; o > 0; o /= 2) dot[j] += __shfl_xor_sync(0xffffffffu, dot[j], o);
            if constexpr (kWide) {
                __syncthreads();
                if (lane == 0)
#pragma unroll
                    for (int j = 0; j < kGroup; ++j) red[warp * kGroup + j] = dot[j];
                __syncthreads();
                if (threadIdx.x < kGroup && j0 + static_cast<int>(threadIdx.x) < p.k) {
                    float s = 0.f;
                    for (int u = 0; u < kRowWarps; ++u) s += red[u * kGroup + threadIdx.x];
                    p.dweights[token * p.k + j0 + threadIdx.x] = s;
                }
            } else if (lane == 0) {
#pragma unroll
                for (int j = 0; j < kGroup; ++j)
                    if (j0 + j < p.k) p.dweights[token * p.k + j0 + j] = dot[j];
            }
        }
    }
    if (p.rows_out) clear_rows<T, kBytes>(p, item, lane, 32);
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
// Bytes of the pieces that rows of all these matrices divide into.
int piece_bytes(std::initializer_list<Matrix> all, int64_t width, int dtype) {
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

enum RowOp { kDispatch, kCombine, kCombineBwd };
template <typename T, int kBytes>
cudaError_t combine_bwd_run(const RowParams& p, cudaStream_t stream) {
    // a block to a token where a warp to each would leave most of the machine idle
    const bool wide = p.tokens < num_sms() * kRowWarps * 2 && p.parts > 32;
    const int64_t blocks = std::max(wide ? static_cast<int64_t>(p.tokens) : ceil_div(p.tokens, kRowWarps),
                                    p.rows_out ? ceil_div(p.rows, kRowsToClear * kRowWarps) : 0);
    if (blocks == 0) return cudaSuccess;
    const auto kernel = wide ? (p.k == 1 ? combine_bwd_kernel<T, kBytes, true, 1> : p.k == 2 ? combine_bwd_kernel<T, kBytes, true, 2> : combine_bwd_kernel<T, kBytes, true, 4>)
                             : (p.k == 1 ? combine_bwd_kernel<T, kBytes, false, 1> : p.k == 2 ? combine_bwd_kernel<T, kBytes, false, 2> : combine_bwd_kernel<T, kBytes, false, 4>);
    return launch_beside(kernel, dim3(static_cast<unsigned>(blocks)), kRowThreads, 0, 1, stream, p);
}
template <typename T, int kBytes>
cudaError_t rows_run(RowOp op, RowParams p, int64_t width, cudaStream_t stream) {
    p.parts = static_cast<int>(width * static_cast<int64_t>(sizeof(T)) / kBytes);
    if (op == kCombineBwd) return combine_bwd_run<T, kBytes>(p, stream);
    const bool dispatch = op == kDispatch;
    const int64_t segments = std::min<int64_t>(ceil_div(p.parts, 32 * (dispatch ? kDispatchDeep : kCombineDeep)), 65535);
    const int64_t blocks = std::max(ceil_div(p.tokens, kRowWarps), dispatch ? ceil_div(p.rows, kRowsToClear * kRowWarps) : 0);
    if (blocks == 0) return cudaSuccess;
    const auto kernel = dispatch ? dispatch_kernel<T, kBytes> : combine_kernel<T, kBytes>;
    return launch_beside(kernel, dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(segments)), kRowThreads, 0, 1, stream, p);
}
cudaError_t rows_launch(RowOp op, const RowParams& p, int bytes, int64_t width, int dtype, cudaStream_t stream) {
    if (dtype == PF_BF16) {
        switch (bytes) {
            case 16: return rows_run<__nv_bfloat16, 16>(op, p, width, stream);
            case 8: return rows_run<__nv_bfloat16, 8>(op, p, width, stream);
            case 4: return rows_run<__nv_bfloat16, 4>(op, p, width, stream);
            default: return rows_run<__nv_bfloat16, 2>(op, p, width, stream);
        }
    }
    switch (bytes) {
        case 16: return rows_run<float, 16>(op, p, width, stream);
        case 8: return rows_run<float, 8>(op, p, width, stream);
        default: return rows_run<float, 4>(op, p, width, stream);
    }
}

}  // namespace
}  // namespace pf

using namespace pf;

extern "C" {

int64_t pf_expert_rows(int64_t tokens, int k, int experts, int64_t capacity) {
    if (tokens < 0 || k < 1 || experts < 1 || capacity < 0) return 0;
    return capacity > 0 ? experts * capacity : tokens * k;
}

int pf_expert_sort(const int32_t* ids, int64_t tokens, int k, int experts, int64_t capacity, int32_t* slots, int32_t* sources, int32_t* counts,
                   int32_t* offsets, void* cuda_stream) {
    if (tokens < 0 || k < 1 || experts < 1 || capacity < 0) return PF_ERR_INVALID_ARG;
    if (k > (1 << 16) || tokens > (1LL << 30) / k || experts > kMostExperts || capacity > (1LL << 30) / experts) return PF_ERR_UNSUPPORTED;
    const int64_t a = tokens * k, rows = pf_expert_rows(tokens, k, experts, capacity);
    if (!list_valid(ids, a) || !list_valid(slots, a) || !list_valid(sources, rows) || !list_valid(counts, 1) || !list_valid(offsets, 1))
        return PF_ERR_INVALID_ARG;
    const SortParams p{ids, slots, sources, counts, offsets, static_cast<int>(a), experts, static_cast<int>(capacity), static_cast<int>(rows)};
    const size_t smem = sizeof(int) * static_cast<size_t>(experts) * (kSortWarps + 3);      // 152 KB for the most experts
    static std::atomic<uint64_t> allowed{0};
    if (smem > 48 * 1024)
        PF_CUDA(allow_dynamic_smem(reinterpret_cast<const void*>(&sort_kernel), sizeof(int) * kMostExperts * (kSortWarps + 3), allowed));
    int blocks = 1;
    while (blocks < kSortBlocks && static_cast<int64_t>(blocks) * kSortThreads < a) blocks *= 2;
    PF_CUDA(launch_beside(sort_kernel, dim3(static_cast<unsigned>(blocks)), kSortThreads, smem, blocks, static_cast<cudaStream_t>(cuda_stream), p));
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
    PF_CUDA(rows_launch(kDispatch, p, piece_bytes({{tokens ? x : nullptr, ldx}, {xs, ldxs}}, width, dtype), width, dtype, static_cast<cudaStream_t>(cuda_stream)));
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
    PF_CUDA(rows_launch(kCombine, p, piece_bytes({{rows ? ys : nullptr, ldys}, {y, ldy}}, width, dtype), width, dtype, static_cast<cudaStream_t>(cuda_stream)));
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
    PF_CUDA(rows_launch(kCombineBwd, p, piece_bytes({{rows ? ys : nullptr, ldys}, {tokens ? dy : nullptr, lddy}, {p.rows_out, lddys}}, width, dtype), width,
                        dtype, static_cast<cudaStream_t>(cuda_stream)));
    return PF_OK;
}

}  // extern "C"
