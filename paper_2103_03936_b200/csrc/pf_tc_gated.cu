// Second products of a gated layer with its gate, on the tensor cores:  g = T0 V0^T + b0,  u = T1 V1^T + b1,
//   forward   y = act(g) u
//   backward  dZ0 = dY u act'(g),  dZ1 = dY act(g)      (g and u are computed again: a stash would be 2 m n elements)
//
// A pair of CTAs computes tiles of 256 rows x 128 columns of g and of u at the same time (cta_group::2: each CTA holds 128 of the rows of T and 64 of those of V
// and receives its rows x all columns), two accumulators of 128 columns each in tensor memory, twice, so that the products of the next tile run under the gate
// of the present one.  Forward, a contraction of up to 256 leaves room for the rows of T0 and T1 to stay in shared memory: a pair walks over a run of neighbouring
// tiles, row after row, and only V0 and V1 come through the ring (16 KB a CTA for 64 contraction elements of a tile).  Else both come, and a pair takes every pairs-th tile.
// The gate is what the tensor cores wait for, so sixteen warps share it; results leave by TMA.
// Forward, two teams of eight warps take every other tile, so that while some wait for tensor memory or barriers others compute.  Backward (bound by memory) all
// take each tile; dY comes by TMA, two tiles ahead, and dZ0 leaves from its place.
//
// Forward, 16384 x 4096 over 64 (floor: y at the copy's rate, 21 us): stores straight from registers, 32 bytes a lane, 52 us; through shared memory with plain stores 57;
// by TMA, one team, 66; two teams 51; two teams with panels of 64 columns (128 bytes a row) 45, without releases at the cluster's scope (arrive_relaxed) 39, with fewer
// special functions 37.5 (max(0, .): 24).  Backward there (dY, dZ0, dZ1: 62 us): 93; dY one tile ahead 100, not ahead (two teams) 118.
#include <cuda.h>

#include <algorithm>

#include "pf_tc.h"
#include "pf_tc_gated.cuh"
#include "pf_tc_host.h"
#include "pf_tc_pair_prims.cuh"

namespace pf {
namespace tc {
namespace {

constexpr int kEpiWarps = 16;
constexpr int kGatedThreads = (4 + kEpiWarps) * 32;      // T producer, MMA issue, V producer, dY producer, gate
constexpr uint32_t kPanel = 16384;                       // 128 rows x 64 bf16
constexpr uint32_t kHalfPanel = 8192;                    // 64 rows
constexpr uint32_t kRoom = 224 * 1024;                   // of T, the ring, and what follows
constexpr uint32_t kTile = 32768;                        // 128 rows x 128 bf16: four panels of 128 rows x 32 (64 bytes a row)
constexpr uint32_t kWarpTile = 2048;                     // a warp's 32 rows x 32
constexpr int kGatedStages = 8;
constexpr int kDyTiles = 3;                              // backward, dY: of this tile, of the next, and where dZ0 of the last one leaves from

struct GatedParams {
    int M, N, nkb, tiles_n, total, stages;
    const void* bias;                          // [2, N] bf16, or null
    int64_t bias_step;
    __nv_bfloat16* y;                          // forward, of rows that TMA cannot store; else null
    int64_t ldy;
    unsigned int* status;
};
struct GatedCtl {
    uint64_t full[kGatedStages], empty[kGatedStages];
    uint64_t t_full, t_empty;
    uint64_t acc_full[2], acc_empty[2];
    uint64_t dy_full[kDyTiles], dy_empty[kDyTiles];
    uint32_t tmem_base;
    uint32_t abort;
};

__device__ __forceinline__ uint4 pack_eight(const float* v) {
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}

// A warp's 32 rows x 32 columns (64 bytes a row, 16-byte pieces exchanged by the row as TMA does) to rows of any pitch and alignment: whole 16-byte pieces of the
// destination, put together from five words with a funnel shift, eight rows to an instruction, then what is left of a row in front and behind.
__device__ __forceinline__ void store_any(uint32_t tile, __nv_bfloat16* C, int64_t ldc, int row0, int col0, int rows, int cols, int lane) {
    const int p = lane & 3, count = min(32, cols - col0);
    auto word = [&](int r, int w) {      // (behind the row's end any)
        return ld_shared_u32(tile + static_cast<uint32_t>(r) * 64u + ((static_cast<uint32_t>(w >> 2) ^ (static_cast<uint32_t>(r >> 1) & 3u)) << 4) + (w & 3) * 4u);
    };
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {
        const int r = i * 8 + (lane >> 2);
        if (row0 + r >= rows) continue;
        unsigned short* const d = reinterpret_cast<unsigned short*>(C) + static_cast<int64_t>(row0 + r) * ldc + col0;
        auto element = [&](int e) { return static_cast<unsigned short>(word(r, e >> 1) >> ((e & 1) * 16)); };
        const int head = static_cast<int>((0u - static_cast<uint32_t>(reinterpret_cast<uintptr_t>(d))) & 15u) >> 1;      // elements before the first whole piece
        const int e = head + 8 * p;
        if (e + 8 <= count) {
            uint32_t w[5];
#pragma unroll
            for (int k = 0; k < 5; ++k) w[k] = word(r, min(15, (e >> 1) + k));
            const uint32_t bit = (e & 1) * 16;
            *reinterpret_cast<uint4*>(d + e) = make_uint4(__funnelshift_r(w[0], w[1], bit), __funnelshift_r(w[1], w[2], bit), __funnelshift_r(w[2], w[3], bit),
                                                          __funnelshift_r(w[3], w[4], bit));
        }
        const int behind = count > head ? head + ((count - head) & ~7) : min(head, count);
        for (int k = p; k < min(head, count); k += 4) d[k] = element(k);
        for (int k = behind + p; k < count; k += 4) d[k] = element(k);
    }
}

// Arrival on a barrier of the pair's leader of warps that have read tensor memory (their loads are done): nothing that they wrote has to be seen with it, and a release
// of the cluster's scope waits for all of it, a quarter of the warps' time.
__device__ __forceinline__ void arrive_relaxed(uint32_t cluster_bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// 32 accumulator columns of a row with their bias.
__device__ __forceinline__ void add_bias32(float (&v)[32], const __nv_bfloat16* bias, int col, int n, int lane) {
    const unsigned short* const b = reinterpret_cast<const unsigned short*>(bias);
    const float mine = col + lane < n ? __uint_as_float(static_cast<uint32_t>(b[col + lane]) << 16) : 0.f;
#pragma unroll
    for (int e = 0; e < 32; ++e) v[e] += __shfl_sync(0xffffffffu, mine, e);
}
__device__ __forceinline__ void load_columns(uint32_t at, float (&v)[32]) {
    tmem_ld32(at, reinterpret_cast<uint32_t(&)[32]>(v));
}

// kResident: T stays in shared memory.  kWide (forward, results by TMA): panels of 64 columns leave, else of 32.  tmOut: y, or dZ; tmdY: backward.
template <bool kResident, bool kBwd, int kAct, bool kWide>
__global__ void __launch_bounds__(kGatedThreads, 1)
tc_gated_kernel(const __grid_constant__ CUtensorMap tmT, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmOut,
                const __grid_constant__ CUtensorMap tmdY, const GatedParams p) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    uint8_t* const smem = smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
    GatedCtl* const ctl = reinterpret_cast<GatedCtl*>(smem);
    const uint32_t t_smem = smem_u32(smem + 1024);
    const uint32_t ring = kResident ? t_smem + static_cast<uint32_t>(p.nkb) * 2 * kPanel : t_smem;
    constexpr uint32_t kStage = 2 * kHalfPanel + (kResident ? 0 : 2 * kPanel), kVOff = kResident ? 0 : 2 * kPanel;
    const uint32_t out = t_smem + kRoom - (kWide ? 2 : 1) * kTile;                 // y, or dZ1
    const uint32_t dys = out - kDyTiles * kTile;                 // backward: dY, in whose place dZ0 goes
    constexpr int kTeams = kBwd ? 1 : 2, kTeamWarps = kEpiWarps / kTeams;      // of the gate: tiles that are in work at a time
    volatile uint32_t* const abort_flag = &ctl->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = static_cast<int>(blockIdx.x) >> 1, pairs = static_cast<int>(gridDim.x) >> 1;
    // Runs of neighbouring tiles, or every pairs-th: what is written at one time then lies together.
    const int step = kResident ? 1 : pairs;
    const int beg = kResident ? static_cast<int>(static_cast<int64_t>(p.total) * pair / pairs) : pair;
    const int end = kResident ? static_cast<int>(static_cast<int64_t>(p.total) * (pair + 1) / pairs) : p.total;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(smem_u32(&ctl->full[s]), kResident ? 1 : 2);      // (the leader's: its producers arrive with the bytes of both CTAs)
            mbar_init(smem_u32(&ctl->empty[s]), 1);
        }
        mbar_init(smem_u32(&ctl->t_full), 1);
        mbar_init(smem_u32(&ctl->t_empty), 1);
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&ctl->acc_full[b]), 1);
            mbar_init(smem_u32(&ctl->acc_empty[b]), 2 * kTeamWarps);    // (the leader's)
        }
        for (int b = 0; b < kDyTiles; ++b) {
            mbar_init(smem_u32(&ctl->dy_full[b]), 1);
            mbar_init(smem_u32(&ctl->dy_empty[b]), kEpiWarps);
        }
        ctl->abort = 0;
        fence_barrier_init();
        fence_proxy_async_smem();
        tma_prefetch_desc(&tmT);
        tma_prefetch_desc(&tmV);
        tma_prefetch_desc(&tmOut);
        if (kBwd) tma_prefetch_desc(&tmdY);
    }
    if (warp == 1) tmem_alloc_pair(smem_u32(&ctl->tmem_base), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    cluster_sync_all();
    pdl_wait();
    pdl_launch_dependents();
    const uint32_t tmem = ctl->tmem_base;
    const uint32_t full0 = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]);

    if (warp == 0 || warp == 2) {
        if (elect_one()) {
            // ------------------------------------------------------------ producers (T: warp 0, V: warp 2)
            bool ok = true;
            const uint32_t full_leader0 = map_to_cta(full0, 0);
            if (kResident && warp == 0) {
                const uint32_t bar = map_to_cta(smem_u32(&ctl->t_full), 0);
                uint32_t ph = 1;
                for (int t = beg; t < end && ok;) {
                    const int tm = t / p.tiles_n, row = tm * 256 + static_cast<int>(rank) * 128;
                    ok = mbar_wait(smem_u32(&ctl->t_empty), ph, abort_flag, p.status);
                    if (!ok) break;
                    if (rank == 0) mbar_expect_tx(smem_u32(&ctl->t_full), static_cast<uint32_t>(p.nkb) * 4 * kPanel);
                    for (int kb = 0; kb < p.nkb; ++kb)
                        for (int g = 0; g < 2; ++g) tma_load_3d_pair(t_smem + static_cast<uint32_t>(2 * kb + g) * kPanel, &tmT, bar, kb * 64, row, g);
                    ph ^= 1u;
                    t = (tm + 1) * p.tiles_n;
                }
            } else {
                const CUtensorMap* const map = warp == 0 ? &tmT : &tmV;
                const uint32_t bytes = warp == 0 ? kPanel : kHalfPanel, off = warp == 0 ? 0u : kVOff;
                uint32_t s = 0, ph = 1;
                for (int t = beg; t < end && ok; t += step) {
                    const int tm = t / p.tiles_n;
                    const int row = warp == 0 ? tm * 256 + static_cast<int>(rank) * 128 : (t - tm * p.tiles_n) * 128 + static_cast<int>(rank) * 64;
                    for (int kb = 0; kb < p.nkb; ++kb) {
                        ok = mbar_wait(empty0 + 8 * s, ph, abort_flag, p.status);
                        if (!ok) break;
                        const uint32_t dst = ring + s * kStage + off, bar = full_leader0 + 8 * s;
                        if (rank == 0) mbar_expect_tx(full0 + 8 * s, 4 * bytes);
                        tma_load_3d_pair(dst, map, bar, kb * 64, row, 0);
                        tma_load_3d_pair(dst + bytes, map, bar, kb * 64, row, 1);
                        if (++s == static_cast<uint32_t>(p.stages)) { s = 0; ph ^= 1u; }
                    }
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            // ------------------------------------------------------------ MMA issue (leader only)
            constexpr uint32_t idesc = make_idesc_bf16(256, 128, 0, 0);
            const uint64_t t_desc = make_smem_desc(t_smem, 16, 1024), ring_desc = make_smem_desc(ring, 16, 1024);
            uint32_t s = 0, ph = 0, t_ph = 0, j = 0;
            int tm_now = -1;
            bool ok = true;
            // both CTAs must have been given the same tensor-memory columns
            if (ld_cluster_u32(map_to_cta(smem_u32(&ctl->tmem_base), 1)) != tmem) {
                *abort_flag = 1u;
                if (p.status) atomicExch(p.status, kStatusTimeout);
                ok = false;
            }
            for (int t = beg; t < end && ok; t += step, ++j) {
                const int tm = t / p.tiles_n;
                if (kResident && tm != tm_now) {
                    if (tm_now >= 0) tc_commit_pair(smem_u32(&ctl->t_empty));      // (once the products of the row before are done)
                    ok = mbar_wait(smem_u32(&ctl->t_full), t_ph, abort_flag, p.status);
                    if (!ok) break;
                    t_ph ^= 1u;
                    tm_now = tm;
                }
                const uint32_t buf = j & 1u;
                ok = mbar_wait_cluster(smem_u32(&ctl->acc_empty[buf]), ((j >> 1) & 1u) ^ 1u, abort_flag, p.status);
                if (!ok) break;
                tc_fence_after();
                const uint32_t d = tmem + buf * 256;
                for (int kb = 0; kb < p.nkb; ++kb) {
                    ok = mbar_wait(full0 + 8 * s, ph, abort_flag, p.status);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t stage = ring_desc + ((s * kStage) >> 4);
                    const uint64_t a0 = kResident ? t_desc + static_cast<uint32_t>(kb) * (2 * kPanel >> 4) : stage, b0 = stage + (kVOff >> 4);
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const uint64_t a = a0 + g * (kPanel >> 4), b = b0 + g * (kHalfPanel >> 4);
                        tc_mma_bf16_pair(d + g * 128, a, b, idesc, kb > 0 ? 1u : 0u);
                        tc_mma_bf16_pair(d + g * 128, a + 2, b + 2, idesc, 1u);
                        tc_mma_bf16_pair(d + g * 128, a + 4, b + 4, idesc, 1u);
                        tc_mma_bf16_pair(d + g * 128, a + 6, b + 6, idesc, 1u);
                    }
                    tc_commit_pair(empty0 + 8 * s);
                    if (++s == static_cast<uint32_t>(p.stages)) { s = 0; ph ^= 1u; }
                }
                if (ok) tc_commit_pair(smem_u32(&ctl->acc_full[buf]));
            }
        }
    } else if (warp == 3) {
        if (kBwd && elect_one()) {
            // ------------------------------------------------------------ dY of this CTA's rows
            bool ok = true;
            uint32_t b = 0, ph = 1;
            for (int t = beg; t < end && ok; t += step) {
                const int tm = t / p.tiles_n, tn = t - tm * p.tiles_n;
                const uint32_t bar = smem_u32(&ctl->dy_full[b]);
                ok = mbar_wait(smem_u32(&ctl->dy_empty[b]), ph, abort_flag, p.status);
                if (!ok) break;
                mbar_expect_tx(bar, kTile);
                for (int c = 0; c < 4; ++c)
                    tma_load_3d(dys + b * kTile + static_cast<uint32_t>(c) * 4 * kWarpTile, &tmdY, bar, tn * 128 + c * 32, tm * 256 + static_cast<int>(rank) * 128, 0);
                if (++b == kDyTiles) { b = 0; ph ^= 1u; }
            }
        }
    } else {
        // ---------------------------------------------------------------- gate
        const int q = warp & 3, w = (warp - 4) >> 2;      // rows 32 q (the quadrant of tensor memory that the warp may touch)
        const int team = kTeams == 2 ? w >> 1 : 0;
        constexpr int kChunks = kTeams;                   // of 32 columns, side by side
        const int c0 = kTeams == 2 ? (w & 1) * 2 : w;
        const uint32_t lane_base = tmem + (static_cast<uint32_t>(q * 32) << 16) + c0 * 32;
        const uint32_t own = static_cast<uint32_t>(lane) * 64u, sw = (static_cast<uint32_t>(lane) >> 1) & 3u;
        const uint32_t panel = out + static_cast<uint32_t>(w * 4 + q) * (kWide ? 2 * kWarpTile : kWarpTile);
        const uint32_t dy_place = static_cast<uint32_t>(c0 * 4 + q) * kWarpTile;
        const __nv_bfloat16* const bias = static_cast<const __nv_bfloat16*>(p.bias);
        const uint32_t acc_empty_leader0 = map_to_cta(smem_u32(&ctl->acc_empty[0]), 0);
        bool ok = true;
        uint32_t j = static_cast<uint32_t>(team), dy = 0, dy_last = 0, dy_ph = 0;
        for (int t = beg + team * step; t < end && ok; t += kTeams * step, j += kTeams) {
            const int tm = t / p.tiles_n, row0 = tm * 256 + static_cast<int>(rank) * 128 + q * 32;
            const uint32_t buf = j & 1u;
            ok = mbar_wait_warp(smem_u32(&ctl->acc_full[buf]), (j >> 1) & 1u, abort_flag, p.status);
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int ch = 0; ch < kChunks; ++ch) {
                const int col0 = (t - tm * p.tiles_n) * 128 + (c0 + ch) * 32;
                float g[32], u[32];
                load_columns(lane_base + buf * 256 + ch * 32, g);
                load_columns(lane_base + buf * 256 + 128 + ch * 32, u);
                tmem_ld_wait();
                if (ch == kChunks - 1) tc_fence_before();
                __syncwarp();
                if (lane == 0 && ch == kChunks - 1) arrive_relaxed(acc_empty_leader0 + 8 * buf);
                if (bias) {
                    add_bias32(g, bias, col0, p.N, lane);
                    add_bias32(u, bias + p.bias_step, col0, p.N, lane);
                }
                const uint32_t mine = panel + own;
                if constexpr (!kBwd) {
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        const float2 v = split(gated2<kAct>(f2(g[e], g[e + 1]), f2(u[e], u[e + 1])));
                        g[e] = v.x;
                        g[e + 1] = v.y;
                    }
                    if (!kWide || ch == 0) {      // what was there before has left its place
                        if (lane == 0) tma_store_wait_read<0>();
                        __syncwarp();
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (kWide) st_shared_v4(panel + lane * 128u + ((static_cast<uint32_t>(4 * ch + i) ^ (lane & 7u)) << 4), pack_eight(g + 8 * i));
                        else st_shared_v4(mine + ((static_cast<uint32_t>(i) ^ sw) << 4), pack_eight(g + 8 * i));
                    }
                    if (kWide && ch == 0) continue;
                } else {
                    ok = mbar_wait_warp(smem_u32(&ctl->dy_full[dy]), dy_ph, abort_flag, p.status);
                    if (!ok) break;
                    const uint32_t dy_mine = dys + dy * kTile + dy_place + own;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t piece = (static_cast<uint32_t>(i) ^ sw) << 4;
                        const uint4 v = ld_shared_v4(dy_mine + piece);
                        const uint32_t ws[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int e = 0; e < 8; e += 2) {
                            const uint32_t two = ws[e >> 1];
                            F2 dg, du;
                            gated_grad2<kAct>(f2(g[8 * i + e], g[8 * i + e + 1]), f2(u[8 * i + e], u[8 * i + e + 1]),
                                              f2(__uint_as_float(two << 16), __uint_as_float(two & 0xffff0000u)), &dg, &du);
                            const float2 a = split(dg), b = split(du);
                            g[8 * i + e] = a.x;
                            g[8 * i + e + 1] = a.y;
                            u[8 * i + e] = b.x;
                            u[8 * i + e + 1] = b.y;
                        }
                    }
                    if (lane == 0) {      // the last tile's results have left their places, of which dY may have one
                        tma_store_wait_read<0>();
                        if (j > 0) mbar_arrive(smem_u32(&ctl->dy_empty[dy_last]));
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t piece = (static_cast<uint32_t>(i) ^ sw) << 4;
                        st_shared_v4(dy_mine + piece, pack_eight(g + 8 * i));
                        st_shared_v4(mine + piece, pack_eight(u + 8 * i));
                    }
                }
                if (kBwd || p.y == nullptr) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        if constexpr (kWide) {
                            if (row0 < p.M && col0 - 32 < p.N) tma_store_3d(&tmOut, panel, col0 - 32, row0, 0);
                        } else if (row0 < p.M && col0 < p.N) {
                            if constexpr (kBwd) tma_store_3d(&tmOut, dys + dy * kTile + dy_place, col0, row0, 0);
                            tma_store_3d(&tmOut, panel, col0, row0, kBwd ? 1 : 0);
                        }
                        tma_store_commit();
                    }
                    if (kBwd) {
                        dy_last = dy;
                        if (++dy == kDyTiles) { dy = 0; dy_ph ^= 1u; }
                    }
                } else {
                    __syncwarp();
                    if (col0 < p.N) store_any(panel, p.y, p.ldy, row0, col0, p.M, p.N, lane);
                    __syncwarp();
                }
            }
        }
        if (lane == 0) tma_store_wait_read<0>();
    }
    // Where a wait has run out, copies and products may be under way, on whose barriers nothing can be built any more: they are given a millisecond (a thousand times what
    // one takes) before this CTA's memory and its partner's are free.
    if (*abort_flag) {
        const long long t0 = clock64();
        while (clock64() - t0 < kWaitCycleLimit / 2000) {}
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();          // neither CTA leaves (or frees tensor memory) while the other may still signal it
    if (warp == 1) {
        __syncwarp();
        tmem_dealloc_pair(tmem, 512);
    }
}

// Maps of y, dY and dZ: boxes of 32 columns (64 bytes, the span of the exchange of pieces) x box_rows rows of one matrix.
bool cached_map_half(CUtensorMap* map, const void* p, int64_t groups, int64_t rows, int64_t cols, int64_t ld, int64_t gs, int box_rows) {
    return cached_map(map, MapKey{p, {groups, rows, cols, ld, gs, box_rows, -8, 0}}, [&](EncodeTiledFn fn) {
        const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(groups)};
        const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(gs) * 2};
        const cuuint32_t box[3] = {32u, static_cast<cuuint32_t>(box_rows), 1u}, estr[3] = {1u, 1u, 1u};
        return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    });
}

template <bool kResident, bool kBwd, bool kWide>
int gated_launch(int act, const CUtensorMap (&maps)[4], const GatedParams& p, cudaStream_t stream) {
    void (*kernel)(CUtensorMap, CUtensorMap, CUtensorMap, CUtensorMap, GatedParams) =
        act == PF_GATE_SILU ? tc_gated_kernel<kResident, kBwd, PF_GATE_SILU, kWide> : act == PF_GATE_GELU ? tc_gated_kernel<kResident, kBwd, PF_GATE_GELU, kWide>
        : act == PF_GATE_SIGMOID ? tc_gated_kernel<kResident, kBwd, PF_GATE_SIGMOID, kWide> : tc_gated_kernel<kResident, kBwd, PF_GATE_RELU, kWide>;
    const size_t smem = 2048 + kRoom;
    if (allow_smem(kernel, smem) != cudaSuccess) return PF_ERR_CUDA;
    const int pairs = std::min(p.total, num_sms() / 2);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(pairs * 2)); cfg.blockDim = dim3(kGatedThreads); cfg.dynamicSmemBytes = smem; cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, kernel, maps[0], maps[1], maps[2], maps[3], p) != cudaSuccess) return PF_ERR_CUDA;
    count_launch();
    return PF_OK;
}

}  // namespace

int gated(const GatedArgs& a, cudaStream_t stream) {
    const int64_t tiles_n = ceil_div(a.n, 128), total = ceil_div(a.m, 256) * tiles_n;
    if (total > 0x7fffffff || a.m > 0x7fffffff || a.n > 0x7fffffff) return PF_ERR_UNSUPPORTED;
    const bool bwd = a.dY != nullptr, direct = bwd || tma_out(a.y, a.ldy, a.n);
    CUtensorMap maps[4];
    bool ok = cached_map_3d(&maps[0], a.T, 2, a.m, a.r, a.ldt, a.st, 128) && cached_map_3d(&maps[1], a.V, 2, a.n, a.r, a.ldv, a.sv, 64);
    maps[2] = maps[3] = maps[0];
    const int nkb = static_cast<int>(ceil_div(a.r, 64));
    const bool resident = !bwd && nkb <= 4, wide = !bwd && direct && nkb <= 3;      // (as far as three stages or more are left)
    if (ok && wide) ok = cached_map_3d(&maps[2], a.y, 1, a.m, a.n, a.ldy, 0, 32);
    else if (ok && direct) ok = cached_map_half(&maps[2], a.y, bwd ? 2 : 1, a.m, a.n, a.ldy, bwd ? a.sz : a.m * a.ldy, 32);
    if (ok && bwd) ok = cached_map_half(&maps[3], a.dY, 1, a.m, a.n, a.lddy, a.m * a.lddy, 128);
    if (!ok) return PF_ERR_CUDA;
    GatedParams p = {};
    p.M = static_cast<int>(a.m); p.N = static_cast<int>(a.n);
    p.nkb = nkb;
    p.tiles_n = static_cast<int>(tiles_n); p.total = static_cast<int>(total);
    p.bias = a.bias; p.bias_step = a.n;
    p.y = direct ? nullptr : static_cast<__nv_bfloat16*>(a.y); p.ldy = a.ldy;
    p.status = device_status_ptr();
    // what y, or dY and dZ1, leave: a resident T takes 32 KB for 64 contraction elements, a stage 16 (with T 48).  (Backward, with a resident T: 99 us, so 97 at 16384 x 4096
    // over 128; over 256 there is no room, and runs of neighbouring tiles took 131, every pairs-th 120.)
    const int room = static_cast<int>((kRoom - (bwd ? 1 + kDyTiles : wide ? 2 : 1) * kTile) / 16384);
    p.stages = resident ? std::min(kGatedStages, room - 2 * nkb) : room / 3;
    if (bwd) return gated_launch<false, true, false>(a.act, maps, p, stream);
    if (wide) return gated_launch<true, false, true>(a.act, maps, p, stream);
    return resident ? gated_launch<true, false, false>(a.act, maps, p, stream) : gated_launch<false, false, false>(a.act, maps, p, stream);
}

}  // namespace tc
}  // namespace pf
