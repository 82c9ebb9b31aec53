// Gated factorized layers, y = act(x U0 V0^T + b0) * (x U1 V1^T + b1), forward and backward.
//
// bf16: T = x U for both pairs in one launch, then both second products with the gate in one (pf_tc_gated.cu); the gate's operands never
// reach memory; T, and backward dZ, are rounded to bf16, as the tensor cores read them (and as in the factorized layers beside this one).
// Matrices that TMA cannot read are copied first.
// fp32: both pairs' products beside one another (pf_tc_f32.cu) for some rows at a time and the gate over their results, which then still are in L2; the smallest
// ones, those that TMA cannot read, and bf16 layers wider than 2^22 by the grouped layer (bf16: g and u are rounded on the way).
// Backward: the gate's operands again, dZ of both pairs, then the gradients of both.
#include <algorithm>

#include "pf_internal.h"
#include "pf_tc.h"
#include "pf_tc_gated.cuh"

namespace pf {
namespace {

struct GateParams {
    void* z;                 // [2, rows, ldz]: g and u; backward: becomes dZ
    const void* bias;
    const void* dY;
    void* y;
    int64_t ldz, sz, lddy, ldy, rows;
    int cols;
};
__device__ __forceinline__ float get(const float* p) { return *p; }
__device__ __forceinline__ float get(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// Bound by L2: three or five numbers read and written for each output.
template <typename T, int kAct, bool kBwd>
__global__ void __launch_bounds__(256) gate_kernel(const GateParams p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    T* const z0 = static_cast<T*>(p.z);
    T* const z1 = z0 + p.sz;
    const T* const bias = static_cast<const T*>(p.bias);
    const T* const dY = static_cast<const T*>(p.dY);
    T* const y = static_cast<T*>(p.y);
    for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y)
        for (int c = blockIdx.x * 256 + threadIdx.x; c < p.cols; c += gridDim.x * 256) {
            const float g = get(z0 + row * p.ldz + c) + (bias ? get(bias + c) : 0.f), u = get(z1 + row * p.ldz + c) + (bias ? get(bias + p.cols + c) : 0.f);
            if constexpr (kBwd) {
                float value, slope;
                gate_slope<kAct, true>(g, &value, &slope);
                const float dy = get(dY + row * p.lddy + c);
                put(z0 + row * p.ldz + c, dy * slope * u);
                put(z1 + row * p.ldz + c, dy * value);
            } else {
                put(y + row * p.ldy + c, gate<kAct>(g) * u);
            }
        }
}
template <typename T, bool kBwd>
cudaError_t gate_launch(int act, const GateParams& p, cudaStream_t stream) {
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(ceil_div(p.cols, 256), 1024)), static_cast<unsigned>(std::min<int64_t>(p.rows, 4096)));
    const auto kernel = act == PF_GATE_SILU ? gate_kernel<T, PF_GATE_SILU, kBwd> : act == PF_GATE_GELU ? gate_kernel<T, PF_GATE_GELU, kBwd>
                        : act == PF_GATE_SIGMOID ? gate_kernel<T, PF_GATE_SIGMOID, kBwd> : gate_kernel<T, PF_GATE_RELU, kBwd>;
    return launch_beside(kernel, grid, 256, 0, 1, stream, p);
}
template <bool kBwd>
cudaError_t gate_any(int dtype, int act, const GateParams& p, cudaStream_t stream) {
    return dtype == PF_BF16 ? gate_launch<__nv_bfloat16, kBwd>(act, p, stream) : gate_launch<float, kBwd>(act, p, stream);
}

// Rows at a time of what does not take the tensor cores' gate: both results of at most 2^23 elements each.
int64_t rows_at_once(int64_t m, int64_t n) { return std::max<int64_t>(1, std::min(m, std::max<int64_t>(128, (1LL << 23) / n / 128 * 128))); }
int64_t z_pitch(int64_t n) { return (n + 7) / 8 * 8; }

struct GatedWs {
    size_t off_grouped, off_z, off_sums, total;
};
int64_t t_pitch(int64_t r, int dtype) { return dtype == PF_BF16 ? tc::gated_t_pitch(r) : (r + 7) / 8 * 8; }
bool on_tensor_cores(int64_t k, int64_t n, int64_t r, int dtype) { return dtype == PF_BF16 && tc::gated_fits(k, n, r); }
GatedWs gated_ws(int64_t m, int64_t k, int64_t n, int64_t r, int dtype, bool bwd) {
    GatedWs w = {};
    const int64_t rows = rows_at_once(m, n);
    const bool fused = on_tensor_cores(k, n, r, dtype);
    size_t grouped = 0;
    size_t off = align_up(static_cast<size_t>(2) * m * t_pitch(r, dtype) * dtype_size(dtype), 256);      // T
    w.off_grouped = off;
    if (fused) {
        grouped = tc::gated_first_workspace(m, k, n, r);
    } else {
        for (const int64_t part : {rows, m % rows}) grouped = std::max(grouped, pf_lowrank_linear_grouped_workspace(2, part, k, n, r, dtype, 0));
        if (dtype == PF_F32) {
            for (const int64_t part : {rows, m % rows}) grouped = std::max(grouped, tc::f32_gated_workspace(part, k, n, r, false));
            if (bwd) grouped = std::max(grouped, tc::f32_gated_workspace(m, k, n, r, true));
        }
    }
    if (bwd) grouped = std::max(grouped, pf_lowrank_linear_grouped_workspace(2, m, k, n, r, dtype, 1));
    off += align_up(grouped, 256);
    w.off_z = off;
    if (bwd || !fused) off += align_up(static_cast<size_t>(2) * (bwd ? m : rows) * z_pitch(n) * dtype_size(dtype), 256);
    w.off_sums = off;
    if (bwd) off += align_up(sizeof(float) * act_bwd_chunks(m) * static_cast<size_t>(n), 256);
    w.total = off;
    return w;
}

struct Matrices {
    const void* x;
    int64_t ldx;
    const void* U;
    int64_t ldu, su;
    const void* V;
    int64_t ldv, sv;
    int64_t m, k, n, r;
    int dtype;
};
int validate_gated(const Matrices& a, int act, const void* bias) {
    if (!valid_dtype(a.dtype) || a.m < 0 || a.k < 1 || a.n < 1 || a.r < 1 || a.su < 0 || a.sv < 0) return PF_ERR_INVALID_ARG;
    if (act < PF_GATE_SILU || act > PF_GATE_RELU) return PF_ERR_INVALID_ARG;
    if ((!a.x && a.m > 0) || !a.U || !a.V || a.ldx < a.k || a.ldu < a.r || a.ldv < a.r) return PF_ERR_INVALID_ARG;
    if (!elem_aligned(a.x, a.dtype) || !elem_aligned(a.U, a.dtype) || !elem_aligned(a.V, a.dtype) || !elem_aligned(bias, a.dtype)) return PF_ERR_INVALID_ARG;
    if (a.m > (1LL << 30) || a.k > (1LL << 30) || a.n > (1LL << 30) || a.r > (1LL << 20)) return PF_ERR_UNSUPPORTED;
    if (a.su < (a.k - 1) * a.ldu + a.r || a.sv < (a.n - 1) * a.ldv + a.r) return PF_ERR_INVALID_ARG;
    return PF_OK;
}
bool stash_valid(const void* T, int64_t ldt, int64_t st, const Matrices& a) {
    return !T || (ldt >= a.r && elem_aligned(T, a.dtype) && (a.m == 0 || st >= (a.m - 1) * ldt + a.r));
}
const void* moved(const void* p, int64_t elems, int dtype) { return static_cast<const char*>(p) + elems * static_cast<int64_t>(dtype_size(dtype)); }
void* moved(void* p, int64_t elems, int dtype) { return static_cast<char*>(p) + elems * static_cast<int64_t>(dtype_size(dtype)); }

tc::GroupedArgs grouped_args(const Matrices& a, const void* T, int64_t ldt, int64_t st, char* ws, cudaStream_t stream) {
    tc::GroupedArgs g;
    g.groups = 2; g.x = a.x; g.ldx = a.ldx; g.U = a.U; g.ldu = a.ldu; g.su = a.su; g.V = a.V; g.ldv = a.ldv; g.sv = a.sv;
    g.T = const_cast<void*>(T); g.ldt = ldt; g.st = st; g.m = a.m; g.k = a.k; g.n = a.n; g.r = a.r; g.ws = ws; g.stream = stream;
    return g;
}
// z [2, a.m, ldz] of both pairs, sz elements apart, by the grouped layer or both pairs at once.  need_t: T is to be computed (kept, if it is not null), else it is given.
int both_pairs(const Matrices& a, void* T, int64_t ldt, int64_t st, bool need_t, void* z, int64_t ldz, int64_t sz, char* ws, size_t room, cudaStream_t stream) {
    if (a.dtype == PF_F32 && !small::f32_fits(a.m, a.k, a.n, a.r, false)) {
        tc::GroupedArgs g = grouped_args(a, T, ldt, st, ws, stream);
        g.y = z; g.ldy = ldz; g.sy = sz;
        int handled = 0;
        const int rc = tc::f32_gated_fwd(g, need_t, &handled);
        if (rc != PF_OK || handled) return rc;
    }
    return pf_lowrank_linear_grouped_fwd(2, a.x, a.ldx, 0, a.U, a.ldu, a.su, a.V, a.ldv, a.sv, z, ldz, sz, need_t ? T : nullptr, ldt, st, a.m, a.k, a.n, a.r, a.dtype, ws,
                                         room, stream);
}

}  // namespace
}  // namespace pf

using namespace pf;

extern "C" {

size_t pf_lowrank_linear_gated_workspace(int64_t m, int64_t k, int64_t n, int64_t r, int dtype, int is_bwd) {
    if (!valid_dtype(dtype) || m < 0 || k < 1 || n < 1 || r < 1 || m > (1LL << 30) || k > (1LL << 30) || n > (1LL << 30) || r > (1LL << 20)) return 0;
    return gated_ws(m, k, n, r, dtype, is_bwd != 0).total;
}

int pf_lowrank_linear_gated_fwd(const void* x, int64_t ldx, const void* U, int64_t ldu, int64_t su, const void* V, int64_t ldv, int64_t sv,
                                const void* bias, int act, void* y, int64_t ldy, void* T_stash, int64_t ldt, int64_t st, int64_t m, int64_t k, int64_t n,
                                int64_t r, int dtype, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const Matrices a = {x, ldx, U, ldu, su, V, ldv, sv, m, k, n, r, dtype};
    int rc = validate_gated(a, act, bias);
    if (rc != PF_OK) return rc;
    if ((!y && m > 0) || ldy < n || !elem_aligned(y, dtype) || !stash_valid(T_stash, ldt, st, a)) return PF_ERR_INVALID_ARG;
    const GatedWs w = gated_ws(m, k, n, r, dtype, false);
    rc = check_ws(workspace, workspace_bytes, w.total);
    if (rc != PF_OK || m == 0) return rc;
    char* const ws = static_cast<char*>(workspace);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (on_tensor_cores(k, n, r, dtype)) {
        const tc::GroupedArgs g = grouped_args(a, T_stash, ldt, st, ws + w.off_grouped, stream);
        tc::GatedArgs ga;
        int handled = 0;
        rc = tc::gated_first(g, true, ws, nullptr, 0, &ga, &handled);
        if (rc != PF_OK || !handled) return rc != PF_OK ? rc : PF_ERR_CUDA;      // (a driver without tensor maps)
        ga.bias = bias; ga.act = act; ga.y = y; ga.ldy = ldy;
        return tc::gated(ga, stream);
    }
    const int64_t rows = rows_at_once(m, n), ldz = z_pitch(n);
    void* const z = ws + w.off_z;
    for (int64_t i = 0; i < m; i += rows) {
        const int64_t part = std::min(rows, m - i);
        Matrices some = a;
        some.x = moved(x, i * ldx, dtype);
        some.m = part;
        rc = both_pairs(some, T_stash ? moved(T_stash, i * ldt, dtype) : nullptr, ldt, st, true, z, ldz, part * ldz, ws + w.off_grouped, w.off_z - w.off_grouped, stream);
        if (rc != PF_OK) return rc;
        const GateParams p = {z, bias, nullptr, moved(y, i * ldy, dtype), ldz, part * ldz, 0, ldy, part, static_cast<int>(n)};
        PF_CUDA(gate_any<false>(dtype, act, p, stream));
    }
    return PF_OK;
}

int pf_lowrank_linear_gated_bwd(const void* x, int64_t ldx, const void* U, int64_t ldu, int64_t su, const void* V, int64_t ldv, int64_t sv,
                                const void* bias, int act, const void* dY, int64_t lddy, const void* T_stash, int64_t ldt, int64_t st, void* dX,
                                int64_t lddx, void* dU, int64_t lddu, int64_t sdu, void* dV, int64_t lddv, int64_t sdv, void* dbias, int64_t m, int64_t k,
                                int64_t n, int64_t r, int dtype, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const Matrices a = {x, ldx, U, ldu, su, V, ldv, sv, m, k, n, r, dtype};
    int rc = validate_gated(a, act, bias);
    if (rc != PF_OK) return rc;
    if ((!dY && m > 0) || lddy < n || !elem_aligned(dY, dtype) || !stash_valid(T_stash, ldt, st, a)) return PF_ERR_INVALID_ARG;
    if (!dU || lddu < r || !elem_aligned(dU, dtype) || sdu < (k - 1) * lddu + r || !dV || lddv < r || !elem_aligned(dV, dtype) || sdv < (n - 1) * lddv + r ||
        (dX && (lddx < k || !elem_aligned(dX, dtype))) || !elem_aligned(dbias, dtype))
        return PF_ERR_INVALID_ARG;
    const GatedWs w = gated_ws(m, k, n, r, dtype, true);
    rc = check_ws(workspace, workspace_bytes, w.total);
    if (rc != PF_OK) return rc;
    char* const ws = static_cast<char*>(workspace);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    void* const z = ws + w.off_z;
    const int64_t ldz = z_pitch(n), sz = m * ldz;
    const void* T = T_stash;
    if (m > 0) {
        if (on_tensor_cores(k, n, r, dtype)) {
            tc::GroupedArgs g = grouped_args(a, T_stash, ldt, st, ws + w.off_grouped, stream);
            g.dY = dY; g.lddy = lddy;
            tc::GatedArgs ga;
            int handled = 0;
            rc = tc::gated_first(g, !T_stash, ws, z, ldz, &ga, &handled);      // (a copy of dY in the place of dZ0: the gate reads each tile of it before it writes that)
            if (rc != PF_OK || !handled) return rc != PF_OK ? rc : PF_ERR_CUDA;
            ga.bias = bias; ga.act = act; ga.y = z; ga.ldy = ldz; ga.sz = sz;
            rc = tc::gated(ga, stream);
            if (rc != PF_OK) return rc;
            T = ga.T; ldt = ga.ldt; st = ga.st;
        } else {
            const int64_t rows = rows_at_once(m, n);
            if (!T_stash) { T = ws; ldt = t_pitch(r, dtype); st = m * ldt; }
            for (int64_t i = 0; i < m; i += rows) {
                const int64_t part = std::min(rows, m - i);
                Matrices some = a;
                some.x = moved(x, i * ldx, dtype);
                some.m = part;
                rc = both_pairs(some, const_cast<void*>(moved(T, i * ldt, dtype)), ldt, st, !T_stash, moved(z, i * ldz, dtype), ldz, sz, ws + w.off_grouped,
                                w.off_z - w.off_grouped, stream);
                if (rc != PF_OK) return rc;
                const GateParams p = {moved(z, i * ldz, dtype), bias, moved(dY, i * lddy, dtype), nullptr, ldz, sz, lddy, 0, part, static_cast<int>(n)};
                PF_CUDA(gate_any<true>(dtype, act, p, stream));
            }
        }
    }
    if (dbias) {
        for (int g = 0; g < 2; ++g) {
            void* const db = moved(dbias, g * n, dtype);
            if (m == 0) PF_CUDA(cudaMemsetAsync(db, 0, n * dtype_size(dtype), stream));
            else PF_CUDA(act_bwd(nullptr, 0, moved(z, g * sz, dtype), ldz, db, m, n, PF_ACT_NONE, dtype, reinterpret_cast<float*>(ws + w.off_sums), stream));
        }
    }
    if (dtype == PF_F32 && m > 0 && !small::f32_fits(m, k, n, r, true)) {
        tc::GroupedArgs g = grouped_args(a, T, ldt, st, ws + w.off_grouped, stream);
        g.dY = z; g.lddy = ldz; g.sdy = sz; g.dX = dX; g.lddx = lddx; g.dU = dU; g.lddu = lddu; g.sdu = sdu; g.dV = dV; g.lddv = lddv; g.sdv = sdv;
        int handled = 0;
        rc = tc::f32_gated_bwd(g, &handled);
        if (rc != PF_OK || handled) return rc;
    }
    return pf_lowrank_linear_grouped_bwd(2, x, ldx, 0, U, ldu, su, V, ldv, sv, z, ldz, sz, T, ldt, st, dX, lddx, 0, dU, lddu, sdu, dV, lddv, sdv, m, k, n, r,
                                         dtype, ws + w.off_grouped, w.off_z - w.off_grouped, cuda_stream);
}

}  // extern "C"
