// The gate of a gated layer with waits that run out: in some pairs of blocks copies are expected to bring 16 bytes more than they do, so that what waits for them
// gives up.  The copies themselves, and all accesses, are as they always are.
#include "pf_tc_pair_prims.cuh"

namespace pf {
namespace tc {
__device__ __forceinline__ void mbar_expect_some(uint32_t bar, uint32_t bytes) { mbar_expect_tx(bar, bytes + (blockIdx.x % 64 == 4 ? 16 : 0)); }
}  // namespace tc
}  // namespace pf

#define mbar_expect_tx mbar_expect_some
#include "pf_tc_gated.cu"
#undef mbar_expect_tx

// What the library has elsewhere.
namespace pf {
__device__ unsigned int g_waits_status;
void count_launch(int) {}
unsigned int* device_status_ptr() {
    void* p = nullptr;
    return cudaGetSymbolAddress(&p, g_waits_status) == cudaSuccess ? static_cast<unsigned int*>(p) : nullptr;
}
}  // namespace pf

// T [2, m, r], V [2, n, r] (r a multiple of 8), dY [m, n] or null, out: y [m, n] or dZ [2, m, n].
extern "C" int waits_gated(const void* T, const void* V, const void* dY, void* out, long long m, long long n, long long r) {
    pf::tc::GatedArgs a;
    a.T = T; a.ldt = r; a.st = m * r; a.V = V; a.ldv = r; a.sv = n * r; a.m = m; a.n = n; a.r = r;
    a.dY = dY; a.lddy = n; a.act = PF_GATE_SILU; a.y = out; a.ldy = n; a.sz = m * n;
    return pf::tc::gated(a, nullptr);
}
// The status of what has run, which is cleared; -1: an error.
extern "C" int waits_status(void) {
    unsigned int v = 0;
    const unsigned int zero = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&v, pf::g_waits_status, sizeof(v)) != cudaSuccess ||
        cudaMemcpyToSymbol(pf::g_waits_status, &zero, sizeof(zero)) != cudaSuccess)
        return -1;
    return static_cast<int>(v);
}
