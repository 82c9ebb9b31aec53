// The kernels over a vocabulary's rows with waits that run out: in some blocks the last copy of a row is expected to bring 16 bytes more than it does, so that what
// waits for it gives up.  The copies themselves, and all accesses, are as they always are.
#include "pf_tc_prims.cuh"

namespace pf {
namespace tc {
constexpr uint32_t kWholeChunk = 16384;      // of 256 threads
__device__ __forceinline__ void mbar_expect_some(uint32_t bar, uint32_t bytes) {
    mbar_expect_tx(bar, bytes + (blockIdx.x % 64 == 5 && bytes < kWholeChunk ? 16 : 0));
}
}  // namespace tc
}  // namespace pf

#define mbar_expect_tx mbar_expect_some
#include "pf_vocab.cu"
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

// The status of what has run, which is cleared; -1: an error.
extern "C" int waits_status(void) {
    unsigned int v = 0;
    const unsigned int zero = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&v, pf::g_waits_status, sizeof(v)) != cudaSuccess ||
        cudaMemcpyToSymbol(pf::g_waits_status, &zero, sizeof(zero)) != cudaSuccess)
        return -1;
    return static_cast<int>(v);
}
