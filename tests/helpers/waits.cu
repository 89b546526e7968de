// waits.cu -- what jb_tcgen05.cuh does when a wait is not served, and shared memory left full of a pattern, for the tests.
#include <cstdint>

#include <cuda_runtime.h>

#include "jb_tcgen05.cuh"

namespace {

// A barrier that nobody arrives at. out: what the wait said, *failed after it, cycles of it; of the longest of 32 looks; of a
// second wait, which finds *failed set; what that one said.
__global__ void unserved_kernel(long long* out) {
    __shared__ unsigned long long bar;
    __shared__ int failed;
    if (threadIdx.x == 0) {
        jb::barrier_init(jb::shared_address(&bar), 1);
        jb::barriers_initialized();
        failed = 0;
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    const uint32_t at = jb::shared_address(&bar);
    long long look = 0;
    for (int i = 0; i < 32; ++i) {
        const long long a = clock64();
        if (jb::barrier_sleep(at, 0)) failed = 2;  // what it says is asked for, or nothing waits for it
        look = max(look, clock64() - a);
    }
    const long long b = clock64();
    const bool first = jb::barrier_wait(at, 0, &failed);
    const long long c = clock64();
    const int after = *static_cast<volatile int*>(&failed);
    const bool second = jb::barrier_wait(at, 0, &failed);
    const long long d = clock64();
    out[0] = first;
    out[1] = after;
    out[2] = c - b;
    out[3] = look;
    out[4] = d - c;
    out[5] = second;
}

__global__ void fill_kernel(uint32_t pattern, int words) {
    extern __shared__ uint32_t all[];
    for (int i = threadIdx.x; i < words; i += blockDim.x) static_cast<volatile uint32_t*>(all)[i] = pattern;
}

}  // namespace

#define EXPORT extern "C" __attribute__((visibility("default")))

EXPORT int unserved_wait(long long* out) {
    unserved_kernel<<<1, 32>>>(out);
    return static_cast<int>(cudaGetLastError());
}

// All of every SM's shared memory that a CTA can have.
EXPORT int fill_shared(uint32_t pattern) {
    constexpr int kBytes = 227 * 1024;
    cudaError_t e = cudaFuncSetAttribute(fill_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e != cudaSuccess) return static_cast<int>(e);
    fill_kernel<<<152 * 4, 1024, kBytes>>>(pattern, kBytes / 4);
    return static_cast<int>(cudaGetLastError());
}
