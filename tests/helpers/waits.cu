// waits.cu -- what jb_tcgen05.cuh does when a wait is not served and when products are waited for at the end, and shared memory
// left full of a pattern, for the tests.
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

// 64 products of tiles of ones, 128 x 64 by 64 columns, issued by the elected lane and drained: every sum is 64 x 64, and out[i]
// what lane i of the first warp reads right after the drain.
__global__ void drain_kernel(float* out) {
    extern __shared__ char dynamic[];
    __shared__ unsigned long long bar;
    __shared__ uint32_t tmem;
    const uint32_t tiles = (jb::shared_address(dynamic) + 1023) & ~1023u;  // 128 rows of 128 bytes, then 64
    uint32_t* words = reinterpret_cast<uint32_t*>(dynamic + (tiles - jb::shared_address(dynamic)));
    for (int i = threadIdx.x; i < 192 * 32; i += blockDim.x) words[i] = 0x3F803F80u;
    if (threadIdx.x == 0) {
        jb::barrier_init(jb::shared_address(&bar), 1);
        jb::barriers_initialized();
    }
    if (threadIdx.x < 32) jb::tmem_alloc(jb::shared_address(&tmem), 64);
    jb::shared_to_async_proxy();
    jb::tc_fence_before();
    __syncthreads();
    jb::tc_fence_after();
    if (threadIdx.x < 32) {
        const uint32_t d = jb::same(tmem), a = jb::tile_descriptor(tiles, 16), b = jb::tile_descriptor(tiles + 128 * 128, 16);
        for (int i = 0; i < 64; ++i) {
            if (jb::elected())
                for (int k = 0; k < 4; ++k) jb::tc_product(d, a + 2 * k, b + 2 * k, jb::product_descriptor(64, false), i > 0 || k > 0);
            __syncwarp();
        }
        jb::tc_drain(jb::shared_address(&bar));
        jb::tc_fence_after();
        uint32_t x[32];
        jb::tmem_load32(d, x);
        jb::tc_wait_loads();
        float sum = 0.0f;
        for (int i = 0; i < 32; ++i) sum += __uint_as_float(x[i]);
        out[threadIdx.x] = sum / 32;
        jb::tc_fence_before();
        __syncwarp();
        jb::tmem_free(tmem, 64);
    }
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

EXPORT int drained_products(float* out) {
    constexpr int kBytes = 1024 + 192 * 128;
    drain_kernel<<<1, 128, kBytes>>>(out);
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
