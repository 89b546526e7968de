// jb_tcgen05.cuh -- mbarriers, asynchronous copies and the fifth generation's tensor-core instructions as functions.
#pragma once
#include <cstdint>

#include <cuda_runtime.h>

namespace jb {

__device__ __forceinline__ uint32_t shared_address(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// --- mbarriers ---------------------------------------------------------------------------

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barriers_initialized() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void barrier_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Whether the phase of this parity has ended; the thread may sleep for up to about a millisecond before it says no.
__device__ __forceinline__ bool barrier_sleep(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 1000000;\n selp.u32 %0, 1, 0, p;\n}"
        : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
// Waits for the phase of this parity to end. A wait of over about two seconds gives up and sets *failed, and one that finds it
// set gives up after a look: then the roles of the CTA leave their loops, or go through the rest of them, a look a wait, where
// other warps need their part in a barrier. Few polls: those of waiting warps took 40 % of all instructions without sleep and
// with a look at the clock each.
constexpr long long kPatience = 4000000000ll;  // cycles
static __device__ __noinline__ bool barrier_wait_long(uint32_t bar, uint32_t parity, volatile int* failed) {
    const long long start = clock64();
    for (;;) {
        if (*failed) return false;
        for (int i = 0; i < 32; ++i)
            if (barrier_sleep(bar, parity)) return true;
        if (clock64() - start > kPatience) {
            *failed = 1;
            return false;
        }
    }
}
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, volatile int* failed) {
    return barrier_sleep(bar, parity) || barrier_wait_long(bar, parity, failed);
}

// The same for a wait that may end some hundred cycles late: the warp sleeps between its looks and leaves the others' issue
// slots alone (a sixth of all instructions were looks of warps that had nothing else to do).
__device__ __forceinline__ bool barrier_wait_idle(uint32_t bar, uint32_t parity, volatile int* failed) {
    for (int i = 0; i < 64; ++i) {
        uint32_t done;
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
            : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done != 0) return true;
        __nanosleep(128);
    }
    return barrier_wait(bar, parity, failed);
}

// A value that all lanes have, told to the compiler to be so: what products take is then formed once for the warp and not
// moved over from lanes for each of them (a product took 75 cycles of its warp without).
__device__ __forceinline__ int same(int x) { return __shfl_sync(0xFFFFFFFFu, x, 0); }
__device__ __forceinline__ uint32_t same(uint32_t x) { return __shfl_sync(0xFFFFFFFFu, x, 0); }

// True in one lane of a converged warp: what it alone does keeps its operands the same for the whole warp.
__device__ __forceinline__ bool elected() {
    uint32_t e;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xFFFFFFFF;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(e));
    return e != 0;
}

// --- copies ------------------------------------------------------------------------------

// Announces a copy's bytes at the barrier and arrives there; the phase ends when they have come, too.
__device__ __forceinline__ void barrier_arrive_bytes(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void barrier_arrive_count(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
// A box of a tensor with four dimensions, the first one contiguous; x times the element's size is a multiple of 16 bytes.
__device__ __forceinline__ void copy_box(uint32_t to, const void* map, int x, int y, int z, int w, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(to),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
                 : "memory");
}
// What this thread wrote to shared memory becomes visible to the tensor cores' reads.
__device__ __forceinline__ void shared_to_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// --- tensor memory and products ------------------------------------------------------------

__device__ __forceinline__ void tmem_alloc(uint32_t to, uint32_t columns) {  // a warp
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns) {  // the same warp
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_loads() { __syncwarp(); asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_stores() { __syncwarp(); asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// An arrival at `bar` when all products that this thread has issued are done.
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Waits for all products that the warp has issued, which a commit knows of in the lane that issued them: the elected one, the same
// at each time. The whole warp; a barrier with one arrival that nothing else uses.
__device__ __forceinline__ void tc_drain(uint32_t bar) {
    __syncwarp();
    if (elected()) {
        int late = 0;
        tc_commit(bar);
        barrier_wait(bar, 0, &late);
    }
    __syncwarp();
}

// A tile in shared memory with rows of 128 bytes, 16-byte pieces of row r at (piece ^ r % 8), 1024-byte aligned: the lower
// word of its descriptor, to which bytes / 16 can be added; the upper word is the same for all. `leading`: bytes from one
// 64-element panel to the next where the panels' direction is not the product's (unused otherwise).
__device__ __forceinline__ uint32_t tile_descriptor(uint32_t at, uint32_t leading) { return (leading >> 4) << 16 | at >> 4; }
constexpr uint32_t kTileDescriptor = (1024u >> 4) | 1u << 14 | 2u << 29;  // eight rows, version, swizzle of 128 bytes

// bf16 products with fp32 sums, M = 128: N columns; `across`: B's rows in memory are its product's summed index.
__host__ __device__ constexpr uint32_t product_descriptor(int n, bool across) {
    return 1u << 4 | 1u << 7 | 1u << 10 | (across ? 1u << 16 : 0u) | static_cast<uint32_t>(n >> 3) << 17 | (128u >> 4) << 24;
}
// D = A B (+ D): A and B in shared memory; 16 summed elements.
__device__ __forceinline__ void tc_product(uint32_t d, uint32_t a, uint32_t b, uint32_t how, bool add) {
    asm volatile(
        "{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.b32 p, %5, 0;\n mov.b64 a, {%1, %4};\n mov.b64 b, {%2, %4};\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}" ::"r"(d), "r"(a), "r"(b), "r"(how), "r"(kTileDescriptor), "r"(static_cast<uint32_t>(add))
        : "memory");
}
// The same with A in tensor memory, two elements a column.
__device__ __forceinline__ void tc_product_from_tmem(uint32_t d, uint32_t a, uint32_t b, uint32_t how, bool add) {
    asm volatile(
        "{\n .reg .pred p;\n .reg .b64 b;\n setp.ne.b32 p, %5, 0;\n mov.b64 b, {%2, %4};\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}" ::"r"(d), "r"(a), "r"(b), "r"(how), "r"(kTileDescriptor), "r"(static_cast<uint32_t>(add))
        : "memory");
}

// These are the whole warp's: lanes that took another way have to be back.
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t* x) {
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
        "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]), "=r"(x[8]), "=r"(x[9]), "=r"(x[10]),
          "=r"(x[11]), "=r"(x[12]), "=r"(x[13]), "=r"(x[14]), "=r"(x[15]), "=r"(x[16]), "=r"(x[17]), "=r"(x[18]), "=r"(x[19]), "=r"(x[20]),
          "=r"(x[21]), "=r"(x[22]), "=r"(x[23]), "=r"(x[24]), "=r"(x[25]), "=r"(x[26]), "=r"(x[27]), "=r"(x[28]), "=r"(x[29]), "=r"(x[30]), "=r"(x[31])
        : "r"(at));
}
__device__ __forceinline__ void tmem_store32(uint32_t at, const uint32_t* x) {
    __syncwarp();
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
        "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(at),
        "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]), "r"(x[10]), "r"(x[11]),
        "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]), "r"(x[16]), "r"(x[17]), "r"(x[18]), "r"(x[19]), "r"(x[20]), "r"(x[21]), "r"(x[22]),
        "r"(x[23]), "r"(x[24]), "r"(x[25]), "r"(x[26]), "r"(x[27]), "r"(x[28]), "r"(x[29]), "r"(x[30]), "r"(x[31])
        : "memory");
}

__device__ __forceinline__ void tmem_load16(uint32_t at, uint32_t* x) {
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]), "=r"(x[8]), "=r"(x[9]), "=r"(x[10]),
          "=r"(x[11]), "=r"(x[12]), "=r"(x[13]), "=r"(x[14]), "=r"(x[15])
        : "r"(at));
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t* x) {
    __syncwarp();
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(at), "r"(x[0]),
        "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]), "r"(x[10]), "r"(x[11]), "r"(x[12]), "r"(x[13]),
        "r"(x[14]), "r"(x[15])
        : "memory");
}

}  // namespace jb
