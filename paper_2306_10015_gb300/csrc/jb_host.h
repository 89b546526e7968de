// jb_host.h -- what the entry points of the C ABI share.
#pragma once
#include <cstdint>
#include <new>

#include <cuda_runtime.h>

#include "jb.h"

#define JB_EXPORT extern "C" __attribute__((visibility("default")))

namespace jb {

// [p, p + n * es) fits in the address space (written so that n * es cannot wrap).
inline bool range_fits(uint64_t p, uint64_t n, uint64_t es) { return n <= (UINT64_MAX - p) / es; }

// Runs an entry point's body; a host allocation failure (or any other C++
// exception) becomes a status instead of crossing the C interface.
template <typename F>
int guarded(F&& body) noexcept {
    try {
        return body();
    } catch (const std::bad_alloc&) {
        return JB_ERR_NO_MEMORY;
    } catch (...) {
        return JB_ERR_INVALID_ARG;
    }
}

// libjb links the CUDA runtime statically: its last-error state is its own, so the
// errors of a caller's runtime (torch's, say) are neither seen nor cleared here. A
// failed call of this library's is cleared from that state (cudaGetLastError) so that
// it cannot be reported again by a later, unrelated call.
inline int cuda_status(cudaError_t e) {
    if (e == cudaSuccess) return JB_OK;
    (void)cudaGetLastError();
    return JB_ERR_CUDA;
}

}  // namespace jb
