// jb_tensor_map.h -- the driver's function that describes a tensor to TMA copies.
#pragma once
#include <atomic>

#include <cuda.h>
#include <cuda_runtime.h>

namespace jb {

using Encode = decltype(&cuTensorMapEncodeTiled);

// Asked for once.
inline cudaError_t encoder(Encode& encode) {
    static std::atomic<void*> known;
    void* f = known.load(std::memory_order_acquire);
    if (f == nullptr) {
        cudaDriverEntryPointQueryResult found;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
        if (e != cudaSuccess) return e;
        if (found != cudaDriverEntryPointSuccess || f == nullptr) return cudaErrorNotSupported;
        known.store(f, std::memory_order_release);
    }
    encode = reinterpret_cast<Encode>(f);
    return cudaSuccess;
}

}  // namespace jb
