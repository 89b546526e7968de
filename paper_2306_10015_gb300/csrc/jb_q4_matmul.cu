// jb_q4_matmul.cu -- products of a few rows with a matrix of 4-bit weights (the format of jb_perturb_q4):
//   y[i][o] = sum_k x[i][k] level[code[o][k]] scale[o][k / 64] + bias[o]
#include <cuda_bf16.h>

#include "jb_draft.h"
#include "jb_internal.h"
#include "jb_launch.cuh"

namespace jb {
namespace {

constexpr int kMatThreads = 256;

struct Params {
    Q4Matmul m;
    float levels[16];
};

__device__ __forceinline__ float value(const float* p) { return *p; }
__device__ __forceinline__ float value(const __nv_bfloat16* p) { return __bfloat162float(*p); }

// A warp takes a row of the matrix, a lane 16 codes of it at a time, against 8 rows of x.
template <typename T>
__global__ void __launch_bounds__(kMatThreads) q4_matmul_kernel(const __grid_constant__ Params p) {
    __shared__ float levels[16];
    const Q4Matmul& m = p.m;
    if (threadIdx.x < 16) levels[threadIdx.x] = p.levels[threadIdx.x];
    after_previous();
    let_next_start();
    __syncthreads();
    const int o = blockIdx.x * (kMatThreads / 32) + static_cast<int>(threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (o >= m.out) return;
    const T* x = static_cast<const T*>(m.x);
    for (int first = 0; first < m.n; first += 8) {
        float sum[8] = {};
        for (int k = 16 * lane; k < m.in; k += 512) {
            const uint64_t at = static_cast<uint64_t>(o) * m.in + k;
            const uint64_t codes = *reinterpret_cast<const uint64_t*>(m.codes + at / 2);
            float w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = levels[codes >> (4 * e) & 15];
            const float scale = m.scale[at / 64];
            for (int i = 0; i < 8 && first + i < m.n; ++i) {
                float part = 0.0f;
                const T* row = x + (first + i) * m.x_row + k;
#pragma unroll
                for (int e = 0; e < 16; ++e) part = fmaf(w[e], value(row + e), part);
                sum[i] = fmaf(part, scale, sum[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            for (int u = 16; u > 0; u /= 2) sum[i] += __shfl_xor_sync(0xFFFFFFFFu, sum[i], u);
            if (lane != 0 || first + i >= m.n) continue;
            if (m.bias != nullptr) sum[i] += value(static_cast<const T*>(m.bias) + o);
            T* y = static_cast<T*>(m.y) + (first + i) * m.y_row + o;
            if constexpr (sizeof(T) == 4) *y = sum[i];
            else *y = __float2bfloat16_rn(sum[i]);
        }
    }
}

}  // namespace

cudaError_t launch_q4_matmul(const Q4Matmul& m, cudaStream_t s) {
    Params p;
    p.m = m;
    q4_levels_host(p.levels);
    const unsigned ctas = (m.out + kMatThreads / 32 - 1) / (kMatThreads / 32);
    return m.bf16 ? launch(q4_matmul_kernel<__nv_bfloat16>, ctas, kMatThreads, 0, 0, s, p) : launch(q4_matmul_kernel<float>, ctas, kMatThreads, 0, 0, s, p);
}

}  // namespace jb
