// jb_append.cu -- new tokens on their way into the cache: queries and keys turned by their positions, keys and values
// written to their pages.
//
// Pair j of a head is turned by the angle 2 pi (t s_j mod 2^64) / 2^64, t the token's position and s_j the pair's step in
// 2^-64 of a turn. The product is exact, so that the angle of position 2^30 is as good as that of position 1; it is
// rounded once, to fp32, as a part of half a turn.
//   (a, b) -> (a cos - b sin, b cos + a sin), in fp32, rounded once more to the storage type
//
// Every byte is read once and written once, which bounds it. A CTA takes a token, or a part of its heads where there are
// few tokens: its threads form the token's cosines and sines once in shared memory, one pair each, then take 16-byte
// vectors of all heads. 8191 tokens of 32 query and 32 key heads of 128 in bf16: 69.6 us, 5.8 TB/s; one token 2.5 us, a launch and
// a chain of table, steps and sines.
#include <cuda_bf16.h>

#include "jb_draft.h"
#include "jb_launch.cuh"

namespace jb {
namespace {

constexpr int kThreads = 128;
constexpr int kMaxPairs = kMaxHeadDim / 2;

enum Pairing { kHalves, kNext, kOddHalves };  // kOddHalves: half of the turned elements is no multiple of a vector

struct Params {
    Pages pages;
    Append a;
    uint32_t units, vecs;         // units of a head that is turned; 16-byte vectors of a head
    uint64_t magic, vec_magic;    // 2^32 / units and 2^32 / vecs rounded up: u magic >> 32 is u / units while u is below 2^22
};

template <typename T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int kElems = 4;
    static __device__ __forceinline__ void read(const uint4& v, float (&x)[4]) {
        x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 write(const float (&x)[4]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int kElems = 8;
    static __device__ __forceinline__ void read(const uint4& v, float (&x)[8]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ uint4 write(const float (&x)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

__device__ __forceinline__ float2 turned(float a, float b, float2 cs) {
    return make_float2(fmaf(a, cs.x, -(b * cs.y)), fmaf(b, cs.x, a * cs.y));
}

template <typename T, Pairing kPairing>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ Params p) {
    constexpr int kElems = Vec<T>::kElems;
    __shared__ float2 cs[kMaxPairs];
    __shared__ float heads[kPairing == kOddHalves ? kThreads / 32 : 1][kPairing == kOddHalves ? kMaxHeadDim : 1];
    const Append& a = p.a;
    const int i = blockIdx.x, half = a.dims / 2;
    after_previous();
    let_next_start();
    const long long turns = a.turns[i];
    for (int j = threadIdx.x; j < half; j += kThreads) {
        const long long part = static_cast<long long>(static_cast<uint64_t>(turns) * a.steps[j]);
        sincospif(__ll2float_rn(part) * 0x1p-63f, &cs[j].y, &cs[j].x);
    }
    // the token's place; a token without one is not written, and its queries are turned all the same
    const int row = a.rows[i], pos = a.pos[i];
    int page = -1;
    if (row >= 0 && row < p.pages.n_rows && pos >= 0 && pos / p.pages.page_tokens < p.pages.row_pages)
        page = p.pages.table[static_cast<size_t>(row) * p.pages.row_pages + pos / p.pages.page_tokens];
    const bool placed = page >= 0 && page < p.pages.n_pages;
    const uint64_t place = placed ? page * a.page_stride + pos % p.pages.page_tokens * a.to_token : 0;
    __syncthreads();
    // source and destination of head h, queries first; nullptr: not to be written
    const auto source = [&](int h) {
        const int kind = h < a.q_heads ? 0 : 1;
        return a.from[kind] + i * a.token_stride[kind] + (kind ? h - a.q_heads : h) * a.head_stride[kind];
    };
    const auto destination = [&](int h) -> char* {
        if (h < a.q_heads) return a.q_out + i * a.out_token + h * a.out_head;
        return placed ? a.to[0] + place + (h - a.q_heads) * a.to_head : nullptr;
    };
    const uint32_t all = a.q_heads + a.heads, vecs = p.vecs;
    if constexpr (kPairing == kOddHalves) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = kThreads / 32;
        for (uint32_t h = blockIdx.y * warps + warp; h < all; h += gridDim.y * warps) {
            const char* from = source(h);
            char* to = destination(h);
            for (uint32_t v = lane; v < vecs; v += 32) {
                float x[kElems];
                Vec<T>::read(reinterpret_cast<const uint4*>(from)[v], x);
#pragma unroll
                for (int e = 0; e < kElems; ++e) heads[warp][v * kElems + e] = x[e];
            }
            __syncwarp();
            if (to != nullptr)
                for (uint32_t v = lane; v < vecs; v += 32) {
                    float x[kElems];
#pragma unroll
                    for (int e = 0; e < kElems; ++e) {
                        const int j = v * kElems + e;
                        x[e] = heads[warp][j];
                        if (j < half) x[e] = turned(x[e], heads[warp][j + half], cs[j]).x;
                        else if (j < a.dims) x[e] = turned(heads[warp][j - half], x[e], cs[j - half]).y;
                    }
                    reinterpret_cast<uint4*>(to)[v] = Vec<T>::write(x);
                }
            __syncwarp();
        }
    } else {
        const uint32_t pairs = kPairing == kHalves ? half / kElems : 0;  // units that are two vectors
        constexpr int kUnroll = 2;
        const uint32_t total = all * p.units, step = gridDim.y * kThreads;
        for (uint32_t first = blockIdx.y * kThreads + threadIdx.x; first < total; first += kUnroll * step) {
            uint4 lo[kUnroll], hi[kUnroll];
            char* to[kUnroll];
            uint32_t at[kUnroll];
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                const uint32_t u = first + k * step;
                to[k] = nullptr;
                if (u >= total) continue;
                const uint32_t h = static_cast<uint32_t>(u * p.magic >> 32), unit = u - h * p.units;
                const uint4* from = reinterpret_cast<const uint4*>(source(h));
                to[k] = destination(h);
                at[k] = unit;
                if (kPairing == kHalves && unit < pairs) {
                    lo[k] = from[unit];
                    hi[k] = from[unit + pairs];
                } else {
                    lo[k] = from[unit + pairs];
                }
            }
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                if (to[k] == nullptr) continue;
                uint4* out = reinterpret_cast<uint4*>(to[k]);
                const uint32_t unit = at[k];
                if constexpr (kPairing == kHalves) {
                    if (unit >= pairs) {
                        out[unit + pairs] = lo[k];
                        continue;
                    }
                    float x[kElems], y[kElems];
                    Vec<T>::read(lo[k], x);
                    Vec<T>::read(hi[k], y);
#pragma unroll
                    for (int e = 0; e < kElems; ++e) {
                        const float2 t = turned(x[e], y[e], cs[unit * kElems + e]);
                        x[e] = t.x;
                        y[e] = t.y;
                    }
                    out[unit] = Vec<T>::write(x);
                    out[unit + pairs] = Vec<T>::write(y);
                } else {
                    float x[kElems];
                    Vec<T>::read(lo[k], x);
#pragma unroll
                    for (int e = 0; e < kElems; e += 2) {
                        const int j = (unit * kElems + e) / 2;
                        if (j >= half) continue;
                        const float2 t = turned(x[e], x[e + 1], cs[j]);
                        x[e] = t.x;
                        x[e + 1] = t.y;
                    }
                    out[unit] = Vec<T>::write(x);
                }
            }
        }
    }
    // values
    if (!placed) return;
    const uint32_t total = a.heads * vecs;
    for (uint32_t u = blockIdx.y * kThreads + threadIdx.x; u < total; u += gridDim.y * kThreads) {
        const uint32_t h = static_cast<uint32_t>(u * p.vec_magic >> 32), v = u - h * vecs;
        const char* from = a.from[2] + i * a.token_stride[2] + h * a.head_stride[2];
        reinterpret_cast<uint4*>(a.to[1] + place + h * a.to_head)[v] = reinterpret_cast<const uint4*>(from)[v];
    }
}

uint64_t magic_of(uint32_t d) { return ((1ull << 32) + d - 1) / d; }

}  // namespace

cudaError_t launch_append(const Pages& pages, const Append& a, cudaStream_t s) {
    const int elems = a.bf16 ? 8 : 4, half = a.dims / 2;
    const Pairing pairing = a.interleaved ? kNext : half % elems == 0 ? kHalves : kOddHalves;
    Params p = {pages, a};
    p.vecs = a.head_dim / elems;
    p.units = pairing == kHalves ? p.vecs - half / elems : p.vecs;
    p.magic = magic_of(p.units);
    p.vec_magic = magic_of(p.vecs);
    // a token's heads are shared out while that fills the GPU
    const uint32_t most = ((a.q_heads + a.heads) * p.units + kThreads - 1) / kThreads, want = (152u * 8 + a.n - 1) / a.n;
    const dim3 grid(a.n, most < want ? most : want);
    const auto start = [&](auto kernel) { return launch(kernel, grid, kThreads, 0, 0, s, p); };
    using B = __nv_bfloat16;
    switch (pairing) {
        case kNext: return a.bf16 ? start(append_kernel<B, kNext>) : start(append_kernel<float, kNext>);
        case kHalves: return a.bf16 ? start(append_kernel<B, kHalves>) : start(append_kernel<float, kHalves>);
        default: return a.bf16 ? start(append_kernel<B, kOddHalves>) : start(append_kernel<float, kOddHalves>);
    }
}

}  // namespace jb
