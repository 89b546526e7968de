// jb_q4_tiles.cu -- large products with 4-bit weights on tcgen05: tiles of 128 rows of the matrix by all rows of x.
//
// Three kernels. The first converts x: to fp16, scaled by a power of two for each row so that the largest is near 2^15 (fp32:
// an upper and a lower part, which are rows of their own; see jb_q4_matmul.cu for what that keeps). The second multiplies: the
// matrix's 128-row tiles, 256 columns (four blocks) at a time, are one line of steps, of which every CTA takes an equal
// stretch; sums of what a CTA has of a tile go to the workspace. The third adds them up in the order of the line, multiplies
// by the power of two and adds the bias.
//
// In the second kernel codes and converted inputs come by TMA, in rows of 128 bytes. Eight warps turn codes into numbers: a
// thread has a row, reads its block's 32 bytes, and a table with a copy for each lane gives each byte's two levels as two
// fp16, which go to tensor memory (levels never pass through shared memory again). One warp issues the block's products, 64
// columns deep, the levels from tensor memory, the inputs from shared memory; four warps take the block's sums from tensor
// memory and add them up in fp32, times the block's scale, a thread a row. So a scale is applied in fp32 and once, and a
// weight's level enters off by at most 1.6e-4 of itself (see kLevelScale; fp32: with 22 bits, from two products).
//
// Blocks pass from role to role in pairs: with one at a time the waits and commits of the warp that issues products, 160
// cycles a block, bounded it (33 us for one row times 20480 x 5120). 17 bf16 rows times 5120 x 20480: 27.6 us, 4 of
// them the two kernels around it, for 8.9 us of bytes; 64 rows times 20480 x 5120 36 us. Nothing is busy all the time there: of the
// 47 thousand cycles of the warp that issues products (clock reads around its waits) 28 go to the 337 products, some 80 cycles
// each whatever the rows of x are, 6.5 to waits for levels, 6.4 for room for sums, 6 for the first inputs. Warps that decode
// wait 21 of 43 thousand for room for levels, which products give back; shared memory's pipe is busy 41 % of the time, the
// tensor pipe 12.5 %.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "jb_draft.h"
#include "jb_internal.h"
#include "jb_launch.cuh"
#include "jb_q4_halves.cuh"
#include "jb_tcgen05.cuh"
#include "jb_tensor_map.h"

namespace jb {
namespace {

constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kRows = 128, kStepBlocks = 4;
constexpr int kDecodeWarps = 8, kSumWarps = 4;
constexpr int kTileThreads = 32 * (kDecodeWarps + kSumWarps + 2);
template <typename T>
constexpr int kMostRows = sizeof(T) == 4 ? 32 : 64;  // rows of x at a time
constexpr int kTileCtas = 160;          // most

// Rows of converted x: n rounded up to a product's 16 columns, upper parts and then lower parts.
__host__ __device__ constexpr int padded_rows(int n) { return (n + 15) / 16 * 16; }

struct Line {  // of steps
    int steps, each, extra;  // of a tile; of a CTA, and the first `extra` CTAs one more
    __host__ __device__ long long bound(int w) const { return static_cast<long long>(each) * w + (w < extra ? w : extra); }
    __host__ __device__ int owner(long long x) const {
        const long long longer = (each + 1ll) * extra;
        return static_cast<int>(x < longer ? x / (each + 1) : extra + (x - longer) / each);
    }
};

struct TileParams {
    CUtensorMap codes, inputs;
    Q4Matmul m;
    float levels[16];
    Line line;
    int rows, pad;    // rows of x in this pass, and what they are padded to
    int first;        // row of x
    int parts;        // most parts of a tile
    __half* converted;  // [2 pad or pad][in]
    float* powers;      // [pad]
    float* sums;        // [tile][part][row of x][row of the matrix]
};

__device__ __forceinline__ void read8(const float* from, float (&x)[8]) {
    const float4 a = reinterpret_cast<const float4*>(from)[0], b = reinterpret_cast<const float4*>(from)[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
__device__ __forceinline__ void read8(const __nv_bfloat16* from, float (&x)[8]) {
    const uint4 v = *reinterpret_cast<const uint4*>(from);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(w[e] << 16);
        x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    }
}

// A CTA a row of x; rows past the last are zeros.
template <typename T>
__global__ void __launch_bounds__(512) q4_convert_kernel(const __grid_constant__ TileParams p) {
    constexpr bool kF32 = sizeof(T) == 4;
    constexpr int kKept = 4;  // pieces of 8 that a thread keeps between its two looks
    __shared__ float most_of[16];
    after_previous();
    let_next_start();
    const int row = blockIdx.x, in = p.m.in, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T* x = static_cast<const T*>(p.m.x) + (p.first + row) * p.m.x_row;
    const bool real = row < p.rows;
    float v[kKept][8];
    float most = 0.0f;
    const auto look = [&](const float (&w)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, isfinite(w[i]) ? fabsf(w[i]) : 0.0f);
    };
#pragma unroll
    for (int u = 0; u < kKept; ++u) {
        const int k = 8 * (threadIdx.x + 512 * u);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[u][i] = 0.0f;
        if (real && k < in) read8(x + k, v[u]);
        look(v[u]);
    }
    for (int k = 8 * (threadIdx.x + 512 * kKept); real && k < in; k += 8 * 512) {
        float w[8];
        read8(x + k, w);
        look(w);
    }
#pragma unroll
    for (int d = 16; d > 0; d /= 2) most = fmaxf(most, __shfl_xor_sync(kAll, most, d));
    if (lane == 0) most_of[warp] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) most = fmaxf(most, most_of[i]);
    const int e = exponent_of(most);
    const float down = scaled_down(e);
    if (threadIdx.x == 0) p.powers[row] = scaled_up<kF32>(e);
    __half* upper = p.converted + static_cast<size_t>(row) * in;
    __half* lower = upper + static_cast<size_t>(p.pad) * in;
    const auto convert = [&](const float (&w)[8], int k) {
        uint32_t a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) split<kF32>(w[2 * i] * down, w[2 * i + 1] * down, a[i], b[i]);
        *reinterpret_cast<uint4*>(upper + k) = make_uint4(a[0], a[1], a[2], a[3]);
        if (kF32) *reinterpret_cast<uint4*>(lower + k) = make_uint4(b[0], b[1], b[2], b[3]);
    };
#pragma unroll
    for (int u = 0; u < kKept; ++u) {
        const int k = 8 * (threadIdx.x + 512 * u);
        if (k < in) convert(v[u], k);
    }
    for (int k = 8 * (threadIdx.x + 512 * kKept); k < in; k += 8 * 512) {
        float w[8] = {};
        if (real) read8(x + k, w);
        convert(w, k);
    }
}

// kPad: rows of x, padded.
template <typename T, int kPad>
struct Tiles {
    static constexpr bool kF32 = sizeof(T) == 4;
    static constexpr int kColumns = kF32 ? 2 * kPad : kPad;      // of a product
    static constexpr int kLevels = kF32 ? 64 : 32;               // columns of tensor memory of a block's levels
    static constexpr int kBuffersA = kF32 ? 2 : 4;               // pairs of blocks whose levels are there
    static constexpr int kSums = kBuffersA * 2 * kLevels;        // where sums begin
    static constexpr int kBuffersD = (512 - kSums) / (2 * kColumns) >= 4 ? 4 : 2;
    static constexpr uint32_t kCodeBytes = kRows * 128, kInputBytes = kColumns * 128, kStageBytes = kCodeBytes + kStepBlocks * kInputBytes;
    static constexpr int kStages = 160 * 1024 / kStageBytes >= 4 ? 4 : 160 * 1024 / kStageBytes >= 3 ? 3 : 2;
    static constexpr uint32_t kTable = 65536;
    static constexpr int kShared = 1024 + kTable + kStages * kStageBytes;
    static_assert(kSums + kBuffersD * 2 * kColumns <= 512 && kShared <= 226 * 1024);
};

struct TileControl {
    unsigned long long full[4], inputs[4], empty[4], levels[4], levels_read[4], sums[4], sums_read[4], drained;
    uint32_t tmem;
    int failed;
};

template <typename T, int kPad>
__global__ void __launch_bounds__(kTileThreads, 1) q4_tiles_kernel(const __grid_constant__ TileParams p) {
    using S = Tiles<T, kPad>;
    constexpr bool kF32 = S::kF32;
    extern __shared__ char dynamic[];
    __shared__ TileControl c;
    const int warp = same(static_cast<int>(threadIdx.x) >> 5), lane = threadIdx.x & 31;
    const uint32_t base = (shared_address(dynamic) + 1023) & ~1023u, table = base, stages = base + S::kTable;
    char* const table_at = dynamic + (base - shared_address(dynamic));
    {   // the table: 256 bytes for each byte of codes, with a copy of its two levels for each lane
        for (int i = threadIdx.x; i < 256 * 16; i += kTileThreads) {
            const int byte = i / 16, quad = i % 16;
            if (!kF32 && quad >= 8) continue;
            const float a = p.levels[byte & 15] * kLevelScale<kF32>, b = p.levels[byte >> 4] * kLevelScale<kF32>;
            const uint32_t w = halves(a, b);
            const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&w));
            const uint32_t v = kF32 ? halves(a - h.x, b - h.y) : w;
            *reinterpret_cast<uint4*>(table_at + byte * 256 + quad * 16) = make_uint4(w, v, w, v);
        }
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < 4; ++i) {
            barrier_init(shared_address(&c.full[i]), 1);
            barrier_init(shared_address(&c.inputs[i]), 1);
            barrier_init(shared_address(&c.empty[i]), kDecodeWarps + 1);
            barrier_init(shared_address(&c.levels[i]), kDecodeWarps / 2);
            barrier_init(shared_address(&c.levels_read[i]), 1);
            barrier_init(shared_address(&c.sums[i]), 1);
            barrier_init(shared_address(&c.sums_read[i]), kSumWarps);
        }
        barrier_init(shared_address(&c.drained), 1);
        c.failed = 0;
        barriers_initialized();
    }
    if (warp == kDecodeWarps + kSumWarps) tmem_alloc(shared_address(&c.tmem), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // Only what the kernel before this one writes waits for its end: that one starts this one when all before itself are done.
    let_next_start();
    const uint32_t tmem = same(c.tmem);
    const Q4Matmul& m = p.m;
    const int blocks = m.in / 64, steps = p.line.steps;
    const long long begin = p.line.bound(blockIdx.x), end = p.line.bound(blockIdx.x + 1);
    const auto blocks_of = [&](int step) { return min(kStepBlocks, blocks - step * kStepBlocks); };
    const auto wait = [&](unsigned long long* bar, uint32_t parity) { return __all_sync(kAll, barrier_wait(shared_address(bar), parity, &c.failed)); };

    if (warp < kDecodeWarps) {  // codes to levels: groups of four warps take pairs of blocks in turn
        const int group = warp >> 2, row = threadIdx.x & 127;
        const uint32_t place = lane * (kF32 ? 8 : 4), to = tmem + (static_cast<uint32_t>(32 * (warp & 3)) << 16);
        uint32_t pair = 0, stage = 0;
        int step = static_cast<int>(begin % steps);
        bool ok = true;
        for (long long x = begin; ok && x < end; ++x, ++stage) {
            const uint32_t slot = stage % S::kStages;
            ok = wait(&c.full[slot], stage / S::kStages & 1);
            const int here = blocks_of(step);
            const uint32_t codes = stages + slot * S::kStageBytes + row * 128;
            for (int first = 0; ok && first < here; first += 2, ++pair) {
                if ((pair & 1) != static_cast<uint32_t>(group)) continue;
                const uint32_t buffer = pair % S::kBuffersA;
                ok = wait(&c.levels_read[buffer], (pair / S::kBuffersA & 1) ^ 1);
                tc_fence_after();
                // all reads of the pair under way together (fp32: of a block; a second block that is not there is decoded too)
                constexpr int kTogether = kF32 ? 1 : 2;
#pragma unroll 1
                for (int b0 = 0; b0 < 2; b0 += kTogether) {
                    uint32_t w[kTogether][8], upper[kTogether][32];
                    [[maybe_unused]] uint32_t lower[32];
#pragma unroll
                    for (int b = 0; b < kTogether; ++b)
#pragma unroll
                        for (int half = 0; half < 2; ++half)  // 16 bytes of a block's 32
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                         : "=r"(w[b][4 * half]), "=r"(w[b][4 * half + 1]), "=r"(w[b][4 * half + 2]), "=r"(w[b][4 * half + 3])
                                         : "r"(codes + (((2 * (first + b0 + b) + half) ^ (row & 7)) << 4)));
#pragma unroll
                    for (int b = 0; b < kTogether; ++b)
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const uint32_t at = __byte_perm(w[b][e / 4], place, 0x5504 | e % 4 << 4) + table;  // place, the byte, 0, 0
                            if constexpr (kF32) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(upper[b][e]), "=r"(lower[e]) : "r"(at));
                            else asm volatile("ld.shared.b32 %0, [%1];" : "=r"(upper[b][e]) : "r"(at));
                        }
#pragma unroll
                    for (int b = 0; b < kTogether; ++b) {
                        const uint32_t there = to + (2 * buffer + b0 + b) * S::kLevels;
                        tmem_store32(there, upper[b]);
                        if constexpr (kF32) tmem_store32(there + 32, lower);
                    }
                }
                tc_wait_stores();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive(shared_address(&c.levels[buffer]));
            }
            __syncwarp();
            if (lane == 0) barrier_arrive(shared_address(&c.empty[slot]));
            if (++step == steps) step = 0;
        }
    } else if (warp < kDecodeWarps + kSumWarps) {  // sums of blocks, times their scales
        const int row = threadIdx.x & 127;
        const uint32_t from = tmem + S::kSums + (static_cast<uint32_t>(32 * (warp & 3)) << 16);
        float acc[kPad];
#pragma unroll
        for (int i = 0; i < kPad; ++i) acc[i] = 0.0f;
        uint32_t pair = 0;
        int step = static_cast<int>(begin % steps), tile = static_cast<int>(begin / steps);
        float next[kStepBlocks];
        const auto scales_of = [&](int at_tile, int at_step) {
            const int o = at_tile * kRows + row;
            const float* scale = m.scale + static_cast<int64_t>(o) * blocks + at_step * kStepBlocks;
#pragma unroll
            for (int b = 0; b < kStepBlocks; ++b) next[b] = 0.0f;
            if (o >= m.out) return;
            if (blocks % 4 == 0 && reinterpret_cast<uint64_t>(m.scale) % 16 == 0) {
                const float4 v = __ldg(reinterpret_cast<const float4*>(scale));
                next[0] = v.x, next[1] = v.y, next[2] = v.z, next[3] = v.w;
            } else {
#pragma unroll
                for (int b = 0; b < kStepBlocks; ++b)
                    if (b < blocks_of(at_step)) next[b] = __ldg(scale + b);
            }
        };
        if (begin < end) scales_of(tile, step);
        bool ok = true;
        for (long long x = begin; x < end; ++x) {
            const int here = blocks_of(step);
            float scale[kStepBlocks];
#pragma unroll
            for (int b = 0; b < kStepBlocks; ++b) scale[b] = next[b];
            const int this_tile = tile;
            if (++step == steps) {
                step = 0;
                ++tile;
            }
            if (x + 1 < end) scales_of(tile, step);
#pragma unroll
            for (int first = 0; first < kStepBlocks; first += 2) {
                if (first >= here) break;
                const uint32_t buffer = pair % S::kBuffersD, at = from + buffer * 2 * S::kColumns;
                ok = wait(&c.sums[buffer], pair / S::kBuffersD & 1) && ok;
                tc_fence_after();
                ++pair;
                const bool two = first + 1 < here;
#pragma unroll
                for (int i = 0; i < kPad; i += 16) {
                    uint32_t d[2][16];
                    [[maybe_unused]] uint32_t l[2][16];
                    tmem_load16(at + i, d[0]);
                    tmem_load16(at + S::kColumns + i, d[1]);
                    if constexpr (kF32) {
                        tmem_load16(at + kPad + i, l[0]);
                        tmem_load16(at + S::kColumns + kPad + i, l[1]);
                    }
                    tc_wait_loads();
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        if (b == 1 && !two) continue;  // what an earlier pair left there
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            float v = __uint_as_float(d[b][k]);
                            if constexpr (kF32) v += __uint_as_float(l[b][k]);
                            acc[i + k] = fmaf(v, scale[first + b], acc[i + k]);
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive(shared_address(&c.sums_read[buffer]));
            }
            if (step != 0 && x + 1 < end) continue;
            // the tile's part, or all of it
            const long long start = static_cast<long long>(this_tile) * steps;
            const int part = static_cast<int>(blockIdx.x) - p.line.owner(start);
            float* to = p.sums + (static_cast<size_t>(this_tile) * p.parts + part) * p.rows * kRows + row;
#pragma unroll
            for (int i = 0; i < kPad; ++i) {
                if (i < p.rows) to[static_cast<size_t>(i) * kRows] = ok ? acc[i] : NAN;
                acc[i] = 0.0f;
            }
        }
    } else if (warp == kDecodeWarps + kSumWarps) {  // products
        constexpr uint32_t kF16 = 1u << 4 | 128u >> 4 << 24;  // fp16, fp32 sums, 128 rows
        constexpr uint32_t kBoth = kF16 | static_cast<uint32_t>(S::kColumns >> 3) << 17, kUpper = kF16 | static_cast<uint32_t>(kPad >> 3) << 17;
        uint32_t pair = 0, stage = 0;
        int step = static_cast<int>(begin % steps);
        bool ok = true;
        for (long long x = begin; ok && x < end; ++x, ++stage) {
            const uint32_t slot = stage % S::kStages;
            ok = wait(&c.inputs[slot], stage / S::kStages & 1);
            const int here = blocks_of(step);
            for (int first = 0; ok && first < here; first += 2, ++pair) {
                const uint32_t buffer = pair % S::kBuffersA, sums = pair % S::kBuffersD;
                ok = wait(&c.sums_read[sums], (pair / S::kBuffersD & 1) ^ 1) && wait(&c.levels[buffer], pair / S::kBuffersA & 1);
                if (!ok) break;
                tc_fence_after();
                const uint32_t in = tile_descriptor(stages + slot * S::kStageBytes + S::kCodeBytes + first * S::kInputBytes, 16);
                const uint32_t a = tmem + buffer * 2 * S::kLevels, d = tmem + S::kSums + sums * 2 * S::kColumns;
                const bool two = first + 1 < here;
                if (elected()) {
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        if (b == 1 && !two) continue;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            tc_product_from_tmem(d + b * S::kColumns, a + b * S::kLevels + 8 * k, in + ((b * S::kInputBytes + k * 32) >> 4), kBoth, k > 0);
                        if constexpr (kF32) {
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                tc_product_from_tmem(d + b * S::kColumns, a + b * S::kLevels + 32 + 8 * k, in + ((b * S::kInputBytes + k * 32) >> 4), kUpper, true);
                        }
                    }
                    tc_commit(shared_address(&c.levels_read[buffer]));
                    tc_commit(shared_address(&c.sums[sums]));
                    if (first + 2 >= here) tc_commit(shared_address(&c.empty[slot]));
                }
                __syncwarp();
            }
            if (++step == steps) step = 0;
        }
        if (!ok) tc_drain(shared_address(&c.drained));  // what is under way ends before tensor memory is given back
    } else {  // copies; codes of the first stages go ahead of the inputs, which another kernel may still be converting
        const uint32_t all = static_cast<uint32_t>(end - begin);
        const int from_step = static_cast<int>(begin % steps), from_tile = static_cast<int>(begin / steps);
        uint32_t asked = 0;
        int code_step = from_step, code_tile = from_tile;
        const auto codes = [&] {
            const uint32_t slot = asked++ % S::kStages, bar = shared_address(&c.full[slot]);
            if (lane == 0) {
                barrier_arrive_bytes(bar, S::kCodeBytes);
                copy_box(stages + slot * S::kStageBytes, &p.codes, code_step * 128, code_tile * kRows, 0, 0, bar);
            }
            if (++code_step == steps) {
                code_step = 0;
                ++code_tile;
            }
        };
        while (asked < all && asked < S::kStages) codes();
        if (all > 0) after_previous();
        int step = from_step;
        uint32_t stage = 0;
        for (; stage < all; ++stage) {
            const uint32_t slot = stage % S::kStages, to = stages + slot * S::kStageBytes + S::kCodeBytes, bar = shared_address(&c.inputs[slot]);
            if (!wait(&c.empty[slot], (stage / S::kStages & 1) ^ 1)) break;
            if (asked == stage) codes();
            const int here = blocks_of(step);
            if (lane == 0) barrier_arrive_bytes(bar, here * S::kInputBytes);
            __syncwarp();
            if (lane < here) copy_box(to + lane * S::kInputBytes, &p.inputs, (step * kStepBlocks + lane) * 64, 0, 0, 0, bar);
            if (++step == steps) step = 0;
        }
        // what is under way arrives before the role ends, whatever became of the others
        int late = 0;
        for (uint32_t k = asked < S::kStages ? 0 : asked - S::kStages; k < asked; ++k) barrier_wait(shared_address(&c.full[k % S::kStages]), k / S::kStages & 1, &late);
        for (uint32_t k = stage < S::kStages ? 0 : stage - S::kStages; k < stage; ++k) barrier_wait(shared_address(&c.inputs[k % S::kStages]), k / S::kStages & 1, &late);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kDecodeWarps + kSumWarps) tmem_free(c.tmem, 512);
}

// A thread a result.
template <typename T>
__global__ void __launch_bounds__(128) q4_join_kernel(const __grid_constant__ TileParams p) {
    after_previous();
    let_next_start();
    const int tile = blockIdx.x, i = blockIdx.y, o = tile * kRows + static_cast<int>(threadIdx.x);
    if (o >= p.m.out) return;
    const long long start = static_cast<long long>(tile) * p.line.steps;
    const int parts = p.line.owner(start + p.line.steps - 1) - p.line.owner(start) + 1;
    const float* from = p.sums + (static_cast<size_t>(tile) * p.parts * p.rows + i) * kRows + threadIdx.x;
    float v = 0.0f;
#pragma unroll 4
    for (int k = 0; k < parts; ++k) v += __ldcg(from + static_cast<size_t>(k) * p.rows * kRows);
    v *= p.powers[i];
    T* y = static_cast<T*>(p.m.y) + (p.first + i) * p.m.y_row + o;
    if constexpr (sizeof(T) == 4) {
        if (p.m.bias != nullptr) v += static_cast<const float*>(p.m.bias)[o];
        *y = v;
    } else {
        if (p.m.bias != nullptr) v += __bfloat162float(static_cast<const __nv_bfloat16*>(p.m.bias)[o]);
        *y = __float2bfloat16_rn(v);
    }
}

int steps_of(int in) { return (in / 64 + kStepBlocks - 1) / kStepBlocks; }

// CTAs that the line is dealt to, and most parts of a tile.
Line line_of(int out, int in, int ctas) {
    const long long total = static_cast<long long>((out + kRows - 1) / kRows) * steps_of(in);
    return {steps_of(in), static_cast<int>(total / ctas), static_cast<int>(total % ctas)};
}
int parts_of(const Line& l) { return l.each == 0 ? l.steps : (l.steps + l.each - 1) / l.each + 1; }

constexpr int kTileDevices = 64;
cudaError_t sms_of(int& sms) {
    static std::atomic<int> known[kTileDevices];
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    sms = device < kTileDevices ? known[device].load(std::memory_order_relaxed) : 0;
    if (sms > 0) return cudaSuccess;
    e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e != cudaSuccess) return e;
    if (sms > kTileCtas) sms = kTileCtas;
    if (device < kTileDevices) known[device].store(sms, std::memory_order_relaxed);
    return cudaSuccess;
}

cudaError_t describe(CUtensorMap& map, CUtensorMapDataType type, const void* at, cuuint64_t inner, cuuint64_t outer, cuuint64_t stride, cuuint32_t box_inner,
                     cuuint32_t box_outer) {
    Encode encode = nullptr;
    const cudaError_t e = encoder(encode);
    if (e != cudaSuccess) return e;
    const cuuint64_t dims[4] = {inner, outer, 1, 1}, strides[3] = {stride, stride * outer, stride * outer};
    const cuuint32_t boxes[4] = {box_inner, box_outer, 1, 1}, steps[4] = {1, 1, 1, 1};
    const CUresult r = encode(&map, type, 4, const_cast<void*>(at), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <typename T, int kPad>
cudaError_t launch_pad(const TileParams& p, int ctas, cudaStream_t s) {
    using S = Tiles<T, kPad>;
    static std::atomic<bool> ready[kTileDevices];
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device >= kTileDevices || !ready[device].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(q4_tiles_kernel<T, kPad>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kShared);
        if (e != cudaSuccess) return e;
        if (device < kTileDevices) ready[device].store(true, std::memory_order_relaxed);
    }
    return launch(q4_tiles_kernel<T, kPad>, ctas, kTileThreads, S::kShared, 0, s, p);
}

template <typename T>
cudaError_t launch_type(const Q4Matmul& m, cudaStream_t s) {
    constexpr int kParts = sizeof(T) == 4 ? 2 : 1;
    int sms = 0;
    cudaError_t e = sms_of(sms);
    if (e != cudaSuccess) return e;
    TileParams p;
    p.m = m;
    q4_levels_host(p.levels);
    const int tiles = (m.out + kRows - 1) / kRows;
    const long long total = static_cast<long long>(tiles) * steps_of(m.in);
    const int ctas = total < sms ? static_cast<int>(total) : sms;
    p.line = line_of(m.out, m.in, ctas);
    p.parts = parts_of(p.line);
    e = describe(p.codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, m.codes, m.in / 2, m.out, m.in / 2, 128, kRows);
    if (e != cudaSuccess) return e;
    for (p.first = 0; p.first < m.n; p.first += kMostRows<T>) {
        p.rows = m.n - p.first < kMostRows<T> ? m.n - p.first : kMostRows<T>;
        p.pad = padded_rows(p.rows);
        char* ws = static_cast<char*>(m.ws);
        p.converted = reinterpret_cast<__half*>(ws);
        ws += static_cast<size_t>(kParts) * p.pad * m.in * 2;
        p.powers = reinterpret_cast<float*>(ws);
        p.sums = p.powers + kMostRows<__nv_bfloat16>;
        e = describe(p.inputs, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, p.converted, m.in, kParts * p.pad, m.in * 2, 64, kParts * p.pad);
        if (e != cudaSuccess) return e;
        e = launch(q4_convert_kernel<T>, p.pad, 512, 0, 0, s, p);
        if (e != cudaSuccess) return e;
        if (p.pad == 16) e = launch_pad<T, 16>(p, ctas, s);
        else if (p.pad == 32) e = launch_pad<T, 32>(p, ctas, s);
        else if constexpr (kMostRows<T> == 64) e = p.pad == 48 ? launch_pad<T, 48>(p, ctas, s) : launch_pad<T, 64>(p, ctas, s);
        if (e != cudaSuccess) return e;
        e = launch(q4_join_kernel<T>, dim3(tiles, p.rows), 128, 0, 0, s, p);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

bool q4_by_tiles(int n, int out, int in, int bf16) {
    // Three launches pay from some columns of the product on (rows of x, in fp32 two for each): the fewer the larger the matrix is
    // and the longer its rows are, as a CTA of the other kernel holds so much input. Measured over 48 shapes with cold weights, the
    // other kernel and this one in us, bf16 unless fp32 is said:
    //   32768 x 1024, 16 rows 16.0 and 15.9, 17 rows 19.2 and 16.3; 4096 x 1024, 24 rows 6.9 and 8.0, 32 rows 8.2 and 8.1;
    //   1024 x 1024, 24 rows 5.7 and 6.6, 32 rows 6.9 and 6.6, fp32 12 rows 5.8 and 6.8, 16 rows 6.9 and 6.8;
    //   2048 x 2048, 12 rows 6.3 and 7.1, 16 rows 7.4 and 7.4; 3000 x 3008, 9 rows 8.6 and 9.1, 12 rows 10.0 and 9.1;
    //   4096 x 4096, 8 rows 9.5 and 11.6, 9 rows 11.9 and 11.7, fp32 4 rows 11.6 and 12.0, 5 rows 13.0 and 12.1;
    //   20480 x 5120, 6 rows 24.2 and 26.0, 8 rows 26.2 and 26.0, fp32 3 rows 29.4 and 32.3, 4 rows 32.5 and 32.4;
    //   32000 x 4096, 6 rows 31.3 and 29.9, 7 rows 37.7 and 29.9; 8192 x 8192, 3 rows 17.9 and 20.0, 4 rows 21.3 and 20.0;
    //   5120 x 20480, 1 row 27.1 and 24.9, 2 rows 24.5 and 25.0, 5 rows 24.9 and 26.0, 6 rows 28.9 and 26.0, fp32 1 row 32.4 and 31.2;
    //   4096 x 16384, 1 row 16.6 and 19.1, 4 rows 19.3 and 19.1, 6 rows 24.2 and 20.1.
    // Over all of them the side that is taken costs 0.8 % more than the faster one on average, more than a quarter only where at most
    // 1024 rows of the matrix are 16384 long or longer.
    const long long size = static_cast<long long>(out) * in, columns = static_cast<long long>(n) * (bf16 ? 1 : 2);
    if (size < 1ll << 19) return false;
    if (in < 2048) return columns >= (size >= 1ll << 23 ? 17 : size >= 1ll << 21 ? 24 : 32);
    if (size >= 1ll << 25 && in >= 13000) return columns * in >= 20480;
    if (size >= 1ll << 26) return columns >= 7 || columns * in >= 1ll << 15;
    if (size >= 1ll << 25 || in >= 4096) return columns > 8;
    return columns * in >= 1ll << 15;
}

uint64_t q4_workspace(int n, int out, int in, int bf16) {
    if (!q4_by_tiles(n, out, in, bf16)) return 0;
    const int most = bf16 ? kMostRows<__nv_bfloat16> : kMostRows<float>, rows = n < most ? n : most, tiles = (out + kRows - 1) / kRows;
    const long long total = static_cast<long long>(tiles) * steps_of(in);
    // parts are most with the most CTAs
    const int parts = parts_of(line_of(out, in, static_cast<int>(total < kTileCtas ? total : kTileCtas)));
    return static_cast<uint64_t>(bf16 ? 1 : 2) * padded_rows(rows) * in * 2 + 4ull * kMostRows<__nv_bfloat16> + 4ull * tiles * parts * rows * kRows;
}

cudaError_t launch_q4_tiles(const Q4Matmul& m, cudaStream_t s) {
    return m.bf16 ? launch_type<__nv_bfloat16>(m, s) : launch_type<float>(m, s);
}

}  // namespace jb
