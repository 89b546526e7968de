// jb_q4_matmul.cu -- products of very few rows, or with small matrices, of 4-bit weights (the format of jb_perturb_q4; the
// others are in jb_q4_tiles.cu):
//   y[i][o] = sum_k x[i][k] level[code[o][k]] scale[o][k / 64] + bias[o]
//
// The weights are read once, 4.5 bits each, and that bounds it while turning codes into numbers keeps up: a byte is a pair
// of codes, and a table in shared memory with a copy for each lane (no bank conflicts) has the pair's two levels as two fp16,
// which is how mma.m16n8k16 takes them. So 16 rows of the matrix by 64 columns, a block each, are 16 table reads a lane and
// four products with up to 8 rows of x; tokens are the product's columns.
//
// Numbers. fp16 has 11 bits: a level is off by at most 1.6e-4 of itself (see kLevelScale), beside the 2^-9 of a bf16 result. bf16 inputs fit fp16 with
// all their bits once they are scaled by a power of two, chosen for each row (of a CTA's slice of the columns) so that the
// largest is near 2^15 (what is 2^-28 of it or smaller loses bits, 2^-40 of it is lost). fp32: levels and inputs are two fp16 each, 22 bits
// and more; the inputs' two parts are two columns of the product, and a table read is two words (the product of two lower
// parts, at most 2^-22, is left out). A block's sum is fp32 and
// meets its scale once; sums over blocks, warps and CTAs are fp32, in an order that does not depend on the launch's timing.
//
// A CTA of 16 warps has a slice of the columns, whose inputs it keeps in shared memory, and takes tiles of 16 rows: warps
// split the slice, and their sums are joined in shared memory. Where the inputs of all columns do not fit, a cluster of CTAs
// has a slice each and their sums are joined through distributed shared memory. A warp copies its codes and scales ahead
// (cp.async) to a ring of its own: loads to registers are waited for all together, and with six blocks ahead that left
// 8 KB under way on an SM (one row times 20480 x 5120: 47 us). It takes two or four blocks of a row at a time, because each
// line that a copy touches takes a turn of the pipe that serves shared memory, too, as a table read does (one block: 28 us).
// One bf16 row times 20480 x 5120 takes 19.4 us, 3.05 TB/s, where the bytes take 8.7. That pipe is what is busiest, 64 % of the
// time (issue slots 48 %, tensor pipes 15 %); the rest is the table and the inputs at the start, and tiles that do not divide
// evenly: CTAs have work for 91 % of the rounds there, by launch_tiles' estimate, and for 70 % with 5120 x 20480 (27.1 us).
#include <atomic>
#include <type_traits>

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "jb_draft.h"
#include "jb_internal.h"
#include "jb_launch.cuh"
#include "jb_q4_halves.cuh"

namespace jb {
namespace {

namespace cg = cooperative_groups;

constexpr int kMatWarps = 16, kMatThreads = 32 * kMatWarps;
constexpr int kUnit = 512;          // columns of a row that a warp converts at a time
constexpr int kPad = 8;             // halves between rows of inputs: reads of 8 rows meet no bank twice
constexpr int kRed = 20;            // floats from column to column of a tile's sums, for the same reason
constexpr int kMostColumns = 64;    // of the product at a time

struct Params {
    Q4Matmul m;
    float levels[16];
    int first, rows;     // rows of x in this pass
    int columns;         // of the product: rows, or twice as many
    int slice;           // columns of a CTA's slice
    int ways, at_once;   // warps that split a slice; tiles of 16 rows that a CTA takes at a time
    int slots;           // rounds of tiles whose warps' sums are joined at a time
    int kept;            // tiles whose sums a CTA keeps until the cluster joins them
};

// What a kernel for so many columns of the product / 8 is made of.
template <typename T, int kTiles>
struct Shape {
    static constexpr bool kF32 = sizeof(T) == 4;
    static constexpr int kSpan = kTiles == 1 ? 4 : 2;           // neighbouring blocks of a row that a warp takes
    static constexpr int kAhead = 2;                            // of them copied ahead
    static constexpr int kPitch = kSpan * 32 + 32;              // bytes from row to row: reads of 8 rows meet no bank twice
    static constexpr int kStage = 16 * kPitch + kSpan * 64;     // codes, and scales by block and row
    // From byte to byte in the table: with 256 bytes the byte and the lane's place are put together by one permutation,
    // with 128 by a shift and a selection, for less memory.
    static constexpr int kShift = kF32 || kTiles == 1 ? 8 : 7;
};
// Shared memory, in bytes: table, rings, powers of two and rows' maxima, inputs, warps' sums, kept sums.
struct Layout {
    int rings, powers, inputs, sums, kept, all;
};
__host__ __device__ inline int round16(int x) { return (x + 15) & ~15; }
template <typename S>
__host__ __device__ inline Layout layout_of(int rows, int columns, int slice, int slots, int kept) {
    Layout l;
    l.rings = 256 << S::kShift;
    l.powers = l.rings + kMatWarps * S::kAhead * S::kStage;
    l.inputs = l.powers + 2 * kMostColumns * 4;
    l.sums = l.inputs + round16(columns * (slice + kPad) * 2);
    l.kept = l.sums + slots * kMatWarps * rows * kRed * 4;
    l.all = l.kept + kept * rows * 16 * 4;
    return l;
}

__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 16 inputs of a row in fp32.
__device__ __forceinline__ void read16(const float* from, float (&x)[16]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 v = reinterpret_cast<const float4*>(from)[i];
        x[4 * i] = v.x, x[4 * i + 1] = v.y, x[4 * i + 2] = v.z, x[4 * i + 3] = v.w;
    }
}
__device__ __forceinline__ void read16(const __nv_bfloat16* from, float (&x)[16]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint4 v = reinterpret_cast<const uint4*>(from)[i];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[8 * i + 2 * e] = __uint_as_float(w[e] << 16);
            x[8 * i + 2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        }
    }
}

// The slice's inputs as the product takes them, and their powers of two. A warp takes 512 columns of a row at a time; what
// it has read for the row's maximum it keeps, if that is one unit.
template <typename T>
__device__ void stage(const Params& p, const Layout& l, char* shared, int from) {
    constexpr bool kF32 = sizeof(T) == 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, groups = (p.slice + kUnit - 1) / kUnit, units = p.rows * groups;
    float* powers = reinterpret_cast<float*>(shared + l.powers);
    int* most_of = reinterpret_cast<int*>(powers + kMostColumns);
    __half* inputs = reinterpret_cast<__half*>(shared + l.inputs);
    const T* x = static_cast<const T*>(p.m.x);
    const int here = min(p.slice, p.m.in - from);
    float v[16];
    const auto read = [&](int row, int k) {
        if (k < here) {
            read16(x + (p.first + row) * p.m.x_row + from + k, v);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = 0.0f;
        }
    };
    for (int u = warp; u < units; u += kMatWarps) {
        const int row = u / groups;
        read(row, (u - row * groups) * kUnit + 16 * lane);
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, isfinite(v[i]) ? fabsf(v[i]) : 0.0f);
#pragma unroll
        for (int d = 16; d > 0; d /= 2) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
        if (lane == 0) atomicMax(&most_of[row], __float_as_int(most));  // not negative: ordered as integers are
    }
    __syncthreads();
    for (int u = warp; u < units; u += kMatWarps) {
        const int row = u / groups, k = (u - row * groups) * kUnit + 16 * lane;
        if (units > kMatWarps) read(row, k);
        const int e = exponent_of(__int_as_float(most_of[row]));
        const float down = scaled_down(e);
        if (lane == 0) powers[row] = scaled_up<kF32>(e);
        if (k >= p.slice) continue;
        uint32_t w[8], r[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) split<kF32>(v[2 * i] * down, v[2 * i + 1] * down, w[i], r[i]);
        __half* to = inputs + (kF32 ? 2 * row : row) * (p.slice + kPad) + k;
        reinterpret_cast<uint4*>(to)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(to)[1] = make_uint4(w[4], w[5], w[6], w[7]);
        if (kF32) {
            to += p.slice + kPad;
            reinterpret_cast<uint4*>(to)[0] = make_uint4(r[0], r[1], r[2], r[3]);
            reinterpret_cast<uint4*>(to)[1] = make_uint4(r[4], r[5], r[6], r[7]);
        }
    }
}

__device__ __forceinline__ void copy16(uint32_t to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copy8(uint32_t to, const void* from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copy4(uint32_t to, const void* from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory"); }

// kTiles: columns of the product / 8.
template <typename T, int kTiles>
__global__ void __launch_bounds__(kMatThreads, 1) q4_matmul_kernel(const __grid_constant__ Params p) {
    using S = Shape<T, kTiles>;
    constexpr bool kF32 = S::kF32;
    extern __shared__ __align__(256) char shared[];
    const Q4Matmul& m = p.m;
    const Layout l = layout_of<S>(p.rows, p.columns, p.slice, p.slots, p.kept);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, t = lane & 3;
    {   // the table: the entry of a byte, with a copy for each lane
        __shared__ uint32_t pairs[256][kF32 ? 2 : 1];
        if (threadIdx.x < 256) {
            const float a = p.levels[threadIdx.x & 15] * kLevelScale<kF32>, b = p.levels[threadIdx.x >> 4] * kLevelScale<kF32>;
            const uint32_t w = halves(a, b);
            pairs[threadIdx.x][0] = w;
            if (kF32) {
                const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&w));
                pairs[threadIdx.x][kF32 ? 1 : 0] = halves(a - h.x, b - h.y);
            }
        }
        __syncthreads();
        constexpr int kQuads = kF32 ? 16 : 8;  // 16-byte pieces of an entry
        for (int i = threadIdx.x; i < 256 * kQuads; i += kMatThreads) {
            const uint32_t w = pairs[i / kQuads][0], v = kF32 ? pairs[i / kQuads][kF32 ? 1 : 0] : w;
            *reinterpret_cast<uint4*>(shared + (i / kQuads << S::kShift) + i % kQuads * 16) = make_uint4(w, v, w, v);
        }
    }
    int* most_of = reinterpret_cast<int*>(shared + l.powers) + kMostColumns;
    if (threadIdx.x < kMostColumns) most_of[threadIdx.x] = 0;
    __syncthreads();
    const cg::cluster_group cluster = cg::this_cluster();
    const int rank = cluster.block_rank(), ranks = cluster.num_blocks();
    const int from = rank * p.slice, blocks = max(0, min(p.slice, m.in - from)) / 64;
    const int tiles = (m.out + 15) / 16, way = warp % p.ways, mine = warp / p.ways;  // the last warps may have nothing to do
    const int stride = gridDim.x / ranks * p.at_once, first_tile = blockIdx.x / ranks * p.at_once;
    const int spans = (p.slice / 64 + S::kSpan - 1) / S::kSpan, each = (spans + p.ways - 1) / p.ways;  // of a slice; for a warp
    const int rounds = (tiles - first_tile + stride - 1) / stride;  // the same for all warps of the cluster
    after_previous();
    let_next_start();

    // A span's copies: 16 bytes a lane, of 32 / (2 kSpan) rows at a time; 4 bytes a lane of scales.
    constexpr int kSpan = S::kSpan, kLanes = 2 * kSpan, kRows = 32 / kLanes, kScaleRows = 32 / kSpan;
    const uint32_t ring = static_cast<uint32_t>(__cvta_generic_to_shared(shared)) + l.rings + warp * (S::kAhead * S::kStage);
    const uint32_t code_to = ring + lane / kLanes * S::kPitch + lane % kLanes * 16, scale_to = ring + 16 * S::kPitch + lane % kSpan * 64 + lane / kSpan * 4;
    const bool whole = reinterpret_cast<uint64_t>(m.codes) % 16 == 0, idle = mine >= p.at_once;
    int ahead_round = 0, ahead_j = 0;
    const auto ask = [&](int stage) {
        if (ahead_round < rounds && !idle) {
            const int row = (first_tile + ahead_round * stride + mine) * 16, last = m.out - 1 - row, block = (way + p.ways * ahead_j) * kSpan;
            const int64_t at = static_cast<int64_t>(row) * m.in + from + 64 * block;
            if (block + lane % kLanes / 2 < blocks) {
                const uint32_t to = code_to + stage * S::kStage;
                const uint8_t* codes = m.codes + at / 2 + lane % kLanes * 16;
#pragma unroll
                for (int k = 0; k < 16; k += kRows) {
                    const uint8_t* here = codes + static_cast<int64_t>(min(k + lane / kLanes, last)) * (m.in / 2);
                    if (whole) {
                        copy16(to + k * S::kPitch, here);
                    } else {
                        copy8(to + k * S::kPitch, here);
                        copy8(to + k * S::kPitch + 8, here + 8);
                    }
                }
            }
            if (block + lane % kSpan < blocks) {
                const float* scales = m.scale + at / 64 + lane % kSpan;
#pragma unroll
                for (int k = 0; k < 16; k += kScaleRows)
                    copy4(scale_to + stage * S::kStage + k * 4, scales + static_cast<int64_t>(min(k + lane / kSpan, last)) * (m.in / 64));
            }
            if (++ahead_j == each) {
                ahead_j = 0;
                ++ahead_round;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const uint32_t place = lane * (kF32 ? 8 : 4);  // of the lane's copy in an entry
    const char* staged = shared + l.rings + warp * (S::kAhead * S::kStage);
    const float* powers = reinterpret_cast<const float*>(shared + l.powers);
    const uint32_t inputs = static_cast<uint32_t>(__cvta_generic_to_shared(shared)) + l.inputs + (r * (p.slice + kPad) + 16 * t) * 2;
    const uint32_t real = 8 * (kTiles - 1) + r < p.columns;  // this lane's column of the product's last 8
    float* sums = reinterpret_cast<float*>(shared + l.sums);
    float* kept = reinterpret_cast<float*>(shared + l.kept);
    const T* bias = static_cast<const T*>(m.bias);
    T* y = static_cast<T*>(m.y) + p.first * m.y_row;
    const auto store = [&](int tile, int column, int row, float v) {
        const int o = tile * 16 + row;
        if (o >= m.out) return;
        if constexpr (kF32) {
            if (bias != nullptr) v += bias[o];
            y[column * m.y_row + o] = v;
        } else {
            if (bias != nullptr) v += __bfloat162float(bias[o]);
            y[column * m.y_row + o] = __float2bfloat16_rn(v);
        }
    };

#pragma unroll
    for (int u = 0; u < S::kAhead; ++u) ask(u);
    stage<T>(p, l, shared, from);
    __syncthreads();
    float acc[kTiles][4];
#pragma unroll
    for (int n = 0; n < kTiles; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.0f;
    // kCount blocks of a span from its block `first` on, whose codes have arrived
    const auto work = [&](const char* stage, int span, int first, auto count) {
        constexpr int kCount = decltype(count)::value;
        float part[kCount][kTiles][4], scale[kCount][2];
        uint32_t codes[kCount][4];
#pragma unroll
        for (int c = 0; c < kCount; ++c) {
            const char* at = stage + (first + c) * 32 + t * 8;
            const uint2 low = *reinterpret_cast<const uint2*>(at + r * S::kPitch), high = *reinterpret_cast<const uint2*>(at + (r + 8) * S::kPitch);
            codes[c][0] = low.x, codes[c][1] = low.y, codes[c][2] = high.x, codes[c][3] = high.y;
            const float* scales = reinterpret_cast<const float*>(stage + 16 * S::kPitch) + (first + c) * 16 + r;
            scale[c][0] = scales[0];
            scale[c][1] = scales[8];
#pragma unroll
            for (int n = 0; n < kTiles; ++n) part[c][n][0] = part[c][n][1] = part[c][n][2] = part[c][n][3] = 0.0f;
        }
        const uint32_t in = inputs + (span * kSpan + first) * 128;
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // 8 columns of a lane's 16
            uint32_t upper[kCount][2][4];  // of two products
            [[maybe_unused]] uint32_t lower[kCount][2][4];
#pragma unroll
            for (int c = 0; c < kCount; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {       // bytes
#pragma unroll
                    for (int g = 0; g < 2; ++g) {   // rows r and r + 8
                        const uint32_t w = codes[c][2 * g + h];
                        uint32_t at;
                        if constexpr (S::kShift == 8) at = __byte_perm(w, place, 0x5504 | e << 4);  // place, byte e, 0, 0
                        else at = ((8 * e >= 7 ? w >> (8 * e - 7) : w << 7) & (255u << 7)) | place;
                        if constexpr (kF32) {
                            const uint2 v = *reinterpret_cast<const uint2*>(shared + at);
                            upper[c][e / 2][g + e % 2 * 2] = v.x;
                            lower[c][e / 2][g + e % 2 * 2] = v.y;
                        } else {
                            upper[c][e / 2][g + e % 2 * 2] = *reinterpret_cast<const uint32_t*>(shared + at);
                        }
                    }
                }
#pragma unroll
            for (int n = 0; n < kTiles; ++n)
#pragma unroll
                for (int c = 0; c < kCount; ++c) {
                    uint4 b = make_uint4(0, 0, 0, 0);  // the last columns may not be real
                    asm volatile(
                        "{\n .reg .pred p;\n setp.ne.u32 p, %5, 0;\n @p ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];\n}"
                        : "+r"(b.x), "+r"(b.y), "+r"(b.z), "+r"(b.w)
                        : "r"(in + 16 * n * (p.slice + kPad) + c * 128 + 16 * h), "r"(n == kTiles - 1 ? real : 1u));
                    mma(part[c][n], upper[c][0], b.x, b.y);
                    mma(part[c][n], upper[c][1], b.z, b.w);
                    if constexpr (kF32) {  // lower parts of levels with upper parts of inputs
                        if (r & 1) b = make_uint4(0, 0, 0, 0);
                        mma(part[c][n], lower[c][0], b.x, b.y);
                        mma(part[c][n], lower[c][1], b.z, b.w);
                    }
                }
        }
#pragma unroll
        for (int c = 0; c < kCount; ++c)
#pragma unroll
            for (int n = 0; n < kTiles; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[n][i] = fmaf(part[c][n][i], scale[c][i / 2], acc[n][i]);
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    const int kWarp = p.rows * kRed;  // floats of a warp's sums
    const auto together = [&]() {     // the warps of a tile
        if (p.ways == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + mine), "r"(32 * p.ways) : "memory");
    };
    int stage_now = 0, slot = 0, held = 0;  // held: rounds whose sums are kept
    for (int round = 0; round < rounds;) {
        if (!idle) {
#pragma unroll 1
            for (int j = 0; j < each; ++j) {
                asm volatile("cp.async.wait_group %0;" ::"n"(S::kAhead - 1) : "memory");
                __syncwarp();
                const int span = way + p.ways * j, here = min(kSpan, blocks - span * kSpan);
                const char* stage = staged + stage_now * S::kStage;
                int first = 0;
                if constexpr (kTiles <= 2) {  // two blocks at a time: their reads and products do not wait for one another
#pragma unroll 1
                    for (; first + 1 < here; first += 2) work(stage, span, first, Two());
                }
#pragma unroll 1
                for (; first < here; ++first) work(stage, span, first, One());
                __syncwarp();
                ask(stage_now);
                stage_now = stage_now == S::kAhead - 1 ? 0 : stage_now + 1;
            }
            float* here = sums + (slot * kMatWarps + warp) * kWarp;
#pragma unroll
            for (int n = 0; n < kTiles; ++n) {
                if constexpr (kF32) {
                    if (4 * n + t < p.rows) {
                        here[(4 * n + t) * kRed + r] = acc[n][0] + acc[n][1];
                        here[(4 * n + t) * kRed + r + 8] = acc[n][2] + acc[n][3];
                    }
                } else {
                    if (8 * n + 2 * t < p.rows) {
                        here[(8 * n + 2 * t) * kRed + r] = acc[n][0];
                        here[(8 * n + 2 * t) * kRed + r + 8] = acc[n][2];
                    }
                    if (8 * n + 2 * t + 1 < p.rows) {
                        here[(8 * n + 2 * t + 1) * kRed + r] = acc[n][1];
                        here[(8 * n + 2 * t + 1) * kRed + r + 8] = acc[n][3];
                    }
                }
                acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.0f;
            }
        }
        ++round;
        if (++slot < p.slots && round < rounds) continue;
        // the sums of `slot` rounds' tiles: all warps' in the order of the ways
        if (!idle) {
            together();
            for (int i = 32 * way + lane; i < slot * p.rows * 16; i += 32 * p.ways) {
                const int k = i / (p.rows * 16), column = i / 16 - k * p.rows, row = i & 15;
                const float* parts = sums + (k * kMatWarps + mine * p.ways) * kWarp + column * kRed + row;
                float v = 0.0f;
#pragma unroll 4
                for (int w = 0; w < p.ways; ++w) v += parts[w * kWarp];
                v *= powers[column];
                if (ranks > 1) kept[(((held + k) * p.at_once + mine) * p.rows + column) * 16 + row] = v;
                else store(first_tile + (round - slot + k) * stride + mine, column, row, v);
            }
            together();
        }
        held += slot;
        slot = 0;
        if (ranks == 1 || ((held + p.slots) * p.at_once <= p.kept && round < rounds)) continue;
        cluster.sync();
        const int values = held * p.at_once * p.rows * 16;
        for (int i = rank * kMatThreads + static_cast<int>(threadIdx.x); i < values; i += ranks * kMatThreads) {
            const int row = i & 15, column = (i >> 4) % p.rows, k = (i >> 4) / p.rows;
            float v = 0.0f;
            for (int w = 0; w < ranks; ++w) v += *cluster.map_shared_rank(kept + i, w);
            store(first_tile + (round - held + k / p.at_once) * stride + k % p.at_once, column, row, v);
        }
        cluster.sync();  // until every CTA's memory has been read
        held = 0;
    }
}

constexpr int kMostShared = 227 * 1024 - 2560;  // of a CTA, beside the table's source

// Clusters of so many CTAs that run at once, asked for once (a cluster's CTAs share a part of the GPU, whose number of SMs
// need not be a multiple of theirs), and the kernel's share of shared memory set.
constexpr int kMatDevices = 64;
template <auto kKernel>
cudaError_t resident(int ranks, int& clusters) {
    static std::atomic<int> known[kMatDevices][4];
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const int which = ranks == 1 ? 0 : ranks == 2 ? 1 : ranks == 4 ? 2 : 3;
    clusters = device < kMatDevices ? known[device][which].load(std::memory_order_relaxed) : 0;
    if (clusters > 0) return cudaSuccess;
    e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute a;
    a.id = cudaLaunchAttributeClusterDimension;
    a.val.clusterDim.x = ranks;
    a.val.clusterDim.y = a.val.clusterDim.z = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(ranks);
    c.blockDim = dim3(kMatThreads);
    c.dynamicSmemBytes = kMostShared;
    c.attrs = &a;
    c.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&clusters, kKernel, &c);
    if (e != cudaSuccess) return e;
    if (clusters < 1) return cudaErrorInvalidConfiguration;
    if (device < kMatDevices) known[device][which].store(clusters, std::memory_order_relaxed);
    return cudaSuccess;
}

template <typename T, int kTiles>
cudaError_t launch_tiles(Params p, int ranks, cudaStream_t s) {
    int clusters = 0;
    const cudaError_t e = resident<q4_matmul_kernel<T, kTiles>>(ranks, clusters);
    if (e != cudaSuccess) return e;
    using S = Shape<T, kTiles>;
    const int tiles = (p.m.out + 15) / 16, blocks = p.slice / 64;
    // How many warps split a slice: what leaves the fewest of them waiting, for one another's spans, for the last tiles and
    // for want of a tile (three warps of 16 without one cost less than a tile in three of a round)
    const int spans = (blocks + S::kSpan - 1) / S::kSpan;
    double best = 0.0;
    for (int ways = kMatWarps; ways >= 1; --ways) {
        const int at_once = kMatWarps / ways, each = (spans + ways - 1) / ways, rounds = (tiles + at_once * clusters - 1) / (at_once * clusters);
        const double busy = static_cast<double>(spans) / (static_cast<double>(each) * ways) * tiles / (static_cast<double>(rounds) * at_once * clusters) *
                            (0.5 + 0.5 * ways * at_once / kMatWarps);
        if (busy <= best * 1.01) continue;
        best = busy;
        p.ways = ways;
        p.at_once = at_once;
    }
    const int used = (tiles + p.at_once - 1) / p.at_once < clusters ? (tiles + p.at_once - 1) / p.at_once : clusters;
    const int rounds = (tiles + p.at_once * used - 1) / (p.at_once * used);
    // sums of as many rounds as there is room for are joined at a time, and kept until the cluster joins them
    const int room = kMostShared - layout_of<S>(p.rows, p.columns, p.slice, 0, 0).all, round_bytes = kMatWarps * p.rows * kRed * 4;
    const int tile_bytes = ranks > 1 ? p.rows * 16 * 4 : 0;
    p.slots = rounds;
    while (p.slots > 1 && p.slots * (round_bytes + p.at_once * tile_bytes) > (room < 48 * 1024 ? room : 48 * 1024)) --p.slots;
    p.kept = 0;
    if (ranks > 1) {
        const int most = (room - p.slots * round_bytes) / tile_bytes, want = (rounds + p.slots - 1) / p.slots * p.slots * p.at_once;
        p.kept = want < most ? want : most;
        if (p.kept < p.slots * p.at_once) return cudaErrorInvalidConfiguration;
    }
    const int shared = layout_of<S>(p.rows, p.columns, p.slice, p.slots, p.kept).all;
    return launch(q4_matmul_kernel<T, kTiles>, used * ranks, kMatThreads, shared, ranks, s, p);
}

// Calls f with the number of the product's columns / 8 as a constant.
template <typename F>
auto with_tiles(int columns, F f) {
    switch ((columns + 7) / 8) {
        case 1: return f(std::integral_constant<int, 1>());
        case 2: return f(std::integral_constant<int, 2>());
        case 3: return f(std::integral_constant<int, 3>());
        case 4: return f(std::integral_constant<int, 4>());
        case 5: return f(std::integral_constant<int, 5>());
        case 6: return f(std::integral_constant<int, 6>());
        case 7: return f(std::integral_constant<int, 7>());
        default: return f(std::integral_constant<int, 8>());
    }
}

template <typename T>
cudaError_t launch_t(Params p, cudaStream_t s) {
    const Q4Matmul& m = p.m;
    const int each = sizeof(T) == 2 ? 1 : 2;  // columns of the product for a row of x
    // The fewest CTAs that hold a slice each of the inputs of the rows at hand and sums of 16 tiles beside them; fewer rows
    // at a time where eight do not, or where they do not hold the last rows (few columns come with a larger table)
    const auto fit = [&](int rows, int ranks) {
        const int slice = (m.in / 64 + ranks - 1) / ranks * 64;
        return with_tiles(rows * each, [&](auto tiles) { return layout_of<Shape<T, tiles.value>>(rows, rows * each, slice, 1, ranks > 1 ? kMatWarps : 0).all <= kMostShared; });
    };
    const auto fits = [&](int rows, int ranks) { return fit(rows, ranks) && (m.n % rows == 0 || fit(m.n % rows, ranks)); };
    int rows = m.n < kMostColumns / each ? m.n : kMostColumns / each, ranks = 1;
    for (;; rows = (rows + 1) / 2) {
        ranks = 1;
        while (ranks < 8 && !fits(rows, ranks)) ranks *= 2;
        if (fits(rows, ranks) || rows == 1) break;
    }
    p.slice = (m.in / 64 + ranks - 1) / ranks * 64;
    for (p.first = 0; p.first < m.n; p.first += rows) {
        p.rows = m.n - p.first < rows ? m.n - p.first : rows;
        p.columns = p.rows * each;
        const cudaError_t e = with_tiles(p.columns, [&](auto tiles) { return launch_tiles<T, tiles.value>(p, ranks, s); });
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_q4_matmul(const Q4Matmul& m, cudaStream_t s) {
    if (q4_by_tiles(m.n, m.out, m.in, m.bf16) && reinterpret_cast<uint64_t>(m.codes) % 16 == 0) return launch_q4_tiles(m, s);
    Params p;
    p.m = m;
    q4_levels_host(p.levels);
    return m.bf16 ? launch_t<__nv_bfloat16>(p, s) : launch_t<float>(p, s);
}

}  // namespace jb
