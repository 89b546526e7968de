// jb_tree.cu -- attention of trees of drafted tokens over the pages of a cache: every node sees the tokens of its row
// before the tree, its ancestors and itself.
//   out = sum_t exp(x_t) v_t / sum_t exp(x_t),  x_t as in jb_attend.cu, positions by depth
//
// Here fp32, on the FMA units (bf16: jb_tree_bf16.cu). A CTA has a block of rows, whose queries are in shared memory, and lets
// the row's keys and values pass by in tiles, which a warp copies ahead (TMA, swizzled by 128 bytes so that 16 rows of keys are
// read without conflicts). A warp takes 8 rows and a part of a tile's positions, and the parts meet at the block's end: half of
// its lanes have four of the rows each, so that a step of four elements is four reads of queries, which all of them share, and
// one or two of keys for up to 16 packed products a lane; weights pass through shared memory to the same rows' lanes, which then
// have columns of the values. The maximum of a row stays as it was until a score exceeds it by 2^8, so that lanes compare
// notes only then.
//
// FMA units bound it where trees are large (four rows of 2000 to 4000 tokens, trees of 64 nodes, 8 query heads of each of 8 key
// heads of 128: 664 us, 38 of 74 TFLOP/s) and HBM where they are small (24 rows of 65 to 2000 tokens, 32 heads of 128, trees of 8
// nodes: 160 us for 72 us of bytes; up to 33 nodes: 253 us). Two warps a scheduler reach neither: each waits for its own
// reads of shared memory and copies of two tiles ahead are all that fits. With 16 rows a warp and the same parts small trees
// took 1.3 to 2.3 times as long, large ones 0.95 to 1.15 times.
#include <numeric>

#include <cuda_bf16.h>

#include "jb_tcgen05.cuh"
#include "jb_tree.cuh"

namespace jb {
namespace {

constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kWarps = 8, kWorkThreads = 32 * kWarps, kThreads = kWorkThreads + 32;  // the last warp copies
constexpr int kRows = 4;        // of a lane; a warp has two times as many
constexpr float kSlack = 8.0f;  // how far a row may exceed its maximum before sums are scaled, in powers of two
constexpr int kSms = 160;       // most

// Heads of up to D elements; kGroups groups of rows, and kWays warps that share a group's positions.
template <int D, int kGroups_>
struct Shape {
    static constexpr int kGroups = kGroups_, kWays = kWarps / kGroups;
    static constexpr int kCtas = D == 64 ? 2 : 1;                    // on an SM
    static constexpr int kBlock = 2 * kRows * kGroups;
    static constexpr int kTile = D == 256 ? 32 : 64, kPos = kTile / kWays, kEach = kPos / 16;  // of a warp; of a lane
    static constexpr int kStages = 2;
    static constexpr int kPanels = D / 32, kPitch = 2 * kRows + 4;    // floats from position to position of the weights
    static constexpr uint32_t kPanel = kTile * 128, kTileBytes = kPanels * kPanel;
    using C = Cut<kBlock, kTile, 1>;
    using Deal = Dealer<C, kThreads>;
    static constexpr int kShared = 1024 + 2 * kStages * kTileBytes + 4 * (kBlock * D + kWarps * kPos * kPitch);
    static_assert(kEach >= 1 && kPos % 16 == 0 && kPos <= 32);
};

struct F32Params {
    TreeParams t;
    CUtensorMap keys, values;
    int box;  // groups of a box, which lie in one page
};

template <typename S>
struct Control {
    unsigned long long full[S::kStages], empty[S::kStages];
    unsigned missing[S::kStages];  // groups of a tile whose page is missing
    int failed, more;
    typename S::Deal deal;
    Piece piece;
    Nodes nodes;
    int depth[S::kBlock], node[S::kBlock];
    float slope[S::kBlock], most[S::kBlock], sum[S::kBlock];
    long long sums[kThreads / 32], found[2];
};

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 read4(uint32_t at) { return *static_cast<const float4*>(__cvta_shared_to_generic(at)); }

// A barrier of the warps that compute, true if x is in one of their threads.
__device__ __forceinline__ bool any_of(bool x) {
    uint32_t any;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.or.pred p, 1, %2, q;\n selp.u32 %0, 1, 0, p;\n}"
                 : "=r"(any) : "r"(static_cast<uint32_t>(x)), "n"(kWorkThreads) : "memory");
    return any != 0;
}

template <typename S, int D>
__device__ void copy_role(const F32Params& f, typename S::Deal deal, Control<S>& c, uint32_t ring) {
    constexpr int kTileGroups = S::kTile / kGroup;
    const TreeParams& p = f.t;
    const int lane = threadIdx.x & 31, panel = lane % S::kPanels, group = lane / S::kPanels * f.box;
    const bool mine = group < kTileGroups && 32 * panel < p.a.head_dim;
    const uint32_t box_bytes = f.box * kGroup * 128;
    uint32_t copies = 0;
    const auto last = [&] {  // what is under way arrives before the role ends, whatever became of the others
        int late = 0;
        for (uint32_t k = copies < S::kStages ? 0 : copies - S::kStages; k < copies; ++k)
            barrier_wait(shared_address(&c.full[k % S::kStages]), k / S::kStages & 1, &late);
    };
    Piece s;
    while (deal.take(p, s)) {
        const int* table = p.pages.table + static_cast<size_t>(s.span.row) * p.pages.row_pages;
        for (int tile = s.span.first_tile + s.from; tile < s.span.first_tile + s.to; ++tile, ++copies) {
            const int g = tile * kTileGroups + group, page = mine && g * kGroup < s.span.len ? table[g / p.page_groups] : -1;
            const bool real = page >= 0 && page < p.pages.n_pages;
            const unsigned boxes = __ballot_sync(kAll, real);
            unsigned missing = 0;  // groups, from the boxes of the first panel
            for (int k = 0; k < kTileGroups; ++k)
                if (!(boxes >> (k / f.box * S::kPanels) & 1u)) missing |= 1u << k;
            const uint32_t stage = copies % S::kStages, bar = shared_address(&c.full[stage]), to = ring + 2 * stage * S::kTileBytes + panel * S::kPanel + group * (kGroup * 128);
            if (!__all_sync(kAll, barrier_wait(shared_address(&c.empty[stage]), (copies / S::kStages & 1) ^ 1, &c.failed))) return last();
            if (lane == 0) {
                *static_cast<volatile unsigned*>(&c.missing[stage]) = missing;
                barrier_arrive_bytes(bar, 2 * __popc(boxes) * box_bytes);
            }
            __syncwarp();
            if (real) {
                copy_box(to, &f.keys, 32 * panel, g % p.page_groups * kGroup, s.head, page, bar);
                copy_box(to + S::kTileBytes, &f.values, 32 * panel, g % p.page_groups * kGroup, s.head, page, bar);
            }
            __syncwarp();
        }
    }
    last();
}

// kExtra: a cap or a bias on the scores.
template <typename S, int D, bool kExtra>
__device__ void work_role(const TreeParams& p, Control<S>& c, uint32_t ring, float* queries, float* all_weights) {
    constexpr int kEach = S::kEach, kPos = S::kPos, kPairs = D / 32;  // pairs of columns of a lane
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = warp % S::kGroups, way = warp / S::kGroups, d = p.a.head_dim;
    const int half = lane >> 4, place = lane & 15, row0 = group * (2 * kRows) + half * kRows;  // the lane's first row
    float* weights = all_weights + warp * (kPos * S::kPitch);
    const uint32_t query_at = shared_address(queries) + row0 * (D * 4), weights_at = shared_address(weights) + half * kRows * 4;
    const Piece& s = c.piece;
    uint32_t tiles = 0;
    int tree = -1;
    bool ok = true;  // a wait that gives up leaves the loops as they are: other warps may wait for this one
    for (;;) {
        any_of(false);  // nobody reads the last piece, its queries and its parts any more
        if (threadIdx.x == 0) c.more = c.deal.take(p, c.piece);
        any_of(false);
        if (c.more == 0) break;
        if (s.tree != tree) fill_nodes<kWorkThreads>(p, s.span, c.nodes, threadIdx.x, any_of);
        tree = s.tree;
        const int rows = s.span.nodes * p.a.group;
        const bool whole = s.from == 0 && s.to == s.span.tiles;
        if (threadIdx.x == 0 && s.from == 0 && !whole) take_note(p, {s.span.first, s.head, s.block, c.deal.last_of(s), rows, {}});
        for (int u = threadIdx.x; u < S::kBlock * (D / 4); u += kWorkThreads) {
            const int r = u / (D / 4), e = u % (D / 4) * 4, all = s.block * S::kBlock + r, node = all / p.a.group, h = all - node * p.a.group;
            float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (all < rows && e < d)
                x = load4(reinterpret_cast<const float*>(p.a.q) + (s.span.first + node) * p.a.q_row + (s.head * p.a.group + h) * p.a.q_head + e);
            *reinterpret_cast<float4*>(queries + r * D + e) = x;
        }
        if (threadIdx.x < S::kBlock) {
            const int all = s.block * S::kBlock + threadIdx.x, node = all < rows ? all / p.a.group : 0;
            c.node[threadIdx.x] = node;
            c.depth[threadIdx.x] = all < rows ? c.nodes.depth[node] : -1;
            c.slope[threadIdx.x] = kExtra && all < rows && p.a.slopes != nullptr ? p.a.slopes[s.head * p.a.group + all - node * p.a.group] * kLog2e : 0.0f;
        }
        any_of(false);
        const bool idle = s.block * S::kBlock + group * 2 * kRows >= rows;
        float m[kRows], l[kRows];
        float2 acc[kRows][kPairs];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            m[i] = kLowest;
            l[i] = 0.0f;
#pragma unroll
            for (int q = 0; q < kPairs; ++q) acc[i][q] = make_float2(0.0f, 0.0f);
        }
        for (int tile = s.span.first_tile + s.from; tile < s.span.first_tile + s.to; ++tile, ++tiles) {
            const uint32_t stage = tiles % S::kStages, keys = ring + 2 * stage * S::kTileBytes, values = keys + S::kTileBytes;
            const int t0 = tile * S::kTile + way * kPos;
            ok = barrier_wait(shared_address(&c.full[stage]), tiles / S::kStages & 1, &c.failed) && ok;
            __syncwarp();
            if (!idle) {
                const unsigned missing = *static_cast<volatile unsigned*>(&c.missing[stage]) >> (way * kPos / kGroup);
                const bool edge = missing != 0 || s.span.base - t0 < kPos || (p.a.window > 0 && t0 < static_cast<long long>(s.span.base) + kMaxNodes - p.a.window);
                // scores of the lane's rows at positions place and place + 16 of the warp's
                float2 x[kRows][kEach];
#pragma unroll
                for (int i = 0; i < kRows; ++i)
#pragma unroll
                    for (int j = 0; j < kEach; ++j) x[i][j] = make_float2(0.0f, 0.0f);
                const uint32_t key_at = keys + (way * kPos + place) * 128;
#pragma unroll 1
                for (int panel = 0; 32 * panel < d; ++panel) {
#pragma unroll
                    for (int piece = 0; piece < 8; ++piece) {  // beyond the head's end copies put zeros
                        const uint32_t at = key_at + panel * S::kPanel + ((piece ^ (place & 7)) << 4);
                        float4 k[kEach];
#pragma unroll
                        for (int j = 0; j < kEach; ++j) k[j] = read4(at + j * (16 * 128));
#pragma unroll
                        for (int i = 0; i < kRows; ++i) {
                            const float4 q = read4(query_at + i * (D * 4) + panel * 128 + piece * 16);
#pragma unroll
                            for (int j = 0; j < kEach; ++j) {
                                x[i][j] = __ffma2_rn(make_float2(q.x, q.y), make_float2(k[j].x, k[j].y), x[i][j]);
                                x[i][j] = __ffma2_rn(make_float2(q.z, q.w), make_float2(k[j].z, k[j].w), x[i][j]);
                            }
                        }
                    }
                }
                unsigned seen[kRows];
                if (edge) {
                    const int mine = row0 + (lane & (kRows - 1));
                    unsigned bits = seen_of(p, s.span, c.nodes, c.node[mine], c.depth[mine], t0);
                    if (missing & 1u) bits &= 0xFFFF0000u;
                    if (missing & 2u) bits &= 0x0000FFFFu;
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < kRows; ++i) seen[i] = __shfl_sync(kAll, bits, (lane & 16) + i);
                }
                bool rises = false;
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
#pragma unroll
                    for (int j = 0; j < kEach; ++j) {
                        const int at = place + 16 * j;
                        float y = x[i][j].x + x[i][j].y;
                        const bool sees = !edge || (seen[i] >> at & 1u);
                        if constexpr (kExtra) {
                            const int t = t0 + at, depth = c.depth[row0 + i];
                            int back = t - s.span.base - depth;
                            if (t >= s.span.base && sees) back = c.nodes.depth[t - s.span.base] - depth;
                            y = score<true>(p, y, c.slope[row0 + i], back);
                        } else {
                            y *= p.a.scale * kLog2e;
                        }
                        y = sees ? y : -INFINITY;
                        rises = rises || (y > m[i] && (m[i] == kLowest || y - m[i] > kSlack));
                        x[i][j].x = y;
                    }
                }
                if (__any_sync(kAll, rises)) {
#pragma unroll
                    for (int i = 0; i < kRows; ++i) {
                        float top = m[i];
#pragma unroll
                        for (int j = 0; j < kEach; ++j) top = fmaxf(top, x[i][j].x);
#pragma unroll
                        for (int u = 1; u < 16; u *= 2) top = fmaxf(top, __shfl_xor_sync(kAll, top, u));
                        const float k = exp2_approx(m[i] - top);
                        m[i] = top;
                        l[i] *= k;
#pragma unroll
                        for (int q = 0; q < kPairs; ++q) acc[i][q] = __fmul2_rn(acc[i][q], make_float2(k, k));
                    }
                }
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    float w[kRows];
#pragma unroll
                    for (int i = 0; i < kRows; ++i) {
                        w[i] = exp2_approx(x[i][j].x - m[i]);
                        l[i] += w[i];
                    }
#pragma unroll
                    for (int i = 0; i < kRows; i += 4)
                        *reinterpret_cast<float4*>(weights + (place + 16 * j) * S::kPitch + half * kRows + i) = make_float4(w[i], w[i + 1], w[i + 2], w[i + 3]);
                }
                __syncwarp();
                // columns 4 place .. + 3 of every 64
                const uint32_t value_at = values + (place >> 3) * S::kPanel + way * kPos * 128;
                const auto add = [&](int u, auto sees) {
                    float w[kRows];
#pragma unroll
                    for (int i = 0; i < kRows; i += 4) {
                        const float4 y = read4(weights_at + u * (S::kPitch * 4) + i * 4);
                        w[i] = y.x, w[i + 1] = y.y, w[i + 2] = y.z, w[i + 3] = y.w;
                    }
#pragma unroll
                    for (int q = 0; q < kPairs; q += 2) {
                        const float4 v = read4(value_at + q * S::kPanel + u * 128 + (((place & 7) ^ (u & 7)) << 4));
#pragma unroll
                        for (int i = 0; i < kRows; ++i) {
                            if (!sees(i)) continue;
                            acc[i][q] = __ffma2_rn(make_float2(w[i], w[i]), make_float2(v.x, v.y), acc[i][q]);
                            acc[i][q + 1] = __ffma2_rn(make_float2(w[i], w[i]), make_float2(v.z, v.w), acc[i][q + 1]);
                        }
                    }
                };
                if (edge) {  // a value that is not seen must not reach the sum, whatever it holds
#pragma unroll 1
                    for (int u = 0; u < kPos; ++u) add(u, [&](int i) { return (seen[i] >> u & 1u) != 0; });
                } else {
#pragma unroll 4
                    for (int u = 0; u < kPos; ++u) add(u, [](int) { return true; });
                }
                __syncwarp();
            }
            if (lane == 0) barrier_arrive(shared_address(&c.empty[stage]));
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i)
#pragma unroll
            for (int u = 1; u < 16; u *= 2) l[i] += __shfl_xor_sync(kAll, l[i], u);
        // the ways' parts one after the other, through the queries' place
        for (int w = 1; w < S::kWays; ++w) {
            any_of(false);
            if (way == w && !idle) {
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    if (place == 0) {
                        c.most[row0 + i] = m[i];
                        c.sum[row0 + i] = l[i];
                    }
#pragma unroll
                    for (int q = 0; q < kPairs; q += 2)
                        *reinterpret_cast<float4*>(queries + (row0 + i) * D + 32 * q + 4 * place) = make_float4(acc[i][q].x, acc[i][q].y, acc[i][q + 1].x, acc[i][q + 1].y);
                }
            }
            any_of(false);
            if (way == 0 && !idle) {
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    const float other = c.most[row0 + i], top = fmaxf(m[i], other), k = exp2_approx(m[i] - top), by = exp2_approx(other - top);
                    m[i] = top;
                    l[i] = fmaf(c.sum[row0 + i], by, l[i] * k);
#pragma unroll
                    for (int q = 0; q < kPairs; q += 2) {
                        const float4 o = load4(queries + (row0 + i) * D + 32 * q + 4 * place);
                        acc[i][q] = make_float2(fmaf(o.x, by, acc[i][q].x * k), fmaf(o.y, by, acc[i][q].y * k));
                        acc[i][q + 1] = make_float2(fmaf(o.z, by, acc[i][q + 1].x * k), fmaf(o.w, by, acc[i][q + 1].y * k));
                    }
                }
            }
        }
        if (way != 0 || idle) continue;
        float* slot = slot_of<typename S::C, D>(p, gridDim.x, blockIdx.x, s.from == 0);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int row = row0 + i, all = s.block * S::kBlock + row, node = c.node[row], h = all - node * p.a.group;
            if (all >= rows) continue;
            const bool none = c.depth[row] < 0;  // its chain of parents is not valid
            const float k = !ok ? NAN : whole ? (l[i] > 0.0f ? 1.0f / l[i] : 0.0f) : 1.0f;
            float* to = whole ? reinterpret_cast<float*>(p.a.out) + (s.span.first + node) * p.a.out_row + (s.head * p.a.group + h) * p.a.out_head : slot + row * D;
            if (!whole && place == 0) {
                slot[S::kBlock * D + row] = none ? kLowest : m[i];
                slot[S::kBlock * D + S::kBlock + row] = none ? 0.0f : l[i];
            }
#pragma unroll
            for (int q = 0; q < kPairs; q += 2) {
                const int e = 32 * q + 4 * place;
                if (e >= d) continue;
                *reinterpret_cast<float4*>(to + e) = none ? make_float4(0.0f, 0.0f, 0.0f, 0.0f)
                                                          : make_float4(acc[i][q].x * k, acc[i][q].y * k, acc[i][q + 1].x * k, acc[i][q + 1].y * k);
            }
        }
    }
}

template <int D, int kGroups, bool kExtra>
__global__ void __launch_bounds__(kThreads, Shape<D, kGroups>::kCtas) tree_kernel(const __grid_constant__ F32Params f) {
    using S = Shape<D, kGroups>;
    const TreeParams& p = f.t;
    extern __shared__ char dynamic[];
    __shared__ Control<S> c;
    const int warp = same(static_cast<int>(threadIdx.x) >> 5);
    const uint32_t ring = (shared_address(dynamic) + 1023) & ~1023u;
    float* queries = reinterpret_cast<float*>(dynamic + (ring - shared_address(dynamic)) + 2 * S::kStages * S::kTileBytes);
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            barrier_init(shared_address(&c.full[i]), 1);
            barrier_init(shared_address(&c.empty[i]), kWarps);
        }
        c.failed = 0;
        barriers_initialized();
    }
    __syncthreads();
    after_previous();
    let_next_start();
    typename S::Deal deal;
    const bool work = deal.start(p, blockIdx.x, gridDim.x, c.sums, c.found);
    if (threadIdx.x == 0) {
        take_note(p, {});
        c.deal = deal;
    }
    if (work) {
        if (warp == kWarps) copy_role<S, D>(f, deal, c, ring);
        else work_role<S, D, kExtra>(p, c, ring, queries, queries + S::kBlock * D);
    }
    __syncthreads();
    write_zeros<float, typename S::C, kThreads>(p);
}

template <int D, int kGroups, bool kExtra>
cudaError_t launch_extra(const TreeParams& p, cudaStream_t s) {
    using S = Shape<D, kGroups>;
    int ctas = 0;
    cudaError_t e = resident<tree_kernel<D, kGroups, kExtra>>(S::kShared, S::kCtas, kSms * S::kCtas, ctas);
    if (e != cudaSuccess) return e;
    F32Params f;
    f.t = p;
    f.box = std::gcd(p.page_groups, S::kTile / kGroup);
    Encode encode = nullptr;
    e = encoder(encode);
    if (e == cudaSuccess) e = describe_pool(encode, f.keys, p, p.a.k, f.box, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4);
    if (e == cudaSuccess) e = describe_pool(encode, f.values, p, p.a.v, f.box, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4);
    if (e == cudaSuccess) e = launch(tree_kernel<D, kGroups, kExtra>, ctas, kThreads, S::kShared, 0, s, f);
    return e != cudaSuccess || ctas == 1 ? e : launch_join<float, D, typename S::C>(p, ctas, s);
}

template <int D, int kGroups>
cudaError_t launch_groups(const TreeParams& p, cudaStream_t s) {
    return p.a.slopes != nullptr || p.a.softcap > 0.0f ? launch_extra<D, kGroups, true>(p, s) : launch_extra<D, kGroups, false>(p, s);
}

// Blocks of 16 rows for small trees, of 32 for others. Measured with 16 rows of 400 to 1000 tokens, 32 heads of 128, the first
// and the second in us: trees of 8 nodes 115 and 168, of 16 134 and 175, of 20 234 and 183, of 64 520 and 403.
template <int D>
cudaError_t launch_d(const TreeParams& p, cudaStream_t s) {
    if constexpr (D < 256)
        if (static_cast<long long>(p.trees.n_nodes) * p.a.group <= 16ll * p.trees.n) return launch_groups<D, 2>(p, s);
    return launch_groups<D, 4>(p, s);
}

template <int D>
constexpr size_t floats_of() { return workspace_floats(kSms * Shape<D, 4>::kCtas, Shape<D, 4>::kBlock, D); }

}  // namespace

uint64_t tree_workspace(int bf16, int head_dim) {
    if (bf16) return tree_workspace_bf16(head_dim);
    return sizeof(float) * (head_dim <= 64 ? floats_of<64>() : head_dim <= 128 ? floats_of<128>() : floats_of<256>());
}

cudaError_t launch_tree(const Pages& pages, const Trees& trees, const TreeAttend& a, cudaStream_t s) {
    const float cap = a.softcap > 0.0f ? a.softcap : 1.0f;
    const TreeParams p = {pages, trees, a, pages.page_tokens / kGroup, a.scale / cap, cap * kLog2e};
    if (a.bf16) return launch_tree_bf16(p, s);
    return a.head_dim <= 64 ? launch_d<64>(p, s) : a.head_dim <= 128 ? launch_d<128>(p, s) : launch_d<256>(p, s);
}

}  // namespace jb
