// jb_tree.cuh -- what the kernels of jb_tree.cu share: which queries and positions a tree has, who sees whom, how the
// work is dealt out, and how parts of one row's attention are joined.
//
// The rows of a block are (node, query head of the key head) pairs, nodes first: row r is node r / group. Tiles of
// positions of all (tree, key head, block of rows) are one line, with kCost more for each block, and every CTA of a
// persistent grid takes an equal stretch of it, whatever the rows' lengths. Blocks that a boundary cuts leave (weighted
// values, maximum, sum) in the workspace, which join_kernel adds up in the order of the line: results do not depend on
// which CTA was first.
#pragma once
#include <atomic>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "jb_draft.h"
#include "jb_launch.cuh"
#include "jb_scores.cuh"
#include "jb_tensor_map.h"

namespace jb {
namespace {

constexpr int kGroup = 16;          // pages hold a multiple of so many tokens
constexpr int kMaskWords = kMaxNodes / 32;

}  // namespace

struct TreeParams {
    Pages pages;
    Trees trees;
    TreeAttend a;
    int page_groups;        // groups in a page
    float cap_in, cap_out;  // softcap: scale / cap, cap / ln 2
};

uint64_t tree_workspace_bf16(int head_dim);
cudaError_t launch_tree_bf16(const TreeParams& p, cudaStream_t s);

namespace {

// Tree i: its queries, its row's positions that some node sees, [lo, len), the nodes' among them [base, len), and their
// tiles. tiles == 0: a tree without nodes or one that is not valid, whose queries get zeros.
struct Span {
    int row, first, nodes, base, len, lo, first_tile, tiles, blocks;
};

// kRows rows of a block, kTile positions of a tile, the cost of a block in tiles.
template <int kRows_, int kTile_, int kCost_>
struct Cut {
    static constexpr int kRows = kRows_, kTile = kTile_, kCost = kCost_;
};

template <typename C>
__device__ __forceinline__ Span span_of(const TreeParams& p, int i) {
    Span s;
    s.row = p.trees.rows[i];
    const long long from = p.trees.starts[i], to = p.trees.starts[i + 1];
    const bool listed = from >= 0 && from < to && to <= p.trees.n_nodes;
    s.first = listed ? static_cast<int>(from) : 0;
    s.nodes = listed ? static_cast<int>(to - from) : 0;
    s.base = s.len = s.lo = s.first_tile = s.tiles = s.blocks = 0;
    if (!listed || s.nodes > kMaxNodes || s.row < 0 || s.row >= p.pages.n_rows) return s;
    const int len = p.pages.lens[s.row];
    if (len < s.nodes || len > p.pages.row_pages * p.pages.page_tokens) return s;
    s.len = len;
    s.base = len - s.nodes;
    if (p.a.window > 0) s.lo = max(0, s.base - p.a.window + 1);  // what a root sees
    s.first_tile = s.lo / C::kTile;
    s.tiles = (s.len - 1) / C::kTile + 1 - s.first_tile;
    s.blocks = (s.nodes * p.a.group + C::kRows - 1) / C::kRows;  // group is at most 65536
    return s;
}

// Tiles [from, to) of a block of rows of a tree's key head, at least one.
struct Piece {
    int tree, head, block, from, to;
    long long begin;  // where the block starts on the line
    Span span;
};

__device__ __forceinline__ long long quotient(long long a, long long b) {
    return ((a | b) >> 32) == 0 ? static_cast<long long>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b)) : a / b;
}

// The line, and which CTA has which of it: `each` tiles, and the first `extra` CTAs one more.
struct Line {
    long long total, each;
    int workers, extra;

    __device__ long long bound(int w) const { return each * w + min(w, extra); }
    __device__ int owner(long long x) const {
        const long long longer = (each + 1) * extra;
        return x < longer ? static_cast<int>(quotient(x, each + 1)) : extra + static_cast<int>(quotient(x - longer, each));
    }
};

// Sum of v over the threads before this one, and over all. sums: kThreads / 32 words.
template <int kThreads>
__device__ __forceinline__ long long before_thread(long long v, long long* sums, long long& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long in = v;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const long long o = __shfl_up_sync(0xFFFFFFFFu, in, d);
        if (lane >= d) in += o;
    }
    if (lane == 31) sums[warp] = in;
    __syncthreads();
    long long base = 0;
    total = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) base += sums[w];
        total += sums[w];
    }
    __syncthreads();
    return base + in - v;
}

// Deals a CTA's stretch of the line out in pieces.
template <typename C, int kThreads>
struct Dealer {
    long long next, end, at;  // at: the tree's part of the line before `next`
    Line line;
    int tree;
    Span span;

    // What a tree takes of the line.
    static __device__ long long cost_of(const TreeParams& p, const Span& s) {
        return s.tiles == 0 ? 0 : static_cast<long long>(s.tiles + C::kCost) * s.blocks * p.a.heads;
    }
    static __device__ long long cost_of(const TreeParams& p, int i) { return i < p.trees.n ? cost_of(p, span_of<C>(p, i)) : 0; }

    // The CTA together; kThreads of them. False: the CTA has nothing to do. found: two words of shared memory.
    __device__ bool start(const TreeParams& p, int worker, int ctas, long long* sums, long long* found) {
        long long total = 0, here = 0, mine = 0, before = 0;
        const bool few = p.trees.n <= kThreads;
        for (int first = 0; first < p.trees.n; first += kThreads) {
            mine = cost_of(p, first + static_cast<int>(threadIdx.x));
            before = before_thread<kThreads>(mine, sums, here);
            total += here;
        }
        line.total = total;
        line.workers = static_cast<int>(min(static_cast<long long>(ctas), max(1ll, total / (C::kCost + 1))));
        line.each = quotient(total, line.workers);
        line.extra = static_cast<int>(total - line.each * line.workers);
        next = end = 0;
        if (worker >= line.workers || total == 0) return false;
        next = line.bound(worker);
        end = line.bound(worker + 1);
        // the tree with the place `next`
        const auto look = [&](int i) {
            if (before <= next && next < before + mine) {
                found[0] = i;
                found[1] = before;
            }
        };
        if (few) {
            look(threadIdx.x);
        } else {
            long long base = 0;
            for (int first = 0; base <= next; first += kThreads, base += here) {
                mine = cost_of(p, first + static_cast<int>(threadIdx.x));
                before = base + before_thread<kThreads>(mine, sums, here);
                look(first + threadIdx.x);
            }
        }
        __syncthreads();
        tree = static_cast<int>(found[0]);
        at = next - found[1];
        span = span_of<C>(p, tree);
        return true;
    }
    __device__ bool take(const TreeParams& p, Piece& s) {
        while (next < end) {
            while (at >= cost_of(p, span)) {
                at -= cost_of(p, span);
                ++tree;
                span = span_of<C>(p, tree);
            }
            const int cost = span.tiles + C::kCost, pair = static_cast<int>(quotient(at, cost));
            const int from = static_cast<int>(at - static_cast<long long>(pair) * cost);
            const int to = static_cast<int>(min(static_cast<long long>(cost), from + (end - next)));
            s.begin = next - from;
            next += to - from;
            at += to - from;
            if (to <= C::kCost) continue;  // none of its tiles
            s.tree = tree;
            s.span = span;
            s.head = pair / span.blocks;
            s.block = pair - s.head * span.blocks;
            s.from = max(0, from - C::kCost);
            s.to = to - C::kCost;
            return true;
        }
        return false;
    }
    // The CTA with the block's last tile.
    __device__ int last_of(const Piece& s) const { return line.owner(s.begin + s.span.tiles + C::kCost - 1); }
};

// Who sees whom in a tree: depth of each node (-1: its chain of parents is not valid, and it sees nothing), and of its
// ancestors and itself those within the window, as bits.
struct Nodes {
    unsigned mask[kMaskWords][kMaxNodes];
    int depth[kMaxNodes];
    short jump[kMaxNodes];
};

// kThreads threads together, `rank` among them; any(x): a barrier of them, true if x is in one of them. The chains are
// walked by doubling: after round r a node has the ancestors up to 2^r steps away.
template <int kThreads, typename Any>
__device__ __forceinline__ void fill_nodes(const TreeParams& p, const Span& s, Nodes& t, int rank, Any any) {
    constexpr int kBad = 1 << 20, kEach = (kMaxNodes + kThreads - 1) / kThreads;
    const int words = (s.nodes + 31) / 32;
    bool more = false;
    any(false);  // nobody reads the last tree's any more
    for (int j = rank; j < s.nodes; j += kThreads) {
        const int up = p.trees.parents[s.first + j];
        const bool inner = up >= 0 && up < j;
        t.jump[j] = static_cast<short>(inner ? up : -1);
        t.depth[j] = inner ? 1 : up == -1 ? 0 : kBad;
        for (int w = 0; w < kMaskWords; ++w) t.mask[w][j] = w == j >> 5 ? 1u << (j & 31) : 0;
        more = more || inner;
    }
    while (any(more)) {  // at most 8 rounds: a chain has at most 255 steps
        unsigned mask[kEach][kMaskWords];
        int depth[kEach], jump[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int j = rank + e * kThreads, up = j < s.nodes ? t.jump[j] : -1;
            jump[e] = up;
            if (up < 0) continue;
            depth[e] = min(t.depth[j] + t.depth[up], kBad);
            jump[e] = t.jump[up];
#pragma unroll
            for (int w = 0; w < kMaskWords; ++w)
                if (w < words) mask[e][w] = t.mask[w][j] | t.mask[w][up];
        }
        any(false);
        more = false;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int j = rank + e * kThreads;
            if (j >= s.nodes || t.jump[j] < 0) continue;
            t.depth[j] = depth[e];
            t.jump[j] = static_cast<short>(jump[e]);
#pragma unroll
            for (int w = 0; w < kMaskWords; ++w)
                if (w < words) t.mask[w][j] = mask[e][w];
            more = more || jump[e] >= 0;
        }
    }
    for (int j = rank; j < s.nodes; j += kThreads) {
        const bool valid = t.depth[j] < kBad;
        const int from = valid && p.a.window > 0 ? t.depth[j] - p.a.window : -1;  // ancestors up to this depth are not seen
        if (valid && from < 0) continue;
        for (int w = 0; w < kMaskWords; ++w) {
            unsigned keep = 0;
            for (unsigned m = valid ? t.mask[w][j] : 0; m != 0; m &= m - 1)
                if (t.depth[32 * w + __ffs(m) - 1] > from) keep |= m & -m;
            t.mask[w][j] = keep;
        }
    }
    any(false);
    for (int j = rank; j < s.nodes; j += kThreads)
        if (t.depth[j] >= kBad) t.depth[j] = -1;
    any(false);
}

// Bits of the 32 positions from t on that lie in [lo, hi).
__device__ __forceinline__ unsigned between(int t, int lo, int hi) {
    const int a = max(lo - t, 0), b = min(hi - t, 32);
    if (a >= b) return 0;
    return (b == 32 ? 0xFFFFFFFFu : (1u << b) - 1u) & ~((1u << a) - 1u);
}

// Which of the 32 positions from t on a node of this depth sees.
__device__ __forceinline__ unsigned seen_of(const TreeParams& p, const Span& s, const Nodes& nodes, int node, int depth, int t) {
    if (depth < 0) return 0;
    const int lo = p.a.window > 0 ? max(0, min(s.base, s.base + depth - p.a.window + 1)) : 0;
    unsigned bits = between(t, lo, s.base);
    const int off = t - s.base;
    if (off <= -32 || off >= kMaxNodes) return bits;
    if (off < 0) return bits | nodes.mask[0][node] << -off;
    const int w = off >> 5;
    return bits | __funnelshift_r(nodes.mask[w][node], w + 1 < kMaskWords ? nodes.mask[w + 1][node] : 0u, off & 31);
}

template <typename T>
__device__ __forceinline__ void store_out(T* to, float v);
template <>
__device__ __forceinline__ void store_out<float>(float* to, float v) { *to = v; }
template <>
__device__ __forceinline__ void store_out<__nv_bfloat16>(__nv_bfloat16* to, float v) { *to = __float2bfloat16_rn(v); }

// Zeros for the queries of trees that are not valid.
template <typename T, typename C, int kThreads>
__device__ __forceinline__ void write_zeros(const TreeParams& p) {
    const int d = p.a.head_dim;
    const long long values = static_cast<long long>(p.a.heads) * p.a.group * d;
    for (int i = blockIdx.x; i < p.trees.n; i += gridDim.x) {
        const Span s = span_of<C>(p, i);
        if (s.tiles > 0) continue;
        for (int j = 0; j < s.nodes; ++j)
            for (long long u = threadIdx.x; u < values; u += kThreads)
                store_out(reinterpret_cast<T*>(p.a.out) + (s.first + j) * p.a.out_row + u / d * p.a.out_head + u % d, 0.0f);
    }
}

// The workspace: a note of each CTA, the block that it is the first to have a part of and not the last (rows 0: none); then
// partial results, o[rows][D], m[rows], l[rows]. The first part of a block is in its CTA's slot 1, the others in their
// CTAs' slots 0, so that the end of one block and the start of the next do not meet.
struct Note {
    int first, head, block, last, rows;  // first: node of the tree; last: CTA with the block's end; rows: of the tree
    int pad[3];                          // slots begin on 16 bytes
};
__host__ __device__ constexpr size_t slot_floats(int rows, int d) { return static_cast<size_t>(rows) * (d + 2); }
__host__ __device__ constexpr size_t workspace_floats(int ctas, int rows, int d) { return ctas * (sizeof(Note) / 4 + 2 * slot_floats(rows, d)); }
template <typename C, int D>
__device__ __forceinline__ float* slot_of(const TreeParams& p, int ctas, int worker, bool first) {
    return p.a.ws + ctas * (sizeof(Note) / 4) + slot_floats(C::kRows, D) * (2 * static_cast<size_t>(worker) + (first ? 1 : 0));
}
__device__ __forceinline__ void take_note(const TreeParams& p, const Note& n) { reinterpret_cast<Note*>(p.a.ws)[blockIdx.x] = n; }

// CTA (b, slice) joins a slice of the rows of the block that CTA b has the first part of. A thread adds up four values of
// every part of a row, four parts at a time so that the loads do not wait for one another: a chain of reads (note, then
// maxima, sums and values) is what takes the time. (Four rows one after the other: 3.6 us more
// for 24 ragged rows.)
constexpr int kJoinThreads = 256;
template <typename T, int D, typename C>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ TreeParams p) {
    constexpr int kQuads = D / 4, kAt = kJoinThreads / kQuads, kAhead = 4;  // rows; parts
    constexpr int kRows = C::kRows;
    after_previous();
    let_next_start();
    const Note n = reinterpret_cast<const Note*>(p.a.ws)[blockIdx.x];
    const int quad = threadIdx.x % kQuads, b = blockIdx.x, row = blockIdx.y * kAt + threadIdx.x / kQuads;
    if (4 * quad >= p.a.head_dim || row >= min(kRows, n.rows - n.block * kRows)) return;
    float m = kLowest, l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int w = b; w <= n.last; w += kAhead) {
        float mw[kAhead], lw[kAhead];
        float4 ow[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const float* slot = slot_of<C, D>(p, gridDim.x, min(w + k, n.last), w + k == b);
            mw[k] = w + k <= n.last ? __ldcg(slot + kRows * D + row) : kLowest;
            lw[k] = w + k <= n.last ? __ldcg(slot + kRows * D + kRows + row) : 0.0f;
            ow[k] = w + k <= n.last ? __ldcg(reinterpret_cast<const float4*>(slot + row * D) + quad) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const float top = fmaxf(m, mw[k]), f = exp2_approx(m - top), g = exp2_approx(mw[k] - top);
            l = fmaf(g, lw[k], l * f);
            o = make_float4(fmaf(g, ow[k].x, o.x * f), fmaf(g, ow[k].y, o.y * f), fmaf(g, ow[k].z, o.z * f), fmaf(g, ow[k].w, o.w * f));
            m = top;
        }
    }
    const float inverse = l > 0.0f ? 1.0f / l : 0.0f;
    const int all = n.block * kRows + row, node = all / p.a.group, h = all - node * p.a.group;
    T* out = reinterpret_cast<T*>(p.a.out) + (n.first + node) * p.a.out_row + (n.head * p.a.group + h) * p.a.out_head + 4 * quad;
    store_out(out, o.x * inverse);
    store_out(out + 1, o.y * inverse);
    store_out(out + 2, o.z * inverse);
    store_out(out + 3, o.w * inverse);
}

// Four dimensions, boxes with 128 bytes of the first one, their 16-byte pieces swizzled.
inline bool encoded(Encode encode, CUtensorMap& map, const void* from, CUtensorMapDataType type, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* boxes) {
    const cuuint32_t steps[4] = {1, 1, 1, 1};
    return encode(&map, type, 4, const_cast<void*>(from), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A layer's keys or values, [pages][heads][tokens][elements], in boxes of `box` groups of tokens.
inline cudaError_t describe_pool(Encode encode, CUtensorMap& map, const TreeParams& p, const char* pool, int box, CUtensorMapDataType type, int bytes) {
    const cuuint64_t page = static_cast<cuuint64_t>(p.a.heads) * p.a.head_dim * p.pages.page_tokens;
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(p.a.head_dim), static_cast<cuuint64_t>(p.pages.page_tokens), static_cast<cuuint64_t>(p.a.heads),
                                static_cast<cuuint64_t>(p.pages.n_pages)};
    const cuuint64_t strides[3] = {p.a.token_stride * bytes, p.a.head_stride * bytes, (p.pages.n_pages > 1 ? p.a.page_stride : page) * bytes};
    const cuuint32_t boxes[4] = {static_cast<cuuint32_t>(128 / bytes), static_cast<cuuint32_t>(box * kGroup), 1, 1};
    return encoded(encode, map, pool, type, dims, strides, boxes) ? cudaSuccess : cudaErrorInvalidValue;
}

template <typename T, int D, typename C>
cudaError_t launch_join(const TreeParams& p, int ctas, cudaStream_t s) {
    constexpr int kAt = kJoinThreads / (D / 4);
    return launch(join_kernel<T, D, C>, dim3(ctas, (C::kRows + kAt - 1) / kAt), kJoinThreads, 0, 0, s, p);
}

// CTAs of a kernel, `each` on an SM and `most` at most: the device's SMs are asked for once, and the kernel's share of shared memory set.
constexpr int kDevices = 64;
template <auto kKernel>
cudaError_t resident(int shared, int each, int most, int& ctas) {
    static std::atomic<int> known[kDevices];
    int device = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    ctas = device < kDevices ? known[device].load(std::memory_order_relaxed) : 0;
    if (ctas > 0) return cudaSuccess;
    e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e != cudaSuccess) return e;
    ctas = sms * each < most ? sms * each : most;
    if (device < kDevices) known[device].store(ctas, std::memory_order_relaxed);
    return cudaSuccess;
}

}  // namespace
}  // namespace jb
