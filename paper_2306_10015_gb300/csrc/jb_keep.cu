// jb_keep.cu -- of a row's drafted tokens the path to one of them stays.
//
// The nodes of a tree are the last tokens of its row. Those on the path to the leaf move, in order, to the places behind
// the tokens before the tree; the row ends there, and pages behind it are given back. A node's place on the path is not
// behind its place in the tree, so that moving them one after the other, each column of 16 bytes by itself, overwrites
// nothing that is still to be moved.
//
// One CTA checks the list, walks the paths (a warp a tree, the parents in shared memory) and, if nothing is wrong, writes
// lengths, tables and counts and leaves the moves in the workspace; a second kernel moves the tokens of all layers over
// the whole GPU. HBM bounds that one: what moves is read once and written once (64 trees of up to 64 nodes, 24 layers of 32
// heads of 64 in bf16: 59 us, 6.2 TB/s; the plan 12 us, four chains of memory latencies, under the last call's end).
#include "jb_draft.h"
#include "jb_launch.cuh"

namespace jb {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;

// Without the end of the last page, which may lie past 2^31 - 1.
__device__ __forceinline__ int pages_of(int tokens, int page_tokens) { return tokens / page_tokens + (tokens % page_tokens != 0); }

// Workspace: header; count[n], moves of each tree; from[n_nodes] and to[n_nodes] as (page, place in it), a tree's moves
// at its nodes' places in the list.
struct Moves {
    int* count;
    int2* from;
    int2* to;

    __device__ Moves(int* ws, const Trees& t)
        : count(ws + kHeaderWords + 4 * static_cast<size_t>(t.n_nodes)), from(reinterpret_cast<int2*>(ws + kHeaderWords)), to(from + t.n_nodes) {}
};

__global__ void __launch_bounds__(kPlanThreads) keep_plan_kernel(Pages p, Trees t, const int* leaves, int* status, int* ws) {
    extern __shared__ unsigned seen[];  // a bit for each row
    __shared__ short parents[kPlanWarps][kMaxNodes], path[kPlanWarps][kMaxNodes];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    after_previous();
    let_next_start();
    const Moves moves(ws, t);
    for (int i = threadIdx.x; i < (p.n_rows + 31) / 32; i += kPlanThreads) seen[i] = 0;
    __syncthreads();
    const int room = p.row_pages * p.page_tokens;
    bool bad = false;
    for (int i = warp; i < t.n; i += kPlanWarps) {
        const int row = t.rows[i], first = t.starts[i], leaf = leaves[i];
        const int nodes = static_cast<int>(min(static_cast<long long>(t.starts[i + 1]) - first, static_cast<long long>(kMaxNodes + 1)));
        const bool fits = row >= 0 && row < p.n_rows && first >= 0 && nodes >= 0 && nodes <= kMaxNodes && first <= t.n_nodes - nodes &&
                          leaf >= -1 && leaf < nodes && p.lens[row] >= nodes && p.lens[row] <= room;
        int count = -1;  // kept nodes; -1: something is wrong
        if (fits) {
            for (int j = lane; j < nodes; j += 32) {
                const int up = t.parents[first + j];
                parents[warp][j] = static_cast<short>(up >= -1 && up < j ? up : -2);
            }
            __syncwarp();
            if (lane == 0) {  // from the leaf up, to the end of path
                int depth = 0, j = leaf;
                while (j >= 0) {
                    path[warp][kMaxNodes - 1 - depth++] = static_cast<short>(j);
                    j = parents[warp][j];
                }
                count = j == -1 ? depth : -1;
                if (atomicOr(&seen[row >> 5], 1u << (row & 31)) >> (row & 31) & 1u) count = -1;
            }
            count = __shfl_sync(0xFFFFFFFFu, count, 0);
            __syncwarp();
        }
        const int base = fits ? p.lens[row] - nodes : 0;
        const int* entry = p.table + static_cast<size_t>(fits ? row : 0) * p.row_pages;
        int still = 0;  // nodes that are where they belong
        for (int k = lane; k < ((count + 31) & ~31); k += 32) {
            const int j = k < count ? path[warp][kMaxNodes - count + k] : k;
            const unsigned moved = __ballot_sync(0xFFFFFFFFu, j != k);
            if (moved == 0) {
                still = min(k - lane + 32, count);
                continue;
            }
            if (still == k - lane) still += __ffs(moved) - 1;
            if (j == k) continue;
            const int src = base + j, dst = base + k, a = entry[src / p.page_tokens], b = entry[dst / p.page_tokens];
            if (a < 0 || a >= p.n_pages || b < 0 || b >= p.n_pages || p.refs[b] != 1) {
                bad = true;  // a missing page, or one that other rows name too
                continue;
            }
            moves.from[first + k] = make_int2(a, src % p.page_tokens);
            moves.to[first + k] = make_int2(b, dst % p.page_tokens);
        }
        bad = bad || count < 0;
        // moves[first + still ..]: once a node moves, all later ones do
        still = __shfl_sync(0xFFFFFFFFu, still, 0);
        if (lane == 0) moves.count[i] = count < 0 ? 0 : count << 16 | still;
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) {
        ws[0] = bad ? 0 : 1;
        *status = bad ? -1 : 0;
    }
    if (bad) return;
    for (int i = warp; i < t.n; i += kPlanWarps) {
        const int row = t.rows[i], len = p.lens[row], kept = len - (t.starts[i + 1] - t.starts[i]) + (moves.count[i] >> 16);
        int* entry = p.table + static_cast<size_t>(row) * p.row_pages;
        for (int j = pages_of(kept, p.page_tokens) + lane; j < pages_of(len, p.page_tokens); j += 32) {
            const int page = entry[j];
            entry[j] = -1;
            if (page >= 0 && page < p.n_pages) atomicSub(&p.refs[page], 1);
        }
        __syncwarp();
        if (lane == 0) p.lens[row] = kept;
    }
}

// A thread takes a column of 16 bytes of a tree's moved tokens in one pool. blockIdx.x: tree and part of the columns,
// blockIdx.y: the pool.
constexpr int kMoveThreads = 256;
constexpr int kAhead = 8;  // tokens read before the first of them is written
__global__ void __launch_bounds__(kMoveThreads) keep_move_kernel(Pages p, Trees t, const __grid_constant__ Pools pools, int parts, const int* ws) {
    after_previous();
    let_next_start();
    if (ws[0] == 0) return;
    const Moves moves(const_cast<int*>(ws), t);
    const int i = blockIdx.x / parts, column = (blockIdx.x - i * parts) * kMoveThreads + threadIdx.x;
    const int columns = pools.slabs * pools.row_vecs;
    if (column >= columns) return;
    const int count = moves.count[i] >> 16, first = t.starts[i];
    const uint64_t row_bytes = 16ull * pools.row_vecs;
    const uint32_t slab = column / pools.row_vecs;
    char* base = pools.base[blockIdx.y] + slab * (p.page_tokens * row_bytes) + 16ull * (column - slab * pools.row_vecs);
    const auto at = [&](const int2& m) { return reinterpret_cast<uint4*>(base + m.x * pools.stride + m.y * row_bytes); };
    for (int k = moves.count[i] & 0xFFFF; k < count; k += kAhead) {
        uint4 x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (k + u < count) x[u] = *at(moves.from[first + k + u]);
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (k + u < count) *at(moves.to[first + k + u]) = x[u];
    }
}

}  // namespace

cudaError_t launch_keep_plan(const Pages& p, const Trees& t, const int* leaves, int* status, int* ws, cudaStream_t s) {
    return launch(keep_plan_kernel, 1, kPlanThreads, 4ull * ((p.n_rows + 31) / 32), 0, s, p, t, leaves, status, ws);
}

cudaError_t launch_keep_move(const Pages& p, const Trees& t, const Pools& pools, const int* ws, cudaStream_t s) {
    const int parts = static_cast<int>((static_cast<uint64_t>(pools.slabs) * pools.row_vecs + kMoveThreads - 1) / kMoveThreads);
    return launch(keep_move_kernel, dim3(static_cast<unsigned>(t.n) * parts, pools.n), kMoveThreads, 0, 0, s, p, t, pools, parts, ws);
}

}  // namespace jb
