// jb_tree.cu -- attention of trees of drafted tokens over the pages of a cache: every node sees the tokens of its row
// before the tree, its ancestors and itself.
//   out = sum_t exp(x_t) v_t / sum_t exp(x_t),  x_t as in jb_attend.cu, positions by depth
#include <atomic>

#include <cuda_bf16.h>

#include "jb_tree.cuh"

namespace jb {
namespace {

constexpr int kThreads = 128;
constexpr int kRows = 16;   // rows of a block
constexpr int kTile = 32;   // positions of a tile
using C = Cut<kRows, kTile, 1>;

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
template <int D>
struct Shared {
    float q[kRows][D];
    float k[kTile][D + 4];
    float v[kTile][D];
    float w[kTile][kRows];
    unsigned seen[kRows];
    float factor[kRows];
    Nodes nodes;
    long long sums[kThreads / 32], found[2];
};

// fp32 arithmetic on the FMA units, tiles of 32 positions against blocks of 16 rows in shared memory.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) tree_kernel(const __grid_constant__ TreeParams p) {
    constexpr int kQuads = D / 4, kGroups = kThreads / kQuads, kEach = kRows / kGroups;  // rows whose values a thread adds up
    extern __shared__ __align__(16) char dynamic[];
    Shared<D>& sh = *reinterpret_cast<Shared<D>*>(dynamic);
    const int d = p.a.head_dim;
    after_previous();
    let_next_start();
    Dealer<C, kThreads> deal;
    const bool work = deal.start(p, blockIdx.x, gridDim.x, sh.sums, sh.found);
    int tree = -1;
    Piece s;
    Note cut = {};
    while (work && deal.take(p, s)) {
        if (s.tree != tree) fill_nodes<kThreads>(p, s.span, sh.nodes, threadIdx.x, [](bool x) { return __syncthreads_or(x); });
        tree = s.tree;
        const int rows = s.span.nodes * p.a.group;
        __syncthreads();
        for (int u = threadIdx.x; u < kRows * kQuads; u += kThreads) {
            const int r = u / kQuads, e = u % kQuads * 4, all = s.block * kRows + r, node = all / p.a.group, h = all - node * p.a.group;
            float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (all < rows && e < d)
                x = load4(reinterpret_cast<const T*>(p.a.q) + (s.span.first + node) * p.a.q_row + (s.head * p.a.group + h) * p.a.q_head + e);
            *reinterpret_cast<float4*>(&sh.q[r][e]) = x;
        }
        // scores: row threadIdx.x / 8, positions threadIdx.x % 8 + 8 i
        const int r = threadIdx.x >> 3, c = threadIdx.x & 7, all = s.block * kRows + r;
        const bool real = all < rows;
        const int node = real ? all / p.a.group : 0, depth = real ? sh.nodes.depth[node] : -1;
        const float slope = real && p.a.slopes != nullptr ? p.a.slopes[s.head * p.a.group + all - node * p.a.group] * kLog2e : 0.0f;
        const int quad = threadIdx.x % kQuads * 4, group = threadIdx.x / kQuads;
        float m = kLowest, l = 0.0f;
        float4 acc[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) acc[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        const int* table = p.pages.table + static_cast<size_t>(s.span.row) * p.pages.row_pages;
        for (int tile = s.span.first_tile + s.from; tile < s.span.first_tile + s.to; ++tile) {
            const int t0 = tile * kTile;
            __syncthreads();
            for (int u = threadIdx.x; u < kTile * kQuads; u += kThreads) {
                const int t = t0 + u / kQuads, e = u % kQuads * 4;
                float4 k = make_float4(0.0f, 0.0f, 0.0f, 0.0f), v = k;
                if (t >= s.span.lo && t < s.span.len && e < d) {
                    const int page = table[t / p.pages.page_tokens];
                    if (page >= 0 && page < p.pages.n_pages) {
                        const uint64_t at = page * p.a.page_stride + s.head * p.a.head_stride + t % p.pages.page_tokens * p.a.token_stride + e;
                        k = load4(reinterpret_cast<const T*>(p.a.k) + at);
                        v = load4(reinterpret_cast<const T*>(p.a.v) + at);
                    }
                }
                *reinterpret_cast<float4*>(&sh.k[u / kQuads][e]) = k;
                *reinterpret_cast<float4*>(&sh.v[u / kQuads][e]) = v;
            }
            unsigned seen = seen_of(p, s.span, sh.nodes, node, depth, t0);
#pragma unroll
            for (int g = 0; g < kTile; g += kGroup) {  // a missing page is not seen
                const int page = t0 + g < s.span.len ? table[(t0 + g) / p.pages.page_tokens] : -1;
                if (page < 0 || page >= p.pages.n_pages) seen &= ~(0xFFFFu << g);
            }
            if (c == 0) sh.seen[r] = seen;
            __syncthreads();
            float x[kTile / 8] = {};
            for (int e = 0; e < D; e += 4) {
                const float4 q = *reinterpret_cast<const float4*>(&sh.q[r][e]);
#pragma unroll
                for (int i = 0; i < kTile / 8; ++i) {
                    const float4 k = *reinterpret_cast<const float4*>(&sh.k[c + 8 * i][e]);
                    x[i] = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, fmaf(q.w, k.w, x[i]))));
                }
            }
            float high = kLowest;
#pragma unroll
            for (int i = 0; i < kTile / 8; ++i) {
                const int t = t0 + c + 8 * i;
                const bool sees = seen >> (c + 8 * i) & 1u;
                const int where = t < s.span.base || !sees ? t : s.span.base + sh.nodes.depth[t - s.span.base];
                x[i] = sees ? score<true>(p, x[i], slope, where - s.span.base - depth) : -INFINITY;
                high = fmaxf(high, x[i]);
            }
#pragma unroll
            for (int u = 1; u < 8; u *= 2) high = fmaxf(high, __shfl_xor_sync(0xFFFFFFFFu, high, u));
            const float top = fmaxf(m, high), f = exp2_approx(m - top);
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < kTile / 8; ++i) {
                x[i] = exp2_approx(x[i] - top);
                sum += x[i];
                sh.w[c + 8 * i][r] = x[i];
            }
#pragma unroll
            for (int u = 1; u < 8; u *= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, u);
            l = fmaf(l, f, sum);
            m = top;
            if (c == 0) sh.factor[r] = f;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const float k = sh.factor[group * kEach + i];
                acc[i] = make_float4(acc[i].x * k, acc[i].y * k, acc[i].z * k, acc[i].w * k);
            }
            for (int u = 0; u < kTile; ++u) {
                const float4 v = *reinterpret_cast<const float4*>(&sh.v[u][quad]);
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    // a value that is not seen must not reach the sum, whatever it holds
                    if (!(sh.seen[group * kEach + i] >> u & 1u)) continue;
                    const float w = sh.w[u][group * kEach + i];
                    acc[i] = make_float4(fmaf(w, v.x, acc[i].x), fmaf(w, v.y, acc[i].y), fmaf(w, v.z, acc[i].z), fmaf(w, v.w, acc[i].w));
                }
            }
        }
        const bool whole = s.from == 0 && s.to == s.span.tiles;
        float* slot = slot_of<C, D>(p, gridDim.x, blockIdx.x, s.from == 0);
        if (s.from == 0 && !whole) cut = {s.span.first, s.head, s.block, deal.last_of(s), s.span.nodes * p.a.group, {}};
        __syncthreads();
        if (c == 0) {
            sh.factor[r] = l > 0.0f ? 1.0f / l : 0.0f;
            if (!whole) {
                slot[kRows * D + r] = m;
                slot[kRows * D + kRows + r] = l;
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int row = group * kEach + i, all_i = s.block * kRows + row;
            if (!whole) {
                *reinterpret_cast<float4*>(slot + row * D + quad) = acc[i];
            } else if (all_i < rows && quad < d) {
                const float k = sh.factor[row];
                const int n = all_i / p.a.group, h = all_i - n * p.a.group;
                T* out = reinterpret_cast<T*>(p.a.out) + (s.span.first + n) * p.a.out_row + (s.head * p.a.group + h) * p.a.out_head + quad;
                store_out(out, acc[i].x * k);
                store_out(out + 1, acc[i].y * k);
                store_out(out + 2, acc[i].z * k);
                store_out(out + 3, acc[i].w * k);
            }
        }
    }
    if (threadIdx.x == 0) take_note(p, cut);
    write_zeros<T, C, kThreads>(p);
}

// SMs of a device and CTAs of a kernel on one, asked for once.
constexpr int kDevices = 64;
template <auto kKernel>
cudaError_t resident(int threads, int shared, int& ctas) {
    static std::atomic<int> known[kDevices];
    int device = 0, sms = 0, each = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    ctas = device < kDevices ? known[device].load(std::memory_order_relaxed) : 0;
    if (ctas > 0) return cudaSuccess;
    if (shared > 48 * 1024) e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, kKernel, threads, shared);
    if (e != cudaSuccess) return e;
    ctas = sms * each < kMaxCtas ? sms * each : kMaxCtas;
    if (ctas < 1) return cudaErrorInvalidConfiguration;
    if (device < kDevices) known[device].store(ctas, std::memory_order_relaxed);
    return cudaSuccess;
}

template <typename T, int D>
cudaError_t launch_d(const TreeParams& p, cudaStream_t s) {
    constexpr int shared = sizeof(Shared<D>);
    int ctas = 0;
    cudaError_t e = resident<tree_kernel<T, D>>(kThreads, shared, ctas);
    if (e != cudaSuccess) return e;
    e = launch(tree_kernel<T, D>, ctas, kThreads, shared, 0, s, p);
    return e != cudaSuccess || ctas == 1 ? e : launch_join<T, D, C>(p, ctas, s);
}

template <typename T>
cudaError_t launch_t(const TreeParams& p, cudaStream_t s) {
    return p.a.head_dim <= 64 ? launch_d<T, 64>(p, s) : p.a.head_dim <= 128 ? launch_d<T, 128>(p, s) : launch_d<T, 256>(p, s);
}

}  // namespace

uint64_t tree_workspace(int bf16, int head_dim) {
    if (bf16) return tree_workspace_bf16(head_dim);
    return sizeof(float) * workspace_floats(kMaxCtas, kRows, head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256);
}

cudaError_t launch_tree(const Pages& pages, const Trees& trees, const TreeAttend& a, cudaStream_t s) {
    const float cap = a.softcap > 0.0f ? a.softcap : 1.0f;
    const TreeParams p = {pages, trees, a, pages.page_tokens / kGroup, a.scale / cap, cap * kLog2e};
    return a.bf16 ? launch_tree_bf16(p, s) : launch_t<float>(p, s);
}

}  // namespace jb
