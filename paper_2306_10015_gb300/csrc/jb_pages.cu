// jb_pages.cu -- the pages of a cache: reserve, free, fork, compact, write.
//
// Which pages are free is decided on the device: nothing is read back, and the ids are those of
// the definition (the lowest free ones, in the order of the list), whatever the launch. A plan
// kernel ranks the free pages in one cluster of CTAs, each over a slice of the counts; what moves
// data runs after it over the whole GPU.
#include <cooperative_groups.h>

#include "jb_answer.h"

namespace jb {
namespace {

namespace cg = cooperative_groups;

constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;
constexpr unsigned kAll = 0xFFFFFFFFu;

__device__ __forceinline__ int warp_inclusive(int v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int o = __shfl_up_sync(kAll, v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// Exclusive prefix of v over the CTA's threads; `total` is the sum. sums: kPlanWarps words.
__device__ __forceinline__ int block_exclusive(int v, int* sums, int& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int in = warp_inclusive(v);
    if (lane == 31) sums[warp] = in;
    __syncthreads();
    const int all = warp_inclusive(lane < kPlanWarps ? sums[lane] : 0);
    const int before = __shfl_sync(kAll, all, warp == 0 ? 0 : warp - 1);
    total = __shfl_sync(kAll, all, 31);
    __syncthreads();
    return in - v + (warp == 0 ? 0 : before);
}

__device__ __forceinline__ int block_sum(int v, int* sums) {
    int total;
    block_exclusive(v, sums, total);
    return total;
}

// emit(page, rank) for the pages of [lo, hi) with flag(page), ascending, ranks from `start` on;
// ranks from `stop` on are left out.
template <typename Flag, typename Emit>
__device__ __forceinline__ void ranked(int lo, int hi, int start, int stop, int* sums, Flag flag, Emit emit) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int tile = lo; tile < hi && start < stop; tile += 4 * kPlanThreads) {
        unsigned bits[4];
        int mine = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int page = tile + warp * 128 + k * 32 + lane;
            bits[k] = __ballot_sync(kAll, page < hi && flag(page));
            mine += __popc(bits[k]);
        }
        int total;
        // the warp's count enters the prefix once, by its first lane
        int rank = start + block_exclusive(lane == 0 ? mine : 0, sums, total);
        rank = __shfl_sync(kAll, rank, 0);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int r = rank + __popc(bits[k] & ((1u << lane) - 1u));
            if ((bits[k] >> lane & 1u) && r < stop) emit(tile + warp * 128 + k * 32 + lane, r);
            rank += __popc(bits[k]);
        }
        start += total;
    }
}

__device__ __forceinline__ int pages_of(long long tokens, int page_tokens) {
    return static_cast<int>((tokens + page_tokens - 1) / page_tokens);
}

// Tokens of a row, within what its row of the table can hold.
__device__ __forceinline__ int row_len(const Pages& p, int row) {
    return min(max(p.lens[row], 0), p.row_pages * p.page_tokens);
}

// The cluster's slice of the pages, and the free pages before it and in all.
struct Slice {
    int lo, hi, before, total;
};

// `mine`: a word of shared memory that the other CTAs read. Ends with the CTAs in step.
template <typename Flag>
__device__ __forceinline__ Slice count_pages(int n_pages, int* sums, int* mine, Flag flag) {
    const cg::cluster_group cluster = cg::this_cluster();
    const int ctas = cluster.num_blocks(), rank = cluster.block_rank();
    const int per = (n_pages + ctas - 1) / ctas;
    Slice s;
    s.lo = min(rank * per, n_pages);
    s.hi = min(s.lo + per, n_pages);
    int n = 0;
    for (int i = s.lo + threadIdx.x; i < s.hi; i += kPlanThreads) n += flag(i) ? 1 : 0;
    n = block_sum(n, sums);
    if (threadIdx.x == 0) *mine = n;
    cluster.sync();
    s.before = s.total = 0;
    for (int c = 0; c < ctas; ++c) {
        const int v = *cluster.map_shared_rank(mine, c);
        if (c < rank) s.before += v;
        s.total += v;
    }
    cluster.sync();
    return s;
}

__device__ __forceinline__ void clear_seen(unsigned* seen, int n_rows) {
    for (int i = threadIdx.x; i < (n_rows + 31) / 32; i += kPlanThreads) seen[i] = 0;
}

// Marks a row; true if it was marked before.
__device__ __forceinline__ bool seen_before(unsigned* seen, int row) {
    const unsigned bit = 1u << (row & 31);
    return (atomicOr(&seen[row >> 5], bit) & bit) != 0;
}

// Dynamic shared memory of the plans: base[n + 1], then a bit for each row.
__device__ __forceinline__ int owner_of(const int* base, int n, int rank) {
    int lo = 0, hi = n - 1;  // the last i with base[i] <= rank
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (base[mid] <= rank) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__global__ void __launch_bounds__(kPlanThreads) reserve_kernel(Pages p, const int* rows, const int* tokens, int n,
                                                               int* status) {
    extern __shared__ int dynamic[];
    __shared__ int sums[kPlanWarps];
    __shared__ int free_here;
    int* base = dynamic;
    unsigned* seen = reinterpret_cast<unsigned*>(dynamic + n);
    const cg::cluster_group cluster = cg::this_cluster();

    // every CTA works the list out for itself
    clear_seen(seen, p.n_rows);
    __syncthreads();
    int need_all = 0;
    bool bad = false;
    for (int first = 0; first < n; first += kPlanThreads) {
        const int i = first + threadIdx.x;
        int need = 0;
        if (i < n) {
            const int row = rows[i], more = tokens[i];
            if (row < 0 || row >= p.n_rows || more < 0 || seen_before(seen, row)) {
                bad = true;
            } else {
                const int len = row_len(p, row);
                const long long want = static_cast<long long>(len) + more;
                if (want > static_cast<long long>(p.row_pages) * p.page_tokens) bad = true;
                else need = pages_of(want, p.page_tokens) - pages_of(len, p.page_tokens);
            }
        }
        int total;
        const int at = need_all + block_exclusive(need, sums, total);
        if (i < n) base[i] = at;
        // more than all pages: the exact number no longer matters, but it must not wrap
        need_all = min(need_all + total, 0x3FFFFFFF);
    }
    bad = __syncthreads_or(bad);
    const Slice s = count_pages(p.n_pages, sums, &free_here, [&](int i) { return p.refs[i] == 0; });
    const bool first_thread = cluster.block_rank() == 0 && threadIdx.x == 0;
    if (bad || need_all > s.total) {
        if (first_thread) *status = bad ? -1 : need_all - s.total;
        return;
    }
    ranked(s.lo, s.hi, s.before, need_all, sums, [&](int page) { return p.refs[page] == 0; },
           [&](int page, int rank) {
               const int i = owner_of(base, n, rank);
               const int row = rows[i];
               const int at = pages_of(row_len(p, row), p.page_tokens) + rank - base[i];
               p.table[static_cast<size_t>(row) * p.row_pages + at] = page;
               p.refs[page] = 1;
           });
    cluster.sync();  // the lengths are read until here
    if (cluster.block_rank() == 0) {
        for (int i = threadIdx.x; i < n; i += kPlanThreads) p.lens[rows[i]] = row_len(p, rows[i]) + tokens[i];
        if (threadIdx.x == 0) *status = 0;
    }
}

// One CTA a row. Entries are taken out one by one, so a row listed twice is released once.
__global__ void __launch_bounds__(256) free_kernel(Pages p, const int* rows) {
    const int row = rows[blockIdx.x];
    if (row < 0 || row >= p.n_rows) return;
    int* entry = p.table + static_cast<size_t>(row) * p.row_pages;
    for (int j = threadIdx.x; j < p.row_pages; j += 256) {
        if (entry[j] < 0) continue;
        const int page = atomicExch(&entry[j], -1);
        if (page >= 0 && page < p.n_pages) atomicSub(&p.refs[page], 1);
    }
    if (threadIdx.x == 0) p.lens[row] = 0;
}

// Workspace of a fork: header, fresh[n] (the page that takes the last tokens, or -1), len[n] (tokens
// of the parent, or -1: nothing to do), stage[n][row_pages] (the parents' entries).
__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(Pages p, const int* parents, const int* children,
                                                                 int n, int* status, int* ws) {
    extern __shared__ int dynamic[];
    __shared__ int sums[kPlanWarps];
    __shared__ int free_here;
    int* base = dynamic;
    unsigned* seen = reinterpret_cast<unsigned*>(dynamic + n);
    const cg::cluster_group cluster = cg::this_cluster();
    int* fresh = ws + kHeaderWords;
    int* len = fresh + n;

    clear_seen(seen, p.n_rows);
    __syncthreads();
    int need_all = 0;
    bool bad = false;
    for (int first = 0; first < n; first += kPlanThreads) {
        const int i = first + threadIdx.x;
        int need = 0;
        if (i < n) {
            const int a = parents[i], b = children[i];
            if (a < 0 || a >= p.n_rows || b < 0 || b >= p.n_rows || seen_before(seen, b)) bad = true;
            else need = a != b && row_len(p, a) % p.page_tokens != 0;
        }
        int total;
        const int at = need_all + block_exclusive(need, sums, total);
        if (i < n) base[i] = at;
        need_all += total;
    }
    bad = __syncthreads_or(bad);
    const Slice s = count_pages(p.n_pages, sums, &free_here, [&](int i) { return p.refs[i] == 0; });
    const bool go = !bad && need_all <= s.total;
    if (cluster.block_rank() == 0) {
        for (int i = threadIdx.x; i < n; i += kPlanThreads) {
            const bool moves = go && parents[i] != children[i];
            len[i] = moves ? row_len(p, parents[i]) : -1;
            if (!(moves && len[i] % p.page_tokens != 0)) fresh[i] = -1;
        }
        if (threadIdx.x == 0) *status = bad ? -1 : max(need_all - s.total, 0);
    }
    if (!go) return;
    ranked(s.lo, s.hi, s.before, need_all, sums, [&](int page) { return p.refs[page] == 0; },
           [&](int page, int rank) {
               fresh[owner_of(base, n, rank)] = page;
               p.refs[page] = 1;
           });
}

// A run of 16-byte vectors, four in flight a thread.
template <typename At>
__device__ __forceinline__ void copy_vectors(uint32_t first, uint32_t n, uint32_t step, At at) {
    uint32_t v = first;
    for (; v + 3 * step < n; v += 4 * step) {
        uint4 x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = *reinterpret_cast<const uint4*>(at(v + k * step).first);
#pragma unroll
        for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(at(v + k * step).second) = x[k];
    }
    for (; v < n; v += step) *reinterpret_cast<uint4*>(at(v).second) = *reinterpret_cast<const uint4*>(at(v).first);
}

struct Ends {
    const char* first;
    char* second;
};

// One CTA for a pair's last page in one pool: the valid tokens of each slab.
__global__ void __launch_bounds__(256) fork_copy_kernel(Pages p, const __grid_constant__ Pools pools,
                                                        const int* parents, int n, const int* ws) {
    const int i = blockIdx.x / pools.n, pool = blockIdx.x % pools.n;
    const int to = ws[kHeaderWords + i], len = ws[kHeaderWords + n + i];
    if (to < 0) return;
    const int from = p.table[static_cast<size_t>(parents[i]) * p.row_pages + len / p.page_tokens];
    if (from < 0 || from >= p.n_pages) return;
    const uint32_t run = (len % p.page_tokens) * pools.row_vecs, whole = p.page_tokens * pools.row_vecs;
    const char* src = pools.base[pool] + from * pools.stride;
    char* dst = pools.base[pool] + to * pools.stride;
    copy_vectors(threadIdx.x, run * pools.slabs, 256, [&](uint32_t v) {
        const uint64_t at = 16ull * (v / run * whole + v % run);
        return Ends{src + at, dst + at};
    });
}

// The parents' entries are set aside before any row is written: a parent may be a child too.
__global__ void __launch_bounds__(256) fork_stage_kernel(Pages p, const int* parents, int n, int* ws) {
    const int i = blockIdx.x, len = ws[kHeaderWords + n + i];
    if (len < 0) return;
    const int full = len / p.page_tokens;
    const int* entry = p.table + static_cast<size_t>(parents[i]) * p.row_pages;
    int* stage = ws + kHeaderWords + 2 * n + static_cast<size_t>(i) * p.row_pages;
    for (int j = threadIdx.x; j < full; j += 256) {
        const int page = entry[j];
        stage[j] = page;
        if (page >= 0 && page < p.n_pages) atomicAdd(&p.refs[page], 1);
    }
}

__global__ void __launch_bounds__(256) fork_rows_kernel(Pages p, const int* children, int n, const int* ws) {
    const int i = blockIdx.x, len = ws[kHeaderWords + n + i];
    if (len < 0) return;
    const int full = len / p.page_tokens, fresh = ws[kHeaderWords + i], child = children[i];
    int* entry = p.table + static_cast<size_t>(child) * p.row_pages;
    const int* stage = ws + kHeaderWords + 2 * n + static_cast<size_t>(i) * p.row_pages;
    for (int j = threadIdx.x; j < p.row_pages; j += 256) {
        const int old = entry[j];
        if (old >= 0 && old < p.n_pages) atomicSub(&p.refs[old], 1);
        const int now = j < full ? stage[j] : j == full ? fresh : -1;
        if (now != old) entry[j] = now;
    }
    if (threadIdx.x == 0) p.lens[child] = len;
}

// Workspace of a compaction: header (moves, pages in use), from[n_pages / 2 + 1], to[...], the new id
// of each page that moves.
__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(Pages p, int* status, int* ws) {
    __shared__ int sums[kPlanWarps];
    __shared__ int used_here, holes_here, movers_here;
    const cg::cluster_group cluster = cg::this_cluster();
    int* from = ws + kHeaderWords;
    int* to = from + p.n_pages / 2 + 1;
    int* moved = to + p.n_pages / 2 + 1;
    const auto used = [&](int page) { return p.refs[page] > 0; };
    const int n_live = count_pages(p.n_pages, sums, &used_here, used).total;
    const auto hole = [&](int page) { return page < n_live && !used(page); };
    const auto mover = [&](int page) { return page >= n_live && used(page); };
    const Slice h = count_pages(p.n_pages, sums, &holes_here, hole);
    const Slice m = count_pages(p.n_pages, sums, &movers_here, mover);
    ranked(h.lo, h.hi, h.before, h.total, sums, hole, [&](int page, int rank) { to[rank] = page; });
    ranked(m.lo, m.hi, m.before, m.total, sums, mover, [&](int page, int rank) { from[rank] = page; });
    cluster.sync();  // both lists are whole
    const int step = cluster.num_blocks() * kPlanThreads;
    for (int i = cluster.block_rank() * kPlanThreads + threadIdx.x; i < m.total; i += step) {
        moved[from[i]] = to[i];
        p.refs[to[i]] = p.refs[from[i]];
        p.refs[from[i]] = 0;
    }
    if (cluster.block_rank() == 0 && threadIdx.x == 0) {
        ws[0] = m.total;
        ws[1] = n_live;
        if (status != nullptr) *status = n_live;
    }
}

__global__ void __launch_bounds__(256) compact_copy_kernel(Pages p, const __grid_constant__ Pools pools, const int* ws) {
    const int* from = ws + kHeaderWords;
    const int* to = from + p.n_pages / 2 + 1;
    const uint32_t vecs = pools.slabs * p.page_tokens * pools.row_vecs;
    const uint64_t units = static_cast<uint64_t>(ws[0]) * pools.n;
    for (uint64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const uint32_t i = static_cast<uint32_t>(u / pools.n), pool = static_cast<uint32_t>(u % pools.n);
        const char* src = pools.base[pool] + from[i] * pools.stride;
        char* dst = pools.base[pool] + to[i] * pools.stride;
        copy_vectors(threadIdx.x, vecs, 256, [&](uint32_t v) { return Ends{src + 16ull * v, dst + 16ull * v}; });
    }
}

__global__ void __launch_bounds__(256) compact_table_kernel(Pages p, const int* ws) {
    const int n_live = ws[1];
    if (ws[0] == 0) return;
    const int* moved = ws + kHeaderWords + 2 * (p.n_pages / 2 + 1);
    const size_t n = static_cast<size_t>(p.n_rows) * p.row_pages;
    for (size_t i = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<size_t>(gridDim.x) * 256) {
        const int page = p.table[i];
        if (page >= n_live && page < p.n_pages) p.table[i] = moved[page];
    }
}

// One thread a 16-byte vector: the keys' vectors first, then the values'.
__global__ void __launch_bounds__(256) write_kernel(Pages p, const Write w) {
    const uint32_t token_vecs = w.heads * w.head_vecs;
    const uint64_t each = static_cast<uint64_t>(w.n) * token_vecs;
    for (uint64_t u = blockIdx.x * 256ull + threadIdx.x; u < 2 * each; u += gridDim.x * 256ull) {
        const int which = u >= each;
        const uint64_t at = u - (which ? each : 0);
        const int i = static_cast<int>(at / token_vecs);
        const uint32_t in = static_cast<uint32_t>(at % token_vecs), head = in / w.head_vecs, vec = in % w.head_vecs;
        const int row = w.rows[i], pos = w.pos[i];
        if (row < 0 || row >= p.n_rows || pos < 0 || pos / p.page_tokens >= p.row_pages) continue;
        const int page = p.table[static_cast<size_t>(row) * p.row_pages + pos / p.page_tokens];
        if (page < 0 || page >= p.n_pages) continue;
        const char* src = w.from[which] + i * w.token_stride[which] + head * w.head_stride[which] + 16ull * vec;
        char* dst = w.to[which] + page * w.page_stride + head * w.to_head + (pos % p.page_tokens) * w.to_token + 16ull * vec;
        *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(src);
    }
}

// Ranking the free pages of a small cache takes one CTA; eight share larger ones.
constexpr int kOneCtaPages = 16384;

template <typename... Params, typename... Args>
cudaError_t launch_plan(void (*kernel)(Params...), int n_pages, size_t shared, cudaStream_t s, Args... args) {
    if (shared > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(shared));
        if (e != cudaSuccess) return e;
    }
    cudaLaunchAttribute cluster;
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = n_pages <= kOneCtaPages ? 1 : 8;
    cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(cluster.val.clusterDim.x);
    c.blockDim = dim3(kPlanThreads);
    c.dynamicSmemBytes = shared;
    c.stream = s;
    c.attrs = &cluster;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, kernel, static_cast<Params>(args)...);
}

size_t plan_shared(const Pages& p, int n) { return 4ull * n + 4ull * ((p.n_rows + 31) / 32); }

}  // namespace

cudaError_t launch_reserve(const Pages& p, const int* rows, const int* tokens, int n, int* status, cudaStream_t s) {
    return launch_plan(reserve_kernel, p.n_pages, plan_shared(p, n), s, p, rows, tokens, n, status);
}

cudaError_t launch_free(const Pages& p, const int* rows, int n, cudaStream_t s) {
    free_kernel<<<n, 256, 0, s>>>(p, rows);
    return cudaGetLastError();
}

cudaError_t launch_fork_plan(const Pages& p, const int* parents, const int* children, int n, int* status, int* ws,
                             cudaStream_t s) {
    return launch_plan(fork_plan_kernel, p.n_pages, plan_shared(p, n), s, p, parents, children, n, status, ws);
}

cudaError_t launch_fork_copy(const Pages& p, const Pools& pools, const int* parents, int n, const int* ws,
                             cudaStream_t s) {
    fork_copy_kernel<<<n * pools.n, 256, 0, s>>>(p, pools, parents, n, ws);
    return cudaGetLastError();
}

cudaError_t launch_fork_rows(const Pages& p, const int* parents, const int* children, int n, int* ws, cudaStream_t s) {
    fork_stage_kernel<<<n, 256, 0, s>>>(p, parents, n, ws);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    fork_rows_kernel<<<n, 256, 0, s>>>(p, children, n, ws);
    return cudaGetLastError();
}

cudaError_t launch_compact_plan(const Pages& p, int* status, int* ws, cudaStream_t s) {
    return launch_plan(compact_plan_kernel, p.n_pages, 0, s, p, status, ws);
}

cudaError_t launch_compact_copy(const Pages& p, const Pools& pools, const int* ws, cudaStream_t s) {
    compact_copy_kernel<<<152 * 8, 256, 0, s>>>(p, pools, ws);
    return cudaGetLastError();
}

cudaError_t launch_compact_table(const Pages& p, const int* ws, cudaStream_t s) {
    const uint64_t n = static_cast<uint64_t>(p.n_rows) * p.row_pages;
    const uint64_t blocks = (n + 255) / 256;
    compact_table_kernel<<<static_cast<unsigned>(blocks < 1216 ? blocks : 1216), 256, 0, s>>>(p, ws);
    return cudaGetLastError();
}

cudaError_t launch_write(const Pages& p, const Write& w, cudaStream_t s) {
    const uint64_t n = 2ull * w.n * w.heads * w.head_vecs, blocks = (n + 255) / 256;
    write_kernel<<<static_cast<unsigned>(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(p, w);
    return cudaGetLastError();
}

}  // namespace jb
