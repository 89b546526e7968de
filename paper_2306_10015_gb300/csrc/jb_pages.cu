// jb_pages.cu -- the pages of a cache: reserve, free, fork, compact, write.
//
// Which pages are free is decided on the device: nothing is read back, and the ids are those of
// the definition (the lowest free ones, in the order of the list), whatever the launch. A plan
// kernel ranks the free pages in one cluster of CTAs, each over a slice of the counts; what moves
// data runs after it over the whole GPU, and HBM bounds it. Small caches are bound by launches, which is why
// a plan also writes the tables.
// Measured (GPU time): 24 prompts forked to 8 answers each in 24 layers, 1.1 GB written: 194 us (a prompt's page
// is read from HBM once); 3000 pages of 131 KB freed, moved and reserved: 248 us, 6.5 TB/s; the same with 35
// pages: 15 us; 8191 new tokens of 3 KB keys and values each: 17 us, 5.9 TB/s; 64 new tokens: 2.6 us.
#include <cooperative_groups.h>

#include "jb_answer.h"
#include "jb_launch.cuh"

namespace jb {
namespace {

namespace cg = cooperative_groups;

constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;
constexpr unsigned kAll = 0xFFFFFFFFu;

template <typename V>
__device__ __forceinline__ V warp_inclusive(V v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const V o = __shfl_up_sync(kAll, v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// Exclusive prefix of v over the CTA's threads; `total` is the sum. sums: kPlanWarps words.
template <typename V>
__device__ __forceinline__ V block_exclusive(V v, V* sums, V& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const V in = warp_inclusive(v);
    if (lane == 31) sums[warp] = in;
    __syncthreads();
    const V all = warp_inclusive(lane < kPlanWarps ? sums[lane] : V(0));
    const V before = __shfl_sync(kAll, all, warp == 0 ? 0 : warp - 1);
    total = __shfl_sync(kAll, all, 31);
    __syncthreads();
    return in - v + (warp == 0 ? V(0) : before);
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

// The plan's CTAs, in step.
struct Team {
    cg::cluster_group cluster;
    int ctas, rank;

    __device__ Team() : cluster(cg::this_cluster()), ctas(cluster.num_blocks()), rank(cluster.block_rank()) {}
    __device__ void sync() const {
        if (ctas > 1) cluster.sync();
        else __syncthreads();
    }
    // The sum of v over the CTAs, and over those before this one. word: one of shared memory, not used for
    // anything else.
    __device__ int sum(int v, int* word, int& before) const {
        if (threadIdx.x == 0) *word = v;
        sync();
        int all = 0;
        before = 0;
        for (int c = 0; c < ctas; ++c) {
            const int x = *cluster.map_shared_rank(word, c);
            if (c < rank) before += x;
            all += x;
        }
        return all;
    }
};

// The team's slice of the pages, and the flagged ones before it, in it and in all.
struct Slice {
    int lo, hi, before, here, total;
};

template <typename Flag>
__device__ __forceinline__ int count_pages(int lo, int hi, int* sums, Flag flag) {
    int n = 0;
    for (int i = lo + static_cast<int>(threadIdx.x); i < hi; i += kPlanThreads) n += flag(i) ? 1 : 0;
    return block_sum(n, sums);
}

template <typename Flag>
__device__ __forceinline__ Slice slice_of(const Team& team, int n_pages, int* sums, int* word, Flag flag) {
    const int per = (n_pages + team.ctas - 1) / team.ctas;
    Slice s;
    s.lo = min(team.rank * per, n_pages);
    s.hi = min(s.lo + per, n_pages);
    s.here = count_pages(s.lo, s.hi, sums, flag);
    s.total = team.sum(s.here, word, s.before);
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

// Dynamic shared memory of the plans: base[n], then a bit for each row.
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
    __shared__ long long wide_sums[kPlanWarps];
    __shared__ int free_here;
    int* base = dynamic;
    unsigned* seen = reinterpret_cast<unsigned*>(dynamic + n);
    after_previous();
    let_next_start();
    const Team team;

    // every CTA works the list out for itself
    clear_seen(seen, p.n_rows);
    __syncthreads();
    long long need_all = 0;  // rows of 2^27 pages may be asked for
    bool bad = false;
    for (int first = 0; first < n; first += kPlanThreads) {
        const int i = first + threadIdx.x;
        long long need = 0;
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
        long long total;
        const long long at = need_all + block_exclusive(need, wide_sums, total);
        if (i < n) base[i] = static_cast<int>(min(at, 0x7FFFFFFFll));  // looked at if all are fewer than the pages
        need_all += total;
    }
    bad = __syncthreads_or(bad);
    const Slice s = slice_of(team, p.n_pages, sums, &free_here, [&](int i) { return p.refs[i] == 0; });
    if (bad || need_all > s.total) {
        if (team.rank == 0 && threadIdx.x == 0) *status = bad ? -1 : static_cast<int>(min(need_all - s.total, 0x7FFFFFFFll));
        team.sync();  // until every CTA's memory has been read
        return;
    }
    ranked(s.lo, s.hi, s.before, static_cast<int>(need_all), sums, [&](int page) { return p.refs[page] == 0; },
           [&](int page, int rank) {
               const int i = owner_of(base, n, rank);
               const int row = rows[i];
               const int at = pages_of(row_len(p, row), p.page_tokens) + rank - base[i];
               p.table[static_cast<size_t>(row) * p.row_pages + at] = page;
               p.refs[page] = 1;
           });
    team.sync();  // the lengths are read until here
    if (team.rank == 0) {
        for (int i = threadIdx.x; i < n; i += kPlanThreads) p.lens[rows[i]] = row_len(p, rows[i]) + tokens[i];
        if (threadIdx.x == 0) *status = 0;
    }
}

// One CTA a row. Entries are taken out one by one, so a row listed twice is released once.
__global__ void __launch_bounds__(256) free_kernel(Pages p, const int* rows) {
    after_previous();
    let_next_start();
    const int row = rows[blockIdx.x];
    if (row < 0 || row >= p.n_rows) return;
    int* entry = p.table + static_cast<size_t>(row) * p.row_pages;
    const int pages = pages_of(row_len(p, row), p.page_tokens);
    __syncthreads();  // the length is read until here
    for (int j = threadIdx.x; j < pages; j += 256) {
        const int page = atomicExch(&entry[j], -1);
        if (page >= 0 && page < p.n_pages) atomicSub(&p.refs[page], 1);
    }
    if (threadIdx.x == 0) p.lens[row] = 0;
}

// Workspace of a fork: header, from[n] and to[n] (the pages of the last tokens, -1: nothing to copy), len[n]
// (tokens of the parent, -1: nothing to do), stage[n][row_pages] (the parents' entries).
__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(Pages p, const int* parents, const int* children,
                                                                 int n, int* status, int* ws) {
    extern __shared__ int dynamic[];
    __shared__ int sums[kPlanWarps];
    __shared__ int free_here;
    int* base = dynamic;
    unsigned* seen = reinterpret_cast<unsigned*>(dynamic + n);
    after_previous();
    let_next_start();
    const Team team;
    int* from = ws + kHeaderWords;
    int* to = from + n;
    int* len = to + n;
    int* stage = len + n;

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
    const Slice s = slice_of(team, p.n_pages, sums, &free_here, [&](int i) { return p.refs[i] == 0; });
    const bool go = !bad && need_all <= s.total;
    if (team.rank == 0) {
        for (int i = threadIdx.x; i < n; i += kPlanThreads) {
            const int a = parents[i];
            const bool moves = go && a != children[i];
            const int tokens = moves ? row_len(p, a) : -1;
            len[i] = tokens;
            from[i] = moves && tokens % p.page_tokens != 0 ? p.table[static_cast<size_t>(a) * p.row_pages + tokens / p.page_tokens] : -1;
        }
        if (threadIdx.x == 0) *status = bad ? -1 : max(need_all - s.total, 0);
    }
    if (!go) {
        team.sync();  // until every CTA's memory has been read
        return;
    }
    ranked(s.lo, s.hi, s.before, need_all, sums, [&](int page) { return p.refs[page] == 0; },
           [&](int page, int rank) {
               to[owner_of(base, n, rank)] = page;
               p.refs[page] = 1;
           });
    team.sync();
    // The parents' entries are set aside before any row is written: a parent may be a child too. A warp takes a
    // pair at a time.
    const int lane = threadIdx.x & 31, warp = team.rank * kPlanWarps + static_cast<int>(threadIdx.x >> 5), warps = team.ctas * kPlanWarps;
    for (int i = warp; i < n; i += warps) {
        const int full = len[i] < 0 ? 0 : len[i] / p.page_tokens;
        const int* entry = p.table + static_cast<size_t>(parents[i]) * p.row_pages;
        for (int j = lane; j < full; j += 32) {
            const int page = entry[j];
            stage[static_cast<size_t>(i) * p.row_pages + j] = page;
            if (page >= 0 && page < p.n_pages) atomicAdd(&p.refs[page], 1);
        }
    }
    team.sync();
    for (int i = warp; i < n; i += warps) {
        const int tokens = len[i];
        if (tokens < 0) continue;
        const int child = children[i], full = tokens / p.page_tokens, pages = pages_of(tokens, p.page_tokens);
        const int had = pages_of(row_len(p, child), p.page_tokens);
        int* entry = p.table + static_cast<size_t>(child) * p.row_pages;
        __syncwarp();  // the length is read until here
        for (int j = lane; j < max(pages, had); j += 32) {
            const int old = j < had ? entry[j] : -1;
            if (old >= 0 && old < p.n_pages) atomicSub(&p.refs[old], 1);
            entry[j] = j < full ? stage[static_cast<size_t>(i) * p.row_pages + j] : j < pages ? to[i] : -1;
        }
        if (lane == 0) p.lens[child] = tokens;
    }
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

// `splits` CTAs for a pair's last page in one pool: the valid tokens of each slab.
__global__ void __launch_bounds__(256) fork_copy_kernel(Pages p, const __grid_constant__ Pools pools, int n, int splits,
                                                        const int* ws) {
    after_previous();
    let_next_start();
    const int split = blockIdx.x % splits, unit = blockIdx.x / splits, i = unit / pools.n, pool = unit % pools.n;
    const int from = ws[kHeaderWords + i], to = ws[kHeaderWords + n + i], len = ws[kHeaderWords + 2 * n + i];
    if (from < 0 || from >= p.n_pages) return;
    const uint32_t run = (len % p.page_tokens) * pools.row_vecs, whole = p.page_tokens * pools.row_vecs;
    const char* src = pools.base[pool] + from * pools.stride;
    char* dst = pools.base[pool] + to * pools.stride;
    copy_vectors(split * 256 + threadIdx.x, run * pools.slabs, splits * 256, [&](uint32_t v) {
        const uint64_t at = 16ull * (v / run * whole + v % run);
        return Ends{src + at, dst + at};
    });
}

// Workspace of a compaction: header (moves, pages in use), from[n_pages / 2 + 1], to[...], the new id
// of each page that moves.
__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(Pages p, int* status, int* ws) {
    __shared__ int sums[kPlanWarps];
    __shared__ int used_here, low_here;
    after_previous();
    let_next_start();
    const Team team;
    int* from = ws + kHeaderWords;
    int* to = from + p.n_pages / 2 + 1;
    int* moved = to + p.n_pages / 2 + 1;
    const auto used = [&](int page) { return p.refs[page] > 0; };
    const Slice s = slice_of(team, p.n_pages, sums, &used_here, used);
    const int n_live = s.total;
    // pages in use below n_live: of the slices on both sides they are known
    const int low = s.hi <= n_live ? s.here : s.lo >= n_live ? 0 : count_pages(s.lo, n_live, sums, used);
    int before;
    const int low_all = team.sum(low, &low_here, before);
    const int moves = n_live - low_all;
    // the first page's rank among the holes, and of the first page from n_live on among the movers
    ranked(s.lo, min(s.hi, n_live), s.lo - s.before, moves, sums, [&](int page) { return !used(page); },
           [&](int page, int rank) { to[rank] = page; });
    const int start = max(s.lo, n_live);
    ranked(start, s.hi, s.before + low - low_all, moves, sums, used, [&](int page, int rank) { from[rank] = page; });
    team.sync();  // both lists are whole
    const int step = team.ctas * kPlanThreads;
    for (int i = team.rank * kPlanThreads + static_cast<int>(threadIdx.x); i < moves; i += step) {
        moved[from[i]] = to[i];
        p.refs[to[i]] = p.refs[from[i]];
        p.refs[from[i]] = 0;
    }
    if (team.rank == 0 && threadIdx.x == 0) {
        ws[0] = moves;
        ws[1] = n_live;
        if (status != nullptr) *status = n_live;
    }
}

// The first table_ctas CTAs put the new ids into the table, the others move pages, 16 KB at a time.
constexpr int kChunk = 4 * 256;  // 16-byte vectors
constexpr int kWaves = 128;      // of CTAs to an SM
__global__ void __launch_bounds__(256) compact_move_kernel(Pages p, const __grid_constant__ Pools pools, int table_ctas, const int* ws) {
    after_previous();
    let_next_start();
    const int moves = ws[0], n_live = ws[1];
    if (moves == 0) return;
    const int* from = ws + kHeaderWords;
    const int* to = from + p.n_pages / 2 + 1;
    const int* moved = to + p.n_pages / 2 + 1;
    if (static_cast<int>(blockIdx.x) < table_ctas) {
        const size_t n = static_cast<size_t>(p.n_rows) * p.row_pages, step = table_ctas * 256ull;
        for (size_t i = blockIdx.x * 256ull + threadIdx.x; i < n; i += step) {
            const int page = p.table[i];
            if (page >= n_live && page < p.n_pages) p.table[i] = moved[page];
        }
        return;
    }
    const uint32_t vecs = pools.slabs * p.page_tokens * pools.row_vecs, chunks = (vecs + kChunk - 1) / kChunk;
    const uint64_t units = static_cast<uint64_t>(moves) * pools.n * chunks;
    for (uint64_t u = blockIdx.x - table_ctas; u < units; u += gridDim.x - table_ctas) {
        const uint64_t page = u / chunks;
        const uint32_t first = static_cast<uint32_t>(u - page * chunks) * kChunk + threadIdx.x;
        const uint32_t i = static_cast<uint32_t>(page / pools.n), pool = static_cast<uint32_t>(page - static_cast<uint64_t>(i) * pools.n);
        const char* src = pools.base[pool] + from[i] * pools.stride;
        char* dst = pools.base[pool] + to[i] * pools.stride;
        uint4 x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (first + k * 256 < vecs) x[k] = __ldcs(reinterpret_cast<const uint4*>(src) + first + k * 256);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (first + k * 256 < vecs) __stcs(reinterpret_cast<uint4*>(dst) + first + k * 256, x[k]);
    }
}

// A warp takes kVecs vectors a lane of a token's keys (blockIdx.y even) or values.
constexpr int kVecs = 4;
__global__ void __launch_bounds__(256) write_kernel(Pages p, const __grid_constant__ Write w) {
    after_previous();
    let_next_start();
    const int i = blockIdx.x * 8 + static_cast<int>(threadIdx.x >> 5), which = blockIdx.y & 1;
    if (i >= w.n) return;
    const int row = w.rows[i], pos = w.pos[i];
    if (row < 0 || row >= p.n_rows || pos < 0 || pos / p.page_tokens >= p.row_pages) return;
    const int page = p.table[static_cast<size_t>(row) * p.row_pages + pos / p.page_tokens];
    if (page < 0 || page >= p.n_pages) return;
    const char* src = w.from[which] + i * w.token_stride[which];
    char* dst = w.to[which] + page * w.page_stride + pos % p.page_tokens * w.to_token;
    const uint32_t first = (blockIdx.y >> 1) * 32 * kVecs + (threadIdx.x & 31), vecs = w.heads * w.head_vecs;
    uint4 x[kVecs];
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
        const uint32_t v = first + 32 * k, head = static_cast<uint32_t>(v * w.magic >> 32);
        if (v < vecs) x[k] = *reinterpret_cast<const uint4*>(src + head * w.head_stride[which] + 16 * (v - head * w.head_vecs));
    }
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
        const uint32_t v = first + 32 * k, head = static_cast<uint32_t>(v * w.magic >> 32);
        if (v < vecs) *reinterpret_cast<uint4*>(dst + head * w.to_head + 16 * (v - head * w.head_vecs)) = x[k];
    }
}

// Dynamic shared memory of a plan, and the most that one takes.
constexpr size_t plan_shared(int n_rows, int n) { return 4ull * n + 4ull * ((n_rows + 31) / 32); }
constexpr int kMostShared = static_cast<int>(plan_shared(kMaxRows, kMaxListed));

// A small plan takes one CTA; eight share larger ones. work: pages to rank and entries to write.
constexpr uint64_t kOneCta = 16384;

template <typename... Params, typename... Args>
cudaError_t launch_plan(void (*kernel)(Params...), uint64_t work, size_t shared, cudaStream_t s, const Args&... args) {
    if (shared > 48 * 1024) {  // the limit is the kernel's, not the call's: every host thread sets the same one
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
        if (e != cudaSuccess) return e;
    }
    const unsigned ctas = work <= kOneCta ? 1 : 8;
    return launch(kernel, ctas, kPlanThreads, shared, ctas, s, args...);
}

}  // namespace

cudaError_t launch_reserve(const Pages& p, const int* rows, const int* tokens, int n, int* status, cudaStream_t s) {
    return launch_plan(reserve_kernel, p.n_pages, plan_shared(p.n_rows, n), s, p, rows, tokens, n, status);
}

cudaError_t launch_free(const Pages& p, const int* rows, int n, cudaStream_t s) {
    return launch(free_kernel, n, 256, 0, 0, s, p, rows);
}

cudaError_t launch_fork_plan(const Pages& p, const int* parents, const int* children, int n, int* status, int* ws,
                             cudaStream_t s) {
    return launch_plan(fork_plan_kernel, p.n_pages + static_cast<uint64_t>(n) * p.row_pages, plan_shared(p.n_rows, n), s, p, parents,
                       children, n, status, ws);
}

cudaError_t launch_fork_copy(const Pages& p, const Pools& pools, int n, const int* ws, cudaStream_t s) {
    // few pages are shared out further, so that every SM has some
    const int units = n * static_cast<int>(pools.n), splits = units >= 2048 ? 1 : units >= 512 ? 4 : 8;
    return launch(fork_copy_kernel, static_cast<unsigned>(units) * splits, 256, 0, 0, s, p, pools, n, splits, ws);
}

cudaError_t launch_compact_plan(const Pages& p, int* status, int* ws, cudaStream_t s) {
    return launch_plan(compact_plan_kernel, p.n_pages, 0, s, p, status, ws);
}

cudaError_t launch_compact_move(const Pages& p, const Pools& pools, bool table, const int* ws, cudaStream_t s) {
    const uint64_t blocks = (static_cast<uint64_t>(p.n_rows) * p.row_pages + 255) / 256;
    const int table_ctas = table ? static_cast<int>(blocks < 152 ? blocks : 152) : 0;
    // Waves of short CTAs even out what memory serves unevenly: 152 x 8 CTAs that stay 273 us for 3000 pages of
    // 131 KB, 152 x 128 248 us. No more than there can be chunks to move.
    const uint64_t chunks = (static_cast<uint64_t>(pools.slabs) * p.page_tokens * pools.row_vecs + kChunk - 1) / kChunk;
    const uint64_t most = (p.n_pages / 2 + 1ull) * pools.n * chunks, room = 152 * kWaves;
    return launch(compact_move_kernel, static_cast<unsigned>(most < room ? most : room) + table_ctas, 256, 0, 0, s, p, pools, table_ctas, ws);
}

cudaError_t launch_write(const Pages& p, const Write& w, cudaStream_t s) {
    const unsigned vecs = w.heads * w.head_vecs, parts = (vecs + 32 * kVecs - 1) / (32 * kVecs);
    cudaLaunchConfig_t c = {};
    cudaLaunchAttribute a;
    a.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a.val.programmaticStreamSerializationAllowed = 1;
    c.gridDim = dim3((w.n + 7u) / 8u, 2 * parts);
    c.blockDim = dim3(256);
    c.stream = s;
    c.attrs = &a;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, write_kernel, p, w);
}

}  // namespace jb
