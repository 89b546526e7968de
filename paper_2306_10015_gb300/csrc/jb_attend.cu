// jb_attend.cu -- attention of single queries over the pages of a cache.
//
// A query reads each key and value of its row once and does 4 g operations per element with g
// query heads to a key head, so the bytes bound it: the kernels stream pages from HBM and keep all
// state in registers. Work is cut evenly whatever the rows' lengths: the 16-token groups of all
// (query, key head) pairs are one line, every warp takes an equal stretch of it and works alone. A pair
// that crosses a boundary is joined from partial (maximum, sum, weighted values) by the warp that
// finishes last, 8 or 16 parts at a time.
//
// Softmax is kept with a running maximum, so that one pass is enough:
//   m' = max(m, max_t x_t), s' = s e^(m - m') + sum e^(x_t - m'), o' likewise.
//
// Why a warp and not a CTA: warps that add up their parts of a pair at a barrier cost 2.7 us a pair, which is
// all that 40 tokens take (256 rows of 20 to 60 tokens, 32 heads of 128: 74 us, now 43). Why equal pieces
// decided at the start: keeping a share back for the warps that are done first was slower everywhere (by 2 to
// 30 %), and so were twice as many CTAs as run at once (1 to 20 %): a warp that is done leaves its bandwidth to
// the others, and every further piece costs a start and a join.
//
// What it is not made for: the tokens of a prompt, each of which streams its row's keys and values for itself (one
// of 2048 bf16 tokens, 32 heads of 128: 5.1 ms), and groups of more than 8 (fp32) or 16 (bf16) query heads, which
// read them once for each block of so many heads (16 fp32 heads of 256: 2.2 times the floor).
#include <atomic>

#include <cuda_bf16.h>

#include "jb_answer.h"
#include "jb_launch.cuh"

namespace jb {
namespace {

constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kGroup = 16;         // tokens a warp takes at a time; pages hold a multiple of it
constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kMaxWorkers = 2048;  // warps of the persistent grid; the workspace has two slots for each
constexpr int kLevels = 4;         // of joining 8 or 16 parts of a pair at a time: 8^4 >= kMaxWorkers
constexpr int kLeast = 4;          // groups of a stretch, where that leaves one to each CTA
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.0e38f;

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

struct Params {
    Pages pages;
    Attend a;
    int blocks;        // blocks of query heads to a key head
    int page_groups;   // groups in a page
    float cap_in, cap_out;  // softcap: scale / cap, cap / ln 2
};

// Partial results of a stretch: o[heads][D], m[heads], s[heads], for the query heads that are worked on
// together.
__host__ __device__ constexpr int slot_floats(int heads, int d) { return heads * (d + 2); }

// Groups that query i reads: [first, first + groups), of tokens lo to pos.
struct Span {
    int row, lo, pos, first, groups;
};

__device__ __forceinline__ Span span_of(const Params& p, int i) {
    Span s;
    s.row = p.a.rows[i];
    s.pos = p.a.pos[i];
    s.lo = s.first = s.groups = 0;
    if (s.row < 0 || s.row >= p.pages.n_rows || s.pos < 0 || s.pos >= p.pages.row_pages * p.pages.page_tokens) {
        s.pos = -1;
        return s;
    }
    if (p.a.window > 0) s.lo = max(0, s.pos - p.a.window + 1);
    s.first = s.lo / kGroup;
    s.groups = s.pos / kGroup - s.first + 1;
    return s;
}

// Groups [from, to) of a (query, key head, block of query heads).
struct Stretch {
    int query, head, block, from, to;
    long long begin;  // where the pair starts on the line
    Span span;
};

// a / b; 64-bit division only where it is needed.
__device__ __forceinline__ long long quotient(long long a, long long b) {
    return ((a | b) >> 32) == 0 ? static_cast<long long>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b)) : a / b;
}

static_assert(kMaxListed <= kThreads * kThreads, "a thread's run of queries");

// The line of groups, and which warp has which of them: `each`, and the first `extra` warps one more.
struct Line {
    long long total, each;
    int workers, extra;

    __device__ long long bound(int w) const { return each * w + min(w, extra); }
    __device__ int owner(long long x) const {
        const long long longer = (each + 1) * extra;
        return x < longer ? static_cast<int>(quotient(x, each + 1)) : extra + static_cast<int>(quotient(x - longer, each));
    }
};

// Deals the line out.
struct Dealer {
    long long next, end;
    Line line;
    int worker;
    int query;
    long long at;         // groups of the query before `next`
    Span span;

    // The CTA together. sums: kThreads + 1 words of shared memory.
    __device__ void start(const Params& p, long long* sums) {
        const int n = p.a.n, pairs = p.a.heads * p.blocks, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        const int per = (n + kThreads - 1) / kThreads;
        // groups of each thread's run of queries
        long long mine = 0;
        for (int k = 0; k < per; ++k) {
            const int i = static_cast<int>(threadIdx.x) * per + k;
            if (i < n) mine += span_of(p, i).groups;
        }
        scan(mine, sums);
        line.total = sums[kThreads] * pairs;
        // neighbours on the line are on different SMs, so that few stretches use all of them
        worker = warp * gridDim.x + blockIdx.x;
        // few groups: one to a warp on every SM, then kLeast before the next warps get some (one row of 2048
        // tokens, 32 heads: 16.9 us with one group a warp, 13.4 with four)
        line.workers = static_cast<int>(min(static_cast<long long>(gridDim.x) * kWarps,
                                            max(min(max(1ll, line.total), static_cast<long long>(gridDim.x)), line.total / kLeast)));
        next = end = 0;
        if (worker >= line.workers || line.total == 0) return;
        line.each = quotient(line.total, line.workers);
        line.extra = static_cast<int>(line.total - line.each * line.workers);
        next = line.bound(worker);
        end = line.bound(worker + 1);
        // the run with the warp's first group: groups before a query are multiples of `pairs`
        const long long goal = quotient(next, pairs);
        int run = 0;
#pragma unroll
        for (int k = 0; k < kThreads; k += 32) {
            const unsigned here = __ballot_sync(kAll, sums[k + lane] <= goal && goal < sums[k + lane + 1]);
            if (here != 0) run = k + __ffs(here) - 1;
        }
        long long base = sums[run];
        query = run * per;
        for (int k = 0; per > 1 && k < per; k += 32) {  // and the query within the run
            const int i = query + lane;
            const int g = k + lane < per && i < n ? span_of(p, i).groups : 0;
            long long in = g;  // a query may have 2^27
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const long long o = __shfl_up_sync(kAll, in, d);
                if (lane >= d) in += o;
            }
            const unsigned past = __ballot_sync(kAll, base + in > goal);
            if (past != 0) {
                const int l = __ffs(past) - 1;
                base += __shfl_sync(kAll, in - g, l);
                query += l;
                break;
            }
            base += __shfl_sync(kAll, in, 31);
            query += 32;
        }
        span = span_of(p, query);
        at = next - base * pairs;
    }

    // sums[i] = sum of v over threads before i, sums[kThreads] = of all.
    __device__ static void scan(long long v, long long* sums) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        __shared__ long long warp_sums[kWarps];
        long long in = v;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const long long o = __shfl_up_sync(kAll, in, d);
            if (lane >= d) in += o;
        }
        if (lane == 31) warp_sums[warp] = in;
        __syncthreads();
        for (int w = 0; w < warp; ++w) in += warp_sums[w];
        sums[threadIdx.x + 1] = in;
        if (threadIdx.x == 0) sums[0] = 0;
        __syncthreads();
    }

    __device__ bool take(const Params& p, Stretch& s) {
        if (next >= end) return false;
        const long long pairs = p.a.heads * p.blocks;
        while (at >= span.groups * pairs) {
            at -= span.groups * pairs;
            ++query;
            span = span_of(p, query);
        }
        s.query = query;
        s.span = span;
        const int pair = static_cast<int>(quotient(at, span.groups));
        s.head = pair / p.blocks;
        s.block = pair % p.blocks;
        s.from = static_cast<int>(at - static_cast<long long>(pair) * span.groups);
        s.to = static_cast<int>(min(static_cast<long long>(span.groups), s.from + (end - next)));
        s.begin = next - s.from;
        next += s.to - s.from;
        at += s.to - s.from;
        return true;
    }
};

template <typename T>
__device__ __forceinline__ void store_out(T* to, float v);
template <>
__device__ __forceinline__ void store_out<float>(float* to, float v) { *to = v; }
template <>
__device__ __forceinline__ void store_out<__nv_bfloat16>(__nv_bfloat16* to, float v) { *to = __float2bfloat16_rn(v); }

// The workspace: a counter for each slot and level, zero between calls, then the slots. Part 0 of a pair
// is in its worker's slot 1, the others in their workers' slots 0, so that a worker's end of one pair
// and start of the next do not meet.
__host__ __device__ constexpr size_t counters() { return static_cast<size_t>(kLevels) * 2 * kMaxWorkers; }
static_assert(counters() * 4 == 65536, "what jb.h says of the workspace");
__device__ __forceinline__ int slot_index(int first, int part) { return 2 * (first + part) + (part == 0 ? 1 : 0); }
__device__ __forceinline__ float* slot_of(const Params& p, int heads, int d, int index) {
    return p.a.ws + counters() + static_cast<size_t>(slot_floats(heads, d)) * index;
}

// Zeros for the queries that see nothing.
template <typename T>
__device__ __forceinline__ void write_zeros(const Params& p) {
    const int d = p.a.head_dim, heads = p.a.heads * p.a.group;
    for (int i = blockIdx.x; i < p.a.n; i += gridDim.x) {
        if (span_of(p, i).groups > 0) continue;
        for (int u = threadIdx.x; u < heads * d; u += kThreads)
            store_out(reinterpret_cast<T*>(p.a.out) + i * p.a.out_row + u / d * p.a.out_head + u % d, 0.0f);
    }
}

// A stretch's part is in its slot. The warp that hands in the last of kRadix parts joins them, and so on
// up to the whole pair, which it stores. The order of the sums is that of the line, whoever joins. A
// join is a chain of waits on L2, so its loads are issued together, kDeep float4 of each part at a time.
template <typename T, int D, int kH, int kRadix, int kDeep>
__device__ __forceinline__ void join_up(const Params& p, int first, int index, int count, int query, int head, int block) {
    const int lane = threadIdx.x & 31;
    const int heads_here = min(kH, p.a.group - block * kH), d = p.a.head_dim;
    int* counter = reinterpret_cast<int*>(p.a.ws);
    for (int reach = 1;; reach *= kRadix, counter += 2 * kMaxWorkers) {  // a part stands for `reach` stretches
        const int team = index / kRadix, members = min(kRadix, count - team * kRadix);
        if (members > 1) {
            const int base = slot_index(first, team * kRadix * reach);
            __syncwarp();
            int before = 0;
            if (lane == 0) {
                __threadfence();
                before = atomicAdd(&counter[base], 1);
                __threadfence();
            }
            before = __shfl_sync(kAll, before, 0);
            __syncwarp();  // every lane reads what lane 0 may read now
            if (before + 1 < members) return;
            if (lane == 0) counter[base] = 0;
            const bool last = count <= kRadix;
            const auto slot = [&](int i) { return slot_of(p, kH, D, slot_index(first, (team * kRadix + i) * reach)); };
            // lane h: head h's maxima and sums
            float f[kRadix], li[kRadix], m = kLowest, l = 0.0f, inverse = 0.0f;
#pragma unroll
            for (int i = 0; i < kRadix; ++i) {
                const bool real = i < members && lane < heads_here;
                f[i] = real ? __ldcg(slot(i) + kH * D + lane) : kLowest;
                li[i] = real ? __ldcg(slot(i) + kH * D + kH + lane) : 0.0f;
            }
            for (int from = 0; from < heads_here * D; from += 128 * kDeep) {
                float4 x[kDeep][kRadix];
#pragma unroll
                for (int j = 0; j < kDeep; ++j) {
                    const int e = from + 128 * j + 4 * lane;
#pragma unroll
                    for (int i = 0; i < kRadix; ++i)
                        x[j][i] = i < members && e < heads_here * D ? __ldcg(reinterpret_cast<const float4*>(slot(i) + e))
                                                                    : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                }
                if (from == 0) {
#pragma unroll
                    for (int i = 0; i < kRadix; ++i) m = fmaxf(m, f[i]);
#pragma unroll
                    for (int i = 0; i < kRadix; ++i) {
                        f[i] = exp2_approx(f[i] - m);
                        l = fmaf(f[i], li[i], l);
                    }
                    inverse = l > 0.0f ? 1.0f / l : 0.0f;
                }
#pragma unroll
                for (int j = 0; j < kDeep; ++j) {
                    const int e = from + 128 * j + 4 * lane, h = min(e / D, heads_here - 1);
                    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                    for (int i = 0; i < kRadix; ++i) {
                        const float k = __shfl_sync(kAll, f[i], h);
                        o = make_float4(fmaf(k, x[j][i].x, o.x), fmaf(k, x[j][i].y, o.y), fmaf(k, x[j][i].z, o.z), fmaf(k, x[j][i].w, o.w));
                    }
                    const float scale = __shfl_sync(kAll, inverse, h);
                    if (e >= heads_here * D) continue;
                    if (!last) {
                        *reinterpret_cast<float4*>(slot(0) + e) = o;
                    } else if (e % D < d) {
                        T* out = reinterpret_cast<T*>(p.a.out) + query * p.a.out_row + (head * p.a.group + block * kH + h) * p.a.out_head + e % D;
                        store_out(out, o.x * scale);
                        store_out(out + 1, o.y * scale);
                        store_out(out + 2, o.z * scale);
                        store_out(out + 3, o.w * scale);
                    }
                }
            }
            if (last) return;
            if (lane < heads_here) {
                slot(0)[kH * D + lane] = m;
                slot(0)[kH * D + kH + lane] = l;
            }
        }
        index = team;
        count = (count + kRadix - 1) / kRadix;
    }
}

// A warp has at most two pairs that are cut: its first and its last. They are noted here, and handed in
// when the warp has nothing else to do (and the registers of its products are free).
struct Noted {
    int query, head, block, first, count;
};

__device__ __forceinline__ void note(Noted& to, const Dealer& deal, const Stretch& s) {
    const int first = deal.line.owner(s.begin), last = deal.line.owner(s.begin + s.span.groups - 1);
    if ((threadIdx.x & 31) == 0) to = {s.query, s.head, s.block, first, last - first + 1};
}

template <typename T, int D, int kH>
__device__ __forceinline__ void hand_in(const Params& p, const Noted* noted, int n, int worker) {
    __syncwarp();
    for (int i = 0; i < n; ++i) {
        const Noted c = noted[i];
        // parts of one float4 a lane are joined 16 at a time, longer ones 8 at a time
        if (min(kH, p.a.group - c.block * kH) * D <= 128)
            join_up<T, D, kH, 16, 1>(p, c.first, worker - c.first, c.count, c.query, c.head, c.block);
        else
            join_up<T, D, kH, 8, D == 64 ? 2 : 4>(p, c.first, worker - c.first, c.count, c.query, c.head, c.block);
    }
}

// 16 bytes from global to shared memory, asynchronously; zeros if not `real`.
__device__ __forceinline__ void copy_async(uint32_t to, const void* from, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void wait_copies() {
    asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}
__device__ __forceinline__ void prefetch(const void* p) { asm volatile("prefetch.global.L1 [%0];" ::"l"(p)); }

// The stretches whose copies are under way, in the order of the line; a ring for each warp.
constexpr int kQueue = 4;

// A warp copies its groups, whole rows at a time, kStages ahead into a ring of its own, across the ends of
// stretches, so that it waits neither for other warps nor between pairs. 16-byte pieces of row t are stored at
// column (piece ^ t % 8): reads of one column of 8 rows, and of one row, are free of bank conflicts.
template <typename T, int D>
struct Feed {
    static constexpr int kStages = sizeof(T) == 4 && D >= 128 ? 1 : 2;    // groups that a warp copies ahead
    static constexpr int kPieces = D * static_cast<int>(sizeof(T)) / 16;  // of a row
    static constexpr int kLanes = kPieces < 32 ? kPieces : 32;            // of them that copy one row
    static constexpr int kRows = 32 / kLanes;                             // rows that the warp copies at a time
    static constexpr uint32_t kRowBytes = D * sizeof(T);
    static constexpr uint32_t kGroupBytes = kGroup * kRowBytes;           // keys, and as much for the values
    static constexpr uint32_t kStageBytes = 2 * kGroupBytes;
    static constexpr int kRing = kStages * kStageBytes;
    static constexpr int kElems = 16 / sizeof(T);
    static_assert(kStages + 1 < kQueue);

    uint32_t ring;       // shared address of the warp's ring
    Stretch* queue;
    int queued;          // stretches put there so far
    const int* table;
    uint64_t at;         // the key head's, this lane's row and piece, in elements
    int group, stop, page, lo, pos;
    uint32_t missing;    // stages that hold a group whose page is missing

    __device__ void ahead(const Params& p) { page = group < stop ? table[group / p.page_groups] : -1; }

    // Goes on to the dealer's next stretch, whose first page it looks up.
    __device__ void next(const Params& p, Dealer& deal, int heads_together) {
        Stretch s;
        if (!deal.take(p, s)) {
            group = stop = 0;
            return;
        }
        const int lane = threadIdx.x & 31;
        if (lane == 0) queue[queued % kQueue] = s;
        ++queued;
        table = p.pages.table + static_cast<size_t>(s.span.row) * p.pages.row_pages;
        at = s.head * p.a.head_stride + lane / kLanes * p.a.token_stride + kElems * (lane % kLanes);
        group = s.span.first + s.from;
        stop = s.span.first + s.to;
        lo = s.span.lo;
        pos = s.span.pos;
        ahead(p);
        // the queries that will be wanted: 128 bytes a lane
        constexpr int kLines = static_cast<int>(D * sizeof(T) / 128);
        const int h = min(s.block * heads_together + lane / kLines, p.a.group - 1), e = lane % kLines * static_cast<int>(128 / sizeof(T));
        if (lane / kLines < heads_together && e < p.a.head_dim)
            prefetch(reinterpret_cast<const T*>(p.a.q) + s.query * p.a.q_row + (s.head * p.a.group + h) * p.a.q_head + e);
    }

    // kApart: keys and values are asked and waited for one after the other.
    template <bool kApart>
    __device__ void start(const Params& p, Dealer& deal, int heads_together) {
        queued = 0;
        missing = 0;
        next(p, deal, heads_together);
#pragma unroll
        for (int i = 0; i < kStages; ++i) {
            if constexpr (kApart) {
                ask_keys(p, i);
                ask_values(p, i, deal, heads_together);
            } else {
                ask(p, i, deal, heads_together);
            }
        }
    }

    // Copies the group's keys, values or both; the values alone after the keys.
    template <bool kKeys, bool kValues>
    __device__ __forceinline__ void copy(const Params& p, int stage) {
        bool real = !(missing >> stage & 1u);
        if constexpr (kKeys) {
            real = page >= 0 && page < p.pages.n_pages;
            missing = (missing & ~(1u << stage)) | (real ? 0u : 1u << stage);
        }
        if (!real) return;
        const int row = (threadIdx.x & 31) / kLanes, piece = threadIdx.x % kLanes;
        const uint64_t from = at + page * p.a.page_stride + group % p.page_groups * kGroup * p.a.token_stride;
        const T* kp = reinterpret_cast<const T*>(p.a.k) + from;
        const T* vp = reinterpret_cast<const T*>(p.a.v) + from;
        const uint32_t to = ring + stage * kStageBytes + row * kRowBytes;
        const int token = group * kGroup + row;
#pragma unroll
        for (int j = 0; j < kGroup; j += kRows)
#pragma unroll
            for (int i = 0; i < kPieces; i += kLanes) {
                // what is not seen is not read: a value must not reach the sum, whatever it holds
                const bool seen = kElems * (piece + i) < p.a.head_dim && token + j >= lo && token + j <= pos;
                const uint32_t place = to + j * kRowBytes + (((piece + i) ^ ((row + j) & 7)) << 4);
                if constexpr (kKeys) copy_async(place, kp + j * p.a.token_stride + kElems * i, seen);
                if constexpr (kValues) copy_async(place + kGroupBytes, vp + j * p.a.token_stride + kElems * i, seen);
            }
    }
    __device__ __forceinline__ void advance(const Params& p, Dealer& deal, int heads_together) {
        if (++group < stop) ahead(p);
        else next(p, deal, heads_together);
    }
    __device__ __forceinline__ void ask_keys(const Params& p, int stage) {
        if (group < stop) copy<true, false>(p, stage);
        commit_copies();
    }
    // Of the group whose keys were asked for last; goes on to the next one.
    __device__ __forceinline__ void ask_values(const Params& p, int stage, Dealer& deal, int heads_together) {
        if (group < stop) {
            copy<false, true>(p, stage);
            advance(p, deal, heads_together);
        }
        commit_copies();
    }
    __device__ __forceinline__ void ask(const Params& p, int stage, Dealer& deal, int heads_together) {
        if (group < stop) {
            copy<true, true>(p, stage);
            advance(p, deal, heads_together);
        }
        commit_copies();
    }

    // Waits for the keys in `stage`; false if the group's page is missing.
    __device__ __forceinline__ bool keys_ready(int stage) {
        wait_copies<2 * kStages - 1>();
        __syncwarp();
        return !(missing >> stage & 1u);
    }
    // Waits for the values, the keys of a later group having been asked for.
    __device__ __forceinline__ void values_ready() {
        wait_copies<2 * kStages - 1>();
        __syncwarp();
    }

    // Waits for the group in `stage`; false if its page is missing.
    __device__ __forceinline__ bool ready(int stage) {
        wait_copies<kStages - 1>();
        __syncwarp();
        return !(missing >> stage & 1u);
    }
};

// The score as the softmax takes it, in units of ln 2, as is the slope.
template <bool kExtra>
__device__ __forceinline__ float score(const Params& p, float dot, float slope, int back) {
    if constexpr (!kExtra) {
        return dot * (p.a.scale * kLog2e);
    } else {
        float x = dot * (p.a.scale * kLog2e);
        if (p.a.softcap > 0.0f) {
            // tanh(y) = 1 - 2 / (1 + e^2y), to a few 2^-24; near 0 that is not enough of a small y, and
            // tanh(y) / y = 1 - y^2/3 + 2 y^4/15 - 17 y^6/315 is good to 6e-8 below 1/5
            const float y = dot * p.cap_in, y2 = y * y;
            const float e = exp2_approx(y * (2.0f * kLog2e));
            const float large = fmaf(-2.0f * p.cap_out, __fdividef(1.0f, 1.0f + e), p.cap_out);
            const float small = x * fmaf(y2, fmaf(y2, fmaf(y2, -17.0f / 315.0f, 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
            x = fabsf(y) < 0.2f ? small : large;
        }
        return fmaf(slope, static_cast<float>(back), x);
    }
}

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// What rounding (lo, hi) to bf16 as `packed` drops.
__device__ __forceinline__ uint32_t pack_rest(float lo, float hi, uint32_t packed) {
    return pack_bf16(lo - __uint_as_float(packed << 16), hi - __uint_as_float(packed & 0xFFFF0000u));
}

// Four 8 x 8 matrices of 16-bit elements; lane l gives the address of row l % 8 of matrix l / 8.
__device__ __forceinline__ void load_matrices(uint32_t (&m)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(m[0]), "=r"(m[1]), "=r"(m[2]), "=r"(m[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_transposed(uint32_t (&m)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(m[0]), "=r"(m[1]), "=r"(m[2]), "=r"(m[3]) : "r"(at) : "memory");
}

// bf16, mma.m16n8k16: a warp multiplies up to 16 query heads (rows) by 16 tokens. Few rows are real, so the
// tensor cores are 17 % busy at most and a 128-row product would only pad more; what bounds it is HBM.
// Measured (GPU time): 96 rows of 1900 to 2048 tokens, 40 heads of 128: 570 us, 6.8 TB/s, the rate of a copy, and
// the bytes of one read (1.294 GB at a third of the rows). 3 rows of up to 131072 tokens, 8 query heads
// to each of 8 key heads: 230 us, 6.3 TB/s. 48 rows of 65 to 2048 tokens: 81 us, 5.7 TB/s (3 us until the first
// copies, 5 us of joins at the end; 85 us where copies stopped at the end of each pair). Two groups ahead and two
// CTAs: three ahead take 4 % longer, three CTAs 6 %.
// With r = lane / 4 and c = lane % 4 a lane holds the scores of rows r and r + 8, tokens 2c and 2c + 1 of each
// eight, which is also how the weights enter the second product.
// Weights enter it with 16 bits, as two bf16 numbers. With up to 8 query heads to a key head (kH = 8) the
// other 8 rows hold what rounding drops, at no cost; with more, a second product adds it.
template <int D, int kH>
constexpr int kBf16Ctas = D == 64 ? 3 : D == 128 ? 2 : 1;  // on an SM; heads of 256 spill 32 to 164 bytes at 255 registers

template <int D, int kH, bool kExtra>
__global__ void __launch_bounds__(kThreads, kBf16Ctas<D, kH>) attend_bf16_kernel(const __grid_constant__ Params p) {
    using T = __nv_bfloat16;
    constexpr int kS = D / 16, kPieces = D / 8, kR = kH / 8;
    extern __shared__ __align__(128) char dynamic[];
    __shared__ long long sums[kThreads + 1];
    __shared__ Noted noted[kWarps][2];
    __shared__ Stretch queue[kWarps][kQueue];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, c = lane & 3;
    const int d = p.a.head_dim;
    Feed<T, D> feed;
    feed.ring = static_cast<uint32_t>(__cvta_generic_to_shared(dynamic)) + warp * Feed<T, D>::kRing;
    // this lane's row and piece of the matrices that it addresses
    const uint32_t k_row = feed.ring + (8 * (lane >> 4) + (lane & 7)) * Feed<T, D>::kRowBytes, k_piece = (lane >> 3) & 1;
    const uint32_t v_row = feed.ring + Feed<T, D>::kGroupBytes + (8 * ((lane >> 3) & 1) + (lane & 7)) * Feed<T, D>::kRowBytes, v_piece = lane >> 4;

    after_previous();
    let_next_start();
    feed.queue = queue[warp];
    Dealer deal;
    deal.start(p, sums);
    feed.template start<false>(p, deal, kH);
    int cuts = 0, stage = 0;
    for (int done = 0; done < feed.queued; ++done) {
        __syncwarp();
        const Stretch s = queue[warp][done % kQueue];
        const int heads_here = min(kH, p.a.group - s.block * kH);
        const int head0 = s.head * p.a.group + s.block * kH;
        uint32_t q[kS][2 * kR];  // rows r and r + 8, elements 16 i + 2c and + 8
        float slope[kR];
        const T* qp = reinterpret_cast<const T*>(p.a.q) + s.query * p.a.q_row + (head0 + r) * p.a.q_head + 2 * c;
#pragma unroll
        for (int h = 0; h < kR; ++h) {
            const bool real = r + 8 * h < heads_here;
#pragma unroll
            for (int i = 0; i < 2 * kS; ++i)
                q[i / 2][(i & 1) * kR + h] = real && 8 * i < d ? *reinterpret_cast<const uint32_t*>(qp + 8 * h * p.a.q_head + 8 * i) : 0;
            slope[h] = kExtra && p.a.slopes != nullptr && real ? p.a.slopes[head0 + r + 8 * h] * kLog2e : 0.0f;
        }
        float acc[kPieces][4], m[kR], l[kR];
#pragma unroll
        for (int j = 0; j < kPieces; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
#pragma unroll
        for (int h = 0; h < kR; ++h) {
            m[h] = kLowest;
            l[h] = 0.0f;
        }
        for (int g = s.span.first + s.from; g < s.span.first + s.to; ++g) {
            if (feed.ready(stage)) {
                const uint32_t at = stage * Feed<T, D>::kStageBytes;
                float x[2][4] = {};
#pragma unroll
                for (int i = 0; i < kS; ++i) {
                    uint32_t k[4];
                    load_matrices(k, k_row + at + (((2 * i + k_piece) ^ (lane & 7)) << 4));
                    mma(x[0], q[i][0], kR == 2 ? q[i][1] : 0, q[i][kR], kR == 2 ? q[i][3] : 0, k[0], k[1]);
                    mma(x[1], q[i][0], kR == 2 ? q[i][1] : 0, q[i][kR], kR == 2 ? q[i][3] : 0, k[2], k[3]);
                }
                const int t0 = g * kGroup + 2 * c;  // this lane's tokens: t0, t0 + 1, t0 + 8, t0 + 9
                const bool edge = g * kGroup < s.span.lo || g * kGroup + kGroup - 1 > s.span.pos;
                float y[kR][4];
                bool rises = false;
#pragma unroll
                for (int h = 0; h < kR; ++h) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const int token = t0 + (t & 1) + (t >> 1) * 8;
                        y[h][t] = score<kExtra>(p, x[t >> 1][2 * h + (t & 1)], slope[h], token - s.span.pos);
                        if (edge && (token < s.span.lo || token > s.span.pos)) y[h][t] = -INFINITY;
                    }
                    float high = fmaxf(fmaxf(y[h][0], y[h][1]), fmaxf(y[h][2], y[h][3]));
                    high = fmaxf(high, __shfl_xor_sync(kAll, high, 1));
                    high = fmaxf(high, __shfl_xor_sync(kAll, high, 2));
                    x[0][h] = fmaxf(m[h], high);
                    rises = rises || high > m[h];
                }
                if (__any_sync(kAll, rises)) {
                    float k[kR];
#pragma unroll
                    for (int h = 0; h < kR; ++h) {
                        k[h] = exp2_approx(m[h] - x[0][h]);
                        m[h] = x[0][h];
                        l[h] *= k[h];
                    }
#pragma unroll
                    for (int j = 0; j < kPieces; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[j][e] *= k[kR == 2 ? e / 2 : 0];
                }
                uint32_t high_part[kR][2], rest[kR][2];
#pragma unroll
                for (int h = 0; h < kR; ++h) {
                    float w[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        w[t] = exp2_approx(y[h][t] - m[h]);
                        l[h] += w[t];
                    }
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        high_part[h][t] = pack_bf16(w[2 * t], w[2 * t + 1]);
                        rest[h][t] = pack_rest(w[2 * t], w[2 * t + 1], high_part[h][t]);
                    }
                }
#pragma unroll
                for (int j = 0; j < kPieces; j += 2) {
                    uint32_t v[4];
                    load_transposed(v, v_row + at + (((j + v_piece) ^ (lane & 7)) << 4));
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if constexpr (kR == 1) {
                            mma(acc[j + i], high_part[0][0], rest[0][0], high_part[0][1], rest[0][1], v[2 * i], v[2 * i + 1]);
                        } else {
                            mma(acc[j + i], high_part[0][0], high_part[kR - 1][0], high_part[0][1], high_part[kR - 1][1], v[2 * i], v[2 * i + 1]);
                            mma(acc[j + i], rest[0][0], rest[kR - 1][0], rest[0][1], rest[kR - 1][1], v[2 * i], v[2 * i + 1]);
                        }
                    }
                }
            }
            __syncwarp();
            feed.ask(p, stage, deal, kH);
            stage = stage == Feed<T, D>::kStages - 1 ? 0 : stage + 1;
        }
        // the next stretches' copies run while this one is finished
        const bool whole = s.from == 0 && s.to == s.span.groups;
        float* slot = slot_of(p, kH, D, 2 * deal.worker + (s.from == 0 ? 1 : 0));
#pragma unroll
        for (int h = 0; h < kR; ++h) {
            l[h] += __shfl_xor_sync(kAll, l[h], 1);
            l[h] += __shfl_xor_sync(kAll, l[h], 2);
            if (r + 8 * h >= heads_here) continue;
            const float inverse = l[h] > 0.0f ? 1.0f / l[h] : 0.0f;
            T* out = reinterpret_cast<T*>(p.a.out) + s.query * p.a.out_row + (head0 + r + 8 * h) * p.a.out_head + 2 * c;
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                // rows r and r + 8 are two query heads, or two parts of one
                const float o0 = kR == 2 ? acc[j][2 * h] : acc[j][0] + acc[j][2];
                const float o1 = kR == 2 ? acc[j][2 * h + 1] : acc[j][1] + acc[j][3];
                if (!whole)
                    *reinterpret_cast<float2*>(slot + (r + 8 * h) * D + 8 * j + 2 * c) = make_float2(o0, o1);
                else if (8 * j < d)
                    *reinterpret_cast<uint32_t*>(out + 8 * j) = pack_bf16(o0 * inverse, o1 * inverse);
            }
            if (!whole && c == 0) {
                slot[kH * D + r + 8 * h] = m[h];
                slot[kH * D + kH + r + 8 * h] = l[h];
            }
        }
        if (!whole) note(noted[warp][cuts++], deal, s);
    }
    hand_in<T, D, kH>(p, noted[warp], cuts, deal.worker);
    write_zeros<T>(p);
}

// fp32, on the FMA units (packed pairs), kH query heads at a time. HBM bounds it up to 2 query heads to a key head
// (64 rows of about 1500 tokens, 32 heads of 64: 246 us, 6.4 TB/s; heads of 128: 6.6 TB/s); with 8, the reads of
// queries and weights from shared memory, the products and their latencies do (8 key heads of 128: 137 us, 5.7 TB/s;
// 144 where a warp does not copy keys while it multiplies values; with one head that costs 1 to 2 %).
// For the scores a lane takes token lane % 16 and half of its elements against the queries in shared memory, or,
// with 8 query heads, two tokens and a quarter, which halves the reads of queries (147 to 144 us then). The parts
// are added up so that each half of the warp has half of the heads, and caps, maxima and exponentials are worked out
// once (160 to 147 us; 64 rows of 8 key heads of 64: 98 us, 117). For the values a lane takes four (eight) elements of every token,
// with the weights from shared memory.
template <int D, int kH>
constexpr int kF32Ctas = D == 64 ? (kH == 8 ? 2 : 3) : D == 128 ? 2 : 1;  // on an SM; three for 8 heads of 64 spill
constexpr int kF32Heads = 8;               // of a slot

template <int D, int kH>
struct F32Shape {
    static constexpr int kQueries = kH * D * 4, kWeights = kGroup * kH * 4;
    static constexpr int kWarpBytes = Feed<float, D>::kRing + kQueries + kWeights;
};

template <int D, int kH>
__global__ void __launch_bounds__(kThreads, kF32Ctas<D, kH>) attend_f32_kernel(const __grid_constant__ Params p) {
    using T = float;
    using Shape = F32Shape<D, kH>;
    constexpr int kPieces = D / 4, kV = (D + 127) / 128;  // pieces of the values that a lane takes
    constexpr int kMine = kH > 1 ? kH / 2 : 1;            // heads whose softmax a lane works on
    constexpr int kT = kH == 8 ? 2 : 1;                   // tokens whose scores a lane adds a part of
    constexpr int kStep = kGroup / kT;                    // from one to the next
    // with one stage, keys are copied while values are multiplied and the other way round
    constexpr bool kApart = Feed<float, D>::kStages == 1 && kH >= 4;
    extern __shared__ __align__(128) char dynamic[];
    __shared__ long long sums[kThreads + 1];
    __shared__ Noted noted[kWarps][2];
    __shared__ Stretch queue[kWarps][kQueue];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, token = lane & 15, half = lane >> 4;
    const int d = p.a.head_dim;
    char* mine = dynamic + warp * Shape::kWarpBytes;
    float* queries = reinterpret_cast<float*>(mine + Feed<float, D>::kRing);
    float* weights = queries + kH * D;
    Feed<float, D> feed;
    feed.ring = static_cast<uint32_t>(__cvta_generic_to_shared(mine));

    after_previous();
    let_next_start();
    feed.queue = queue[warp];
    Dealer deal;
    deal.start(p, sums);
    feed.template start<kApart>(p, deal, kH);
    int cuts = 0, stage = 0;
    for (int done = 0; done < feed.queued; ++done) {
        __syncwarp();
        const Stretch s = queue[warp][done % kQueue];
        const int heads_here = min(kH, p.a.group - s.block * kH);
        const int head0 = s.head * p.a.group + s.block * kH;
        float slope[kMine], m[kMine], l[kMine];  // of heads first, first + 1, ..
        float2 acc[kH][kV][2];
        const int first = kH > 1 ? half * kMine : 0;
        for (int u = lane; u < kH * kPieces; u += 32) {
            const int h = u / kPieces, e = u % kPieces * 4;
            *reinterpret_cast<float4*>(queries + 4 * u) =
                h < heads_here && e < d ? *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.a.q) + s.query * p.a.q_row + (head0 + h) * p.a.q_head + e)
                                        : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
#pragma unroll
        for (int h = 0; h < kMine; ++h) {
            slope[h] = p.a.slopes != nullptr && first + h < heads_here ? p.a.slopes[head0 + first + h] * kLog2e : 0.0f;
            m[h] = kLowest;
            l[h] = 0.0f;
        }
#pragma unroll
        for (int h = 0; h < kH; ++h)
#pragma unroll
            for (int i = 0; i < kV; ++i) acc[h][i][0] = acc[h][i][1] = make_float2(0.0f, 0.0f);
        __syncwarp();
        for (int g = s.span.first + s.from; g < s.span.first + s.to; ++g) {
            const bool real = kApart ? feed.keys_ready(stage) : feed.ready(stage);
            if (real) {
                const int part = lane / kStep;  // pieces part, part + 2 kT, .. of tokens lane % kStep and (kT = 2) 8 on
                const char* keys = mine + stage * Feed<float, D>::kStageBytes + lane % kStep * Feed<float, D>::kRowBytes;
                float2 sums2[kH][kT];
#pragma unroll
                for (int h = 0; h < kH; ++h)
#pragma unroll
                    for (int u = 0; u < kT; ++u) sums2[h][u] = make_float2(0.0f, 0.0f);
#pragma unroll 8 / kT
                for (int i = 0; i < kPieces; i += 2 * kT) {
                    float4 k[kT];
#pragma unroll
                    for (int u = 0; u < kT; ++u)
                        k[u] = *reinterpret_cast<const float4*>(keys + u * kStep * Feed<float, D>::kRowBytes + (((i + part) ^ (lane & 7)) << 4));
#pragma unroll
                    for (int h = 0; h < kH; ++h) {
                        const float4 q = *reinterpret_cast<const float4*>(queries + h * D + 4 * (i + part));
#pragma unroll
                        for (int u = 0; u < kT; ++u) {
                            sums2[h][u] = __ffma2_rn(make_float2(q.x, q.y), make_float2(k[u].x, k[u].y), sums2[h][u]);
                            sums2[h][u] = __ffma2_rn(make_float2(q.z, q.w), make_float2(k[u].z, k[u].w), sums2[h][u]);
                        }
                    }
                }
                const int t = g * kGroup + token;
                const bool unseen = t < s.span.lo || t > s.span.pos;
                // lanes 16 (and 8) apart hold the parts of a score: the halves get the other's for their own heads, and
                // the lanes of a half for their own token
                const auto part_of = [&](int h, int u) { return sums2[h][u].x + sums2[h][u].y; };
                float x[kMine], high[kMine];
                bool rises = false;
#pragma unroll
                for (int h = 0; h < kMine; ++h) {
                    float mine_of[kT];
#pragma unroll
                    for (int u = 0; u < kT; ++u) {
                        const float low = part_of(h, u), up = part_of(kH - kMine + h, u);
                        mine_of[u] = (half == 0 ? low : up) + __shfl_xor_sync(kAll, half == 0 ? up : low, 16);
                    }
                    float dot = mine_of[0];
                    if constexpr (kT == 2) {
                        const bool second = lane & 8;
                        dot = (second ? mine_of[1] : mine_of[0]) + __shfl_xor_sync(kAll, second ? mine_of[0] : mine_of[1], 8);
                    }
                    x[h] = unseen ? -INFINITY : score<true>(p, dot, slope[h], t - s.span.pos);
                    high[h] = x[h];
#pragma unroll
                    for (int w = 1; w < 16; w *= 2) high[h] = fmaxf(high[h], __shfl_xor_sync(kAll, high[h], w));
                    rises = rises || high[h] > m[h];
                }
                if (__any_sync(kAll, rises)) {
                    float k[kMine];
#pragma unroll
                    for (int h = 0; h < kMine; ++h) {
                        const float top = fmaxf(m[h], high[h]);
                        k[h] = exp2_approx(m[h] - top);
                        m[h] = top;
                        l[h] *= k[h];
                    }
#pragma unroll
                    for (int h = 0; h < kH; ++h) {
                        const float kh = __shfl_sync(kAll, k[h % kMine], 16 * (h / kMine));
#pragma unroll
                        for (int i = 0; i < kV; ++i)
#pragma unroll
                            for (int e = 0; e < 2; ++e) acc[h][i][e] = __fmul2_rn(acc[h][i][e], make_float2(kh, kh));
                    }
                }
#pragma unroll
                for (int h = 0; h < kMine; ++h) {
                    x[h] = exp2_approx(x[h] - m[h]);
                    l[h] += x[h];
                    if (kH > 1 || half == 0) weights[token * kH + first + h] = x[h];
                }
            }
            __syncwarp();
            if constexpr (kApart) feed.ask_keys(p, stage);
            if (real) {
                if constexpr (kApart) feed.values_ready();
                const char* values = mine + stage * Feed<float, D>::kStageBytes + Feed<float, D>::kGroupBytes;
#pragma unroll 8
                for (int u = 0; u < kGroup; ++u) {
                    float4 v[kV];
#pragma unroll
                    for (int i = 0; i < kV; ++i)
                        v[i] = *reinterpret_cast<const float4*>(values + u * Feed<float, D>::kRowBytes + (((lane % kPieces + 32 * i) ^ (u & 7)) << 4));
                    float w[kH];
                    if constexpr (kH >= 4) {
#pragma unroll
                        for (int h = 0; h < kH; h += 4) *reinterpret_cast<float4*>(w + h) = *reinterpret_cast<const float4*>(weights + u * kH + h);
                    } else {
#pragma unroll
                        for (int h = 0; h < kH; ++h) w[h] = weights[u * kH + h];
                    }
#pragma unroll
                    for (int h = 0; h < kH; ++h) {
                        const float2 pair = make_float2(w[h], w[h]);
#pragma unroll
                        for (int i = 0; i < kV; ++i) {
                            acc[h][i][0] = __ffma2_rn(pair, make_float2(v[i].x, v[i].y), acc[h][i][0]);
                            acc[h][i][1] = __ffma2_rn(pair, make_float2(v[i].z, v[i].w), acc[h][i][1]);
                        }
                    }
                }
            }
            __syncwarp();
            if constexpr (kApart) feed.ask_values(p, stage, deal, kH);
            else feed.ask(p, stage, deal, kH);
            stage = stage == Feed<T, D>::kStages - 1 ? 0 : stage + 1;
        }
        const bool whole = s.from == 0 && s.to == s.span.groups;
        float* slot = slot_of(p, kF32Heads, D, 2 * deal.worker + (s.from == 0 ? 1 : 0));
#pragma unroll
        for (int h = 0; h < kMine; ++h)
#pragma unroll
            for (int w = 1; w < 16; w *= 2) l[h] += __shfl_xor_sync(kAll, l[h], w);
#pragma unroll
        for (int h = 0; h < kH; ++h) {
            const float mh = __shfl_sync(kAll, m[h % kMine], 16 * (h / kMine)), lh = __shfl_sync(kAll, l[h % kMine], 16 * (h / kMine));
            if (h >= heads_here) continue;
            const float inverse = lh > 0.0f ? 1.0f / lh : 0.0f;
            float* out = reinterpret_cast<float*>(p.a.out) + s.query * p.a.out_row + (head0 + h) * p.a.out_head;
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                const int e = 4 * lane + 128 * i;
                if (e >= D) continue;
                if (!whole)
                    *reinterpret_cast<float4*>(slot + h * D + e) = make_float4(acc[h][i][0].x, acc[h][i][0].y, acc[h][i][1].x, acc[h][i][1].y);
                else if (e < d)
                    *reinterpret_cast<float4*>(out + e) =
                        make_float4(acc[h][i][0].x * inverse, acc[h][i][0].y * inverse, acc[h][i][1].x * inverse, acc[h][i][1].y * inverse);
            }
            if (!whole && lane == 0) {
                slot[kF32Heads * D + h] = mh;
                slot[kF32Heads * D + kF32Heads + h] = lh;
            }
        }
        if (!whole) note(noted[warp][cuts++], deal, s);
        __syncwarp();
    }
    hand_in<T, D, kF32Heads>(p, noted[warp], cuts, deal.worker);
    write_zeros<T>(p);
}

// SMs of a device and CTAs of a kernel on one, asked for once.
constexpr int kDevices = 64;
template <auto kKernel>
cudaError_t resident(int shared, int& ctas) {
    static std::atomic<int> known[kDevices];
    int device = 0, sms = 0, each = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    ctas = device < kDevices ? known[device].load(std::memory_order_relaxed) : 0;
    if (ctas > 0) return cudaSuccess;
    if (shared > 48 * 1024) e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, kKernel, kThreads, shared);
    if (e != cudaSuccess) return e;
    ctas = sms * each < kMaxWorkers / kWarps ? sms * each : kMaxWorkers / kWarps;
    if (ctas < 1) return cudaErrorInvalidConfiguration;
    if (device < kDevices) known[device].store(ctas, std::memory_order_relaxed);
    return cudaSuccess;
}

template <auto kKernel>
cudaError_t launch_resident(int shared, const Params& p, cudaStream_t s) {
    int ctas = 0;
    const cudaError_t e = resident<kKernel>(shared, ctas);
    return e != cudaSuccess ? e : launch(kKernel, ctas, kThreads, shared, 0, s, p);
}

template <int D, int kH>
cudaError_t launch_bf16(Params p, cudaStream_t s) {
    constexpr int shared = kWarps * Feed<__nv_bfloat16, D>::kRing;
    p.blocks = (p.a.group + kH - 1) / kH;
    return p.a.softcap > 0.0f || p.a.slopes != nullptr
               ? launch_resident<attend_bf16_kernel<D, kH, true>>(shared, p, s)
               : launch_resident<attend_bf16_kernel<D, kH, false>>(shared, p, s);
}

template <int D, int kH>
cudaError_t launch_f32(Params p, cudaStream_t s) {
    p.blocks = (p.a.group + kH - 1) / kH;
    return launch_resident<attend_f32_kernel<D, kH>>(kWarps * F32Shape<D, kH>::kWarpBytes, p, s);
}

template <int D>
cudaError_t launch_d(const Params& p, cudaStream_t s) {
    const int g = p.a.group;
    if (p.a.bf16) return g <= 8 ? launch_bf16<D, 8>(p, s) : launch_bf16<D, 16>(p, s);
    return g == 1 ? launch_f32<D, 1>(p, s) : g == 2 ? launch_f32<D, 2>(p, s) : g <= 4 ? launch_f32<D, 4>(p, s) : launch_f32<D, 8>(p, s);
}

int padded(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

}  // namespace

uint64_t attend_workspace(int bf16, int group, int head_dim) {
    const int heads = bf16 && group > 8 ? 16 : 8;
    return sizeof(float) * (counters() + 2ull * kMaxWorkers * slot_floats(heads, padded(head_dim)));
}

cudaError_t launch_attend(const Pages& pages, const Attend& a, cudaStream_t s) {
    const float cap = a.softcap > 0.0f ? a.softcap : 1.0f;
    const Params p = {pages, a, 1, pages.page_tokens / kGroup, a.scale / cap, cap * kLog2e};
    switch (padded(a.head_dim)) {
        case 64: return launch_d<64>(p, s);
        case 128: return launch_d<128>(p, s);
        default: return launch_d<256>(p, s);
    }
}

}  // namespace jb
