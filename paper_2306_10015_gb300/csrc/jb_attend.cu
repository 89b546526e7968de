// jb_attend.cu -- attention of single queries over the pages of a cache.
//
// A query reads each key and value of its row once and does 4 g operations per element with g
// query heads to a key head, so the bytes bound it: the kernels stream pages from HBM and keep all
// state in registers. Work is cut evenly whatever the rows' lengths: the 16-token groups of all
// (query, key head) pairs are one line, every CTA takes an equal stretch of it, and pairs that
// cross a boundary are joined by a second kernel from partial (maximum, sum, weighted values).
//
// Softmax is kept with a running maximum, so that one pass is enough:
//   m' = max(m, max_t x_t), s' = s e^(m - m') + sum e^(x_t - m'), o' likewise.
#include <atomic>

#include <cuda_bf16.h>

#include "jb_answer.h"

namespace jb {
namespace {

constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kGroup = 16;       // tokens a warp takes at a time; pages hold a multiple of it
constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kTile = kWarps;    // groups that a CTA takes at a time: one a warp
constexpr int kHeads = 8;        // query heads of one key head that are worked on together
constexpr int kMaxCtas = 1024;   // of the persistent grid; the workspace has two slots for each
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.0e38f;

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Cached pages are read once: no place in L1 for them.
__device__ __forceinline__ uint4 load_stream(const void* p) {
    uint4 v;
    asm("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
        : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
        : "l"(p));
    return v;
}

struct Params {
    Pages pages;
    Attend a;
    int blocks;        // blocks of kHeads query heads to a key head
    int page_groups;   // groups in a page
};

// The partial result of a stretch: o[kHeads][D], m[kHeads], s[kHeads].
__host__ __device__ constexpr int slot_floats(int d) { return kHeads * (d + 2); }

// Which pair a CTA started and did not finish: joined from slot 1 of the CTA and slot 0 of the
// `parts` - 1 that follow.
struct Unfinished {
    int query, head, block, parts;
};

// Groups that query i reads: [first, last] of them, none if last < first.
struct Span {
    int row, lo, pos, first, last;
    __device__ int tiles() const { return (last - first + kTile) / kTile; }
};

__device__ __forceinline__ Span span_of(const Params& p, int i) {
    Span s;
    s.row = p.a.rows[i];
    s.pos = p.a.pos[i];
    s.lo = s.first = 0;
    s.last = -1;
    if (s.row < 0 || s.row >= p.pages.n_rows || s.pos < 0 || s.pos >= p.pages.row_pages * p.pages.page_tokens) {
        s.pos = -1;
        return s;
    }
    if (p.a.window > 0) s.lo = max(0, s.pos - p.a.window + 1);
    s.first = s.lo / kGroup;
    s.last = s.pos / kGroup;
    return s;
}

// A stretch of one (query, key head, block of query heads): tiles [from, to) of `tiles`.
struct Stretch {
    int query, head, block, from, to, tiles;
    Span span;
};

// a / b; 64-bit division only where it is needed.
__device__ __forceinline__ long long quotient(long long a, long long b) {
    return ((a | b) >> 32) == 0 ? static_cast<long long>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b)) : a / b;
}

static_assert(kMaxListed <= kThreads * kThreads, "a thread's run of queries is searched by one thread each");

// Deals the line of tiles out. All threads of a CTA go through it together.
struct Dealer {
    long long next, end, total;
    int ctas;
    int query;
    long long at;         // tiles of the query before `next`
    Span span;

    __device__ static long long bound(long long total, int ctas, int cta) {
        const long long each = quotient(total, ctas);
        return each * cta + quotient((total - each * ctas) * cta, ctas);
    }

    // sums: kThreads + 1 words of shared memory, found: two.
    __device__ void start(const Params& p, long long* sums, long long* found) {
        const int n = p.a.n, pairs = p.a.heads * p.blocks;
        const int per = (n + kThreads - 1) / kThreads;
        // tiles of each thread's run of queries
        const int mine_from = static_cast<int>(threadIdx.x) * per, mine_to = min(n, mine_from + per);
        long long mine = 0;
        for (int i = mine_from; i < mine_to; ++i) mine += span_of(p, i).tiles();
        scan(mine, sums);
        total = sums[kThreads] * pairs;
        ctas = static_cast<int>(min(static_cast<long long>(gridDim.x), max(1ll, total)));
        if (static_cast<int>(blockIdx.x) >= ctas || total == 0) {
            next = end = 0;
            return;
        }
        next = bound(total, ctas, blockIdx.x);
        end = bound(total, ctas, blockIdx.x + 1);
        // the run with the tile `next`, then the query: tiles before a query are multiples of `pairs`
        const long long goal = quotient(next, pairs);
        if (sums[threadIdx.x] <= goal && goal < sums[threadIdx.x + 1]) {
            found[0] = mine_from;
            found[1] = sums[threadIdx.x];
        }
        __syncthreads();
        if (per > 1) {  // at most kThreads queries (of kMaxListed) are a run
            const long long base = found[1];
            const int i = static_cast<int>(found[0]) + threadIdx.x;
            scan(static_cast<int>(threadIdx.x) < per && i < n ? span_of(p, i).tiles() : 0, sums);
            if (base + sums[threadIdx.x] <= goal && goal < base + sums[threadIdx.x + 1]) {
                found[0] = i;
                found[1] = base + sums[threadIdx.x];
            }
            __syncthreads();
        }
        query = static_cast<int>(found[0]);
        span = span_of(p, query);
        at = next - found[1] * pairs;
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
        while (span.tiles() == 0 || at >= span.tiles() * pairs) {
            at -= span.tiles() * pairs;
            ++query;
            span = span_of(p, query);
        }
        s.query = query;
        s.span = span;
        s.tiles = span.tiles();
        const int pair = static_cast<int>(quotient(at, s.tiles));
        s.head = pair / p.blocks;
        s.block = pair % p.blocks;
        s.from = static_cast<int>(at - static_cast<long long>(pair) * s.tiles);
        s.to = static_cast<int>(min(static_cast<long long>(s.tiles), s.from + (end - next)));
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

// Adds up the warps' results, kPart elements of each head from `first` on, and stores the result itself
// or its part of a slot of the workspace. part: [kWarps][kHeads][kPart]; top, sum: [kWarps][kHeads].
template <typename T, int D, int kPart>
__device__ __forceinline__ void finish(const Params& p, const Stretch& s, int heads_here, int first, const float* part,
                                       const float* top, const float* sum) {
    const int d = p.a.head_dim;
    const bool whole = s.from == 0 && s.to == s.tiles;
    float* slot = p.a.ws + static_cast<size_t>(slot_floats(D)) * (2 * blockIdx.x + (s.from == 0 ? 1 : 0));
    for (int u = threadIdx.x; u < heads_here * kPart; u += kThreads) {
        const int h = u / kPart, e = first + u % kPart;
        float m = kLowest;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) m = fmaxf(m, top[w * kHeads + h]);
        float o = 0.0f, l = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float c = exp2_approx(top[w * kHeads + h] - m);
            o = fmaf(c, part[w * kHeads * kPart + u], o);
            l = fmaf(c, sum[w * kHeads + h], l);
        }
        if (whole) {
            const int head = (s.head * p.a.group) + s.block * kHeads + h;
            if (e < d)
                store_out(reinterpret_cast<T*>(p.a.out) + s.query * p.a.out_row + head * p.a.out_head + e, l > 0.0f ? o / l : 0.0f);
        } else {
            slot[h * D + e] = o;
            if (e == 0) {
                slot[kHeads * D + h] = m;
                slot[kHeads * D + kHeads + h] = l;
            }
        }
    }
}

// Which pair the CTA leaves for the second kernel, and zeros for the queries that see nothing.
template <typename T>
__device__ __forceinline__ void write_rest(const Params& p) {
    const int d = p.a.head_dim, heads = p.a.heads * p.a.group;
    for (int i = blockIdx.x; i < p.a.n; i += gridDim.x) {
        if (span_of(p, i).pos >= 0) continue;
        for (int u = threadIdx.x; u < heads * d; u += kThreads)
            store_out(reinterpret_cast<T*>(p.a.out) + i * p.a.out_row + u / d * p.a.out_head + u % d, 0.0f);
    }
}

__device__ __forceinline__ Unfinished* unfinished(const Params& p, int d_padded) {
    return reinterpret_cast<Unfinished*>(p.a.ws + static_cast<size_t>(slot_floats(d_padded)) * 2 * kMaxCtas);
}

__device__ __forceinline__ void note_unfinished(const Params& p, const Dealer& deal, const Stretch& s, bool any, int d_padded) {
    if (threadIdx.x != 0) return;
    Unfinished u = {0, 0, 0, 0};
    if (any && s.from == 0 && s.to < s.tiles) {
        const long long stop = deal.next - s.to + s.tiles;  // where the pair ends on the line
        u = {s.query, s.head, s.block, 1};
        while (Dealer::bound(deal.total, deal.ctas, blockIdx.x + u.parts) < stop) ++u.parts;
    }
    unfinished(p, d_padded)[blockIdx.x] = u;
}

// The score as the softmax takes it, in units of ln 2.
template <bool kExtra>
__device__ __forceinline__ float score(const Params& p, float dot, float slope, int back) {
    if constexpr (!kExtra) {
        return dot * (p.a.scale * kLog2e);
    } else {
        float x = dot * p.a.scale;
        if (p.a.softcap > 0.0f) {
            // tanh(y) = 1 - 2 / (1 + e^2y): absolute error of a few 2^-24 of the cap
            const float e = exp2_approx(x / p.a.softcap * (2.0f * kLog2e));
            x = p.a.softcap * (1.0f - __fdividef(2.0f, 1.0f + e));
        }
        return fmaf(slope, static_cast<float>(back), x) * kLog2e;
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

// 16 bytes from global to shared memory, asynchronously; zeros if not `real`.
__device__ __forceinline__ void copy_async(uint32_t to, const void* from, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void wait_copies() {
    asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
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

// bf16, mma.m16n8k16 with 8 query heads x 16 tokens a warp. Each warp copies its own groups, whole rows at a
// time, kStages ahead into a ring of its own, so that warps never wait for one another; 16-byte pieces of row t
// are stored at column (piece ^ t % 8), which makes the reads of 8 rows free of bank conflicts.
// The 16-row operand has 8 query heads; for P its other 8 rows hold what rounding P to bf16 drops, so
// that the weights enter with 16 bits at no cost.
template <int D>
struct Bf16Shape {
    static constexpr int kS = D / 16;                  // steps of the scores' inner product
    static constexpr int kPieces = D / 8;              // of a row
    static constexpr int kRows = 32 / kPieces;         // that the warp copies at a time
    static constexpr int kGroupBytes = kGroup * D * 2; // keys, and as much for the values
    static constexpr int kStages = D == 64 ? 4 : 2;
    static constexpr int kPart = D / 2;  // elements of the output that the warps add up at a time
    static constexpr int kCtas = D == 64 ? 3 : D == 128 ? 2 : 1;  // on an SM
    static constexpr int kRing = kWarps * kStages * 2 * kGroupBytes;
    static constexpr int kShared = kRing + kWarps * kHeads * kPart * 4;
};

template <int D, bool kExtra>
__global__ void __launch_bounds__(kThreads, Bf16Shape<D>::kCtas) attend_bf16_kernel(const __grid_constant__ Params p) {
    using Shape = Bf16Shape<D>;
    using T = __nv_bfloat16;
    constexpr int kS = Shape::kS, kPieces = Shape::kPieces, kRows = Shape::kRows, kStages = Shape::kStages, kPart = Shape::kPart;
    constexpr uint32_t kGroupBytes = Shape::kGroupBytes, kStageBytes = 2 * kGroupBytes, kRowBytes = D * 2;
    extern __shared__ __align__(128) char dynamic[];
    float* part = reinterpret_cast<float*>(dynamic + Shape::kRing);
    __shared__ long long sums[kThreads + 1], found[2];
    __shared__ float top[kWarps * kHeads], sum[kWarps * kHeads];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, c = lane & 3;
    const int d = p.a.head_dim;
    const uint32_t ring = static_cast<uint32_t>(__cvta_generic_to_shared(dynamic)) + warp * kStages * kStageBytes;
    // this lane's row and piece of a copy, and of the matrices that it addresses
    const int row = lane / kPieces, piece = lane % kPieces;
    const uint32_t k_row = ring + (8 * (lane >> 4) + (lane & 7)) * kRowBytes, k_piece = (lane >> 3) & 1;
    const uint32_t v_row = ring + kGroupBytes + (8 * ((lane >> 3) & 1) + (lane & 7)) * kRowBytes, v_piece = lane >> 4;

    // Copies of a stretch's groups: what is next to be asked for, and which of the stages hold a group
    // whose page is missing.
    struct Feed {
        const int* table;
        uint64_t at;         // the key head's, this lane's row and piece, in elements
        int group, stop, page, lo, pos;
        uint32_t missing;
    } feed = {};
    const auto ahead = [&] { feed.page = feed.group < feed.stop ? feed.table[feed.group / p.page_groups] : -1; };
    const auto open = [&](const Stretch& s) {
        feed.table = p.pages.table + static_cast<size_t>(s.span.row) * p.pages.row_pages;
        feed.at = s.head * p.a.head_stride + row * p.a.token_stride + 8 * piece;
        feed.group = s.span.first + s.from * kTile + warp;
        feed.stop = min(s.span.last + 1, s.span.first + s.to * kTile);
        feed.lo = s.span.lo;
        feed.pos = s.span.pos;
        feed.missing = 0;
        ahead();
    };
    const auto ask = [&](int stage) {
        if (feed.group < feed.stop) {
            const bool real = feed.page >= 0 && feed.page < p.pages.n_pages;
            feed.missing = (feed.missing & ~(1u << stage)) | (real ? 0u : 1u << stage);
            if (real) {
                const uint64_t at = feed.at + feed.page * p.a.page_stride + feed.group % p.page_groups * kGroup * p.a.token_stride;
                const T* kp = reinterpret_cast<const T*>(p.a.k) + at;
                const T* vp = reinterpret_cast<const T*>(p.a.v) + at;
                const uint32_t to = ring + stage * kStageBytes + row * kRowBytes;
                const int token = feed.group * kGroup + row;
                const bool inside = 8 * piece < d;
#pragma unroll
                for (int j = 0; j < kGroup; j += kRows) {
                    const uint32_t place = to + j * kRowBytes + ((piece ^ ((row + j) & 7)) << 4);
                    copy_async(place, kp + j * p.a.token_stride, inside);
                    // a value that is not seen must not reach the sum, whatever it holds
                    copy_async(place + kGroupBytes, vp + j * p.a.token_stride, inside && token + j >= feed.lo && token + j <= feed.pos);
                }
            }
            feed.group += kTile;
            ahead();
        }
        commit_copies();
    };

    Dealer deal;
    deal.start(p, sums, found);
    Stretch s, after;
    bool any = deal.take(p, s), more = any;
    if (more) {
        open(s);
#pragma unroll
        for (int i = 0; i < kStages; ++i) ask(i);
    }
    while (more) {
        const int heads_here = min(kHeads, p.a.group - s.block * kHeads);
        const int head0 = s.head * p.a.group + s.block * kHeads;
        uint32_t q[kS][2];
        const T* qp = reinterpret_cast<const T*>(p.a.q) + s.query * p.a.q_row + (head0 + r) * p.a.q_head + 2 * c;
#pragma unroll
        for (int i = 0; i < kS; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                q[i][h] = r < heads_here && 16 * i + 8 * h < d ? *reinterpret_cast<const uint32_t*>(qp + 16 * i + 8 * h) : 0;
        const float slope = kExtra && p.a.slopes != nullptr && r < heads_here ? p.a.slopes[head0 + r] : 0.0f;

        float acc[kPieces][4];
#pragma unroll
        for (int j = 0; j < kPieces; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
        float m = kLowest, l = 0.0f;
        const int stop = feed.stop;
        int stage = 0;
        for (int g = s.span.first + s.from * kTile + warp; g < stop; g += kTile) {
            wait_copies<kStages - 1>();
            __syncwarp();
            const uint32_t at = stage * kStageBytes;
            if (!(feed.missing >> stage & 1u)) {
                float x[2][4] = {};
#pragma unroll
                for (int i = 0; i < kS; ++i) {
                    uint32_t k[4];
                    load_matrices(k, k_row + at + (((2 * i + k_piece) ^ (lane & 7)) << 4));
                    mma(x[0], q[i][0], 0, q[i][1], 0, k[0], k[1]);
                    mma(x[1], q[i][0], 0, q[i][1], 0, k[2], k[3]);
                }
                const int t0 = g * kGroup + 2 * c;  // this lane's tokens: t0, t0 + 1, t0 + 8, t0 + 9
                const bool edge = g * kGroup < s.span.lo || g * kGroup + kGroup - 1 > s.span.pos;
                float y[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int token = t0 + (t & 1) + (t >> 1) * 8;
                    y[t] = score<kExtra>(p, x[t >> 1][t & 1], slope, token - s.span.pos);
                    if (edge && (token < s.span.lo || token > s.span.pos)) y[t] = -INFINITY;
                }
                float high = fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3]));
                high = fmaxf(high, __shfl_xor_sync(kAll, high, 1));
                high = fmaxf(high, __shfl_xor_sync(kAll, high, 2));
                if (__any_sync(kAll, high > m)) {
                    const float next = fmaxf(m, high), k = exp2_approx(m - next);
                    m = next;
                    l *= k;
#pragma unroll
                    for (int j = 0; j < kPieces; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[j][e] *= k;
                }
                float w[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    w[t] = exp2_approx(y[t] - m);
                    l += w[t];
                }
                const uint32_t a0 = pack_bf16(w[0], w[1]), a2 = pack_bf16(w[2], w[3]);
                const uint32_t a1 = pack_bf16(w[0] - __uint_as_float(a0 << 16), w[1] - __uint_as_float(a0 & 0xFFFF0000u));
                const uint32_t a3 = pack_bf16(w[2] - __uint_as_float(a2 << 16), w[3] - __uint_as_float(a2 & 0xFFFF0000u));
#pragma unroll
                for (int j = 0; j < kPieces; j += 2) {
                    uint32_t v[4];
                    load_transposed(v, v_row + at + (((j + v_piece) ^ (lane & 7)) << 4));
                    mma(acc[j], a0, a1, a2, a3, v[0], v[1]);
                    mma(acc[j + 1], a0, a1, a2, a3, v[2], v[3]);
                }
            }
            __syncwarp();
            ask(stage);
            stage = stage == kStages - 1 ? 0 : stage + 1;
        }
        // the next stretch's copies run while this one is added up
        more = deal.take(p, after);
        if (more) {
            open(after);
#pragma unroll
            for (int i = 0; i < kStages; ++i) ask(i);
        }
        l += __shfl_xor_sync(kAll, l, 1);
        l += __shfl_xor_sync(kAll, l, 2);
        if (c == 0) {
            top[warp * kHeads + r] = m;
            sum[warp * kHeads + r] = l;
        }
#pragma unroll
        for (int h = 0; h < D / kPart; ++h) {
            if (r < heads_here) {
                float* to = part + (warp * kHeads + r) * kPart;
#pragma unroll
                for (int j = 0; j < kPart / 8; ++j) {
                    const float(&x)[4] = acc[h * (kPart / 8) + j];
                    *reinterpret_cast<float2*>(to + 8 * j + 2 * c) = make_float2(x[0] + x[2], x[1] + x[3]);
                }
            }
            __syncthreads();
            finish<T, D, kPart>(p, s, heads_here, h * kPart, part, top, sum);
            __syncthreads();
        }
        if (!more) break;
        s = after;
    }
    note_unfinished(p, deal, s, any, D);
    write_rest<T>(p);
}

// fp32, on the FMA units. kH query heads at a time. For the scores lane (r, c) takes key token r,
// elements 16 s + 4 c .. + 3, against the queries in shared memory, and the quad adds up; for the
// values a lane takes elements 4 lane .. + 3 of every token, with the weights from the lanes that
// hold them.
template <int D, int kH>
__global__ void __launch_bounds__(kThreads) attend_f32_kernel(const __grid_constant__ Params p) {
    constexpr int kS = D / 16, kV = (D + 127) / 128;
    __shared__ long long sums[kThreads + 1], found[2];
    __shared__ __align__(16) float part[kWarps * kHeads * D];
    __shared__ __align__(16) float queries[kH * D];
    __shared__ float top[kWarps * kHeads], sum[kWarps * kHeads];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, c = lane & 3;
    const int d = p.a.head_dim;

    Dealer deal;
    deal.start(p, sums, found);
    Stretch s;
    bool any = false;
    while (deal.take(p, s)) {
        any = true;
        const int heads_here = min(kHeads, p.a.group - s.block * kHeads);
        const int head0 = s.head * p.a.group + s.block * kHeads;
        for (int u = threadIdx.x; u < kH * D; u += kThreads) {
            const int h = u / D, e = u % D;
            queries[u] = h < heads_here && e < d
                             ? reinterpret_cast<const float*>(p.a.q)[s.query * p.a.q_row + (head0 + h) * p.a.q_head + e]
                             : 0.0f;
        }
        __syncthreads();
        float slope[kH], m[kH], l[kH], acc[kH][kV][4];
#pragma unroll
        for (int h = 0; h < kH; ++h) {
            slope[h] = p.a.slopes != nullptr && h < heads_here ? p.a.slopes[head0 + h] : 0.0f;
            m[h] = kLowest;
            l[h] = 0.0f;
#pragma unroll
            for (int i = 0; i < kV; ++i) acc[h][i][0] = acc[h][i][1] = acc[h][i][2] = acc[h][i][3] = 0.0f;
        }
        const int* table = p.pages.table + static_cast<size_t>(s.span.row) * p.pages.row_pages;
        const int stop = min(s.span.last + 1, s.span.first + s.to * kTile);
        for (int g = s.span.first + s.from * kTile + warp; g < stop; g += kTile) {
            const int page = table[g / p.page_groups];
            if (page < 0 || page >= p.pages.n_pages) continue;
            const uint64_t at = page * p.a.page_stride + s.head * p.a.head_stride + g % p.page_groups * kGroup * p.a.token_stride;
            const float* kp = reinterpret_cast<const float*>(p.a.k) + at;
            const float* vp = reinterpret_cast<const float*>(p.a.v) + at;
            float x[2][kH] = {};
#pragma unroll
            for (int i = 0; i < kS; ++i) {
                if (16 * i + 4 * c >= d) break;
                float4 kf[2];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const uint4 v = load_stream(kp + (8 * t + r) * p.a.token_stride + 16 * i + 4 * c);
                    kf[t] = make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
                }
#pragma unroll
                for (int h = 0; h < kH; ++h) {
                    const float4 q = *reinterpret_cast<const float4*>(queries + h * D + 16 * i + 4 * c);
#pragma unroll
                    for (int t = 0; t < 2; ++t)
                        x[t][h] = fmaf(q.w, kf[t].w, fmaf(q.z, kf[t].z, fmaf(q.y, kf[t].y, fmaf(q.x, kf[t].x, x[t][h]))));
                }
            }
            const bool edge = g * kGroup < s.span.lo || g * kGroup + kGroup - 1 > s.span.pos;
            float w[2][kH];
#pragma unroll
            for (int h = 0; h < kH; ++h) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    float y = x[t][h];
                    y += __shfl_xor_sync(kAll, y, 1);
                    y += __shfl_xor_sync(kAll, y, 2);
                    const int token = g * kGroup + 8 * t + r;
                    y *= p.a.scale;
                    if (p.a.softcap > 0.0f) y = p.a.softcap * tanhf(y / p.a.softcap);
                    y = fmaf(slope[h], static_cast<float>(token - s.span.pos), y);
                    if (edge && (token < s.span.lo || token > s.span.pos)) y = -INFINITY;
                    w[t][h] = y;
                }
                float high = fmaxf(w[0][h], w[1][h]);
                high = fmaxf(high, __shfl_xor_sync(kAll, high, 4));
                high = fmaxf(high, __shfl_xor_sync(kAll, high, 8));
                high = fmaxf(high, __shfl_xor_sync(kAll, high, 16));
                if (high > m[h]) {
                    const float k = exp2_approx((m[h] - high) * kLog2e);
                    m[h] = high;
                    l[h] *= k;
#pragma unroll
                    for (int i = 0; i < kV; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[h][i][e] *= k;
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    w[t][h] = exp2_approx((w[t][h] - m[h]) * kLog2e);
                    l[h] += w[t][h];
                }
            }
#pragma unroll
            for (int t = 0; t < kGroup; ++t) {
                const int token = g * kGroup + t;
                if (edge && (token < s.span.lo || token > s.span.pos)) continue;  // the warp agrees
                float4 v[kV];
#pragma unroll
                for (int i = 0; i < kV; ++i) {
                    uint4 u = make_uint4(0, 0, 0, 0);
                    if (128 * i + 4 * lane < d) u = load_stream(vp + t * p.a.token_stride + 128 * i + 4 * lane);
                    v[i] = make_float4(__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w));
                }
#pragma unroll
                for (int h = 0; h < kH; ++h) {
                    const float weight = __shfl_sync(kAll, w[t >> 3][h], (t & 7) * 4);
#pragma unroll
                    for (int i = 0; i < kV; ++i) {
                        acc[h][i][0] = fmaf(weight, v[i].x, acc[h][i][0]);
                        acc[h][i][1] = fmaf(weight, v[i].y, acc[h][i][1]);
                        acc[h][i][2] = fmaf(weight, v[i].z, acc[h][i][2]);
                        acc[h][i][3] = fmaf(weight, v[i].w, acc[h][i][3]);
                    }
                }
            }
        }
#pragma unroll
        for (int h = 0; h < kH; ++h) {
            l[h] += __shfl_xor_sync(kAll, l[h], 4);
            l[h] += __shfl_xor_sync(kAll, l[h], 8);
            l[h] += __shfl_xor_sync(kAll, l[h], 16);
            if (lane == 0) {
                top[warp * kHeads + h] = m[h] * kLog2e;
                sum[warp * kHeads + h] = l[h];
            }
#pragma unroll
            for (int i = 0; i < kV; ++i)
                if (128 * i + 4 * lane < D)
                    *reinterpret_cast<float4*>(part + (warp * kHeads + h) * D + 128 * i + 4 * lane) =
                        make_float4(acc[h][i][0], acc[h][i][1], acc[h][i][2], acc[h][i][3]);
        }
        __syncthreads();
        finish<float, D, D>(p, s, heads_here, 0, part, top, sum);
        __syncthreads();
    }
    note_unfinished(p, deal, s, any, D);
    write_rest<float>(p);
}

// Joins a pair's partial results; one CTA for each CTA that left one, in the order of the line.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) join_kernel(const __grid_constant__ Params p) {
    const Unfinished u = unfinished(p, D)[blockIdx.x];
    if (u.parts == 0) return;
    const int heads_here = min(kHeads, p.a.group - u.block * kHeads), d = p.a.head_dim;
    const auto slot = [&](int i) {
        return p.a.ws + static_cast<size_t>(slot_floats(D)) * (2 * (blockIdx.x + i) + (i == 0 ? 1 : 0));
    };
    for (int e = threadIdx.x; e < heads_here * D; e += kThreads) {
        const int h = e / D;
        float m = kLowest;
        for (int i = 0; i < u.parts; ++i) m = fmaxf(m, slot(i)[kHeads * D + h]);
        float o = 0.0f, l = 0.0f;
        for (int i = 0; i < u.parts; ++i) {
            const float* f = slot(i);
            const float c = exp2_approx(f[kHeads * D + h] - m);
            o = fmaf(c, f[e], o);
            l = fmaf(c, f[kHeads * D + kHeads + h], l);
        }
        if (e % D < d)
            store_out(reinterpret_cast<T*>(p.a.out) + u.query * p.a.out_row + (u.head * p.a.group + u.block * kHeads + h) * p.a.out_head + e % D,
                      l > 0.0f ? o / l : 0.0f);
    }
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
    ctas = sms * each < kMaxCtas ? sms * each : kMaxCtas;
    if (device < kDevices) known[device].store(ctas, std::memory_order_relaxed);
    return cudaSuccess;
}

template <auto kKernel>
cudaError_t launch_both(int shared, void (*join)(Params), const Params& p, cudaStream_t s) {
    int ctas = 0;
    cudaError_t e = resident<kKernel>(shared, ctas);
    if (e != cudaSuccess) return e;
    kKernel<<<ctas, kThreads, shared, s>>>(p);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    join<<<ctas, kThreads, 0, s>>>(p);
    return cudaGetLastError();
}

template <int D>
cudaError_t launch_d(const Params& p, cudaStream_t s) {
    if (p.a.bf16) {
        constexpr int shared = Bf16Shape<D>::kShared;
        return p.a.softcap > 0.0f || p.a.slopes != nullptr
                   ? launch_both<attend_bf16_kernel<D, true>>(shared, join_kernel<__nv_bfloat16, D>, p, s)
                   : launch_both<attend_bf16_kernel<D, false>>(shared, join_kernel<__nv_bfloat16, D>, p, s);
    }
    const int g = p.a.group;
    return g == 1   ? launch_both<attend_f32_kernel<D, 1>>(0, join_kernel<float, D>, p, s)
           : g == 2 ? launch_both<attend_f32_kernel<D, 2>>(0, join_kernel<float, D>, p, s)
           : g <= 4 ? launch_both<attend_f32_kernel<D, 4>>(0, join_kernel<float, D>, p, s)
                    : launch_both<attend_f32_kernel<D, 8>>(0, join_kernel<float, D>, p, s);
}

int padded(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

}  // namespace

uint64_t attend_workspace(int, int, int, int head_dim) {
    return kMaxCtas * (2ull * slot_floats(padded(head_dim)) * sizeof(float) + sizeof(Unfinished));
}

cudaError_t launch_attend(const Pages& pages, const Attend& a, cudaStream_t s) {
    const Params p = {pages, a, (a.group + kHeads - 1) / kHeads, pages.page_tokens / kGroup};
    switch (padded(a.head_dim)) {
        case 64: return launch_d<64>(p, s);
        case 128: return launch_d<128>(p, s);
        default: return launch_d<256>(p, s);
    }
}

}  // namespace jb
