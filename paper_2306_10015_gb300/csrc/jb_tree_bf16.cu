// jb_tree_bf16.cu -- jb_attend_tree on the tensor cores, for bf16 caches.
//
// A block of 128 rows (node, query head of the key head) is one tile of tcgen05.mma, and its row's keys and values pass by
// it once, 128 (heads of up to 128) or 64 positions at a time:
//   S = Q K^T (fp32, tensor memory), P = exp(S - m), O = O + P V (fp32, tensor memory)
// with the maximum m of the softmax kept as it was until a row exceeds it by 2^8; only then is O multiplied. Weights enter
// the second product as two bf16 numbers, 16 bits of them.
//
// Roles of a CTA, one on an SM: two warps copy keys and values (cp.async, whole rows, any page size and layout) into a
// ring of swizzled tiles; one thread issues the products; four warps, a thread a row, take scores from tensor memory and put
// weights in their place, so that of three score tiles one is being multiplied, one worked on and one its values' operand.
#include <atomic>

#include <cuda_bf16.h>

#include "jb_tcgen05.cuh"
#include "jb_tree.cuh"

namespace jb {
namespace {

using T = __nv_bfloat16;

constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kRows = 128;
constexpr int kSoftmaxWarps = 4, kCopyWarps = 2;
constexpr int kThreads = 256;        // a warp more than have a role: registers are dealt out to four warps at a time
constexpr int kScoreTiles = 3;
constexpr uint32_t kColumns = 512;   // of tensor memory
constexpr float kSlack = 8.0f;       // how far a row may exceed its maximum before sums are scaled, in powers of two

template <int D>
struct Shape {
    static constexpr int kTile = D == 256 ? 64 : 128;
    static constexpr int kSlots = D == 64 ? 8 : D == 128 ? 5 : 4;
    static constexpr int kDepth = kSlots - 2;  // tiles that are copied before the first of them is waited for
    static constexpr uint32_t kTileBytes = kTile * D * 2, kQueryBytes = kRows * D * 2;
    static constexpr uint32_t kPanel = kTile * 128, kQueryPanel = kRows * 128;  // 64 elements of all rows
    static constexpr uint32_t kSums = kScoreTiles * kTile;                      // column of O
    static constexpr int kShared = 1024 + kQueryBytes + kSlots * kTileBytes;
    static_assert(kSums + D <= kColumns);
};

struct Control {
    unsigned long long full[8], empty[8], scores[kScoreTiles], weights[kScoreTiles], queries, sums, drained;
    uint32_t tmem;
    int failed;
    int not_finite;       // a value that some rows see and others do not was not finite, in some tile so far
    unsigned missing[8];  // groups of a tile whose page is missing; copies are at most five tiles ahead of the softmax
};

// Whether some of the positions [t, t + n) are seen by some nodes and not by others.
__device__ __forceinline__ bool edge_of(const TreeParams& p, const Span& s, int t, int n) {
    return t + n > s.base || (p.a.window > 0 && t < static_cast<long long>(s.base) + kMaxNodes - p.a.window);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <int D>
__device__ void copy_role(const TreeParams& p, Dealer<kRows, Shape<D>::kTile, kThreads> deal, Control& c, uint32_t ring) {
    using S = Shape<D>;
    constexpr int kTile = S::kTile, kGroups = kTile / kGroup, kPieces = D / 8, kStep = 32 * kCopyWarps / kPieces, kSteps = kTile / kStep;
    const int u = threadIdx.x - 32 * (kSoftmaxWarps + 1), lane = u & 31, piece = u % kPieces, row0 = u / kPieces;
    const int d = p.a.head_dim, pieces = (d + 15) / 16 * 2;  // products take 16 elements: the last piece may be zeros
    // where this thread's piece of row row0 is in a tile; rows further on are a multiple of 8 rows or 4 rows away
    const uint32_t panel = static_cast<uint32_t>(piece >> 3) * S::kPanel;
    uint32_t next = 0, signalled = 0;
    const auto slot_at = [&](uint32_t i) { return ring + i % S::kSlots * S::kTileBytes; };
    const auto place = [&](uint32_t i, int row) { return slot_at(i) + panel + row * 128 + (((piece & 7) ^ (row & 7)) << 4); };
    uint32_t edges = 0;  // bit i % 32: tile i holds values that some rows do not see
    const auto signal = [&]() {  // tile `signalled` has arrived
        const uint32_t i = signalled++;
        if (edges >> (i % 32) & 1u) {
            edges &= ~(1u << (i % 32));
            // a value that is not finite must not meet a weight of zero: it is taken out here and added at the end to
            // the rows that see it
            bool bad = false;
            if (piece < pieces)
                for (int k = 0; k < kSteps; ++k) {
                    const uint32_t at = place(i, row0 + k * kStep);
                    uint32_t w[4], any = 0;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t mask = ((w[e] & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((w[e] & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
                        w[e] &= ~mask;
                        any |= mask;
                    }
                    if (any == 0) continue;
                    bad = true;
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                }
            if (bad) *static_cast<volatile int*>(&c.not_finite) = 1;
        }
        shared_to_async_proxy();
        __syncwarp();
        if (lane == 0) barrier_arrive(shared_address(&c.full[i % S::kSlots]));
    };
    Piece s;
    uint32_t tiles = 0;
    while (deal.take(p, s)) {
        const int* table = p.pages.table + static_cast<size_t>(s.span.row) * p.pages.row_pages;
        // lane g: page and place of the tile's group g
        const auto look_up = [&](int tile) {
            const int group = tile * kGroups + lane;
            return lane < kGroups && group * kGroup < s.span.len ? table[group / p.page_groups] : -1;
        };
        const int stop = s.span.first_tile + s.to;
        int page = look_up(s.span.first_tile + s.from);
        for (int tile = s.span.first_tile + s.from; tile < stop; ++tile, ++tiles) {
            const int t0 = tile * kTile, group = tile * kGroups + lane;
            const bool real = page >= 0 && page < p.pages.n_pages;
            const unsigned missing = ~__ballot_sync(kAll, real) & ((1u << kGroups) - 1u);
            const long long at = real ? static_cast<long long>(page * p.a.page_stride + group % p.page_groups * (kGroup * p.a.token_stride)) : 0;
            if (u == 0) *static_cast<volatile unsigned*>(&c.missing[tiles % 8]) = missing;
            if (tile + 1 < stop) page = look_up(tile + 1);
            const bool edge = edge_of(p, s.span, t0, kTile);
#pragma unroll
            for (int kind = 0; kind < 2; ++kind) {
                const uint32_t i = next++;
                if (!__all_sync(kAll, barrier_wait(shared_address(&c.empty[i % S::kSlots]), (i / S::kSlots & 1) ^ 1, &c.failed))) {
                    copies_wait<0>();
                    return;
                }
                const T* from = reinterpret_cast<const T*>(kind == 0 ? p.a.k : p.a.v) + s.head * p.a.head_stride + 8 * piece;
#pragma unroll
                for (int k = 0; k < kSteps; ++k) {
                    constexpr int kPerGroup = kGroup / kStep > 0 ? kGroup / kStep : 1;
                    const int row = row0 + k * kStep, t = t0 + row;
                    const long long base = __shfl_sync(kAll, at, k / kPerGroup);
                    const bool seen = !(missing >> (k / kPerGroup) & 1u) && t >= s.span.lo && t < s.span.len && 8 * piece < d;
                    if (piece < pieces) copy_async16(place(i, row), from + base + (row % kGroup) * p.a.token_stride, seen);
                }
                copies_commit();
                if (kind == 1 && edge) edges |= 1u << (i % 32);
                if (next > S::kDepth) {
                    copies_wait<S::kDepth>();
                    signal();
                }
            }
        }
    }
    copies_wait<0>();
    while (signalled < next) signal();
}

template <int D>
__device__ void product_role(const TreeParams& p, Dealer<kRows, Shape<D>::kTile, kThreads> deal, Control& c, uint32_t queries, uint32_t ring) {
    using S = Shape<D>;
    constexpr int kTile = S::kTile;
    const int steps = (p.a.head_dim + 15) / 16;
    constexpr uint32_t kScores = product_descriptor(kTile, false);
    const uint32_t values = product_descriptor(16 * steps, true);
    const uint32_t tmem = c.tmem;
    uint32_t tiles = 0, blocks = 0;  // so far
    const auto scores_of = [&](uint32_t tile) {
        const uint32_t i = 2 * tile;
        if (!barrier_wait(shared_address(&c.full[i % S::kSlots]), i / S::kSlots & 1, &c.failed)) return false;
        tc_fence_after();
        const uint32_t k = ring + i % S::kSlots * S::kTileBytes;
        for (int e = 0; e < steps; ++e)
            tc_product(tmem + tile % kScoreTiles * kTile, tile_descriptor(queries + e / 4 * S::kQueryPanel + e % 4 * 32, 16),
                       tile_descriptor(k + e / 4 * S::kPanel + e % 4 * 32, 16), kScores, e > 0);
        tc_commit(shared_address(&c.empty[i % S::kSlots]));
        tc_commit(shared_address(&c.scores[tile % kScoreTiles]));
        return true;
    };
    Piece s;
    while (deal.take(p, s)) {
        const uint32_t n = s.to - s.from;
        if (!barrier_wait(shared_address(&c.queries), blocks++ & 1, &c.failed)) return;
        tc_fence_after();
        if (!scores_of(tiles)) return;
        if (n > 1 && !scores_of(tiles + 1)) return;
        for (uint32_t j = 0; j < n; ++j, ++tiles) {
            const uint32_t i = 2 * tiles + 1, buffer = tiles % kScoreTiles;
            if (!barrier_wait(shared_address(&c.weights[buffer]), tiles / kScoreTiles & 1, &c.failed)) return;
            if (!barrier_wait(shared_address(&c.full[i % S::kSlots]), i / S::kSlots & 1, &c.failed)) return;
            tc_fence_after();
            const uint32_t v = ring + i % S::kSlots * S::kTileBytes, w = tmem + buffer * kTile;
#pragma unroll
            for (int half = 0; half < 2; ++half)  // the weights' upper and lower bits
                for (int e = 0; e < kTile / 16; ++e)
                    tc_product_from_tmem(tmem + S::kSums, w + half * (kTile / 2) + 8 * e, tile_descriptor(v + e * 2048, S::kPanel), values,
                                         j > 0 || half > 0 || e > 0);
            tc_commit(shared_address(&c.empty[i % S::kSlots]));
            tc_commit(shared_address(&c.sums));
            if (j + 2 < n && !scores_of(tiles + 2)) return;
        }
    }
}

template <int D, bool kExtra>
__device__ void softmax_role(const TreeParams& p, Dealer<kRows, Shape<D>::kTile, kThreads> deal, Control& c, Nodes& nodes, uint32_t queries) {
    using S = Shape<D>;
    constexpr int kTile = S::kTile, kPieces = D / 8;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, d = p.a.head_dim;
    const uint32_t tmem = c.tmem + (static_cast<uint32_t>(32 * warp) << 16);
    const float factor = p.a.scale * kLog2e;  // positive unless kExtra
    uint32_t tiles = 0;
    int tree = -1;
    bool ok = true;  // a wait that gives up leaves the loops as they are: other warps may wait for this one
    Piece s;
    while (deal.take(p, s)) {
        if (s.tree != tree)
            fill_nodes<32 * kSoftmaxWarps>(p, s.span, nodes, threadIdx.x, [](bool x) {
                uint32_t any;
                asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.or.pred p, 1, %2, q;\n selp.u32 %0, 1, 0, p;\n}"
                             : "=r"(any) : "r"(static_cast<uint32_t>(x)), "n"(32 * kSoftmaxWarps) : "memory");
                return any != 0;
            });
        tree = s.tree;
        const int rows = s.span.nodes * p.a.group, all = s.block * kRows + threadIdx.x;
        const bool real = all < rows, idle = s.block * kRows + 32 * warp >= rows;  // idle: none of the warp's rows is real
        const int node = real ? all / p.a.group : 0, h = real ? all - node * p.a.group : 0, depth = real ? nodes.depth[node] : -1;
        {   // the warp's queries
            const T* mine = reinterpret_cast<const T*>(p.a.q) + (s.span.first + node) * p.a.q_row + (s.head * p.a.group + h) * p.a.q_head;
            constexpr int kLanes = kPieces < 32 ? kPieces : 32, kAtOnce = 32 / kLanes;
            const int piece = lane % kLanes;
            const unsigned valid = __ballot_sync(kAll, real);
            if (!idle)
#pragma unroll 4
                for (int k = 0; k < 32; k += kAtOnce) {
                    const int r = k + lane / kLanes, row = 32 * warp + r;
                    const T* from = reinterpret_cast<const T*>(__shfl_sync(kAll, reinterpret_cast<unsigned long long>(mine), r));
                    copy_async16(queries + (piece >> 3) * S::kQueryPanel + row * 128 + (((piece & 7) ^ (row & 7)) << 4), from + 8 * piece,
                                 (valid >> r & 1u) && 8 * piece < d);
                }
            copies_commit();
            copies_wait<0>();
            shared_to_async_proxy();
            __syncwarp();
            if (lane == 0) barrier_arrive(shared_address(&c.queries));
        }
        const float slope = kExtra && real && p.a.slopes != nullptr ? p.a.slopes[s.head * p.a.group + h] * kLog2e : 0.0f;
        float m = kLowest, offset = 0.0f, l = 0.0f;  // offset: what is subtracted from scores, in powers of two; 0 before one is seen
        for (int tile = s.span.first_tile + s.from; tile < s.span.first_tile + s.to; ++tile, ++tiles) {
            const int t0 = tile * kTile;
            const uint32_t buffer = tiles % kScoreTiles, at = tmem + buffer * kTile;
            ok = barrier_wait(shared_address(&c.scores[buffer]), tiles / kScoreTiles & 1, &c.failed) && ok;
            tc_fence_after();
            if (!idle) {
                uint32_t raw[kTile];
#pragma unroll
                for (int k = 0; k < kTile; k += 32) tmem_load32(at + k, raw + k);
                tc_wait_loads();
                const unsigned missing = *static_cast<volatile unsigned*>(&c.missing[tiles % 8]);
                const bool edge = missing != 0 || edge_of(p, s.span, t0, kTile);
                if (kExtra || edge) {
#pragma unroll
                    for (int k = 0; k < kTile; k += 32) {
                        unsigned seen = kAll;
                        if (edge) {
                            seen = seen_of(p, s.span, depth, nodes.mask[node], t0 + k);
                            if (missing >> (k / kGroup) & 1u) seen &= 0xFFFF0000u;
                            if (missing >> (k / kGroup + 1) & 1u) seen &= 0x0000FFFFu;
                        }
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            float x = __uint_as_float(raw[k + e]);
                            const bool sees = seen >> e & 1u;
                            if constexpr (kExtra) {
                                const int t = t0 + k + e;
                                int back = t - s.span.base - depth;
                                if (edge && sees && t >= s.span.base) back = nodes.depth[t - s.span.base] - depth;
                                x = score<true>(p, x, slope, back);
                            }
                            raw[k + e] = __float_as_uint(sees ? x : -INFINITY);
                        }
                    }
                }
                float high = kLowest;
#pragma unroll
                for (int k = 0; k < kTile; ++k) high = fmaxf(high, __uint_as_float(raw[k]));
                const float by = kExtra ? 1.0f : factor;
                const bool first = tile == s.span.first_tile + s.from;
                const bool rises = high > m && (m == kLowest || (high - m) * by > kSlack);
                if (__any_sync(kAll, rises)) {
                    float k = 1.0f;
                    if (rises) {
                        const float top = high * by;
                        k = m == kLowest ? 0.0f : exp2_approx(offset - top);
                        m = high;
                        offset = top;
                        l *= k;
                    }
                    if (!first) {
                        ok = barrier_wait(shared_address(&c.sums), (tiles - 1) & 1, &c.failed) && ok;
                        tc_fence_after();
#pragma unroll
                        for (int e = 0; e < D; e += 32) {
                            uint32_t o[32];
                            tmem_load32(tmem + S::kSums + e, o);
                            tc_wait_loads();
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * k);
                            tmem_store32(tmem + S::kSums + e, o);
                        }
                    }
                }
                float part[4] = {};
#pragma unroll
                for (int k = 0; k < kTile; k += 64) {
                    uint32_t upper[32], lower[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const float x0 = __uint_as_float(raw[k + 2 * e]), x1 = __uint_as_float(raw[k + 2 * e + 1]);
                        const float w0 = exp2_approx(kExtra ? x0 - offset : fmaf(x0, by, -offset));
                        const float w1 = exp2_approx(kExtra ? x1 - offset : fmaf(x1, by, -offset));
                        part[e & 1] += w0;
                        part[2 + (e & 1)] += w1;
                        upper[e] = pack_bf16(w0, w1);
                        lower[e] = pack_bf16(w0 - __uint_as_float(upper[e] << 16), w1 - __uint_as_float(upper[e] & 0xFFFF0000u));
                    }
                    tmem_store32(at + k / 2, upper);
                    tmem_store32(at + kTile / 2 + k / 2, lower);
                }
                l += (part[0] + part[1]) + (part[2] + part[3]);
                tc_wait_stores();
            }
            // The product of the tile before this one is done before this one's may start: so its weights' place is free
            // for the scores after next, and no wait is two phases of its barrier away from what it waits for.
            if (tiles > 0) ok = barrier_wait(shared_address(&c.sums), (tiles - 1) & 1, &c.failed) && ok;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(shared_address(&c.weights[buffer]));
        }
        ok = barrier_wait(shared_address(&c.sums), (tiles - 1) & 1, &c.failed) && ok;
        tc_fence_after();
        if (idle) continue;
        const bool whole = s.from == 0 && s.to == s.span.tiles;
        float* slot = slot_of<kRows, D>(p, blockIdx.x, s.from == 0);
        if (!whole && real) {
            slot[kRows * D + threadIdx.x] = m == kLowest || depth < 0 ? kLowest : offset;
            slot[kRows * D + kRows + threadIdx.x] = depth < 0 ? 0.0f : l;
        }
        const float inverse = l > 0.0f ? 1.0f / l : 0.0f;
        const bool mend = *static_cast<volatile int*>(&c.not_finite) != 0;
        T* out = reinterpret_cast<T*>(p.a.out) + (s.span.first + node) * p.a.out_row + (s.head * p.a.group + h) * p.a.out_head;
#pragma unroll
        for (int e = 0; e < D; e += 32) {
            uint32_t o[32];
            tmem_load32(tmem + S::kSums + e, o);
            tc_wait_loads();  // every lane's loads, also of lanes whose row is not real
            if (!real || e >= d) continue;
            if (mend) {  // values that were taken out
                const int* table = p.pages.table + static_cast<size_t>(s.span.row) * p.pages.row_pages;
                for (int tile = s.span.first_tile + s.from; tile < s.span.first_tile + s.to; ++tile) {
                    if (!edge_of(p, s.span, tile * kTile, kTile)) continue;
                    for (int k = 0; k < kTile; k += 32)
                        for (unsigned seen = seen_of(p, s.span, depth, nodes.mask[node], tile * kTile + k); seen != 0; seen &= seen - 1) {
                            const int t = tile * kTile + k + __ffs(seen) - 1, page = table[t / p.pages.page_tokens];
                            if (page < 0 || page >= p.pages.n_pages) continue;
                            const T* v = reinterpret_cast<const T*>(p.a.v) + page * p.a.page_stride + s.head * p.a.head_stride + t % p.pages.page_tokens * p.a.token_stride + e;
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                if (e + i >= d) continue;
                                const float x = __bfloat162float(v[i]);
                                if (!isfinite(x)) o[i] = __float_as_uint(__uint_as_float(o[i]) + x);
                            }
                        }
                }
            }
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
                if (e + i >= d) continue;
                const auto x = [&](int k) { return !ok ? NAN : depth < 0 ? 0.0f : __uint_as_float(o[i + k]); };
                if (!whole) {
                    *reinterpret_cast<float4*>(slot + threadIdx.x * D + e + i) = make_float4(x(0), x(1), x(2), x(3));
                    *reinterpret_cast<float4*>(slot + threadIdx.x * D + e + i + 4) = make_float4(x(4), x(5), x(6), x(7));
                } else {
                    *reinterpret_cast<uint4*>(out + e + i) = make_uint4(pack_bf16(x(0) * inverse, x(1) * inverse), pack_bf16(x(2) * inverse, x(3) * inverse),
                                                                        pack_bf16(x(4) * inverse, x(5) * inverse), pack_bf16(x(6) * inverse, x(7) * inverse));
                }
            }
        }
        tc_fence_before();
    }
}

template <int D, bool kExtra>
__global__ void __launch_bounds__(kThreads, 1) tree_bf16_kernel(const __grid_constant__ TreeParams p) {
    using S = Shape<D>;
    extern __shared__ char dynamic[];
    __shared__ Control c;
    __shared__ Nodes nodes;
    __shared__ long long sums[kThreads / 32], found[2];
    const int warp = threadIdx.x >> 5;
    const uint32_t queries = (shared_address(dynamic) + 1023) & ~1023u, ring = queries + S::kQueryBytes;
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kSlots; ++i) {
            barrier_init(shared_address(&c.full[i]), kCopyWarps);
            barrier_init(shared_address(&c.empty[i]), 1);
        }
        for (int i = 0; i < kScoreTiles; ++i) {
            barrier_init(shared_address(&c.scores[i]), 1);
            barrier_init(shared_address(&c.weights[i]), kSoftmaxWarps);
        }
        barrier_init(shared_address(&c.queries), kSoftmaxWarps);
        barrier_init(shared_address(&c.sums), 1);
        barrier_init(shared_address(&c.drained), 1);
        c.failed = c.not_finite = 0;
        barriers_initialized();
    }
    if (warp == kSoftmaxWarps) tmem_alloc(shared_address(&c.tmem), kColumns);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    after_previous();
    let_next_start();
    Dealer<kRows, S::kTile, kThreads> deal;
    if (deal.start(p, blockIdx.x, gridDim.x, sums, found)) {
        if (warp < kSoftmaxWarps) {
            softmax_role<D, kExtra>(p, deal, c, nodes, queries);
        } else if (warp == kSoftmaxWarps) {
            if ((threadIdx.x & 31) == 0) {
                product_role<D>(p, deal, c, queries, ring);
                if (*static_cast<volatile int*>(&c.failed)) {  // what is under way ends before tensor memory is given back
                    int late = 0;
                    tc_commit(shared_address(&c.drained));
                    barrier_wait(shared_address(&c.drained), 0, &late);
                }
            }
            __syncwarp();
        } else if (warp <= kSoftmaxWarps + kCopyWarps) {
            copy_role<D>(p, deal, c, ring);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kSoftmaxWarps) tmem_free(c.tmem, kColumns);
    write_zeros<T, kRows, S::kTile, kThreads>(p);
}

// SMs of a device, asked for once, and the kernel's share of shared memory set.
constexpr int kDevices = 64;
template <auto kKernel>
cudaError_t resident(int shared, int& ctas) {
    static std::atomic<int> known[kDevices];
    int device = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    ctas = device < kDevices ? known[device].load(std::memory_order_relaxed) : 0;
    if (ctas > 0) return cudaSuccess;
    e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e != cudaSuccess) return e;
    ctas = sms < kMaxTcCtas ? sms : kMaxTcCtas;
    if (device < kDevices) known[device].store(ctas, std::memory_order_relaxed);
    return cudaSuccess;
}

template <int D, bool kExtra>
cudaError_t launch_extra(const TreeParams& p, cudaStream_t s) {
    constexpr int slices = kRows / (128 / (D / 4));
    int ctas = 0;
    cudaError_t e = resident<tree_bf16_kernel<D, kExtra>>(Shape<D>::kShared, ctas);
    if (e != cudaSuccess) return e;
    e = launch(tree_bf16_kernel<D, kExtra>, ctas, kThreads, Shape<D>::kShared, 0, s, p);
    return e != cudaSuccess || ctas == 1 ? e : launch_join<T, D, kRows, Shape<D>::kTile>(p, ctas, slices, s);
}

template <int D>
cudaError_t launch_d(const TreeParams& p, cudaStream_t s) {
    return p.a.softcap > 0.0f || p.a.slopes != nullptr || !(p.a.scale > 0.0f) ? launch_extra<D, true>(p, s) : launch_extra<D, false>(p, s);
}

}  // namespace

uint64_t tree_workspace_bf16(int head_dim) {
    return sizeof(float) * 2ull * kMaxTcCtas * slot_floats(kRows, head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256);
}

cudaError_t launch_tree_bf16(const TreeParams& p, cudaStream_t s) {
    return p.a.head_dim <= 64 ? launch_d<64>(p, s) : p.a.head_dim <= 128 ? launch_d<128>(p, s) : launch_d<256>(p, s);
}

}  // namespace jb
