// jb_tree_bf16.cu -- jb_attend_tree on the tensor cores, for bf16 caches.
//
// A group of 128 rows (node, query head of the key head) is one tile of tcgen05.mma, and its row's keys and values pass by
// it once, 64 positions at a time:
//   S = Q K^T (fp32, tensor memory), P = exp(S - m), O = O + P V (fp32, tensor memory)
// with the maximum m of the softmax kept as it was until a row exceeds it by 2^8; only then is O multiplied. Weights enter
// the second product as two bf16 numbers, 16 bits of them.
//
// A block is one group, with two CTAs on an SM (one with heads of more than 128), or, for large trees, two groups in a CTA with
// an SM to itself, which share the tiles of keys and values and twice as many of them ahead. Roles: a warp copies keys and values
// (TMA, boxes of a page's tokens, any page size and layout) into swizzled tiles, and queries where a group is whole nodes; one
// or two warps look after values that some rows do not see, and copy queries otherwise; a warp for each group issues its
// products; four warps for each group, a thread a row, take scores from tensor memory and put weights in their place.
//
// What bounds it. Large trees: the softmax's warps, two on a scheduler. Three rows of 58000 tokens, 64 nodes by 8 query heads,
// 8 key heads of 128, capped: 549 us, issue slots 55 % used, packed fp32 units half, tensor pipes 45 % (one group a block:
// 643 us). 16 chains of 255 behind 400 to 1800 tokens, 40 heads of 128: 198 us, 24 % of the rate of plain products; a block has
// a dozen to three dozen tiles, and its first scores wait for its queries. Small trees: memory latency. 24 rows of 65 to 2000
// tokens, up to 33 nodes, 32 heads of 128: 70 us for 36 us of bytes; the tiles that fit beside the queries are two ahead.
//
// Loops are kept short: a warp that runs alone through code that is longer than its instruction cache waits for
// instructions (128 positions of a thread unrolled: 8000 cycles for as many positions). Nor is cp.async for keys and
// values: a warp issued one in 170 cycles, 10000 for 128 positions. Eight warps for a group's softmax, two threads a row, were
// no faster (757 and 741 us for the long rows): what they gain in waits they lose in registers and barriers.
#include <algorithm>
#include <numeric>

#include <cuda_bf16.h>

#include "jb_tcgen05.cuh"
#include "jb_tree.cuh"

namespace jb {
namespace {

using T = __nv_bfloat16;

constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kRows = 128, kTile = 64;  // of a product's tile
constexpr int kScoreTiles = 2;
constexpr float kSlack = 8.0f;       // how far a row may exceed its maximum before sums are scaled, in powers of two

// What a score goes through on its way to the softmax.
enum Scores { kPlain, kCapped, kBiased };  // a positive scale alone; a cap; a bias, with or without a cap, or any scale

// Heads of up to D elements, blocks of kGroups x 128 rows.
template <int D, int kGroups>
struct Shape {
    static_assert(kGroups == 1 || D <= 128);
    static constexpr int kBlock = kGroups * kRows;
    using C = Cut<kBlock, kTile, 2>;
    // Warps: of the softmax, one for each group's products, one that copies, the helpers.
    static constexpr int kSoftmaxWarps = 4 * kGroups, kHelpWarps = 3 - kGroups, kHelpThreads = 32 * kHelpWarps;
    static constexpr int kCopyWarp = kSoftmaxWarps + kGroups, kFirstHelper = 32 * (kCopyWarp + 1), kThreads = kFirstHelper + kHelpThreads;
    using Deal = Dealer<C, kThreads>;
    static constexpr int kCtas = D == 256 || kGroups == 2 ? 1 : 2;     // on an SM
    static constexpr int kSlots = D == 64 || kGroups == 2 ? 8 : 4;
    static constexpr int kQueries = D == 64 ? 2 : 1;   // blocks of queries that there is room for
    static constexpr uint32_t kTileBytes = kTile * D * 2, kQueryBytes = kRows * D * 2;  // of a group
    static constexpr uint32_t kPanel = kTile * 128, kQueryPanel = kRows * 128;  // 64 elements of all rows
    static constexpr uint32_t kSums = kScoreTiles * kTile;                      // column of a group's O
    static constexpr uint32_t kGroupColumns = D == 256 ? 512 : 256, kColumns = kGroups * kGroupColumns;  // of tensor memory
    static constexpr int kGroupsOf = kGroups;
    static __device__ __forceinline__ int groups_of(const TreeParams& p, const Piece& s) {  // of the block that have rows
        return kGroups == 1 || s.span.nodes * p.a.group - s.block * kBlock <= kRows ? 1 : 2;
    }
    static __device__ __forceinline__ uint32_t query_of(uint32_t block, uint32_t group) { return (block * kGroups + group) * kQueryBytes; }
    static constexpr int kShared = 1024 + kQueries * kGroups * kQueryBytes + kSlots * kTileBytes;
    static_assert(kSums + D <= kGroupColumns && kColumns <= 512 && kSlots % 2 == 0);  // even: values are always in odd slots
};

struct TcParams {
    TreeParams t;
    CUtensorMap keys, values;  // [pages][heads][tokens][elements]
    CUtensorMap queries;       // [nodes][heads][query heads of one][elements]
    int box;                   // groups of a box, which lie in one page
    int query_box;             // whether a block of queries is a box, too: whole nodes; else threads copy them
};

struct Control {
    unsigned long long full[8], clean[8], empty[8], edges[8], queries[2], queries_read[2], drained[2];
    unsigned long long scores[2][kScoreTiles], weights[2][kScoreTiles], sums[2];  // of each group of rows
    uint32_t tmem;
    int failed;
    // Block b's place b % 8 is b + 1 if a value in it that some rows see and others do not was not finite. A block has a tile at
    // least, and helpers are at most five tiles ahead of the softmax, as copies are.
    uint32_t not_finite[8];
    unsigned missing[8];     // groups of a tile whose page is missing; copies are at most five tiles ahead of the softmax
};

// Whether some of the positions [t, t + n) are seen by some nodes and not by others. t + n itself may leave 31 bits.
__device__ __forceinline__ bool edge_of(const TreeParams& p, const Span& s, int t, int n) {
    return s.base - t < n || (p.a.window > 0 && t < static_cast<long long>(s.base) + kMaxNodes - p.a.window);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Keys and values of the blocks' tiles, in the order in which they are needed. Lane i copies box i of a tile: `box` groups of
// 64 elements.
template <typename S, int D>
__device__ void copy_role(const TcParams& tc, typename S::Deal deal, Control& c, uint32_t queries, uint32_t ring) {
    constexpr int kGroups = kTile / kGroup, kPanels = D / 64;
    const TreeParams& p = tc.t;
    const int lane = threadIdx.x & 31, panel = lane % kPanels, group = lane / kPanels * tc.box;  // group: of the tile
    const bool mine = group < kGroups && 64 * panel < p.a.head_dim;
    const uint32_t box_bytes = tc.box * kGroup * 128;
    uint32_t copies = 0, tiles = 0, edges = 0, blocks = 0;
    const auto last = [&] {  // what is under way arrives before the role ends, whatever became of the others
        int late = 0;
        for (uint32_t k = copies < S::kSlots ? 0 : copies - S::kSlots; k < copies; ++k)
            barrier_wait(shared_address(&c.full[k % S::kSlots]), k / S::kSlots & 1, &late);
        if (tc.query_box)
            for (uint32_t k = blocks < S::kQueries ? 0 : blocks - S::kQueries; k < blocks; ++k)
                barrier_wait(shared_address(&c.queries[k % S::kQueries]), k / S::kQueries & 1, &late);
    };
    Piece s;
    while (deal.take(p, s)) {
        const int* table = p.pages.table + static_cast<size_t>(s.span.row) * p.pages.row_pages;
        const auto look_up = [&](int tile) {
            const int g = tile * kGroups + group;
            return mine && g * kGroup < s.span.len ? table[g / p.page_groups] : -1;
        };
        const int stop = s.span.first_tile + s.to;
        int page = look_up(s.span.first_tile + s.from);
        for (int tile = s.span.first_tile + s.from; tile < stop; ++tile, ++tiles) {
            const bool real = page >= 0 && page < p.pages.n_pages;
            const int y = (tile * kGroups + group) % p.page_groups * kGroup, w = page;
            const unsigned boxes = __ballot_sync(kAll, real);
            unsigned missing = 0;  // groups, from the boxes of the first panel
            for (int g = 0; g < kGroups; ++g)
                if (!(boxes >> (g / tc.box * kPanels) & 1u)) missing |= 1u << g;
            if (lane == 0) *static_cast<volatile unsigned*>(&c.missing[tiles % 8]) = missing;
            if (tile + 1 < stop) page = look_up(tile + 1);
            const uint32_t bytes = __popc(boxes) * box_bytes;
#pragma unroll 1
            for (int kind = 0; kind < 2; ++kind) {
                const uint32_t i = copies, slot = i % S::kSlots, at = ring + slot * S::kTileBytes;
                if (!__all_sync(kAll, barrier_wait(shared_address(&c.empty[slot]), (i / S::kSlots & 1) ^ 1, &c.failed))) return last();
                if (kind == 1 && missing != 0) {  // what tiles before left there is no number to meet a weight of zero
                    for (int g = 0; g < kGroups; ++g)
                        if (missing >> g & 1u)
                            for (int u = lane; u < kPanels * kGroup * 8; u += 32)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + u / (kGroup * 8) * S::kPanel + g * (kGroup * 128) + u % (kGroup * 8) * 16), "r"(0)
                                             : "memory");
                    shared_to_async_proxy();
                }
                __syncwarp();
                if (lane == 0) {
                    barrier_arrive_bytes(shared_address(&c.full[slot]), bytes);
                    if (kind == 1) {
                        if (edge_of(p, s.span, tile * kTile, kTile)) barrier_arrive(shared_address(&c.edges[edges++ % 8]));
                        else barrier_arrive_count(shared_address(&c.clean[slot]), S::kHelpWarps);
                    }
                }
                __syncwarp();
                if (real) copy_box(at + panel * S::kPanel + group * (kGroup * 128), kind == 0 ? &tc.keys : &tc.values, 64 * panel, y, s.head, w, shared_address(&c.full[slot]));
                ++copies;
                if (tc.query_box && kind == 0 && tile == s.span.first_tile + s.from) {
                    const uint32_t b = blocks % S::kQueries;
                    if (!__all_sync(kAll, barrier_wait(shared_address(&c.queries_read[b]), (blocks / S::kQueries & 1) ^ 1, &c.failed))) return last();
                    const int groups = S::groups_of(p, s), g = lane / kPanels, x = 64 * (lane % kPanels);
                    if (lane == 0) barrier_arrive_bytes(shared_address(&c.queries[b]), groups * ((p.a.head_dim + 63) / 64) * S::kQueryPanel);
                    __syncwarp();
                    if (g < groups && x < p.a.head_dim)
                        copy_box(queries + S::query_of(b, g) + x / 64 * S::kQueryPanel, &tc.queries, x, 0, s.head,
                                 s.span.first + (s.block * S::kGroupsOf + g) * (kRows / p.a.group), shared_address(&c.queries[b]));
                    ++blocks;
                }
            }
        }
    }
    last();
}

// 128 rows of queries from row `first` of the tree's on, by all helpers. Rows that are not real stay what they were: their results go nowhere.
template <typename S, int D>
__device__ void copy_queries(const TreeParams& p, const Piece& s, int first, uint32_t to) {
    constexpr int kPieces = D / 8, kStep = S::kHelpThreads / kPieces;
    const int u = threadIdx.x - S::kFirstHelper, piece = u % kPieces, row0 = u / kPieces, rows = s.span.nodes * p.a.group;
    const int rows_here = min(kRows, rows - first);
    int all = first + row0, node = all / p.a.group, h = all - node * p.a.group;
    const T* from = reinterpret_cast<const T*>(p.a.q) + s.span.first * p.a.q_row + static_cast<uint64_t>(s.head) * p.a.group * p.a.q_head + 8 * piece;
    const bool held = 8 * piece < p.a.head_dim;
    constexpr int kAhead = 8;
    static_assert(kRows % (kAhead * kStep) == 0);
#pragma unroll 1
    for (int row = row0; row < rows_here; row += kAhead * kStep) {
        uint4 x[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            x[k] = held && all < rows ? *reinterpret_cast<const uint4*>(from + node * p.a.q_row + h * p.a.q_head) : make_uint4(0, 0, 0, 0);
            all += kStep;
            for (h += kStep; h >= p.a.group; h -= p.a.group) ++node;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int r = row + k * kStep;
            const uint32_t at = to + static_cast<uint32_t>(piece >> 3) * S::kQueryPanel + r * 128 + (((piece & 7) ^ (r & 7)) << 4);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x[k].x), "r"(x[k].y), "r"(x[k].z), "r"(x[k].w) : "memory");
        }
    }
}

// A value that is not finite must not meet a weight of zero: it is taken out here and added at the end to the rows that see
// it. So are the rows outside [lo, hi), which nobody sees. True if there was one inside. Panels that heads of `d` elements do not
// reach are not copied and hold anything: a pattern found there sent every later block of the CTA through put_back (8 chains of
// 255, 4 heads of 192: 2930 us, with zeros there 54).
template <typename S, int D>
__device__ bool clean_values(uint32_t tile, int d, int lo, int hi) {
    const int u = threadIdx.x - S::kFirstHelper, pieces = (D == 256 ? (d + 63) / 64 : D / 64) * (kTile * 8);
    constexpr int kAhead = S::kHelpWarps == 1 ? 8 : 2;
    static_assert(kTile * 8 % (kAhead * S::kHelpThreads) == 0);
    bool bad = false;
#pragma unroll 1
    for (int i = u; i < pieces; i += kAhead * S::kHelpThreads) {
        uint32_t w[kAhead][4];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[k][0]), "=r"(w[k][1]), "=r"(w[k][2]), "=r"(w[k][3]) : "r"(tile + (i + k * S::kHelpThreads) * 16) : "memory");
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int at = i + k * S::kHelpThreads, row = at / 8 % kTile;
            const bool inside = row >= lo && row < hi;
            uint32_t any = 0;  // an exponent of ones carries over into the sign's place
#pragma unroll
            for (int e = 0; e < 4; ++e) any |= (w[k][e] & 0x7F807F80u) + 0x00800080u;
            any &= 0x80008000u;
            if (any == 0 && inside) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t mask = ((w[k][e] & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((w[k][e] & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
                w[k][e] = inside ? w[k][e] & ~mask : 0;
            }
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(tile + at * 16), "r"(w[k][0]), "r"(w[k][1]), "r"(w[k][2]), "r"(w[k][3]) : "memory");
            bad = bad || inside;
        }
    }
    return bad;
}

template <typename S, int D>
__device__ void help_role(const TcParams& tc, typename S::Deal deal, Control& c, uint32_t queries, uint32_t ring) {
    const TreeParams& p = tc.t;
    const int lane = threadIdx.x & 31;
    uint32_t blocks = 0, done = 0, tiles = 0, edges = 0;
    const auto tell = [&](unsigned long long* bar) {
        shared_to_async_proxy();
        __syncwarp();
        if (lane == 0) barrier_arrive(shared_address(bar));
    };
    const auto block = [&](const Piece& s) {
        if (tc.query_box) return true;
        const uint32_t b = blocks % S::kQueries;
        if (!__all_sync(kAll, barrier_wait(shared_address(&c.queries_read[b]), (blocks / S::kQueries & 1) ^ 1, &c.failed))) return false;
        ++blocks;
        for (int g = 0; g < S::groups_of(p, s); ++g) copy_queries<S, D>(p, s, s.block * S::kBlock + g * kRows, queries + S::query_of(b, g));
        tell(&c.queries[b]);
        return true;
    };
    Piece s, next;
    bool more = deal.take(p, s);
    if (more && !block(s)) return;
    while (more) {
        more = deal.take(p, next);
        if (S::kQueries > 1 && more && !block(next)) return;
        for (int tile = s.span.first_tile + s.from; tile < s.span.first_tile + s.to; ++tile, ++tiles) {
            if (!edge_of(p, s.span, tile * kTile, kTile)) continue;
            const uint32_t i = 2 * tiles + 1, slot = i % S::kSlots, e = edges++;
            // first that its copy has begun: the slot's own phase may be any before that
            if (!__all_sync(kAll, barrier_wait_idle(shared_address(&c.edges[e % 8]), e / 8 & 1, &c.failed))) return;
            if (!__all_sync(kAll, barrier_wait(shared_address(&c.full[slot]), i / S::kSlots & 1, &c.failed))) return;
            if (clean_values<S, D>(ring + slot * S::kTileBytes, p.a.head_dim, s.span.lo - tile * kTile, s.span.len - tile * kTile))
                *static_cast<volatile uint32_t*>(&c.not_finite[done % 8]) = done + 1;
            tell(&c.clean[slot]);
        }
        ++done;
        // with room for one block of queries the next can come only when this one has been read to its end
        if (S::kQueries == 1 && more && !block(next)) return;
        s = next;
    }
}

// Products of group g's rows.
template <typename S, int D>
__device__ void product_role(const TreeParams& p, typename S::Deal deal, Control& c, int g, uint32_t queries, uint32_t ring) {
    const int steps = (p.a.head_dim + 15) / 16;
    constexpr uint32_t scores = product_descriptor(kTile, false);
    constexpr bool kDeep = S::kSlots >= 8;
    const uint32_t values = product_descriptor(16 * steps, true);
    const uint32_t tmem = same(c.tmem) + g * S::kGroupColumns;
    uint32_t tiles = 0, mine = 0;  // so far; mine: of those that the group has rows for
    // The whole warp runs this and one lane issues: operands are then the warp's, which products want them to be.
    const auto wait = [&](unsigned long long* bar, uint32_t parity) {
        const bool ok = __all_sync(kAll, barrier_wait(shared_address(bar), parity, &c.failed));
        tc_fence_after();
        return ok;
    };
    const auto came = [&](uint32_t copy) { return wait(&c.full[copy % S::kSlots], copy / S::kSlots & 1); };
    Piece s;
    for (uint32_t blocks = 0; same(static_cast<int>(deal.take(p, s))) != 0; ++blocks) {
        const uint32_t n = same(s.to - s.from), b = blocks % S::kQueries;
        if (!wait(&c.queries[b], blocks / S::kQueries & 1)) return;
        if (g >= same(S::groups_of(p, s))) {  // nothing to do, which the copies have to know
            for (uint32_t copy = 2 * tiles; copy < 2 * (tiles + n); ++copy) {
                if (!came(copy)) return;
                if (elected()) barrier_arrive(shared_address(&c.empty[copy % S::kSlots]));
                __syncwarp();
            }
            if (elected()) barrier_arrive(shared_address(&c.queries_read[b]));
            __syncwarp();
            tiles += n;
            continue;
        }
        const uint32_t q = tile_descriptor(queries + S::query_of(b, g), 16);
        const auto scores_of = [&](uint32_t tile, bool last) {  // of the block's tile
            const uint32_t slot = 2 * (tiles + tile) % S::kSlots, k = tile_descriptor(ring + slot * S::kTileBytes, 16), buffer = (mine + tile) % kScoreTiles;
            if (elected()) {
#pragma unroll
                for (int e = 0; e < D / 16; ++e)
                    if (e < steps)
                        tc_product(tmem + buffer * kTile, q + ((e / 4 * S::kQueryPanel + e % 4 * 32) >> 4), k + ((e / 4 * S::kPanel + e % 4 * 32) >> 4), scores, e > 0);
                tc_commit(shared_address(&c.empty[slot]));
                tc_commit(shared_address(&c.scores[g][buffer]));
                if (last) tc_commit(shared_address(&c.queries_read[b]));
            }
            __syncwarp();
        };
        // A tile's scores take the place of the weights of two tiles before, whose product has to be done. That of a block's
        // first tile is, for the weights after them were given later than it ended.
        if (!came(2 * tiles)) return;
        scores_of(0, n == 1);
        if (n > 1) {
            if (!came(2 * (tiles + 1)) || (mine > 0 && !wait(&c.sums[g], (mine - 1) & 1))) return;
            scores_of(1, n == 2);
        }
        for (uint32_t j = 0; j < n; ++j) {
            const uint32_t i = 2 * (tiles + j) + 1, slot = i % S::kSlots, turn = mine + j, buffer = turn % kScoreTiles;
            // What has come by now is looked at before the weights, from which on every look counts; with few slots keys have not
            if (!came(i) || !wait(&c.clean[slot], i / S::kSlots & 1)) return;
            if (kDeep && j + 2 < n && !came(i + 3)) return;
            if (!wait(&c.weights[g][buffer], turn / kScoreTiles & 1)) return;
            const uint32_t v = tile_descriptor(ring + slot * S::kTileBytes, S::kPanel), w = tmem + buffer * kTile;
            if (elected()) {
#pragma unroll
                for (int half = 0; half < 2; ++half)  // the weights' upper and lower bits
#pragma unroll
                    for (int e = 0; e < kTile / 16; ++e)
                        tc_product_from_tmem(tmem + S::kSums, w + e * 16 + half * 8, v + (e * 2048 >> 4), values, half > 0 || e > 0 || j > 0);
                tc_commit(shared_address(&c.empty[slot]));
                tc_commit(shared_address(&c.sums[g]));
            }
            __syncwarp();
            if (j + 2 < n) {
                if ((!kDeep && !came(i + 3)) || !wait(&c.sums[g], turn & 1)) return;
                scores_of(j + 2, j + 3 == n);
            }
        }
        tiles += n;
        mine += n;
    }
}

// A barrier of the softmax warps, true if x is in one of their threads.
template <int kSoftmaxWarps>
__device__ __forceinline__ bool any_of(bool x) {
    uint32_t any;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.or.pred p, 1, %2, q;\n selp.u32 %0, 1, 0, p;\n}"
                 : "=r"(any) : "r"(static_cast<uint32_t>(x)), "n"(32 * kSoftmaxWarps) : "memory");
    return any != 0;
}

// Adds to o, 32 elements of a row's sums from element e on, the values that were taken out and that the row sees.
__device__ __noinline__ void put_back(const TreeParams& p, const Piece& s, const Nodes& nodes, int node, int depth, int e, uint32_t* o) {
    const int* table = p.pages.table + static_cast<size_t>(s.span.row) * p.pages.row_pages;
    for (int tile = s.span.first_tile + s.from; tile < s.span.first_tile + s.to; ++tile) {
        if (!edge_of(p, s.span, tile * kTile, kTile)) continue;
        for (int k = 0; k < kTile; k += 32)
            for (unsigned seen = seen_of(p, s.span, nodes, node, depth, tile * kTile + k); seen != 0; seen &= seen - 1) {
                const int t = tile * kTile + k + __ffs(seen) - 1, page = table[t / p.pages.page_tokens];
                if (page < 0 || page >= p.pages.n_pages) continue;
                const T* v = reinterpret_cast<const T*>(p.a.v) + page * p.a.page_stride + s.head * p.a.head_stride + t % p.pages.page_tokens * p.a.token_stride + e;
                for (int i = 0; i < 32 && e + i < p.a.head_dim; ++i) {
                    const float x = __bfloat162float(v[i]);
                    if (!isfinite(x)) o[i] = __float_as_uint(__uint_as_float(o[i]) + x);
                }
            }
    }
}

// What the softmax's warps work on, held for all of them in shared memory: their registers are for scores.
template <typename Deal>
struct Work {
    Deal deal;
    Piece piece;
    int more;
    uint32_t blocks;  // so far, the piece's among them
};

template <typename S, int D, Scores kScores>
__device__ void softmax_role(const TreeParams& p, Control& c, Work<typename S::Deal>& work, Nodes& nodes) {
    using C = typename S::C;
    // Whether a tile's scores stay in registers from one pass to the next. Where a cap is put on them between the passes that
    // pays (729 -> 636 us for three rows of 58000 tokens), and without one a short loop that takes them from tensor memory
    // twice does (78 us and not 84 for 24 ragged rows).
    constexpr bool kHeld = kScores == kCapped;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = warp / 4, row = threadIdx.x, d = p.a.head_dim;
    const uint32_t tmem = c.tmem + g * S::kGroupColumns + (static_cast<uint32_t>(32 * (warp % 4)) << 16);
    const float by = kScores == kPlain ? p.a.scale * kLog2e : 1.0f;
    uint32_t tiles = 0, mine = 0;  // so far; mine: of those that the group has rows for
    int tree = -1;
    bool ok = true;  // a wait that gives up leaves the loops as they are: other warps may wait for this one
    const Piece& s = work.piece;
    for (;;) {
        any_of<S::kSoftmaxWarps>(false);  // nobody reads the last piece any more
        if (threadIdx.x == 0) {
            work.more = work.deal.take(p, work.piece);
            ++work.blocks;
        }
        any_of<S::kSoftmaxWarps>(false);
        if (work.more == 0) break;
        if (s.tree != tree) fill_nodes<32 * S::kSoftmaxWarps>(p, s.span, nodes, threadIdx.x, any_of<S::kSoftmaxWarps>);
        tree = s.tree;
        const int rows = s.span.nodes * p.a.group, all = s.block * S::kBlock + row;
        if (threadIdx.x == 0 && s.from == 0 && s.to != s.span.tiles) take_note(p, {s.span.first, s.head, s.block, work.deal.last_of(s), rows, {}});
        if (g >= S::groups_of(p, s)) {
            tiles += s.to - s.from;
            continue;
        }
        const bool real = all < rows, idle = s.block * S::kBlock + 32 * warp >= rows;  // idle: none of the warp's rows is real
        const int node = real ? all / p.a.group : 0, h = real ? all - node * p.a.group : 0, depth = real ? nodes.depth[node] : -1;
        const float slope = kScores == kBiased && real && p.a.slopes != nullptr ? p.a.slopes[s.head * p.a.group + h] * kLog2e : 0.0f;
        // m: the largest score, in kPlain before the scale, which may bring anything finite into range; after it what is not
        // above kLowest counts as infinite. offset: what is subtracted from scores, in powers of two; 0 before one is seen
        float m = -INFINITY, offset = 0.0f, l = 0.0f;
        for (int tile = s.span.first_tile + s.from; tile < s.span.first_tile + s.to; ++tile, ++tiles, ++mine) {
            const int t0 = tile * kTile;
            const uint32_t buffer = mine % kScoreTiles, at = tmem + buffer * kTile;
            ok = barrier_wait(shared_address(&c.scores[g][buffer]), mine / kScoreTiles & 1, &c.failed) && ok;
            tc_fence_after();
            if (!idle) {
                const unsigned missing = *static_cast<volatile unsigned*>(&c.missing[tiles % 8]);
                const bool edge = missing != 0 || edge_of(p, s.span, t0, kTile);
                float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                const auto seen_at = [&](int i) {  // of 32 positions
                    unsigned seen = seen_of(p, s.span, nodes, node, depth, t0 + 32 * i);
                    if (missing >> (2 * i) & 1u) seen &= 0xFFFF0000u;
                    if (missing >> (2 * i + 1) & 1u) seen &= 0x0000FFFFu;
                    return seen;
                };
                uint32_t x[kHeld ? kTile : 1];
                if constexpr (kHeld) {
#pragma unroll
                    for (int k = 0; k < kTile; k += 32) tmem_load32(at + k, x + k);
                    tc_wait_loads();
                    float most[2] = {};
#pragma unroll
                    for (int k = 0; k < kTile; ++k) most[k & 1] = fmaxf(most[k & 1], fabsf(__uint_as_float(x[k])));
                    if (__all_sync(kAll, fmaxf(most[0], most[1]) * fabsf(p.cap_in) < kSmallCap)) {
#pragma unroll
                        for (int k = 0; k < kTile; k += 2) {
                            const float2 y = capped_small(p, make_float2(__uint_as_float(x[k]), __uint_as_float(x[k + 1])));
                            x[k] = __float_as_uint(y.x);
                            x[k + 1] = __float_as_uint(y.y);
                        }
                    } else {
#pragma unroll 1
                        for (int k = 0; k < kTile; k += 16) {
                            uint32_t raw[16];
                            tmem_load16(at + k, raw);
                            tc_wait_loads();
#pragma unroll
                            for (int e = 0; e < 16; ++e) raw[e] = __float_as_uint(capped(p, __uint_as_float(raw[e])));
                            tmem_store16(at + k, raw);
                        }
                        tc_wait_stores();
#pragma unroll
                        for (int k = 0; k < kTile; k += 32) tmem_load32(at + k, x + k);
                        tc_wait_loads();
                    }
                    if (edge) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const unsigned seen = seen_at(i);
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!(seen >> e & 1u)) x[32 * i + e] = __float_as_uint(-INFINITY);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < kTile; ++k) tops[k % 4] = fmaxf(tops[k % 4], __uint_as_float(x[k]));
                } else if (kScores == kBiased || edge) {  // scores are put back as the softmax takes them
                    unsigned seen[2] = {kAll, kAll};
                    if (edge) seen[0] = seen_at(0), seen[1] = seen_at(1);
                    uint32_t raw[16];
                    tmem_load16(at, raw);
#pragma unroll 1
                    for (int k = 0; k < kTile; k += 16) {
                        const unsigned sees = seen[k >> 5] >> (k & 16);
                        uint32_t y[16];
                        tc_wait_loads();
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            y[e] = raw[e];
                            if constexpr (kScores == kBiased) {
                                const int t = t0 + k + e;
                                int back = t - s.span.base - depth;
                                if (t >= s.span.base && (sees >> e & 1u)) back = nodes.depth[t - s.span.base] - depth;
                                y[e] = __float_as_uint(score<true>(p, __uint_as_float(raw[e]), slope, back));
                            }
                        }
                        if (k + 16 < kTile) tmem_load16(at + k + 16, raw);
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            if (!(sees >> e & 1u)) y[e] = __float_as_uint(-INFINITY);
                            tops[e % 4] = fmaxf(tops[e % 4], __uint_as_float(y[e]));
                        }
                        tmem_store16(at + k, y);
                    }
                    tc_wait_stores();
                } else {
                    uint32_t raw[kTile];
#pragma unroll
                    for (int k = 0; k < kTile; k += 32) tmem_load32(at + k, raw + k);
                    tc_wait_loads();
#pragma unroll
                    for (int k = 0; k < kTile; ++k) tops[k % 4] = fmaxf(tops[k % 4], __uint_as_float(raw[k]));
                }
                const float high = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
                const float top = high * by;
                const bool rises = high > m && top > kLowest && (m == -INFINITY || (high - m) * by > kSlack);
                if (__any_sync(kAll, rises)) {
                    float k = 1.0f;
                    if (rises) {
                        k = m == -INFINITY ? 0.0f : exp2_approx(offset - top);
                        m = high;
                        offset = top;
                        l *= k;
                    }
                    if (tile != s.span.first_tile + s.from) {
                        ok = barrier_wait(shared_address(&c.sums[g]), (mine - 1) & 1, &c.failed) && ok;
                        tc_fence_after();
#pragma unroll 1
                        for (int e = 0; e < D; e += 16) {
                            uint32_t o[16];
                            tmem_load16(tmem + S::kSums + e, o);
                            tc_wait_loads();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * k);
                            tmem_store16(tmem + S::kSums + e, o);
                        }
                    }
                }
                float2 part[2] = {};
                const float2 by2 = make_float2(by, by), less = make_float2(-offset, -offset);
                // 16 scores to the upper bits of their weights, then the lower ones
                const auto weights_of = [&](const uint32_t* score, uint32_t to) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float2 y = __ffma2_rn(make_float2(__uint_as_float(score[2 * e]), __uint_as_float(score[2 * e + 1])), by2, less);
                        y.x = exp2_approx(y.x);
                        y.y = exp2_approx(y.y);
                        part[e & 1] = __fadd2_rn(part[e & 1], y);
                        w[e] = pack_bf16(y.x, y.y);
                        const float2 rest = __fadd2_rn(y, make_float2(-__uint_as_float(w[e] << 16), -__uint_as_float(w[e] & 0xFFFF0000u)));
                        w[8 + e] = pack_bf16(rest.x, rest.y);
                    }
                    tmem_store16(to, w);
                };
                if constexpr (kHeld) {
#pragma unroll
                    for (int k = 0; k < kTile; k += 16) weights_of(x + k, at + k);
                } else {
                    uint32_t raw[16];
                    tmem_load16(at, raw);
#pragma unroll 1
                    for (int k = 0; k < kTile; k += 16) {
                        uint32_t now[16];
                        tc_wait_loads();
#pragma unroll
                        for (int e = 0; e < 16; ++e) now[e] = raw[e];
                        if (k + 16 < kTile) tmem_load16(at + k + 16, raw);
                        weights_of(now, at + k);
                    }
                }
                l += (part[0].x + part[0].y) + (part[1].x + part[1].y);
                tc_wait_stores();
            }
            // The product of the tile before this one is done before this one's may start: so no wait is two phases of
            // its barrier away from what it waits for.
            if (mine > 0) ok = barrier_wait(shared_address(&c.sums[g]), (mine - 1) & 1, &c.failed) && ok;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(shared_address(&c.weights[g][buffer]));
        }
        const bool whole = s.from == 0 && s.to == s.span.tiles;
        ok = barrier_wait(shared_address(&c.sums[g]), (mine - 1) & 1, &c.failed) && ok;
        tc_fence_after();
        if (idle) continue;
        float* slot = slot_of<C, D>(p, gridDim.x, blockIdx.x, s.from == 0);
        if (!whole && real) {
            slot[S::kBlock * D + row] = m == -INFINITY || depth < 0 ? kLowest : offset;
            slot[S::kBlock * D + S::kBlock + row] = depth < 0 ? 0.0f : l;
        }
        const float inverse = l > 0.0f ? 1.0f / l : 0.0f;
        const uint32_t blocks = work.blocks;
        const bool mend = *static_cast<volatile uint32_t*>(&c.not_finite[(blocks - 1) % 8]) == blocks;
        T* out = reinterpret_cast<T*>(p.a.out) + (s.span.first + node) * p.a.out_row + (s.head * p.a.group + h) * p.a.out_head;
#pragma unroll 1
        for (int e = 0; e < D; e += 32) {
            uint32_t o[32];
            tmem_load32(tmem + S::kSums + e, o);
            tc_wait_loads();  // every lane's loads, also of lanes whose row is not real
            if (!real || e >= d) continue;
            if (mend) {
                uint32_t copy[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) copy[i] = o[i];
                put_back(p, s, nodes, node, depth, e, copy);
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = copy[i];
            }
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
                if (e + i >= d) continue;
                const auto x = [&](int k) { return !ok ? NAN : depth < 0 ? 0.0f : __uint_as_float(o[i + k]); };
                if (!whole) {
                    *reinterpret_cast<float4*>(slot + row * D + e + i) = make_float4(x(0), x(1), x(2), x(3));
                    *reinterpret_cast<float4*>(slot + row * D + e + i + 4) = make_float4(x(4), x(5), x(6), x(7));
                } else {
                    *reinterpret_cast<uint4*>(out + e + i) = make_uint4(pack_bf16(x(0) * inverse, x(1) * inverse), pack_bf16(x(2) * inverse, x(3) * inverse),
                                                                        pack_bf16(x(4) * inverse, x(5) * inverse), pack_bf16(x(6) * inverse, x(7) * inverse));
                }
            }
        }
        tc_fence_before();
    }
}

template <int D, int kGroups, Scores kScores>
__global__ void __launch_bounds__(Shape<D, kGroups>::kThreads, Shape<D, kGroups>::kCtas) tree_bf16_kernel(const __grid_constant__ TcParams tc) {
    using S = Shape<D, kGroups>;
    constexpr int kThreads = S::kThreads, kSoftmaxWarps = S::kSoftmaxWarps;
    const TreeParams& p = tc.t;
    extern __shared__ char dynamic[];
    __shared__ Control c;
    __shared__ Nodes nodes;
    __shared__ Work<typename S::Deal> work;
    __shared__ long long sums[kThreads / 32], found[2];
    const int warp = same(static_cast<int>(threadIdx.x) >> 5);
    const uint32_t queries = (shared_address(dynamic) + 1023) & ~1023u, ring = queries + S::kQueries * kGroups * S::kQueryBytes;
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kSlots; ++i) {
            barrier_init(shared_address(&c.full[i]), 1);
            barrier_init(shared_address(&c.clean[i]), S::kHelpWarps);
            barrier_init(shared_address(&c.empty[i]), kGroups);
        }
        for (int i = 0; i < 8; ++i) {
            barrier_init(shared_address(&c.edges[i]), 1);
            c.not_finite[i] = 0;
        }
        for (int g = 0; g < kGroups; ++g) {
            for (int i = 0; i < kScoreTiles; ++i) {
                barrier_init(shared_address(&c.scores[g][i]), 1);
                barrier_init(shared_address(&c.weights[g][i]), 4);
            }
            barrier_init(shared_address(&c.sums[g]), 1);
            barrier_init(shared_address(&c.drained[g]), 1);
        }
        for (int i = 0; i < S::kQueries; ++i) {
            barrier_init(shared_address(&c.queries[i]), tc.query_box ? 1 : S::kHelpWarps);
            barrier_init(shared_address(&c.queries_read[i]), kGroups);
        }
        c.failed = 0;
        barriers_initialized();
    }
    if (warp == kSoftmaxWarps) tmem_alloc(shared_address(&c.tmem), S::kColumns);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    after_previous();
    let_next_start();
    typename S::Deal deal;
    if (deal.start(p, blockIdx.x, gridDim.x, sums, found)) {
        if (warp < kSoftmaxWarps) {
            if (threadIdx.x == 0) {
                take_note(p, {});
                work.deal = deal;
                work.blocks = 0;
            }
            softmax_role<S, D, kScores>(p, c, work, nodes);
        } else if (warp < S::kCopyWarp) {
            const int g = warp - kSoftmaxWarps;
            product_role<S, D>(p, deal, c, g, queries, ring);
            // what is under way ends before tensor memory is given back
            if (__any_sync(kAll, *static_cast<volatile int*>(&c.failed) != 0)) tc_drain(shared_address(&c.drained[g]));
        } else if (warp == S::kCopyWarp) {
            copy_role<S, D>(tc, deal, c, queries, ring);
        } else {
            help_role<S, D>(tc, deal, c, queries, ring);
        }
    } else if (threadIdx.x == 0) {
        take_note(p, {});
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kSoftmaxWarps) tmem_free(c.tmem, S::kColumns);
    write_zeros<T, typename S::C, kThreads>(p);
}

template <int D, int kGroups>
constexpr int max_ctas() { return 160 * Shape<D, kGroups>::kCtas; }

// Queries in blocks of whole nodes: false where a block is none, or strides are none of a box (one query for all nodes, say).
bool describe_queries(Encode encode, CUtensorMap& map, const TreeParams& p) {
    if (kRows % p.a.group != 0 || p.a.q_head == 0 || p.a.q_row == 0) return false;
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(p.a.head_dim), static_cast<cuuint64_t>(p.a.group), static_cast<cuuint64_t>(p.a.heads),
                                static_cast<cuuint64_t>(p.trees.n_nodes)};
    const cuuint64_t strides[3] = {p.a.q_head * sizeof(T), p.a.q_head * p.a.group * sizeof(T), p.a.q_row * sizeof(T)};
    const cuuint32_t boxes[4] = {64, static_cast<cuuint32_t>(p.a.group), 1, static_cast<cuuint32_t>(kRows / p.a.group)};
    return encoded(encode, map, p.a.q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, dims, strides, boxes);
}

template <int D, int kGroups, Scores kScores>
cudaError_t launch_scores(const TreeParams& p, cudaStream_t s) {
    using S = Shape<D, kGroups>;
    int ctas = 0;
    cudaError_t e = resident<tree_bf16_kernel<D, kGroups, kScores>>(S::kShared, S::kCtas, max_ctas<D, kGroups>(), ctas);
    if (e != cudaSuccess) return e;
    TcParams tc;
    tc.t = p;
    tc.box = std::gcd(p.page_groups, kTile / kGroup);
    Encode encode = nullptr;
    e = encoder(encode);
    if (e == cudaSuccess) e = describe_pool(encode, tc.keys, p, p.a.k, tc.box, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, sizeof(T));
    if (e == cudaSuccess) e = describe_pool(encode, tc.values, p, p.a.v, tc.box, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, sizeof(T));
    if (e == cudaSuccess) tc.query_box = describe_queries(encode, tc.queries, p);
    if (e == cudaSuccess) e = launch(tree_bf16_kernel<D, kGroups, kScores>, ctas, S::kThreads, S::kShared, 0, s, tc);
    return e != cudaSuccess || ctas == 1 ? e : launch_join<T, D, typename S::C>(p, ctas, s);
}

template <int D, int kGroups>
cudaError_t launch_groups(const TreeParams& p, cudaStream_t s) {
    if (p.a.slopes != nullptr || (p.a.softcap == 0.0f && !(p.a.scale > 0.0f))) return launch_scores<D, kGroups, kBiased>(p, s);
    return p.a.softcap > 0.0f ? launch_scores<D, kGroups, kCapped>(p, s) : launch_scores<D, kGroups, kPlain>(p, s);
}

template <int D>
cudaError_t launch_d(const TreeParams& p, cudaStream_t s) {
    // Two groups where trees have more than one's rows on average. Measured with 16 rows of 400 to 1800 tokens, 40 heads of 128,
    // one group and two in us: chains of 127 105 and 145, of 129 164 and 154, of 192 182 and 171, of 256 201 and 198.
    if constexpr (D <= 128)
        if (static_cast<long long>(p.trees.n_nodes) * p.a.group > static_cast<long long>(kRows) * p.trees.n) return launch_groups<D, 2>(p, s);
    return launch_groups<D, 1>(p, s);
}

template <int D, int kGroups>
constexpr size_t floats_of() { return workspace_floats(max_ctas<D, kGroups>(), Shape<D, kGroups>::kBlock, D); }

}  // namespace

uint64_t tree_workspace_bf16(int head_dim) {
    const size_t floats = head_dim <= 64    ? std::max(floats_of<64, 1>(), floats_of<64, 2>())
                          : head_dim <= 128 ? std::max(floats_of<128, 1>(), floats_of<128, 2>())
                                            : floats_of<256, 1>();
    return sizeof(float) * floats;
}

cudaError_t launch_tree_bf16(const TreeParams& p, cudaStream_t s) {
    return p.a.head_dim <= 64 ? launch_d<64>(p, s) : p.a.head_dim <= 128 ? launch_d<128>(p, s) : launch_d<256>(p, s);
}

}  // namespace jb
