// jb_sample.cu -- the next token of each row from its logits and a random word.
//
// Weights are integers (w = rint(2^30 exp(y))), so a sum of them is the same in every order and the
// token is a function of the logits' bits, the settings and the word alone. What is kept is a prefix
// of the order (logit descending, index ascending). Its end is found without sorting: a histogram over
// y of counts and weights gives the bin that holds the end, the bin's tokens are collected and ranked.
// A bin with too many tokens is cut again, by key and at last by index, until they fit.
//
// A row is one cluster of CTAs that read it from L2 in each of their few passes (a batch of logits is
// smaller than L2); histograms and sums are joined through distributed shared memory.
//
// What bounds it is not the bytes: for few rows a chain of a dozen barriers (one fp32 row of 50272 tokens: 8 us
// without filters, 14 with top-k or with all filters, 18 with top-p), for many the instructions, about 90 for each
// token (256 bf16 rows: 20 us without filters, 33 with top-k, 67 with top-p: 15 of them the exponentials and
// shared-memory additions of the histogram, 9 the sum of what is kept, 7 the search for the bin's tokens; 45
// where top-p keeps few tokens, whose list serves the rest of the draw).
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "jb_answer.h"
#include "jb_launch.cuh"

namespace jb {
namespace {

namespace cg = cooperative_groups;

constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kIndexBins = 1024;       // bins of an index, 2^18 tokens at most
constexpr int kMaxCluster = 8;
constexpr int kSms = 152;
constexpr int kResident = 1024;        // threads on an SM: 64 registers each (4 bytes spilled); 1536 and 2048 are slower
constexpr int kMaxSlice = 65536;       // tokens of one CTA: sums of halves of their weights fit 32 bits
constexpr int kLarge = 512;            // threads of a CTA, 256 for small vocabularies
constexpr int kSmallVocab = 8192;
constexpr int kSteps = 16;             // of 32 units, that a warp's part of a slice has at most
constexpr float kReach = 21.5f;        // weights round to 0 below y = -31 ln 2 = -21.49
constexpr float kOne = 1073741824.0f;  // 2^30, the weight of the largest logit
typedef unsigned long long u64;

// Logits as unsigned keys in the same order; 0 and -0 are one, NaN goes below -inf.
__device__ __forceinline__ uint32_t key_of(float l) {
    if (l != l) return 0;
    const uint32_t b = __float_as_uint(l + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t kNothing = 0x007FFFFFu;  // key of -inf; nothing at or below it is drawn

__device__ __forceinline__ float logit_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}

// Eight logits at a time; NaN past the end. In a row whose largest logit is +inf those stand for 0 and all
// others for -inf.
constexpr int kUnit = 8;
template <typename T>
__device__ __forceinline__ void load_unit(const T* row, int j, int vocab, bool wide, bool infinite, float (&x)[kUnit]) {
    if (wide && j + kUnit <= vocab) {
        if constexpr (sizeof(T) == 2) {
            const uint4 v = *reinterpret_cast<const uint4*>(row + j);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < kUnit; ++i) x[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
        } else {
            const float4 a = *reinterpret_cast<const float4*>(row + j), b = *reinterpret_cast<const float4*>(row + j + 4);
            x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kUnit; ++i) x[i] = j + i < vocab ? static_cast<float>(row[j + i]) : NAN;
    }
    if (infinite) {
#pragma unroll
        for (int i = 0; i < kUnit; ++i) x[i] = x[i] == INFINITY ? 0.0f : -INFINITY;
    }
}

struct Row {
    float top;      // the largest logit
    float inverse;  // 1 / temperature

    // NaN stays NaN, and weighs 0
    __device__ float scaled(float x) const { return (x - top) * inverse; }
    __device__ static uint32_t weight_of(float y) { return __float2uint_rn(expf(y) * kOne); }
    __device__ uint32_t weight(float x) const { return weight_of(scaled(x)); }
};

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

// Exclusive prefix over the CTA's threads and the total. sums: a word for each of kWarps warps.
template <int kWarps, typename V>
__device__ __forceinline__ V block_exclusive(V v, V* sums, V& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const V in = warp_inclusive(v);
    if (lane == 31) sums[warp] = in;
    __syncthreads();
    const V all = warp_inclusive(lane < kWarps ? sums[lane] : V(0));
    const V before = __shfl_sync(kAll, all, warp == 0 ? 0 : warp - 1);
    total = __shfl_sync(kAll, all, 31);
    __syncthreads();
    return in - v + (warp == 0 ? V(0) : before);
}

// Adds to to[at] in shared memory if b < limit, without a branch.
__device__ __forceinline__ void add_below(float b, float limit, uint32_t to, uint32_t v) {
    asm volatile("{.reg .pred p; setp.lt.f32 p, %0, %1; @p red.shared.add.u32 [%2], %3;}" ::"f"(b), "f"(limit), "r"(to), "r"(v) : "memory");
}
// The halves of a weight; few have an upper one.
__device__ __forceinline__ void add_halves_below(float b, float limit, uint32_t low, uint32_t high, uint32_t w) {
    asm volatile(
        "{.reg .pred p, q; setp.lt.f32 p, %0, %1; setp.ne.and.u32 q, %5, 0, p;"
        "@p red.shared.add.u32 [%2], %4; @q red.shared.add.u32 [%3], %5;}" ::"f"(b), "f"(limit), "r"(low), "r"(high), "r"(w & 0xFFFFu), "r"(w >> 16)
        : "memory");
}
__device__ __forceinline__ uint32_t shared_address(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// A token's place in the order as a number: larger comes first.
__device__ __forceinline__ u64 place_of(uint32_t key, uint32_t index) { return static_cast<u64>(key) << 32 | ~index; }

// The tokens that a histogram is taken of, places from `first` down to `last`, and its bins.
enum Bins { kByScore, kByKey, kByIndex };
struct Among {
    u64 first, last;
    Bins bins;
    float scale;   // bins for each unit of y (kByScore)
    uint32_t key;  // the largest key (kByKey)
    int shift;     // bits of key or index within a bin
};

// Where a histogram's running count or weight reaches its goal.
struct Crossing {
    int bin;     // -1: nowhere
    int count;   // tokens in the bins before (of all bins, if nowhere)
    u64 mass;    // their weight
    u64 goal;
};

// The weight that a share of top_p of a weight is.
__device__ __forceinline__ u64 share_of(float top_p, u64 mass) {
    return max(1ull, static_cast<u64>(ceil(fmax(static_cast<double>(top_p), 0.0) * static_cast<double>(mass))));
}

template <int kThreads>
struct Shared {
    static constexpr int kBins = 4 * kThreads;
    uint32_t count[kBins], low[kBins], high[kBins];  // tokens, and their weights' halves
    u64 list[kThreads], order[kThreads];             // tokens of the bin; in the first CTA, in order
    u64 sums[32];
    int counts[32];
    float top;
    int total_count, listed, index;
    u64 total_mass, all;                             // of the bins; of all tokens
    uint32_t least, most;                            // keys of the bin's tokens
    Crossing crossing;
    u64 cut, cut_mass;
    u64 steps[kThreads / 32][kSteps];                // kept weight of each warp's runs of 32 units
};

// A row's settings.
struct Settings {
    const Sample& p;
    int row, top_k;
    float top_p;
    uint32_t least, random;  // the least weight (min_p), the word
};

template <typename T, int kThreads>
struct Draw {
    static constexpr int kWarps = kThreads / 32, kBins = Shared<kThreads>::kBins;
    static_assert(kBins >= kIndexBins);
    const T* row;
    int vocab, rank, ctas, from, to;  // units of this warp
    bool wide, infinite;
    Row r;
    Shared<kThreads>& sh;
    cg::cluster_group cluster;

    __device__ __forceinline__ Shared<kThreads>& of(int cta) { return *cluster.map_shared_rank(&sh, cta); }

    __device__ __forceinline__ void sync() {
        if (ctas > 1) cluster.sync();
        else __syncthreads();
    }

    // f(logits, first index) for the warp's units, a thread's indices ascending.
    template <typename F>
    __device__ __forceinline__ void each_unit(F f) {
        for (int u = from + static_cast<int>(threadIdx.x & 31); u < to; u += 32) {
            float x[kUnit];
            load_unit(row, u * kUnit, vocab, wide, infinite, x);
            f(x, u * kUnit);
        }
    }
    // f(logit, index) for the set bits of a unit's mask. Few are: they are loaded again, one by one.
    template <typename F>
    __device__ __forceinline__ void each_set(unsigned mask, int j, F f) {
        for (; mask != 0; mask &= mask - 1) {
            const int at = j + __ffs(mask) - 1;
            float x = static_cast<float>(row[at]);
            if (infinite) x = x == INFINITY ? 0.0f : -INFINITY;
            f(x, at);
        }
    }

    // Bin of a token; -1 if it is not among them.
    __device__ __forceinline__ int bin_of(const Among& a, float x, int index) const {
        const uint32_t key = key_of(x);
        const u64 place = place_of(key, index);
        if (key <= kNothing || place > a.first || place < a.last) return -1;
        if (a.bins == kByScore) return static_cast<int>(fminf(r.scaled(x) * a.scale, static_cast<float>(kBins)));
        return a.bins == kByKey ? static_cast<int>((a.key - key) >> a.shift) : index >> a.shift;
    }
    // The unit's tokens that may be among them (no NaN).
    __device__ __forceinline__ unsigned near(const Among& a, const float (&x)[kUnit]) const {
        const float least = a.last == 0 ? -INFINITY : logit_of(static_cast<uint32_t>(a.last >> 32));
        unsigned mask = 0;
#pragma unroll
        for (int i = 0; i < kUnit; ++i) mask |= x[i] >= least ? 1u << i : 0u;
        return mask;
    }

    // Counts of the bins need no weights: a token without weight only follows all others.
    template <bool kCounts, bool kMasses>
    __device__ __forceinline__ void fill(const Among& a) {
        constexpr float kLimit = static_cast<float>(kBins);
        const uint32_t counts = shared_address(sh.count), lows = shared_address(sh.low), highs = shared_address(sh.high);
        u64 all = 0;
        each_unit([&](const float (&x)[kUnit], int j) {
            if (a.bins == kByScore && a.last == 0) {  // all tokens
#pragma unroll
                for (int i = 0; i < kUnit; ++i) {
                    const float y = r.scaled(x[i]), b = y * a.scale;  // NaN is in no bin
                    const uint32_t at = 4 * static_cast<uint32_t>(b);
                    if constexpr (kCounts) add_below(b, kLimit, counts + at, 1);
                    if constexpr (kMasses) {
                        const uint32_t w = Row::weight_of(y);
                        add_halves_below(b, kLimit, lows + at, highs + at, w);
                        all += w;
                    }
                }
            } else {
                each_set(near(a, x), j, [&](float v, int index) {
                    const int bin = bin_of(a, v, index);
                    const float b = bin < 0 ? kLimit : static_cast<float>(bin);
                    const uint32_t at = 4u * static_cast<uint32_t>(bin);
                    if constexpr (kCounts) add_below(b, kLimit, counts + at, 1);
                    if constexpr (kMasses) add_halves_below(b, kLimit, lows + at, highs + at, r.weight(v));
                });
            }
        });
        if constexpr (kMasses) {
#pragma unroll
            for (int d = 16; d > 0; d /= 2) all += __shfl_xor_sync(kAll, all, d);
            if ((threadIdx.x & 31) == 0 && all > 0) atomicAdd(&sh.all, all);
        }
    }

    // The sum of v over the cluster's CTAs, one a lane; adds those of lanes below `rank` to `before`.
    template <typename V>
    __device__ __forceinline__ static V sum_to(V v, int rank, V& before) {
        V in = v;
#pragma unroll
        for (int d = 1; d < kMaxCluster; d *= 2) {
            const V o = __shfl_up_sync(kAll, in, d);
            if (static_cast<int>(threadIdx.x & 31) >= d) in += o;
        }
        before += rank > 0 ? __shfl_sync(kAll, in, rank > 0 ? rank - 1 : 0) : V(0);
        return __shfl_sync(kAll, in, kMaxCluster - 1);
    }

    // Where the tokens' number (kCounts) or else their weight reaches `goal` (0: a share of top_p of all weights).
    template <bool kCounts, bool kMasses>
    __device__ Crossing find(const Among& a, u64 goal, float top_p) {
        for (int i = threadIdx.x; i < kBins; i += kThreads) sh.count[i] = sh.low[i] = sh.high[i] = 0;
        if (threadIdx.x == 0) sh.all = 0;
        __syncthreads();
        fill<kCounts, kMasses>(a);
        sync();
        // each CTA joins a section of the bins, a thread a few in a row
        constexpr int kMost = kBins / kThreads;
        const int section = kBins / ctas, share = (section + kThreads - 1) / kThreads;
        const int begin = static_cast<int>(threadIdx.x) * share;
        const int first = rank * section + begin;
        int count[kMost];
        u64 mass[kMost];
        int n = 0;
        u64 m = 0;
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            count[i] = 0;
            mass[i] = 0;
            if (i < share && begin + i < section) {
                for (int c = 0; c < ctas; ++c) {
                    if constexpr (kCounts) count[i] += of(c).count[first + i];
                    if constexpr (kMasses) mass[i] += of(c).low[first + i] + (static_cast<u64>(of(c).high[first + i]) << 16);
                }
            }
            n += count[i];
            m += mass[i];
        }
        int total_count = 0, before = 0;
        u64 total_mass = 0, mass_before = 0;
        if constexpr (kCounts) before = block_exclusive<kWarps>(n, sh.counts, total_count);
        if constexpr (kMasses) mass_before = block_exclusive<kWarps>(m, sh.sums, total_mass);
        if (threadIdx.x == 0) {
            sh.total_count = total_count;
            sh.total_mass = total_mass;
        }
        sync();
        // a lane reads a CTA's totals
        const int lane = threadIdx.x & 31;
        const Shared<kThreads>& other = of(min(lane, ctas - 1));
        const bool real = lane < ctas;
        const int all_count = kCounts ? sum_to(real ? other.total_count : 0, rank, before) : 0;
        const u64 binned = kMasses ? sum_to(real ? other.total_mass : 0, rank, mass_before) : 0;
        u64 none = 0;
        if (goal == 0) goal = share_of(top_p, sum_to(real ? other.all : 0, 0, none));
        const auto tell = [&](const Crossing& x) {
            for (int c = 0; c < ctas; ++c) of(c).crossing = x;
        };
        if ((kCounts ? static_cast<u64>(all_count) : binned) < goal) {
            if (rank == 0 && threadIdx.x == 0) tell({-1, all_count, binned, goal});
        } else {
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                const u64 x = kCounts ? static_cast<u64>(before) : mass_before;
                const u64 y = x + (kCounts ? static_cast<u64>(count[i]) : mass[i]);
                if (x < goal && y >= goal) tell({first + i, before, mass_before, goal});
                before += count[i];
                mass_before += mass[i];
            }
        }
        sync();
        return sh.crossing;
    }

    // The bin's tokens (with all_before, and those of the bins before, by score): their number, or more than
    // kThreads if they do not fit the first CTA's list.
    __device__ int collect(const Among& a, int bin, bool all_before) {
        if (threadIdx.x == 0) {
            sh.listed = 0;
            sh.least = 0xFFFFFFFFu;
            sh.most = 0;
        }
        __syncthreads();
        uint32_t least = 0xFFFFFFFFu, most = 0;
        each_unit([&](const float (&x)[kUnit], int j) {
            unsigned mask = 0;
            if (a.bins == kByScore) {  // the bin's edges, in the same arithmetic
                const float from = all_before ? 0.0f : static_cast<float>(bin), to = static_cast<float>(bin + 1);
#pragma unroll
                for (int i = 0; i < kUnit; ++i) {
                    const float b = r.scaled(x[i]) * a.scale;
                    mask |= b >= from && b < to ? 1u << i : 0u;
                }
            } else {
                mask = near(a, x);
            }
            each_set(mask, j, [&](float v, int index) {
                const int b = bin_of(a, v, index);
                if (b != bin && !(all_before && b >= 0 && b < bin)) return;
                const uint32_t key = key_of(v);
                least = min(least, key);
                most = max(most, key);
                if (*static_cast<volatile int*>(&sh.listed) > kThreads) return;  // too many in any case
                const int at = atomicAdd(&sh.listed, 1);
                if (at < kThreads) sh.list[at] = place_of(key, index);
            });
        });
        least = __reduce_min_sync(kAll, least);
        most = __reduce_max_sync(kAll, most);
        if ((threadIdx.x & 31) == 0) {
            atomicMin(&sh.least, least);
            atomicMax(&sh.most, most);
        }
        sync();
        const int lane = threadIdx.x & 31;
        return __reduce_add_sync(kAll, lane < ctas ? min(of(min(lane, ctas - 1)).listed, kThreads + 1) : 0);
    }

    // The first CTA: the place of the thread's token in the order of the n that are listed; 0 past them.
    __device__ __forceinline__ u64 ranked(int n) {
        const int i = threadIdx.x;
        u64 place = 0;
        if (i < n) {
            int at = i, c = 0;
            while (at >= of(c).listed) at -= of(c++).listed;
            place = of(c).list[at];
            sh.order[i] = place;
        }
        __syncthreads();
        int before = 0;
        for (int j = 0; j < n; ++j) before += sh.order[j] > place ? 1 : 0;
        __syncthreads();
        if (i < n) sh.order[before] = place;
        __syncthreads();
        return i < n ? sh.order[i] : 0;
    }

    // Ranks the n listed tokens and tells every CTA the place of the one that reaches the goal, `count`
    // tokens of weight `mass` being before them.
    __device__ void choose(int n, bool tokens, u64 goal, u64 count, u64 mass) {
        if (rank == 0) {
            const int i = threadIdx.x;
            const u64 place = ranked(n);
            const u64 w = i < n ? r.weight(logit_of(static_cast<uint32_t>(place >> 32))) : 0;
            u64 all;
            const u64 x = block_exclusive<kWarps>(w, sh.sums, all);
            const bool here = tokens ? count + i + 1 == goal : mass + x < goal && mass + x + w >= goal;
            if (i < n && here) {
                for (int c = 0; c < ctas; ++c) {
                    of(c).cut = place;
                    of(c).cut_mass = mass + x + w;
                }
            }
        }
        sync();
    }

    // The whole draw by the first CTA, where everything that is kept is among the n listed tokens: the first
    // top_k, and of those what reaches `goal` (0: a share of top_p of them).
    __device__ void draw_listed(const Settings& t, int n, int top_k, u64 goal) {
        const int i = threadIdx.x;
        const u64 place = ranked(n);
        const float x = i < n ? logit_of(static_cast<uint32_t>(place >> 32)) : -INFINITY;
        const uint32_t w = i < min(n, top_k) ? r.weight(x) : 0, index = ~static_cast<uint32_t>(place);
        u64 mass, total;
        const u64 before = block_exclusive<kWarps>(static_cast<u64>(w), sh.sums, mass);
        if (goal == 0 && t.top_p < 1.0f) goal = share_of(t.top_p, mass);
        const bool in = goal == 0 || before < goal;
        const uint32_t kept = in && w >= t.least ? w : 0;
        block_exclusive<kWarps>(static_cast<u64>(kept), sh.sums, total);
        sh.list[i] = static_cast<u64>(index) << 32 | kept;  // of this CTA: all have been read
        __syncthreads();
        u64 run = 0;  // of kept tokens with a lower index
        for (int j = 0; j < n; ++j) {
            const u64 other = sh.list[j];
            if (static_cast<uint32_t>(other >> 32) < index) run += static_cast<uint32_t>(other);
        }
        const u64 aim = __umul64hi(static_cast<u64>(t.random) << 32, total);
        if (kept > 0 && run <= aim && aim < run + kept) {
            t.p.tokens[t.row] = static_cast<int>(index);
            if (t.p.logprobs != nullptr) t.p.logprobs[t.row] = r.scaled(x) - logf(static_cast<float>(total) * (1.0f / kOne));
        }
    }

    // The end of what is kept by the number of tokens or else by weight: `last` is the place of its last token (0:
    // nothing is cut off), `mass` its weight; both tell of an earlier end before. True if the draw is done.
    template <bool kTokens>
    __device__ __forceinline__ bool cut_off(const Settings& t, bool nucleus, bool counted, u64& last, u64& mass) {
        // tokens more than ln(vocab / (1 - p)) below the largest together weigh less than 1 - p of it; 0.1
        // for roundings, which are larger where weights are below five units
        float reach = kTokens ? kReach : logf(static_cast<float>(vocab) / (1.0f - fmaxf(t.top_p, 0.0f))) + 0.1f;
        if (!(reach < 19.0f)) reach = kReach;
        u64 goal = kTokens ? static_cast<u64>(t.top_k) : counted ? share_of(t.top_p, mass) : 0;  // 0: known with the weights
        Among a = {~0ull, last, kByScore, -kBins / reach, 0, 0};
        // where few are kept one list holds them all, ties apart, and the first CTA does the rest
        bool whole = kTokens ? t.top_k <= kThreads / 2 : !counted;
        int count = 0;  // of tokens before `a`, and their weight; `last` stays if the goal is not reached
        mass = 0;
        // by score, twice if it was not within reach or the list was not enough; by key at most four times (32
        // bits, 10 at a time); by index, 256 to a bin: those fit
        for (int round = 0; round < 8; ++round) {
            const u64 left = goal == 0 ? 0 : goal - (kTokens ? count : mass);
            Crossing x;
            if (kTokens && (whole || !nucleus)) x = find<kTokens, !kTokens>(a, left, t.top_p);
            else x = find<kTokens, true>(a, left, t.top_p);
            if (goal == 0) goal = x.goal;
            if (x.bin < 0) {
                if (a.bins == kByScore && reach < kReach) {
                    reach = kReach;
                    a.scale = -kBins / reach;
                    continue;
                }
                if (kTokens && whole && nucleus) {  // all are kept, and now their weight is wanted
                    whole = false;
                    continue;
                }
                mass += x.mass;
                break;
            }
            // tokens before the bin weigh at least as much each as one on its upper edge: are they few?
            if (!kTokens) whole = whole && static_cast<float>(x.mass) <= kThreads / 2 * kOne * expf(static_cast<float>(x.bin) / a.scale);
            int n = collect(a, x.bin, whole);
            if (whole) {
                if (n <= kThreads) {
                    if (rank == 0) draw_listed(t, n, kTokens ? t.top_k : vocab, kTokens ? 0 : goal);
                    sync();  // until every CTA's memory has been read
                    return true;
                }
                sync();
                whole = false;
                if (kTokens) continue;
                n = collect(a, x.bin, false);
            }
            count += x.count;
            mass += x.mass;
            if (n <= kThreads) {
                choose(n, kTokens, goal, count, mass);
                last = sh.cut;
                mass = sh.cut_mass;
                break;
            }
            uint32_t lowest = 0xFFFFFFFFu, highest = 0;
            for (int c = 0; c < ctas; ++c) {
                lowest = min(lowest, of(c).least);
                highest = max(highest, of(c).most);
            }
            sync();  // read by all before it is set anew
            a.first = min(a.first, place_of(highest, 0));
            a.last = max(a.last, place_of(lowest, 0xFFFFFFFFu));
            a.key = highest;
            a.bins = lowest == highest ? kByIndex : kByKey;
            a.shift = lowest == highest ? 8 : max(0, 22 - __clz(highest - lowest));
        }
        return false;
    }

    // Of the unit's tokens, which may be kept: at or above x, and with y at or above y. It only saves weighing: none that
    // is kept may be left out.
    __device__ __forceinline__ unsigned candidates(const float(&x)[kUnit], float least_x, float least_y) const {
        unsigned mask = 0;
#pragma unroll
        for (int i = 0; i < kUnit; ++i) mask |= x[i] >= least_x ? 1u << i : 0u;
        if (least_y > -INFINITY) {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) mask &= r.scaled(x[i]) >= least_y ? ~0u : ~(1u << i);
        }
        return mask;
    }

    __device__ __forceinline__ static float max_of(float v) {
#pragma unroll
        for (int d = 16; d > 0; d /= 2) v = fmaxf(v, __shfl_xor_sync(kAll, v, d));
        return v;
    }

    __device__ void run(const Sample& p, int i) {
        const float temperature = p.temperature == nullptr ? 1.0f : p.temperature[i];
        const int top_k = p.top_k == nullptr ? 0 : p.top_k[i];
        const float min_p = p.min_p == nullptr ? 0.0f : p.min_p[i];
        const float top_p = p.top_p == nullptr ? 1.0f : p.top_p[i];
        const uint32_t random = p.words[i];
        float top = -INFINITY;
        each_unit([&](const float (&x)[kUnit], int) {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) top = fmaxf(top, x[i]);  // NaN is passed over
        });
        top = max_of(top);
        if ((threadIdx.x & 31) == 0) sh.counts[threadIdx.x >> 5] = __float_as_int(top);
        if (threadIdx.x == 0) sh.index = 0x7FFFFFFF;
        __syncthreads();
        const int lane = threadIdx.x & 31;
        top = max_of(lane < kWarps ? __int_as_float(sh.counts[lane]) : -INFINITY);
        if (ctas > 1) {
            if (threadIdx.x == 0) sh.top = top;
            sync();
            top = max_of(of(min(lane, ctas - 1)).top);
        }

        const bool none = top == -INFINITY;
        if (none || !(temperature >= 0x1p-64f) || top_k == 1) {  // the first of the largest
            int first = 0x7FFFFFFF;
            each_unit([&](const float (&x)[kUnit], int j) {
#pragma unroll
                for (int i = 0; i < kUnit; ++i) first = min(first, x[i] == top ? j + i : 0x7FFFFFFF);
            });
            first = __reduce_min_sync(kAll, first);
            if ((threadIdx.x & 31) == 0) atomicMin(&sh.index, first);
            sync();
            if (rank == 0 && threadIdx.x == 0) {
                for (int c = 0; c < ctas; ++c) first = min(first, of(c).index);
                p.tokens[i] = none ? -1 : first;
                if (p.logprobs != nullptr) p.logprobs[i] = none ? -INFINITY : 0.0f;
            }
            sync();  // until every CTA's memory has been read
            return;
        }
        infinite = top == INFINITY;
        r.top = infinite ? 0.0f : top;
        r.inverse = __frcp_rn(temperature);
        const uint32_t least = min_p > 0.0f ? static_cast<uint32_t>(ceil(fmin(static_cast<double>(min_p), 1.0) * 1073741824.0)) : 0;
        u64 last = 0, mass = 0;
        const bool counted = top_k > 0 && top_k < vocab, nucleus = top_p < 1.0f;
        // the end of what is kept, first by top_k and then, among that, by top_p
        const Settings settings = {p, i, top_k, top_p, least, random};
        if (counted && cut_off<true>(settings, nucleus, counted, last, mass)) return;
        if (nucleus && cut_off<false>(settings, nucleus, counted, last, mass)) return;

        // what is kept; few tokens are where something is cut off, and only those are weighed
        const float least_x = last == 0 ? -INFINITY : logit_of(static_cast<uint32_t>(last >> 32));
        const int last_index = static_cast<int>(~static_cast<uint32_t>(last));
        // a weight is rounded to the least one from half a unit below it on; 0.01 for the roundings of y, logf and expf
        const float least_y = least > 0 ? logf((static_cast<float>(least) - 0.5f) * (1.0f / kOne)) - 0.01f : -INFINITY;
        const bool cut = last != 0 || least > 0;
        const auto kept = [&](float x, int index) -> uint32_t {
            if (x == least_x && index > last_index && last != 0) return 0;
            const uint32_t w = r.weight(x);
            return w >= least ? w : 0;
        };
        const auto weigh = [&](const float(&x)[kUnit], int j) -> u64 {
            u64 sum = 0;
            if (cut) {
                each_set(candidates(x, least_x, least_y), j, [&](float v, int at) { sum += kept(v, at); });
            } else {
#pragma unroll
                for (int k = 0; k < kUnit; ++k) sum += r.weight(x[k]);
            }
            return sum;
        };
        // sums of the warp's steps of 32 units, kept for finding the token's
        const int warp = threadIdx.x >> 5;
        u64 sum = 0;
        for (int u = from; u < to; u += 32) {
            u64 mine = 0;
            if (u + lane < to) {
                float x[kUnit];
                load_unit(row, (u + lane) * kUnit, vocab, wide, infinite, x);
                mine = weigh(x, (u + lane) * kUnit);
            }
#pragma unroll
            for (int d = 16; d > 0; d /= 2) mine += __shfl_xor_sync(kAll, mine, d);
            if (lane == 0) sh.steps[warp][(u - from) / 32] = mine;
            sum += mine;
        }
        __syncwarp();
        u64 here;
        // one thread a warp counts: its prefix is the warp's
        u64 before = block_exclusive<kWarps>(lane == 0 ? sum : 0, sh.sums, here);
        before = __shfl_sync(kAll, before, 0);
        if (threadIdx.x == 0) sh.total_mass = here;
        sync();
        const u64 all = sum_to(lane < ctas ? of(min(lane, ctas - 1)).total_mass : 0, rank, before);
        const u64 aim = __umul64hi(static_cast<u64>(random) << 32, all);
        if (aim >= before && aim < before + sum) {  // the warp that has the token
            u64 run = before;
            int u = from;
            for (int step = 0; run + sh.steps[warp][step] <= aim; ++step, u += 32) run += sh.steps[warp][step];
            float x[kUnit];
            u64 mine = 0;
            if (u + lane < to) {
                load_unit(row, (u + lane) * kUnit, vocab, wide, infinite, x);
                mine = weigh(x, (u + lane) * kUnit);
            }
            const u64 in = run + warp_inclusive(mine);
            if (aim >= in - mine && aim < in) {
                u64 sofar = in - mine;
#pragma unroll
                for (int k = 0; k < kUnit; ++k) {
                    const u64 w = x[k] >= least_x ? kept(x[k], (u + lane) * kUnit + k) : 0;
                    if (aim >= sofar && aim < sofar + w) {
                        p.tokens[i] = (u + lane) * kUnit + k;
                        if (p.logprobs != nullptr) p.logprobs[i] = r.scaled(x[k]) - logf(static_cast<float>(all) * (1.0f / kOne));
                    }
                    sofar += w;
                }
            }
        }
        sync();  // until every CTA has read the others' memory
    }
};

static_assert(kMaxSlice / kUnit / 32 <= kSteps * (kLarge / 32) && kSmallVocab / kUnit / 32 <= kSteps * 8, "a warp's steps");

__host__ __device__ constexpr int units_per_warp(int vocab, int warps) {
    return ((vocab + kUnit - 1) / kUnit + warps - 1) / warps;
}

template <typename T, int kThreads>
__global__ void __launch_bounds__(kThreads, kResident / kThreads) sample_kernel(Sample p) {
    __shared__ Shared<kThreads> sh;
    after_previous();
    let_next_start();
    const cg::cluster_group cluster = cg::this_cluster();
    const int ctas = cluster.num_blocks(), rank = cluster.block_rank(), i = blockIdx.x / ctas;
    const T* row = reinterpret_cast<const T*>(p.logits) + static_cast<uint64_t>(i) * p.row_stride;
    // a warp's tokens are consecutive, and so are the warps': indices ascend with (CTA, warp)
    constexpr int kWarps = kThreads / 32;
    const int units = (p.vocab + kUnit - 1) / kUnit, per = units_per_warp(p.vocab, ctas * kWarps);
    const int from = min((rank * kWarps + static_cast<int>(threadIdx.x >> 5)) * per, units);
    const bool wide = reinterpret_cast<uint64_t>(row) % 16 == 0;
    Draw<T, kThreads> draw = {row, p.vocab, rank, ctas, from, min(from + per, units), wide, false, {}, sh, cluster};
    draw.run(p, i);
}

template <typename T>
cudaError_t launch_t(const Sample& p, cudaStream_t s) {
    // few tokens: CTAs of 256 threads, more of which fit an SM
    const bool small = p.vocab <= kSmallVocab;
    const int threads = small ? 256 : kLarge, tokens = threads * kUnit, room = kSms * (kResident / threads);
    int ctas = 1;
    // as many CTAs as run at once and have a unit for every thread; more where a slice would be too long
    const auto more = [&](int c) {
        return units_per_warp(p.vocab, c * threads / 32) * (threads / 32) * kUnit > kMaxSlice ||
               (2ll * c * p.n <= room && p.vocab > c * tokens);
    };
    while (ctas < kMaxCluster && more(ctas)) ctas *= 2;
    if (static_cast<long long>(p.n) * ctas > 0x7FFFFFFFll) return cudaErrorInvalidValue;
    return launch(small ? sample_kernel<T, 256> : sample_kernel<T, kLarge>, static_cast<unsigned>(p.n) * ctas, threads, 0, ctas, s, p);
}

}  // namespace

cudaError_t launch_sample(const Sample& p, cudaStream_t s) {
    return p.bf16 ? launch_t<__nv_bfloat16>(p, s) : launch_t<float>(p, s);
}

}  // namespace jb
