// jb_sample.cu -- the next token of each row from its logits and a random word.
//
// Weights are integers (w = rint(2^30 exp(y))), so a sum of them is the same in every order and the
// token is a function of the logits' bits, the settings and the word alone. What is kept is a prefix
// of the order (logit descending, index ascending); its end is found by descending through the digits
// of the logits' ordered keys with a histogram of counts and weights for each digit.
#include <cuda_bf16.h>

#include "jb_answer.h"

namespace jb {
namespace {

constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
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

struct Row {
    uint32_t top;   // key of the largest logit
    float high;     // the largest logit
    float inverse;  // 1 / temperature
    u64 cut;        // least weight (min_p)

    __device__ float scaled(uint32_t key) const { return key == top ? 0.0f : (logit_of(key) - high) * inverse; }
    __device__ u64 weight(uint32_t key) const {
        if (key <= kNothing) return 0;
        return static_cast<u64>(__float2ll_rn(expf(scaled(key)) * kOne));
    }
};

template <typename T>
__device__ __forceinline__ uint32_t load_key(const T* row, int j);
template <>
__device__ __forceinline__ uint32_t load_key<float>(const float* row, int j) { return key_of(row[j]); }
template <>
__device__ __forceinline__ uint32_t load_key<__nv_bfloat16>(const __nv_bfloat16* row, int j) { return key_of(__bfloat162float(row[j])); }

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

// Exclusive prefix over the CTA's threads and the total.
template <typename V>
__device__ __forceinline__ V block_exclusive(V v, V* sums, V& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const V in = warp_inclusive(v);
    if (lane == 31) sums[warp] = in;
    __syncthreads();
    const V all = warp_inclusive(sums[lane]);
    const V before = __shfl_sync(kAll, all, warp == 0 ? 0 : warp - 1);
    total = __shfl_sync(kAll, all, 31);
    __syncthreads();
    return in - v + (warp == 0 ? V(0) : before);
}

// The end of what is kept: keys above `key`, and of the tokens with that key the first `ties`.
struct End {
    uint32_t key;
    int ties;
    u64 mass;  // weight of what is kept
};

struct Shared {
    int count[256];
    u64 mass[256];
    u64 sums[kWarps];
    int counts[kWarps];
    uint32_t key;
    int above;
    u64 mass_above;
    int found;
};

// The end of the shortest prefix of the order, within `within`, that has `goal` tokens (by_mass
// false) or weighs `goal` (by_mass true). Tokens of weight 0 are not counted: they are never drawn.
template <typename T>
__device__ End descend(const T* row, int vocab, const Row& r, const End& within, bool by_mass, u64 goal, Shared& sh) {
    uint32_t prefix = 0;
    int above = 0;
    u64 mass_above = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (threadIdx.x < 256) {
            sh.count[threadIdx.x] = 0;
            sh.mass[threadIdx.x] = 0;
        }
        __syncthreads();
        for (int j = threadIdx.x; j < vocab; j += kThreads) {
            const uint32_t key = load_key(row, j);
            if (key < within.key || (shift < 24 && (key ^ prefix) >> (shift + 8) != 0)) continue;
            const u64 w = r.weight(key);
            if (w == 0) continue;
            atomicAdd(&sh.count[key >> shift & 255], 1);
            atomicAdd(&sh.mass[key >> shift & 255], w);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            int digit = 255;
            for (; digit > 0; --digit) {
                const bool last = by_mass ? mass_above + sh.mass[digit] >= goal
                                          : static_cast<u64>(above) + sh.count[digit] >= goal;
                if (last) break;
                above += sh.count[digit];
                mass_above += sh.mass[digit];
            }
            sh.key = prefix | static_cast<uint32_t>(digit) << shift;
            sh.above = above;
            sh.mass_above = mass_above;
        }
        __syncthreads();
        prefix = sh.key;
        above = sh.above;
        mass_above = sh.mass_above;
        __syncthreads();
    }
    End e;
    e.key = prefix;
    const u64 w = r.weight(prefix);
    int most = prefix == within.key ? within.ties : 0x7FFFFFFF;  // tokens with this key
    // sh.count holds the last digit's histogram: tokens with exactly this key
    most = min(most, sh.count[prefix & 255]);
    const u64 wanted = by_mass ? (w == 0 ? 0 : (goal - min(goal, mass_above) + w - 1) / w) : goal - min(goal, static_cast<u64>(above));
    e.ties = static_cast<int>(min(static_cast<u64>(most), wanted));
    e.mass = mass_above + w * e.ties;
    __syncthreads();
    return e;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_kernel(Sample p) {
    __shared__ Shared sh;
    const int i = blockIdx.x;
    const T* row = reinterpret_cast<const T*>(p.logits) + static_cast<uint64_t>(i) * p.row_stride;

    uint32_t top = 0;
    for (int j = threadIdx.x; j < p.vocab; j += kThreads) top = max(top, load_key(row, j));
    top = __reduce_max_sync(kAll, top);
    if ((threadIdx.x & 31) == 0) sh.counts[threadIdx.x >> 5] = static_cast<int>(top);
    __syncthreads();
    top = __reduce_max_sync(kAll, static_cast<uint32_t>(sh.counts[threadIdx.x & 31]));
    __syncthreads();
    if (top <= kNothing) {
        if (threadIdx.x == 0) {
            p.tokens[i] = -1;
            if (p.logprobs != nullptr) p.logprobs[i] = -INFINITY;
        }
        return;
    }
    const float temperature = p.temperature == nullptr ? 1.0f : p.temperature[i];
    const bool greedy = !(temperature >= 0x1p-64f);
    Row r;
    r.top = top;
    r.high = logit_of(top);
    r.inverse = greedy ? 1.0f : __frcp_rn(temperature);
    const float min_p = p.min_p == nullptr ? 0.0f : p.min_p[i];
    r.cut = min_p > 0.0f ? static_cast<u64>(ceil(fmin(static_cast<double>(min_p), 1.0) * 1073741824.0)) : 0;
    const int top_k = greedy ? 1 : p.top_k == nullptr ? 0 : p.top_k[i];
    const double top_p = p.top_p == nullptr ? 1.0 : static_cast<double>(p.top_p[i]);

    // everything that has a weight
    End end = {kNothing + 1, 0x7FFFFFFF, 0};
    if (top_k > 0 && top_k < p.vocab) {
        end = descend(row, p.vocab, r, end, false, static_cast<u64>(top_k), sh);
    } else {
        u64 sum = 0;
        for (int j = threadIdx.x; j < p.vocab; j += kThreads) sum += r.weight(load_key(row, j));
        block_exclusive(sum, sh.sums, end.mass);
    }
    if (top_p < 1.0) {
        const u64 goal = max(1ull, static_cast<u64>(ceil(fmax(top_p, 0.0) * static_cast<double>(end.mass))));
        end = descend(row, p.vocab, r, end, true, goal, sh);
    }
    // weights of what is kept, in the order of the indices
    const auto kept = [&](uint32_t key, int tie) -> u64 {
        if (key < end.key || (key == end.key && tie >= end.ties)) return 0;
        const u64 w = r.weight(key);
        return w >= r.cut ? w : 0;
    };
    u64 all = 0;
    int ties = 0;
    for (int first = 0; first < p.vocab; first += kThreads) {
        const int j = first + threadIdx.x;
        const uint32_t key = j < p.vocab ? load_key(row, j) : 0;
        int here;
        const int tie = ties + block_exclusive(key == end.key ? 1 : 0, sh.counts, here);
        u64 sum;
        block_exclusive(kept(key, tie), sh.sums, sum);
        all += sum;
        ties += here;
    }
    const u64 aim = __umul64hi(static_cast<u64>(p.words[i]) << 32, all);
    u64 run = 0;
    ties = 0;
    for (int first = 0; first < p.vocab; first += kThreads) {
        const int j = first + threadIdx.x;
        const uint32_t key = j < p.vocab ? load_key(row, j) : 0;
        int here;
        const int tie = ties + block_exclusive(key == end.key ? 1 : 0, sh.counts, here);
        u64 sum;
        const u64 w = kept(key, tie);
        const u64 before = run + block_exclusive(w, sh.sums, sum);
        if (w > 0 && before <= aim && aim < before + w) {
            p.tokens[i] = j;
            if (p.logprobs != nullptr) p.logprobs[i] = r.scaled(key) - logf(static_cast<float>(all) * (1.0f / kOne));
        }
        run += sum;
        ties += here;
        if (run > aim) break;
    }
}

}  // namespace

cudaError_t launch_sample(const Sample& p, cudaStream_t s) {
    if (p.bf16) sample_kernel<__nv_bfloat16><<<p.n, kThreads, 0, s>>>(p);
    else sample_kernel<float><<<p.n, kThreads, 0, s>>>(p);
    return cudaGetLastError();
}

}  // namespace jb
