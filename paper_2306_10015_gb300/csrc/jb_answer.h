// jb_answer.h -- launch descriptors of the calls that write answers, shared by their host side
// (jb_answer_capi.cpp) and the kernels (jb_pages.cu, jb_attend.cu, jb_sample.cu). Not part of the
// public interface.
#pragma once
#include <cstdint>

#include <cuda_runtime.h>

namespace jb {

constexpr int kMaxRows = 65536;          // rows of a cache
constexpr int kMaxListed = 16384;        // rows or pairs listed in one call
constexpr int kLayersPerLaunch = 128;    // layers whose pages one launch copies
constexpr int kMaxHeadDim = 256;
constexpr int kMaxVocab = 1 << 18;       // sums of 2^18 weights of 2^30 stay below 2^48

// jb_pages as the kernels take it.
struct Pages {
    int* table;
    int* lens;
    int* refs;
    int n_rows, row_pages, n_pages, page_tokens;
};

// Where the pages of layers with the same geometry are. A page is `slabs` runs (heads, or the
// whole page where tokens come first) of page_tokens rows of row_vecs 16-byte vectors.
struct Pools {
    uint64_t stride;  // bytes from page to page
    uint32_t slabs;
    uint32_t row_vecs;
    uint32_t n;       // pools: the keys and the values of each layer
    char* base[2 * kLayersPerLaunch];
};

cudaError_t launch_reserve(const Pages& p, const int* rows, const int* tokens, int n, int* status, cudaStream_t s);
cudaError_t launch_free(const Pages& p, const int* rows, int n, cudaStream_t s);
cudaError_t launch_fork_plan(const Pages& p, const int* parents, const int* children, int n, int* status, int* ws,
                             cudaStream_t s);
cudaError_t launch_fork_copy(const Pages& p, const Pools& pools, int n, const int* ws, cudaStream_t s);
cudaError_t launch_compact_plan(const Pages& p, int* status, int* ws, cudaStream_t s);
cudaError_t launch_compact_move(const Pages& p, const Pools& pools, bool table, const int* ws, cudaStream_t s);

// Words of the workspaces, in 4-byte units.
constexpr int kHeaderWords = 16;
inline uint64_t fork_words(const Pages& p, int n) {
    return kHeaderWords + 3ull * n + static_cast<uint64_t>(n) * p.row_pages;
}
inline uint64_t compact_words(const Pages& p) {  // moves (from, to), new ids
    return kHeaderWords + 2ull * (p.n_pages / 2 + 1) + p.n_pages;
}

struct Write {
    const char* from[2];         // keys, values
    uint64_t token_stride[2];    // bytes
    uint64_t head_stride[2];
    char* to[2];
    uint64_t page_stride, to_head, to_token;  // bytes
    const int* rows;
    const int* pos;
    int n, heads;
    uint32_t head_vecs;          // 16-byte vectors of a head
    uint64_t magic;              // 2^32 / head_vecs rounded up: v magic >> 32 is v / head_vecs below 2^20, the
                                 // limit of a token's vectors
};
cudaError_t launch_write(const Pages& p, const Write& w, cudaStream_t s);

struct Attend {
    const char* q;
    char* out;
    uint64_t q_row, q_head, out_row, out_head;          // elements
    const char* k;
    const char* v;
    uint64_t page_stride, head_stride, token_stride;    // elements
    const int* rows;
    const int* pos;
    const float* slopes;
    float* ws;
    float scale, softcap;
    int window, n, heads, group, head_dim, bf16;
};
uint64_t attend_workspace(int bf16, int group, int head_dim);
cudaError_t launch_attend(const Pages& p, const Attend& a, cudaStream_t s);

struct Sample {
    const void* logits;
    uint64_t row_stride;
    int bf16, n, vocab;
    const float* temperature;
    const int* top_k;
    const float* top_p;
    const float* min_p;
    const uint32_t* words;
    int* tokens;
    float* logprobs;
};
cudaError_t launch_sample(const Sample& p, cudaStream_t s);

}  // namespace jb
