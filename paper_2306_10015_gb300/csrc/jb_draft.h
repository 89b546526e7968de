// jb_draft.h -- launch descriptors of the calls that work on drafted tokens and of the products with 4-bit weights,
// shared by their host side (jb_draft_capi.cpp) and the kernels (jb_append.cu, jb_keep.cu, jb_tree.cu, jb_q4_matmul.cu).
// Not part of the public interface.
#pragma once
#include <cstdint>

#include <cuda_runtime.h>

#include "jb_answer.h"

namespace jb {

constexpr int kMaxNodes = 256;           // drafted tokens of a tree
constexpr int kMaxInner = 65536;         // columns of a matrix of 4-bit weights
constexpr int kMaxOutputs = 1 << 30;     // its rows
constexpr int kMaxMatmulRows = 1 << 30;  // rows that it is multiplied with: passes over them end below 2^31
constexpr int kMaxAppendVecs = 1 << 20;  // 16-byte vectors of a token's queries and keys

struct Append {
    const char* from[3];        // queries, keys, values; strides in bytes
    uint64_t token_stride[3], head_stride[3];
    char* q_out;
    uint64_t out_token, out_head;
    char* to[2];                // the layer's keys, values
    uint64_t page_stride, to_head, to_token;
    const uint64_t* steps;
    const int* rows;
    const int* pos;
    const int* turns;
    int n, q_heads, heads, head_dim, dims, interleaved, bf16;
};
cudaError_t launch_append(const Pages& p, const Append& a, cudaStream_t s);

// jb_trees as the kernels take it.
struct Trees {
    const int* rows;
    const int* starts;
    const int* parents;
    int n, n_nodes;
};

// Words of a workspace of jb_cache_keep: header, moves of each tree, then (page, place) from and to of each node.
inline uint64_t keep_words(int n, int n_nodes) { return kHeaderWords + static_cast<uint64_t>(n) + 4ull * n_nodes; }
cudaError_t launch_keep_plan(const Pages& p, const Trees& t, const int* leaves, int* status, int* ws, cudaStream_t s);
cudaError_t launch_keep_move(const Pages& p, const Trees& t, const Pools& pools, const int* ws, cudaStream_t s);

struct TreeAttend {
    const char* q;
    char* out;
    uint64_t q_row, q_head, out_row, out_head;          // elements
    const char* k;
    const char* v;
    uint64_t page_stride, head_stride, token_stride;    // elements
    const float* slopes;
    float* ws;
    float scale, softcap;
    int window, heads, group, head_dim, bf16;
};
uint64_t tree_workspace(int bf16, int head_dim);
cudaError_t launch_tree(const Pages& p, const Trees& t, const TreeAttend& a, cudaStream_t s);

struct Q4Matmul {
    const uint8_t* codes;
    const float* scale;
    const void* x;
    const void* bias;
    void* y;
    uint64_t x_row, y_row;  // elements
    void* ws;
    int n, out, in, bf16;
};
// What levels are multiplied by before they become fp16, and sums divided by. fp32: so that their lower parts are normal numbers.
// bf16: the 16 levels happen to lie near numbers of fp16 then, off by at most 1.59e-4 of themselves and 0.9e-4 in the root mean
// square (times 1: 3.66e-4 and 1.7e-4; the best of all multiples of 2^-10 between 1 and 2, with which the levels -1 and 1 are exact).
template <bool kF32>
constexpr float kLevelScale = kF32 ? 1024.0f : 1391.0f / 1024.0f;

// Large products, by tcgen05: whether one is, its workspace and its launch.
bool q4_by_tiles(int n, int out, int in, int bf16);
uint64_t q4_workspace(int n, int out, int in, int bf16);
cudaError_t launch_q4_tiles(const Q4Matmul& m, cudaStream_t s);
cudaError_t launch_q4_matmul(const Q4Matmul& m, cudaStream_t s);

}  // namespace jb
