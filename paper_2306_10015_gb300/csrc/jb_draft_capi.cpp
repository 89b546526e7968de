// jb_draft_capi.cpp -- the entry points that work on drafted tokens, and the products with 4-bit weights (declared in
// include/jb.h): argument checks and launches. What the lists say is checked by the kernels, on the device.
#include <cmath>

#include "jb.h"
#include "jb_check.h"
#include "jb_draft.h"
#include "jb_host.h"

using namespace jb;

namespace {

int check_trees(const jb_trees* in, Trees& out) {
    if (in == nullptr || in->n < 0 || in->n > kMaxListed || in->n_nodes < 0) return JB_ERR_INVALID_ARG;
    if (in->n > 0 && (in->rows == nullptr || in->starts == nullptr)) return JB_ERR_INVALID_ARG;
    if (in->n_nodes > 0 && in->parents == nullptr) return JB_ERR_INVALID_ARG;
    if (!aligned(in->rows, 4) || !aligned(in->starts, 4) || !aligned(in->parents, 4)) return JB_ERR_MISALIGNED;
    out = {in->rows, in->starts, in->parents, in->n, in->n_nodes};
    return JB_OK;
}

// Rows of runs: `n` rows at `base` + i * row bytes, each with `heads` runs of `len` bytes `head` apart.
struct Runs {
    uint64_t base, n, row, heads, head, len;

    uint64_t extent() const { return (heads - 1) * head + len; }  // of a row
    uint64_t end() const { return base + (n - 1) * row + extent(); }
};

// Whether the addresses of all runs exist; strides are at most 2^48 elements and counts below 2^31 x 2^16, so products
// are formed in 128 bits.
bool fits(const Runs& r) {
    const unsigned __int128 last = static_cast<unsigned __int128>(r.n - 1) * r.row + static_cast<unsigned __int128>(r.heads - 1) * r.head + r.len;
    return last + r.base <= UINT64_MAX;
}

// Whether two sets of runs share no byte, as far as that can be told: they lie apart, or have the same step from row to
// row and rows that lie apart within it, as the parts of one matrix of queries, keys and values do.
bool apart(const Runs& a, const Runs& b) {
    if (a.end() <= b.base || b.end() <= a.base) return true;
    if (a.row != b.row || a.row == 0 || a.extent() > a.row || b.extent() > b.row) return false;
    const uint64_t at = b.base >= a.base ? (b.base - a.base) % a.row : (a.row - (a.base - b.base) % a.row) % a.row;
    return at >= a.extent() && at + b.extent() <= a.row;
}

}  // namespace

JB_EXPORT int jb_cache_append(const jb_pages* pages, const jb_kv* layer, const jb_rotation* rotation, const void* d_q,
                              uint64_t q_token_stride, uint64_t q_head_stride, int q_heads, void* d_q_out,
                              uint64_t out_token_stride, uint64_t out_head_stride, const void* d_k, uint64_t k_token_stride,
                              uint64_t k_head_stride, const void* d_v, uint64_t v_token_stride, uint64_t v_head_stride,
                              const int32_t* d_rows, const int32_t* d_pos, const int32_t* d_turns, int n,
                              struct CUstream_st* stream) {
    return guarded([&] {
        Pages p;
        JB_TRY(check_pages(pages, p));
        if (layer == nullptr || rotation == nullptr) return static_cast<int>(JB_ERR_INVALID_ARG);
        JB_TRY(check_layer(*layer, p));
        if (rotation->dims < 2 || rotation->dims % 2 != 0 || rotation->dims > layer->head_dim || rotation->steps == nullptr)
            return static_cast<int>(JB_ERR_INVALID_ARG);
        if (!aligned(rotation->steps, 8)) return static_cast<int>(JB_ERR_MISALIGNED);
        if (q_heads < 0 || q_heads > 65536) return static_cast<int>(JB_ERR_INVALID_ARG);
        const uint64_t es = size_of(layer->dtype), head_bytes = layer->head_dim * es;
        if ((static_cast<uint64_t>(q_heads) + layer->heads) * (head_bytes / 16) > static_cast<uint64_t>(kMaxAppendVecs))
            return static_cast<int>(JB_ERR_INVALID_ARG);
        JB_TRY(check_list(d_rows, d_pos, n, INT32_MAX));
        if (n == 0) return static_cast<int>(JB_OK);
        const int32_t* turns = d_turns != nullptr ? d_turns : d_pos;
        if (!aligned(turns, 4)) return static_cast<int>(JB_ERR_MISALIGNED);
        if (d_k == nullptr || d_v == nullptr || (q_heads > 0 && (d_q == nullptr || d_q_out == nullptr)))
            return static_cast<int>(JB_ERR_INVALID_ARG);
        if (!aligned(d_k, 16) || !aligned(d_v, 16)) return static_cast<int>(JB_ERR_MISALIGNED);
        JB_TRY(check_strides(k_token_stride, k_head_stride, es));
        JB_TRY(check_strides(v_token_stride, v_head_stride, es));
        const auto runs = [&](const void* at, uint64_t token, uint64_t head, int heads) {
            return Runs{reinterpret_cast<uint64_t>(at), static_cast<uint64_t>(n), token * es, static_cast<uint64_t>(heads), head * es, head_bytes};
        };
        const Runs k = runs(d_k, k_token_stride, k_head_stride, layer->heads), v = runs(d_v, v_token_stride, v_head_stride, layer->heads);
        if (!fits(k) || !fits(v)) return static_cast<int>(JB_ERR_INVALID_ARG);
        // what is read and what is written share no byte, but for queries that are turned where they are
        const uint64_t page = static_cast<uint64_t>(layer->heads) * layer->head_dim * p.page_tokens;
        const uint64_t cache_bytes = (layer->page_stride * (p.n_pages - 1) + page) * es;
        const Runs pools[2] = {{reinterpret_cast<uint64_t>(layer->k), 1, 0, 1, 0, cache_bytes}, {reinterpret_cast<uint64_t>(layer->v), 1, 0, 1, 0, cache_bytes}};
        for (const Runs& pool : pools)
            if (!apart(k, pool) || !apart(v, pool)) return static_cast<int>(JB_ERR_INVALID_ARG);
        if (q_heads > 0) {
            if (!aligned(d_q, 16) || !aligned(d_q_out, 16)) return static_cast<int>(JB_ERR_MISALIGNED);
            JB_TRY(check_strides(q_token_stride, q_head_stride, es));
            JB_TRY(check_strides(out_token_stride, out_head_stride, es));
            const Runs q = runs(d_q, q_token_stride, q_head_stride, q_heads), out = runs(d_q_out, out_token_stride, out_head_stride, q_heads);
            if (!fits(q) || !fits(out)) return static_cast<int>(JB_ERR_INVALID_ARG);
            if (outputs_overlap(n, out_token_stride, q_heads, out_head_stride, layer->head_dim)) return static_cast<int>(JB_ERR_INVALID_ARG);
            const bool in_place = q.base == out.base && (n == 1 || q.row == out.row) && (q_heads == 1 || q.head == out.head);
            if ((!in_place && !apart(q, out)) || !apart(k, out) || !apart(v, out)) return static_cast<int>(JB_ERR_INVALID_ARG);
            for (const Runs& pool : pools)
                if (!apart(q, pool) || !apart(out, pool)) return static_cast<int>(JB_ERR_INVALID_ARG);
        }
        Append a;
        a.from[0] = static_cast<const char*>(d_q);
        a.from[1] = static_cast<const char*>(d_k);
        a.from[2] = static_cast<const char*>(d_v);
        a.token_stride[0] = q_token_stride * es;
        a.token_stride[1] = k_token_stride * es;
        a.token_stride[2] = v_token_stride * es;
        a.head_stride[0] = q_head_stride * es;
        a.head_stride[1] = k_head_stride * es;
        a.head_stride[2] = v_head_stride * es;
        a.q_out = static_cast<char*>(d_q_out);
        a.out_token = out_token_stride * es;
        a.out_head = out_head_stride * es;
        a.to[0] = static_cast<char*>(layer->k);
        a.to[1] = static_cast<char*>(layer->v);
        a.page_stride = layer->page_stride * es;
        a.to_head = head_bytes * (layer->by_token ? 1 : p.page_tokens);
        a.to_token = head_bytes * (layer->by_token ? layer->heads : 1);
        a.steps = rotation->steps;
        a.rows = d_rows;
        a.pos = d_pos;
        a.turns = turns;
        a.n = n;
        a.q_heads = q_heads;
        a.heads = layer->heads;
        a.head_dim = layer->head_dim;
        a.dims = rotation->dims;
        a.interleaved = rotation->interleaved != 0;
        a.bf16 = layer->dtype == JB_BF16;
        return cuda_status(launch_append(p, a, stream));
    });
}

JB_EXPORT uint64_t jb_cache_keep_workspace(const jb_trees* trees) {
    Trees t;
    return check_trees(trees, t) == JB_OK ? 4 * keep_words(t.n, t.n_nodes) : 0;
}

JB_EXPORT int jb_cache_keep(const jb_pages* pages, const jb_kv* layers, int n_layers, const jb_trees* trees, const int32_t* d_leaves,
                            int32_t* d_status, void* workspace, uint64_t workspace_bytes, struct CUstream_st* stream) {
    return guarded([&] {
        Pages p;
        Trees t;
        JB_TRY(check_pages(pages, p));
        JB_TRY(check_layers(layers, n_layers, p));
        JB_TRY(check_trees(trees, t));
        if (d_status == nullptr || (t.n > 0 && d_leaves == nullptr)) return static_cast<int>(JB_ERR_INVALID_ARG);
        if (!aligned(d_status, 4) || !aligned(d_leaves, 4)) return static_cast<int>(JB_ERR_MISALIGNED);
        if (t.n == 0) return cuda_status(cudaMemsetAsync(d_status, 0, 4, stream));
        JB_TRY(check_workspace(workspace, workspace_bytes, 4 * keep_words(t.n, t.n_nodes)));
        int* ws = static_cast<int*>(workspace);
        JB_TRY(cuda_status(launch_keep_plan(p, t, d_leaves, d_status, ws, stream)));
        return for_pools(layers, n_layers, [&](const Pools& pools, bool) { return launch_keep_move(p, t, pools, ws, stream); });
    });
}

JB_EXPORT uint64_t jb_attend_tree_workspace(const jb_kv* layer) {
    if (layer == nullptr || layer->head_dim < 1 || layer->head_dim > kMaxHeadDim) return 0;
    return tree_workspace(layer->dtype == JB_BF16, layer->head_dim);
}

JB_EXPORT int jb_attend_tree(const jb_pages* pages, const jb_kv* layer, const jb_scores* scores, const jb_trees* trees, const void* d_q,
                             uint64_t q_row_stride, uint64_t q_head_stride, int q_heads, void* d_out, uint64_t out_row_stride,
                             uint64_t out_head_stride, void* workspace, uint64_t workspace_bytes, struct CUstream_st* stream) {
    return guarded([&] {
        Pages p;
        Trees t;
        JB_TRY(check_pages(pages, p));
        if (layer == nullptr) return static_cast<int>(JB_ERR_INVALID_ARG);
        JB_TRY(check_layer(*layer, p));
        JB_TRY(check_scores(scores));
        JB_TRY(check_trees(trees, t));
        if (q_heads < 1 || q_heads > 65536 || q_heads % layer->heads != 0) return static_cast<int>(JB_ERR_INVALID_ARG);
        if (t.n == 0 || t.n_nodes == 0) return static_cast<int>(JB_OK);
        if (d_q == nullptr || d_out == nullptr) return static_cast<int>(JB_ERR_INVALID_ARG);
        if (!aligned(d_q, 16) || !aligned(d_out, 16) || !aligned(scores->slopes, 4)) return static_cast<int>(JB_ERR_MISALIGNED);
        const uint64_t es = size_of(layer->dtype);
        JB_TRY(check_strides(q_row_stride, q_head_stride, es));
        JB_TRY(check_strides(out_row_stride, out_head_stride, es));
        const Runs q = {reinterpret_cast<uint64_t>(d_q), static_cast<uint64_t>(t.n_nodes), q_row_stride * es, static_cast<uint64_t>(q_heads),
                        q_head_stride * es, layer->head_dim * es};
        const Runs out = {reinterpret_cast<uint64_t>(d_out), static_cast<uint64_t>(t.n_nodes), out_row_stride * es, static_cast<uint64_t>(q_heads),
                          out_head_stride * es, layer->head_dim * es};
        if (!fits(q) || !fits(out)) return static_cast<int>(JB_ERR_INVALID_ARG);
        // outputs that share bytes would hold whichever was written last; a query may be read after another's output is written
        if (outputs_overlap(t.n_nodes, out_row_stride, q_heads, out_head_stride, layer->head_dim) || !apart(q, out))
            return static_cast<int>(JB_ERR_INVALID_ARG);
        JB_TRY(check_workspace(workspace, workspace_bytes, jb_attend_tree_workspace(layer)));
        TreeAttend a;
        a.q = static_cast<const char*>(d_q);
        a.out = static_cast<char*>(d_out);
        a.q_row = q_row_stride;
        a.q_head = q_head_stride;
        a.out_row = out_row_stride;
        a.out_head = out_head_stride;
        a.k = static_cast<const char*>(layer->k);
        a.v = static_cast<const char*>(layer->v);
        a.page_stride = layer->page_stride;
        a.head_stride = static_cast<uint64_t>(layer->head_dim) * (layer->by_token ? 1 : p.page_tokens);
        a.token_stride = static_cast<uint64_t>(layer->head_dim) * (layer->by_token ? layer->heads : 1);
        a.slopes = scores->slopes;
        a.ws = static_cast<float*>(workspace);
        a.scale = scores->scale;
        a.softcap = scores->softcap;
        a.window = scores->window;
        a.heads = layer->heads;
        a.group = q_heads / layer->heads;
        a.head_dim = layer->head_dim;
        a.bf16 = layer->dtype == JB_BF16;
        return cuda_status(launch_tree(p, t, a, stream));
    });
}

JB_EXPORT uint64_t jb_q4_matmul_workspace(int out_features, int in_features, int dtype, int n) {
    if ((dtype != JB_F32 && dtype != JB_BF16) || out_features < 1 || out_features > kMaxOutputs || in_features < 64 || in_features % 64 != 0 || in_features > kMaxInner || n < 0 || n > kMaxMatmulRows) return 0;
    return q4_workspace(n, out_features, in_features, dtype == JB_BF16);
}

JB_EXPORT int jb_q4_matmul(const jb_q4_segment* weights, int out_features, int in_features, int dtype, const void* d_x, uint64_t x_row_stride,
                           int n, const void* d_bias, void* d_y, uint64_t y_row_stride, void* workspace, uint64_t workspace_bytes,
                           struct CUstream_st* stream) {
    return guarded([&] {
        if (dtype != JB_F32 && dtype != JB_BF16) return static_cast<int>(JB_ERR_UNSUPPORTED_DTYPE);
        if (weights == nullptr || out_features < 1 || out_features > kMaxOutputs || in_features < 64 || in_features % 64 != 0 || in_features > kMaxInner || n < 0 || n > kMaxMatmulRows ||
            x_row_stride > (1ull << 48) || y_row_stride > (1ull << 48))
            return static_cast<int>(JB_ERR_INVALID_ARG);
        if (weights->numel != static_cast<uint64_t>(out_features) * in_features) return static_cast<int>(JB_ERR_INVALID_ARG);
        if (n == 0) return static_cast<int>(JB_OK);
        if (weights->codes == nullptr || weights->scale == nullptr || d_x == nullptr || d_y == nullptr) return static_cast<int>(JB_ERR_INVALID_ARG);
        const uint64_t es = size_of(dtype);
        if (!aligned(weights->codes, 8) || !aligned(weights->scale, 4) || !aligned(d_x, 16) || x_row_stride * es % 16 != 0 || !aligned(d_y, es) ||
            !aligned(d_bias, es))
            return static_cast<int>(JB_ERR_MISALIGNED);
        const Runs x = {reinterpret_cast<uint64_t>(d_x), static_cast<uint64_t>(n), x_row_stride * es, 1, 0, in_features * es};
        const Runs y = {reinterpret_cast<uint64_t>(d_y), static_cast<uint64_t>(n), y_row_stride * es, 1, 0, out_features * es};
        const Runs bias = {reinterpret_cast<uint64_t>(d_bias), 1, 0, 1, 0, out_features * es};
        const Runs codes = {reinterpret_cast<uint64_t>(weights->codes), 1, 0, 1, 0, weights->numel / 2};
        const Runs scale = {reinterpret_cast<uint64_t>(weights->scale), 1, 0, 1, 0, weights->numel / 16};
        if (!fits(x) || !fits(y) || !fits(bias) || !fits(codes) || !fits(scale)) return static_cast<int>(JB_ERR_INVALID_ARG);
        if ((n > 1 && y_row_stride < static_cast<uint64_t>(out_features)) || !apart(x, y) || !apart(codes, y) || !apart(scale, y) ||
            (d_bias != nullptr && !apart(bias, y)))
            return static_cast<int>(JB_ERR_INVALID_ARG);
        const uint64_t need = q4_workspace(n, out_features, in_features, dtype == JB_BF16);
        if (need > 0) JB_TRY(check_workspace(workspace, workspace_bytes, need));
        const Q4Matmul m = {weights->codes, weights->scale, d_x, d_bias, d_y, x_row_stride, y_row_stride, workspace, n, out_features, in_features, dtype == JB_BF16};
        return cuda_status(launch_q4_matmul(m, stream));
    });
}
