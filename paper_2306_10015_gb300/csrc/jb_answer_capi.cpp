// jb_answer_capi.cpp -- the entry points that write answers with the perturbed model (declared in
// include/jb.h): argument checks and launches. Lengths, page tables and counts stay on the device;
// the kernels themselves check what they read there.
#include <cmath>

#include "jb.h"
#include "jb_answer.h"
#include "jb_host.h"

namespace {

using jb::cuda_status;
using jb::guarded;
using jb::range_fits;

bool aligned(const void* p, uint64_t to) { return reinterpret_cast<uint64_t>(p) % to == 0; }

int check_pages(const jb_pages* in, jb::Pages& out) {
    if (in == nullptr || in->table == nullptr || in->lens == nullptr || in->refs == nullptr) return JB_ERR_INVALID_ARG;
    if (in->n_rows < 1 || in->n_rows > jb::kMaxRows || in->row_pages < 1 || in->n_pages < 1) return JB_ERR_INVALID_ARG;
    if (in->page_tokens < 16 || in->page_tokens > 1024 || in->page_tokens % 16 != 0) return JB_ERR_INVALID_ARG;
    if (static_cast<int64_t>(in->row_pages) * in->page_tokens > INT32_MAX) return JB_ERR_INVALID_ARG;
    if (in->n_pages > (1 << 30)) return JB_ERR_INVALID_ARG;
    if (!aligned(in->table, 4) || !aligned(in->lens, 4) || !aligned(in->refs, 4)) return JB_ERR_MISALIGNED;
    out = {in->table, in->lens, in->refs, in->n_rows, in->row_pages, in->n_pages, in->page_tokens};
    return JB_OK;
}

int check_list(const int32_t* a, const int32_t* b, int n, int most) {
    if (n < 0 || n > most || (n > 0 && (a == nullptr || b == nullptr))) return JB_ERR_INVALID_ARG;
    return aligned(a, 4) && aligned(b, 4) ? JB_OK : JB_ERR_MISALIGNED;
}

uint64_t size_of(int dtype) { return dtype == JB_F32 ? 4 : 2; }

int check_layer(const jb_kv& l, const jb::Pages& p) {
    if (l.dtype != JB_F32 && l.dtype != JB_BF16) return JB_ERR_UNSUPPORTED_DTYPE;
    if (l.k == nullptr || l.v == nullptr || l.heads < 1 || l.heads > 65536 || l.head_dim < 1 || l.head_dim > jb::kMaxHeadDim)
        return JB_ERR_INVALID_ARG;
    const uint64_t es = size_of(l.dtype);
    if (l.head_dim * es % 16 != 0 || l.page_stride % (16 / es) != 0 || !aligned(l.k, 16) || !aligned(l.v, 16))
        return JB_ERR_MISALIGNED;
    const uint64_t page = static_cast<uint64_t>(l.heads) * l.head_dim * p.page_tokens;
    if (l.page_stride < page || l.page_stride > (1ull << 62) / es / p.n_pages || l.heads * (l.head_dim * es / 16) > (1u << 20))
        return JB_ERR_INVALID_ARG;
    const uint64_t span = l.page_stride * (p.n_pages - 1) + page;
    if (!range_fits(reinterpret_cast<uint64_t>(l.k), span, es) || !range_fits(reinterpret_cast<uint64_t>(l.v), span, es))
        return JB_ERR_INVALID_ARG;
    return JB_OK;
}

// Checks all layers; they have to share their geometry.
int check_layers(const jb_kv* layers, int n, const jb::Pages& p) {
    if (n < 1 || layers == nullptr) return JB_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i) {
        const int rc = check_layer(layers[i], p);
        if (rc != JB_OK) return rc;
        if (layers[i].heads != layers[0].heads || layers[i].head_dim != layers[0].head_dim || layers[i].dtype != layers[0].dtype ||
            (layers[i].by_token != 0) != (layers[0].by_token != 0) || layers[i].page_stride != layers[0].page_stride)
            return JB_ERR_INVALID_ARG;
    }
    return JB_OK;
}

// Calls f with the pools of up to kLayersPerLaunch layers at a time.
template <typename F>
int for_pools(const jb_kv* layers, int n, F f) {
    const jb_kv& l = layers[0];
    const uint64_t es = size_of(l.dtype);
    for (int first = 0; first < n; first += jb::kLayersPerLaunch) {
        jb::Pools pools;
        pools.stride = l.page_stride * es;
        pools.slabs = l.by_token ? 1 : l.heads;
        pools.row_vecs = static_cast<uint32_t>((l.by_token ? l.heads : 1) * (l.head_dim * es / 16));
        pools.n = 0;
        for (int i = first; i < n && i < first + jb::kLayersPerLaunch; ++i) {
            pools.base[pools.n++] = static_cast<char*>(layers[i].k);
            pools.base[pools.n++] = static_cast<char*>(layers[i].v);
        }
        const int rc = cuda_status(f(pools, first == 0));
        if (rc != JB_OK) return rc;
    }
    return JB_OK;
}

int check_workspace(const void* ws, uint64_t have, uint64_t need) {
    if (ws == nullptr || have < need) return JB_ERR_INVALID_ARG;
    return aligned(ws, 16) ? JB_OK : JB_ERR_MISALIGNED;
}

int check_strides(uint64_t a, uint64_t b, uint64_t es) {
    if (a > (1ull << 48) || b > (1ull << 48)) return JB_ERR_INVALID_ARG;
    return a * es % 16 == 0 && b * es % 16 == 0 ? JB_OK : JB_ERR_MISALIGNED;
}

// Whether two of `na` x `nb` runs of `len` elements at i * sa + j * sb share some: those of (i, j) and (i2, j2) do if
// (i - i2) sa and (j2 - j) sb are less than `len` apart. Counts are below 2^31, one of them at most 2^16, and strides at
// most 2^48, so that no product with the smaller count wraps.
bool outputs_overlap(uint64_t na, uint64_t sa, uint64_t nb, uint64_t sb, uint64_t len) {
    if ((na > 1 && sa < len) || (nb > 1 && sb < len)) return true;
    if (na < 2 || nb < 2) return false;
    if (na < nb) return outputs_overlap(nb, sb, na, sa, len);
    if (sa >= (nb - 1) * sb + len || sb / sa >= na) return false;  // one within the other, as a row holds its heads
    for (uint64_t j = 1; j < nb; ++j) {                            // the two i's nearest to j
        const uint64_t i = j * sb / sa, past = j * sb % sa;
        if ((i < na && past < len) || (i + 1 < na && sa - past < len)) return true;
    }
    return false;
}

#define JB_TRY(x)                     \
    do {                              \
        const int rc_ = (x);          \
        if (rc_ != JB_OK) return rc_; \
    } while (0)

}  // namespace

JB_EXPORT int jb_cache_reserve(const jb_pages* pages, const int32_t* d_rows, const int32_t* d_tokens, int n,
                               int32_t* d_status, struct CUstream_st* stream) {
    return guarded([&] {
        jb::Pages p;
        JB_TRY(check_pages(pages, p));
        JB_TRY(check_list(d_rows, d_tokens, n, jb::kMaxListed));
        if (d_status == nullptr) return static_cast<int>(JB_ERR_INVALID_ARG);
        if (!aligned(d_status, 4)) return static_cast<int>(JB_ERR_MISALIGNED);
        if (n == 0) return cuda_status(cudaMemsetAsync(d_status, 0, 4, stream));
        return cuda_status(jb::launch_reserve(p, d_rows, d_tokens, n, d_status, stream));
    });
}

JB_EXPORT int jb_cache_free(const jb_pages* pages, const int32_t* d_rows, int n, struct CUstream_st* stream) {
    return guarded([&] {
        jb::Pages p;
        JB_TRY(check_pages(pages, p));
        JB_TRY(check_list(d_rows, d_rows, n, INT32_MAX));
        if (n == 0) return static_cast<int>(JB_OK);
        return cuda_status(jb::launch_free(p, d_rows, n, stream));
    });
}

JB_EXPORT uint64_t jb_cache_workspace(const jb_pages* pages, int n) {
    jb::Pages p;
    if (check_pages(pages, p) != JB_OK || n < 0) return 0;
    return 4 * (n > 0 ? jb::fork_words(p, n) : jb::compact_words(p));
}

JB_EXPORT int jb_cache_fork(const jb_pages* pages, const jb_kv* layers, int n_layers, const int32_t* d_parents,
                            const int32_t* d_children, int n, int32_t* d_status, void* workspace,
                            uint64_t workspace_bytes, struct CUstream_st* stream) {
    return guarded([&] {
        jb::Pages p;
        JB_TRY(check_pages(pages, p));
        JB_TRY(check_layers(layers, n_layers, p));
        JB_TRY(check_list(d_parents, d_children, n, jb::kMaxListed));
        if (d_status == nullptr) return static_cast<int>(JB_ERR_INVALID_ARG);
        if (!aligned(d_status, 4)) return static_cast<int>(JB_ERR_MISALIGNED);
        if (n == 0) return cuda_status(cudaMemsetAsync(d_status, 0, 4, stream));
        JB_TRY(check_workspace(workspace, workspace_bytes, 4 * jb::fork_words(p, n)));
        int* ws = static_cast<int*>(workspace);
        JB_TRY(cuda_status(jb::launch_fork_plan(p, d_parents, d_children, n, d_status, ws, stream)));
        return for_pools(layers, n_layers, [&](const jb::Pools& pools, bool) { return jb::launch_fork_copy(p, pools, n, ws, stream); });
    });
}

JB_EXPORT int jb_cache_compact(const jb_pages* pages, const jb_kv* layers, int n_layers, int32_t* d_status,
                               void* workspace, uint64_t workspace_bytes, struct CUstream_st* stream) {
    return guarded([&] {
        jb::Pages p;
        JB_TRY(check_pages(pages, p));
        JB_TRY(check_layers(layers, n_layers, p));
        if (!aligned(d_status, 4)) return static_cast<int>(JB_ERR_MISALIGNED);
        JB_TRY(check_workspace(workspace, workspace_bytes, 4 * jb::compact_words(p)));
        int* ws = static_cast<int*>(workspace);
        JB_TRY(cuda_status(jb::launch_compact_plan(p, d_status, ws, stream)));
        return for_pools(layers, n_layers, [&](const jb::Pools& pools, bool first) {
            return jb::launch_compact_move(p, pools, first, ws, stream);
        });
    });
}

JB_EXPORT int jb_cache_write(const jb_pages* pages, const jb_kv* layer, const void* d_k, uint64_t k_token_stride,
                             uint64_t k_head_stride, const void* d_v, uint64_t v_token_stride, uint64_t v_head_stride,
                             const int32_t* d_rows, const int32_t* d_pos, int n, struct CUstream_st* stream) {
    return guarded([&] {
        jb::Pages p;
        JB_TRY(check_pages(pages, p));
        if (layer == nullptr) return static_cast<int>(JB_ERR_INVALID_ARG);
        JB_TRY(check_layer(*layer, p));
        JB_TRY(check_list(d_rows, d_pos, n, INT32_MAX));
        if (n == 0) return static_cast<int>(JB_OK);
        if (d_k == nullptr || d_v == nullptr) return static_cast<int>(JB_ERR_INVALID_ARG);
        if (!aligned(d_k, 16) || !aligned(d_v, 16)) return static_cast<int>(JB_ERR_MISALIGNED);
        const uint64_t es = size_of(layer->dtype);
        JB_TRY(check_strides(k_token_stride, k_head_stride, es));
        JB_TRY(check_strides(v_token_stride, v_head_stride, es));
        jb::Write w;
        w.from[0] = static_cast<const char*>(d_k);
        w.from[1] = static_cast<const char*>(d_v);
        w.token_stride[0] = k_token_stride * es;
        w.token_stride[1] = v_token_stride * es;
        w.head_stride[0] = k_head_stride * es;
        w.head_stride[1] = v_head_stride * es;
        w.to[0] = static_cast<char*>(layer->k);
        w.to[1] = static_cast<char*>(layer->v);
        w.page_stride = layer->page_stride * es;
        w.to_head = layer->head_dim * es * (layer->by_token ? 1 : p.page_tokens);
        w.to_token = layer->head_dim * es * (layer->by_token ? layer->heads : 1);
        w.rows = d_rows;
        w.pos = d_pos;
        w.n = n;
        w.heads = layer->heads;
        w.head_vecs = static_cast<uint32_t>(layer->head_dim * es / 16);
        w.magic = ((1ull << 32) + w.head_vecs - 1) / w.head_vecs;
        return cuda_status(jb::launch_write(p, w, stream));
    });
}

JB_EXPORT uint64_t jb_attend_workspace(const jb_kv* layer, int q_heads) {
    if (layer == nullptr || layer->heads < 1 || q_heads < layer->heads || layer->head_dim < 1 || layer->head_dim > jb::kMaxHeadDim)
        return 0;
    return jb::attend_workspace(layer->dtype == JB_BF16, q_heads / layer->heads, layer->head_dim);
}

JB_EXPORT int jb_attend(const jb_pages* pages, const jb_kv* layer, const jb_scores* scores, const void* d_q,
                        uint64_t q_row_stride, uint64_t q_head_stride, int q_heads, const int32_t* d_rows,
                        const int32_t* d_pos, int n, void* d_out, uint64_t out_row_stride, uint64_t out_head_stride,
                        void* workspace, uint64_t workspace_bytes, struct CUstream_st* stream) {
    return guarded([&] {
        jb::Pages p;
        JB_TRY(check_pages(pages, p));
        if (layer == nullptr || scores == nullptr) return static_cast<int>(JB_ERR_INVALID_ARG);
        JB_TRY(check_layer(*layer, p));
        if (q_heads < 1 || q_heads > 65536 || q_heads % layer->heads != 0) return static_cast<int>(JB_ERR_INVALID_ARG);
        if (!std::isfinite(scores->scale) || !std::isfinite(scores->softcap) || scores->softcap < 0.0f || scores->window < 0)
            return static_cast<int>(JB_ERR_INVALID_ARG);
        if (scores->softcap > 0.0f && (scores->softcap > 1e30f || !std::isfinite(scores->scale / scores->softcap)))
            return static_cast<int>(JB_ERR_INVALID_ARG);
        JB_TRY(check_list(d_rows, d_pos, n, INT32_MAX));
        if (n == 0) return static_cast<int>(JB_OK);
        if (d_q == nullptr || d_out == nullptr) return static_cast<int>(JB_ERR_INVALID_ARG);
        if (!aligned(d_q, 16) || !aligned(d_out, 16) || !aligned(scores->slopes, 4)) return static_cast<int>(JB_ERR_MISALIGNED);
        const uint64_t es = size_of(layer->dtype);
        JB_TRY(check_strides(q_row_stride, q_head_stride, es));
        JB_TRY(check_strides(out_row_stride, out_head_stride, es));
        // outputs that share bytes would hold whichever was written last
        if (outputs_overlap(n, out_row_stride, q_heads, out_head_stride, layer->head_dim)) return static_cast<int>(JB_ERR_INVALID_ARG);
        JB_TRY(check_workspace(workspace, workspace_bytes, jb_attend_workspace(layer, q_heads)));
        jb::Attend a;
        a.k = static_cast<const char*>(layer->k);
        a.v = static_cast<const char*>(layer->v);
        a.q_row = q_row_stride;
        a.q_head = q_head_stride;
        a.out_row = out_row_stride;
        a.out_head = out_head_stride;
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
        for (int64_t first = 0; first < n; first += jb::kMaxListed) {
            a.q = static_cast<const char*>(d_q) + static_cast<uint64_t>(first) * q_row_stride * es;
            a.out = static_cast<char*>(d_out) + static_cast<uint64_t>(first) * out_row_stride * es;
            a.rows = d_rows + first;
            a.pos = d_pos + first;
            a.n = static_cast<int>(n - first < jb::kMaxListed ? n - first : jb::kMaxListed);
            JB_TRY(cuda_status(jb::launch_attend(p, a, stream)));
        }
        return static_cast<int>(JB_OK);
    });
}

JB_EXPORT int jb_sample(const void* d_logits, uint64_t row_stride, int dtype, int n, int vocab,
                        const jb_sampling* sampling, const uint32_t* d_words, int32_t* d_tokens, float* d_logprobs,
                        struct CUstream_st* stream) {
    return guarded([&] {
        if (dtype != JB_F32 && dtype != JB_BF16) return static_cast<int>(JB_ERR_UNSUPPORTED_DTYPE);
        if (n < 0 || vocab < 1 || vocab > jb::kMaxVocab || sampling == nullptr || row_stride > (1ull << 48))
            return static_cast<int>(JB_ERR_INVALID_ARG);
        if (n == 0) return static_cast<int>(JB_OK);
        if (d_logits == nullptr || d_words == nullptr || d_tokens == nullptr) return static_cast<int>(JB_ERR_INVALID_ARG);
        if (!aligned(d_logits, size_of(dtype)) || !aligned(d_words, 4) || !aligned(d_tokens, 4) || !aligned(d_logprobs, 4) ||
            !aligned(sampling->temperature, 4) || !aligned(sampling->top_k, 4) || !aligned(sampling->top_p, 4) || !aligned(sampling->min_p, 4))
            return static_cast<int>(JB_ERR_MISALIGNED);
        const jb::Sample p = {d_logits, row_stride, dtype == JB_BF16, n, vocab, sampling->temperature, sampling->top_k,
                              sampling->top_p, sampling->min_p, d_words, d_tokens, d_logprobs};
        return cuda_status(jb::launch_sample(p, stream));
    });
}
