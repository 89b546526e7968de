// jb_check.h -- argument checks that the entry points of jb_answer_capi.cpp and jb_draft_capi.cpp share.
#pragma once
#include <cmath>
#include <cstdint>

#include "jb.h"
#include "jb_answer.h"
#include "jb_host.h"

#define JB_TRY(x)                     \
    do {                              \
        const int rc_ = (x);          \
        if (rc_ != JB_OK) return rc_; \
    } while (0)

namespace jb {

inline bool aligned(const void* p, uint64_t to) { return reinterpret_cast<uint64_t>(p) % to == 0; }

inline int check_pages(const jb_pages* in, Pages& out) {
    if (in == nullptr || in->table == nullptr || in->lens == nullptr || in->refs == nullptr) return JB_ERR_INVALID_ARG;
    if (in->n_rows < 1 || in->n_rows > kMaxRows || in->row_pages < 1 || in->n_pages < 1) return JB_ERR_INVALID_ARG;
    if (in->page_tokens < 16 || in->page_tokens > 1024 || in->page_tokens % 16 != 0) return JB_ERR_INVALID_ARG;
    if (static_cast<int64_t>(in->row_pages) * in->page_tokens > INT32_MAX) return JB_ERR_INVALID_ARG;
    if (in->n_pages > (1 << 30)) return JB_ERR_INVALID_ARG;
    if (!aligned(in->table, 4) || !aligned(in->lens, 4) || !aligned(in->refs, 4)) return JB_ERR_MISALIGNED;
    out = {in->table, in->lens, in->refs, in->n_rows, in->row_pages, in->n_pages, in->page_tokens};
    return JB_OK;
}

inline int check_list(const int32_t* a, const int32_t* b, int n, int most) {
    if (n < 0 || n > most || (n > 0 && (a == nullptr || b == nullptr))) return JB_ERR_INVALID_ARG;
    return aligned(a, 4) && aligned(b, 4) ? JB_OK : JB_ERR_MISALIGNED;
}

inline uint64_t size_of(int dtype) { return dtype == JB_F32 ? 4 : 2; }

inline int check_layer(const jb_kv& l, const Pages& p) {
    if (l.dtype != JB_F32 && l.dtype != JB_BF16) return JB_ERR_UNSUPPORTED_DTYPE;
    if (l.k == nullptr || l.v == nullptr || l.heads < 1 || l.heads > 65536 || l.head_dim < 1 || l.head_dim > kMaxHeadDim)
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
inline int check_layers(const jb_kv* layers, int n, const Pages& p) {
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
    for (int first = 0; first < n; first += kLayersPerLaunch) {
        Pools pools;
        pools.stride = l.page_stride * es;
        pools.slabs = l.by_token ? 1 : l.heads;
        pools.row_vecs = static_cast<uint32_t>((l.by_token ? l.heads : 1) * (l.head_dim * es / 16));
        pools.n = 0;
        for (int i = first; i < n && i < first + kLayersPerLaunch; ++i) {
            pools.base[pools.n++] = static_cast<char*>(layers[i].k);
            pools.base[pools.n++] = static_cast<char*>(layers[i].v);
        }
        const int rc = cuda_status(f(pools, first == 0));
        if (rc != JB_OK) return rc;
    }
    return JB_OK;
}

inline int check_scores(const jb_scores* s) {
    if (s == nullptr || !std::isfinite(s->scale) || !std::isfinite(s->softcap) || s->softcap < 0.0f || s->window < 0) return JB_ERR_INVALID_ARG;
    if (s->softcap > 0.0f && (s->softcap > 1e30f || !std::isfinite(s->scale / s->softcap))) return JB_ERR_INVALID_ARG;
    return JB_OK;
}

inline int check_workspace(const void* ws, uint64_t have, uint64_t need) {
    if (ws == nullptr || have < need) return JB_ERR_INVALID_ARG;
    return aligned(ws, 16) ? JB_OK : JB_ERR_MISALIGNED;
}

inline int check_strides(uint64_t a, uint64_t b, uint64_t es) {
    if (a > (1ull << 48) || b > (1ull << 48)) return JB_ERR_INVALID_ARG;
    return a * es % 16 == 0 && b * es % 16 == 0 ? JB_OK : JB_ERR_MISALIGNED;
}

// Whether two of `na` x `nb` runs of `len` elements at i * sa + j * sb share some: those of (i, j) and (i2, j2) do if
// (i - i2) sa and (j2 - j) sb are less than `len` apart. Counts are below 2^31, one of them at most 2^16, and strides at
// most 2^48, so that no product with the smaller count wraps.
inline bool outputs_overlap(uint64_t na, uint64_t sa, uint64_t nb, uint64_t sb, uint64_t len) {
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

}  // namespace jb
