// The C ABI of the 4-bit key/value cache: argument checks and launches.
#include <cmath>

#include "qp_kv_attention.hpp"

using namespace qp;

namespace qp {
#define QP_KV_EXTERN_DIM(D) \
    extern template hipError_t at_dim<D>(const KvLayer &, int, const KvView &, const KvView &, const KvAttn &, void *, hipStream_t)
QP_KV_EXTERN_DIM(64);
QP_KV_EXTERN_DIM(80);
QP_KV_EXTERN_DIM(96);
QP_KV_EXTERN_DIM(128);
QP_KV_EXTERN_DIM(256);
}  // namespace qp

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
qp_status hip_status(hipError_t e) { return e == hipSuccess ? QP_OK : QP_EHIP; }

bool sizes_ok(const qp_kv_cache_t *c)
{
    if (!c || c->reserved != 0u) return false;
    const uint32_t d = c->head_dim, t = c->page_tokens;
    if (d != 64u && d != 80u && d != 96u && d != 128u && d != 256u) return false;
    if (t != 32u && t != 64u && t != 128u && t != 256u) return false;
    return c->kv_heads >= 1u && c->kv_heads <= 1024u;
}
uint32_t page_shift(const qp_kv_cache_t *c)
{
    return c->page_tokens == 32u ? 5u : c->page_tokens == 64u ? 6u : c->page_tokens == 128u ? 7u : 8u;
}
uint64_t slab_bytes(const qp_kv_cache_t *c) { return (uint64_t)c->page_tokens * (c->head_dim + 16u); }

qp_status check_cache(const qp_kv_cache_t *c)
{
    if (!sizes_ok(c) || !c->pages_dev || !aligned16(c->pages_dev)) return QP_EINVAL;
    if (c->layers < 1u || c->layers > 65536u || c->n_pages < 1u || c->n_pages > kKvMaxPages) return QP_EINVAL;
    // at most 2^16 layers x 2^24 pages x 2^27 bytes of a page: compared in parts that fit 64 bits
    const uint64_t pages = (uint64_t)c->layers * c->n_pages, page = slab_bytes(c) * c->kv_heads;
    return c->pages_bytes / page >= pages ? QP_OK : QP_ENOSPC;
}
qp_status check_rows(const qp_kv_cache_t *c, const qp_kv_rows_t *r)
{
    if (!r || !r->table_dev || !r->lengths_dev || !aligned4(r->table_dev) || !aligned4(r->lengths_dev)) return QP_EINVAL;
    if (r->rows < 1u || r->rows > kKvMaxRows || r->pages_per_row < 1u) return QP_EINVAL;
    return (uint64_t)r->pages_per_row * c->page_tokens < (1ull << 31) ? QP_OK : QP_EINVAL;
}
qp_status check_pool(uint32_t n_pages, const void *pool, size_t bytes)
{
    if (!pool || !aligned4(pool)) return QP_EINVAL;
    return bytes >= qp_kv_pool_bytes(n_pages) ? QP_OK : QP_ENOSPC;
}
// What reserve, fork, free and compact have in common.
qp_status check_books(const qp_kv_cache_t *c, const qp_kv_rows_t *r, const void *pool, size_t bytes)
{
    qp_status st = check_cache(c);
    if (st != QP_OK) return st;
    if ((st = check_rows(c, r)) != QP_OK) return st;
    return check_pool(c->n_pages, pool, bytes);
}

bool dtype_ok(uint32_t d) { return d == QP_F32 || d == QP_BF16; }
qp_status check_view(const qp_kv_view_t *v, uint64_t tokens, uint64_t heads, uint32_t dim, bool written)
{
    if (!v || !v->data_dev || !aligned16(v->data_dev) || !dtype_ok(v->dtype) || v->reserved != 0u) return QP_EINVAL;
    const uint64_t unit = v->dtype == QP_F32 ? 4u : 8u;    // elements in 16 bytes
    if (v->token_stride % unit || v->head_stride % unit || v->token_stride >> 40 || v->head_stride >> 40) return QP_EINVAL;
    if (!written) return QP_OK;
    // no two elements at one place: tokens outside heads, or heads outside tokens
    const uint64_t t = v->token_stride, h = v->head_stride;
    const bool tokens_out = (heads == 1u || h >= dim) && (tokens == 1u || t >= (heads - 1u) * h + dim);
    const bool heads_out = (tokens == 1u || t >= dim) && (heads == 1u || h >= (tokens - 1u) * t + dim);
    return tokens_out || heads_out ? QP_OK : QP_EINVAL;
}
KvView view_of(const qp_kv_view_t *v)
{
    const uint64_t size = v->dtype == QP_F32 ? 4u : 2u;
    return KvView{static_cast<unsigned char *>(v->data_dev), v->token_stride * size, v->head_stride * size};
}

qp_status check_tokens(const qp_kv_cache_t *c, const qp_kv_rows_t *r, uint32_t layer, const int32_t *begin, uint64_t tokens, uint64_t heads)
{
    qp_status st = check_cache(c);
    if (st != QP_OK) return st;
    if ((st = check_rows(c, r)) != QP_OK) return st;
    if (layer >= c->layers || !begin || !aligned4(begin)) return QP_EINVAL;
    return tokens < (1ull << 31) && tokens * heads < (1ull << 31) ? QP_OK : QP_EINVAL;
}
KvLayer layer_of(const qp_kv_cache_t *c, const qp_kv_rows_t *r, uint32_t layer, const int32_t *begin, uint64_t tokens)
{
    KvLayer l;
    l.page_bytes = slab_bytes(c) * c->kv_heads;
    l.pages = static_cast<unsigned char *>(c->pages_dev) + (uint64_t)layer * c->n_pages * l.page_bytes;
    l.table = r->table_dev;
    l.lengths = r->lengths_dev;
    l.begin = begin;
    l.slab_bytes = (uint32_t)slab_bytes(c);
    l.n_pages = c->n_pages;
    l.rows = r->rows;
    l.pages_per_row = r->pages_per_row;
    l.kv_heads = c->kv_heads;
    l.tokens = (uint32_t)tokens;
    l.page_shift = page_shift(c);
    return l;
}
KvPages pages_of(const qp_kv_cache_t *c)
{
    KvPages p;
    p.pages = static_cast<unsigned char *>(c->pages_dev);
    p.page_bytes = slab_bytes(c) * c->kv_heads;
    p.layer_bytes = p.page_bytes * c->n_pages;
    p.layers = c->layers;
    p.n_pages = c->n_pages;
    p.page_shift = page_shift(c);
    return p;
}

}  // namespace

extern "C" {

size_t qp_kv_page_bytes(const qp_kv_cache_t *cache) { return sizes_ok(cache) ? (size_t)(slab_bytes(cache) * cache->kv_heads) : 0; }

size_t qp_kv_pool_bytes(uint32_t n_pages)
{
    return n_pages < 1u || n_pages > kKvMaxPages ? 0 : (QP_KV_POOL_HEADER + 6u * (size_t)n_pages) * sizeof(int32_t);
}

qp_status qp_kv_pool_init(uint32_t n_pages, void *pool_dev, size_t pool_bytes, void *stream)
{
    if (n_pages < 1u || n_pages > kKvMaxPages) return QP_EINVAL;
    const qp_status st = check_pool(n_pages, pool_dev, pool_bytes);
    if (st != QP_OK) return st;
    return hip_status(launch_kv_pool_init(n_pages, pool_dev, static_cast<hipStream_t>(stream)));
}

qp_status qp_kv_reserve(const qp_kv_cache_t *cache, const qp_kv_rows_t *rows, const int32_t *want_dev, void *pool_dev,
                        size_t pool_bytes, void *stream)
{
    const qp_status st = check_books(cache, rows, pool_dev, pool_bytes);
    if (st != QP_OK) return st;
    if (!want_dev || !aligned4(want_dev)) return QP_EINVAL;
    return hip_status(launch_kv_reserve(pages_of(cache), *rows, want_dev, pool_dev, static_cast<hipStream_t>(stream)));
}

qp_status qp_kv_fork(const qp_kv_cache_t *cache, const qp_kv_rows_t *rows, const int32_t *parent_dev, void *pool_dev,
                     size_t pool_bytes, void *stream)
{
    const qp_status st = check_books(cache, rows, pool_dev, pool_bytes);
    if (st != QP_OK) return st;
    if (!parent_dev || !aligned4(parent_dev)) return QP_EINVAL;
    return hip_status(launch_kv_fork(pages_of(cache), *rows, parent_dev, pool_dev, static_cast<hipStream_t>(stream)));
}

qp_status qp_kv_free(const qp_kv_cache_t *cache, const qp_kv_rows_t *rows, const int32_t *keep_dev, void *pool_dev,
                     size_t pool_bytes, void *stream)
{
    const qp_status st = check_books(cache, rows, pool_dev, pool_bytes);
    if (st != QP_OK) return st;
    if (!keep_dev || !aligned4(keep_dev)) return QP_EINVAL;
    return hip_status(launch_kv_free(pages_of(cache), *rows, keep_dev, pool_dev, static_cast<hipStream_t>(stream)));
}

qp_status qp_kv_compact(const qp_kv_cache_t *cache, const qp_kv_rows_t *rows, void *pool_dev, size_t pool_bytes, void *stream)
{
    const qp_status st = check_books(cache, rows, pool_dev, pool_bytes);
    if (st != QP_OK) return st;
    return hip_status(launch_kv_compact(pages_of(cache), *rows, pool_dev, static_cast<hipStream_t>(stream)));
}

qp_status qp_kv_append(const qp_kv_cache_t *cache, const qp_kv_rows_t *rows, uint32_t layer, const int32_t *token_begin_dev,
                       uint64_t tokens, const qp_kv_view_t *k, const qp_kv_view_t *v, void *stream)
{
    const qp_status st = check_tokens(cache, rows, layer, token_begin_dev, tokens, cache ? cache->kv_heads : 0u);
    if (st != QP_OK) return st;
    if (tokens == 0u) return QP_OK;
    if (check_view(k, tokens, cache->kv_heads, cache->head_dim, false) != QP_OK ||
        check_view(v, tokens, cache->kv_heads, cache->head_dim, false) != QP_OK || k->dtype != v->dtype)
        return QP_EINVAL;
    return hip_status(launch_kv_append(layer_of(cache, rows, layer, token_begin_dev, tokens), cache->head_dim, (int)k->dtype,
                                       view_of(k), view_of(v), static_cast<hipStream_t>(stream)));
}

qp_status qp_kv_read(const qp_kv_cache_t *cache, const qp_kv_rows_t *rows, uint32_t layer, const int32_t *token_begin_dev,
                     const int32_t *first_dev, uint64_t tokens, const qp_kv_view_t *k, const qp_kv_view_t *v, void *stream)
{
    const qp_status st = check_tokens(cache, rows, layer, token_begin_dev, tokens, cache ? cache->kv_heads : 0u);
    if (st != QP_OK) return st;
    if (!aligned4(first_dev)) return QP_EINVAL;
    if (tokens == 0u) return QP_OK;
    if (check_view(k, tokens, cache->kv_heads, cache->head_dim, true) != QP_OK ||
        check_view(v, tokens, cache->kv_heads, cache->head_dim, true) != QP_OK || k->dtype != v->dtype)
        return QP_EINVAL;
    return hip_status(launch_kv_read(layer_of(cache, rows, layer, token_begin_dev, tokens), cache->head_dim, (int)k->dtype,
                                     first_dev, view_of(k), view_of(v), static_cast<hipStream_t>(stream)));
}

size_t qp_kv_attention_workspace_bytes(const qp_kv_cache_t *cache, const qp_kv_rows_t *rows, uint64_t tokens, uint32_t q_heads)
{
    if (!sizes_ok(cache) || !rows || rows->rows < 1u || rows->rows > kKvMaxRows || rows->pages_per_row < 1u) return 0;
    if ((uint64_t)rows->pages_per_row * cache->page_tokens >= (1ull << 31)) return 0;
    if (q_heads == 0u || q_heads % cache->kv_heads || q_heads / cache->kv_heads > 1024u) return 0;
    if (tokens >= (1ull << 31) || tokens * q_heads >= (1ull << 31)) return 0;
    const KvLayer c = layer_of(cache, rows, 0, nullptr, tokens);
    size_t few;
    return at_bytes(c, cache->head_dim, q_heads / cache->kv_heads, few);
}

qp_status qp_kv_attention(const qp_kv_cache_t *cache, const qp_kv_rows_t *rows, uint32_t layer, const int32_t *token_begin_dev,
                          uint64_t tokens, const qp_kv_view_t *q, const qp_kv_view_t *out, const qp_kv_attn_cfg_t *cfg,
                          void *ws_dev, size_t ws_bytes, void *stream)
{
    if (!cfg || !cache) return QP_EINVAL;
    const qp_status st = check_tokens(cache, rows, layer, token_begin_dev, tokens, cfg->q_heads);
    if (st != QP_OK) return st;
    if (!(cfg->scale > 0.0f) || !std::isfinite(cfg->scale) || cfg->causal > 1u || cfg->window >> 31) return QP_EINVAL;
    if (cfg->window != 0u && cfg->causal == 0u) return QP_EINVAL;
    if (cfg->q_heads == 0u || cfg->q_heads % cache->kv_heads || cfg->q_heads / cache->kv_heads > 1024u) return QP_EINVAL;
    if (tokens == 0u) return QP_OK;
    if (check_view(q, tokens, cfg->q_heads, cache->head_dim, false) != QP_OK ||
        check_view(out, tokens, cfg->q_heads, cache->head_dim, true) != QP_OK || q->dtype != out->dtype)
        return QP_EINVAL;
    if (!ws_dev || !aligned16(ws_dev)) return QP_EINVAL;
    if (ws_bytes < qp_kv_attention_workspace_bytes(cache, rows, tokens, cfg->q_heads)) return QP_ENOSPC;
    const KvLayer c = layer_of(cache, rows, layer, token_begin_dev, tokens);
    const KvAttn a{cfg->scale, cfg->q_heads / cache->kv_heads, cfg->causal, cfg->window};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int dt = (int)q->dtype;
    switch (cache->head_dim) {
        case 64: return hip_status(at_dim<64>(c, dt, view_of(q), view_of(out), a, ws_dev, s));
        case 80: return hip_status(at_dim<80>(c, dt, view_of(q), view_of(out), a, ws_dev, s));
        case 96: return hip_status(at_dim<96>(c, dt, view_of(q), view_of(out), a, ws_dev, s));
        case 128: return hip_status(at_dim<128>(c, dt, view_of(q), view_of(out), a, ws_dev, s));
        default: return hip_status(at_dim<256>(c, dt, view_of(q), view_of(out), a, ws_dev, s));
    }
}

}  // extern "C"
