// C ABI of the paged cache and of the attention that reads it (see include/slimspec.h): argument checks on the host, then the launches.
#include "cache.hpp"

using namespace slimspec;

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool rows_aligned(int64_t stride) { return stride >= 0 && (stride & 7) == 0; }

// Checks a cache's description and, where it is right, says it the kernels' way.
int check_cache(const slimspec_cache *c, CacheView &out)
{
    if (!c || !c->k || !c->v || !c->table || !c->held || !c->lens || !c->refs) return SLIMSPEC_INVALID_ARGUMENT;
    if (c->layers < 1 || c->pages < 1 || c->heads < 1 || c->page_size < 1 || c->head_dim < 1 || c->slots < 1 || c->slot_pages < 1) return SLIMSPEC_INVALID_ARGUMENT;
    if (c->dtype != SLIMSPEC_BF16 && c->dtype != SLIMSPEC_F16) return SLIMSPEC_INVALID_ARGUMENT;
    if (c->layer_stride < 0 || c->page_stride < 0 || c->head_stride < c->head_dim || c->place_stride < c->head_dim) return SLIMSPEC_INVALID_ARGUMENT;
    if ((c->layers > 1 && c->layer_stride == 0) || (c->pages > 1 && c->page_stride == 0)) return SLIMSPEC_INVALID_ARGUMENT;
    if ((c->head_dim & 7) || c->head_dim > SLIMSPEC_CACHE_MAX_HEAD_DIM) return SLIMSPEC_UNSUPPORTED;
    if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1))) return SLIMSPEC_UNSUPPORTED;
    // index arithmetic: places and entries of a slot in 31 bits, elements in 64, a page's places from its first in 31 bits of bytes
    if ((int64_t)c->slot_pages * c->page_size >= (int64_t)1 << 31 || c->place_stride > (int64_t)1 << 20) return SLIMSPEC_UNSUPPORTED;
    if (c->layers > 1024 || c->heads > 1024) return SLIMSPEC_UNSUPPORTED;
    if (((c->layer_stride | c->page_stride | c->head_stride | c->place_stride) & 7)) return SLIMSPEC_UNSUPPORTED;
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->refs)) return SLIMSPEC_UNSUPPORTED;
    int shift = 0;
    while (1 << shift < c->page_size) ++shift;
    out = CacheView{static_cast<uint16_t *>(c->k), static_cast<uint16_t *>(c->v), c->layer_stride, c->page_stride, c->head_stride, c->place_stride,
                    c->table, c->held, c->lens, c->refs, c->layers, c->pages, c->heads, shift, c->head_dim, c->slots, c->slot_pages};
    return SLIMSPEC_OK;
}

int check_batch(const slimspec_batch *b, BatchView &out)
{
    if (!b || b->n < 0 || b->tokens < 0) return SLIMSPEC_INVALID_ARGUMENT;
    if (b->n > 0 && (!b->slots || !b->first)) return SLIMSPEC_INVALID_ARGUMENT;
    if (b->n > SLIMSPEC_CACHE_MAX_SEQUENCES) return SLIMSPEC_UNSUPPORTED;
    out = BatchView{b->slots, b->first, b->n, b->tokens};
    return SLIMSPEC_OK;
}

int done(hipError_t e) { return e == hipSuccess ? SLIMSPEC_OK : fail_hip(e); }

}  // namespace

extern "C" {

size_t slimspec_tree_attention_workspace_bytes(const slimspec_cache *cache, const slimspec_batch *batch, int32_t q_heads)
{
    CacheView c;
    if (check_cache(cache, c) != SLIMSPEC_OK || !batch || batch->n < 0 || batch->tokens < 0 || batch->n > SLIMSPEC_CACHE_MAX_SEQUENCES) return 0;
    if (q_heads < 1 || q_heads % c.heads || q_heads > 65535 || (int64_t)batch->tokens * q_heads >= (int64_t)1 << 31) return 0;
    return tree_attention_workspace_bytes(batch->n, batch->tokens, q_heads, c.heads, c.head_dim);
}

int slimspec_tree_attention(const slimspec_cache *cache, int32_t layer,
                            const void *q, int32_t q_heads, int64_t q_token_stride, int64_t q_head_stride,
                            const slimspec_batch *batch, const uint64_t *mask, int32_t mask_words, float scale,
                            void *out, int64_t out_token_stride, int64_t out_head_stride, float *lse,
                            void *workspace, size_t workspace_bytes, void *stream)
{
    CacheView c;
    BatchView b;
    int st = check_cache(cache, c);
    if (st != SLIMSPEC_OK) return st;
    if ((st = check_batch(batch, b)) != SLIMSPEC_OK) return st;
    if (layer < 0 || layer >= c.layers) return SLIMSPEC_INVALID_ARGUMENT;
    if (q_heads < 1 || q_heads % c.heads || !(scale - scale == 0.f)) return SLIMSPEC_INVALID_ARGUMENT;      // (a scale that is a finite number)
    if (mask && (mask_words < 1 || mask_words > SLIMSPEC_TREE_MAX_WORDS)) return SLIMSPEC_INVALID_ARGUMENT;
    if (q_token_stride < 0 || q_head_stride < 0 || out_token_stride < 0 || out_head_stride < 0) return SLIMSPEC_INVALID_ARGUMENT;
    if (q_heads > 65535 || (int64_t)b.tokens * q_heads >= (int64_t)1 << 31) return SLIMSPEC_UNSUPPORTED;       // query rows are counted in 31 bits
    if (!rows_aligned(q_token_stride) || !rows_aligned(q_head_stride) || !rows_aligned(out_token_stride) || !rows_aligned(out_head_stride)) return SLIMSPEC_UNSUPPORTED;
    if (b.n == 0 || b.tokens == 0) return SLIMSPEC_OK;
    if (!q || !out || !workspace) return SLIMSPEC_INVALID_ARGUMENT;
    if (!aligned16(q) || !aligned16(out) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return SLIMSPEC_UNSUPPORTED;
    if (workspace_bytes < tree_attention_workspace_bytes(b.n, b.tokens, q_heads, c.heads, c.head_dim)) return SLIMSPEC_WORKSPACE_TOO_SMALL;
    const TreeCall call{static_cast<const uint16_t *>(q), static_cast<uint16_t *>(out), lse, mask, q_token_stride, q_head_stride,
                        out_token_stride, out_head_stride, q_heads, mask ? mask_words : 0, scale, cache->dtype == SLIMSPEC_F16};
    return done(launch_tree_attention(c, layer, call, b, workspace, static_cast<hipStream_t>(stream)));
}

int slimspec_tree_mask(const int32_t *parents, const slimspec_batch *batch, int32_t words, uint64_t *mask, void *stream)
{
    if (!batch || batch->n < 0 || batch->tokens < 0 || (batch->n > 0 && !batch->first)) return SLIMSPEC_INVALID_ARGUMENT;
    if (words < 1 || words > SLIMSPEC_TREE_MAX_WORDS) return SLIMSPEC_INVALID_ARGUMENT;
    if (batch->n > SLIMSPEC_CACHE_MAX_SEQUENCES) return SLIMSPEC_UNSUPPORTED;
    if (batch->n == 0 || batch->tokens == 0) return SLIMSPEC_OK;
    if (!parents || !mask) return SLIMSPEC_INVALID_ARGUMENT;
    return done(launch_tree_mask(parents, BatchView{batch->slots, batch->first, batch->n, batch->tokens}, words, mask, static_cast<hipStream_t>(stream)));
}

int slimspec_cache_reserve(const slimspec_cache *cache, const slimspec_batch *batch, int32_t *report, void *stream)
{
    CacheView c;
    BatchView b;
    int st = check_cache(cache, c);
    if (st != SLIMSPEC_OK) return st;
    if ((st = check_batch(batch, b)) != SLIMSPEC_OK) return st;
    if (!report) return SLIMSPEC_INVALID_ARGUMENT;
    return done(launch_cache_reserve(c, b, report, static_cast<hipStream_t>(stream)));
}

int slimspec_cache_append(const slimspec_cache *cache, int32_t first_layer, int32_t n_layers,
                          const void *k_new, const void *v_new, int64_t new_layer_stride, int64_t new_token_stride, int64_t new_head_stride,
                          const slimspec_batch *batch, void *stream)
{
    CacheView c;
    BatchView b;
    int st = check_cache(cache, c);
    if (st != SLIMSPEC_OK) return st;
    if ((st = check_batch(batch, b)) != SLIMSPEC_OK) return st;
    if (first_layer < 0 || n_layers < 1 || n_layers > c.layers - first_layer) return SLIMSPEC_INVALID_ARGUMENT;
    if (new_layer_stride < 0 || new_token_stride < 0 || new_head_stride < 0) return SLIMSPEC_INVALID_ARGUMENT;
    if (!rows_aligned(new_layer_stride) || !rows_aligned(new_token_stride) || !rows_aligned(new_head_stride)) return SLIMSPEC_UNSUPPORTED;
    if (b.n == 0 || b.tokens == 0) return SLIMSPEC_OK;
    if (!k_new || !v_new) return SLIMSPEC_INVALID_ARGUMENT;
    if (!aligned16(k_new) || !aligned16(v_new)) return SLIMSPEC_UNSUPPORTED;
    const NewRows rows{static_cast<const uint16_t *>(k_new), static_cast<const uint16_t *>(v_new), new_layer_stride, new_token_stride, new_head_stride};
    return done(launch_cache_append(c, first_layer, n_layers, rows, b, static_cast<hipStream_t>(stream)));
}

int slimspec_cache_compact(const slimspec_cache *cache, const slimspec_batch *batch,
                           const int32_t *path, int32_t width, const int32_t *accepted, int32_t *new_lens, void *stream)
{
    CacheView c;
    BatchView b;
    int st = check_cache(cache, c);
    if (st != SLIMSPEC_OK) return st;
    if ((st = check_batch(batch, b)) != SLIMSPEC_OK) return st;
    if (width < 1) return SLIMSPEC_INVALID_ARGUMENT;
    if (b.n == 0) return SLIMSPEC_OK;
    if (!path || !accepted || !new_lens || new_lens == cache->lens) return SLIMSPEC_INVALID_ARGUMENT;
    return done(launch_cache_compact(c, b, path, width, accepted, new_lens, static_cast<hipStream_t>(stream)));
}

int slimspec_cache_set_lens(const slimspec_cache *cache, const int32_t *slots, int32_t n, const int32_t *lens, void *stream)
{
    CacheView c;
    const int st = check_cache(cache, c);
    if (st != SLIMSPEC_OK) return st;
    if (n < 0 || (n > 0 && !slots) || lens == cache->lens) return SLIMSPEC_INVALID_ARGUMENT;
    if (n > SLIMSPEC_CACHE_MAX_SEQUENCES) return SLIMSPEC_UNSUPPORTED;
    if (n == 0) return SLIMSPEC_OK;
    return done(launch_cache_set_lens(c, slots, n, lens, static_cast<hipStream_t>(stream)));
}

int slimspec_cache_fork(const slimspec_cache *cache, const int32_t *parents, const int32_t *children, int32_t n, int32_t *report, void *stream)
{
    CacheView c;
    const int st = check_cache(cache, c);
    if (st != SLIMSPEC_OK) return st;
    if (n < 0 || (n > 0 && (!parents || !children)) || !report) return SLIMSPEC_INVALID_ARGUMENT;
    if (n > SLIMSPEC_CACHE_MAX_SEQUENCES) return SLIMSPEC_UNSUPPORTED;
    return done(launch_cache_fork(c, parents, children, n, report, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
