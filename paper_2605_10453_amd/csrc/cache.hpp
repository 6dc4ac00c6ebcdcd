// The paged cache as the kernels see it, and the launchers of its kernels (cache_pages.hip, tree_attention.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "../../include/slimspec.h"
#include "launch.hpp"

namespace slimspec {

constexpr int kMaxSequences = SLIMSPEC_CACHE_MAX_SEQUENCES;

// slimspec_cache with what the kernels index by; log2 of the page size instead of the size
struct CacheView {
    uint16_t *k, *v;
    int64_t layer_stride, page_stride, head_stride, place_stride;
    int32_t *table, *held, *lens, *refs;
    int32_t layers, pages, heads, page_shift, head_dim, slots, slot_pages;
};
struct BatchView { const int32_t *slots, *first; int32_t n, tokens; };

#if defined(__HIPCC__)
// A sequence of the batch.  What the device arrays say is bounded here once: a sequence out of range has no tokens (tokens = 0, valid = false).
// HELD: so is one that does not hold the pages of its committed and new tokens (table entries past them are of other times, or other slots).
struct Sequence { int slot, first, tokens, len; bool valid; };
template <bool HELD = true>
__device__ __forceinline__ Sequence sequence_of(const CacheView &c, const BatchView &b, int i)
{
    Sequence q;
    q.slot = b.slots[i];
    const int lo = b.first[i], hi = b.first[i + 1];
    q.first = lo;
    q.tokens = hi - lo;
    q.valid = q.slot >= 0 && q.slot < c.slots && lo >= 0 && hi >= lo && hi <= b.tokens;
    q.len = q.valid ? c.lens[q.slot] : 0;
    const int pages = HELD && q.valid ? min(c.held[q.slot], c.slot_pages) : c.slot_pages;
    // places are int32: slot_pages * page_size < 2^31, and lens + tokens must stay inside the pages
    q.valid = q.valid && q.len >= 0 && (int64_t)q.len + q.tokens <= (int64_t)pages * (1 << c.page_shift);
    if (!q.valid) { q.tokens = 0; q.len = 0; q.first = 0; }
    return q;
}
// The page that holds a place of a valid sequence's slot, or -1 where the table holds no page number.
__device__ __forceinline__ int page_of(const CacheView &c, int slot, int place)
{
    const int page = c.table[(int64_t)slot * c.slot_pages + (place >> c.page_shift)];
    return (uint32_t)page < (uint32_t)c.pages ? page : -1;
}
#endif

hipError_t launch_tree_mask(const int32_t *parents, const BatchView &b, int words, uint64_t *mask, hipStream_t st);
hipError_t launch_cache_reserve(const CacheView &c, const BatchView &b, int32_t *report, hipStream_t st);
struct NewRows { const uint16_t *k, *v; int64_t layer_stride, token_stride, head_stride; };
hipError_t launch_cache_append(const CacheView &c, int first_layer, int n_layers, const NewRows &rows, const BatchView &b, hipStream_t st);
hipError_t launch_cache_compact(const CacheView &c, const BatchView &b, const int32_t *path, int width, const int32_t *accepted, int32_t *new_lens, hipStream_t st);
hipError_t launch_cache_set_lens(const CacheView &c, const int32_t *slots, int n, const int32_t *lens, hipStream_t st);
hipError_t launch_cache_fork(const CacheView &c, const int32_t *parents, const int32_t *children, int n, int32_t *report, hipStream_t st);

struct TreeCall {
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    const uint64_t *mask;
    int64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;
    int32_t q_heads, mask_words;
    float scale;
    bool f16;
};
size_t tree_attention_workspace_bytes(int n, int tokens, int q_heads, int heads, int head_dim);
hipError_t launch_tree_attention(const CacheView &c, int layer, const TreeCall &call, const BatchView &b, void *workspace, hipStream_t st);

}  // namespace slimspec
