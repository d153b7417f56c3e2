// Sequences whose queries lie packed, one behind the other, over a paged cache (dl_chunk.hip, dl_weigh.hip).
#pragma once

#include "dl_codes.h"

struct dl_packed {
    const int32_t *starts, *lens, *pages;
    int64_t pages_stride;
    uint32_t tokens, most, batch;  // rows of q; max_pages * page_tokens
    __device__ __forceinline__ uint32_t len(uint32_t b) const { return most ? min((uint32_t)max(lens[b], 0), most) : 0u; }
    __device__ __forceinline__ uint32_t start(uint32_t b) const { return min((uint32_t)max(starts[b], 0), tokens); }
    __device__ __forceinline__ uint32_t queries(uint32_t b, uint32_t first) const { return max(start(b + 1u), first) - first; }
};

constexpr float DL_LOG2E = 1.44269504088896340736f, DL_LN2 = 0.69314718055994530942f;

// What dl_chunk_attention_args and dl_kv_weigh_args have in common, looked at from sizes alone / from all of it.
template <class Args>
static inline int dl_packed_sizes(const dl_kv_cache *cache, const Args *args, dl_cache_view *view)
{
    if (!cache || !args) return DL_ERR_INVALID;
    const int rc = dl_cache_check(cache, 0, view);
    if (rc != DL_OK) return rc;
    if (args->type != DL_TYPE_BF16 && args->type != DL_TYPE_F16) return DL_ERR_INVALID;
    if (args->batch < 0 || args->batch > 65535 || args->q_heads < 0 || args->q_heads > 65536 || args->q_heads % cache->heads) return DL_ERR_INVALID;
    if (args->tokens < 0 || args->tokens > DL_MAX_ROWS / 2 || args->tokens * args->q_heads > DL_MAX_ROWS / 2) return DL_ERR_INVALID;
    if (args->max_pages < 0 || args->max_pages > 1 << 30 || args->max_pages * cache->page_tokens > 1 << 30) return DL_ERR_INVALID;
    return DL_OK;
}
template <class Args>
static inline int dl_packed_setup(const dl_kv_cache *cache, const Args *args, size_t needed, dl_packed *p)
{
    if (!args->q_starts || (args->max_pages && (!args->pages || !args->lens))) return DL_ERR_INVALID;
    if (((uint64_t)args->q_starts | (uint64_t)args->pages | (uint64_t)args->lens | (uint64_t)args->lse) % 4u || (uint64_t)args->q % 2u) return DL_ERR_INVALID;
    if (!args->workspace || (uint64_t)args->workspace % 16u || args->workspace_bytes < needed) return DL_ERR_INVALID;
    p->starts = args->q_starts;
    p->lens = args->lens;
    p->pages = args->pages;
    p->pages_stride = args->pages_stride;
    p->tokens = (uint32_t)args->tokens;
    p->most = cache->pages ? (uint32_t)(args->max_pages * cache->page_tokens) : 0u;
    p->batch = (uint32_t)args->batch;
    return DL_OK;
}
