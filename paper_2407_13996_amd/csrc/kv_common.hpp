// The paged key/value cache shared by the cache's kernels: where a token's
// elements lie, and the host's checks of caches, block tables and rows.
#pragma once

#include "host_common.hpp"

namespace sgdrc {

// One layer of a cache, as kernels see it.
struct KvView {
    uint8_t *pool;        // the layer's block in page 0
    uint64_t pool_pages;
    uint32_t shift;       // log2 of a page's bytes
    uint32_t bshift;      // log2 of a block's tokens
    uint32_t heads;
};

struct RowsView {
    const uint8_t *ptr;
    uint64_t token;       // bytes from a token to the next
    uint64_t head;        // bytes from a head to the next
};

// Elements are two bytes.  Inside a head's chunk of a block of 2^bshift tokens:
// byte offsets of 16-byte group ``d8`` of token ``tok``'s K, and of the 8 tokens
// from 8 * t8 on of dimension ``d`` of V.
template <int D>
__device__ __forceinline__ uint32_t k_off(uint32_t d8, uint32_t tok, uint32_t bshift)
{
    return ((d8 << bshift) + tok) * 16u;
}

template <int D>
__device__ __forceinline__ uint32_t v_off(uint32_t t8, uint32_t d, uint32_t bshift)
{
    return ((uint32_t)D * 2u << bshift) + (t8 * (uint32_t)D + d) * 16u;
}

// Bytes of a head's chunk.
template <int D>
__device__ __forceinline__ uint32_t head_bytes(uint32_t bshift)
{
    return (uint32_t)D * 4u << bshift;
}

int check_kv_cache(const sgdrc_kv_cache *c);
int check_kv_blocks(const sgdrc_kv_blocks *b, uint32_t block_tokens);
int check_rows(const sgdrc_rows *r, const char *name);
int check_aligned(const void *p, uint32_t bytes, const char *name);

inline KvView kv_view(const sgdrc_kv_cache *c, uint32_t layer)
{
    return {static_cast<uint8_t *>(c->pool) + layer * c->layer_stride, c->pool_pages, c->page_shift,
            (uint32_t)__builtin_ctz(c->block_tokens), c->kv_heads};
}

// Entries of a row of block tables.
inline uint32_t blocks_width(const sgdrc_kv_blocks *b) { return b->width ? b->width : b->stride; }

inline RowsView rows_view(const sgdrc_rows *r)
{
    return {static_cast<const uint8_t *>(r->ptr), r->token_stride * 2u, r->head_stride * 2u};
}

}  // namespace sgdrc
