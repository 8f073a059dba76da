// What the paged key/value cache's kernels share: where a token's elements lie,
// the loop over tiles, and the host's checks of caches, block tables and rows.
#pragma once

#include "host_common.hpp"

namespace sgdrc {

constexpr uint32_t kDevErrSeq = 16u;              // a length, row start, slot or path out of range

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

// The gate's two schedules with one call of ``body``, for bodies so large that
// a copy per schedule would cost registers and code: under a static schedule
// as static_tile_loop, otherwise tickets of one queue for the whole device
// (the host asks for a gate without queue groups), and the tiles left if no
// workgroup reached an allowed CU to the last workgroup of the grid (flagged).
// ``body(tile, err)`` as in gated_tile_loop; every thread of the workgroup runs
// the same iterations.  ``prologue`` may read operands, so workgroups on CUs
// outside the mask do not run it (unless tiles are left): it would take from the
// streams whose those CUs are.  Where all XCDs are allowed it does not wait for
// the workgroup's own to be known.
template <typename Prologue, typename Body>
__device__ __forceinline__ void single_tile_loop(const Gate &g, uint32_t n_tiles, Prologue prologue, Body body)
{
    __shared__ uint32_t s_ticket;
    __shared__ uint32_t s_flag;
    const auto rank = [&]() {
        uint32_t xcc;
        asm volatile("s_getreg_b32 %0, hwreg(HW_REG_XCC_ID)" : "=s"(xcc));
        return g.xcd_rank[xcc & 0xFu];
    };
    if (g.tlog && blockIdx.x == 0 && threadIdx.x == 0)
        __hip_atomic_store(&g.tlog[0], __builtin_amdgcn_s_memrealtime(), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
    uint32_t err = 0u;
    // where the next tile comes from: the static stride, the queue, what is left
    enum { kStride, kQueue, kLeft };
    uint32_t from = g.statics ? kStride : kQueue;
    uint32_t t = n_tiles;
    // what is left of the queue once the last workgroup has arrived
    auto take_left = [&]() {
        t = __builtin_amdgcn_readfirstlane(
            __hip_atomic_load(&g.q->grp_next[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
        if (t < n_tiles)
            err |= threadIdx.x == 0 ? kDevFlagGateFallback : 0u;
        from = kLeft;
    };
    uint32_t cu = (uint32_t)kMaxCus;
    bool mine = true;
    if (from == kQueue) {
        cu = my_cu_entry(g) & 0xFFFFu;
        if (__builtin_amdgcn_readfirstlane(cu_allowed(g, cu) ? 1u : 0u) == 0u) {
            if (__builtin_amdgcn_readfirstlane(arrive_last(g, &s_flag) ? 1u : 0u) == 0u)
                return;
            take_left();
            mine = t < n_tiles;
        }
    } else if (g.n_allowed_xcd != g.n_xcd) {
        mine = __builtin_amdgcn_readfirstlane(rank()) != 0xFFu;
    }
    if (mine)
        prologue();
    const uint32_t a = rank();
    if (from == kStride && g.log_cu)
        cu = my_cu_entry(g) & 0xFFFFu;
    __syncthreads();
    const uint32_t workers = (gridDim.x / g.n_xcd) * g.n_allowed_xcd;
    if (from == kStride && a != 0xFFu)
        t = (blockIdx.x / g.n_xcd) * g.n_allowed_xcd + a;
    t = __builtin_amdgcn_readfirstlane(t);
    for (;;) {
        uint32_t tile = n_tiles;
        if (from == kQueue) {
            tile = claim_ticket(&g.q->grp_next[0], &s_ticket);
            if (tile >= n_tiles) {
                // (the flag is the same in every lane; without saying so here all
                // that follows, the body's scalars too, would count as per-lane)
                if (__builtin_amdgcn_readfirstlane(arrive_last(g, &s_flag) ? 1u : 0u) == 0u)
                    break;
                take_left();
            }
        }
        if (from != kQueue) {
            tile = t;
            if (tile >= n_tiles)
                break;
            t += from == kStride ? workers : 1u;
        }
        log_tile(g, cu, tile);
        body(__builtin_amdgcn_readfirstlane(tile), err);
    }
    if (from == kLeft) {
        reset_slot(g.q);
        if (g.tlog && threadIdx.x == 0) {
            __builtin_amdgcn_s_waitcnt(0);
            __hip_atomic_store(&g.tlog[1], __builtin_amdgcn_s_memrealtime(), __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (from == kStride)
        static_end(g, a, NoOp(), err);
    else if (err != 0u)
        raise_flag(g.err, err);
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
