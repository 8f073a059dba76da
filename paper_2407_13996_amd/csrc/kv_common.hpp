// What the paged key/value cache's kernels share: where a token's elements lie,
// how V is turned, the loop over tiles, and the host's checks of caches, block tables and rows.
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

constexpr int kKvThreads = 256;

// LDS of a workgroup of kKvThreads that writes V of TOKENS tokens of one head.  V is
// turned on the way: the 8 tokens of an aligned group of slots meet in one
// 16-byte store.  Groups that the tokens do not fill are
// written element by element (every token of a decoding step; the ends of a
// prompt's run).  A group belongs to the tile of its first token.
template <int D, int TOKENS>
struct ValueTurn {
    static constexpr uint32_t kRows = TOKENS + 7;         // the tile's and those of a group that begins in it
    static constexpr uint32_t V16 = D / 8;                // 16-byte pieces of a row
    static constexpr uint32_t kBack = 7u;                 // tokens before the tile that are looked at
    static constexpr uint32_t kSeen = kBack + TOKENS + 7u;
    int64_t slot[kSeen];
    uint32_t bits[2];                                     // leaders of full groups, single tokens
    uint32_t lead[TOKENS / 8 + 1];                        // the leaders
    __attribute__((aligned(16))) uint16_t v[kRows][D + 8];

    // The slots of the tile's tokens and those around it, -1 past the ends, for slots
    // out of range (flagged) and, if ``position`` is given, where that is below 0.
    __device__ __forceinline__ void take_slots(const KvView &c, const int64_t *slots, const int32_t *position,
                                               uint32_t t0, uint32_t n_tokens, uint32_t &err)
    {
        if (threadIdx.x < kSeen) {
            const int64_t i = (int64_t)t0 + threadIdx.x - kBack;
            const bool in = i >= 0 && i < (int64_t)n_tokens;
            int64_t s = in ? slots[i] : -1;
            if (position && in && position[i] < 0)
                s = -1;
            if (s < -1 || (s >= 0 && ((uint64_t)s >> c.bshift) >= c.pool_pages)) {
                err |= kDevErrSeq;
                s = -1;
            }
            slot[threadIdx.x] = s;
        }
    }

    // Which tokens lead a full group, which stand alone (after a barrier).
    __device__ __forceinline__ void sort_out()
    {
        if (threadIdx.x < 64u) {
            bool leads = false, single = false;
            if (threadIdx.x < (uint32_t)TOKENS) {
                const uint32_t x = threadIdx.x + kBack;
                const int64_t s = slot[x];
                if (s >= 0) {
                    const uint32_t in = (uint32_t)s & 7u;
                    bool full = true;
#pragma unroll
                    for (uint32_t q = 0; q < 8u; ++q)
                        full = full && slot[x - in + q] == s - (int64_t)in + (int64_t)q;
                    leads = full && in == 0u;
                    single = !full;
                }
            }
            const uint64_t lb = __ballot(leads), sb = __ballot(single);
            if (leads)
                lead[__popcll(lb & ((1ull << threadIdx.x) - 1ull))] = threadIdx.x;
            if (threadIdx.x == 0u) {
                bits[0] = (uint32_t)lb;
                bits[1] = (uint32_t)sb;
            }
        }
    }

    // The stores, with the tile's rows in ``v`` (after another barrier).
    __device__ __forceinline__ void write(const KvView &c, const RowsView &from, uint32_t t0, uint32_t h)
    {
        const uint32_t leaders = __builtin_amdgcn_readfirstlane(bits[0]);
        const uint32_t singles = __builtin_amdgcn_readfirstlane(bits[1]);
        // the rows past the tile of its last group (tokens that exist: their slots are consecutive)
        if (leaders >> (TOKENS - 7)) {
            const uint32_t last = 31u - (uint32_t)__builtin_clz(leaders);
            const uint32_t n = (last + 8u - TOKENS) * V16;
            for (uint32_t i = threadIdx.x; i < n; i += kKvThreads)
                *reinterpret_cast<u32x4 *>(&v[TOKENS + i / V16][(i % V16) * 8u]) =
                    *reinterpret_cast<const u32x4 *>(from.ptr + (uint64_t)(t0 + TOKENS + i / V16) * from.token +
                                                     h * from.head + (i % V16) * 16u);
            __syncthreads();
        }
        // a thread takes 16 bytes of a group: a dimension of its eight tokens
        for (uint32_t i = threadIdx.x; i < (uint32_t)__builtin_popcount(leaders) * D; i += kKvThreads) {
            const uint32_t x = lead[i / (uint32_t)D], d = i % (uint32_t)D;
            const int64_t s = slot[kBack + x];
            uint8_t *const at = c.pool + ((uint64_t)(s >> c.bshift) << c.shift) + h * head_bytes<D>(c.bshift);
            const uint32_t t8 = ((uint32_t)s & ((1u << c.bshift) - 1u)) >> 3;
            u32x4 o;
#pragma unroll
            for (uint32_t q = 0; q < 4u; ++q)
                o[q] = (uint32_t)v[x + 2u * q][d] | ((uint32_t)v[x + 2u * q + 1u][d] << 16);
            *reinterpret_cast<u32x4 *>(at + v_off<D>(t8, d, c.bshift)) = o;
        }
        if (singles) {
            for (uint32_t i = threadIdx.x; i < (uint32_t)(TOKENS * D); i += kKvThreads) {
                const uint32_t x = i / (uint32_t)D, d = i % (uint32_t)D;
                if ((singles >> x) & 1u) {
                    const int64_t s = slot[kBack + x];
                    uint8_t *const at = c.pool + ((uint64_t)(s >> c.bshift) << c.shift) + h * head_bytes<D>(c.bshift);
                    const uint32_t off = (uint32_t)s & ((1u << c.bshift) - 1u);
                    *reinterpret_cast<uint16_t *>(at + v_off<D>(off >> 3, d, c.bshift) + (off & 7u) * 2u) = v[x][d];
                }
            }
        }
    }
};

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

// The same for bodies that load on into the workgroup's next tiles:
// ``prime(tile, next)`` starts the loads of the first, ``body(tile, next, after, err)``
// works on a tile whose loads are under way and starts those of the two that it
// takes after it (n_tiles or more: none; the queue's tickets are taken ahead for that).
// The body holds a barrier.
template <typename Prime, typename Prologue, typename Body>
__device__ __forceinline__ void single_tile_stream(const Gate &g, uint32_t n_tiles, Prime prime, Prologue prologue,
                                                   Body body)
{
    __shared__ uint32_t s_ticket;
    __shared__ uint32_t s_flag;
    uint32_t xcc;
    asm volatile("s_getreg_b32 %0, hwreg(HW_REG_XCC_ID)" : "=s"(xcc));
    const uint32_t a = g.xcd_rank[xcc & 0xFu];
    if (g.tlog && blockIdx.x == 0 && threadIdx.x == 0)
        __hip_atomic_store(&g.tlog[0], __builtin_amdgcn_s_memrealtime(), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    uint32_t err = 0u;
    const uint32_t workers = (gridDim.x / g.n_xcd) * g.n_allowed_xcd;
    const bool queue = g.statics == 0u;
    uint32_t cu = queue || g.log_cu ? my_cu_entry(g) & 0xFFFFu : (uint32_t)kMaxCus;
    uint32_t t = n_tiles, next = n_tiles, after = n_tiles, step = workers;
    bool left = false;  // working on what the queue has left
    if (!queue) {
        if (a != 0xFFu) {
            t = (blockIdx.x / g.n_xcd) * g.n_allowed_xcd + a;
            next = t + workers;
            after = next + workers;
        }
    } else if (__builtin_amdgcn_readfirstlane(cu_allowed(g, cu) ? 1u : 0u)) {
        t = claim_ticket(&g.q->grp_next[0], &s_ticket);
        next = claim_ticket(&g.q->grp_next[0], &s_ticket);
        after = claim_ticket(&g.q->grp_next[0], &s_ticket);
    }
    bool fresh = true;
    for (;;) {
        t = __builtin_amdgcn_readfirstlane(t);
        next = __builtin_amdgcn_readfirstlane(next);
        after = __builtin_amdgcn_readfirstlane(after);
        if (queue && !left && t >= n_tiles) {
            if (__builtin_amdgcn_readfirstlane(arrive_last(g, &s_flag) ? 1u : 0u) == 0u)
                break;
            // the last workgroup of the grid
            left = fresh = true;
            step = 1u;
            t = __builtin_amdgcn_readfirstlane(
                __hip_atomic_load(&g.q->grp_next[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
            next = t + 1u;
            after = t + 2u;
            if (t < n_tiles)
                err |= threadIdx.x == 0 ? kDevFlagGateFallback : 0u;
        }
        if (t >= n_tiles)
            break;
        if (fresh) {
            prime(t, next);
            prologue();
            __syncthreads();
            fresh = false;
        }
        uint32_t ahead = 0u;
        if (queue && !left && threadIdx.x == 0)
            ahead = __hip_atomic_fetch_add(&g.q->grp_next[0], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        log_tile(g, cu, t);
        body(t, next, after, err);
        t = next;
        next = after;
        if (queue && !left) {
            if (threadIdx.x == 0)
                s_ticket = ahead;
            __syncthreads();
            after = s_ticket;
        } else {
            after += step;
        }
    }
    if (left) {
        reset_slot(g.q);
        if (g.tlog && threadIdx.x == 0) {
            __builtin_amdgcn_s_waitcnt(0);
            __hip_atomic_store(&g.tlog[1], __builtin_amdgcn_s_memrealtime(), __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (!queue)
        static_end(g, a, NoOp(), err);
    else if (err != 0u)
        raise_flag(g.err, err);
}

int check_kv_cache(const sgdrc_kv_cache *c);
int check_kv_blocks(const sgdrc_kv_blocks *b, uint32_t block_tokens);
int check_layer(const sgdrc_kv_cache *c, uint32_t layer);
int check_rows(const sgdrc_rows *r, const char *name);
int check_aligned(const void *p, uint32_t bytes, const char *name);

// Launches kernel ``k`` (a single_tile_loop of ``tiles`` tiles in workgroups of
// ``threads``) on the stream's allowed CUs.
template <typename K, typename... A>
int launch_tiles(sgdrc_ctx *ctx, void *stream, uint64_t tiles, int occ, int threads, K k, A... args)
{
    Ctx *c = nullptr;
    int rc = check_ctx(ctx, &c);
    if (rc)
        return rc;
    Gate g;
    LaunchInfo li;
    rc = make_gate(c, stream, tiles, kStreamGroupCus, &g, &li, false, true);
    if (rc)
        return rc;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(k, dim3(gated_grid(c, occ, tiles, li)), dim3(threads), 0, s, args..., (uint32_t)tiles, g);
    SGDRC_HIP(hipGetLastError());
    return finish_static_tlog(g, s);
}

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
