// The paged key/value cache: block tables and slot maps, the writes of new
// tokens and of accepted drafts.
#include <algorithm>
#include <cmath>

#include "kv_common.hpp"

namespace sgdrc {

constexpr int kKvThreads = 256;
constexpr uint32_t kMapTile = kKvThreads;  // requests and tokens of a map tile, one a thread
constexpr uint32_t kRefused = 0xFFFFFFFFu;

struct MapArgs {
    const uint64_t *ring_pos;
    const int32_t *held, *lens, *fresh;
    uint64_t *ring_pos_out;
    int32_t *held_out, *lens_out;
    uint32_t *ring;
    uint32_t *table;
    uint32_t *q_start;
    int64_t *slots;
    int32_t *request, *position;
    uint32_t ring_size, stride, width, bshift, n_requests, n_tokens;
};

// What a request asks for.  ``ok``: its state is sound and its tokens fit its
// row of the table.
struct MapAsk {
    uint32_t tokens, need, freed;
    bool ok, ended;
};

__device__ __forceinline__ MapAsk map_ask(const MapArgs &a, uint32_t r)
{
    const int64_t len = a.lens[r], held = a.held[r], fresh = a.fresh[r];
    MapAsk q;
    q.ended = fresh < 0;
    q.tokens = q.ended ? 0u : (uint32_t)fresh;
    q.ok = len >= 0 && held >= 0 && held <= (int64_t)a.width && len <= (held << a.bshift);
    const int64_t total = len + (int64_t)q.tokens;
    q.ok = q.ok && total <= ((int64_t)a.width << a.bshift);
    const int64_t blocks = (total + (1 << a.bshift) - 1) >> a.bshift;
    q.need = q.ok && !q.ended && blocks > held ? (uint32_t)(blocks - held) : 0u;
    q.freed = q.ok && q.ended ? (uint32_t)held : 0u;
    return q;
}

// Every workgroup that may have a tile adds up all requests for itself (three
// running sums: tokens, wanted pages, returned pages), so that one launch without any
// exchange between workgroups does: its requests' and tokens' entries follow from
// the sums in LDS.  The state goes to other memory than it is read from for the
// same reason.  A step is bound by the launch and this chain of round trips
// (lengths, sums, table or ring, slot), not by its bytes: 8 requests take 5.2
// us, 2048 of which every ninth ends 13.4 (17 in tiles of four tokens a thread),
// where a thread reads its 8 requests one after the other, and again for the sums.
__global__ __launch_bounds__(kKvThreads) void k_kv_map(MapArgs a, uint32_t n_tiles, Gate g)
{
    __shared__ uint32_t s_q[SGDRC_MAX_REQUESTS + 1];  // first token of each request
    // first wanted page of a request counted from the ring's first free one, or
    // first returned page of an ended one from its end; kRefused: not served
    __shared__ uint32_t s_e[SGDRC_MAX_REQUESTS];
    __shared__ uint64_t s_sum[3][kKvThreads / 64];
    __shared__ uint32_t s_taken, s_given;
    const uint32_t R = a.n_requests;
    uint64_t taken0 = 0, put0 = 0, avail = 0, room = 0;
    uint32_t pro_err = 0u;
    auto prologue = [&]() {
        taken0 = a.ring_pos[0];
        put0 = a.ring_pos[1];
        avail = put0 - taken0;
        room = a.ring_size - avail;
        if (put0 < taken0 || avail > a.ring_size) {
            avail = room = 0;
            pro_err = kDevErrSeq;
        }
        const uint32_t per = (R + kKvThreads - 1u) / kKvThreads;
        const uint32_t r0 = min(threadIdx.x * per, R), r1 = min(r0 + per, R);
        uint64_t sum[3] = {0, 0, 0};
        for (uint32_t r = r0; r < r1; ++r) {
            const MapAsk q = map_ask(a, r);
            sum[0] += q.tokens;
            sum[1] += q.need;
            sum[2] += q.freed;
        }
        const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
        uint64_t run[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            uint64_t v = sum[k];
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const uint64_t o = __shfl_up(v, off, 64);
                v += lane >= (uint32_t)off ? o : 0;
            }
            if (lane == 63u)
                s_sum[k][wave] = v;
            run[k] = v - sum[k];
        }
        if (threadIdx.x == 0)
            s_taken = s_given = 0u;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 3; ++k)
            for (uint32_t w = 0; w < wave; ++w)
                run[k] += s_sum[k][w];
        uint32_t taken = 0u, given = 0u;  // ends of the last pages taken and given back
        for (uint32_t r = r0; r < r1; ++r) {
            const MapAsk q = map_ask(a, r);
            s_q[r] = (uint32_t)min(run[0], (uint64_t)a.n_tokens);
            run[0] += q.tokens;
            const uint64_t end = run[1] + q.need;
            const bool served = q.ok && !q.ended && (q.need == 0u || end <= avail) && run[0] <= a.n_tokens;
            const uint64_t back = run[2] + q.freed;
            const bool fits = q.ok && q.ended && (q.freed == 0u || back <= room);
            if (q.ended)
                s_e[r] = fits ? (uint32_t)(q.freed ? run[2] : 0u) : kRefused;
            else
                s_e[r] = served ? (uint32_t)(q.need ? run[1] : 0u) : kRefused;
            if (served && q.need)
                taken = (uint32_t)end;
            if (fits && q.freed)
                given = (uint32_t)back;
            run[1] = end;
            run[2] = back;
            if (r == R - 1u)
                s_q[R] = (uint32_t)min(run[0], (uint64_t)a.n_tokens);
        }
        if (taken)
            atomicMax(&s_taken, taken);
        if (given)
            atomicMax(&s_given, given);
    };
    auto body = [&](uint32_t t, uint32_t &err) {
        err |= pro_err;
        const uint32_t lane = threadIdx.x & 63u;
        const uint32_t taken_at = (uint32_t)(taken0 % a.ring_size), put_at = (uint32_t)(put0 % a.ring_size);
        if (t == 0u && threadIdx.x == 0u) {
            a.ring_pos_out[0] = taken0 + s_taken;
            a.ring_pos_out[1] = put0 + s_given;
            a.q_start[R] = s_q[R];
        }
        {
            const uint32_t r = t * kMapTile + threadIdx.x;
            uint32_t freed = 0u;
            if (r < R) {
                const MapAsk q = map_ask(a, r);
                const uint32_t e = s_e[r];
                const bool beyond = q.ok && !q.ended && e == kRefused && s_q[r] + q.tokens != s_q[r + 1u];
                const bool on = e != kRefused;
                err |= !q.ok || beyond || (q.ended && !on) ? kDevErrSeq : 0u;
                a.held_out[r] = on ? (q.ended ? 0 : a.held[r] + (int32_t)q.need) : a.held[r];
                a.lens_out[r] = on ? (q.ended ? 0 : a.lens[r] + (int32_t)q.tokens) : a.lens[r];
                a.q_start[r] = s_q[r];
                freed = on ? q.freed : 0u;
            }
            // ended requests' pages, a wavefront for four requests at a time
            for (uint64_t todo = __ballot(freed != 0u); todo;) {
                uint32_t rr[4], n[4], most = 0u;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t l = todo ? (uint32_t)__builtin_ctzll(todo) : 0u;
                    rr[k] = t * kMapTile + (threadIdx.x & ~63u) + l;
                    n[k] = todo ? __shfl(freed, l, 64) : 0u;
                    most = max(most, n[k]);
                    todo &= todo - 1ull;
                }
                for (uint32_t b = lane; b < most; b += 64u) {
                    uint32_t page[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        page[k] = a.table[(uint64_t)rr[k] * a.stride + min(b, max(n[k], 1u) - 1u)];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (b < n[k]) {
                            const uint64_t at = (uint64_t)put_at + s_e[rr[k]] + b;  // below twice the ring's size
                            a.ring[at >= a.ring_size ? at - a.ring_size : at] = page[k];
                        }
                }
            }
        }
        const uint64_t i = (uint64_t)t * kMapTile + threadIdx.x;
        if (i < a.n_tokens) {
            int64_t slot = -1;
            int32_t req = -1, pos = -1;
            if (i < s_q[R]) {
                // the last request that begins at or before token i
                uint32_t lo = 0u, hi = R;
                while (hi - lo > 1u) {
                    const uint32_t mid = (lo + hi) >> 1;
                    if (s_q[mid] <= i)
                        lo = mid;
                    else
                        hi = mid;
                }
                req = (int32_t)lo;
                const uint32_t p = (uint32_t)a.lens[lo] + ((uint32_t)i - s_q[lo]);
                pos = (int32_t)p;
                if (s_e[lo] != kRefused) {
                    const uint32_t b = p >> a.bshift, held = (uint32_t)a.held[lo];
                    uint32_t *const entry = a.table + (uint64_t)lo * a.stride + b;
                    uint32_t page;
                    if (b < held) {
                        page = *entry;
                    } else {
                        uint64_t at = (uint64_t)taken_at + s_e[lo] + (b - held);
                        page = a.ring[at >= a.ring_size ? at - a.ring_size : at];
                        // a new block begins with a new token
                        if ((p & ((1u << a.bshift) - 1u)) == 0u)
                            *entry = page;
                    }
                    slot = (int64_t)(((uint64_t)page << a.bshift) | (p & ((1u << a.bshift) - 1u)));
                }
            }
            a.slots[i] = slot;
            a.request[i] = req;
            a.position[i] = pos;
        }
    };
    single_tile_loop(g, n_tiles, prologue, body);
}

// A tile is TOKENS tokens of one head.  K goes to the cache as it comes, 16 bytes
// at a time; V is turned, the 8 tokens of an aligned group of slots meeting
// in one 16-byte store, through LDS.  Groups that the tokens do not fill are
// written element by element (every token of a decoding step; the ends of a
// prompt's run).  A group belongs to the tile of its first token.  Bound by
// the way from slots and rows through LDS to the stores, which a tile of 32
// goes half as often: 16384 tokens of 8 heads take 33 us so (4.0 TB/s) and 36
// in tiles of 16; 61 tokens, which do not fill the GPU either way, 6.3 and 5.1.
template <int D, int TOKENS>
__global__ __launch_bounds__(kKvThreads) void k_kv_append(KvView c, RowsView k, RowsView v,
                                                          const int64_t *__restrict__ slots,
                                                          uint32_t n_tokens, uint32_t n_tiles, Gate g)
{
    constexpr int kRows = TOKENS + 7;                     // the tile's and those of a group that begins in it
    constexpr uint32_t V16 = D / 8;                       // 16-byte pieces of a row
    constexpr uint32_t kBack = 7u;                        // tokens before the tile that are looked at
    constexpr uint32_t kSeen = kBack + TOKENS + 7u;
    __shared__ int64_t s_slot[kSeen];
    __shared__ uint32_t s_bits[2];                        // leaders of full groups, single tokens
    __shared__ uint32_t s_lead[TOKENS / 8 + 1];    // the leaders
    __shared__ __attribute__((aligned(16))) uint16_t s_v[kRows][D + 8];
    constexpr uint32_t kLoads = (TOKENS * V16 + kKvThreads - 1u) / kKvThreads;
    auto body = [&](uint32_t t, uint32_t &err) {
        const uint32_t h = t % c.heads, t0 = t / c.heads * (uint32_t)TOKENS;
        // K's lanes: 16 tokens side by side (256-byte runs of the cache); V's
        // lanes: along the rows
        const auto k_tok = [](uint32_t i) { return i / (16u * V16) * 16u + i % 16u; };
        const auto k_d8 = [](uint32_t i) { return i % (16u * V16) / 16u; };
        u32x4 kk[kLoads], vv[kLoads];
#pragma unroll
        for (uint32_t j = 0; j < kLoads; ++j) {
            const uint32_t i = j * kKvThreads + threadIdx.x;
            const uint32_t tk = min(t0 + k_tok(i), n_tokens - 1u);
            const uint32_t tv = min(t0 + i / V16, n_tokens - 1u);
            const u32x4 z = {0u, 0u, 0u, 0u};
            kk[j] = vv[j] = z;
            if (i < TOKENS * V16) {
                kk[j] = *reinterpret_cast<const u32x4 *>(k.ptr + tk * k.token + h * k.head + k_d8(i) * 16u);
                vv[j] = *reinterpret_cast<const u32x4 *>(v.ptr + tv * v.token + h * v.head + (i % V16) * 16u);
            }
        }
        __syncthreads();  // the last tile's LDS is read
        if (threadIdx.x < kSeen) {
            const int64_t i = (int64_t)t0 + threadIdx.x - kBack;
            int64_t s = i >= 0 && i < (int64_t)n_tokens ? slots[i] : -1;
            if (s < -1 || (s >= 0 && ((uint64_t)s >> c.bshift) >= c.pool_pages)) {
                err |= kDevErrSeq;
                s = -1;
            }
            s_slot[threadIdx.x] = s;
        }
        __syncthreads();
        if (threadIdx.x < 64u) {
            // token ``threadIdx.x`` of the tile: does it lead a full group, or stand alone
            bool lead = false, single = false;
            if (threadIdx.x < (uint32_t)TOKENS) {
                const uint32_t x = threadIdx.x + kBack;
                const int64_t s = s_slot[x];
                if (s >= 0) {
                    const uint32_t in = (uint32_t)s & 7u;
                    bool full = true;
#pragma unroll
                    for (uint32_t q = 0; q < 8u; ++q)
                        full = full && s_slot[x - in + q] == s - (int64_t)in + (int64_t)q;
                    lead = full && in == 0u;
                    single = !full;
                }
            }
            const uint64_t lb = __ballot(lead), sb = __ballot(single);
            if (lead)
                s_lead[__popcll(lb & ((1ull << threadIdx.x) - 1ull))] = threadIdx.x;
            if (threadIdx.x == 0u) {
                s_bits[0] = (uint32_t)lb;
                s_bits[1] = (uint32_t)sb;
            }
        }
#pragma unroll
        for (uint32_t j = 0; j < kLoads; ++j) {
            const uint32_t i = j * kKvThreads + threadIdx.x;
            if (i < TOKENS * V16) {
                const int64_t s = s_slot[kBack + k_tok(i)];
                if (s >= 0) {
                    uint8_t *const at = c.pool + ((uint64_t)(s >> c.bshift) << c.shift) + h * head_bytes<D>(c.bshift);
                    *reinterpret_cast<u32x4 *>(at + k_off<D>(k_d8(i), (uint32_t)s & ((1u << c.bshift) - 1u), c.bshift)) = kk[j];
                }
                *reinterpret_cast<u32x4 *>(&s_v[i / V16][(i % V16) * 8u]) = vv[j];
            }
        }
        __syncthreads();
        const uint32_t leaders = __builtin_amdgcn_readfirstlane(s_bits[0]);
        const uint32_t singles = __builtin_amdgcn_readfirstlane(s_bits[1]);
        // the rows past the tile of its last group (tokens that exist: their slots are consecutive)
        if (leaders >> (TOKENS - 7)) {
            const uint32_t last = 31u - (uint32_t)__builtin_clz(leaders);
            const uint32_t n = (last + 8u - TOKENS) * V16;
            for (uint32_t i = threadIdx.x; i < n; i += kKvThreads)
                *reinterpret_cast<u32x4 *>(&s_v[TOKENS + i / V16][(i % V16) * 8u]) =
                    *reinterpret_cast<const u32x4 *>(v.ptr + (uint64_t)(t0 + TOKENS + i / V16) * v.token +
                                                     h * v.head + (i % V16) * 16u);
            __syncthreads();
        }
        // a thread takes 16 bytes of a group: a dimension of its eight tokens
        for (uint32_t i = threadIdx.x; i < (uint32_t)__builtin_popcount(leaders) * D; i += kKvThreads) {
            const uint32_t x = s_lead[i / (uint32_t)D], d = i % (uint32_t)D;
            const int64_t s = s_slot[kBack + x];
            uint8_t *const at = c.pool + ((uint64_t)(s >> c.bshift) << c.shift) + h * head_bytes<D>(c.bshift);
            const uint32_t t8 = ((uint32_t)s & ((1u << c.bshift) - 1u)) >> 3;
            u32x4 o;
#pragma unroll
            for (uint32_t q = 0; q < 4u; ++q)
                o[q] = (uint32_t)s_v[x + 2u * q][d] | ((uint32_t)s_v[x + 2u * q + 1u][d] << 16);
            *reinterpret_cast<u32x4 *>(at + v_off<D>(t8, d, c.bshift)) = o;
        }
        if (singles) {
            for (uint32_t i = threadIdx.x; i < (uint32_t)(TOKENS * D); i += kKvThreads) {
                const uint32_t x = i / (uint32_t)D, d = i % (uint32_t)D;
                if ((singles >> x) & 1u) {
                    const int64_t s = s_slot[kBack + x];
                    uint8_t *const at = c.pool + ((uint64_t)(s >> c.bshift) << c.shift) + h * head_bytes<D>(c.bshift);
                    const uint32_t off = (uint32_t)s & ((1u << c.bshift) - 1u);
                    *reinterpret_cast<uint16_t *>(at + v_off<D>(off >> 3, d, c.bshift) + (off & 7u) * 2u) = s_v[x][d];
                }
            }
        }
    };
    single_tile_loop(g, n_tiles, NoOp(), body);
}

struct CommitArgs {
    uint64_t layer_stride;
    const uint32_t *table;
    const int32_t *lens, *totals, *path, *accepted;  // totals: may be NULL
    int32_t *lens_out;
    uint32_t stride, width, path_stride;
};

constexpr uint32_t kCommitBatch = 8;  // path entries whose loads are in flight together

// A tile is one request in one layer.  A path ascends, so entry j's source
// (path[j] >= j) is never the destination of an earlier entry, and a thread
// that owns a column (16 bytes of K, one element of V) may load the sources of
// several entries before it stores any.  Bound by the scattered accesses that the
// layout asks for: a token's K is 16 bytes every 16 block_tokens, its V 2 bytes
// in every 16.  64 requests of 32 layers and 8 heads of 128 that keep 6 of 60
// tokens take 109 us, K and V half each; for 42 MB moved the L2 reads 2.1 million
// times from memory (267 MB by its 128-byte lines) and writes 91 MB, 3.3 TB/s
// together.  (Whole 16-byte groups of V, read and written again, took 104, and would
// rewrite tokens that are not this call's.)
template <int D>
__global__ __launch_bounds__(kKvThreads) void k_kv_commit(KvView c, CommitArgs a, uint32_t n_requests,
                                                          uint32_t n_tiles, Gate g)
{
    // each path entry's two pages, as byte offsets (from ~0: it does not move), and tokens in them
    __shared__ uint64_t s_from[SGDRC_MAX_NODES], s_to[SGDRC_MAX_NODES];
    __shared__ uint32_t s_src[SGDRC_MAX_NODES], s_dst[SGDRC_MAX_NODES];
    __shared__ uint32_t s_n;
    auto body = [&](uint32_t t, uint32_t &err) {
        const uint32_t r = t % n_requests, layer = t / n_requests;
        const int32_t len = a.lens[r], want = a.accepted[r];
        const int32_t cap = (int32_t)(a.width << c.bshift);
        const int32_t total = a.totals ? a.totals[r] : cap;
        const bool sound = len >= 0 && len <= cap && total >= 0 && total <= cap && want >= 0;
        const bool ended = sound && total < len;
        const uint32_t n = sound && !ended ? min((uint32_t)want, a.path_stride) : 0u;
        __syncthreads();  // the last tile's LDS is read
        if (threadIdx.x == 0u)
            s_n = n;
        __syncthreads();
        uint32_t bad = !sound || (uint32_t)want > (ended ? 0u : a.path_stride) ? kDevErrSeq : 0u;
        const uint32_t i = threadIdx.x;
        int32_t node = 0;
        if (i < n) {
            node = a.path[(uint64_t)r * a.path_stride + i];
            const int32_t prev = i ? a.path[(uint64_t)r * a.path_stride + i - 1u] : -1;
            if (node <= prev || node >= total - len)
                atomicMin(&s_n, i);
        }
        __syncthreads();
        const uint32_t good = s_n;
        if (good < n)
            bad = kDevErrSeq;
        if (i < good && (uint32_t)node != i) {
            const uint32_t from = (uint32_t)len + (uint32_t)node, to = (uint32_t)len + i;
            uint32_t pe = 0u;
            const uint32_t pf = checked_page(a.table, (uint64_t)r * a.stride + (from >> c.bshift), c.pool_pages, pe);
            const uint32_t pt = checked_page(a.table, (uint64_t)r * a.stride + (to >> c.bshift), c.pool_pages, pe);
            bad |= pe;
            s_from[i] = pe ? ~0ull : (uint64_t)pf << c.shift;
            s_to[i] = (uint64_t)pt << c.shift;
            s_src[i] = from & ((1u << c.bshift) - 1u);
            s_dst[i] = to & ((1u << c.bshift) - 1u);
        } else if (i < good) {
            s_from[i] = ~0ull;
        }
        err |= bad;
        if (layer == 0u && threadIdx.x == 0u)
            a.lens_out[r] = ended ? total : len + (int32_t)good;
        __syncthreads();
        uint8_t *const base = c.pool + layer * a.layer_stride;
        const uint32_t n_v = c.heads * (uint32_t)D, n_k = c.heads * (uint32_t)(D / 8);
        for (uint32_t m0 = 0; m0 < good; m0 += kCommitBatch) {
            for (uint32_t col = threadIdx.x; col < n_v; col += kKvThreads) {
                const uint32_t h = col / (uint32_t)D, d = col % (uint32_t)D;
                uint8_t *const hb = base + h * head_bytes<D>(c.bshift);
                uint16_t v[kCommitBatch];
#pragma unroll
                for (uint32_t q = 0; q < kCommitBatch; ++q) {
                    const uint32_t m = m0 + q;
                    v[q] = 0;
                    if (m < good && s_from[m] != ~0ull)
                        v[q] = *reinterpret_cast<const uint16_t *>(hb + s_from[m] + v_off<D>(s_src[m] >> 3, d, c.bshift) +
                                                                   (s_src[m] & 7u) * 2u);
                }
#pragma unroll
                for (uint32_t q = 0; q < kCommitBatch; ++q) {
                    const uint32_t m = m0 + q;
                    if (m < good && s_from[m] != ~0ull)
                        *reinterpret_cast<uint16_t *>(hb + s_to[m] + v_off<D>(s_dst[m] >> 3, d, c.bshift) +
                                                      (s_dst[m] & 7u) * 2u) = v[q];
                }
            }
            for (uint32_t col = threadIdx.x; col < n_k; col += kKvThreads) {
                const uint32_t h = col / (uint32_t)(D / 8), d8 = col % (uint32_t)(D / 8);
                uint8_t *const hb = base + h * head_bytes<D>(c.bshift);
                u32x4 v[kCommitBatch];
#pragma unroll
                for (uint32_t q = 0; q < kCommitBatch; ++q) {
                    const uint32_t m = m0 + q;
                    v[q] = u32x4{0u, 0u, 0u, 0u};
                    if (m < good && s_from[m] != ~0ull)
                        v[q] = *reinterpret_cast<const u32x4 *>(hb + s_from[m] + k_off<D>(d8, s_src[m], c.bshift));
                }
#pragma unroll
                for (uint32_t q = 0; q < kCommitBatch; ++q) {
                    const uint32_t m = m0 + q;
                    if (m < good && s_from[m] != ~0ull)
                        *reinterpret_cast<u32x4 *>(hb + s_to[m] + k_off<D>(d8, s_dst[m], c.bshift)) = v[q];
                }
            }
        }
    };
    single_tile_loop(g, n_tiles, NoOp(), body);
}

// ------------------------------------------------------------------- checks

int check_aligned(const void *p, uint32_t bytes, const char *name)
{
    if (!p || (reinterpret_cast<uintptr_t>(p) & (bytes - 1u)))
        return set_error(SGDRC_EINVAL, "%s: NULL or not %u-byte aligned", name, bytes);
    return SGDRC_OK;
}

static int check_block_tokens(uint32_t n)
{
    if (n < 16 || n > 1024 || (n & (n - 1)))
        return set_error(SGDRC_EINVAL, "block_tokens %u is not a power of two in 16..1024", n);
    return SGDRC_OK;
}

int check_kv_cache(const sgdrc_kv_cache *c)
{
    if (!c)
        return set_error(SGDRC_EINVAL, "cache is NULL");
    int rc = check_shift(c->page_shift);
    if (rc || (rc = check_aligned(c->pool, 256, "cache.pool")) || (rc = check_block_tokens(c->block_tokens)))
        return rc;
    if (c->dtype != SGDRC_BF16 && c->dtype != SGDRC_F16)
        return set_error(SGDRC_EINVAL, "cache: dtype %u is neither bf16 nor f16", c->dtype);
    if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 256)
        return set_error(SGDRC_EINVAL, "cache: head_dim %u is not 64, 96, 128 or 256", c->head_dim);
    if (c->kv_heads < 1 || c->kv_heads > SGDRC_MAX_KV_HEADS)
        return set_error(SGDRC_EINVAL, "cache: kv_heads %u outside 1..%d", c->kv_heads, SGDRC_MAX_KV_HEADS);
    if (c->pool_pages == 0 || c->pool_pages > (1ull << 32))
        return set_error(SGDRC_EINVAL, "cache: pool_pages outside 1..2^32");
    if (c->n_layers < 1 || c->n_layers > 65536)
        return set_error(SGDRC_EINVAL, "cache: n_layers %u outside 1..65536", c->n_layers);
    const uint64_t block = 4ull * c->kv_heads * c->block_tokens * c->head_dim;
    const uint64_t page = 1ull << c->page_shift;
    if (block > page)
        return set_error(SGDRC_EINVAL, "cache: a block of %llu bytes does not fit a page", (unsigned long long)block);
    if (c->n_layers > 1) {
        if (c->layer_stride & 255u)
            return set_error(SGDRC_EINVAL, "cache: layer_stride is not a multiple of 256");
        const bool inside = c->layer_stride >= block && c->layer_stride <= page / c->n_layers;
        const bool apart = c->layer_stride >= page && c->layer_stride / page >= c->pool_pages &&
                           c->layer_stride <= (1ull << 62) / c->n_layers;
        if (!inside && !apart)
            return set_error(SGDRC_EINVAL, "cache: the layers overlap");
    }
    return SGDRC_OK;
}

int check_kv_blocks(const sgdrc_kv_blocks *b, uint32_t block_tokens)
{
    if (!b)
        return set_error(SGDRC_EINVAL, "blocks is NULL");
    if (b->n_requests < 1 || b->n_requests > SGDRC_MAX_REQUESTS)
        return set_error(SGDRC_EINVAL, "n_requests %u outside 1..%d", b->n_requests, SGDRC_MAX_REQUESTS);
    const uint32_t width = blocks_width(b);
    if (width < 1 || (uint64_t)width * block_tokens > 0x7FFFFFFFull)
        return set_error(SGDRC_EINVAL, "a table row of %u blocks: none, or 2^31 tokens or more", width);
    if (width > b->stride)
        return set_error(SGDRC_EINVAL, "a table row of %u blocks, %u entries apart", width, b->stride);
    return check_aligned(b->table, 4, "blocks.table");
}

int check_rows(const sgdrc_rows *r, const char *name)
{
    if (!r)
        return set_error(SGDRC_EINVAL, "%s is NULL", name);
    const int rc = check_aligned(r->ptr, 16, name);
    if (rc)
        return rc;
    if ((r->token_stride | r->head_stride) & 7u)
        return set_error(SGDRC_EINVAL, "%s: strides must be multiples of 8 elements", name);
    if (r->token_stride > (1ull << 30) || r->head_stride > (1ull << 30))
        return set_error(SGDRC_EINVAL, "%s: stride above 2^30 elements", name);
    return SGDRC_OK;
}

static int kv_layer(const sgdrc_kv_cache *c, uint32_t layer)
{
    if (layer >= c->n_layers)
        return set_error(SGDRC_EINVAL, "layer %u of %u", layer, c->n_layers);
    return SGDRC_OK;
}

// Launches kernel ``k`` of ``tiles`` tiles on the stream's allowed CUs.
template <typename K, typename... A>
static int launch_tiles(sgdrc_ctx *ctx, void *stream, uint64_t tiles, int occ, K k, A... args)
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
    hipLaunchKernelGGL(k, dim3(gated_grid(c, occ, tiles, li)), dim3(kKvThreads), 0, s, args..., (uint32_t)tiles, g);
    SGDRC_HIP(hipGetLastError());
    return finish_static_tlog(g, s);
}

// Tiles of 16 tokens as long as the GPU holds them all at once.
constexpr uint64_t kAppendShort = 2048;

template <int D, int TOKENS>
static int launch_append_tiles(sgdrc_ctx *ctx, const sgdrc_kv_cache *cache, uint32_t layer, const sgdrc_rows *k,
                               const sgdrc_rows *v, const int64_t *slots, uint32_t n_tokens, void *stream)
{
    static const int occ = occupancy(k_kv_append<D, TOKENS>, kKvThreads);
    const uint64_t tiles = ((uint64_t)n_tokens + TOKENS - 1u) / TOKENS * cache->kv_heads;
    return launch_tiles(ctx, stream, tiles, occ, k_kv_append<D, TOKENS>, kv_view(cache, layer), rows_view(k),
                        rows_view(v), slots, n_tokens);
}

template <int D>
static int launch_append(sgdrc_ctx *ctx, const sgdrc_kv_cache *cache, uint32_t layer, const sgdrc_rows *k,
                         const sgdrc_rows *v, const int64_t *slots, uint32_t n_tokens, void *stream)
{
    return ((uint64_t)n_tokens + 15u) / 16u * cache->kv_heads <= kAppendShort
               ? launch_append_tiles<D, 16>(ctx, cache, layer, k, v, slots, n_tokens, stream)
               : launch_append_tiles<D, 32>(ctx, cache, layer, k, v, slots, n_tokens, stream);
}

template <int D>
static int launch_commit(sgdrc_ctx *ctx, const sgdrc_kv_cache *cache, const CommitArgs &a, uint32_t n_requests,
                         void *stream)
{
    static const int occ = occupancy(k_kv_commit<D>, kKvThreads);
    return launch_tiles(ctx, stream, (uint64_t)n_requests * cache->n_layers, occ, k_kv_commit<D>, kv_view(cache, 0), a,
                        n_requests);
}

static int commit(sgdrc_ctx *ctx, const sgdrc_kv_cache *cache, const sgdrc_kv_blocks *blocks, const int32_t *d_lens,
                  const int32_t *d_totals, const int32_t *d_path, uint32_t path_stride, const int32_t *d_accepted,
                  int32_t *d_lens_out, void *stream)
{
    int rc = check_kv_cache(cache);
    if (rc || (rc = check_kv_blocks(blocks, cache->block_tokens)))
        return rc;
    if ((rc = check_aligned(d_lens, 4, "lens")) || (rc = check_aligned(d_path, 4, "path")) ||
        (rc = check_aligned(d_accepted, 4, "accepted")) || (rc = check_aligned(d_lens_out, 4, "lens_out")))
        return rc;
    if (d_lens == d_lens_out || d_totals == d_lens_out)
        return set_error(SGDRC_EINVAL, "lens_out shares memory with lens or totals");
    if (path_stride < 1 || path_stride > SGDRC_MAX_NODES)
        return set_error(SGDRC_EINVAL, "path_stride %u outside 1..%d", path_stride, SGDRC_MAX_NODES);
    const CommitArgs a = {cache->n_layers > 1 ? cache->layer_stride : 0, blocks->table, d_lens, d_totals, d_path, d_accepted,
                          d_lens_out, blocks->stride, blocks_width(blocks), path_stride};
    switch (cache->head_dim) {
    case 64: return launch_commit<64>(ctx, cache, a, blocks->n_requests, stream);
    case 96: return launch_commit<96>(ctx, cache, a, blocks->n_requests, stream);
    case 128: return launch_commit<128>(ctx, cache, a, blocks->n_requests, stream);
    default: return launch_commit<256>(ctx, cache, a, blocks->n_requests, stream);
    }
}

}  // namespace sgdrc

using namespace sgdrc;

extern "C" {

int colored_kv_map(sgdrc_ctx *ctx, uint32_t block_tokens, const sgdrc_kv_state *in, const sgdrc_kv_state *out,
                   uint32_t *d_ring, uint32_t ring_size, const sgdrc_kv_blocks *blocks, const int32_t *d_new,
                   uint32_t *d_q_start, int64_t *d_slots, int32_t *d_request, int32_t *d_position, uint32_t n_tokens,
                   void *stream)
{
    clear_error();
    int rc = check_block_tokens(block_tokens);
    if (rc || (rc = check_kv_blocks(blocks, block_tokens)))
        return rc;
    if (!in || !out)
        return set_error(SGDRC_EINVAL, "in or out is NULL");
    if ((rc = check_aligned(in->ring_pos, 8, "in.ring_pos")) || (rc = check_aligned(in->held, 4, "in.held")) ||
        (rc = check_aligned(in->lens, 4, "in.lens")) || (rc = check_aligned(out->ring_pos, 8, "out.ring_pos")) ||
        (rc = check_aligned(out->held, 4, "out.held")) || (rc = check_aligned(out->lens, 4, "out.lens")) ||
        (rc = check_aligned(d_ring, 4, "ring")) || (rc = check_aligned(d_new, 4, "new")) ||
        (rc = check_aligned(d_q_start, 4, "q_start")))
        return rc;
    if (in->ring_pos == out->ring_pos || in->held == out->held || in->lens == out->lens)
        return set_error(SGDRC_EINVAL, "in and out share memory");
    if (ring_size == 0)
        return set_error(SGDRC_EINVAL, "ring_size is 0");
    if (n_tokens > 0x7FFFFFFFu)
        return set_error(SGDRC_EINVAL, "n_tokens above 2^31 - 1");
    if (n_tokens && ((rc = check_aligned(d_slots, 8, "slots")) || (rc = check_aligned(d_request, 4, "request")) ||
                     (rc = check_aligned(d_position, 4, "position"))))
        return rc;
    const MapArgs a = {in->ring_pos, in->held, in->lens, d_new, out->ring_pos, out->held, out->lens, d_ring,
                       blocks->table, d_q_start, d_slots, d_request, d_position, ring_size, blocks->stride,
                       blocks_width(blocks), (uint32_t)__builtin_ctz(block_tokens), blocks->n_requests, n_tokens};
    const uint64_t tiles = std::max<uint64_t>((blocks->n_requests + kMapTile - 1u) / kMapTile,
                                              ((uint64_t)n_tokens + kMapTile - 1u) / kMapTile);
    static const int occ = occupancy(k_kv_map, kKvThreads);
    return launch_tiles(ctx, stream, tiles, occ, k_kv_map, a);
}

int colored_kv_append(sgdrc_ctx *ctx, const sgdrc_kv_cache *cache, uint32_t layer, const sgdrc_rows *k,
                      const sgdrc_rows *v, const int64_t *d_slots, uint32_t n_tokens, void *stream)
{
    clear_error();
    int rc = check_kv_cache(cache);
    if (rc || (rc = kv_layer(cache, layer)))
        return rc;
    if (n_tokens > 0x7FFFFFFFu || (uint64_t)n_tokens * cache->kv_heads / 16u >= (1ull << 31) - 65536u)
        return set_error(SGDRC_EINVAL, "too many tokens");
    if (n_tokens && ((rc = check_rows(k, "k")) || (rc = check_rows(v, "v")) ||
                     (rc = check_aligned(d_slots, 8, "slots"))))
        return rc;
    if (n_tokens == 0) {
        Ctx *c = nullptr;
        return check_ctx(ctx, &c);
    }
    switch (cache->head_dim) {
    case 64: return launch_append<64>(ctx, cache, layer, k, v, d_slots, n_tokens, stream);
    case 96: return launch_append<96>(ctx, cache, layer, k, v, d_slots, n_tokens, stream);
    case 128: return launch_append<128>(ctx, cache, layer, k, v, d_slots, n_tokens, stream);
    default: return launch_append<256>(ctx, cache, layer, k, v, d_slots, n_tokens, stream);
    }
}

int colored_kv_commit(sgdrc_ctx *ctx, const sgdrc_kv_cache *cache, const sgdrc_kv_blocks *blocks,
                      const int32_t *d_lens, const int32_t *d_path, uint32_t path_stride, const int32_t *d_accepted,
                      int32_t *d_lens_out, void *stream)
{
    clear_error();
    return commit(ctx, cache, blocks, d_lens, nullptr, d_path, path_stride, d_accepted, d_lens_out, stream);
}

int colored_kv_commit_within(sgdrc_ctx *ctx, const sgdrc_kv_cache *cache, const sgdrc_kv_blocks *blocks,
                             const int32_t *d_lens, const int32_t *d_totals, const int32_t *d_path,
                             uint32_t path_stride, const int32_t *d_accepted, int32_t *d_lens_out, void *stream)
{
    clear_error();
    const int rc = check_aligned(d_totals, 4, "totals");
    return rc ? rc
              : commit(ctx, cache, blocks, d_lens, d_totals, d_path, path_stride, d_accepted, d_lens_out, stream);
}

}  // extern "C"
