// Queries and keys between projection and attention: the norm of each head, the
// rotation by the token's place, the write of the queries and, to the paged
// cache, of keys and values, in one pass.
#include <algorithm>
#include <cmath>

#include "kv_common.hpp"

namespace sgdrc {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

struct RotateArgs {
    RowsView q, k, v;
    uint8_t *q_out;
    uint64_t out_token, out_head;  // bytes
    const int64_t *slots;
    const int32_t *position;
    const uint8_t *q_norm, *k_norm;
    const float *freq;
    uint32_t n_heads, n_tokens, turn, norm_dtype, interleaved;  // turn: rotated pieces' pairs of a row
    float eps;
    uint32_t row_end;           // tiles of rows
    uint32_t q_tiles, k_tiles;  // of them along the heads of queries and of keys
    uint32_t q_heads, k_heads;  // heads of one
};

// Two 16-bit numbers as fp32, and back (rounded to nearest even).
template <int DT>
__device__ __forceinline__ f32x2 widen(uint32_t w)
{
    if (DT == SGDRC_BF16)
        return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)};
    const f16x2 v = __builtin_bit_cast(f16x2, w);
    return f32x2{(float)v.x, (float)v.y};
}

template <int DT>
__device__ __forceinline__ uint32_t narrow(float x, float y)
{
    const f32x2 v = {x, y};
    if (DT == SGDRC_BF16)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
    else
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}

// 16 bytes from anywhere.
struct __attribute__((packed, aligned(2))) Bytes16 {
    u32x4 v;
};

__device__ __forceinline__ u32x4 load_any(const void *p) { return static_cast<const Bytes16 *>(p)->v; }

// Eight weights of a norm, from weight ``i`` on.
__device__ __forceinline__ void norm_weights(const uint8_t *w, uint32_t dtype, uint32_t i, float (&f)[8])
{
    u32x4 a = load_any(w + i * (dtype == SGDRC_F32 ? 4u : 2u)), b = {0u, 0u, 0u, 0u};
    if (dtype == SGDRC_F32) {
        b = load_any(w + i * 4u + 16u);
        const uint32_t x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            f[e] = __uint_as_float(x[e]);
    } else {
        const uint32_t x[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const f32x2 v = dtype == SGDRC_BF16 ? widen<SGDRC_BF16>(x[e]) : widen<SGDRC_F16>(x[e]);
            f[2 * e] = v.x;
            f[2 * e + 1] = v.y;
        }
    }
}

// ``v`` of another lane of the same 16: CTRL is a DPP control that swaps neighbours
// (0xB1), pairs (0x4E), or mirrors 8 lanes (0x141) or 16 (0x140).
template <int CTRL>
__device__ __forceinline__ float lane_swap(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}

// Sum over groups of G lanes (mirroring does for exchanging halves whose lanes hold the same).
template <uint32_t G>
__device__ __forceinline__ float lanes_sum(float v)
{
    v += lane_swap<0xB1>(v);
    v += lane_swap<0x4E>(v);
    if (G >= 8)
        v += lane_swap<0x141>(v);
    if (G >= 16)
        v += lane_swap<0x140>(v);
    return v;
}

// A row is shared by D / 16 lanes, each of which has two 16-byte pieces: of what turns,
// pieces j and j + rot / 16, whose elements turn with each other (halves) or among
// themselves (neighbours); the lanes behind share what does not turn alike.  So a
// rotation stays within a lane, and a norm is a sum over a few lanes.
struct Turn {
    float f[8], g[8];  // the pairs' elements
};

// The elements of a lane's pieces.
template <int DT>
__device__ __forceinline__ Turn turn_in(u32x4 x0, u32x4 x1, bool mixed)
{
    uint32_t fw[4] = {x0.x, x0.y, x0.z, x0.w}, gw[4] = {x1.x, x1.y, x1.z, x1.w};
    if (mixed) {
        const uint32_t w[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
#pragma unroll
        for (uint32_t e = 0; e < 4u; ++e) {
            fw[e] = __builtin_amdgcn_perm(w[2 * e + 1], w[2 * e], 0x05040100u);
            gw[e] = __builtin_amdgcn_perm(w[2 * e + 1], w[2 * e], 0x07060302u);
        }
    }
    Turn t;
#pragma unroll
    for (uint32_t e = 0; e < 4u; ++e) {
        const f32x2 a0 = widen<DT>(fw[e]), a1 = widen<DT>(gw[e]);
        t.f[2 * e] = a0.x;
        t.f[2 * e + 1] = a0.y;
        t.g[2 * e] = a1.x;
        t.g[2 * e + 1] = a1.y;
    }
    return t;
}

// The pieces of elements times r.
template <int DT>
__device__ __forceinline__ void turn_out(const Turn &t, float r, bool mixed, u32x4 &y0, u32x4 &y1)
{
    uint32_t fw[4], gw[4];
#pragma unroll
    for (uint32_t e = 0; e < 4u; ++e) {
        fw[e] = narrow<DT>(r * t.f[2 * e], r * t.f[2 * e + 1]);
        gw[e] = narrow<DT>(r * t.g[2 * e], r * t.g[2 * e + 1]);
    }
    y0 = u32x4{fw[0], fw[1], fw[2], fw[3]};
    y1 = u32x4{gw[0], gw[1], gw[2], gw[3]};
    if (mixed) {
        uint32_t w[8];
#pragma unroll
        for (uint32_t e = 0; e < 4u; ++e) {
            w[2 * e] = __builtin_amdgcn_perm(gw[e], fw[e], 0x05040100u);
            w[2 * e + 1] = __builtin_amdgcn_perm(gw[e], fw[e], 0x07060302u);
        }
        y0 = u32x4{w[0], w[1], w[2], w[3]};
        y1 = u32x4{w[4], w[5], w[6], w[7]};
    }
}

// 1 / the length of a row over sqrt(D).
template <uint32_t G, int D>
__device__ __forceinline__ float turn_norm(const Turn &t, float eps)
{
    float sum = 0.0f;
#pragma unroll
    for (uint32_t e = 0; e < 8u; ++e)
        sum = __builtin_fmaf(t.g[e], t.g[e], __builtin_fmaf(t.f[e], t.f[e], sum));
    return rsqrtf(lanes_sum<G>(sum) * (1.0f / D) + eps);
}

// The weights of a lane's pairs (1 without).
__device__ __forceinline__ void turn_weights(const uint8_t *w, uint32_t dtype, bool on, bool mixed, uint32_t p0,
                                             uint32_t p1, float (&fc)[8], float (&gc)[8])
{
#pragma unroll
    for (uint32_t e = 0; e < 8u; ++e)
        fc[e] = gc[e] = 1.0f;
    if (w && on) {
        float x[2][8];
        norm_weights(w, dtype, p0 * 8u, x[0]);
        norm_weights(w, dtype, p1 * 8u, x[1]);
#pragma unroll
        for (uint32_t e = 0; e < 8u; ++e) {
            fc[e] = mixed ? x[e / 4u][2u * (e % 4u)] : x[0][e];
            gc[e] = mixed ? x[e / 4u][2u * (e % 4u) + 1u] : x[1][e];
        }
    }
}

// Sine and cosine of position * freq: turns, and what they leave of a whole number, in 64 bits.
__device__ __forceinline__ void turn_angle(int32_t position, float freq, float &sn, float &cs)
{
    const double rev = (double)position * (double)freq * 0.15915494309189533577;
    sincospif(2.0f * (float)(rev - __builtin_rint(rev)), &sn, &cs);
}

// Two kinds of tiles.  Rows, queries or keys: tokens side by side (a key's 16-byte pieces of
// neighbouring tokens lie side by side in the cache), a token's angles, worked out
// once by the row's lanes and multiplied with the norm's weights, serve the tile's
// heads, of which U are on their way at a time, loaded together and then stored, so
// that no load queues behind a store.  Values: as in k_kv_append.
//
// 16384 tokens of 32 + 8 + 8 heads of 128, 403 MB: 91 us on MI355X (4.5 TB/s), without norms and
// rotation too: the movement in this shape bounds it.  A load or store of a wavefront takes 128 bytes of each of
// eight rows, the other halves come by a second one, as a lane's two pieces lie half a
// rotation apart (lanes side by side over whole rows, with a pair's partners
// in other lanes, have not been measured).  U = 2 reloaded one by
// one, four workgroups a CU, 104; U = 8, two workgroups, 102; U = 4, four workgroups, with
// spilled registers, 110; a token's heads side by side, its angles by way of LDS, 114.
template <int DT, int D, int TOKENS>
__global__ __launch_bounds__(kKvThreads) __attribute__((amdgpu_waves_per_eu(3))) void k_kv_rotate(
    KvView c, RotateArgs a, uint32_t n_tiles, Gate g)
{
    constexpr uint32_t P = D / 16;                          // lanes of a row
    constexpr uint32_t G = P <= 4 ? 4 : P <= 8 ? 8 : 16;    // lanes from a row to the next
    constexpr uint32_t kRowTokens = kKvThreads / G;
    constexpr uint32_t U = 4;                               // heads on their way
    constexpr uint32_t V16 = D / 8;
    constexpr uint32_t kLoads = (TOKENS * V16 + kKvThreads - 1u) / kKvThreads;
    __shared__ ValueTurn<D, TOKENS> s;
    const uint32_t j = threadIdx.x % G;
    const bool mixed = a.interleaved != 0u, turns = j < a.turn;
    const uint32_t p0 = turns ? j : j + a.turn, p1 = turns ? j + a.turn : j + P;

    auto rows = [&](uint32_t t, uint32_t &err) __attribute__((always_inline)) {
        const uint32_t per = a.q_tiles + a.k_tiles, ht = t % per;
        const bool is_k = ht >= a.q_tiles;
        const uint32_t most = is_k ? a.k_heads : a.q_heads, h0 = (is_k ? ht - a.q_tiles : ht) * most;
        const uint32_t n = min(most, (is_k ? c.heads : a.n_heads) - h0);
        const uint32_t tok = t / per * kRowTokens + threadIdx.x / G;
        const uint32_t tt = min(tok, a.n_tokens - 1u);
        const uint64_t stride = is_k ? a.k.head : a.q.head;
        const uint8_t *const from = is_k ? a.k.ptr + tt * a.k.token : a.q.ptr + tt * a.q.token;
        // (rows of tokens that are left out are read, too: no load waits for the position)
        u32x4 x[U][2];
        auto load = [&](uint32_t h) __attribute__((always_inline)) {
#pragma unroll
            for (uint32_t i = 0; i < U; ++i) {
                const uint8_t *const row = from + (h0 + min(h + i, n - 1u)) * stride;
                x[i][0] = x[i][1] = u32x4{0u, 0u, 0u, 0u};
                if (j < P && h + i < n) {
                    x[i][0] = load_nt(row + p0 * 16u);
                    x[i][1] = load_nt(row + p1 * 16u);
                }
            }
        };
        load(0u);
        const int32_t pos = a.position[tt];
        bool write = tok < a.n_tokens && j < P && pos >= 0;
        uint8_t *to = a.q_out + tt * a.out_token + h0 * a.out_head;
        uint64_t step = a.out_head;
        uint32_t o0 = p0 * 16u, o1 = p1 * 16u;
        if (is_k) {
            const int64_t slot = a.slots[tt];
            const bool out = slot < -1 || (slot >= 0 && ((uint64_t)slot >> c.bshift) >= c.pool_pages);
            err |= out && pos >= 0 ? kDevErrSeq : 0u;
            write = write && slot >= 0 && !out;
            const uint64_t held = write ? (uint64_t)slot : 0ull;
            const uint32_t at = (uint32_t)held & ((1u << c.bshift) - 1u);
            step = head_bytes<D>(c.bshift);
            to = c.pool + ((held >> c.bshift) << c.shift) + h0 * step;
            o0 = k_off<D>(p0, at, c.bshift);
            o1 = k_off<D>(p1, at, c.bshift);
        }
        // For pair e: (f, g) -> (f fc - g gs, f fs + g gc), with the weights of f and g
        // multiplied in.
        const uint8_t *const weights = is_k ? a.k_norm : a.q_norm;
        float fc[8], fs[8], gc[8], gs[8];
        turn_weights(weights, a.norm_dtype, j < P, mixed, p0, p1, fc, gc);
#pragma unroll
        for (uint32_t e = 0; e < 8u; ++e)
            fs[e] = gs[e] = 0.0f;
        if (turns) {
            const u32x4 f0 = load_any(a.freq + (mixed ? p0 * 4u : j * 8u));
            const u32x4 f1 = load_any(a.freq + (mixed ? p1 * 4u : j * 8u + 4u));
            const uint32_t freq[8] = {f0.x, f0.y, f0.z, f0.w, f1.x, f1.y, f1.z, f1.w};
#pragma unroll
            for (uint32_t e = 0; e < 8u; ++e) {
                float cs, sn;
                turn_angle(pos, __uint_as_float(freq[e]), sn, cs);
                fs[e] = fc[e] * sn;
                gs[e] = gc[e] * sn;
                fc[e] *= cs;
                gc[e] *= cs;
                __builtin_amdgcn_sched_barrier(0);  // (one after the other: registers)
            }
        }
        for (uint32_t h = 0; h < n; h += U) {
            if (h)
                load(h);
#pragma unroll
            for (uint32_t i = 0; i < U; ++i) {
                const Turn e = turn_in<DT>(x[i][0], x[i][1], mixed);
                const float r = weights ? turn_norm<G, D>(e, a.eps) : 1.0f;
                Turn o;
#pragma unroll
                for (uint32_t k = 0; k < 8u; ++k) {
                    o.f[k] = e.f[k] * fc[k];
                    o.g[k] = e.g[k] * gc[k];
                }
                if (turns) {  // (what does not turn stays as it is, infinities too)
#pragma unroll
                    for (uint32_t k = 0; k < 8u; ++k) {
                        o.f[k] = __builtin_fmaf(-e.g[k], gs[k], o.f[k]);
                        o.g[k] = __builtin_fmaf(e.f[k], fs[k], o.g[k]);
                    }
                }
                u32x4 y0, y1;
                turn_out<DT>(o, r, mixed, y0, y1);
                if (write && h + i < n) {
                    store_nt(to + o0, y0);
                    store_nt(to + o1, y1);
                }
                to += step;
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    auto values = [&](uint32_t t, uint32_t &err) {
        const uint32_t h = t % c.heads, t0 = t / c.heads * (uint32_t)TOKENS;
        u32x4 vv[kLoads];
#pragma unroll
        for (uint32_t l = 0; l < kLoads; ++l) {
            const uint32_t i = l * kKvThreads + threadIdx.x;
            const uint32_t tv = min(t0 + i / V16, a.n_tokens - 1u);
            vv[l] = u32x4{0u, 0u, 0u, 0u};
            if (i < TOKENS * V16)
                vv[l] = *reinterpret_cast<const u32x4 *>(a.v.ptr + tv * a.v.token + h * a.v.head + (i % V16) * 16u);
        }
        __syncthreads();  // the last tile's LDS is read
        s.take_slots(c, a.slots, a.position, t0, a.n_tokens, err);
        __syncthreads();
        s.sort_out();
#pragma unroll
        for (uint32_t l = 0; l < kLoads; ++l) {
            const uint32_t i = l * kKvThreads + threadIdx.x;
            if (i < TOKENS * V16)
                *reinterpret_cast<u32x4 *>(&s.v[i / V16][(i % V16) * 8u]) = vv[l];
        }
        __syncthreads();
        s.write(c, a.v, t0, h);
    };
    auto body = [&](uint32_t t, uint32_t &err) {
        if (t < a.row_end)
            rows(t, err);
        else
            values(t - a.row_end, err);
    };
    single_tile_loop(g, n_tiles, NoOp(), body);
}

// Tiles of rows that the GPU holds at once, about: heads are put together as long as there
// are more.
constexpr uint64_t kRowTiles = 2048;

template <int DT, int D, int TOKENS>
static int launch_rotate(sgdrc_ctx *ctx, const sgdrc_kv_cache *cache, uint32_t layer, RotateArgs a, void *stream)
{
    constexpr uint32_t P = D / 16, G = P <= 4 ? 4 : P <= 8 ? 8 : 16, kRowTokens = kKvThreads / G;
    static const int occ = occupancy(k_kv_rotate<DT, D, TOKENS>, kKvThreads);
    const uint32_t heads = a.n_heads + cache->kv_heads;
    const uint64_t row_groups = ((uint64_t)a.n_tokens + kRowTokens - 1u) / kRowTokens;
    const uint32_t most = (uint32_t)std::min<uint64_t>(heads, (row_groups * heads + kRowTiles - 1u) / kRowTiles);
    const auto tiles_of = [&](uint32_t n, uint32_t &tile) {
        const uint32_t t = (n + most - 1u) / most;
        tile = (n + t - 1u) / t;
        return (n + tile - 1u) / tile;
    };
    a.q_tiles = tiles_of(a.n_heads, a.q_heads);
    a.k_tiles = tiles_of(cache->kv_heads, a.k_heads);
    const uint64_t rows = row_groups * (a.q_tiles + a.k_tiles);
    const uint64_t tiles = rows + ((uint64_t)a.n_tokens + TOKENS - 1u) / TOKENS * cache->kv_heads;
    if (tiles >= (1ull << 31))
        return set_error(SGDRC_EINVAL, "too many tokens");
    a.row_end = (uint32_t)rows;
    return launch_tiles(ctx, stream, tiles, occ, kKvThreads, k_kv_rotate<DT, D, TOKENS>, kv_view(cache, layer), a);
}

template <int DT, int D>
static int launch_rotate_size(sgdrc_ctx *ctx, const sgdrc_kv_cache *cache, uint32_t layer, const RotateArgs &a,
                              void *stream)
{
    // (as colored_kv_append: tiles of 16 values as long as the GPU holds them all at once)
    return ((uint64_t)a.n_tokens + 15u) / 16u * cache->kv_heads <= 2048u
               ? launch_rotate<DT, D, 16>(ctx, cache, layer, a, stream)
               : launch_rotate<DT, D, 32>(ctx, cache, layer, a, stream);
}

template <int DT>
static int launch_rotate_dim(sgdrc_ctx *ctx, const sgdrc_kv_cache *cache, uint32_t layer, const RotateArgs &a,
                             void *stream)
{
    switch (cache->head_dim) {
    case 64: return launch_rotate_size<DT, 64>(ctx, cache, layer, a, stream);
    case 96: return launch_rotate_size<DT, 96>(ctx, cache, layer, a, stream);
    case 128: return launch_rotate_size<DT, 128>(ctx, cache, layer, a, stream);
    default: return launch_rotate_size<DT, 256>(ctx, cache, layer, a, stream);
    }
}

static int check_rotation(const sgdrc_rotation *r, uint32_t head_dim)
{
    if (!r)
        return set_error(SGDRC_EINVAL, "rotation is NULL");
    if (r->rot_dims > head_dim || r->rot_dims % 16u)
        return set_error(SGDRC_EINVAL, "rotation: rot_dims %u is not a multiple of 16 up to %u", r->rot_dims, head_dim);
    if (r->interleaved > 1u || r->norm_dtype > SGDRC_F16)
        return set_error(SGDRC_EINVAL, "rotation: interleaved %u, norm_dtype %u", r->interleaved, r->norm_dtype);
    if (!(r->eps >= 0.0f) || !std::isfinite(r->eps))
        return set_error(SGDRC_EINVAL, "rotation: eps is negative or not finite");
    int rc = r->rot_dims ? check_aligned(r->freq, 4, "rotation.freq") : SGDRC_OK;
    const uint32_t size = r->norm_dtype == SGDRC_F32 ? 4u : 2u;
    for (const void *w : {r->q_norm, r->k_norm})
        if (!rc && w)
            rc = check_aligned(w, size, "rotation: weights");
    return rc;
}

}  // namespace sgdrc

using namespace sgdrc;

extern "C" int colored_kv_append_rotated(sgdrc_ctx *ctx, const sgdrc_kv_cache *cache, uint32_t layer,
                                         const sgdrc_rows *q, uint32_t n_heads, const sgdrc_rows *q_out,
                                         const sgdrc_rows *k, const sgdrc_rows *v, const int64_t *d_slots,
                                         const int32_t *d_position, uint32_t n_tokens, const sgdrc_rotation *rotation,
                                         void *stream)
{
    clear_error();
    int rc = check_kv_cache(cache);
    if (rc || (rc = check_layer(cache, layer)) || (rc = check_rotation(rotation, cache->head_dim)))
        return rc;
    if (n_heads < 1 || n_heads > SGDRC_MAX_HEADS || n_heads % cache->kv_heads)
        return set_error(SGDRC_EINVAL, "%u heads on %u key/value heads", n_heads, cache->kv_heads);
    if (n_tokens > 0x7FFFFFFFu)
        return set_error(SGDRC_EINVAL, "too many tokens");
    if (n_tokens && ((rc = check_rows(q, "q")) || (rc = check_rows(q_out, "q_out")) || (rc = check_rows(k, "k")) ||
                     (rc = check_rows(v, "v")) || (rc = check_aligned(d_slots, 8, "slots")) ||
                     (rc = check_aligned(d_position, 4, "position"))))
        return rc;
    if (n_tokens == 0) {
        Ctx *c = nullptr;
        return check_ctx(ctx, &c);
    }
    const RotateArgs a = {rows_view(q), rows_view(k), rows_view(v), static_cast<uint8_t *>(q_out->ptr),
                          q_out->token_stride * 2u, q_out->head_stride * 2u, d_slots, d_position,
                          static_cast<const uint8_t *>(rotation->q_norm), static_cast<const uint8_t *>(rotation->k_norm),
                          rotation->freq, n_heads, n_tokens, rotation->rot_dims / 16u, rotation->norm_dtype,
                          rotation->interleaved, rotation->eps, 0u, 0u, 0u, 0u, 0u};
    return cache->dtype == SGDRC_BF16 ? launch_rotate_dim<SGDRC_BF16>(ctx, cache, layer, a, stream)
                                      : launch_rotate_dim<SGDRC_F16>(ctx, cache, layer, a, stream);
}
