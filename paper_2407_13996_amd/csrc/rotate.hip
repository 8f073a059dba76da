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
    uint32_t row_tiles, head_tiles;  // tiles of queries and keys; of them along the heads
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

// Eight elements of weights of a norm.
__device__ __forceinline__ void norm_weights(const uint8_t *w, uint32_t dtype, uint32_t at, float (&f)[8])
{
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
        if (dtype == SGDRC_F32)
            f[i] = reinterpret_cast<const float *>(w)[at + i];
        else if (dtype == SGDRC_BF16)
            f[i] = __uint_as_float((uint32_t) reinterpret_cast<const uint16_t *>(w)[at + i] << 16);
        else
            f[i] = (float)reinterpret_cast<const _Float16 *>(w)[at + i];
    }
}

// Tiles of rows (queries and keys): a row is shared by D / 16 lanes, each of which has
// two 16-byte pieces whose elements turn together: pieces j and j + rot / 16 where
// the halves of the rotated part are paired, 2 j and 2 j + 1 where neighbours are
// (and in what does not turn).  So a rotation stays within a lane, a norm is a sum
// over a few lanes, and a token's angles, worked out once, serve HEADS heads.
// Tiles of values: as in k_kv_append.
template <int DT, int D, int HEADS, int TOKENS>
__global__ __launch_bounds__(kKvThreads) void k_kv_rotate(KvView c, RotateArgs a, uint32_t n_tiles, Gate g)
{
    constexpr uint32_t P = D / 16;                          // lanes of a row
    constexpr uint32_t G = P <= 4 ? 4 : P <= 8 ? 8 : 16;    // lanes from a row to the next
    constexpr uint32_t kRowTokens = kKvThreads / G;
    constexpr uint32_t V16 = D / 8;
    constexpr uint32_t kLoads = (TOKENS * V16 + kKvThreads - 1u) / kKvThreads;
    __shared__ ValueTurn<D, TOKENS> s;
    const uint32_t j = threadIdx.x % G;
    const bool turns = j < a.turn;
    const uint32_t p0 = turns && !a.interleaved ? j : 2u * j, p1 = turns && !a.interleaved ? j + a.turn : 2u * j + 1u;

    auto rows = [&](uint32_t t, uint32_t &err) {
        const uint32_t h0 = t % a.head_tiles * HEADS;
        const uint32_t tok = t / a.head_tiles * kRowTokens + threadIdx.x / G;
        const uint32_t tt = min(tok, a.n_tokens - 1u);
        const int32_t pos = a.position[tt];
        const bool on = tok < a.n_tokens && j < P && pos >= 0;
        const uint32_t heads = a.n_heads + c.heads;
        u32x4 x[HEADS][2];
#pragma unroll
        for (uint32_t i = 0; i < HEADS; ++i) {
            const uint32_t h = min(h0 + i, heads - 1u);
            const bool is_k = h >= a.n_heads;
            const uint8_t *const row = is_k ? a.k.ptr + tt * a.k.token + (h - a.n_heads) * a.k.head
                                            : a.q.ptr + tt * a.q.token + h * a.q.head;
            const u32x4 z = {0u, 0u, 0u, 0u};
            x[i][0] = on ? *reinterpret_cast<const u32x4 *>(row + p0 * 16u) : z;
            x[i][1] = on ? *reinterpret_cast<const u32x4 *>(row + p1 * 16u) : z;
        }
        int64_t slot = a.slots[tt];
        if (slot < -1 || (slot >= 0 && ((uint64_t)slot >> c.bshift) >= c.pool_pages)) {
            err |= pos >= 0 ? kDevErrSeq : 0u;
            slot = -1;
        }
        float cs[8], sn[8];
        if (turns) {
#pragma unroll
            for (uint32_t e = 0; e < 8u; ++e) {
                // turns, and what they leave of a whole number, in 64 bits
                const double rev = (double)pos * (double)a.freq[j * 8u + e] * 0.15915494309189533577;
                sincospif(2.0f * (float)(rev - __builtin_rint(rev)), &sn[e], &cs[e]);
            }
        }
#pragma unroll
        for (uint32_t i = 0; i < HEADS; ++i) {
            const uint32_t h = h0 + i;
            const bool is_k = h >= a.n_heads;
            float f[2][8];
#pragma unroll
            for (uint32_t q = 0; q < 2u; ++q)
#pragma unroll
                for (uint32_t e = 0; e < 4u; ++e) {
                    const uint32_t word = x[i][q][e];
                    const f32x2 w = widen<DT>(word);
                    f[q][2 * e] = w.x;
                    f[q][2 * e + 1] = w.y;
                }
            const uint8_t *const norm = is_k ? a.k_norm : a.q_norm;
            if (norm) {
                float sum = 0.0f;
#pragma unroll
                for (uint32_t e = 0; e < 8u; ++e)
                    sum += f[0][e] * f[0][e] + f[1][e] * f[1][e];
#pragma unroll
                for (uint32_t off = 1; off < G; off <<= 1)
                    sum += __shfl_xor(sum, off, 64);
                const float r = 1.0f / __builtin_sqrtf(sum * (1.0f / D) + a.eps);
                float w0[8], w1[8];
                if (j < P) {
                    norm_weights(norm, a.norm_dtype, p0 * 8u, w0);
                    norm_weights(norm, a.norm_dtype, p1 * 8u, w1);
#pragma unroll
                    for (uint32_t e = 0; e < 8u; ++e) {
                        f[0][e] *= r * w0[e];
                        f[1][e] *= r * w1[e];
                    }
                }
            }
            // (what does not turn stays as it is, infinities too)
            if (turns) {
                float u[8], w[8];
#pragma unroll
                for (uint32_t e = 0; e < 8u; ++e) {
                    u[e] = a.interleaved ? f[e / 4][2 * (e % 4)] : f[0][e];
                    w[e] = a.interleaved ? f[e / 4][2 * (e % 4) + 1] : f[1][e];
                }
#pragma unroll
                for (uint32_t e = 0; e < 8u; ++e) {
                    const float x0 = u[e] * cs[e] - w[e] * sn[e], x1 = u[e] * sn[e] + w[e] * cs[e];
                    u[e] = x0;
                    w[e] = x1;
                }
                if (a.interleaved) {
#pragma unroll
                    for (uint32_t e = 0; e < 8u; ++e) {
                        f[e / 4][2 * (e % 4)] = u[e];
                        f[e / 4][2 * (e % 4) + 1] = w[e];
                    }
                } else {
#pragma unroll
                    for (uint32_t e = 0; e < 8u; ++e) {
                        f[0][e] = u[e];
                        f[1][e] = w[e];
                    }
                }
            }
            u32x4 o[2];
#pragma unroll
            for (uint32_t q = 0; q < 2u; ++q)
#pragma unroll
                for (uint32_t e = 0; e < 4u; ++e)
                    o[q][e] = narrow<DT>(f[q][2 * e], f[q][2 * e + 1]);
            if (on && h < heads) {
                if (!is_k) {
                    uint8_t *const to = a.q_out + tok * a.out_token + h * a.out_head;
                    *reinterpret_cast<u32x4 *>(to + p0 * 16u) = o[0];
                    *reinterpret_cast<u32x4 *>(to + p1 * 16u) = o[1];
                } else if (slot >= 0) {
                    uint8_t *const to = c.pool + ((uint64_t)(slot >> c.bshift) << c.shift) +
                                        (h - a.n_heads) * head_bytes<D>(c.bshift);
                    const uint32_t at = (uint32_t)slot & ((1u << c.bshift) - 1u);
                    *reinterpret_cast<u32x4 *>(to + k_off<D>(p0, at, c.bshift)) = o[0];
                    *reinterpret_cast<u32x4 *>(to + k_off<D>(p1, at, c.bshift)) = o[1];
                }
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
        if (t < a.row_tiles)
            rows(t, err);
        else
            values(t - a.row_tiles, err);
    };
    single_tile_loop(g, n_tiles, NoOp(), body);
}

template <int DT, int D, int HEADS, int TOKENS>
static int launch_rotate(sgdrc_ctx *ctx, const sgdrc_kv_cache *cache, uint32_t layer, RotateArgs a, void *stream)
{
    constexpr uint32_t P = D / 16, G = P <= 4 ? 4 : P <= 8 ? 8 : 16, kRowTokens = kKvThreads / G;
    static const int occ = occupancy(k_kv_rotate<DT, D, HEADS, TOKENS>, kKvThreads);
    a.head_tiles = (a.n_heads + cache->kv_heads + HEADS - 1u) / HEADS;
    const uint64_t row_tiles = ((uint64_t)a.n_tokens + kRowTokens - 1u) / kRowTokens * a.head_tiles;
    const uint64_t tiles = row_tiles + ((uint64_t)a.n_tokens + TOKENS - 1u) / TOKENS * cache->kv_heads;
    if (tiles >= (1ull << 31))
        return set_error(SGDRC_EINVAL, "too many tokens");
    a.row_tiles = (uint32_t)row_tiles;
    return launch_tiles(ctx, stream, tiles, occ, kKvThreads, k_kv_rotate<DT, D, HEADS, TOKENS>, kv_view(cache, layer),
                        a);
}

template <int DT, int D>
static int launch_rotate_size(sgdrc_ctx *ctx, const sgdrc_kv_cache *cache, uint32_t layer, const RotateArgs &a,
                              void *stream)
{
    const uint64_t rows = (uint64_t)a.n_tokens * (a.n_heads + cache->kv_heads);
    return rows <= 16384u ? launch_rotate<DT, D, 1, 16>(ctx, cache, layer, a, stream)
                          : launch_rotate<DT, D, 4, 32>(ctx, cache, layer, a, stream);
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
                          rotation->interleaved, rotation->eps, 0u, 0u};
    return cache->dtype == SGDRC_BF16 ? launch_rotate_dim<SGDRC_BF16>(ctx, cache, layer, a, stream)
                                      : launch_rotate_dim<SGDRC_F16>(ctx, cache, layer, a, stream);
}
