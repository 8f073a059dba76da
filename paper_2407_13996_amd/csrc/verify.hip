// Verification of drafted trees: which nodes a sampler of the target's
// probabilities would have taken, and its next token.
#include <algorithm>

#include "kv_common.hpp"

namespace sgdrc {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int kVerifyThreads = 1024;
constexpr uint32_t kVerifyWaves = kVerifyThreads / 64;
constexpr uint32_t kSpan = 1024;       // elements that a wavefront takes at once, 16 a lane
constexpr uint32_t kMaxChunks = 512;   // of a row: the sums that are kept

struct VerifyArgs {
    const uint8_t *target, *draft;
    uint64_t target_stride, draft_stride;  // bytes
    const int32_t *tokens, *parents;
    const float *uniform;
    const uint32_t *q_start;
    const int32_t *lens, *totals;
    int32_t *path, *accepted, *next;
    uint32_t vocab, n_tokens, max_nodes, path_stride, chunk;  // chunk: elements, a multiple of kSpan
};

// A probability as it counts: 0 if not positive, no infinities.
__device__ __forceinline__ float counts(float p) { return fminf(fmaxf(p, 0.0f), 3.402823466e38f); }

template <int DT> struct Row {
    static constexpr uint32_t size = DT == SGDRC_F32 ? 4 : 2, vec = 16 / size;
};

// 16 bytes of a row from an element's address on.
struct __attribute__((packed, aligned(2))) Bytes16 {
    u32x4 v;
};

template <int DT>
__device__ __forceinline__ float row_at(const uint8_t *row, uint32_t i)
{
    if (DT == SGDRC_F32)
        return reinterpret_cast<const float *>(row)[i];
    if (DT == SGDRC_BF16)
        return __uint_as_float((uint32_t) reinterpret_cast<const uint16_t *>(row)[i] << 16);
    return (float)reinterpret_cast<const _Float16 *>(row)[i];
}

// Elements i .. i + 16 / size of a row (0 past its end).
template <int DT>
__device__ __forceinline__ void row_load(const uint8_t *row, uint32_t i, uint32_t vocab, float (&f)[Row<DT>::vec])
{
    constexpr uint32_t n = Row<DT>::vec;
    if (i + n <= vocab) {
        const u32x4 w = reinterpret_cast<const Bytes16 *>(row + (uint64_t)i * Row<DT>::size)->v;
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (uint32_t e = 0; e < n; ++e) {
            if (DT == SGDRC_F32) {
                f[e] = __uint_as_float(x[e % 4u]);
            } else if (DT == SGDRC_BF16) {
                f[e] = __uint_as_float(e % 2u ? x[e / 2u] & 0xFFFF0000u : x[e / 2u] << 16);
            } else {
                const f16x2 h = __builtin_bit_cast(f16x2, x[e / 2u]);
                f[e] = e % 2u ? (float)h.y : (float)h.x;
            }
        }
    } else {
#pragma unroll
        for (uint32_t e = 0; e < n; ++e)
            f[e] = i + e < vocab ? row_at<DT>(row, i + e) : 0.0f;
    }
#pragma unroll
    for (uint32_t e = 0; e < n; ++e)
        f[e] = counts(f[e]);
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1)
        v += __shfl_xor(v, off, 64);
    return v;  // the same bits in every lane
}

// The sum of all lanes up to this one.
__device__ __forceinline__ double wave_scan(double v, uint32_t lane)
{
#pragma unroll
    for (uint32_t off = 1; off < 64u; off <<= 1) {
        const double o = __shfl_up(v, off, 64);
        v += lane >= off ? o : 0.0;
    }
    return v;
}

// A workgroup takes a request: its nodes' tokens, random numbers and
// probabilities are fetched together, the walk is then a chain of comparisons on
// LDS.  Only a rejection (with draft rows) and the last draw need a row as a whole; they
// sum it in chunks, whose sums are kept, so that the draw looks up the
// chunk that the random number falls in and goes through that one again.
template <int DT>
__global__ __launch_bounds__(kVerifyThreads) void k_draft_verify(VerifyArgs a, uint32_t n_tiles, Gate g)
{
    constexpr uint32_t N = Row<DT>::vec;
    __shared__ int32_t s_tok[SGDRC_MAX_NODES], s_par[SGDRC_MAX_NODES], s_path[SGDRC_MAX_NODES];
    __shared__ float s_u[SGDRC_MAX_NODES], s_p[SGDRC_MAX_NODES], s_q[SGDRC_MAX_NODES];
    __shared__ uint32_t s_ex[SGDRC_MAX_NODES];  // tokens ruled out at the node (without draft rows)
    __shared__ double s_chunk[kMaxChunks];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool drawn = a.draft != nullptr;
    const uint32_t n_chunks = (a.vocab + a.chunk - 1u) / a.chunk;

    auto body = [&](uint32_t r, uint32_t &err) {
        const uint32_t q0 = a.q_start[r], q1 = a.q_start[r + 1u];
        uint32_t n = q1 - q0;
        if (q1 < q0 || q1 > a.n_tokens) {
            err |= kDevErrSeq;
            n = 0u;
        }
        if (a.lens && (int64_t)a.totals[r] - a.lens[r] < (int64_t)n)
            n = 0u;
        if (n > a.max_nodes) {
            err |= kDevErrSeq;
            n = a.max_nodes;
        }
        n = __builtin_amdgcn_readfirstlane(n);
        __syncthreads();  // the last tile's LDS is read
        if (threadIdx.x < n) {
            const uint32_t i = threadIdx.x;
            const int32_t tok = a.tokens[q0 + i];
            int32_t par = i ? a.parents[q0 + i] : -1;
            if (par < 0 || par >= (int32_t)i)
                par = -1;
            const bool in = tok >= 0 && tok < (int32_t)a.vocab;
            const uint64_t row = q0 + (uint32_t)max(par, 0);
            s_tok[i] = in ? tok : -1;
            s_par[i] = par;
            s_u[i] = a.uniform[q0 + i];
            s_p[i] = in && i ? counts(row_at<DT>(a.target + row * a.target_stride, tok)) : 0.0f;
            s_q[i] = !drawn ? 1.0f : in && i ? counts(row_at<DT>(a.draft + row * a.draft_stride, tok)) : 0.0f;
        }
        __syncthreads();
        int32_t par[SGDRC_MAX_NODES / 64];  // of nodes 64 k + lane
#pragma unroll
        for (int k = 0; k < SGDRC_MAX_NODES / 64; ++k)
            par[k] = k * 64u + lane < n ? s_par[k * 64u + lane] : -2;

        // where the walk stands: the node, the last child looked at, and what is left of the
        // distribution there
        uint32_t cur = 0u, last = 0u, depth = n ? 1u : 0u, n_ex = 0u;
        double c = 0.0, left = 1.0;
        bool summed = false;  // s_chunk holds the sums of what is left
        auto rows = [&](const uint8_t *&p, const uint8_t *&q) {
            p = a.target + (uint64_t)(q0 + cur) * a.target_stride;
            q = drawn ? a.draft + (uint64_t)(q0 + cur) * a.draft_stride : p;
        };
        auto gone = [&](uint32_t t) {
            bool x = false;
            for (uint32_t i = 0; i < n_ex; ++i)
                x = x || s_ex[i] == t;
            return x;
        };
        // weights of elements i ..  of what is left
        auto weights = [&](const uint8_t *p, const uint8_t *q, uint32_t i, bool ex, double (&w)[N]) {
            float fp[N], fq[N];
            row_load<DT>(p, i, a.vocab, fp);
            if (drawn)
                row_load<DT>(q, i, a.vocab, fq);
#pragma unroll
            for (uint32_t e = 0; e < N; ++e) {
                w[e] = drawn ? fmax((double)fp[e] - c * (double)fq[e], 0.0) : (double)fp[e];
                if (ex && gone(i + e))
                    w[e] = 0.0;
            }
        };
        // whether a ruled-out token lies in the chunk
        auto touched = [&](uint32_t ch) {
            bool x = false;
            for (uint32_t i = 0; i < n_ex; ++i)
                x = x || s_ex[i] / a.chunk == ch;
            return x;
        };
        auto sum_row = [&]() {
            const uint8_t *p, *q;
            rows(p, q);
            __syncthreads();  // the last sums are read
            for (uint32_t ch = wave; ch < n_chunks; ch += kVerifyWaves) {
                const bool ex = touched(ch);
                const uint32_t end = min((ch + 1u) * a.chunk, a.vocab);
                double sum = 0.0;
                for (uint32_t i = ch * a.chunk + lane * N; i < end; i += 64u * N) {
                    double w[N];
                    weights(p, q, i, ex, w);
#pragma unroll
                    for (uint32_t e = 0; e < N; ++e)
                        sum += w[e];
                }
                sum = wave_sum(sum);
                if (lane == 0u)
                    s_chunk[ch] = sum;
            }
            __syncthreads();
            double all = 0.0;
            for (uint32_t ch = lane; ch < n_chunks; ch += 64u)
                all += s_chunk[ch];
            summed = true;
            left = wave_sum(all);
        };

        if (threadIdx.x == 0u)
            s_path[0] = 0;
        while (depth != 0u && depth < a.path_stride) {
            uint32_t child = n;
#pragma unroll
            for (int k = SGDRC_MAX_NODES / 64 - 1; k >= 0; --k) {
                const uint64_t m = __ballot(par[k] == (int32_t)cur && k * 64u + lane > last);
                child = m ? k * 64u + (uint32_t)__builtin_ctzll(m) : child;
            }
            child = __builtin_amdgcn_readfirstlane(child);
            // (where nothing is left no child can be accepted)
            if (child >= n || __builtin_amdgcn_readfirstlane(left > 0.0 ? 0u : 1u))
                break;
            last = child;
            const uint32_t t = __builtin_amdgcn_readfirstlane((uint32_t)s_tok[child]);
            if ((int32_t)t < 0) {
                err |= kDevErrSeq;
                continue;
            }
            const double q = s_q[child];
            double w = fmax((double)s_p[child] - (drawn ? c * q : 0.0), 0.0);
            if (gone(t))
                w = 0.0;
            const bool yes = w > 0.0 && (double)s_u[child] * q * left < w;
            if (__builtin_amdgcn_readfirstlane(yes ? 1u : 0u)) {
                if (threadIdx.x == 0u)
                    s_path[depth] = (int32_t)child;
                cur = child;
                depth += 1u;
                c = 0.0;
                left = 1.0;
                n_ex = 0u;
                summed = false;
                continue;
            }
            if (drawn) {
                c += left;
            } else {
                __syncthreads();
                if (threadIdx.x == 0u)
                    s_ex[n_ex] = t;
                n_ex += 1u;
            }
            sum_row();
        }
        if (n) {
            if (!summed)
                sum_row();
            if (__builtin_amdgcn_readfirstlane(left > 0.0 ? 0u : 1u)) {
                // nothing is left: the row itself
                c = 0.0;
                n_ex = 0u;
                sum_row();
            }
        }
        int32_t next = -1;
        if (n && wave == 0u) {
            const uint8_t *p, *q;
            rows(p, q);
            const double goal = (double)s_u[0] * left;
            // The chunk that the goal falls in, of which a lane holds 8.  (Where rounding
            // leaves the goal above all sums: the last that holds anything.)
            constexpr uint32_t kHeld = kMaxChunks / 64u;
            double mine = 0.0;
            for (uint32_t k = 0; k < kHeld; ++k)
                mine += lane * kHeld + k < n_chunks ? s_chunk[lane * kHeld + k] : 0.0;
            const double upto = wave_scan(mine, lane);
            const uint64_t past = __ballot(mine > 0.0 && upto > goal), some = __ballot(mine > 0.0);
            if (some) {
                const uint32_t l = past ? (uint32_t)__builtin_ctzll(past) : 63u - (uint32_t)__builtin_clzll(some);
                double before = __shfl(upto - mine, l, 64), run = before;
                uint32_t ch = 0u;
                bool found = false;
                for (uint32_t k = 0; k < kHeld; ++k) {
                    const uint32_t x = l * kHeld + k;
                    const double s = x < n_chunks ? s_chunk[x] : 0.0;
                    if (s > 0.0 && !found) {
                        ch = x;
                        before = run;
                        run += s;
                        found = run > goal;
                    }
                }
                ch = __builtin_amdgcn_readfirstlane(ch);
                // the element likewise, 16 in a row to a lane
                const bool ex = touched(ch);
                const uint32_t end = min((ch + 1u) * a.chunk, a.vocab);
                for (uint32_t i0 = ch * a.chunk; i0 < end; i0 += kSpan) {
                    double w[16];
#pragma unroll
                    for (uint32_t k = 0; k < 16u / N; ++k) {
                        double x[N];
                        weights(p, q, i0 + lane * 16u + k * N, ex, x);
#pragma unroll
                        for (uint32_t e = 0; e < N; ++e)
                            w[k * N + e] = x[e];
                    }
                    double sum = 0.0;
#pragma unroll
                    for (uint32_t e = 0; e < 16u; ++e)
                        sum += w[e];
                    const double to = wave_scan(sum, lane);
                    const uint64_t over = __ballot(sum > 0.0 && before + to > goal), any = __ballot(sum > 0.0);
                    if (any) {
                        const uint32_t le = over ? (uint32_t)__builtin_ctzll(over) : 63u - (uint32_t)__builtin_clzll(any);
                        double at = before + (to - sum);
                        uint32_t pick = 0u;
                        bool got = false;
#pragma unroll
                        for (uint32_t e = 0; e < 16u; ++e)
                            if (w[e] > 0.0 && !got) {
                                pick = e;
                                at += w[e];
                                got = at > goal;
                            }
                        next = (int32_t)(i0 + le * 16u + __shfl(pick, le, 64));
                    }
                    if (over)
                        break;
                    before += __shfl(to, 63, 64);
                }
            }
            err |= next < 0 ? kDevErrSeq : 0u;
        }
        __syncthreads();  // the path
        if (threadIdx.x < a.path_stride)
            a.path[(uint64_t)r * a.path_stride + threadIdx.x] = threadIdx.x < depth ? s_path[threadIdx.x] : -1;
        if (threadIdx.x == 0u) {
            a.accepted[r] = (int32_t)depth;
            a.next[r] = next;
        }
    };
    single_tile_loop(g, n_tiles, NoOp(), body);
}

template <int DT>
static int launch_verify(sgdrc_ctx *ctx, const VerifyArgs &a, uint32_t n_requests, void *stream)
{
    static const int occ = occupancy(k_draft_verify<DT>, kVerifyThreads);
    return launch_tiles(ctx, stream, n_requests, occ, kVerifyThreads, k_draft_verify<DT>, a);
}

}  // namespace sgdrc

using namespace sgdrc;

extern "C" int colored_draft_verify(sgdrc_ctx *ctx, uint32_t dtype, uint32_t vocab, const void *d_target,
                                    uint64_t target_stride, const void *d_draft, uint64_t draft_stride,
                                    const int32_t *d_tokens, const int32_t *d_parents, const float *d_uniform,
                                    uint32_t n_tokens, const uint32_t *d_q_start, uint32_t n_requests,
                                    uint32_t max_nodes, const int32_t *d_lens, const int32_t *d_totals, int32_t *d_path,
                                    uint32_t path_stride, int32_t *d_accepted, int32_t *d_next, void *stream)
{
    clear_error();
    if (dtype > SGDRC_F16)
        return set_error(SGDRC_EINVAL, "unknown dtype %u", dtype);
    const uint32_t size = dtype == SGDRC_F32 ? 4u : 2u;
    if (vocab < 1 || vocab > 0x7FFFFFFFu)
        return set_error(SGDRC_EINVAL, "vocab %u outside 1..2^31 - 1", vocab);
    if (n_requests < 1 || n_requests > SGDRC_MAX_REQUESTS)
        return set_error(SGDRC_EINVAL, "n_requests %u outside 1..%d", n_requests, SGDRC_MAX_REQUESTS);
    if (max_nodes < 1 || max_nodes > SGDRC_MAX_NODES || path_stride < 1 || path_stride > SGDRC_MAX_NODES)
        return set_error(SGDRC_EINVAL, "max_nodes %u or path_stride %u outside 1..%d", max_nodes, path_stride,
                         SGDRC_MAX_NODES);
    if (target_stride < vocab || target_stride > (1ull << 40) ||
        (d_draft && (draft_stride < vocab || draft_stride > (1ull << 40))))
        return set_error(SGDRC_EINVAL, "rows lie %llu and %llu elements apart", (unsigned long long)target_stride,
                         (unsigned long long)draft_stride);
    int rc = check_aligned(d_q_start, 4, "q_start");
    if (rc || (rc = check_aligned(d_path, 4, "path")) || (rc = check_aligned(d_accepted, 4, "accepted")) ||
        (rc = check_aligned(d_next, 4, "next")))
        return rc;
    if (n_tokens && ((rc = check_aligned(d_target, size, "target")) || (rc = check_aligned(d_tokens, 4, "tokens")) ||
                     (rc = check_aligned(d_parents, 4, "parents")) || (rc = check_aligned(d_uniform, 4, "uniform"))))
        return rc;
    if (d_draft && (rc = check_aligned(d_draft, size, "draft")))
        return rc;
    if ((d_lens != nullptr) != (d_totals != nullptr))
        return set_error(SGDRC_EINVAL, "lens and totals: both or none");
    if (d_lens && ((rc = check_aligned(d_lens, 4, "lens")) || (rc = check_aligned(d_totals, 4, "totals"))))
        return rc;
    const uint32_t chunk = (uint32_t)(((uint64_t)vocab + (uint64_t)kSpan * kMaxChunks - 1u) / ((uint64_t)kSpan * kMaxChunks)) * kSpan;
    const VerifyArgs a = {static_cast<const uint8_t *>(d_target), static_cast<const uint8_t *>(d_draft),
                          target_stride * size, draft_stride * size, d_tokens, d_parents, d_uniform, d_q_start, d_lens,
                          d_totals, d_path, d_accepted, d_next, vocab, n_tokens, max_nodes, path_stride, chunk};
    switch (dtype) {
    case SGDRC_F32: return launch_verify<SGDRC_F32>(ctx, a, n_requests, stream);
    case SGDRC_BF16: return launch_verify<SGDRC_BF16>(ctx, a, n_requests, stream);
    default: return launch_verify<SGDRC_F16>(ctx, a, n_requests, stream);
    }
}
