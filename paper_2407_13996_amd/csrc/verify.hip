// Verification of drafted trees: which nodes a sampler of the target's
// probabilities would have taken, and its next token.
#include <algorithm>

#include "kv_common.hpp"

namespace sgdrc {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int kVerifyThreads = 512;
constexpr uint32_t kVerifyWaves = kVerifyThreads / 64;
constexpr uint32_t kMaxChunks = 512;   // of a row: the sums that are kept
constexpr uint32_t kDrawSpan = 1024;   // elements that the draw looks through at once, 16 a lane

struct VerifyArgs {
    const uint8_t *target, *draft;
    uint64_t target_stride, draft_stride;  // bytes
    const int32_t *tokens, *parents;
    const float *uniform;
    const uint32_t *q_start;
    const int32_t *lens, *totals;
    int32_t *path, *accepted, *next;
    uint32_t vocab, n_tokens, max_nodes, path_stride, chunk;  // chunk: elements, a multiple of kSpan
    uint32_t parts;     // workgroups of a request
    uint64_t *sums;     // with parts: of each request's chunks, as bits
    uint32_t *arrived;  // and how many of its workgroups have theirs
};

// A probability as it counts: 0 if not positive, no infinities.
__device__ __forceinline__ float counts(float p) { return fminf(fmaxf(p, 0.0f), 3.402823466e38f); }

// Elements of 16 bytes.
template <int DT>
constexpr uint32_t kVec = DT == SGDRC_F32 ? 4u : 8u;

// Elements that a wavefront sums at once.
constexpr uint32_t kSpan = 1024u;

template <int DT>
constexpr uint32_t kSize = DT == SGDRC_F32 ? 4u : 2u;

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

// Elements i .. i + N - 1 of a row; near its end the last N that it has, of which
// the first row_skip do not count.
template <int DT, uint32_t N>
__device__ __forceinline__ u32x4 row_load(const uint8_t *row, uint32_t i, uint32_t vocab)
{
    const uint32_t at = min(i, vocab - N);
    if (N == 1)
        return u32x4{__float_as_uint(row_at<DT>(row, at)), 0u, 0u, 0u};
    return reinterpret_cast<const Bytes16 *>(row + (uint64_t)at * kSize<DT>)->v;
}

template <uint32_t N>
__device__ __forceinline__ uint32_t row_skip(uint32_t i, uint32_t vocab)
{
    return i - min(i, vocab - N);
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// The largest bit patterns seen, of whole words (fp32) or of both halves: up to
// row_plain's they are numbers that count as they are, without the clamps.
template <int DT>
__device__ __forceinline__ uint32_t row_top(uint32_t top, u32x4 v)
{
    const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (DT == SGDRC_F32)
            top = max(top, x[e]);
        else
            top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top),
                                                                         __builtin_bit_cast(u16x2, x[e])));
    }
    return top;
}

template <int DT>
__device__ __forceinline__ bool row_plain(uint32_t top)
{
    if (DT == SGDRC_F32)
        return top <= 0x7F7FFFFFu;
    const uint32_t most = DT == SGDRC_BF16 ? 0x7F7Fu : 0x7BFFu;
    return (top & 0xFFFFu) <= most && top >> 16 <= most;
}

// The probabilities in them, as they count (``plain``: as they are).
template <int DT, uint32_t N>
__device__ __forceinline__ void row_floats(u32x4 v, float (&f)[N], bool plain = false)
{
    const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) {
        if (DT == SGDRC_F32 || N == 1) {
            f[e] = __uint_as_float(x[e % 4u]);
        } else if (DT == SGDRC_BF16) {
            f[e] = __uint_as_float(e % 2u ? x[e / 2u] & 0xFFFF0000u : x[e / 2u] << 16);
        } else {
            const f16x2 h = __builtin_bit_cast(f16x2, x[e / 2u]);
            f[e] = e % 2u ? (float)h.y : (float)h.x;
        }
        if (!plain)
            f[e] = counts(f[e]);
    }
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
// LDS.  Only a rejection and the last draw need a row as a whole; they
// sum it in chunks, whose sums are kept: without draft rows a further rejection
// changes one of them, and the draw looks up the chunk that the random number falls
// in and goes through that one again.  Few requests have several workgroups each: all walk
// as far as the first sum, share its chunks, and the last to have its part
// goes on alone (a chain needs no other sum).  N: elements of a load (1 for a vocabulary
// below a vector's); DRAWN: with draft rows.
// Bound by the chain of its trips to memory (a chain of 5 over 32000: 10.5 us with the launch; 32 trees of up to
// 48 certain choices over 50257: 19.6, a row's sum by one workgroup at each node that rejects),
// with many long rows by the pass over them and its 64-bit arithmetic (64 chains of 8 over 131072, 67 MB: 20).
// Spans of 2048 16-bit elements take 22.7 for the trees, two spans ahead 20.2, 1024 threads 27.
template <int DT, uint32_t N, bool DRAWN>
__global__ __launch_bounds__(kVerifyThreads) __attribute__((amdgpu_waves_per_eu(2))) void k_draft_verify(
    VerifyArgs a, uint32_t n_tiles, Gate g)
{
    constexpr uint32_t kLoads = N == 1u ? 1u : kSpan / 64u / N;
    __shared__ int32_t s_tok[SGDRC_MAX_NODES], s_par[SGDRC_MAX_NODES], s_path[SGDRC_MAX_NODES];
    __shared__ float s_u[SGDRC_MAX_NODES], s_p[SGDRC_MAX_NODES], s_q[SGDRC_MAX_NODES];
    __shared__ uint32_t s_ex[SGDRC_MAX_NODES];  // tokens ruled out at the node (without draft rows)
    __shared__ double s_chunk[kMaxChunks];
    __shared__ uint32_t s_last;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t n_chunks = (a.vocab + a.chunk - 1u) / a.chunk;

    auto body = [&](uint32_t tile, uint32_t &err) {
        const uint32_t r = tile / a.parts, part = tile % a.parts;
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
            s_q[i] = !DRAWN ? 1.0f : in && i ? counts(row_at<DT>(a.draft + row * a.draft_stride, tok)) : 0.0f;
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
        bool alone = a.parts == 1u, mine = n ? true : part == 0u;  // no part to share; ours is the request's end
        auto rows = [&](const uint8_t *&p, const uint8_t *&q) {
            p = a.target + (uint64_t)(q0 + cur) * a.target_stride;
            q = DRAWN ? a.draft + (uint64_t)(q0 + cur) * a.draft_stride : p;
        };
        auto gone = [&](uint32_t t) {
            bool x = false;
            for (uint32_t i = 0; i < n_ex; ++i)
                x = x || s_ex[i] == t;
            return x;
        };
        // weights of the elements from i on, of what is left; ``odd``: some do not count
        auto weights = [&](u32x4 vp, u32x4 vq, uint32_t i, bool ex, bool odd, double (&w)[N]) __attribute__((always_inline)) {
            float fp[N], fq[N];
            row_floats<DT, N>(vp, fp);
            row_floats<DT, N>(vq, fq);
            if (odd) {
                const uint32_t skip = row_skip<N>(i, a.vocab);
#pragma unroll
                for (uint32_t e = 0; e < N; ++e)
                    fp[e] = e >= skip ? fp[e] : 0.0f;
            }
#pragma unroll
            for (uint32_t e = 0; e < N; ++e)
                w[e] = DRAWN ? fmax((double)fp[e] - c * (double)fq[e], 0.0) : (double)fp[e];
            if (ex) {
                const uint32_t at = i - row_skip<N>(i, a.vocab);
                for (uint32_t k = 0; k < n_ex; ++k) {
                    const uint32_t t = s_ex[k];
#pragma unroll
                    for (uint32_t e = 0; e < N; ++e)
                        w[e] = at + e == t ? 0.0 : w[e];
                }
            }
        };
        // whether a ruled-out token lies in the chunk
        auto touched = [&](uint32_t ch) {
            bool x = false;
            for (uint32_t i = 0; i < n_ex; ++i)
                x = x || s_ex[i] / a.chunk == ch;
            return __builtin_amdgcn_readfirstlane(x ? 1u : 0u) != 0u;
        };
        // The sums of chunks ``from``, from + by, ... below ``end``: a span's loads go out
        // together, before the one that came before them is summed.
        const uint32_t per = a.chunk / kSpan;  // spans of a chunk
        auto sum_chunks = [&](uint32_t from, uint32_t end, uint32_t by) __attribute__((always_inline)) {
            const uint8_t *p, *q;
            rows(p, q);
            u32x4 vp[2][kLoads], vq[2][kLoads];
            auto fetch = [&](uint32_t i0, int b) __attribute__((always_inline)) {
#pragma unroll
                for (uint32_t k = 0; k < kLoads; ++k) {
                    const uint32_t i = i0 + (k * 64u + lane) * N;
                    vp[b][k] = row_load<DT, N>(p, i, a.vocab);
                    vq[b][k] = u32x4{0u, 0u, 0u, 0u};
                    if (DRAWN)
                        vq[b][k] = row_load<DT, N>(q, i, a.vocab);
                }
            };
            if (from >= end)
                return;
            uint32_t ch = from, j = 0u;  // the span that is summed
            fetch(ch * a.chunk, 0);
            double sum = 0.0;
            bool ex = touched(ch);
            for (bool more = true; more;) {
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    if (!more)
                        break;
                    const uint32_t at = ch * a.chunk + j * kSpan;
                    const bool odd = at + kSpan > a.vocab;
                    const bool last = j + 1u == per;
                    const uint32_t ch2 = last ? ch + by : ch, j2 = last ? 0u : j + 1u;
                    more = ch2 < end;
                    // (always: the loads before would be waited for where one may be missing)
                    fetch(more ? ch2 * a.chunk + j2 * kSpan : at, b ^ 1);
                    uint32_t top = 0u;
#pragma unroll
                    for (uint32_t k = 0; k < kLoads; ++k) {
                        top = row_top<DT>(top, vp[b][k]);
                        if (DRAWN)
                            top = row_top<DT>(top, vq[b][k]);
                    }
                    if (N > 1 && !ex && !odd && __ballot(!row_plain<DT>(top)) == 0ull) {
#pragma unroll
                        for (uint32_t k = 0; k < kLoads; ++k) {
                            float fp[N], fq[N];
                            row_floats<DT, N>(vp[b][k], fp, true);
                            row_floats<DT, N>(vq[b][k], fq, true);
#pragma unroll
                            for (uint32_t e = 0; e < N; ++e)
                                sum += DRAWN ? fmax((double)fp[e] - c * (double)fq[e], 0.0) : (double)fp[e];
                        }
                    } else {
#pragma unroll
                        for (uint32_t k = 0; k < kLoads; ++k) {
                            double w[N];
                            weights(vp[b][k], vq[b][k], at + (k * 64u + lane) * N, ex, odd, w);
#pragma unroll
                            for (uint32_t e = 0; e < N; ++e)
                                sum += w[e];
                        }
                    }
                    if (last) {
                        sum = wave_sum(sum);
                        if (lane == 0u)
                            s_chunk[ch] = sum;
                        sum = 0.0;
                        ex = more && touched(ch2);
                    }
                    ch = ch2;
                    j = j2;
                }
            }
        };
        // (``one``: only that chunk has changed)
        auto sum_row = [&](uint32_t one) __attribute__((always_inline)) {
            __syncthreads();  // the last sums are read
            uint32_t from = wave, end = n_chunks;
            if (one < n_chunks) {
                from = one % kVerifyWaves == wave ? one : n_chunks;
                end = one + 1u;
            } else if (!alone) {
                from = (uint32_t)((uint64_t)n_chunks * part / a.parts) + wave;
                end = (uint32_t)((uint64_t)n_chunks * (part + 1u) / a.parts);
            }
            sum_chunks(from, end, kVerifyWaves);
            __syncthreads();
            if (!alone) {
                // Sums and count are device-scope atomics (the workgroups may sit on
                // different XCDs); each wavefront waits for its sums before it counts.
                uint64_t *const sums = a.sums + (uint64_t)r * n_chunks;
                for (uint32_t ch = from - wave + threadIdx.x; ch < end; ch += kVerifyThreads)
                    __hip_atomic_store(&sums[ch], (uint64_t)__double_as_longlong(s_chunk[ch]), __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
                __builtin_amdgcn_s_waitcnt(0);
                __syncthreads();
                if (threadIdx.x == 0u) {
                    s_last = __hip_atomic_fetch_add(&a.arrived[r], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                             a.parts - 1u;
                    if (s_last)  // zero at rest
                        __hip_atomic_store(&a.arrived[r], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
                __syncthreads();
                mine = __builtin_amdgcn_readfirstlane(s_last) != 0u;
                if (mine)
                    for (uint32_t ch = threadIdx.x; ch < n_chunks; ch += kVerifyThreads)
                        s_chunk[ch] = __longlong_as_double((int64_t)__hip_atomic_load(&sums[ch], __ATOMIC_RELAXED,
                                                                                     __HIP_MEMORY_SCOPE_AGENT));
                alone = true;
                __syncthreads();
            }
            double total = 0.0;
            for (uint32_t ch = lane; ch < n_chunks; ch += 64u)
                total += s_chunk[ch];
            summed = true;
            left = wave_sum(total);
        };

        if (threadIdx.x == 0u)
            s_path[0] = 0;
        // The walk; at its end what the next token is drawn from is summed, and where nothing is
        // left the row itself.
        bool ending = false, whole = false;
        while (n) {
            uint32_t child = n, one = n_chunks;
            if (!ending) {
#pragma unroll
                for (int k = SGDRC_MAX_NODES / 64 - 1; k >= 0; --k) {
                    const uint64_t m = __ballot(par[k] == (int32_t)cur && k * 64u + lane > last);
                    child = m ? k * 64u + (uint32_t)__builtin_ctzll(m) : child;
                }
                child = __builtin_amdgcn_readfirstlane(child);
            }
            const bool some = __builtin_amdgcn_readfirstlane(left > 0.0 ? 1u : 0u) != 0u;
            // (where nothing is left no child can be accepted)
            if (child >= n || !some || depth >= a.path_stride) {
                ending = true;
                if (summed && (some || whole))
                    break;
                if (summed) {
                    whole = true;
                    c = 0.0;
                    n_ex = 0u;
                }
            } else {
                last = child;
                const uint32_t t = __builtin_amdgcn_readfirstlane((uint32_t)s_tok[child]);
                if ((int32_t)t < 0) {
                    err |= kDevErrSeq;
                    continue;
                }
                const double q = s_q[child];
                double w = fmax((double)s_p[child] - (DRAWN ? c * q : 0.0), 0.0);
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
                if (DRAWN) {
                    c += left;
                } else {
                    __syncthreads();
                    if (threadIdx.x == 0u)
                        s_ex[n_ex] = t;
                    n_ex += 1u;
                    one = summed ? t / a.chunk : n_chunks;
                }
            }
            sum_row(one);
            if (!mine)
                break;
        }
        int32_t next = -1;
        if (n && mine && wave == 0u) {
            const uint8_t *p, *q;
            rows(p, q);
            const double goal = (double)s_u[0] * left;
            // The chunk that the goal falls in, of which a lane holds 8.  (Where rounding
            // leaves the goal above all sums: the last that holds anything.)
            constexpr uint32_t kHeld = kMaxChunks / 64u;
            double held = 0.0;
            for (uint32_t k = 0; k < kHeld; ++k)
                held += lane * kHeld + k < n_chunks ? s_chunk[lane * kHeld + k] : 0.0;
            const double upto = wave_scan(held, lane);
            const uint64_t past = __ballot(held > 0.0 && upto > goal), some = __ballot(held > 0.0);
            if (some) {
                const uint32_t l = past ? (uint32_t)__builtin_ctzll(past) : 63u - (uint32_t)__builtin_clzll(some);
                double before = __shfl(upto - held, l, 64), run = before;
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
                for (uint32_t i0 = ch * a.chunk; i0 < end; i0 += kDrawSpan) {
                    double w[16];
#pragma unroll
                    for (uint32_t k = 0; k < 16u / N; ++k) {
                        double x[N];
                        const uint32_t i = i0 + lane * 16u + k * N;
                        const u32x4 vp = row_load<DT, N>(p, i, a.vocab);
                        weights(vp, DRAWN ? row_load<DT, N>(q, i, a.vocab) : vp, i, ex, true, x);
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
                                const uint32_t i = i0 + lane * 16u + e / N * N;
                                pick = i - row_skip<N>(i, a.vocab) + e % N;
                                at += w[e];
                                got = at > goal;
                            }
                        next = (int32_t)__shfl(pick, le, 64);
                    }
                    if (over)
                        break;
                    before += __shfl(to, 63, 64);
                }
            }
            err |= next < 0 ? kDevErrSeq : 0u;
        }
        __syncthreads();  // the path
        if (mine && threadIdx.x < a.path_stride)
            a.path[(uint64_t)r * a.path_stride + threadIdx.x] = threadIdx.x < depth ? s_path[threadIdx.x] : -1;
        if (mine && threadIdx.x == 0u) {
            a.accepted[r] = (int32_t)depth;
            a.next[r] = next;
        }
    };
    single_tile_loop(g, n_tiles, NoOp(), body);
}

template <int DT, uint32_t N, bool DRAWN>
static int launch_verify(sgdrc_ctx *ctx, VerifyArgs a, uint32_t n_requests, void *stream)
{
    static const int occ = occupancy(k_draft_verify<DT, N, DRAWN>, kVerifyThreads);
    const uint64_t pieces = ((uint64_t)a.vocab + kSpan - 1u) / kSpan;
    const uint64_t in_chunk = (pieces + kMaxChunks - 1u) / kMaxChunks;
    a.chunk = (uint32_t)in_chunk * kSpan;
    const uint32_t chunks = (uint32_t)((pieces + in_chunk - 1u) / in_chunk);
    Ctx *c = nullptr;
    int rc = check_ctx(ctx, &c);
    if (rc)
        return rc;
    // Workgroups of a request: one a CU over all requests, each wavefront with a
    // chunk, sums that fit the stream's place for them.  (Chains of 8 nodes over 131072
    // float values, 64 of them: 20.4 us, two workgroups a CU 20.7, without parts 32.3.  One
    // chain: 11.3 either way, without parts 22.4.)
    a.parts = 1u;
    if (n_requests <= kVerifyShared && (uint64_t)n_requests * chunks <= kVerifySums)
        a.parts = std::max(1u, std::min({16u, (uint32_t)stream_allowed_cus(c, stream) / n_requests,
                                         chunks / kVerifyWaves}));
    const uint64_t tiles = (uint64_t)n_requests * a.parts;
    Gate g;
    LaunchInfo li;
    if ((rc = make_gate(c, stream, tiles, kStreamGroupCus, &g, &li, false, true)))
        return rc;
    uint64_t *const place = c->d_verify + (size_t)(g.q - c->d_queues) * (kVerifySums + kVerifyShared);
    a.sums = place;
    a.arrived = reinterpret_cast<uint32_t *>(place + kVerifySums);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    hipLaunchKernelGGL((k_draft_verify<DT, N, DRAWN>), dim3(gated_grid(c, occ, tiles, li)), dim3(kVerifyThreads), 0, s, a,
                       (uint32_t)tiles, g);
    SGDRC_HIP(hipGetLastError());
    return finish_static_tlog(g, s);
}

template <int DT>
static int launch_verify_size(sgdrc_ctx *ctx, const VerifyArgs &a, uint32_t n_requests, void *stream)
{
    if (a.vocab < kVec<DT>)
        return a.draft ? launch_verify<DT, 1, true>(ctx, a, n_requests, stream)
                       : launch_verify<DT, 1, false>(ctx, a, n_requests, stream);
    return a.draft ? launch_verify<DT, kVec<DT>, true>(ctx, a, n_requests, stream)
                   : launch_verify<DT, kVec<DT>, false>(ctx, a, n_requests, stream);
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
    const VerifyArgs a = {static_cast<const uint8_t *>(d_target), static_cast<const uint8_t *>(d_draft),
                          target_stride * size, draft_stride * size, d_tokens, d_parents, d_uniform, d_q_start, d_lens,
                          d_totals, d_path, d_accepted, d_next, vocab, n_tokens, max_nodes, path_stride, 0u, 1u,
                          nullptr, nullptr};
    switch (dtype) {
    case SGDRC_F32: return launch_verify_size<SGDRC_F32>(ctx, a, n_requests, stream);
    case SGDRC_BF16: return launch_verify_size<SGDRC_BF16>(ctx, a, n_requests, stream);
    default: return launch_verify_size<SGDRC_F16>(ctx, a, n_requests, stream);
    }
}
