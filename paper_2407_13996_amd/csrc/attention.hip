// Attention of drafted tokens over the paged key/value cache.
//
// For one key/value head, the query rows of a request are its nodes' G =
// n_heads / kv_heads query heads.  With S^T = K Q^T and O^T = V^T P^T a
// query row is a column of both matrix products, that is, a lane (mod 16) of
// every accumulator, so the softmax's running maximum and sum are one register
// a row, and
// rescaling, masking by node and the final division need no exchange between
// lanes.  The products' operands come straight from the cache: 16 bytes of K
// (8 dims of a token) or of V (8 tokens of a dim) are one lane's share of a
// 16x16x32 MFMA operand.  S^T's accumulators hold four tokens of a row a lane;
// two K tiles, whose rows are tokens 8 (r / 4) + r % 4 and those + 4, leave lane
// group g with tokens 8g .. 8g + 7 of a 32-token step, in order: the P^T
// operand.  No shuffle and no LDS between the two products.
//
// Split: every request's tokens are cut in steps of 32, and the steps of all
// (request, block of rows, head) triples, "segments", form one line, which is
// cut in at most 512 equal ranges, one tile of the schedule each, whatever the
// lengths: long and short requests fill the device alike.  A range's piece of a
// segment that is not all of it leaves its maximum, sum and weighted V in
// the workspace; a second launch joins them.  The cut depends on the lengths
// only, so results do not depend on the CU mask.
#include <algorithm>
#include <cmath>
#include <limits>
#include <mutex>
#include <type_traits>

#include "kv_common.hpp"

namespace sgdrc {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kAttThreads = 256;
constexpr int kAttWaves = kAttThreads / 64;
constexpr uint32_t kStep = 32;            // tokens of a step
constexpr uint32_t kMinSteps = 4;         // steps of a range at least
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct AttArgs {
    KvView c;
    RowsView q;
    uint8_t *o;
    uint64_t o_token, o_head;   // bytes
    float *lse;
    const uint64_t *mask;
    float *work;
    uint32_t n_requests, stride, width, n_tokens, max_nodes, mask_words;
    uint32_t heads, group;      // query heads, query heads of a key/value head
    uint32_t most_ranges;       // pieces that the line of steps is cut in at most
    float scale, softcap;
    float cap_y, cap_lin, cap_out;  // scale / softcap, and scale and softcap in units of log 2
};

// What the kernels read of the requests.  Kernel arguments of their own,
// so that the compiler knows that nothing writes them and reads what is the
// same for a whole wavefront by scalar loads: these have a counter of their
// own, and waiting for a page-table entry does not wait for the K and V in
// flight.
struct Seqs {
    const uint32_t *q_start, *table;
    const int32_t *lens, *totals;
};

#define SGDRC_SEQS_ARGS \
    const uint32_t *__restrict__ q_start, const uint32_t *__restrict__ table, const int32_t *__restrict__ lens, \
        const int32_t *__restrict__ totals

// A request as the kernels see it: device values brought into range.
struct Req {
    uint32_t start, nodes, total, ctx;
    bool ok;
};

__device__ __forceinline__ Req load_req(const AttArgs &a, const Seqs &sq, uint32_t r)
{
    Req q;
    const uint32_t s = sq.q_start[r], e = sq.q_start[r + 1u];
    const int32_t total = sq.totals[r], ctx = sq.lens[r];
    const uint32_t cap = a.width << a.c.bshift;
    q.start = min(s, a.n_tokens);
    const uint32_t end = max(min(e, a.n_tokens), q.start);
    q.nodes = min(end - q.start, a.max_nodes);
    q.total = total < 0 ? 0u : min((uint32_t)total, cap);
    q.ctx = ctx < 0 ? 0u : min((uint32_t)ctx, q.total);
    // lengths of a request without nodes are not used: one that ends in this step
    // has its old length before it and none after
    const bool lengths = total >= 0 && (uint32_t)total <= cap && ctx >= 0 && ctx <= total;
    q.ok = s <= e && e <= a.n_tokens && e - s <= a.max_nodes && (s == e || lengths);
    return q;
}

// Steps of one segment of a request; a request whose cache is empty has one,
// without tokens, which writes its rows.
__device__ __forceinline__ uint32_t seg_steps(const Req &q)
{
    return max((q.total + kStep - 1u) / kStep, 1u);
}

__device__ __forceinline__ uint32_t row_blocks(const Req &q, uint32_t group, uint32_t rb)
{
    return (q.nodes * group + rb - 1u) / rb;
}

// All workgroups: s_line[r] = first step of request r in the line of steps,
// s_line[n_requests] their number.
template <uint32_t THREADS>
__device__ __forceinline__ void plan_line(const AttArgs &a, const Seqs &sq, uint32_t rb, uint32_t *s_line, uint32_t *s_sum,
                                          uint32_t &err)
{
    const uint32_t R = a.n_requests;
    const uint32_t per = (R + THREADS - 1u) / THREADS;
    const uint32_t r0 = min(threadIdx.x * per, R), r1 = min(r0 + per, R);
    uint32_t sum = 0u;
    for (uint32_t r = r0; r < r1; ++r) {
        const Req q = load_req(a, sq, r);
        err |= q.ok ? 0u : kDevErrSeq;
        sum += q.nodes ? seg_steps(q) * row_blocks(q, a.group, rb) * a.c.heads : 0u;
    }
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    uint32_t v = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t o = __shfl_up(v, off, 64);
        v += lane >= (uint32_t)off ? o : 0u;
    }
    if (lane == 63u)
        s_sum[wave] = v;
    __syncthreads();
    uint32_t run = v - sum;
    for (uint32_t w = 0; w < wave; ++w)
        run += s_sum[w];
    for (uint32_t r = r0; r < r1; ++r) {
        s_line[r] = run;
        if (per == 1u) {
            run += sum;
        } else {
            const Req q = load_req(a, sq, r);
            run += q.nodes ? seg_steps(q) * row_blocks(q, a.group, rb) * a.c.heads : 0u;
        }
        if (r == R - 1u)
            s_line[R] = run;
    }
    __syncthreads();
}

// The cut of a line of steps into ranges of almost equal length: range t is
// [cut(t), cut(t + 1)), cut(t) = t steps / ranges, by 32-bit divisions.
struct Cuts {
    uint32_t steps, n, whole, rest;

    __device__ __forceinline__ Cuts(const AttArgs &a, uint32_t line)
    {
        steps = __builtin_amdgcn_readfirstlane(line);
        n = min(a.most_ranges, (steps + kMinSteps - 1u) / kMinSteps);
        whole = steps / max(n, 1u);
        rest = steps - whole * n;
    }

    __device__ __forceinline__ uint32_t cut(uint32_t t) const { return t * whole + t * rest / max(n, 1u); }

    // the range that step ``p`` is in (ranges are at most 512, so that the
    // estimate is at most one off)
    __device__ __forceinline__ uint32_t range_of(uint32_t p) const
    {
        uint32_t t = min((uint32_t)((float)p * ((float)n / (float)steps)), n - 1u);
        if (t && cut(t) > p)
            --t;
        else if (t + 1u < n && cut(t + 1u) <= p)
            ++t;
        return t;
    }
};

// The last request that begins at or before step ``p`` and has any.
__device__ __forceinline__ uint32_t find_request(const uint32_t *s_line, uint32_t R, uint32_t p)
{
    uint32_t lo = 0u, hi = R;
    while (hi - lo > 1u) {
        const uint32_t mid = (lo + hi) >> 1;
        if (s_line[mid] <= p)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// A partial result in the workspace: per row {maximum, sum}, then the rows'
// weighted V.  Range t has two: 2t for a piece that began in an earlier range,
// 2t + 1 for one that goes on in the next.
__device__ __forceinline__ float *part_stats(float *work, uint32_t part, uint32_t rb, uint32_t dim)
{
    return work + (uint64_t)part * rb * (dim + 2u);
}

__device__ __forceinline__ float *part_rows(float *work, uint32_t part, uint32_t rb, uint32_t dim)
{
    return part_stats(work, part, rb, dim) + rb * 2u;
}

template <int DT>
__device__ __forceinline__ f32x4 att_mfma(u32x4 a, u32x4 b, f32x4 c)
{
    if (DT == SGDRC_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
}

// Two fp32 values rounded to nearest even, side by side.
template <int DT>
__device__ __forceinline__ uint32_t pack2(float x, float y)
{
    const f32x2 v = {x, y};
    if (DT == SGDRC_BF16)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
    else
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}

// Two 16-bit elements at a time, without comparisons (their results would
// take scalar registers, of which a step in this state has none left).
// All of a half's bits where its top bit is set in ``x``.
__device__ __forceinline__ uint32_t spread_top(uint32_t x)
{
    return ((x >> 15) & 0x00010001u) * 0xFFFFu;
}

// Halves that hold more than ``least`` - 1 without their sign, by their top bits.
template <uint32_t LEAST>
__device__ __forceinline__ uint32_t top_from(uint32_t x)
{
    return ((x & 0x7FFF7FFFu) + (0x8000u - LEAST) * 0x00010001u) & 0x80008000u;
}

template <int DT>
constexpr uint32_t kInf = DT == SGDRC_BF16 ? 0x7F80u : 0x7C00u;

// The halves' masks of tokens 2 w and 2 w + 1 in ``bits``.
__device__ __forceinline__ uint32_t pair_mask(uint32_t bits, int w)
{
    return spread_top((((bits >> (2 * w)) & 1u) << 15) | (((bits >> (2 * w + 1)) & 1u) << 31));
}

// Marks of infinities and NaN: 1 for +infinity, 64 for -infinity, 4096 for NaN
// (a step has 32 tokens, so a sum of marks tells how many of each).
template <int DT>
constexpr uint32_t kOne = (DT == SGDRC_BF16 ? 0x3F80u : 0x3C00u) * 0x00010001u;

// The marks of two elements of V, which become 0 where they have one.
template <int DT>
__device__ __forceinline__ uint32_t take_marks(uint32_t &x)
{
    constexpr uint32_t m64 = (DT == SGDRC_BF16 ? 0x4280u : 0x5400u) * 0x00010001u;
    constexpr uint32_t m4096 = (DT == SGDRC_BF16 ? 0x4580u : 0x6C00u) * 0x00010001u;
    const uint32_t off = spread_top(top_from<kInf<DT>>(x)), nan = spread_top(top_from<kInf<DT> + 1u>(x));
    const uint32_t neg = spread_top(x);
    x &= ~off;
    return off & ((nan & m4096) | (~nan & ((neg & m64) | (~neg & kOne<DT>))));
}

// What a sum with these marks is: ``n`` of values with weights, ``n0`` of
// values whose weight is 0 (0 times infinity).
__device__ __forceinline__ float marked(float n, float n0)
{
    const uint32_t k = (uint32_t)n;
    float v = k & 63u ? INFINITY : 0.0f;
    v += (k >> 6) & 63u ? -INFINITY : 0.0f;
    return k >> 12 || n0 != 0.0f ? NAN : v;
}

// Each lane's value and that of the lane 16 (32) away, in an order that both
// see alike.
struct Two {
    float a, b;
};

// (the elements go through scalars: a bit cast of a vector's element takes the
// first of them whichever is named)
__device__ __forceinline__ Two swap16(float v)
{
    const uint32_t x = __builtin_bit_cast(uint32_t, v);
    const u32x2 t = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const uint32_t t0 = t[0], t1 = t[1];
    return {__builtin_bit_cast(float, t0), __builtin_bit_cast(float, t1)};
}

__device__ __forceinline__ Two swap32(float v)
{
    const uint32_t x = __builtin_bit_cast(uint32_t, v);
    const u32x2 t = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    const uint32_t t0 = t[0], t1 = t[1];
    return {__builtin_bit_cast(float, t0), __builtin_bit_cast(float, t1)};
}

// A row's four lanes are 16 apart: the values of the others arrive by swaps of
// half and quarter wavefronts, on the vector ALUs.
__device__ __forceinline__ float row_max(float v)
{
    const Two p = swap16(v);
    const Two q = swap32(fmaxf(p.a, p.b));
    return fmaxf(q.a, q.b);
}

__device__ __forceinline__ float row_sum(float v)
{
    const Two p = swap16(v);
    const Two q = swap32(p.a + p.b);
    return q.a + q.b;
}

// ``v``, as a value that the compiler cannot know before this point: what
// follows from it is worked out here, not kept in registers through the loops
// above.
__device__ __forceinline__ uint32_t fresh(uint32_t v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// n low bits, n of any size.
__device__ __forceinline__ uint32_t low8(int32_t n)
{
    return n >= 8 ? 0xFFu : n <= 0 ? 0u : (1u << n) - 1u;
}

// Which of the tokens ctx + j0 .. ctx + j0 + 7 node ``node`` sees, of ``drafted``.
__device__ __forceinline__ uint32_t seen8(const AttArgs &a, uint32_t token, uint32_t node, int32_t j0,
                                          int32_t drafted)
{
    uint32_t v;
    if (!a.mask) {
        v = low8((int32_t)node + 1 - j0);
    } else {
        const uint32_t lo = (uint32_t)max(j0, 0), w = lo >> 6, sh = lo & 63u;
        const uint64_t *const row = a.mask + (uint64_t)token * a.mask_words;
        uint64_t bits = w < a.mask_words ? row[w] >> sh : 0ull;
        if (sh > 56u && w + 1u < a.mask_words)
            bits |= row[w + 1u] << (64u - sh);
        v = (uint32_t)bits & 0xFFu;
        if (j0 < 0)
            v = j0 <= -8 ? 0xFFu : (v << -j0) | low8(-j0);
    }
    return v & low8(drafted - j0);
}

// A range's part of one segment.
struct Piece {
    uint32_t r, h;              // request, key/value head
    uint32_t start, rows, row0; // the request's first token, its rows; the segment's first row
    uint32_t total, ctx;
    uint32_t u0, u1;            // steps
    uint32_t part;              // its place in the workspace
    bool whole;                 // all of the segment
};

// The piece that begins at step ``p`` of the line, in range ``t`` = [lo, hi); all values uniform.
__device__ __forceinline__ Piece take_piece(const AttArgs &a, const Seqs &sq, const uint32_t *s_line, uint32_t rb, uint32_t t,
                                            uint32_t lo, uint32_t hi, uint32_t p)
{
    Piece x;
    x.r = __builtin_amdgcn_readfirstlane(find_request(s_line, a.n_requests, p));
    const Req rq = load_req(a, sq, x.r);
    const uint32_t U = __builtin_amdgcn_readfirstlane(seg_steps(rq));
    x.total = __builtin_amdgcn_readfirstlane(rq.total);
    x.ctx = __builtin_amdgcn_readfirstlane(rq.ctx);
    x.rows = __builtin_amdgcn_readfirstlane(rq.nodes * a.group);
    x.start = __builtin_amdgcn_readfirstlane(rq.start);
    const uint32_t blocks = (x.rows + rb - 1u) / rb;
    const uint32_t at = p - __builtin_amdgcn_readfirstlane(s_line[x.r]);
    const uint32_t seg = at / U;
    x.u0 = at % U;
    x.u1 = min(U, x.u0 + (hi - p));
    x.h = seg / blocks;
    x.row0 = seg % blocks * rb;
    x.whole = x.u0 == 0u && x.u1 == U;
    x.part = 2u * t + (p == lo && x.u0 != 0u ? 0u : 1u);
    return x;
}

// p[i], the same for the whole wavefront and not written by the kernel, by a
// scalar load.
__device__ __forceinline__ uint32_t load_uniform(const uint32_t *p, uint32_t i)
{
    typedef const uint32_t __attribute__((address_space(4))) *Const;
    return reinterpret_cast<Const>(reinterpret_cast<uintptr_t>(p))[__builtin_amdgcn_readfirstlane(i)];
}

// The pages of a step: those of its first and last 16 tokens (a block holds
// whole groups of 16).  Pages past the cache's end are not looked up: their
// entries may hold anything.
struct StepPages {
    uint32_t e[2];
};

__device__ __forceinline__ StepPages step_pages(const uint32_t *row_table, const Piece &x, uint32_t u, uint32_t bshift)
{
    const uint32_t last = x.total ? (x.total - 1u) >> bshift : 0u;
    StepPages s;
#pragma unroll
    for (uint32_t i = 0; i < 2u; ++i)
        s.e[i] = load_uniform(row_table, min((u * kStep + 16u * i) >> bshift, last));
    return s;
}

// The head's chunks on a step's pages.  ``bad``: bit i set where the pool
// does not have page i (then page 0, whose values are not used), both set
// for a cache without tokens.
struct StepAt {
    const uint8_t *p[2];
    uint32_t bad;
};

__device__ __forceinline__ StepAt step_at(const AttArgs &a, const uint8_t *head, const StepPages &s, uint32_t total,
                                          uint32_t &err)
{
    StepAt at;
    at.bad = 0u;
#pragma unroll
    for (uint32_t i = 0; i < 2u; ++i) {
        const bool bad = s.e[i] > (uint32_t)(a.c.pool_pages - 1u);
        at.bad |= bad || total == 0u ? 1u << i : 0u;
        err |= bad && total != 0u ? kDevErrPtRange : 0u;
        at.p[i] = head + ((uint64_t)(bad || total == 0u ? 0u : s.e[i]) << a.c.shift);
    }
    return at;
}

// A wavefront's rows: column ``col`` of block b is row row0 + 16 b + col of
// the request, node row / group, query head h group + row % group.
template <int DT, int D, int NB>
struct Rows {
    u32x4 q[NB][D / 32];
    f32x4 acc[NB][D / 16];      // O^T: dims 16 dd + 4 grp .. + 3 of column col
    float m[NB], l[NB];
    uint32_t tok[NB], node[NB];

    // block b's rows: 16 from row0 + apart * b on
    __device__ __forceinline__ uint32_t find(const AttArgs &a, const Piece &x, uint32_t row0, uint32_t apart, uint32_t col,
                                             int b)
    {
        const uint32_t row = min(row0 + apart * b + col, x.rows - 1u);
        node[b] = row / a.group;
        tok[b] = x.start + node[b];
        return row;
    }

    __device__ __forceinline__ void load_q(const AttArgs &a, const Piece &x, uint32_t row0, uint32_t apart, uint32_t col,
                                           uint32_t grp)
    {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const uint32_t row = find(a, x, row0, apart, col, b);
            const uint8_t *const qp = a.q.ptr + tok[b] * a.q.token + (x.h * a.group + row % a.group) * a.q.head;
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk)
                q[b][kk] = *reinterpret_cast<const u32x4 *>(qp + (kk * 4u + grp) * 16u);
        }
    }

    __device__ __forceinline__ void begin(const AttArgs &a, const Piece &x, uint32_t row0, uint32_t apart, uint32_t col,
                                          uint32_t grp)
    {
        load_q(a, x, row0, apart, col, grp);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            m[b] = -INFINITY;
            l[b] = 0.0f;
#pragma unroll
            for (int dd = 0; dd < D / 16; ++dd)
                acc[b][dd] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }
};

// Scores capped to cap tanh(y), y = s scale / cap, in units of log 2.  From |y|
// = 1/4 on by tanh y = 1 - 2 / (1 + e^2y), whose two terms cancel for small y:
// the error, some 2^-23 of the cap, would be that of the whole score where the cap
// is large.  Below, s scale times tanh(y) / y by its series in y^2, which the
// first term left out changes by 2^-27.  Both are off by 20 2^-24 of the
// result at most, whatever the cap.  (12 requests of up to 6000 tokens, 16 heads
// on 8 of 256: 165 us, 160 with the first form alone.)
// TIGHT: registers are short, and the cap's numbers are read again from the
// kernel's first argument in every step: kept over the loops, they had
// calls without a cap reload spilled scalars each step, 417 us for 400.
template <bool TIGHT, int NB, int ACT = NB>
__device__ __forceinline__ void cap_scores(const AttArgs &args, f32x4 (&s)[NB][2])
{
    typedef const __attribute__((address_space(4))) AttArgs *Args;
    float cap_y = args.cap_y, cap_lin = args.cap_lin, cap_out = args.cap_out;
    if (TIGHT) {
        Args a = (Args)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(a));
        cap_y = a->cap_y, cap_lin = a->cap_lin, cap_out = a->cap_out;
    }
#pragma unroll
    for (int b = 0; b < ACT; ++b)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float y = s[b][x][i] * cap_y, u = y * y;
                float g = __builtin_fmaf(u, 62.0f / 2835.0f, -17.0f / 315.0f);
                g = __builtin_fmaf(u, g, 2.0f / 15.0f);
                g = __builtin_fmaf(u, g, -1.0f / 3.0f);
                g = __builtin_fmaf(u, g, 1.0f);
                const float e = __builtin_amdgcn_exp2f(__builtin_fabsf(y) * (2.0f * kLog2e));
                const float far = cap_out * __builtin_fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + e), 1.0f);
                s[b][x][i] = u < 0.0625f ? s[b][x][i] * cap_lin * g : __builtin_copysignf(far, y);
            }
}

// f16's P is scaled by 2^10: weights down to 2^-34 of the largest stay normal
// or subnormal numbers there (bf16 has fp32's range).
template <int DT>
constexpr float kLift = DT == SGDRC_F16 ? 10.0f : 0.0f;

// Two weights in two numbers each: a smaller one of the type, and what is left,
// rounded.  Neither part of a weight is 0 (down to 2^-33 of the largest in f16),
// so that an infinite value meets no 0.
template <int DT>
__device__ __forceinline__ void split2(float x, float y, uint32_t &most, uint32_t &rest)
{
    if (DT == SGDRC_BF16) {
        // half a unit less, cut to 8 bits
        const uint32_t bx = __builtin_elementwise_sub_sat(__builtin_bit_cast(uint32_t, x), 0x8000u);
        const uint32_t by = __builtin_elementwise_sub_sat(__builtin_bit_cast(uint32_t, y), 0x8000u);
        most = (bx >> 16) | (by & 0xFFFF0000u);
        rest = pack2<DT>(x - __builtin_bit_cast(float, bx & 0xFFFF0000u), y - __builtin_bit_cast(float, by & 0xFFFF0000u));
    } else {
        constexpr float k = 1.0f - 0x1p-12f;
        const f16x2 h = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(x * k, y * k));
        most = __builtin_bit_cast(uint32_t, h);
        rest = pack2<DT>(x - (float)h[0], y - (float)h[1]);
    }
}

// Scores to weights: the running maximum, what was summed under the old one
// rescaled, the weights added up (fp32) and brought to the P^T operand's type.
// A row's sum stays spread over its four lanes until the end.  ACT: the blocks
// that have rows, the first ones.  PARTS: the numbers of the type that hold a
// weight, a product with V each.  With one, rounded to 8 bits in bf16 or 11 in
// f16, the rounded weights add as much to the result's error as its own
// rounding (24 nodes over 131001 tokens, bf16: 2.3e-3 of it off, 1.7e-3 of that by the
// latter).  With two (16 bits and 22) nothing is added: the form for few rows waits
// for memory and has the time (725 us either way for 96 requests of up to 24000
// tokens).  The form for many has not: 495 us for 405 (24 requests of 64 nodes, 64 heads
// on 8) and 151 for 130.
template <int DT, int D, int NB, int PARTS, int ACT = NB>
__device__ __forceinline__ void weigh(Rows<DT, D, NB> &w, const f32x4 (&s)[NB][2], float c2, u32x4 (&pf)[PARTS][NB])
{
#pragma unroll
    for (int b = 0; b < ACT; ++b) {
        float mx = fmaxf(s[b][0][0], s[b][0][1]);
#pragma unroll
        for (int i = 2; i < 8; ++i)
            mx = fmaxf(mx, s[b][i >> 2][i & 3]);
        mx = row_max(mx);
        if (__ballot(mx > w.m[b]) != 0ull) {
            const float mn = fmaxf(w.m[b], mx);
            const float f = __builtin_amdgcn_exp2f((w.m[b] - (mn == -INFINITY ? 0.0f : mn)) * c2);
            w.m[b] = mn;
            w.l[b] *= f;
#pragma unroll
            for (int dd = 0; dd < D / 16; ++dd)
                w.acc[b][dd] *= f;
        }
        const float sub = (w.m[b] == -INFINITY ? 0.0f : w.m[b] * c2) - kLift<DT>;
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i >> 2][i & 3], c2, -sub));
            w.l[b] += p[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (PARTS == 2) {
                uint32_t most, rest;
                split2<DT>(p[2 * i], p[2 * i + 1], most, rest);
                pf[0][b][i] = most;
                pf[1][b][i] = rest;
            } else {
                pf[0][b][i] = pack2<DT>(p[2 * i], p[2 * i + 1]);
            }
        }
    }
}

// A step that reaches into the drafted tokens or past the cache's end: which
// of the lane's eight tokens its rows see (``there``: those that exist).
template <int DT, int D, int NB>
__device__ __forceinline__ void mask_scores(const AttArgs &a, const Rows<DT, D, NB> &w, int32_t j0, int32_t drafted,
                                            uint32_t there, f32x4 (&s)[NB][2], uint32_t (&seen)[NB])
{
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        seen[b] = seen8(a, w.tok[b], w.node[b], j0, drafted) & there;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            s[b][i >> 2][i & 3] = (seen[b] >> i) & 1u ? s[b][i >> 2][i & 3] : -INFINITY;
    }
}

// O^T += V^T P^T where infinities or NaN among the drafted values must not
// meet the weight 0 of a row that does not see them.  They are taken out of V,
// and a product of marks counts those that each row sees: such a sum is
// infinite or NaN, whatever the rest is.  ``load_v(dd)``: V^T's operand.
template <int DT, int D, int NB, int PARTS, typename LoadV>
__device__ __forceinline__ void add_odd(Rows<DT, D, NB> &r, const u32x4 (&pf)[PARTS][NB], const uint32_t (&seen)[NB],
                                        LoadV load_v)
{
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        u32x4 some, none;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t sees = pair_mask(seen[b], w), weight = spread_top(top_from<1u>(pf[0][b][w]) | top_from<1u>(pf[PARTS - 1][b][w]));
            some[w] = sees & weight & kOne<DT>;
            none[w] = sees & ~weight & kOne<DT>;
        }
#pragma unroll
        for (int dd = 0; dd < D / 16; ++dd) {
            u32x4 v = load_v(dd), marks;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t two = v[w];
                marks[w] = take_marks<DT>(two);
                v[w] = two;
            }
            const f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < PARTS; ++k)
                r.acc[b][dd] = att_mfma<DT>(v, pf[k][b], r.acc[b][dd]);
            const f32x4 n = att_mfma<DT>(marks, some, z), n0 = att_mfma<DT>(marks, none, z);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                r.acc[b][dd][i] += marked(n[i], n0[i]);
            __builtin_amdgcn_sched_barrier(0);  // one block's marks at a time
        }
    }
}

// Zeroes what does not exist (``there``: bits of 8 tokens) in 16 bytes of V;
// not zero if a value that is left is infinite or NaN.
template <int DT>
__device__ __forceinline__ uint32_t keep_there(u32x4 &v, uint32_t there)
{
    uint32_t odd = 0u;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        v[w] &= pair_mask(there, w);
        odd |= top_from<kInf<DT>>(v[w]);
    }
    return odd;
}

// A row's result, or its part of one, 4 dims from d on.
template <int DT, int D>
__device__ __forceinline__ void put_row(const AttArgs &a, const Piece &x, uint32_t rb, uint32_t in, uint32_t d, f32x4 v)
{
    const uint32_t row = x.row0 + in;
    if (row >= x.rows)
        return;
    if (x.whole) {
        uint8_t *const op = a.o + (x.start + row / a.group) * a.o_token + (x.h * a.group + row % a.group) * a.o_head + d * 2u;
        const u32x2 two = {pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3])};
        *reinterpret_cast<u32x2 *>(op) = two;
    } else {
        *reinterpret_cast<f32x4 *>(part_rows(a.work, x.part, rb, D) + (uint64_t)in * D + d) = v;
    }
}

// A row's maximum and sum: to the workspace, or as its log-sum-exp.  Returns
// what its weighted V is to be multiplied with.
template <int DT, int D>
__device__ __forceinline__ float put_stats(const AttArgs &a, const Piece &x, uint32_t rb, uint32_t in, float m, float l,
                                           float c2, bool write)
{
    if (write && x.row0 + in < x.rows) {
        if (!x.whole) {
            float *const st = part_stats(a.work, x.part, rb, D) + in * 2u;
            st[0] = m;
            st[1] = l;
        } else if (a.lse) {
            const uint32_t row = x.row0 + in;
            a.lse[(uint64_t)(x.start + row / a.group) * a.heads + x.h * a.group + row % a.group] =
                l == 0.0f ? -INFINITY : (m * c2 - kLift<DT> + __log2f(l)) * kLn2;
        }
    }
    return !x.whole ? 1.0f : l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;  // NaN stays NaN
}

// Few rows (16 of a segment at most): bound by the cache's bytes.  The four
// wavefronts share the rows and take every fourth step.  K and V go from
// memory to the MFMA operands' registers, past the L2, which nothing would
// read them from again; the next step's K is requested as soon as the scores
// have taken this one's, the next V after the products with this one, into the
// same registers, so that a wavefront has a step in flight for the registers
// of one.  96 requests of up to 24000 tokens (4.7 GB, 32 query and 8 key heads
// of 128) take 720 us with the join's 8, 6.6 TB/s; one of 1009 tokens 8 without,
// of which launch, plan and the first loads are nearly all.
template <int DT, int D>
__global__ __launch_bounds__(kAttThreads) __attribute__((amdgpu_waves_per_eu(D < 256 ? 2 : 1))) void k_attend_few(
    AttArgs a, SGDRC_SEQS_ARGS, uint32_t n_tiles, Gate g)
{
    const Seqs sq = {q_start, table, lens, totals};
    constexpr uint32_t WK = kAttWaves;
    constexpr int NB = 1, PARTS = 2, KK = D / 32, DD = D / 16;
    __shared__ uint32_t s_line[SGDRC_MAX_REQUESTS + 1];
    __shared__ uint32_t s_sum[kAttWaves];
    __shared__ float s_ml[kAttWaves][16 * NB][2];
    __shared__ __attribute__((aligned(16))) float s_o[kAttWaves][16][D + 4];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lane = threadIdx.x & 63u;
    const uint32_t col = lane & 15u, grp = lane >> 4;
    const float c2 = a.softcap > 0.0f ? 1.0f : a.scale * kLog2e;
    uint32_t pro_err = 0u;
    auto prologue = [&]() { plan_line<kAttThreads>(a, sq, 16u * NB, s_line, s_sum, pro_err); };
    auto body = [&](uint32_t t, uint32_t &err) {
        err |= pro_err;
        const Cuts cuts(a, s_line[a.n_requests]);
        const uint32_t lo = t < cuts.n ? cuts.cut(t) : 0u;
        const uint32_t hi = t < cuts.n ? cuts.cut(t + 1u) : 0u;
        for (uint32_t p = lo; p < hi;) {
            const Piece x = take_piece(a, sq, s_line, 16u * NB, t, lo, hi, p);
            p += x.u1 - x.u0;
            Rows<DT, D, NB> w;
            w.begin(a, x, 0u, 16u, col, grp);
            const uint32_t *const row_table = sq.table + (uint64_t)x.r * a.stride;
            const uint8_t *const head = a.c.pool + x.h * head_bytes<D>(a.c.bshift);
            const uint32_t bmask = (1u << a.c.bshift) - 1u;
            const int32_t drafted = (int32_t)(x.total - x.ctx);
            // K's lanes: token 8 (col / 4) + col % 4 (+ 4) of a step, in its
            // half col / 8; V's: tokens 8 grp .. + 7, in half grp / 2
            const uint32_t k_tok = (col >> 2) * 8u + (col & 3u);
            const uint32_t k_lane = k_off<D>(grp, k_tok & bmask, a.c.bshift);
            const uint32_t v_lane = v_off<D>((grp * 8u & bmask) >> 3, col, a.c.bshift);
            u32x4 kf[2][KK], vf[DD];
            auto load_k = [&](uint32_t u, const StepAt &at) __attribute__((always_inline)) {
                const uint8_t *const kp = (col < 8u ? at.p[0] : at.p[1]) + k_lane + (u * kStep & bmask) * 16u;
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    kf[0][kk] = load_nt(kp + ((uint32_t)kk * 64u << a.c.bshift));
                    kf[1][kk] = load_nt(kp + ((uint32_t)kk * 64u << a.c.bshift) + 64u);
                }
            };
            auto load_v = [&](uint32_t u, const StepAt &at) __attribute__((always_inline)) {
                const uint8_t *const vp = (grp < 2u ? at.p[0] : at.p[1]) + v_lane + (u * kStep & bmask) * (2u * D);
#pragma unroll
                for (int dd = 0; dd < DD; ++dd)
                    vf[dd] = load_nt(vp + dd * 256);
            };
            uint32_t u = x.u0 + wave;
            if (u < x.u1) {
                StepAt at = step_at(a, head, step_pages(row_table, x, u, a.c.bshift), x.total, err);
                load_k(u, at);
                load_v(u, at);
                StepPages ahead = step_pages(row_table, x, min(u + WK, x.u1 - 1u), a.c.bshift);
                auto scores = [&](f32x4 (&s)[NB][2]) __attribute__((always_inline)) {
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            s[b][q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                            for (int kk = 0; kk < KK; ++kk)
                                s[b][q] = att_mfma<DT>(kf[q][kk], w.q[b][kk], s[b][q]);
                        }
                };
                // K of the next step (past the piece's end its last one again),
                // which becomes ``at``
                auto next_k = [&]() __attribute__((always_inline)) {
                    at = step_at(a, head, ahead, x.total, err);
                    load_k(min(u + WK, x.u1 - 1u), at);
                    asm volatile("" ::: "memory");  // requested here, not where they are used
                    ahead = step_pages(row_table, x, min(u + 2u * WK, x.u1 - 1u), a.c.bshift);
                };
                auto next_v = [&]() __attribute__((always_inline)) {
                    load_v(min(u + WK, x.u1 - 1u), at);
                    asm volatile("" ::: "memory");
                };
                auto products = [&](const u32x4 (&pf)[PARTS][NB]) __attribute__((always_inline)) {
#pragma unroll
                    for (int dd = 0; dd < DD; ++dd)
#pragma unroll
                        for (int b = 0; b < NB; ++b)
#pragma unroll
                            for (int k = 0; k < PARTS; ++k)
                                w.acc[b][dd] = att_mfma<DT>(vf[dd], pf[k][b], w.acc[b][dd]);
                };
                // steps that every row sees whole, in a loop of their own: with
                // the others' code in it the compiler copies the accumulators
                // every time
                const uint32_t seen_steps = min(x.u1, x.ctx / kStep);
                for (; u < seen_steps && at.bad == 0u; u += WK) {
                    f32x4 s[NB][2];
                    u32x4 pf[PARTS][NB];
                    scores(s);
                    next_k();
                    if (a.softcap > 0.0f)
                        cap_scores<false, NB>(a, s);
                    weigh<DT, D, NB, PARTS>(w, s, c2, pf);
                    products(pf);
                    next_v();
                }
                for (; u < x.u1; u += WK) {
                    f32x4 s[NB][2];
                    u32x4 pf[PARTS][NB];
                    uint32_t seen[NB];
                    scores(s);
                    const uint32_t bad = at.bad;
                    next_k();
                    if (a.softcap > 0.0f)
                        cap_scores<false, NB>(a, s);
                    const int32_t j0 = (int32_t)(u * kStep + grp * 8u) - (int32_t)x.ctx;
                    const uint32_t there = (bad >> (grp >> 1)) & 1u ? 0u : low8(drafted - j0);
                    uint32_t odd = 0u;
#pragma unroll
                    for (int dd = 0; dd < DD; ++dd)
                        odd |= keep_there<DT>(vf[dd], there);
                    mask_scores<DT, D, NB>(a, w, j0, drafted, there, s, seen);
                    weigh<DT, D, NB, PARTS>(w, s, c2, pf);
                    if (__ballot(odd != 0u) != 0ull)
                        add_odd<DT, D, NB, PARTS>(w, pf, seen, [&](int dd) { return vf[dd]; });
                    else
                        products(pf);
                    next_v();
                }
            }
            // Join the wavefronts: maxima and sums first, then the weighted V,
            // 16 rows at a time.
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                w.l[b] = row_sum(w.l[b]);
                if (grp == 0u) {
                    s_ml[wave][16 * b + col][0] = w.m[b];
                    s_ml[wave][16 * b + col][1] = w.l[b];
                }
            }
            __syncthreads();
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                float m = -INFINITY, l = 0.0f;
#pragma unroll
                for (uint32_t k = 0; k < WK; ++k)
                    m = fmaxf(m, s_ml[k][16 * b + col][0]);
                const float use = m == -INFINITY ? 0.0f : m;
#pragma unroll
                for (uint32_t k = 0; k < WK; ++k)
                    l += s_ml[k][16 * b + col][1] * __builtin_amdgcn_exp2f((s_ml[k][16 * b + col][0] - use) * c2);
                const float f = __builtin_amdgcn_exp2f((w.m[b] - use) * c2) *
                                put_stats<DT, D>(a, x, 16u * NB, 16u * b + col, m, l, c2, wave == 0u && grp == 0u);
#pragma unroll
                for (int dd = 0; dd < DD; ++dd)
                    *reinterpret_cast<f32x4 *>(&s_o[wave][col][dd * 16 + grp * 4u]) = w.acc[b][dd] * f;
                __syncthreads();
                for (uint32_t i = threadIdx.x; i < 16u * (D / 4); i += kAttThreads) {
                    const uint32_t rr = i / (D / 4), d = i % (D / 4) * 4u;
                    f32x4 v = *reinterpret_cast<const f32x4 *>(&s_o[0][rr][d]);
#pragma unroll
                    for (uint32_t k = 1; k < WK; ++k)
                        v += *reinterpret_cast<const f32x4 *>(&s_o[k][rr][d]);
                    put_row<DT, D>(a, x, 16u * NB, 16u * b + rr, d, v);
                }
                __syncthreads();
            }
        }
    };
    single_tile_loop(g, n_tiles, prologue, body);
}

// The token of a step that lies at place ``p`` of K's LDS: the two K tiles' rows
// one after the other, so that the sixteen lanes that read a tile's rows of one
// 16-byte column meet all banks (in the order of memory every second lane's
// bank is taken twice).
__device__ __forceinline__ uint32_t lds_token(uint32_t p)
{
    return (p >> 2 & 3u) * 8u + (p >> 4 & 1u) * 4u + (p & 3u);
}

// Many rows: NW wavefronts of 16 NB rows each take the same steps, whose K and
// V pass through LDS once for all of them.  Every thread moves its share of a
// step, 16 bytes at a time, in the order of memory, which is the order of the
// MFMA operands: two steps ahead into registers, then to one of two LDS
// buffers, so that one barrier a step is enough.  Blocks of 16 rows go to the
// wavefronts in turn, and a wavefront leaves out those that a segment does not
// have: 192 rows are three blocks on every SIMD.
//
// Bound by the step's chain: the barrier, the operands from LDS (16 KiB a
// wavefront and step at head_dim 128), products, softmax, products follow each
// other, in both wavefronts of a SIMD at the same time, and their times add up
// (measured for 24 requests of 64 nodes, 64 query and 8 key heads, over 2000 to
// 8000 tokens: 408 us with the join's 27, where the arithmetic takes 210 at the
// rate of a large plain product).  Wavefronts of 16 rows, four on a
// SIMD, took 440, steps of 64 tokens 580, two groups of wavefronts half a step
// apart 500 and more, each with registers spilled.
template <int DT, int D, int NB, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2))) void k_attend_many(AttArgs a, SGDRC_SEQS_ARGS, uint32_t n_tiles, Gate g)
{
    const Seqs sq = {q_start, table, lens, totals};
    constexpr uint32_t T = 64u * NW;
    constexpr uint32_t kRows = 16u * NB * NW;
    constexpr int KK = D / 32, DD = D / 16;
    constexpr bool kTight = NB == 2 || D == 256;             // registers are short
    constexpr int VH = kTight ? DD / 4 : DD / 2;             // V's operands at a time
    constexpr uint32_t kPieces = 8u * D;                     // of 16 bytes: K's, then V's
    constexpr uint32_t PER = (kPieces + T - 1u) / T;         // a thread's
    constexpr uint32_t kBuf = kPieces * 16u;
    __shared__ uint32_t s_line[SGDRC_MAX_REQUESTS + 1];
    __shared__ uint32_t s_sum[NW];
    __shared__ __attribute__((aligned(16))) uint8_t s_kv[2u * kBuf];  // two steps
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lane = threadIdx.x & 63u;
    const uint32_t col = lane & 15u, grp = lane >> 4;
    const float c2 = a.softcap > 0.0f ? 1.0f : a.scale * kLog2e;
    uint32_t pro_err = 0u;
    auto prologue = [&]() { plan_line<T>(a, sq, kRows, s_line, s_sum, pro_err); };
    const uint32_t bmask = (1u << a.c.bshift) - 1u;
    // piece j of this thread: which half of the step it lies in, its place in
    // the head's chunk, and what a token further is
    auto half_of = [&](uint32_t i) { return (i < kPieces / 2u ? lds_token(i) >> 4 : (i - kPieces / 2u) / D >> 1); };
    auto place_of = [&](uint32_t i) {
        return i < kPieces / 2u ? k_off<D>(i / 32u, lds_token(i) & bmask, a.c.bshift)
                                : v_off<D>(((i - kPieces / 2u) / D * 8u & bmask) >> 3, i % D, a.c.bshift);
    };
    static_assert((kPieces / 2u) % D == 0u && kPieces / 2u % 32u == 0u, "V's pieces begin a row");
    auto body = [&](uint32_t t, uint32_t &err) {
        err |= pro_err;
        const Cuts cuts(a, s_line[a.n_requests]);
        const uint32_t lo = t < cuts.n ? cuts.cut(t) : 0u;
        const uint32_t hi = t < cuts.n ? cuts.cut(t + 1u) : 0u;
        for (uint32_t p = lo; p < hi;) {
            const Piece x = take_piece(a, sq, s_line, kRows, t, lo, hi, p);
            p += x.u1 - x.u0;
            Rows<DT, D, NB> w;
            w.begin(a, x, x.row0 + 16u * wave, 16u * NW, col, grp);
            const uint32_t *const row_table = sq.table + (uint64_t)x.r * a.stride;
            const uint8_t *const head = a.c.pool + x.h * head_bytes<D>(a.c.bshift);
            const int32_t drafted = (int32_t)(x.total - x.ctx);
            u32x4 st[2][PER];
            uint32_t bads[2] = {0u, 0u};
            auto fetch = [&](uint32_t tid, uint32_t u, const StepPages &sp, u32x4 (&to)[PER], uint32_t &bad) __attribute__((always_inline)) {
                const StepAt at = step_at(a, head, sp, x.total, err);
                bad = at.bad;
                const uint32_t off = u * kStep & bmask;
#pragma unroll
                for (uint32_t j = 0; j < PER; ++j) {
                    const uint32_t i = j * T + tid;
                    if (kPieces % T == 0u || i < kPieces)
                        to[j] = *reinterpret_cast<const u32x4 *>(
                            (half_of(i) ? at.p[1] : at.p[0]) + place_of(i) + off * (i < kPieces / 2u ? 16u : 2u * D));
                }
            };
            // ``edge``: a step that some row does not see whole; ``active``: this
            // wavefront's blocks that have rows
                auto step = [&](auto edge, auto active, uint32_t tid, uint32_t u, u32x4 (&from)[PER], uint32_t &bad_of, uint8_t *buf,
                            StepPages &ahead) __attribute__((always_inline)) {
                constexpr int ACT = active;
                // worked out every time where registers are short: spilled, waiting
                // for its reload would wait for the data on its way too
                const uint32_t in_step = kTight ? fresh(tid) : tid, col = in_step & 15u, grp = in_step >> 4 & 3u;
                const uint32_t bad = bad_of;
                uint32_t odd = 0u;
                if constexpr (edge) {
#pragma unroll
                    for (uint32_t j = 0; j < PER; ++j) {
                        const uint32_t i = j * T + tid;
                        if (i >= kPieces / 2u && i < kPieces) {
                            const uint32_t t8 = (i - kPieces / 2u) / D;
                            const int32_t j0 = (int32_t)(u * kStep + t8 * 8u) - (int32_t)x.ctx;
                            odd |= keep_there<DT>(from[j], (bad >> (t8 >> 1)) & 1u ? 0u : low8(drafted - j0));
                        }
                    }
                }
#pragma unroll
                for (uint32_t j = 0; j < PER; ++j) {
                    const uint32_t i = j * T + tid;
                    if (kPieces % T == 0u || i < kPieces)
                        *reinterpret_cast<u32x4 *>(buf + i * 16u) = from[j];
                }
                if constexpr (edge)
                    odd = __builtin_amdgcn_readfirstlane((uint32_t)__syncthreads_or((int)(odd != 0u)));
                else
                    __syncthreads();
                // past the piece's end its last step again: where loads may or may
                // not have been made, the compiler has to wait for all of them
                // before it uses older ones
                fetch(tid, min(u + 2u, x.u1 - 1u), ahead, from, bad_of);
                ahead = step_pages(row_table, x, min(u + 3u, x.u1 - 1u), a.c.bshift);
                if constexpr (ACT == 0)
                    return;
                const uint8_t *const kb = buf + (grp * 32u + col) * 16u;
                const uint8_t *const vb = buf + kBuf / 2u + (grp * D + col) * 16u;
                // operands in groups, each requested while the one before is
                // used, the first of V's before the softmax (left to itself the
                // compiler waits for each operand in turn)
                u32x4 kf[KK], vf[VH];
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
                    kf[kk] = *reinterpret_cast<const u32x4 *>(kb + kk * 2048);
                __builtin_amdgcn_sched_barrier(0);
                f32x4 s[NB][2];
#pragma unroll
                for (int q = 0; q < 2; ++q) {
#pragma unroll
                    for (int b = 0; b < ACT; ++b)
                        s[b][q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int kk = 0; kk < KK; ++kk) {
#pragma unroll
                        for (int b = 0; b < ACT; ++b)
                            s[b][q] = att_mfma<DT>(kf[kk], w.q[b][kk], s[b][q]);
                        if (q == 0)
                            kf[kk] = *reinterpret_cast<const u32x4 *>(kb + kk * 2048 + 256);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (a.softcap > 0.0f)
                    cap_scores<kTight, NB, ACT>(a, s);
#pragma unroll
                for (int dd = 0; dd < VH; ++dd)
                    vf[dd] = *reinterpret_cast<const u32x4 *>(vb + dd * 256);
                __builtin_amdgcn_sched_barrier(0);
                u32x4 pf[1][NB];
                uint32_t seen[NB];
                if constexpr (edge) {
                    const int32_t j0 = (int32_t)(u * kStep + grp * 8u) - (int32_t)x.ctx;
                    const uint32_t there = (bad >> (grp >> 1)) & 1u ? 0u : low8(drafted - j0);
                    mask_scores<DT, D, NB>(a, w, j0, drafted, there, s, seen);
                }
                weigh<DT, D, NB, 1, ACT>(w, s, c2, pf);
                if (edge && odd != 0u) {
                    add_odd<DT, D, NB, 1>(w, pf, seen, [&](int dd) {
                        return *reinterpret_cast<const u32x4 *>(vb + dd * 256);
                    });
                } else {
#pragma unroll
                    for (int dd = 0; dd < DD; ++dd) {
#pragma unroll
                        for (int b = 0; b < ACT; ++b)
                            w.acc[b][dd] = att_mfma<DT>(vf[dd % VH], pf[0][b], w.acc[b][dd]);
                        if (dd + VH < DD)
                            vf[dd % VH] = *reinterpret_cast<const u32x4 *>(vb + (dd + VH) * 256);
                    }
                }
            };
            fetch(threadIdx.x, x.u0, step_pages(row_table, x, x.u0, a.c.bshift), st[0], bads[0]);
            fetch(threadIdx.x, min(x.u0 + 1u, x.u1 - 1u), step_pages(row_table, x, min(x.u0 + 1u, x.u1 - 1u), a.c.bshift), st[1],
                  bads[1]);
            StepPages ahead = step_pages(row_table, x, min(x.u0 + 2u, x.u1 - 1u), a.c.bshift);
            // steps that every row sees whole in a loop of their own, two at a
            // time: with the others' code in it the compiler copies the
            // accumulators every time
            const uint32_t seen_steps = min(x.u1, x.ctx / kStep);
            uint32_t u = x.u0;
            auto whole = [&](auto active) __attribute__((always_inline)) {
                for (; u + 2u <= seen_steps && (bads[0] | bads[1]) == 0u; u += 2u) {
                    step(std::false_type(), active, threadIdx.x, u, st[0], bads[0], s_kv, ahead);
                    step(std::false_type(), active, threadIdx.x, u + 1u, st[1], bads[1], s_kv + kBuf, ahead);
                }
            };
            // (all wavefronts meet the same barriers, whichever loop they are in)
            const uint32_t first = x.row0 + 16u * wave;
            if (NB == 2 && first + 16u * NW < x.rows)
                whole(std::integral_constant<int, NB>());
            else if (first < x.rows)
                whole(std::integral_constant<int, 1>());
            else
                whole(std::integral_constant<int, 0>());
            const uint32_t edge_tid = fresh(threadIdx.x);
            // Q is read again where registers are short: kept over both loops,
            // some of it was spilled in the first
            if constexpr (kTight) {
                asm volatile("" ::: "memory");
                w.load_q(a, x, first, 16u * NW, edge_tid & 15u, edge_tid >> 4 & 3u);
            } else {
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    w.find(a, x, first, 16u * NW, edge_tid & 15u, b);
            }
            for (; u < x.u1; u += 2u) {
                step(std::true_type(), std::integral_constant<int, NB>(), edge_tid, u, st[0], bads[0], s_kv, ahead);
                if (u + 1u < x.u1)
                    step(std::true_type(), std::integral_constant<int, NB>(), edge_tid, u + 1u, st[1], bads[1], s_kv + kBuf,
                         ahead);
            }
            const uint32_t end_tid = fresh(threadIdx.x), col_e = end_tid & 15u, grp_e = end_tid >> 4 & 3u;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const uint32_t in = 16u * (NW * b + wave) + col_e;
                const float f = put_stats<DT, D>(a, x, kRows, in, w.m[b], row_sum(w.l[b]), c2, grp_e == 0u);
#pragma unroll
                for (int dd = 0; dd < DD; ++dd)
                    put_row<DT, D>(a, x, kRows, in, dd * 16u + grp_e * 4u, w.acc[b][dd] * f);
            }
            __syncthreads();  // the last step is read
        }
    };
    single_tile_loop(g, n_tiles, prologue, body);
}

// Lanes of a join's row (16 bytes each of the first D / 4), and rows of a tile.
constexpr uint32_t join_lanes(uint32_t dim) { return dim <= 64u ? 16u : dim <= 128u ? 32u : 64u; }
constexpr uint32_t join_rows(uint32_t dim) { return kAttThreads / join_lanes(dim); }

// A segment that lies in several ranges, t0 to t1: its rows, of head ``h``.
struct CutSegment {
    uint32_t start, rows, row0, h, t0, t1;
};

constexpr uint32_t kMostRanges = 512;

// Joins the pieces of segments that lie in several ranges; those inside one
// were written whole.  Every workgroup first lists those segments, a cut
// between ranges a thread, the first cut of a segment having it; a tile is
// some rows of one of them.  (Tiles by rows of the output, each with its
// request and cuts to find, took 88 us for 24 requests of 512 rows and 17 for
// one long cache, where these take 25 and 11.)
// Bound by latency: a row's pieces are asked for eight at a time.
template <int DT, int D>
__global__ __launch_bounds__(kAttThreads) void k_attend_join(AttArgs a, SGDRC_SEQS_ARGS, uint32_t rb, uint32_t chunks,
                                                             uint32_t n_tiles, Gate g)
{
    const Seqs sq = {q_start, table, lens, totals};
    constexpr uint32_t LANES = join_lanes(D), AHEAD = 8;
    __shared__ uint32_t s_line[SGDRC_MAX_REQUESTS + 1];
    __shared__ uint32_t s_sum[kAttWaves];
    __shared__ CutSegment s_cut[kMostRanges];
    const uint32_t lane = threadIdx.x % LANES, d = lane * 4u;
    const float c2 = a.softcap > 0.0f ? 1.0f : a.scale * kLog2e;
    uint32_t n_cut = 0u;
    auto prologue = [&]() {
        uint32_t seen_err = 0u;  // raised by the kernel before
        plan_line<kAttThreads>(a, sq, rb, s_line, s_sum, seen_err);
        const Cuts cuts(a, s_line[a.n_requests]);
        for (uint32_t t0 = 0u; t0 + 1u < cuts.n; t0 += kAttThreads) {
            const uint32_t t = t0 + threadIdx.x + 1u;
            bool first = false;
            CutSegment c = {};
            if (t < cuts.n) {
                const uint32_t p = cuts.cut(t), r = find_request(s_line, a.n_requests, p);
                const Req rq = load_req(a, sq, r);
                const uint32_t U = seg_steps(rq), k = (p - s_line[r]) / U, seg0 = s_line[r] + k * U;
                const uint32_t blocks = row_blocks(rq, a.group, rb);
                first = p != seg0 && cuts.cut(t - 1u) <= seg0;
                c = {rq.start, rq.nodes * a.group, k % blocks * rb, k / blocks, t - 1u, cuts.range_of(seg0 + U - 1u)};
            }
            const uint64_t who = __ballot(first);
            if ((threadIdx.x & 63u) == 0u)
                s_sum[threadIdx.x >> 6] = (uint32_t)__popcll(who);
            __syncthreads();
            uint32_t at = n_cut + (uint32_t)__popcll(who & ((1ull << (threadIdx.x & 63u)) - 1ull));
            for (uint32_t w = 0; w < kAttWaves; ++w) {
                at += w < threadIdx.x >> 6 ? s_sum[w] : 0u;
                n_cut += s_sum[w];
            }
            if (first)
                s_cut[at] = c;
            __syncthreads();
        }
        n_cut = __builtin_amdgcn_readfirstlane(n_cut);
    };
    auto body = [&](uint32_t tile, uint32_t &) {
        const uint32_t i = tile / chunks, in = tile % chunks * join_rows(D) + threadIdx.x / LANES;
        if (i >= n_cut)
            return;
        const uint32_t row0 = s_cut[i].row0, row = row0 + in, h = s_cut[i].h, start = s_cut[i].start;
        if (row >= s_cut[i].rows || in >= rb)
            return;
        // a segment's first piece is its range's last, the others their range's first
        const uint32_t t0 = __builtin_amdgcn_readfirstlane(s_cut[i].t0), t1 = __builtin_amdgcn_readfirstlane(s_cut[i].t1);
        auto part_of = [&](uint32_t q) { return 2u * q + (q == t0 ? 1u : 0u); };
        // maximum and sum, so far
        float m = -INFINITY, l = 0.0f;
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        for (uint32_t q0 = t0; q0 <= t1; q0 += LANES) {
            const uint32_t q = min(q0 + lane, t1), n = min(t1 + 1u - q0, LANES);
            f32x4 x[AHEAD];
            auto load = [&](uint32_t k0) __attribute__((always_inline)) {
#pragma unroll
                for (uint32_t e = 0; e < AHEAD; ++e) {
                    x[e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                    if (k0 + e < n && d < (uint32_t)D)
                        x[e] = *reinterpret_cast<const f32x4 *>(part_rows(a.work, part_of(q0 + k0 + e), rb, D) +
                                                                (uint64_t)in * D + d);
                }
                asm volatile("" ::: "memory");
            };
            const f32x2 st = *reinterpret_cast<const f32x2 *>(part_stats(a.work, part_of(q), rb, D) + in * 2u);
            load(0u);
            float mx = fmaxf(m, st[0]);
#pragma unroll
            for (int off = LANES / 2; off >= 1; off >>= 1)
                mx = fmaxf(mx, __shfl_xor(mx, off, 64));
            const float use = mx == -INFINITY ? 0.0f : mx, old = __builtin_amdgcn_exp2f((m - use) * c2);
            const float f = lane < n ? __builtin_amdgcn_exp2f((st[0] - use) * c2) : 0.0f;
            m = mx;
            l = l * old + (lane < n ? st[1] * f : 0.0f);
            v *= old;
            for (uint32_t k0 = 0u;;) {
#pragma unroll
                for (uint32_t e = 0; e < AHEAD; ++e)
                    v += x[e] * __shfl(f, (int)(min(k0 + e, LANES - 1u) + (threadIdx.x & 63u) / LANES * LANES), 64);
                k0 += AHEAD;
                if (k0 >= n)
                    break;
                load(k0);
            }
        }
#pragma unroll
        for (int off = LANES / 2; off >= 1; off >>= 1)
            l += __shfl_xor(l, off, 64);
        const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
        const uint32_t token = start + row / a.group, qh = h * a.group + row % a.group;
        if (d < (uint32_t)D) {
            const u32x2 two = {pack2<DT>(v[0] * inv, v[1] * inv), pack2<DT>(v[2] * inv, v[3] * inv)};
            *reinterpret_cast<u32x2 *>(a.o + token * a.o_token + qh * a.o_head + d * 2u) = two;
        }
        if (a.lse && lane == 0u)
            a.lse[(uint64_t)token * a.heads + qh] = l == 0.0f ? -INFINITY : (m * c2 - kLift<DT> + __log2f(l)) * kLn2;
    };
    single_tile_loop(g, n_tiles, prologue, body);
}

// -------------------------------------------------------------------- host

typedef void (*AttKernel)(AttArgs, const uint32_t *, const uint32_t *, const int32_t *, const int32_t *, uint32_t, Gate);
typedef void (*JoinKernel)(AttArgs, const uint32_t *, const uint32_t *, const int32_t *, const int32_t *, uint32_t,
                           uint32_t, uint32_t, Gate);

// How a call's rows are spread, by the most rows a segment can have: the
// kernel, its wavefronts, blocks of 16 rows of each, and the ranges that the
// line of steps is cut in: 512 where two workgroups fit a CU, 256 where one
// does, so that all are at work at once.  Both sides of each limit, for 32
// requests of 500 to 8000 tokens, 8 key heads of 128: 16 rows 112 us in the
// form for few, 128 in one for 32 of the same kind; 32 rows 133 there, 130
// here; 64 rows 139, in the form of 128 rows 151; 128 rows 189, in the form of
// 256 273.  Heads of 256 leave no registers for two blocks, and no LDS for a
// second workgroup: in 256 ranges 12 requests of up to 6000 tokens and 64 rows
// take 129 us and one of 60000 and 32 rows 102, in 512 140 and 118 (two rounds,
// twice the pieces to join); 32 requests of 500 to 8000 tokens, of 64 rows, 288
// against 279, as shorter ranges end more evenly.
struct AttForm {
    bool many;
    uint32_t nb, waves, ranges;

    uint32_t rows() const { return 16u * nb * (many ? waves : 1u); }
};

static AttForm att_form(uint32_t dim, uint32_t rows)
{
    if (rows <= 16u)
        return {false, 1, 4, dim == 256u ? 256u : 512u};
    if (rows <= 64u)
        return {true, 1, 4, dim == 256u ? 256u : 512u};
    if (dim == 256u || rows <= 128u)
        return {true, 1, 8, 256};
    return {true, 2, 8, 256};
}

template <int DT, int D>
static AttKernel att_kernel_d(AttForm f)
{
    if (!f.many)
        return k_attend_few<DT, D>;
    if (f.waves == 4)
        return k_attend_many<DT, D, 1, 4>;
    if constexpr (D != 256)
        if (f.nb == 2)
            return k_attend_many<DT, D, 2, 8>;
    return k_attend_many<DT, D, 1, 8>;
}

template <int DT>
static AttKernel att_kernel(uint32_t dim, AttForm f, JoinKernel *join)
{
    switch (dim) {
    case 64: *join = k_attend_join<DT, 64>; return att_kernel_d<DT, 64>(f);
    case 96: *join = k_attend_join<DT, 96>; return att_kernel_d<DT, 96>(f);
    case 128: *join = k_attend_join<DT, 128>; return att_kernel_d<DT, 128>(f);
    default: *join = k_attend_join<DT, 256>; return att_kernel_d<DT, 256>(f);
    }
}

template <typename K>
static int att_occupancy(K k, int threads)
{
    static std::mutex mu;
    static std::unordered_map<const void *, int> cache;
    std::lock_guard<std::mutex> lock(mu);
    auto it = cache.find((const void *)k);
    if (it != cache.end())
        return it->second;
    const int n = occupancy(k, threads);
    cache[(const void *)k] = n;
    return n;
}

static int check_att_shape(const sgdrc_kv_cache *cache, uint32_t n_heads, uint32_t max_nodes)
{
    const int rc = check_kv_cache(cache);
    if (rc)
        return rc;
    if (n_heads == 0 || n_heads > SGDRC_MAX_HEADS || n_heads % cache->kv_heads)
        return set_error(SGDRC_EINVAL, "n_heads %u: above %d or not a multiple of %u key/value heads", n_heads,
                         SGDRC_MAX_HEADS, cache->kv_heads);
    if (max_nodes < 1 || max_nodes > SGDRC_MAX_NODES)
        return set_error(SGDRC_EINVAL, "max_nodes %u outside 1..%d", max_nodes, SGDRC_MAX_NODES);
    return SGDRC_OK;
}

static uint64_t att_workspace(const sgdrc_kv_cache *cache, uint32_t n_heads, uint32_t max_nodes)
{
    const AttForm f = att_form(cache->head_dim, max_nodes * (n_heads / cache->kv_heads));
    return 2ull * f.ranges * f.rows() * (cache->head_dim + 2u) * sizeof(float);
}

}  // namespace sgdrc

using namespace sgdrc;

extern "C" {

int sgdrc_tree_attention_workspace(const sgdrc_kv_cache *cache, uint32_t n_heads, uint32_t max_nodes, uint64_t *bytes)
{
    clear_error();
    if (!bytes)
        return set_error(SGDRC_EINVAL, "bytes is NULL");
    const int rc = check_att_shape(cache, n_heads, max_nodes);
    if (rc)
        return rc;
    *bytes = att_workspace(cache, n_heads, max_nodes);
    return SGDRC_OK;
}

int colored_tree_attention(sgdrc_ctx *ctx, const sgdrc_kv_cache *cache, uint32_t layer, const sgdrc_rows *q,
                           uint32_t n_heads, const uint32_t *d_q_start, uint32_t n_tokens, uint32_t max_nodes,
                           const sgdrc_kv_blocks *blocks, const int32_t *d_lens, const int32_t *d_totals,
                           const uint64_t *d_mask, uint32_t mask_words, float scale, float softcap,
                           const sgdrc_rows *o, float *d_lse, void *d_work, uint64_t work_bytes, void *stream)
{
    clear_error();
    int rc = check_att_shape(cache, n_heads, max_nodes);
    if (rc || (rc = check_kv_blocks(blocks, cache->block_tokens)))
        return rc;
    if (layer >= cache->n_layers)
        return set_error(SGDRC_EINVAL, "layer %u of %u", layer, cache->n_layers);
    if (d_mask && (mask_words < 1 || mask_words > SGDRC_MAX_NODES / 64))
        return set_error(SGDRC_EINVAL, "mask_words %u outside 1..%d", mask_words, SGDRC_MAX_NODES / 64);
    if (!(scale > 0.0f) || !std::isfinite(scale))
        return set_error(SGDRC_EINVAL, "scale is not positive and finite");
    if (!(softcap >= 0.0f) || !std::isfinite(softcap))
        return set_error(SGDRC_EINVAL, "softcap is negative or not finite");
    if ((rc = check_aligned(d_q_start, 4, "q_start")) || (rc = check_aligned(d_lens, 4, "lens")) ||
        (rc = check_aligned(d_totals, 4, "totals")) || (rc = check_aligned(d_work, 256, "work")) ||
        (d_mask && (rc = check_aligned(d_mask, 8, "mask"))) || (d_lse && (rc = check_aligned(d_lse, 4, "lse"))))
        return rc;
    if (work_bytes < att_workspace(cache, n_heads, max_nodes))
        return set_error(SGDRC_EINVAL, "workspace of %llu bytes, %llu are needed", (unsigned long long)work_bytes,
                         (unsigned long long)att_workspace(cache, n_heads, max_nodes));
    if (n_tokens > 0x7FFFFFFFu)
        return set_error(SGDRC_EINVAL, "n_tokens above 2^31 - 1");
    const uint32_t group = n_heads / cache->kv_heads;
    const AttForm f = att_form(cache->head_dim, max_nodes * group);
    const uint32_t rb = f.rows();
    const uint64_t seg = ((uint64_t)blocks_width(blocks) * cache->block_tokens + kStep - 1u) / kStep;
    const uint64_t blocks_of_rows = (max_nodes * group + rb - 1u) / rb;
    if (seg * blocks_of_rows * cache->kv_heads > (1ull << 31) / blocks->n_requests)
        return set_error(SGDRC_EINVAL, "more than 2^31 steps of %u tokens at full tables", kStep);
    if (n_tokens && ((rc = check_rows(q, "q")) || (rc = check_rows(o, "o"))))
        return rc;
    Ctx *c = nullptr;
    if ((rc = check_ctx(ctx, &c)))
        return rc;
    if (n_tokens == 0)
        return SGDRC_OK;

    AttArgs a;
    a.c = kv_view(cache, layer);
    a.q = rows_view(q);
    a.o = static_cast<uint8_t *>(o->ptr);
    a.o_token = o->token_stride * 2u;
    a.o_head = o->head_stride * 2u;
    a.lse = d_lse;
    a.mask = d_mask;
    a.work = static_cast<float *>(d_work);
    a.n_requests = blocks->n_requests;
    a.stride = blocks->stride;
    a.width = blocks_width(blocks);
    a.n_tokens = n_tokens;
    a.max_nodes = max_nodes;
    a.mask_words = mask_words;
    a.heads = n_heads;
    a.group = group;
    a.scale = scale;
    a.softcap = softcap;
    // kept finite, so that a score of 0 stays 0 and a cap near fp32's end does not make all scores infinite
    const float most = std::numeric_limits<float>::max();
    a.cap_y = softcap > 0.0f ? std::min(scale / softcap, most) : 0.0f;
    a.cap_lin = std::min(scale * kLog2e, most);
    a.cap_out = std::min(softcap * kLog2e, most);
    a.most_ranges = f.ranges;
    JoinKernel join = nullptr;
    const AttKernel k = cache->dtype == SGDRC_BF16 ? att_kernel<SGDRC_BF16>(cache->head_dim, f, &join)
                                                   : att_kernel<SGDRC_F16>(cache->head_dim, f, &join);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    Gate g;
    LaunchInfo li;
    if ((rc = make_gate(c, stream, f.ranges, kStreamGroupCus, &g, &li, false, true)))
        return rc;
    const int threads = (int)(64u * f.waves);
    hipLaunchKernelGGL(k, dim3(gated_grid(c, att_occupancy(k, threads), f.ranges, li)), dim3(threads), 0, s, a, d_q_start,
                       blocks->table, d_lens, d_totals, f.ranges, g);
    SGDRC_HIP(hipGetLastError());
    if ((rc = finish_static_tlog(g, s)))
        return rc;
    const uint32_t chunks = (std::min(max_nodes * group, rb) + join_rows(cache->head_dim) - 1u) /
                            join_rows(cache->head_dim);
    const uint32_t join_tiles = (f.ranges - 1u) * chunks;
    if ((rc = make_gate(c, stream, join_tiles, kStreamGroupCus, &g, &li, false, true)))
        return rc;
    hipLaunchKernelGGL(join, dim3(gated_grid(c, att_occupancy(join, kAttThreads), join_tiles, li)), dim3(kAttThreads), 0, s, a,
                       d_q_start, blocks->table, d_lens, d_totals, rb, chunks, join_tiles, g);
    SGDRC_HIP(hipGetLastError());
    return finish_static_tlog(g, s);
}

}  // extern "C"
