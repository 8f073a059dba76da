// 4-bit weights with group scales: their layout, and the product with them for
// up to 16 rows of x.
//
//   y[b][m] = sum over groups G of s[m][G] * sum_{k in G} (n[m][k] - z[m][G]) x[b][k]
//
// The 16x16x32 matrix instruction takes W as its A operand (lane l: row l % 16,
// eight columns of lane group l / 16) and x as B (lane l: row l % 16 of x, the same
// columns).  A code becomes an element of A by an OR: the 16-bit pattern of 16
// has its four highest mantissa bits free, so that the pattern with n there is
// 16 + n, exactly, in both types; two codes, 16 bits apart in the word, take a
// shift and an and-or.  The instruction then sums (16 + n) x; the offset's share
// comes from a second one whose A operand is constant, -24 (16 + 8) without stored
// zero points: its result is where the first begins to add.  A group's sum
// (four of its rows in a lane) is scaled in fp32.
#include <algorithm>

#include "kv_common.hpp"

namespace sgdrc {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int kQ4Threads = 512;
constexpr int kQ4Waves = kQ4Threads / 64;
constexpr uint32_t kQ4Block = 1024;        // bytes of a block of codes, 16 rows by 128 columns
constexpr uint32_t kQ4Outside = 0xC0000000u;  // past x (2 MiB at most), with any column's offset added too
                                              // (as the bits of -2.0f an instruction's own constant, no register)

struct Q4View {
    const uint8_t *pool;
    uint64_t pool_pages;
    uint32_t scales, zeros;  // where they begin in the tensor, in 32 bytes
    uint32_t shift;
    uint32_t rows, cols, segs;
};

template <int DT>
__device__ __forceinline__ f32x4 q4_mfma(u32x4 a, u32x4 b, f32x4 c)
{
    if (DT == SGDRC_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
}

// Eight codes of a word as 16 + n, columns in order; ``one`` is q4_one in a
// vector register (an instruction takes one constant from elsewhere).
template <int DT>
constexpr uint32_t q4_one = DT == SGDRC_BF16 ? 0x41804180u : 0x4C004C00u;  // 16, twice

template <int DT>
__device__ __forceinline__ u32x4 q4_codes(uint32_t w, uint32_t one)
{
    constexpr int at = DT == SGDRC_BF16 ? 3 : 6;  // of the lowest free mantissa bit
    constexpr uint32_t field = 0x000F000Fu << at;
    u32x4 a;
    a.x = ((w << at) & field) | one;
    a.y = ((at >= 4 ? w << (at >= 4 ? at - 4 : 0) : w >> (at >= 4 ? 0 : 4 - at)) & field) | one;
    a.z = ((w >> (8 - at)) & field) | one;
    a.w = ((w >> (12 - at)) & field) | one;
    return a;
}

// Eight numbers of 16 bits as fp32.
template <int DT>
__device__ __forceinline__ void q4_widen(u32x4 w, f32x4 &lo, f32x4 &hi)
{
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (DT == SGDRC_BF16) {
            f[2 * i] = __uint_as_float(x[i] << 16);
            f[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
        } else {
            const f16x2 v = __builtin_bit_cast(f16x2, x[i]);
            f[2 * i] = (float)v.x;
            f[2 * i + 1] = (float)v.y;
        }
    }
    lo = f32x4{f[0], f[1], f[2], f[3]};
    hi = f32x4{f[4], f[5], f[6], f[7]};
}

// R blocks of rows a tile.  The segments of the columns are shared out to the
// workgroup's wavefronts in runs of ``run``, whose sums are added in wave order; a
// wavefront goes through its run in units of NS = 4 / R segments, R x NS blocks.  A
// unit's codes (4 KiB) and scales are in flight while the one before is worked on, a
// register of codes is loaded again as soon as it is used, over the ends of tiles
// too; the page-table entries are gathered a unit ahead of that.  x is in LDS in the
// order of the operands (XL), or comes from the L2 a segment ahead.
template <int DT, int PER, bool ZEROS, int R, bool XL>
__global__ __launch_bounds__(kQ4Threads) __attribute__((amdgpu_waves_per_eu(4))) void k_gemv_q4(
    Q4View v, const uint32_t *__restrict__ pt, const uint8_t *__restrict__ x, uint32_t batch, uint32_t run,
    float *__restrict__ y, uint32_t n_tiles, Gate g)
{
    constexpr int NS = 4 / R;
    constexpr int PLANES = ZEROS ? 2 : 1;
    constexpr uint32_t PIECES = 2u * PER;       // of 16 bytes, of a block's scales
    constexpr uint32_t PLANE = 4u * PIECES;     // lanes that fetch a unit's scales
    constexpr uint32_t RB = R == 4 ? 1 : 2;     // buffers of partial sums
    __shared__ f32x4 s_red[RB][kQ4Waves][R][64];
    __shared__ f32x4 s_sc[kQ4Waves][PLANES * PLANE * 2];  // of a unit, fp32: [plane][block][4][PER]
    extern __shared__ u32x4 s_x[];              // [segment][step][4][batch]
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63u;
    const uint32_t col = lane & 15u, grp = lane >> 4;
    const uint32_t x_row = v.cols * 2u;
    const uint32_t x_at = col < batch ? col * x_row + grp * 16u : kQ4Outside;
    const uint32_t x_lds = grp * batch + min(col, batch - 1u);
    const uint32_t first = wave * run, units = (run + NS - 1u) / NS;
    const uint32_t mine = min(run, v.segs > first ? v.segs - first : 0u);  // segments of the wavefront
    const uint32_t row_blocks = (v.rows + 15u) / 16u;
    // the offset's operand: -24 in both types, or -1 where the zero point comes with the group
    constexpr uint32_t kOff = ZEROS ? (DT == SGDRC_BF16 ? 0xBF80BF80u : 0xBC00BC00u)
                                    : (DT == SGDRC_BF16 ? 0xC1C0C1C0u : 0xCE00CE00u);
    uint32_t off_word = kOff, one = q4_one<DT>;
    asm volatile("" : "+v"(off_word), "+v"(one));
    const u32x4 off = {off_word, off_word, off_word, off_word};
    uint32_t bad = 0u;
    // A lane looks up the page of block ``my_code`` of a unit, and has one piece of the
    // scales: of a plane, of a block, from a byte of it on.
    const uint32_t my_code = lane & 3u, my_plane = lane / PLANE, my_block = lane % PLANE / PIECES;
    const uint32_t code_row = my_code / NS, code_seg = my_code % NS, sc_row = my_block / NS, sc_seg = my_block % NS;
    const uint32_t code_off = code_row * v.segs + code_seg, sc_off = sc_row * v.segs + sc_seg;
    // (lanes past the planes look up the last plane's entries: there are none behind the tensor's)
    const uint32_t sc_base = ZEROS && my_plane ? v.zeros : v.scales, sc_byte = lane % PIECES * 16u;
    const uint32_t low10 = (1u << (v.shift - 10u)) - 1u, low5 = (1u << (v.shift - 5u)) - 1u;

    u32x4 w[R][NS];   // a unit's codes
    u32x4 sc;         // this lane's piece of its scales
    u32x4 xs[2][4];   // x of a segment and of the next

    // A unit: its first block, how many row blocks and segments of it there are, and
    // this lane's page-table entries as the table holds them.
    struct Unit {
        uint32_t block, rows, segs, code_page, sc_page;
    };
    auto unit_of = [&](uint32_t t, uint32_t u) __attribute__((always_inline)) {
        Unit d;
        const uint32_t rb = t * R, s = u * NS;
        const bool in = (t < n_tiles) & (s < mine);
        d.rows = in ? min(row_blocks - rb, (uint32_t)R) : 0u;
        d.segs = in ? min(mine - s, (uint32_t)NS) : 0u;
        d.block = in ? rb * v.segs + first + s : 0u;
        // (a block that is not there: the first)
        const uint32_t code = d.block + (code_row < d.rows && code_seg < d.segs ? code_off : 0u);
        const uint32_t scale = d.block + (sc_row < d.rows && sc_seg < d.segs ? sc_off : 0u);
        d.code_page = pt[code >> (v.shift - 10u)];
        d.sc_page = pt[(sc_base + scale * PER) >> (v.shift - 5u)];
        return d;
    };
    auto load_codes = [&](const Unit &d, int b) __attribute__((always_inline)) {
        const uint32_t page = __builtin_amdgcn_readlane(d.code_page, b);
        const uint32_t r = b / NS, i = b % NS;
        const bool ok = r < d.rows && i < d.segs && page < v.pool_pages;
        const uint8_t *const at = v.pool + ((uint64_t)page << v.shift) + (((d.block + r * v.segs + i) & low10) << 10);
        w[r][i] = buf_load_nt(make_rsrc(at, ok ? kQ4Block : 0u), lane * 16u);
    };
    auto load_scales = [&](const Unit &d) __attribute__((always_inline)) {
        // (a block without codes, or without one of its planes, has no scales)
        const bool code_in = code_row < d.rows && code_seg < d.segs;
        const bool sc_in = sc_row < d.rows && sc_seg < d.segs && my_plane < (uint32_t)PLANES;
        const bool code_ok = d.code_page < v.pool_pages, sc_ok = d.sc_page < v.pool_pages;
        bad |= (code_in && !code_ok) || (sc_in && !sc_ok) ? kDevErrPtRange : 0u;
        const uint32_t codes_there = (uint32_t)__ballot(code_ok);
        bool ok = sc_in && sc_ok && ((codes_there >> my_block) & 1u);
        if (ZEROS) {
            const uint64_t planes_there = __ballot(sc_ok);
            ok = ok && ((planes_there >> (my_block * PIECES)) & 1ull) &&
                 ((planes_there >> (PLANE % 64u + my_block * PIECES)) & 1ull);
        }
        sc = u32x4{0u, 0u, 0u, 0u};
        if (ok)
            sc = load_nt(v.pool + ((uint64_t)d.sc_page << v.shift) +
                         ((((sc_base + (d.block + sc_off) * PER) & low5) << 5) + sc_byte));
    };
    const Rsrc xr = make_rsrc(x, batch * x_row);
    auto load_x = [&](uint32_t s, u32x4 (&to)[4]) __attribute__((always_inline)) {
        if (XL) {
            const u32x4 *const from = s_x + min(s, v.segs - 1u) * 16u * batch + x_lds;
#pragma unroll
            for (uint32_t k = 0; k < 4u; ++k)
                to[k] = from[k * 4u * batch];
        } else {
#pragma unroll
            for (uint32_t k = 0; k < 4u; ++k)
                to[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                    xr, s * 128u + 32u * k < v.cols ? x_at + (s * 128u + 32u * k) * 2u : kQ4Outside, 0, 0));
        }
    };
    bool begun = false;
    Unit next_unit;   // the one whose loads are made next
    auto prime = [&](uint32_t t, uint32_t next) __attribute__((always_inline)) {
        const Unit d = unit_of(t, 0u);
        next_unit = unit_of(units > 1u ? t : next, units > 1u ? 1u : 0u);
        load_scales(d);
#pragma unroll
        for (int b = 0; b < 4; ++b)
            load_codes(d, b);
        if (!XL)
            load_x(first, xs[0]);
        begun = false;
    };
    auto prologue = [&]() __attribute__((always_inline)) {
        if (XL) {
            const uint32_t n = v.segs * 16u * batch;
            for (uint32_t i = threadIdx.x; i < n; i += kQ4Threads) {
                const uint32_t b = i % batch, k = i / batch * 8u;  // columns in order: [segment][step][4]
                u32x4 z = {0u, 0u, 0u, 0u};
                if (k < v.cols)
                    z = *reinterpret_cast<const u32x4 *>(x + (uint64_t)b * x_row + k * 2u);
                s_x[i] = z;
            }
        }
    };
    uint32_t turn = 0u;
    auto body = [&](uint32_t t, uint32_t next, uint32_t after, uint32_t &) __attribute__((always_inline)) {
        float total[R][4] = {};
        if (XL && !begun)
            load_x(first, xs[0]);
        begun = true;
        for (uint32_t u = 0; u < units; ++u) {
            const bool end = u + 1u == units;
            const Unit d = next_unit;
            // the entries of the unit after the next
            next_unit = end ? (units > 1u ? unit_of(next, 1u) : unit_of(after, 0u))
                            : u + 2u < units ? unit_of(t, u + 2u) : unit_of(next, 0u);
            // this unit's scales, in fp32
            if (my_plane < (uint32_t)PLANES) {
                f32x4 lo, hi;
                q4_widen<DT>(sc, lo, hi);
                if (ZEROS) {
                    const float add = my_plane ? 16.0f : 0.0f;
                    lo += add;
                    hi += add;
                }
                s_sc[wave][lane * 2u] = lo;
                s_sc[wave][lane * 2u + 1u] = hi;
            }
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                u32x4 xb[4];
#pragma unroll
                for (uint32_t k = 0; k < 4u; ++k)
                    xb[k] = xs[NS > 1 ? i % 2 : 0][k];
                load_x(first + (i + 1 < NS ? u * NS + i + 1u : end ? 0u : (u + 1u) * NS), xs[NS > 1 ? (i + 1) % 2 : 0]);
                constexpr int kSteps = 4 / PER;
#pragma unroll
                for (int p = 0; p < PER; ++p) {
                    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int k = p * kSteps; k < (p + 1) * kSteps; ++k)
                        o = q4_mfma<DT>(off, xb[k], o);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const u32x4 ww = w[r][i];
                        const uint32_t wk[4] = {ww.x, ww.y, ww.z, ww.w};
                        f32x4 acc = ZEROS ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : o;
#pragma unroll
                        for (int k = p * kSteps; k < (p + 1) * kSteps; ++k)
                            acc = q4_mfma<DT>(q4_codes<DT>(wk[k], one), xb[k], acc);
                        const uint32_t at = ((r * NS + i) * 4u + grp) * PER + p;
                        const f32x4 f = s_sc[wave][at];
                        f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
                        if (ZEROS)
                            z = s_sc[wave][PLANE * 2u + at];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float dot = ZEROS ? __builtin_fmaf(z[j], o[j], acc[j]) : acc[j];
                            total[r][j] = __builtin_fmaf(f[j], dot, total[r][j]);
                            // (left to themselves the sums sink to the unit's end, past all loads)
                            asm volatile("" : "+v"(total[r][j]));
                        }
                        if (p == PER - 1) {
                            if (i == 0 && r == 0)
                                load_scales(d);
                            load_codes(d, r * NS + i);
                        }
                        if (p == PER - 1 || PER == 4)
                            __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
            s_red[turn % RB][wave][r][lane] = f32x4{total[r][0], total[r][1], total[r][2], total[r][3]};
        __syncthreads();
        // (with two buffers, one is written again only after the next tile's barrier)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (wave == (turn + r * (kQ4Waves / R)) % (uint32_t)kQ4Waves) {
                f32x4 sum = s_red[turn % RB][0][r][lane];
#pragma unroll
                for (int i = 1; i < kQ4Waves; ++i)
                    sum += s_red[turn % RB][i][r][lane];
                if (col < batch) {
#pragma unroll
                    for (uint32_t j = 0; j < 4u; ++j) {
                        const uint32_t m = (t * R + r) * 16u + grp * 4u + j;
                        if (m < v.rows)
                            y[(uint64_t)col * v.rows + m] = sum[j];
                    }
                }
            }
        }
        turn += 1u;
        if (RB == 1)
            __syncthreads();
    };
    single_tile_stream(g, n_tiles, prime, prologue, body);
    if (bad)
        raise_flag(g.err, bad);
}

// The packed layout is the codes' alone, so the kernel is a copy: 1 byte read and
// half a byte written a weight.  A wavefront takes kPackBlocks blocks in a row, whose
// loads go out together: eight lanes read the 128 codes of a row, 16 each, and have
// by them one word of two pieces, so that both the reads and the stores run over
// whole cache lines; the block's scales go through its first lanes.  The codes are
// read once and stay out of the L2's way (nontemporal).  11008 x 4096: 16.3 us, 4.1 TB/s
// (byte by byte 20.3; one block 20.4, four 19.4; ordinary loads 18.2).
constexpr int kPackThreads = 256;
constexpr uint32_t kPackBlocks = 2;

struct __attribute__((packed, aligned(1))) Codes16 {
    u32x4 v;
};

// The word of 8 codes: column e at bit 4 (e / 2 + 4 (e % 2)).
__device__ __forceinline__ uint32_t q4_word(uint32_t lo, uint32_t hi)
{
    auto two = [](uint32_t x) {
        x &= 0x000F000Fu;
        return (x | x >> 12) & 0xFFu;
    };
    return two(lo) | two(hi) << 8 | two(lo >> 8) << 16 | two(hi >> 8) << 24;
}

// Where a byte of the matrix lies; nullptr and the flag if its page is none.
__device__ __forceinline__ uint8_t *q4_place(const Q4View &v, const uint32_t *pt, uint64_t byte, uint32_t &err)
{
    const uint32_t e = checked_page(pt, byte >> v.shift, v.pool_pages, err);
    return e == kBadPage ? nullptr
                         : const_cast<uint8_t *>(v.pool) + ((uint64_t)e << v.shift) + (byte & ((1ull << v.shift) - 1ull));
}

__global__ __launch_bounds__(kPackThreads) void k_q4_pack(Q4View v, const uint32_t *__restrict__ pt, uint32_t per,
                                                          const uint8_t *__restrict__ codes, uint64_t stride,
                                                          const uint16_t *__restrict__ scales,
                                                          const uint16_t *__restrict__ zeros, uint32_t n_blocks,
                                                          uint32_t n_tiles, Gate g)
{
    constexpr uint32_t kWaves = kPackThreads / 64;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t code_row = lane / 8u, eighth = lane % 8u;  // and the row 8 further
    const uint32_t row = lane / per, grp = lane % per;  // of the block's 16 per scales, one a lane
    const uint32_t n_groups = v.cols * per / 128u;
    const uint32_t at = (((row / 4u) * per + grp) * 4u + row % 4u) * 2u;
    auto body = [&](uint32_t t, uint32_t, uint32_t &err, auto &&) {
        const uint32_t first = (t * kWaves + wave) * kPackBlocks;
        u32x4 c[kPackBlocks][2];
        uint16_t s[kPackBlocks], z[kPackBlocks];
#pragma unroll
        for (uint32_t b = 0; b < kPackBlocks; ++b) {
            const uint32_t block = first + b, tile = block / v.segs, seg = block % v.segs;
            const uint32_t k = seg * 128u + eighth * 16u, gg = seg * per + grp;
            const uint64_t m = tile * 16ull + code_row, mm = tile * 16ull + row;
#pragma unroll
            for (uint32_t h = 0; h < 2u; ++h) {
                c[b][h] = u32x4{0u, 0u, 0u, 0u};
                if (m + 8u * h < v.rows && k < v.cols)
                    c[b][h] = __builtin_nontemporal_load(
                        &reinterpret_cast<const Codes16 *>(codes + (m + 8u * h) * stride + k)->v);
            }
            s[b] = z[b] = 0u;
            if (row < 16u && mm < v.rows && gg < n_groups) {
                s[b] = scales[mm * n_groups + gg];
                if (zeros)
                    z[b] = zeros[mm * n_groups + gg];
            }
        }
#pragma unroll
        for (uint32_t b = 0; b < kPackBlocks; ++b) {
            const uint32_t block = first + b;
            if (block >= n_blocks)
                break;
            if (uint8_t *const p = q4_place(v, pt, (uint64_t)block * kQ4Block, err)) {
                const uint32_t piece = eighth % 2u * 2u;
                uint32_t *const words = reinterpret_cast<uint32_t *>(p) + (piece * 16u + code_row) * 4u + eighth / 2u;
#pragma unroll
                for (uint32_t h = 0; h < 2u; ++h) {
                    words[h * 32u] = q4_word(c[b][h].x, c[b][h].y);
                    words[h * 32u + 64u] = q4_word(c[b][h].z, c[b][h].w);
                }
            }
            if (row < 16u) {
                if (uint8_t *const p = q4_place(v, pt, v.scales * 32ull + (uint64_t)block * (per * 32u) + at, err))
                    *reinterpret_cast<uint16_t *>(p) = s[b];
                if (zeros)
                    if (uint8_t *const p = q4_place(v, pt, v.zeros * 32ull + (uint64_t)block * (per * 32u) + at, err))
                        *reinterpret_cast<uint16_t *>(p) = z[b];
            }
        }
    };
    tile_loop<Claim::Ahead>(g, n_tiles, NoOp(), body);
}

static uint64_t q4_blocks(const sgdrc_q4 *q)
{
    return ((uint64_t)q->rows + 15u) / 16u * ((q->cols + 127u) / 128u);
}

static int check_q4(const sgdrc_q4 *q)
{
    if (!q)
        return set_error(SGDRC_EINVAL, "q is NULL");
    if (q->dtype != SGDRC_BF16 && q->dtype != SGDRC_F16)
        return set_error(SGDRC_EINVAL, "q: dtype %u is neither bf16 nor f16", q->dtype);
    if (q->group != 32 && q->group != 64 && q->group != 128)
        return set_error(SGDRC_EINVAL, "q: group %u is not 32, 64 or 128", q->group);
    if (q->rows == 0 || q->cols == 0 || q->cols % q->group)
        return set_error(SGDRC_EINVAL, "q: %u rows by %u columns in groups of %u", q->rows, q->cols, q->group);
    if (q->cols > 65536)
        return set_error(SGDRC_EINVAL, "q: more than 65536 columns");
    if (q->zeros > 1 || q->reserved)
        return set_error(SGDRC_EINVAL, "q: zeros must be 0 or 1, reserved 0");
    if (q4_blocks(q) >= (1ull << 26))
        return set_error(SGDRC_EINVAL, "q: 2^26 blocks or more");
    return SGDRC_OK;
}

static uint64_t q4_scale_bytes(const sgdrc_q4 *q) { return q4_blocks(q) * (128u / q->group) * 32u; }

static Q4View q4_view(const sgdrc_paged *w, const sgdrc_q4 *q, uint32_t page_shift)
{
    const uint32_t s = (uint32_t)(q4_blocks(q) * (kQ4Block / 32u));
    return {static_cast<const uint8_t *>(w->pool), w->pool_pages, s, s + (uint32_t)(q4_scale_bytes(q) / 32u),
            page_shift, q->rows, q->cols, (q->cols + 127u) / 128u};
}

typedef void (*Q4Kernel)(Q4View, const uint32_t *, const uint8_t *, uint32_t, uint32_t, float *, uint32_t, Gate);

// Which form of the kernel a call takes: the row blocks of a tile, and where x is.
// None changes a result.
//
// A wavefront with u segments goes through a tile in ceil(u / 4), ceil(u / 2) or u
// units for 1, 2 or 4 row blocks, and a CU has ceil(tiles / CUs) tiles one after the
// other or side by side.  A unit with one row block loads x for four segments, with
// four blocks for one, which all blocks share; what it costs grows with the rows of x that
// come out of LDS or the L2, while four blocks cost their codes, and more with zero points.  The form with the
// least cost, in the weights below, is slower than the best of the three by 0.2 to 1.2 % on average
// over each kind of matrix and by 17 % at worst, over 1100 measured calls: all groups, with and without zero points,
// 2048 to 65536 rows, 1024 to 11008 columns, batches 1 to 16.  The weights do not
// know the groups' size; in the lines marked * they take the slower form.
// bf16, 2 MiB pages, groups of 64, copies in turn (400 MB or 10 of them), us:
//                                                 1    2, x in LDS    4, x in the L2
//   4096 x 11008, batch 1                      10.5          14.4              19.6
//   11008 x 4096, batch 1                      10.1          11.8              11.1
//   11008 x 4096, batch 8                      13.7             -              11.4
//   the same, groups of 32 with zero points    13.9             -              14.6  *
//   12288 x 2048, batch 4                      10.2           9.5               8.0
//   9216 x 5120, batch 16                      28.7             -              13.1
//   6144 x 2048, batch 1                        8.0           6.8               7.8
//   16384 x 8192, batch 1                      18.8          18.4              19.8  *
//   16384 x 8192, batch 16                     37.8             -              21.1
struct Q4Plan {
    uint32_t blocks;  // of rows, a tile: 1, 2 or 4
    bool x_lds;
};

constexpr uint64_t kQ4XLds = 24576;  // bytes of x in LDS at most

static Q4Plan q4_plan(const sgdrc_q4 *q, uint32_t batch, uint32_t allowed)
{
    const uint32_t segs = (q->cols + 127u) / 128u;
    const uint64_t row_blocks = ((uint64_t)q->rows + 15u) / 16u, cus = std::max(allowed, 1u);
    const uint64_t run = (segs + kQ4Waves - 1u) / kQ4Waves;
    const bool fits = (uint64_t)segs * 256u * batch <= kQ4XLds;
    const auto rounds = [&](uint64_t blocks) { return (row_blocks + blocks * cus - 1u) / (blocks * cus); };
    const uint64_t one = rounds(1u) * ((run + 3u) / 4u) * (8u + batch);
    const uint64_t two = fits ? rounds(2u) * ((run + 1u) / 2u) * (9u + batch) : ~0ull;
    const uint64_t four = rounds(4u) * (run * (q->zeros ? 9u : 8u) + 1u);
    if (four < one && four < two)
        return {4u, false};
    if (two < one)
        return {2u, true};
    return {1u, fits};
}

template <int DT, int PER, bool ZEROS>
static Q4Kernel q4_form(const Q4Plan &p)
{
    if (p.blocks == 4u)
        return k_gemv_q4<DT, PER, ZEROS, 4, false>;
    if (p.blocks == 2u)
        return k_gemv_q4<DT, PER, ZEROS, 2, true>;
    return p.x_lds ? k_gemv_q4<DT, PER, ZEROS, 1, true> : k_gemv_q4<DT, PER, ZEROS, 1, false>;
}

template <int DT>
static Q4Kernel q4_kernel(const sgdrc_q4 *q, const Q4Plan &p)
{
    switch (128u / q->group) {
    case 1: return q->zeros ? q4_form<DT, 1, true>(p) : q4_form<DT, 1, false>(p);
    case 2: return q->zeros ? q4_form<DT, 2, true>(p) : q4_form<DT, 2, false>(p);
    default: return q->zeros ? q4_form<DT, 4, true>(p) : q4_form<DT, 4, false>(p);
    }
}

constexpr uint32_t kLdsBytes = 163840u;  // of a CU

// Workgroups of a kernel that fit a CU with ``dynamic`` bytes of LDS each beside its own.
static int q4_occupancy(Q4Kernel k, uint32_t dynamic)
{
    struct Fit {
        int regs;
        uint32_t lds;
    };
    static std::mutex mu;
    static std::unordered_map<const void *, Fit> cache;
    std::lock_guard<std::mutex> lock(mu);
    auto it = cache.find((const void *)k);
    if (it == cache.end()) {
        hipFuncAttributes a{};
        Fit f = {occupancy(k, kQ4Threads), kLdsBytes};
        if (hipFuncGetAttributes(&a, (const void *)k) == hipSuccess)
            f.lds = (uint32_t)a.sharedSizeBytes;
        it = cache.emplace((const void *)k, f).first;
    }
    const uint32_t lds = it->second.lds + dynamic;
    return std::min(it->second.regs, (int)(kLdsBytes / std::max(lds, 1u)));
}

}  // namespace sgdrc

using namespace sgdrc;

extern "C" {

int sgdrc_q4_bytes(const sgdrc_q4 *q, uint64_t *bytes)
{
    clear_error();
    const int rc = check_q4(q);
    if (rc)
        return rc;
    if (!bytes)
        return set_error(SGDRC_EINVAL, "bytes is NULL");
    *bytes = q4_blocks(q) * kQ4Block + q4_scale_bytes(q) * (q->zeros ? 2u : 1u);
    return SGDRC_OK;
}

int colored_q4_pack(sgdrc_ctx *ctx, const sgdrc_paged *dst, const sgdrc_q4 *q, const uint8_t *d_codes,
                    uint64_t code_stride, const void *d_scales, const void *d_zeros, uint32_t page_shift, void *stream)
{
    clear_error();
    int rc = check_shift(page_shift);
    if (rc || (rc = check_paged(dst, "dst")) || (rc = check_q4(q)))
        return rc;
    if (!d_codes || !d_scales || (q->zeros != 0) != (d_zeros != nullptr))
        return set_error(SGDRC_EINVAL, "codes or scales NULL, or zero points without q->zeros or the reverse");
    if ((reinterpret_cast<uintptr_t>(d_scales) | reinterpret_cast<uintptr_t>(d_zeros)) & 1u)
        return set_error(SGDRC_EINVAL, "scales and zero points must be 2-byte aligned");
    if (code_stride < q->cols || code_stride > (1ull << 40))
        return set_error(SGDRC_EINVAL, "code_stride %llu", (unsigned long long)code_stride);
    constexpr uint64_t kTile = kPackThreads / 64 * kPackBlocks;
    const uint64_t blocks = q4_blocks(q), tiles = (blocks + kTile - 1) / kTile;
    Ctx *c = nullptr;
    if ((rc = check_ctx(ctx, &c)))
        return rc;
    Gate g;
    LaunchInfo li;
    if ((rc = make_gate(c, stream, tiles, kGemvGroupCus, &g, &li, false, true)))
        return rc;
    static const int occ = occupancy(k_q4_pack, kPackThreads);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(k_q4_pack, dim3(gated_grid(c, occ, tiles, li)), dim3(kPackThreads), 0, s,
                       q4_view(dst, q, page_shift), dst->pt, 128u / q->group, d_codes, code_stride,
                       static_cast<const uint16_t *>(d_scales), static_cast<const uint16_t *>(d_zeros), (uint32_t)blocks,
                       (uint32_t)tiles, g);
    SGDRC_HIP(hipGetLastError());
    return finish_static_tlog(g, s);
}

int colored_gemv_q4(sgdrc_ctx *ctx, const sgdrc_paged *w, const sgdrc_q4 *q, const void *d_x, uint32_t batch,
                    float *d_y, uint32_t page_shift, void *stream)
{
    clear_error();
    int rc = check_shift(page_shift);
    if (rc || (rc = check_paged(w, "w")) || (rc = check_q4(q)))
        return rc;
    if (batch < 1 || batch > SGDRC_MAX_Q4_BATCH)
        return set_error(SGDRC_EINVAL, "batch %u outside 1..%d", batch, SGDRC_MAX_Q4_BATCH);
    if (!d_x || !d_y)
        return set_error(SGDRC_EINVAL, "NULL x or y");
    if ((reinterpret_cast<uintptr_t>(d_x) & 15u) || (reinterpret_cast<uintptr_t>(d_y) & 3u))
        return set_error(SGDRC_EINVAL, "x must be 16-byte and y 4-byte aligned");
    Ctx *c = nullptr;
    if ((rc = check_ctx(ctx, &c)))
        return rc;
    const Q4Plan p = q4_plan(q, batch, (uint32_t)stream_allowed_cus(c, stream));
    const uint32_t segs = (q->cols + 127u) / 128u;
    const uint64_t tiles = (((uint64_t)q->rows + 15u) / 16u + p.blocks - 1u) / p.blocks;
    Gate g;
    LaunchInfo li;
    if ((rc = make_gate(c, stream, tiles, kStreamGroupCus, &g, &li, false, true)))
        return rc;
    const Q4Kernel k = q->dtype == SGDRC_BF16 ? q4_kernel<SGDRC_BF16>(q, p) : q4_kernel<SGDRC_F16>(q, p);
    const uint32_t lds = p.x_lds ? segs * 256u * batch : 0u;
    const int occ = q4_occupancy(k, lds);
    if (occ < 1)
        return set_error(SGDRC_EINVAL, "the kernel does not fit a CU (library fault)");
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(k, dim3(gated_grid(c, occ, tiles, li)), dim3(kQ4Threads), lds, s,
                       q4_view(w, q, page_shift), w->pt, static_cast<const uint8_t *>(d_x), batch,
                       (segs + kQ4Waves - 1u) / kQ4Waves, d_y, (uint32_t)tiles, g);
    SGDRC_HIP(hipGetLastError());
    return finish_static_tlog(g, s);
}

}  // extern "C"
