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

#include "host_common.hpp"

namespace sgdrc {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int kQ4Threads = 512;
constexpr int kQ4Waves = kQ4Threads / 64;
constexpr uint32_t kQ4Block = 1024;        // bytes of a block of codes, 16 rows by 128 columns
constexpr uint32_t kQ4Outside = 0xFFFFFFF0u;  // an offset past any buffer resource

struct Q4View {
    const uint8_t *pool;
    const uint32_t *pt;
    uint64_t pool_pages;
    uint64_t scales, zeros;  // where they begin in the tensor
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

// Eight codes of a word as 16 + n, columns in order.
template <int DT>
__device__ __forceinline__ u32x4 q4_codes(uint32_t w)
{
    constexpr uint32_t one = DT == SGDRC_BF16 ? 0x41804180u : 0x4C004C00u;  // 16, twice
    constexpr int at = DT == SGDRC_BF16 ? 3 : 6;                            // of the lowest free mantissa bit
    constexpr uint32_t field = 0x000F000Fu << at;
    u32x4 a;
    a.x = ((w << at) & field) | one;
    a.y = ((at >= 4 ? w << (at >= 4 ? at - 4 : 0) : w >> (at >= 4 ? 0 : 4 - at)) & field) | one;
    a.z = ((w >> (8 - at)) & field) | one;
    a.w = ((w >> (12 - at)) & field) | one;
    return a;
}

// Two numbers of 16 bits.
template <int DT>
__device__ __forceinline__ void q4_pair(uint32_t w, float &lo, float &hi)
{
    if (DT == SGDRC_BF16) {
        lo = __uint_as_float(w << 16);
        hi = __uint_as_float(w & 0xFFFF0000u);
    } else {
        const f16x2 v = __builtin_bit_cast(f16x2, w);
        lo = (float)v.x;
        hi = (float)v.y;
    }
}

// A tile is a block of 16 rows; its columns' segments are shared out to the
// workgroup's wavefronts in contiguous runs, whose sums are added in wave order.
template <int DT, int PER, bool ZEROS>
__global__ __launch_bounds__(kQ4Threads) void k_gemv_q4(Q4View v, const uint8_t *__restrict__ x, uint32_t batch,
                                                        float *__restrict__ y, uint32_t n_tiles, Gate g)
{
    constexpr uint32_t kScaleBlock = PER * 32u;
    constexpr int SW = 2 * PER;  // words of scales a lane takes
    __shared__ f32x4 s_red[kQ4Waves][64];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63u;
    const uint32_t col = lane & 15u, grp = lane >> 4;
    const uint32_t x_row = v.cols * 2u;
    const uint64_t pmask = (1ull << v.shift) - 1ull;
    const Rsrc xr = make_rsrc(x, batch * x_row);
    const uint32_t x_at = col < batch ? col * x_row + grp * 16u : kQ4Outside;
    const uint32_t s0 = v.segs * wave / (uint32_t)kQ4Waves, s1 = v.segs * (wave + 1u) / (uint32_t)kQ4Waves;
    // the offset's operand: -24 in both types, or -1 where the zero point comes with the group
    constexpr uint32_t kOff = ZEROS ? (DT == SGDRC_BF16 ? 0xBF80BF80u : 0xBC00BC00u)
                                    : (DT == SGDRC_BF16 ? 0xC1C0C1C0u : 0xCE00CE00u);
    const u32x4 off = {kOff, kOff, kOff, kOff};
    auto body = [&](uint32_t t, uint32_t, uint32_t &err, auto &&) {
        f32x4 total = {0.0f, 0.0f, 0.0f, 0.0f};
        for (uint32_t s = s0; s < s1; ++s) {
            const uint64_t block = (uint64_t)t * v.segs + s;
            auto at = [&](uint64_t byte, uint32_t &e) {
                e = __builtin_amdgcn_readfirstlane(checked_page(v.pt, byte >> v.shift, v.pool_pages, err));
                return v.pool + ((uint64_t)e << v.shift) + (byte & pmask);
            };
            uint32_t ec, es, ez = 0u;
            const uint8_t *const pc = at(block * kQ4Block, ec);
            const uint8_t *const ps = at(v.scales + block * kScaleBlock, es);
            const uint8_t *const pz = ZEROS ? at(v.zeros + block * kScaleBlock, ez) : ps;
            const bool ok = ec != kBadPage && es != kBadPage && ez != kBadPage;
            const u32x4 w = buf_load_nt(make_rsrc(pc, ok ? kQ4Block : 0u), lane * 16u);
            uint32_t sc[SW], zp[SW];
            const Rsrc rs = make_rsrc(ps, ok ? kScaleBlock : 0u), rz = make_rsrc(pz, ok ? kScaleBlock : 0u);
#pragma unroll
            for (int i = 0; i < SW; ++i) {
                sc[i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, grp * (uint32_t)SW * 4u + i * 4u, 0, kAuxNt);
                zp[i] = ZEROS ? (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rz, grp * (uint32_t)SW * 4u + i * 4u, 0, kAuxNt) : 0u;
            }
            u32x4 xb[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                xb[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                    xr, s * 128u + 32u * i < v.cols ? x_at + (s * 128u + 32u * i) * 2u : kQ4Outside, 0, 0));
            const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
            constexpr int kSteps = 4 / PER;
#pragma unroll
            for (int p = 0; p < PER; ++p) {
                f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = p * kSteps; i < (p + 1) * kSteps; ++i)
                    o = q4_mfma<DT>(off, xb[i], o);
                f32x4 acc = ZEROS ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : o;
#pragma unroll
                for (int i = p * kSteps; i < (p + 1) * kSteps; ++i)
                    acc = q4_mfma<DT>(q4_codes<DT>(ww[i]), xb[i], acc);
                float f[4], z[4];
                q4_pair<DT>(sc[2 * p], f[0], f[1]);
                q4_pair<DT>(sc[2 * p + 1], f[2], f[3]);
                if (ZEROS) {
                    q4_pair<DT>(zp[2 * p], z[0], z[1]);
                    q4_pair<DT>(zp[2 * p + 1], z[2], z[3]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float a = ZEROS ? __builtin_fmaf(z[j] + 16.0f, o[j], acc[j]) : acc[j];
                    total[j] = __builtin_fmaf(f[j], a, total[j]);
                }
            }
        }
        s_red[wave][lane] = total;
        __syncthreads();
        if (wave == 0u) {
            f32x4 r = s_red[0][lane];
#pragma unroll
            for (int i = 1; i < kQ4Waves; ++i)
                r += s_red[i][lane];
            if (col < batch) {
#pragma unroll
                for (uint32_t j = 0; j < 4u; ++j) {
                    const uint32_t m = t * 16u + grp * 4u + j;
                    if (m < v.rows)
                        y[(uint64_t)col * v.rows + m] = r[j];
                }
            }
        }
        __syncthreads();
    };
    tile_loop<Claim::Ahead>(g, n_tiles, NoOp(), body);
}

// A tile is kPackBlocks blocks; a thread writes a lane's piece of 16 bytes from
// four runs of eight codes, and the threads past the pieces take the scales.
constexpr int kPackThreads = 256;

template <typename F>
__device__ __forceinline__ void q4_store(const Q4View &v, uint64_t byte, uint32_t &err, F store)
{
    const uint32_t e = checked_page(v.pt, byte >> v.shift, v.pool_pages, err);
    if (e != kBadPage)
        store(const_cast<uint8_t *>(v.pool) + ((uint64_t)e << v.shift) + (byte & ((1ull << v.shift) - 1ull)));
}

__global__ __launch_bounds__(kPackThreads) void k_q4_pack(Q4View v, uint32_t per, const uint8_t *__restrict__ codes,
                                                          uint64_t stride, const uint16_t *__restrict__ scales,
                                                          const uint16_t *__restrict__ zeros, uint64_t n_blocks,
                                                          uint32_t n_tiles, Gate g)
{
    constexpr uint32_t kBlocks = kPackThreads / 64;
    auto body = [&](uint32_t t, uint32_t, uint32_t &err, auto &&) {
        const uint64_t block = (uint64_t)t * kBlocks + (threadIdx.x >> 6);
        const uint32_t lane = threadIdx.x & 63u;
        if (block < n_blocks) {
            const uint64_t tile = block / v.segs;
            const uint32_t seg = (uint32_t)(block % v.segs);
            const uint64_t m = tile * 16u + (lane & 15u);
            u32x4 o;
#pragma unroll
            for (uint32_t i = 0; i < 4u; ++i) {
                const uint32_t k = seg * 128u + i * 32u + (lane >> 4) * 8u;
                uint32_t w = 0u;
                if (m < v.rows && k < v.cols) {
                    const uint8_t *const c = codes + m * stride + k;
#pragma unroll
                    for (uint32_t e = 0; e < 8u; ++e)
                        w |= (uint32_t)(c[e] & 15u) << (4u * (e / 2u + 4u * (e % 2u)));
                }
                o[i] = w;
            }
            q4_store(v, block * kQ4Block + lane * 16u, err, [&](uint8_t *p) { *reinterpret_cast<u32x4 *>(p) = o; });
            const uint32_t row = lane / per, grp = lane % per;  // 16 * per scales
            if (row < 16u) {
                const uint64_t mm = tile * 16u + row;
                const uint32_t gg = seg * per + grp, n = v.cols * per / 128u;
                const bool in = mm < v.rows && gg < n;
                const uint64_t at = block * (per * 32u) + (((row / 4u) * per + grp) * 4u + row % 4u) * 2u;
                const uint16_t s = in ? scales[mm * n + gg] : (uint16_t)0;
                q4_store(v, v.scales + at, err, [&](uint8_t *p) { *reinterpret_cast<uint16_t *>(p) = s; });
                if (zeros) {
                    const uint16_t z = in ? zeros[mm * n + gg] : (uint16_t)0;
                    q4_store(v, v.zeros + at, err, [&](uint8_t *p) { *reinterpret_cast<uint16_t *>(p) = z; });
                }
            }
        }
    };
    tile_loop<Claim::Ahead>(g, n_tiles, NoOp(), body);
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
    return SGDRC_OK;
}

static uint64_t q4_blocks(const sgdrc_q4 *q)
{
    return ((uint64_t)q->rows + 15u) / 16u * ((q->cols + 127u) / 128u);
}

static uint64_t q4_scale_bytes(const sgdrc_q4 *q) { return q4_blocks(q) * (128u / q->group) * 32u; }

static Q4View q4_view(const sgdrc_paged *w, const sgdrc_q4 *q, uint32_t page_shift)
{
    const uint64_t s = q4_blocks(q) * kQ4Block;
    return {static_cast<const uint8_t *>(w->pool), w->pt, w->pool_pages, s, s + q4_scale_bytes(q), page_shift,
            q->rows, q->cols, (q->cols + 127u) / 128u};
}

typedef void (*Q4Kernel)(Q4View, const uint8_t *, uint32_t, float *, uint32_t, Gate);

template <int DT, int PER>
static Q4Kernel q4_kernel(const sgdrc_q4 *q)
{
    return q->zeros ? k_gemv_q4<DT, PER, true> : k_gemv_q4<DT, PER, false>;
}

template <int DT>
static Q4Kernel q4_kernel_group(const sgdrc_q4 *q)
{
    return q->group == 128 ? q4_kernel<DT, 1>(q) : q->group == 64 ? q4_kernel<DT, 2>(q) : q4_kernel<DT, 4>(q);
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
    const uint64_t blocks = q4_blocks(q), tiles = (blocks + kPackThreads / 64 - 1) / (kPackThreads / 64);
    if (blocks >= (1ull << 31))
        return set_error(SGDRC_EINVAL, "2^31 blocks or more");
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
                       q4_view(dst, q, page_shift), 128u / q->group, d_codes, code_stride,
                       static_cast<const uint16_t *>(d_scales), static_cast<const uint16_t *>(d_zeros), blocks,
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
    const uint64_t tiles = ((uint64_t)q->rows + 15u) / 16u;
    Gate g;
    LaunchInfo li;
    if ((rc = make_gate(c, stream, tiles, kGemvGroupCus, &g, &li, false, true)))
        return rc;
    const Q4Kernel k = q->dtype == SGDRC_BF16 ? q4_kernel_group<SGDRC_BF16>(q) : q4_kernel_group<SGDRC_F16>(q);
    static const int occ = occupancy(k_gemv_q4<SGDRC_BF16, 4, true>, kQ4Threads);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(k, dim3(gated_grid(c, occ, tiles, li)), dim3(kQ4Threads), 0, s, q4_view(w, q, page_shift),
                       static_cast<const uint8_t *>(d_x), batch, d_y, (uint32_t)tiles, g);
    SGDRC_HIP(hipGetLastError());
    return finish_static_tlog(g, s);
}

}  // extern "C"
