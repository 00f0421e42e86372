// Quantizers of the recipe with one FP32 scale per block of 128 elements (paper Sec. 1 and 3.1: the per-group scheme of the
// systems that MOSS is compared with): activations and gradients in groups of 128 along the columns and / or along the rows,
// weights in blocks of 128 x 128.  For every group or block
//      s = amax / 448 (1 if all are zero),   codes = rne_e4m3(x * fl32(1 / s)), at most 448 in magnitude,
// the reciprocal capped at FLT_MAX.  No maximum of the whole tensor, so every input is read once and nothing waits.
//
// Bound: HBM.  A workgroup holds 128 x 128 elements in registers: 16 lanes side by side in a row (8 columns each), every thread in
// 8 rows that follow each other.  A row's maximum is then four shuffles away, a column's eight rows are the thread's own, two more
// shuffles and one trip through LDS join the 16 threads of a column.  The transposed codes come out of the converter in
// transposed order (four rows of a column at a time), meet in LDS in 8-byte pieces swizzled by column and leave as whole lines.
// Row groups alone need no tile: 16 lanes per group, wherever it lies.
//
// 8192 x 4096, rows / columns / both: 18.3 / 21.8 / 30.5 us (5.5 / 4.7 / 4.5 TB/s; a large copy 5.0); 8192 x 11008 both 75.6 (4.8); an FP32
// weight of 11008 x 4096 with its transposed codes 55.4 (4.9), without 42.6 (5.3), a BF16 weight 36.9 (4.9) and 24.7 (5.5).  With two IEEE divisions per row and per column, shuffles through LDS and
// a clamp per value, which the memory does not hide in so short a kernel, both took 36.4 and 81.4.
#include <type_traits>

#include "moss_internal.h"

namespace moss {
namespace {

constexpr int kBqThreads = 256;
constexpr int kBqTile = 128;

typedef unsigned short bq_u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t bq_pk_max(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(bq_u16x2, a), __builtin_bit_cast(bq_u16x2, b)));
}
__device__ __forceinline__ float bq_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bq_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ __forceinline__ float block_scale(float amax) { return amax > 0.0f ? amax / kE4M3Max : 1.0f; }
__device__ __forceinline__ float block_reciprocal(float s) { return fminf(1.0f / s, 3.402823466e38f); }

// The same of N maxima of BF16 magnitudes at once.  Between 2^-90 and 2^90 a product and two fused steps give the quotient, and the
// approximate reciprocal with two fused steps its reciprocal, rounded as the divisions round them (all 128 mantissas have been compared);
// a wave that has others divides.
template <int N>
__device__ __forceinline__ void block_scales_of(const float (&amax)[N], float (&s)[N], float (&inv)[N])
{
    constexpr uint32_t kLow = (127u - 90u) << 23, kHigh = (127u + 90u) << 23;
    bool unusual = false;
#pragma unroll
    for (int i = 0; i < N; i++) {
        const float c = 1.0f / kE4M3Max, q = amax[i] * c;
        const float t = __builtin_fmaf(__builtin_fmaf(-kE4M3Max, q, amax[i]), c, q);
        s[i] = amax[i] > 0.0f ? t : 1.0f;
        const float r = __builtin_amdgcn_rcpf(s[i]);
        inv[i] = __builtin_fmaf(__builtin_fmaf(-s[i], r, 1.0f), r, r);
        unusual |= amax[i] != 0.0f && __float_as_uint(amax[i]) - kLow > kHigh - kLow;
    }
    if (__any(unusual))
#pragma unroll
        for (int i = 0; i < N; i++) {
            s[i] = block_scale(amax[i]);
            inv[i] = block_reciprocal(s[i]);
        }
}

// Eight neighbours of a row, as they come: four words of BF16 pairs or eight FP32 words
template <bool F32> struct Chunk {
    uint32_t w[F32 ? 8 : 4];
    __device__ __forceinline__ float at(int c) const { return F32 ? __uint_as_float(w[F32 ? c : 0]) : (c & 1) ? bq_hi(w[c >> 1]) : bq_lo(w[c >> 1]); }
};

template <bool F32>
__device__ __forceinline__ Chunk<F32> load_chunk(const void *x, int64_t at)
{
    Chunk<F32> r;
    const uint4 a = ld_stream16((const uint8_t *)x + at * (F32 ? 4 : 2));
    r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w;
    if (F32) {
        const uint4 b = ld_stream16((const uint8_t *)x + at * 4 + 16);
        r.w[F32 ? 4 : 0] = b.x; r.w[F32 ? 5 : 0] = b.y; r.w[F32 ? 6 : 0] = b.z; r.w[F32 ? 7 : 0] = b.w;
    }
    return r;
}

// Maxima of magnitudes as words: pairs of BF16 magnitudes, or FP32 magnitudes (whose order is that of their bits)
template <bool F32> struct Top {
    uint32_t w[F32 ? 8 : 4];
};
template <bool F32>
__device__ __forceinline__ void take(Top<F32> &m, const Chunk<F32> &x)
{
#pragma unroll
    for (int i = 0; i < (F32 ? 8 : 4); i++) {
        if (F32) { const uint32_t a = x.w[i] & 0x7FFFFFFFu; m.w[i] = a > m.w[i] ? a : m.w[i]; }
        else m.w[i] = bq_pk_max(m.w[i], x.w[i] & 0x7FFF7FFFu);
    }
}
// of all eight, as a float
template <bool F32>
__device__ __forceinline__ float top_of(const Top<F32> &m)
{
    uint32_t t = m.w[0];
#pragma unroll
    for (int i = 1; i < (F32 ? 8 : 4); i++) t = F32 ? (m.w[i] > t ? m.w[i] : t) : bq_pk_max(t, m.w[i]);
    if (F32) return __uint_as_float(t);
    return fmaxf(bq_lo(t), bq_hi(t));
}
// (of magnitudes, whose order is that of their bits; rotated inside a row of 16 lanes)
__device__ __forceinline__ float max_of_16_lanes(float magnitude)
{
    uint32_t m = __float_as_uint(magnitude);
    auto rotated = [&](auto by) {
        const uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x120 + decltype(by)::value, 0xF, 0xF, true);
        m = o > m ? o : m;
    };
    rotated(std::integral_constant<int, 8>{});
    rotated(std::integral_constant<int, 4>{});
    rotated(std::integral_constant<int, 2>{});
    rotated(std::integral_constant<int, 1>{});
    return __uint_as_float(m);
}

// Four codes.  The converter itself saturates at +-448 in waves that have set the mode bit for it (FP16_OVFL, which nothing else here
// looks at): one instruction per value less than a clamp ahead of it.
__device__ __forceinline__ void converter_saturates()
{
    __builtin_amdgcn_s_setreg((1 - 1) << 11 | 23 << 6 | 1, 1);   // hwreg(MODE, offset 23, 1 bit) = 1
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d)
{
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

template <bool F32>
__device__ __forceinline__ uint2 row_codes(const Chunk<F32> &x, float inv)
{
    return make_uint2(codes4(x.at(0) * inv, x.at(1) * inv, x.at(2) * inv, x.at(3) * inv),
                      codes4(x.at(4) * inv, x.at(5) * inv, x.at(6) * inv, x.at(7) * inv));
}

// Row groups alone: 16 lanes per group, kDeep groups of a lane in flight
constexpr int kDeep = 4;
__global__ __launch_bounds__(kBqThreads) void k_block128_rows(const uint16_t *__restrict__ x, uint32_t groups, uint32_t per_row, int cols,
                                                              int64_t ld, uint8_t *__restrict__ q, float *__restrict__ s)
{
    converter_saturates();
    const int sub = threadIdx.x & 15;
    const uint32_t step = gridDim.x * (kBqThreads / 16);
    for (uint32_t g0 = blockIdx.x * (kBqThreads / 16) + (threadIdx.x >> 4); g0 < groups; g0 += step * kDeep) {
        Chunk<false> v[kDeep];
        int64_t row[kDeep];
        int col[kDeep];
        bool there[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; u++) {
            const uint32_t g = g0 + u * step;
            row[u] = g / per_row;
            col[u] = (int)(g % per_row) * 128 + sub * 8;
            there[u] = g < groups && g >= g0 && col[u] < cols;
            v[u] = Chunk<false>{};
            if (there[u]) v[u] = load_chunk<false>(x, row[u] * ld + col[u]);
        }
        float amax[kDeep], scale[kDeep], inv[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; u++) {
            Top<false> m{};
            take(m, v[u]);
            amax[u] = max_of_16_lanes(top_of(m));
        }
        block_scales_of(amax, scale, inv);
#pragma unroll
        for (int u = 0; u < kDeep; u++) {
            if (!there[u]) continue;
            st_stream8(q + row[u] * cols + col[u], row_codes(v[u], inv[u]));
            if (sub == 0) s[row[u] * per_row + col[u] / 128] = scale[u];
        }
    }
}

// 128 x 128 elements.  BLOCK: one scale for all of them (weights), else one per row (ROW) and / or per column (COL).
// ROW: codes as the elements lie.  COL: transposed codes.
template <bool F32, bool ROW, bool COL, bool BLOCK>             // (F32 only with BLOCK)
__global__ __launch_bounds__(kBqThreads) void k_block128_tile(const void *__restrict__ x, int64_t rows, int64_t cols, int64_t ld, uint32_t tiles_c,
                                                              uint8_t *__restrict__ q_row, float *__restrict__ s_row,
                                                              uint8_t *__restrict__ q_col, float *__restrict__ s_col)
{
    __shared__ float red[BLOCK ? 4 : 4 * kBqTile];               // per wave: its maximum, or those of the columns
    __shared__ __attribute__((aligned(16))) uint8_t turned[COL ? kBqTile * kBqTile : 16];
    converter_saturates();
    const uint32_t tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
    const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4, wave = threadIdx.x >> 6;
    const int64_t r0 = (int64_t)tr * kBqTile + rg * 8, c0 = (int64_t)tc * kBqTile + cg * 8;
    const int64_t tiles_r = (rows + kBqTile - 1) / kBqTile;

    Chunk<F32> v[8];
    Top<F32> m{};
#pragma unroll
    for (int i = 0; i < 8; i++) {
        v[i] = Chunk<F32>{};
        if (c0 < cols && r0 + i < rows) v[i] = load_chunk<F32>(x, (r0 + i) * ld + c0);
    }
    if (BLOCK || COL)
#pragma unroll
        for (int i = 0; i < 8; i++) take(m, v[i]);

    float inv_col[8];
    if (BLOCK) {
        float t = wave_max_f32(top_of(m));
        if ((threadIdx.x & 63) == 0) red[wave] = t;
        __syncthreads();
        t = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
        const float s = block_scale(t), inv = block_reciprocal(s);
        if (threadIdx.x == 0) {
            if (ROW) s_row[(int64_t)tr * tiles_c + tc] = s;
            if (COL) s_col[(int64_t)tc * tiles_r + tr] = s;
        }
#pragma unroll
        for (int c = 0; c < 8; c++) inv_col[c] = inv;
    } else if (COL) {
        float t[8];
#pragma unroll
        for (int c = 0; c < 8; c++) {
            t[c] = F32 ? __uint_as_float(m.w[F32 ? c : 0]) : (c & 1) ? bq_hi(m.w[c >> 1]) : bq_lo(m.w[c >> 1]);
            t[c] = fmaxf(t[c], __shfl_xor(t[c], 16, 64));
            t[c] = fmaxf(t[c], __shfl_xor(t[c], 32, 64));
        }
        if ((threadIdx.x & 63) < 16)
#pragma unroll
            for (int c = 0; c < 8; c++) red[wave * kBqTile + cg * 8 + c] = t[c];
        __syncthreads();
        float s[8];
#pragma unroll
        for (int c = 0; c < 8; c++) {
            const int at = cg * 8 + c;
            t[c] = fmaxf(fmaxf(red[at], red[kBqTile + at]), fmaxf(red[2 * kBqTile + at], red[3 * kBqTile + at]));
        }
        block_scales_of(t, s, inv_col);
        if (rg == 0)
#pragma unroll
            for (int c = 0; c < 8; c++)
                if (c0 + c < cols) s_col[(c0 + c) * tiles_r + tr] = s[c];
    }
    if (ROW) {
        float s[8], inv[8];
        if (!BLOCK) {
            float amax[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                Top<F32> own{};
                take(own, v[i]);
                amax[i] = max_of_16_lanes(top_of(own));
            }
            block_scales_of(amax, s, inv);
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (r0 + i >= rows) continue;
            if (!BLOCK && cg == 0) s_row[(r0 + i) * tiles_c + tc] = s[i];
            if (c0 < cols) st_stream8(q_row + (r0 + i) * cols + c0, row_codes(v[i], BLOCK ? inv_col[0] : inv[i]));
        }
    }
    if (COL) {
        // eight rows of a column are one 8-byte piece; piece rg of column c lies at place rg ^ cg of its 128 bytes
#pragma unroll
        for (int c = 0; c < 8; c++) {
            const float f = inv_col[c];
            const uint2 w = make_uint2(codes4(v[0].at(c) * f, v[1].at(c) * f, v[2].at(c) * f, v[3].at(c) * f),
                                       codes4(v[4].at(c) * f, v[5].at(c) * f, v[6].at(c) * f, v[7].at(c) * f));
            *reinterpret_cast<uint2 *>(turned + (cg * 8 + c) * kBqTile + ((rg ^ cg) << 3)) = w;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const int col = k * 32 + (threadIdx.x >> 3), u = threadIdx.x & 7, g = col >> 3;
            const uint4 w = *reinterpret_cast<const uint4 *>(turned + col * kBqTile + ((u ^ (g >> 1)) << 4));
            const int64_t c = (int64_t)tc * kBqTile + col, r = (int64_t)tr * kBqTile + u * 16;
            if (c < cols && r < rows) st_stream16(q_col + c * rows + r, (g & 1) ? make_uint4(w.z, w.w, w.x, w.y) : w);
        }
    }
}

template <bool F32, bool ROW, bool COL, bool BLOCK>
int launch_tile(const void *x, int64_t rows, int64_t cols, int64_t ld, uint8_t *q_row, float *s_row, uint8_t *q_col, float *s_col, hipStream_t st)
{
    const int64_t tiles_c = (cols + kBqTile - 1) / kBqTile, tiles = (rows + kBqTile - 1) / kBqTile * tiles_c;
    if (tiles > 0x7FFFFFFF) return MOSS_ERR_SHAPE;
    hipLaunchKernelGGL((k_block128_tile<F32, ROW, COL, BLOCK>), dim3((unsigned)tiles), dim3(kBqThreads), 0, st, x, rows, cols, ld, (uint32_t)tiles_c, q_row,
                       s_row, q_col, s_col);
    MOSS_LAUNCH_CHECK();
    return MOSS_OK;
}

}  // namespace
}  // namespace moss

extern "C" int moss_quant_block128(const void *x_bf16, int64_t rows, int64_t cols, int64_t ld, unsigned flags, uint8_t *q_row, float *s_row,
                                   uint8_t *q_col, float *s_col, void *stream)
{
    using namespace moss;
    const bool row = flags & MOSS_Q_ROW, col = flags & MOSS_Q_COL;
    if ((flags & ~(MOSS_Q_ROW | MOSS_Q_COL)) || !(row || col)) return MOSS_ERR_UNSUPPORTED;
    if (!x_bf16 || (row && (!q_row || !s_row)) || (col && (!q_col || !s_col))) return MOSS_ERR_NULL;
    if (rows <= 0 || cols <= 0 || cols % 32 || (col && rows % 32) || ld < cols || cols > 0x7FFFFFFF) return MOSS_ERR_SHAPE;
    if (ld % 8 || !moss_aligned16(x_bf16)) return MOSS_ERR_ALIGN;
    if (row && (!moss_aligned16(q_row) || ((uintptr_t)s_row & 3))) return MOSS_ERR_ALIGN;
    if (col && (!moss_aligned16(q_col) || ((uintptr_t)s_col & 3))) return MOSS_ERR_ALIGN;
    hipStream_t st = (hipStream_t)stream;
    if (col) {
        const auto launch = row ? launch_tile<false, true, true, false> : launch_tile<false, false, true, false>;
        return launch(x_bf16, rows, cols, ld, q_row, s_row, q_col, s_col, st);
    }
    const int64_t per_row = (cols + 127) / 128, groups = rows * per_row;
    if (groups > 0x7FFFFFFF) return MOSS_ERR_SHAPE;
    int64_t cus = moss_internal_cu_count();
    if (cus <= 0) cus = 256;
    const int64_t per_wg = kBqThreads / 16, most = cus * 8;
    const int64_t wgs = (groups + per_wg - 1) / per_wg;
    hipLaunchKernelGGL(k_block128_rows, dim3((unsigned)(wgs < most ? wgs : most)), dim3(kBqThreads), 0, st, (const uint16_t *)x_bf16,
                       (uint32_t)groups, (uint32_t)per_row, (int)cols, ld, q_row, s_row);
    MOSS_LAUNCH_CHECK();
    return MOSS_OK;
}

extern "C" int moss_quant_block128_weight(const void *w, int w_dtype, int64_t rows, int64_t cols, uint8_t *wq, float *s, uint8_t *wq_t,
                                          float *s_t, void *stream)
{
    using namespace moss;
    if (!w || !wq || !s || (wq_t && !s_t)) return MOSS_ERR_NULL;
    if (w_dtype != MOSS_DT_BF16 && w_dtype != MOSS_DT_F32) return MOSS_ERR_UNSUPPORTED;
    if (rows <= 0 || cols <= 0 || cols % 32 || (wq_t && rows % 32)) return MOSS_ERR_SHAPE;
    if (!moss_aligned16(w) || !moss_aligned16(wq) || ((uintptr_t)s & 3)) return MOSS_ERR_ALIGN;
    if (wq_t && (!moss_aligned16(wq_t) || ((uintptr_t)s_t & 3))) return MOSS_ERR_ALIGN;
    const auto launch = w_dtype == MOSS_DT_F32 ? (wq_t ? launch_tile<true, true, true, true> : launch_tile<true, true, false, true>)
                                               : (wq_t ? launch_tile<false, true, true, true> : launch_tile<false, true, false, true>);
    return launch(w, rows, cols, cols, wq, s, wq_t, s_t, (hipStream_t)stream);
}
