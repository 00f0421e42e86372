// The products of a layer of experts on block-scaled FP8 matrix instructions (paper Sec. 3.1, Fig. 3b), rows grouped by expert:
//   rows   out[r, n] = a_s b_s[g] sum_k a[r, k] 2^(a_e) b[g][n, k]                  for r in group g   (forward, dX)
//   dW     out[g][m, n] = a_s b_s sum_{r in g} a[m, r] 2^(a_e) b[n, r] 2^(b_e)
// How many rows a group has stands in device memory only.  The grid is made for the most tiles that there can be; a workgroup finds its
// tile, or that there is none for it, from the offsets.  Kernel: the small tiles (moss_gemm_mid.h).
#include "moss_gemm_mid.h"
#include "moss_gemm_wide.h"

namespace {

constexpr int64_t kMaxGroups = 1024, kMaxLd = (int64_t)1 << 24;      // (32-bit offsets inside a tile)

int check_common(int64_t rows, int64_t groups, const int32_t *offsets, int out_dtype, int accumulate)
{
    if (rows <= 0 || rows > 0x7FFFFFFF || groups <= 0) return MOSS_ERR_SHAPE;
    if (groups > kMaxGroups) return MOSS_ERR_UNSUPPORTED;
    if (out_dtype != MOSS_DT_BF16 && out_dtype != MOSS_DT_F32) return MOSS_ERR_UNSUPPORTED;
    if (accumulate && out_dtype != MOSS_DT_F32) return MOSS_ERR_UNSUPPORTED;
    return ((uintptr_t)offsets & 3) ? MOSS_ERR_ALIGN : MOSS_OK;
}

// Tiles: 0 .. 4 the small ones, then 128 x 256 and 256 x 256 of the wide kernel and of the large-tile kernel
enum { kHalf = 5, kWide = 6, kLargeHalf = 7, kLarge = 8 };

int rows_kind(int64_t rows, int64_t N, int64_t K, int64_t groups, const uint8_t *a_e, int64_t ld_out)
{
    const int64_t avg = (rows + groups - 1) / groups;
    if (!a_e || K < 128 || N % 8 || ld_out % 8 || avg <= 128) return avg <= 32 ? 0 : avg <= 64 ? 1 : avg <= 128 ? 2 : 3;
    if (moss_internal_gemm_big_groups_ok(N, K, a_e, ld_out)) return avg <= 256 ? kLargeHalf : kLarge;
    return avg <= 256 ? kHalf : kWide;
}

int dw_kind(int64_t rows, int64_t M, int64_t N, int64_t groups)
{
    (void)groups;
    if (rows < 128 || N % 8) return 3;
    return M * N >= 1024 * 1024 ? kWide : kHalf;
}

}  // namespace

extern "C" int moss_gemm_fp8_mx_grouped(int64_t rows, int64_t N, int64_t K, int64_t groups, const int32_t *offsets, const uint8_t *a_q,
                                        const uint8_t *a_e, const float *a_s, const uint8_t *b_q, int64_t ld_b, int64_t b_stride,
                                        const float *b_s, int64_t b_s_stride, void *out, int out_dtype, int64_t ld_out, int accumulate,
                                        void *stream)
{
    using namespace moss;
    if (!offsets || !a_q || !a_s || !b_q || !b_s || !out) return MOSS_ERR_NULL;
    if (N <= 0 || K <= 0 || K % kGroup || ld_out < N || ld_b < K || b_stride < 0 || b_s_stride < 0) return MOSS_ERR_SHAPE;
    const int rc = check_common(rows, groups, offsets, out_dtype, accumulate);
    if (rc) return rc;
    if (K > ((int64_t)1 << 22) || ld_b > kMaxLd) return MOSS_ERR_UNSUPPORTED;
    if (!moss_aligned16(a_q) || !moss_aligned16(b_q) || !moss_aligned16(out) || ld_b % 16 || b_stride % 16) return MOSS_ERR_ALIGN;
    if (((uintptr_t)a_e & 3) || ((uintptr_t)a_s & 3) || ((uintptr_t)b_s & 3)) return MOSS_ERR_ALIGN;
    hipStream_t st = (hipStream_t)stream;
    const int kind = rows_kind(rows, N, K, groups, a_e, ld_out);
    if (kind >= kLargeHalf) {
        const int rc = moss_internal_gemm_big_groups(kind == kLargeHalf, rows, N, K, groups, offsets, a_q, a_e, a_s, b_q, ld_b, b_stride, b_s, b_s_stride,
                                                     out, out_dtype == MOSS_DT_F32, ld_out, accumulate, st);
        if (rc != MOSS_ERR_UNSUPPORTED) return rc;
    }
    if (kind >= kHalf) {
        WideArgs p{};
        p.M = rows; p.N = N; p.K = K;
        p.a_q = a_q; p.a_x = a_e; p.a_s = a_s;
        p.b_q = b_q; p.b_s = b_s;
        p.pitch_a = K / kGroup;
        p.end_a = rows * p.pitch_a;
        p.ld_b = ld_b; p.b_stride = b_stride; p.b_s_stride = b_s_stride;
        p.offsets = offsets; p.groups = (int)groups;
        p.out = out; p.ld_out = ld_out; p.out_f32 = out_dtype == MOSS_DT_F32; p.accumulate = accumulate;
        const int rc = kind == kWide ? launch_wide<kWideGroupRows, 8, 4, 2>(p, st) : launch_wide<kWideGroupRows, 4, 4, 3>(p, st);
        if (rc != MOSS_ERR_UNSUPPORTED) return rc;
    }
    MidGroupArgs p{};
    p.M = rows; p.N = N; p.K = K;
    p.a_q = a_q; p.a_e = a_e; p.a_s = a_s;
    p.b_q = b_q; p.b_s = b_s;
    p.out = out; p.ld_out = ld_out; p.out_f32 = out_dtype == MOSS_DT_F32; p.accumulate = accumulate;
    p.e_dwords = K % 128 == 0;
    p.offsets = offsets; p.groups = (int)groups; p.rows = rows;
    p.ld_b = ld_b; p.b_stride = b_stride; p.b_s_stride = b_s_stride;
    return launch_mid_kind<kMidGroupRows>(kind >= kHalf ? 3 : kind, p, st);
}

extern "C" int moss_gemm_fp8_mx_grouped_dw(int64_t rows, int64_t M, int64_t N, int64_t groups, const int32_t *offsets, const uint8_t *a_q,
                                           const uint8_t *a_e, const float *a_s, const uint8_t *b_q, const uint8_t *b_e, const float *b_s,
                                           void *out, int out_dtype, int accumulate, void *stream)
{
    using namespace moss;
    if (!offsets || !a_q || !a_e || !a_s || !b_q || !b_e || !b_s || !out) return MOSS_ERR_NULL;
    if (M <= 0 || N <= 0 || rows % kGroup) return MOSS_ERR_SHAPE;
    const int rc = check_common(rows, groups, offsets, out_dtype, accumulate);
    if (rc) return rc;
    if (rows > kMaxLd) return MOSS_ERR_UNSUPPORTED;
    if (!moss_aligned16(a_q) || !moss_aligned16(b_q) || !moss_aligned16(out)) return MOSS_ERR_ALIGN;
    if (((uintptr_t)a_e & 3) || ((uintptr_t)a_s & 3) || ((uintptr_t)b_e & 3) || ((uintptr_t)b_s & 3)) return MOSS_ERR_ALIGN;
    hipStream_t st = (hipStream_t)stream;
    const int kind = dw_kind(rows, M, N, groups);
    if (kind >= kHalf) {
        WideArgs p{};
        p.M = M; p.N = N; p.K = rows;
        p.a_q = a_q; p.a_x = a_e; p.a_s = a_s;
        p.b_q = b_q; p.b_x = b_e; p.b_s = b_s;
        p.pitch_a = p.pitch_b = rows / kGroup;
        p.end_a = M * p.pitch_a;
        p.end_b = N * p.pitch_b;
        p.ld_b = rows;
        p.offsets = offsets; p.groups = (int)groups;
        p.out = out; p.ld_out = N; p.out_f32 = out_dtype == MOSS_DT_F32; p.accumulate = accumulate;
        const int rc = kind == kWide ? launch_wide<kWideGroupDw, 8, 4, 2>(p, st) : launch_wide<kWideGroupDw, 4, 4, 3>(p, st);
        if (rc != MOSS_ERR_UNSUPPORTED) return rc;
    }
    MidGroupArgs p{};
    p.M = M; p.N = N; p.K = rows;
    p.a_q = a_q; p.a_e = a_e; p.a_s = a_s;
    p.b_q = b_q; p.b_e = b_e; p.b_s = b_s;
    p.out = out; p.ld_out = N; p.out_f32 = out_dtype == MOSS_DT_F32; p.accumulate = accumulate;
    p.e_dwords = rows % 128 == 0;
    p.offsets = offsets; p.groups = (int)groups; p.rows = rows;
    return launch_mid_kind<kMidGroupDw>(kind >= kHalf ? 3 : kind, p, st);
}
