// The products of a layer of experts on block-scaled FP8 matrix instructions (paper Sec. 3.1, Fig. 3b), rows grouped by expert:
//   rows   out[r, n] = a_s b_s[g] sum_k a[r, k] 2^(a_e) b[g][n, k]                  for r in group g   (forward, dX)
//   dW     out[g][m, n] = a_s b_s sum_{r in g} a[m, r] 2^(a_e) b[n, r] 2^(b_e)
// How many rows a group has stands in device memory only.  The grid is made for the most tiles that there can be; a workgroup finds its
// tile, or that there is none for it, from the offsets.  Kernels: the small tiles (moss_gemm_mid.h), the wide ones (moss_gemm_wide.h) and
// the large-tile kernel (moss_gemm_big.hip).
//
// Bound: the weights' bytes for few rows (32 rows of 8 experts 11008 x 4096 69 to 71 us, 5.2 TB/s; 76 back to back); the matrix unit and power for
// many (16608 rows of 8 experts 11008 x 4096 667 to 721 us, 2.1 to 2.2 PFLOP/s, 762 to 780 back to back; 4096 x 11008 719; dX from one stacked
// transposed weight, 4096 x 11008 again, 778; K = 4064, which ends inside a stage, 1169 in 128 x 128 tiles); dW lines fetched twice where
// rows begin inside them (8 experts 4096 x 4096 over 16608 rows 357 to 365 us into BF16, 1.5 PFLOP/s, 421 into FP32, 511 on top of what is
// there; over 17280, whose groups begin on lines, 315 into BF16), and latency per tile where sums are short (32 experts of 64 rows 1024 x
// 1024 29 to 31 us into BF16, 42 into FP32, 76 on top of what is there; the outputs' bytes 13, 25, 49).
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

// Kinds of tiles: three of the small ones, two of the wide kernel, two of the large-tile kernel
enum { kSmall32, kSmall64, kSmall128, kWideHalf, kWide, kLargeHalf, kLarge };

// Fits to 350 (rows) and 300 (dW) random layers: 4 to 64 experts, 1 to 16384 assignments as routing deals them out, widths 256 to
// 11008; each run in every kind of tiles.  How many tiles the groups have is known to the device only: half a tile more than
// full ones would be for each group.  The kinds chosen took 4 % (2 %) more than the fastest.  us, rows,
// 32 x 32 / 64 x 128 / 128 x 128 / wide 128 x 256 / large 128 x 256 / large 256 x 256:
//     4 rows, 64 experts 384 x 2432            6.3 / 10.3 / 12.6 / 22.3 / 17.3 / 28.6
//     2688 rows, 4 experts 384 x 640          10.0 /  8.0 /  9.1 / 12.0 /  9.9 / 15.6
//     1024 rows, 8 experts 2560 x 2560        35.6 / 24.6 / 17.6 / 26.9 / 21.0 / 33.1
//     8192 rows, 64 experts 3968 x 384         245 /  103 / 65.8 / 38.5 /    - /    -
//     3697 rows, 32 experts 9344 x 896         384 /  191 /  140 / 95.7 / 78.5 /  114
//     16608 rows, 8 experts 11008 x 4096         - / 1629 / 1139 /  963 /  837 /  714
constexpr MossTileCost kRowsCost[7] = {{2.2, 1.11, 0.61, 0.76, 0.37, 32, 32, 4, 2, false}, {2.2, 2.9, 0.64, 1.91, 0.44, 64, 128, 2, 1, false},
                                       {2.2, 3.48, 0.44, 2.06, 0.46, 128, 128, 1, 1, false}, {5.3, 0.81, 0.91, 3.02, 0.08, 128, 256, 1, 1, true},
                                       {}, {2.8, 2.64, 0.68, 2.01, 0.0, 128, 256, 1, 1, true}, {4.7, 3.13, 1.18, 3.86, 0.0, 256, 256, 1, 1, true}};
// (dW in 128 x 128 / wide 128 x 256 / 256 x 256: 1728 rows of 32 groups 384 x 256 9.5 / 13.3 / 16.6, 8960 of 8 512 x 2048
// 33.4 / 24.6 / 32.2, 2016 of 32 2560 x 1152 138 / 83.8 / 69.1.  Rows of a and b hardly ever begin on lines: all are ragged.)
constexpr MossTileCost kDwCost[7] = {{}, {}, {4.2, 0.04, 1.65, 3.91, 0.0, 128, 128, 1, 1, false}, {7.2, 0.69, 1.41, 4.11, 0.0, 128, 256, 1, 1, true},
                                     {7.3, 1.71, 2.69, 4.81, 0.0, 256, 256, 1, 1, true}, {}, {}};

int rows_kind(int64_t rows, int64_t N, int64_t K, int64_t groups, const uint8_t *a_e, int64_t ld_out)
{
    const bool wide = a_e && K >= 128 && N % 8 == 0 && ld_out % 8 == 0, large = moss_internal_gemm_big_groups_ok(N, K, a_e, ld_out);
    const double some = (double)(groups < rows ? groups : rows);
    int best = 0;
    double least = 0.0;
    for (int k = 0; k < 7; k++) {
        const MossTileCost &c = kRowsCost[k];
        if (!c.bm || (k >= kLargeHalf ? !large : k >= kWideHalf && !wide)) continue;
        const double full = (double)rows / c.bm, tiles_m = full < 1.0 ? some : full + 0.5 * some;
        const double us = moss_tile_us(c, tiles_m * (double)moss_ceil_div(N, c.bn), (double)moss_ceil_div(K, 128 * c.k_groups), K % 128 != 0);
        if (k == 0 || us < least) {
            best = k;
            least = us;
        }
    }
    return best;
}

int dw_kind(int64_t rows, int64_t M, int64_t N, int64_t groups)
{
    int best = kSmall128;
    double least = 0.0;
    for (int k = kSmall128; k <= kWide; k++) {
        const MossTileCost &c = kDwCost[k];
        if (k != kSmall128 && (rows < 128 || N % 8)) continue;
        const double each = (double)rows / (double)groups / 128.0;
        const double us = moss_tile_us(c, (double)groups * (double)moss_ceil_div(M, c.bm) * (double)moss_ceil_div(N, c.bn), each < 1.0 ? 1.0 : each, false);
        if (k == kSmall128 || us < least) {
            best = k;
            least = us;
        }
    }
    return best;
}

// the small tiles as moss_gemm_mid.h numbers them
template <moss::MidForm FORM>
int launch_small(int kind, const moss::MidGroupArgs &p, hipStream_t st)
{
    if constexpr (FORM == moss::kMidGroupRows) {
        const int rc = kind == kSmall32 ? moss::launch_mid_kind<FORM, 0>(p, st) : kind == kSmall64 ? moss::launch_mid_kind<FORM, 2>(p, st) : MOSS_ERR_UNSUPPORTED;
        if (rc != MOSS_ERR_UNSUPPORTED) return rc;           // (there may be too many of them)
    }
    return moss::launch_mid_kind<FORM, 3>(p, st);
}

}  // namespace

// The kinds that calls take (the tests hold the choices by them): the tile (rows * 1000 + columns), the large-tile kernel's with a minus
extern "C" int moss_internal_gemm_grouped_tile(int64_t rows, int64_t N, int64_t K, int64_t groups, int64_t has_a_e, int64_t ld_out)
{
    static const uint8_t some[16] __attribute__((aligned(16))) = {};
    const int k = rows_kind(rows, N, K, groups, has_a_e ? some : nullptr, ld_out);
    return (kRowsCost[k].bm * 1000 + kRowsCost[k].bn) * (k >= kLargeHalf ? -1 : 1);
}
extern "C" int moss_internal_gemm_grouped_dw_tile(int64_t rows, int64_t M, int64_t N, int64_t groups)
{
    const int k = dw_kind(rows, M, N, groups);
    return kDwCost[k].bm * 1000 + kDwCost[k].bn;
}

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
    if (kind == kWideHalf) {
        WideArgs p{};
        p.M = rows; p.N = N; p.K = K;
        p.a_q = a_q; p.a_x = a_e; p.a_s = a_s;
        p.b_q = b_q; p.b_s = b_s;
        p.pitch_a = K / kGroup;
        p.end_a = rows * p.pitch_a;
        p.ld_b = ld_b; p.b_stride = b_stride; p.b_s_stride = b_s_stride;
        p.offsets = offsets; p.groups = (int)groups;
        p.out = out; p.ld_out = ld_out; p.out_f32 = out_dtype == MOSS_DT_F32; p.accumulate = accumulate;
        const int rc = launch_wide<kWideGroupRows, 4, 4, 3>(p, st);
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
    return launch_small<kMidGroupRows>(kind, p, st);
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
    if (kind >= kWideHalf) {
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
    return launch_small<kMidGroupDw>(kind, p, st);
}
