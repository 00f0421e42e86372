// Products of FP8 operands with an FP32 scale per block of 128 along the inner dimension (the per-group scheme of the systems that
// MOSS is compared with, paper Sec. 1 and 3.1):
//      out[m, n] (+)= sum_kb a_s[m, kb] b_s[n or n / 128, kb] sum_{k in kb} dec(a[m, k]) dec(b[n, k]).
// The scales cannot leave the main loop: the sum of every block is taken from zero by the matrix unit and added to the accumulators
// times both scales by the vector unit.  Kernels: the wide tiles (moss_gemm_wide.h) and, where few rows leave them idle and for what they
// cannot take, the small tiles (moss_gemm_mid.h); a stage is one block in both.
//
// Bound, large products: matrix unit and vector unit, which take turns in a stage (moss_gemm_wide.h), and power.  8192 x 11008 x 4096 takes 388 to
// 408 us (1.8 to 1.9 PFLOP/s; 435 to 455 twelve times back to back) on quantized data and 511 on random codes, and neither the waits nor
// the barriers left out shorten it; without the copies it takes 18 % less, without the additions on the vector unit 11 %, without the stores 8 %.
// (The MOSS product of the same size, whose scales the matrix instruction applies: 325 us.)  Few rows: the weight's bytes, 17 x 11008 x
// 4096 10.4 us, 4.4 TB/s.  dW, 4096 x 4096 x 2016: 46 to 49 us into BF16, 52 into FP32, 66 on top of what is there.
#include "moss_gemm_mid.h"
#include "moss_gemm_wide.h"

namespace {

enum BlockKind { kBlockSmall, kBlock64, kBlock128, kBlockHalf, kBlockWide, kBlockSmall64 };

// Fits to 400 random products (M 1 to 16384, N 256 to 11008, K 32 to 8192; a scale per 128 rows of b, or per row), each run in every
// kind of tiles: the kind chosen took 0.5 % (1.0 %) more than the fastest of its problem.  us, a scale per
// 128 rows of b, 32 x 32 / 64 x 128 / 128 x 128 / 128 x 256 / 256 x 256:
//     98 x 3840 x 2944     7.3 / 16.6 / 20.2 / 26.6 / 41.0      512 x 4096 x 4096    31.5 / 23.3 / 27.4 / 36.6 / 57.5
//     1086 x 640 x 640     7.4 /  7.4 /  8.6 / 10.7 / 15.6      651 x 4032 x 1216    26.3 / 17.9 / 13.2 / 16.7 / 24.8
//     4553 x 1792 x 2048  80.1 / 45.3 / 31.7 / 26.1 / 36.4      8192 x 11008 x 4096    - /  970 /  618 /  477 /  418
// and per row: 384 x 1664 x 6688 28.2 / 36.5 / 47.4 / 73.1 / 120, 1280 x 2048 x 2944 35.7 / 34.4 / 25.5 / 34.3 / 52.2,
// 4096 x 4096 x 2016 202 / 93.3 / 66.9 / 57.9 / 51.1.
constexpr MossTileCost kCost[2][5] = {{{2.2, 0.73, 0.52, 0.89, 0.12, 32, 32, 4, 2, false},
                                       {4.0, 0.18, 0.53, 1.43, 0.04, 64, 128, 1, 1, true},
                                       {4.5, 0.0, 0.67, 2.19, 0.02, 128, 128, 1, 1, true},
                                       {4.8, 0.0, 0.95, 4.36, 0.03, 128, 256, 1, 1, true},
                                       {5.7, 0.0, 1.56, 8.5, 0.04, 256, 256, 1, 1, true}},
                                      {{2.5, 0.0, 0.78, 1.07, 0.21, 32, 32, 4, 2, false},
                                       {3.6, 0.87, 0.57, 1.03, 0.02, 64, 128, 1, 1, true},
                                       {3.8, 0.99, 0.79, 1.82, 0.01, 128, 128, 1, 1, true},
                                       {4.3, 1.14, 1.19, 3.26, 0.03, 128, 256, 1, 1, true},
                                       {7.3, 0.0, 1.9, 6.9, 0.04, 256, 256, 1, 1, true}}};

// What the wide tiles cannot take (K below a stage, pieces of 16 bytes that end inside a row of the output) goes to small tiles of 32 x 32, K
// split over their waves, or of 64 x 64.  us: 512 x 1001 x 1024 5.5 / 8.6, 1152 x 3968 x 32 27.6 / 12.0, 8192 x 4096 x 64 175 / 56,
// 2048 x 1001 x 4096 33.2 / 25.1, 4096 x 4100 x 1024 122 / 60.
constexpr MossTileCost kCostSmall64 = {4.0, 0.8, 0.31, 0.3, 0.0, 64, 64, 1, 1, false};

double tiles_us(const MossTileCost &c, int64_t M, int64_t N, int64_t K)
{
    return moss_tile_us(c, (double)moss_ceil_div(M, c.bm) * (double)moss_ceil_div(N, c.bn), (double)moss_ceil_div(K, 128 * c.k_groups), K % 128 != 0);
}

int block_kind(int64_t M, int64_t N, int64_t K, int64_t b_block, int64_t ld_out)
{
    if (K < 128 || N % 8 || ld_out % 8) return tiles_us(kCostSmall64, M, N, K) < tiles_us(kCost[0][kBlockSmall], M, N, K) ? kBlockSmall64 : kBlockSmall;
    int best = 0;
    double least = 0.0;
    for (int k = 0; k < 5; k++) {
        const double us = tiles_us(kCost[b_block == 1][k], M, N, K);
        if (k == 0 || us < least) {
            best = k;
            least = us;
        }
    }
    return best;
}

template <moss::WideForm FORM>
int launch_block(int kind, const moss::WideArgs &p, hipStream_t st)
{
    switch (kind) {
        case kBlock64: return moss::launch_wide<FORM, 2, 2, 5>(p, st);
        case kBlock128: return moss::launch_wide<FORM, 4, 2, 4>(p, st);
        case kBlockHalf: return moss::launch_wide<FORM, 4, 4, 3>(p, st);
        default: return moss::launch_wide<FORM, 8, 4, 2>(p, st);
    }
}

}  // namespace

// The tile (rows * 1000 + columns) that a product takes (the tests hold the choice by it)
extern "C" int moss_internal_gemm_block_tile(int64_t M, int64_t N, int64_t K, int64_t b_block, int64_t ld_out)
{
    const int k = block_kind(M, N, K, b_block, ld_out);
    const MossTileCost &c = k == kBlockSmall64 ? kCostSmall64 : kCost[0][k];
    return c.bm * 1000 + c.bn;
}

extern "C" int moss_gemm_fp8_block128(int64_t M, int64_t N, int64_t K, const uint8_t *a_q, const float *a_s, const uint8_t *b_q,
                                      const float *b_s, int64_t b_block, void *out, int out_dtype, int64_t ld_out, int accumulate, void *stream)
{
    using namespace moss;
    if (!a_q || !a_s || !b_q || !b_s || !out) return MOSS_ERR_NULL;
    if (M <= 0 || N <= 0 || K <= 0 || K % 32 || ld_out < N) return MOSS_ERR_SHAPE;
    if (b_block != 1 && b_block != 128) return MOSS_ERR_UNSUPPORTED;
    if (out_dtype != MOSS_DT_BF16 && out_dtype != MOSS_DT_F32) return MOSS_ERR_UNSUPPORTED;
    if (accumulate && out_dtype != MOSS_DT_F32) return MOSS_ERR_UNSUPPORTED;
    if (!moss_aligned16(a_q) || !moss_aligned16(b_q) || !moss_aligned16(out) || ((uintptr_t)a_s & 3) || ((uintptr_t)b_s & 3)) return MOSS_ERR_ALIGN;
    if (K > ((int64_t)1 << 22)) return MOSS_ERR_UNSUPPORTED;      // 32-bit offsets inside a tile
    hipStream_t st = (hipStream_t)stream;
    const int64_t blocks = (K + 127) / 128;
    const int kind = block_kind(M, N, K, b_block, ld_out);
    if (kind != kBlockSmall && kind != kBlockSmall64) {
        WideArgs p{};
        p.M = M; p.N = N; p.K = K;
        p.a_q = a_q; p.b_q = b_q;
        p.a_x = (const uint8_t *)a_s; p.b_x = (const uint8_t *)b_s;
        p.pitch_a = p.pitch_b = 4 * blocks;
        p.end_a = M * 4 * blocks;
        p.end_b = (N + b_block - 1) / b_block * 4 * blocks;
        p.ld_b = K;
        p.out = out; p.ld_out = ld_out; p.out_f32 = out_dtype == MOSS_DT_F32; p.accumulate = accumulate;
        const int rc = b_block == 1 ? launch_block<kWideBlockRows>(kind, p, st) : launch_block<kWideBlock>(kind, p, st);
        if (rc != MOSS_ERR_UNSUPPORTED) return rc;
    }
    MidArgs p{};
    p.M = M; p.N = N; p.K = K;
    p.a_q = a_q; p.a_e = (const uint8_t *)a_s;
    p.b_q = b_q; p.b_e = (const uint8_t *)b_s;
    p.out = out; p.ld_out = ld_out; p.out_f32 = out_dtype == MOSS_DT_F32; p.accumulate = accumulate;
    p.e_dwords = 1;
    if (kind == kBlockSmall64) return b_block == 1 ? launch_mid_kind<kMidBlockRows, 5>(p, st) : launch_mid_kind<kMidBlock, 5>(p, st);
    return b_block == 1 ? launch_mid_kind<kMidBlockRows, 0>(p, st) : launch_mid_kind<kMidBlock, 0>(p, st);
}
