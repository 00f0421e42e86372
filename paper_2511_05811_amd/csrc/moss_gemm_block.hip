// Products of FP8 operands with an FP32 scale per block of 128 along the inner dimension (the per-group scheme of the systems that
// MOSS is compared with, paper Sec. 1 and 3.1):
//      out[m, n] (+)= sum_kb a_s[m, kb] b_s[n or n / 128, kb] sum_{k in kb} dec(a[m, k]) dec(b[n, k]).
// The scales cannot leave the main loop: the sum of every block is taken from zero by the matrix unit and added to the accumulators
// times both scales by the vector unit.  Kernel: the small tiles, whose stage is one block (moss_gemm_mid.h).
#include "moss_gemm_mid.h"
#include "moss_gemm_wide.h"

namespace {

enum BlockKind { kBlockSmall, kBlock64, kBlock128, kBlockHalf, kBlockWide };

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

int moss_block_kind(int64_t M, int64_t N, int64_t K, bool, int64_t ld_out)
{
    if (K < 128 || N % 8 || ld_out % 8) return kBlockSmall;
    if (M * N < 512 * 512) return kBlockSmall;
    return M * N >= 2048 * 4096 ? kBlockWide : kBlockHalf;
}

}  // namespace

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
    const int kind = moss_block_kind(M, N, K, out_dtype == MOSS_DT_F32, ld_out);
    if (kind != kBlockSmall) {
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
    return b_block == 1 ? launch_mid_kind<kMidBlockRows>(0, p, st) : launch_mid_kind<kMidBlock>(0, p, st);
}
