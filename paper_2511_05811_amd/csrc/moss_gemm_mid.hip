// The choice between the small tiles (moss_gemm_mid.h) and the other kernels of moss_gemm_fp8_mx, and their launch.
#include <cmath>

#include "moss_gemm_mid.h"

// Time of a problem in the kernels that could take it, in microseconds: a launch, then per round of tiles over the compute
// units a fixed part (first latency, exponents, epilogue) and a part per iteration (stages of K = 128, dealt over the K groups
// of a tile), each with a share that grows with how full the rounds are.  The constants are fits to 2200 random problems (M 32 to
// 12000, N 256 to 12288, K 128 to 12288; calls back to back on two sets of operands, 256 compute units), each run in every
// kernel that can take it; the fits missed by 2 to 7 % (mean), 10 % at the 10th and 90th percentile.  K % 128 != 0: the rows no longer start on lines and
// the exponents are cut out of two dwords, so that a stage costs more.  "b" marks exponents of b, whose outputs are FP32.
// The fits are from before tiles of 64 x 128 and more, and FP32 outputs of the large ones, stored from the registers: a round of
// these takes up to 3 us less by now, of the large ones up to 5.  What the kernels take now:
//   tile        (M, N, K) measured / model
//   32 x 32     (256, 1024, 1024) 4.4 / 4.5    (17, 11008, 4096) 10.0 / 10.1
//   64 x 64     (1024, 1024, 1024) 6.3 / 7.0   (256, 4096, 4096) 12.0 / 12.3
//   64 x 128    (512, 4096, 1024) 7.8 / 8.9    (512, 4096, 4096) 14.7 / 16.3
//   128 x 128   (2048, 2048, 1024) 10.0 / 12.1 (2048, 2048, 4096) 22.6 / 24.0
//   128 x 192   (2048, 3072, 1024) 12.5 / 15.5 (2048, 3072, 7168) 43.4 / 44.6
//   large       (2048, 4096, 2048) 19.7 / 18.9 (4096, 4096, 4096) 60 / 58      (4096, 4096, 512) b 23.7 / 28.1
//   ... ragged  (11328, 3520, 2080) 105 / 105  (1336, 4096, 4128) 40.9 / 36.4  (2432, 6016, 2656) b 56.0 / 57.3
//   general     (4096, 4096, 2080) 66 / 62     (6321, 2424, 32) 14.8 / 15.9    (2528, 2912, 8032) b 128 / 131
namespace {

double rounds_of(double tiles, double cus) { return tiles <= cus ? 1.0 : std::ceil(tiles / cus); }
double tiles_of(int64_t M, int64_t N, int bm, int bn) { return (double)((M + bm - 1) / bm) * (double)((N + bn - 1) / bn); }

struct Cost {
    double round, round_full, it, it_full;      // per round, and per iteration in a round; their part that goes with its fill
};

double us_of(const Cost &c, double tiles, double cus, double iterations, double per_round = 0.0)
{
    const double n = rounds_of(tiles, cus), u = tiles / (n * cus);
    return 2.2 + n * (c.round + per_round + c.round_full * u + iterations * (c.it + c.it_full * u));
}

struct MidPlan {
    int kind;        // 0 .. 4: the tiles above, smallest first
    double us;
};

MidPlan plan_mid(int64_t M, int64_t N, int64_t K, bool b_exponents, bool accumulate, bool large_ok, double cus)
{
    // [kind 1 .. 4][K % 128 != 0][exponents of b]
    static const Cost cost[4][2][2] = {{{{2.43, 0.59, 0.704, 0.175}, {3.03, 0.63, 0.738, 0.253}}, {{2.38, 0.54, 0.953, 0.381}, {2.90, 0.45, 1.100, 0.565}}},
                                       {{{3.38, 0.86, 0.514, 0.101}, {3.84, 1.03, 0.700, 0.129}}, {{3.27, 0.94, 0.728, 0.210}, {3.82, 1.11, 1.009, 0.285}}},
                                       {{{4.76, 1.22, 0.354, 0.140}, {5.79, 1.68, 0.406, 0.150}}, {{4.78, 1.66, 0.510, 0.179}, {5.56, 1.95, 0.667, 0.206}}},
                                       {{{6.86, 1.59, 0.419, 0.187}, {8.05, 2.53, 0.622, 0.178}}, {{7.90, 2.23, 0.630, 0.205}, {7.67, 2.63, 0.960, 0.267}}}};
    // 32 x 32: one round; two workgroups fit a compute unit, so that more rounds cost less each
    static const double one[2][2][2] = {{{3.71, 0.407}, {4.27, 0.409}}, {{3.90, 0.490}, {4.26, 0.642}}};
    static const double more[2][2][2] = {{{0.95, 0.375}, {1.25, 0.400}}, {{0.95, 0.520}, {1.15, 0.630}}};
    const int r = K % 128 != 0, b = b_exponents;
    const int64_t C = (K + 127) / 128;
    const double it4 = (double)((C + 3) / 4), it2 = (double)((C + 1) / 2), t0 = tiles_of(M, N, 32, 32);
    // (an accumulating round of 128 rows is charged 3 or 5 us, which is also from before: 3520 x 1540 x 1184 with exponents of b 25.0 us in
    // 128 x 192 tiles, 29.1 in the general kernel, which has it)
    const double us[5] = {t0 <= cus ? one[r][b][0] + one[r][b][1] * it4 : 2.2 + rounds_of(t0, cus) * (more[r][b][0] + more[r][b][1] * it4),
                          us_of(cost[0][r][b], tiles_of(M, N, 64, 64), cus, it4), us_of(cost[1][r][b], tiles_of(M, N, 64, 128), cus, it2),
                          us_of(cost[2][r][b], tiles_of(M, N, 128, 128), cus, (double)C, accumulate ? 3.0 : 0.0),
                          us_of(cost[3][r][b], tiles_of(M, N, 128, 192), cus, (double)C, accumulate ? 5.0 : 0.0)};
    MidPlan best{0, us[0]};
    // (128 x 192 is left out where the large tiles can take the problem: they beat it before its loop became a quarter faster.  Since
    // then they do not always: 1333 x 4096 x 11008 69.6 us in half tiles, 62.8 in 128 x 192; 1492 x 3360 x 9344 57.5, 51.1; 2272 x 7712 x
    // 4992 116.0, 95.6; 1499 x 11168 x 3328 83.7, 67.2; but 2048 x 12288 x 4096 105.3, 109.8; 2048 x 4096 x 12288 89.6, 124.7;
    // 8192 x 4096 x 4096 117.0, 160.9.)
    for (int k = 1; k < (large_ok ? 4 : 5); k++)
        if (us[k] < 0.97 * best.us) best = MidPlan{k, us[k]};
    return best;
}

// k_gemm_mx_big, full or half tiles as it chooses them
double us_big(int64_t M, int64_t N, int64_t K, bool b_exponents, double cus)
{
    // [half tiles][K % 128 != 0][exponents of b]
    static const Cost cost[2][2][2] = {{{{8.83, 0.04, 0.832, 0.627}, {16.61, 3.47, 0.888, 0.566}}, {{9.93, 0.04, 0.824, 0.718}, {19.86, 0.0, 0.853, 0.878}}},
                                       {{{3.99, 0.65, 0.605, 0.147}, {5.30, 3.23, 0.667, 0.164}}, {{4.06, 0.05, 0.734, 0.260}, {5.48, 4.20, 0.865, 0.161}}}};
    const bool half = moss_internal_gemm_big_narrow(M, N);
    return us_of(cost[half][K % 128 != 0][b_exponents], tiles_of(M, N, half ? 128 : 256, 256), cus, (double)((K + 127) / 128));
}

// k_gemm: two workgroups run on a compute unit at a time, every stage waits for its own loads, every tile leaves at the
// memory's rate
double us_general(int64_t M, int64_t N, int64_t K, bool b_exponents, double cus)
{
    const double C = (double)((K + 127) / 128), w = tiles_of(M, N, 128, 128) / cus;       // tiles per compute unit
    const double rounds = w <= 2.0 ? 1.0 : std::ceil(w / 2.0), u = w < rounds ? w / rounds : 1.0;
    return b_exponents ? 5.4 + rounds * C * (1.25 + 0.65 * u) + 3.4 * w : 4.6 + rounds * C * (0.96 + 0.6 * u) + 2.2 * w;
}

double model_cus()
{
    const int cus = moss_internal_cu_count();
    return cus <= 0 ? 256 : cus;
}

// The small tiles if they are expected to take at most nine tenths of the time of the kernel that would have the problem
// otherwise (large_ok: k_gemm_mx_big, else k_gemm; three quarters where short K and FP32 outputs make the fits worse, seven
// tenths without exponents of a, which the fits have not seen), kind -1 and that kernel's time if not.
MidPlan plan_small_or_other(int64_t M, int64_t N, int64_t K, const uint8_t *a_e, const uint8_t *b_e, bool accumulate, bool large_ok)
{
    const double cus = model_cus(), other = large_ok ? us_big(M, N, K, b_e != nullptr, cus) : us_general(M, N, K, b_e != nullptr, cus);
    if (K > ((int64_t)1 << 22) || ((uintptr_t)a_e & 3) || ((uintptr_t)b_e & 3)) return MidPlan{-1, other};     // (32-bit offsets inside a tile)
    const MidPlan plan = plan_mid(M, N, K, b_e != nullptr, accumulate, large_ok, cus);
    const double margin = !a_e && plan.kind >= 3 ? 0.7 : b_e && plan.kind >= 3 && !large_ok && K <= 640 ? 0.75 : 0.9;
    return plan.us > margin * other ? MidPlan{-1, other} : plan;
}

}  // namespace

// The kind of tiles (0 .. 4), -1 to leave the problem to the kernel that would have it otherwise.  Over the 2200 problems, with the
// kernels as they were when fitted, the ones that this and the rule below choose took 0.5 % more than the fastest of each
// problem (mean).  With the kernels as they are now it is 1.3 % over 2000 other problems.
int moss_internal_gemm_mid_kind(int64_t M, int64_t N, int64_t K, const uint8_t *a_e, const uint8_t *b_e, int accumulate,
                                bool large_ok)
{
    return plan_small_or_other(M, N, K, a_e, b_e, accumulate != 0, large_ok).kind;
}

// Whether k_gemm_mx_big takes a problem with K % 128 != 0 from the kernel that has it by the rule above: where it is
// expected to be a fourteenth faster (a fifth for a short K with exponents of b, as above).  4096 x 4096 x 2080 66 -> 41 us, 11328 x 3520 x
// 2080 175 -> 105, 4160 x 4480 x 9824 287 -> 223, 2432 x 6016 x 2656 with exponents of b 105 -> 56.
bool moss_internal_gemm_big_ragged(int64_t M, int64_t N, int64_t K, const uint8_t *a_e, const uint8_t *b_e, int accumulate,
                                   int64_t ld_out)
{
    if (!moss_internal_gemm_big_ragged_ok(M, N, K, a_e, b_e, ld_out)) return false;
    const double other = plan_small_or_other(M, N, K, a_e, b_e, accumulate != 0, false).us;
    return us_big(M, N, K, b_e != nullptr, model_cus()) < (b_e && K < 1000 ? 0.8 : 0.93) * other;
}

int moss_internal_gemm_mid(int kind, int64_t M, int64_t N, int64_t K, const uint8_t *a_q, const uint8_t *a_e, const float *a_s,
                           const uint8_t *b_q, const uint8_t *b_e, const float *b_s, void *out, int out_f32, int64_t ld_out,
                           int accumulate, hipStream_t st)
{
    using namespace moss;
    MidArgs p{};
    p.M = M; p.N = N; p.K = K;
    p.a_q = a_q; p.a_e = a_e; p.a_s = a_s;
    p.b_q = b_q; p.b_e = b_e; p.b_s = b_s;
    p.out = out; p.ld_out = ld_out; p.out_f32 = out_f32; p.accumulate = accumulate;
    p.e_dwords = K % 128 == 0;
    switch (kind) {
        case 0: return launch_mid_kind<kMidDense, 0>(p, st);
        case 1: return launch_mid_kind<kMidDense, 1>(p, st);
        case 2: return launch_mid_kind<kMidDense, 2>(p, st);
        case 3: return launch_mid_kind<kMidDense, 3>(p, st);
        default: return launch_mid_kind<kMidDense, 4>(p, st);
    }
}
