// Wide-tile FP8 GEMM for the products of experts and for operands with an FP32 scale per block of 128.
//
// Shape of the kernel
//  * (32 MI) x (64 NJ) outputs per workgroup of 8 waves (2 x 4), two waves per SIMD, (16 MI) x (16 NJ) per wave in 16 x 16 accumulators of
//    V_MFMA_(SCALE_)F32_16X16X128_F8F6F4, all of them vector registers: the blocked forms add to them on the vector unit.  One
//    matrix instruction covers a stage of K = 128, which is a block.
//  * Stages go through SLOTS slots of LDS, filled by direct global->LDS copies of 128 bytes per row.  One barrier per stage, behind the
//    last fragment's reads of a: there the stage's slot is free, for the copies of stage + SLOTS, and the next stage has landed.  Its first fragments
//    are read behind the last matrix instructions of this one, each b fragment behind the instruction that used its registers
//    last.  While one wave waits its neighbour on the SIMD computes.  Tiles of up to 128 rows hold a whole stage in registers, and
//    all its reads stand ahead of the barrier (kHolds).  (128 x 256 takes all 256
//    registers for that: 8 of the form for rows of groups are spilled and 7 of that for dW of groups, with some twenty accesses to scratch
//    memory each.  256 x 256 with a scale per row of b, which does not hold its stage, spills 2.  Scratch counts in vmcnt with the
//    copies, behind those that a wait is for: it can make a wait longer, never shorter.)
//  * Blocked forms: an instruction starts from zero and leaves its sum in one of four parts.  A part is added to the accumulators
//    times its scales when two further instructions have been issued; the matrix unit takes them one after the other, so it has
//    retired by then.  This order is all that protects the read; the instructions are volatile asm and a part passes through an
//    empty one at that place.
//  * Exponents (four bytes) or scales (a float) of a stage are one dword per row.  A thread fetches those of its row for a block of stages
//    ahead into registers and leaves them in a ring in LDS at the end of the block before.
//  * Persistent workgroups walk their tiles in one stream of stages: copies and scales of the next tile are on their way while this one
//    ends.  Three places in that stream are kept: what is computed, what is copied (SLOTS stages ahead) and what is
//    scaled (a block of stages ahead).
//  * K that ends inside a stage, groups of any length: the last stage's copies are moved back to end with the row, and what of
//    a stage does not belong to the sum is zeroed in the fragments of a.  (Where groups lie along K, in those of b and in the exponents
//    as well: rows of other groups or of none may hold NaN.)
//
// A stage takes (us; blocks of 128 of a weight / of rows / dW of groups) 1.56 / 1.90 / 2.3 to 2.7 in 256 x 256 tiles, 0.95 / 1.19 / 1.2 to
// 1.4 in 128 x 256, 0.67 / 0.79 in 128 x 128, 0.53 / 0.57 in 64 x 128; the matrix instructions of 256 x 256 alone 1.05.  Bound: in the
// blocked forms matrix and vector unit take turns (256 x 256: 1.05 us of matrix instructions, and one or two vector instructions per
// output, 0.45 or 0.9 us, make the 1.56 and 1.90; matrix unit busy 48 % of the time, no LDS conflicts), on top of which long runs meet the
// power limit; the copies for dW, whose rows begin anywhere in a line; LDS reads in the smallest tiles.
//
// Operand layout of the instruction: lane (r = lane % 16, q = lane / 16) supplies for row r the bytes K[16q, 16q + 16) in its first four
// registers and K[64 + 16q, 64 + 16q + 16) in the last four; the 32-wide block q of row r is scaled by byte 0 of the lane's
// scale register.  Stage layout in LDS: as in the large-tile kernel.
#pragma once
#include <atomic>
#include <type_traits>

#include "moss_gemm.h"

namespace moss {

enum WideForm { kWideGroupRows, kWideGroupDw, kWideBlock, kWideBlockRows };

struct WideArgs {
    int64_t M, N, K;                  // (kWideGroupDw: K is the length of the rows of a and b)
    const uint8_t *a_q, *b_q;
    const uint8_t *a_x, *b_x;         // exponents or scales (kWideGroupRows: none of b)
    int64_t pitch_a, pitch_b;         // bytes from row to row of them
    int64_t end_a, end_b;             // and of all
    const float *a_s, *b_s;           // the one scale of each; of each group of b (kWideGroupRows)
    int64_t ld_b, b_stride, b_s_stride;      // as in moss_gemm_fp8_mx_grouped (else ld_b = K)
    const int32_t *offsets;
    int groups;
    void *out;
    int64_t ld_out;
    int out_f32, accumulate;
    int tiles_m, tiles_n;             // (kWideGroupRows: tiles_m is not used)
};

extern __shared__ __attribute__((aligned(1024))) uint8_t wide_smem[];

constexpr int kWideThreads = 512;
constexpr int kWideK = 128;

template <int MI, int NJ, int SLOTS>
struct WideShape {
    static constexpr int kBM = 32 * MI, kBN = 64 * NJ;
    static constexpr int kRows = kBM + kBN;
    static constexpr int kSlot = kRows * kWideK;
    static constexpr int kPieces = kRows / 8 / 8;               // 8-row copies per wave and stage
    static constexpr int kRing = SLOTS * kSlot;                 // [2 blocks][kBlock stages][rows] dwords
    // Stages whose scales are fetched together.  Where they are taken from the registers everything that is under way is waited for, which
    // two slots do at every stage, and more of them should not do often.
    static constexpr int kBlock = SLOTS == 2 || NJ == 4 ? 4 : MI == 2 ? 16 : 8;
    static constexpr int kTable = kRing + 2 * kBlock * kRows * 4;    // tiles ahead of each group (kWideGroupRows)
    static_assert(kBM % 64 == 0 && kBN % 64 == 0, "whole copies per wave, whole waves of rows");
    static_assert(MI * NJ % 4 == 0 && MI % 2 == 0, "parts and fragments take turns from stage to stage");
    static constexpr int lds_bytes(WideForm form, int groups) { return kTable + (form == kWideGroupRows ? (groups + 1) * 4 : 0); }
};

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_at1 __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t u32_at1 __attribute__((aligned(1)));

__device__ __forceinline__ void mfma16_from_zero(v4f &d, const v8i &x, const v8i &y)
{
    asm volatile("v_mfma_f32_16x16x128_f8f6f4 %0, %1, %2, 0" : "=&v"(d) : "v"(x), "v"(y));
}
__device__ __forceinline__ void mfma16_scaled(v4f &d, const v8i &x, const v8i &y, uint32_t sx, uint32_t sy)
{
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]" : "+v"(d) : "v"(x), "v"(y), "v"(sx), "v"(sy));
}

// Stores the 16 x 32 outputs of two fragments side by side.  Lane (r, q) holds row r, columns 4 q .. 4 q + 3 of each.  BF16: lanes of
// neighbouring q exchange a fragment each and hold eight columns of one.  (N and ld are multiples of 8: pieces are whole)
__device__ __forceinline__ void store_pair(const v4f &x, const v4f &y, float scale, void *out, int64_t ld, int64_t row, int64_t n, int q, int64_t M,
                                           int64_t N, int out_f32, int accumulate)
{
    if (out_f32) {
#pragma unroll
        for (int f = 0; f < 2; f++) {
            const v4f &d = f ? y : x;
            const int64_t at = n + 16 * f + 4 * q;
            if (row >= M || at >= N) continue;
            float *o = reinterpret_cast<float *>(out) + row * ld + at;
            float4 v = make_float4(d[0] * scale, d[1] * scale, d[2] * scale, d[3] * scale);
            if (accumulate) {
                const float4 old = *reinterpret_cast<const float4 *>(o);
                v.x += old.x; v.y += old.y; v.z += old.z; v.w += old.w;
            }
            *reinterpret_cast<float4 *>(o) = v;
        }
        return;
    }
    uint32_t w[4] = {pack_bf16(x[0] * scale, x[1] * scale), pack_bf16(x[2] * scale, x[3] * scale), pack_bf16(y[0] * scale, y[1] * scale),
                     pack_bf16(y[2] * scale, y[3] * scale)};
#pragma unroll
    for (int k = 0; k < 2; k++) {
        const auto both = __builtin_amdgcn_permlane16_swap(w[k], w[2 + k], false, false);
        w[k] = both[0];
        w[2 + k] = both[1];
    }
    // q even: columns 4 q .. 4 q + 7 of the first fragment, odd: 4 (q - 1) .. of the second
    const int64_t at = n + 16 * (q & 1) + 4 * (q & 2);
    if (row < M && at < N) *reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(out) + row * ld + at) = make_uint4(w[0], w[1], w[2], w[3]);
}

// Weight gradients of groups of any length: an XCD gets an eighth of every group's tiles (side by side, for the L2), the eighths in
// turn, so that all have the same share of long and short sums.  (Whole groups side by side: 8 groups of 4096 x 4096 whose lengths
// differ by a factor of five kept the XCD of the longest for 709 us.)  Tiles of group g in the list of XCD x, and of the first n groups.
__host__ __device__ __forceinline__ uint32_t eighth_begin(uint32_t each, uint32_t part) { return (uint32_t)((uint64_t)each * part >> 3); }
__host__ __device__ __forceinline__ uint32_t eighth_size(uint32_t each, uint32_t part) { return eighth_begin(each, part + 1) - eighth_begin(each, part); }
__host__ __device__ __forceinline__ uint32_t eighths_of(uint32_t each, uint32_t xcd, uint32_t groups)
{
    uint32_t n = (groups >> 3) * each;               // (eight groups in a row give every part once)
    for (uint32_t g = groups & ~7u; g < groups; g++) n += eighth_size(each, (xcd + g) & 7);
    return n;
}

template <WideForm FORM, int MI, int NJ, int SLOTS>
__global__ __launch_bounds__(kWideThreads, 2) void k_gemm_wide(const WideArgs p)
{
    using S = WideShape<MI, NJ, SLOTS>;
    constexpr int kWideBN = S::kBN;
    constexpr bool kBlocked = FORM == kWideBlock || FORM == kWideBlockRows;
    constexpr bool kGroupK = FORM == kWideGroupDw;   // (what is next to a group of K in a row is not its own)
    constexpr int kBM = S::kBM, kPieces = S::kPieces, kBlock = S::kBlock;
    const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 2, wn = wave & 3;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)wide_smem;
    uint32_t *ring = reinterpret_cast<uint32_t *>(wide_smem + S::kRing), *table = reinterpret_cast<uint32_t *>(wide_smem + S::kTable);
    const int64_t ld_a = p.K;

    // (workgroups are dealt round-robin to the XCDs; gridDim.x is a multiple of 8 if one of them has more than one tile)
    const uint32_t each = (uint32_t)p.tiles_m * (uint32_t)p.tiles_n, xcd = blockIdx.x & 7;
    uint32_t total = each, mine = blockIdx.x, step = gridDim.x;
    if constexpr (FORM == kWideGroupRows) {
        if (wave == 0) count_group_tiles<kBM>(table, p.offsets, p.groups, p.M);
        __syncthreads();
        total = (uint32_t)__builtin_amdgcn_readfirstlane((int)table[p.groups]) * (uint32_t)p.tiles_n;
    }
    if constexpr (FORM == kWideGroupDw) {
        total = eighths_of(each, xcd, (uint32_t)p.groups);
        mine >>= 3;
        step >>= 3;
    }
    if (mine >= total) return;
    const int n_tiles = (int)((total - mine + step - 1) / step);

    // Tile k of this workgroup, in bands of 4 tile rows; each XCD gets a contiguous range, or its part of every group
    struct Tile {
        int64_t m0, n0, rows_end;                    // rows of a below rows_end
        int first, end;                              // the sum is over [first, end)
        int group, T;
    };
    auto tile_of = [&](int k) {
        Tile t;
        const uint32_t pid = mine + (uint32_t)k * step;
        uint32_t at = pid;
        if constexpr (FORM != kWideGroupDw) {
            at = xcd_range_tile(pid, total);
        } else {
            at += xcd * (total >> 3);                // (each begins elsewhere in its list)
            if (at >= total) at -= total;
        }
        uint32_t tiles_m = (uint32_t)p.tiles_m;
        t.group = 0;
        t.m0 = 0;
        t.rows_end = p.M;
        t.first = 0;
        t.end = (int)p.K;
        if constexpr (FORM == kWideGroupRows) {
            const GroupTiles of = group_of_tile(table, p.groups, (uint32_t)p.tiles_n, at);
            t.group = of.group;
            tiles_m = of.count;
            at -= of.ahead * (uint32_t)p.tiles_n;
            group_range(p.offsets, t.group, p.M, t.m0, t.rows_end);
        }
        if constexpr (FORM == kWideGroupDw) {
            uint32_t g = __builtin_amdgcn_readfirstlane((int)(at / each)) * 8;
            at -= (g >> 3) * each;
            for (uint32_t n; at >= (n = eighth_size(each, (xcd + g) & 7)); g++) at -= n;
            at += eighth_begin(each, (xcd + g) & 7);
            t.group = (int)g;
            int64_t first, end;
            group_range(p.offsets, t.group, p.K, first, end);
            t.first = (int)first & ~(kGroup - 1);                // (they are multiples of 32 already, by contract)
            t.end = (int)end & ~(kGroup - 1);
        }
        constexpr uint32_t kBand = 4;
        const uint32_t band = at / (kBand * (uint32_t)p.tiles_n), rem = at - band * kBand * (uint32_t)p.tiles_n;
        const uint32_t here = tiles_m - band * kBand < kBand ? tiles_m - band * kBand : kBand;
        t.n0 = (int64_t)__builtin_amdgcn_readfirstlane((int)(rem / here)) * kWideBN;
        t.m0 += (int64_t)__builtin_amdgcn_readfirstlane((int)(band * kBand + rem % here)) * kBM;
        t.T = (t.end - t.first + kWideK - 1) / kWideK;
        if (t.T == 0) t.T = 1;                                   // (nothing to add, but zeros to store)
        return t;
    };
    // first byte of stage P of a row: moved back where the row would end inside it
    const int last_stage = (int)p.K - kWideK;
    auto stage_at = [&](const Tile &t, int P) {
        const int at = t.first + P * kWideK;
        return at < last_stage ? at : last_stage;
    };

    // ---- what is copied
    const int piece0 = wave * kPieces;
    int c_tile = 0, c_P = 0;
    Tile ct = tile_of(0);
    const uint8_t *ca, *cb;
    int c_last_a, c_last_b;
    auto copy_tile = [&]() {
        ca = p.a_q + ct.m0 * ld_a;
        cb = p.b_q + ct.n0 * p.ld_b + (FORM == kWideGroupRows ? ct.group * p.b_stride : 0);
        c_last_a = (int)(ct.rows_end - ct.m0 < kBM ? ct.rows_end - ct.m0 : kBM) - 1;
        c_last_b = (int)(p.N - ct.n0 < kWideBN ? p.N - ct.n0 : kWideBN) - 1;
    };
    uint32_t c_slot = 0;
    const uint8_t *sa_ptr, *sb_ptr;                  // of the stage to copy
    auto copy_begin = [&]() {
        const int at = stage_at(ct, c_P);
        sa_ptr = ca + at;
        sb_ptr = cb + at;
    };
    // 8 rows of a or of b; rows beyond the matrix repeat the last.  (The lane's offset is worked out anew: there are no registers for
    // those of all pieces.)
    auto copy_piece = [&](int x) {
        const bool is_a = piece0 + x < kBM / 8;
        const int r = (piece0 + x - (is_a ? 0 : kBM / 8)) * 8 + (lane >> 3), last = is_a ? c_last_a : c_last_b;
        const uint32_t chunk = (uint32_t)((lane & 7) ^ ((r >> 1) & 7)) * 16;
        const uint32_t off = (uint32_t)(r < last ? r : last) * (uint32_t)(is_a ? ld_a : p.ld_b) + chunk;
        dma16_at(is_a ? sa_ptr : sb_ptr, off, lds0 + c_slot + (uint32_t)piece0 * 1024, x * 1024);
    };
    auto copy_end = [&]() {
        c_slot = c_slot + S::kSlot == SLOTS * S::kSlot ? 0 : c_slot + S::kSlot;
        if (++c_P == ct.T) {
            c_P = 0;
            if (++c_tile < n_tiles) {
                ct = tile_of(c_tile);
                copy_tile();
            }
        }
    };

    // ---- what is scaled: this thread's row, a block of dwords at a time
    int s_tile = 0, s_block = 0, s_blocks = 1, s_T = 1;
    const bool s_is_a = wave < kBM / kWave, s_there = wave < S::kRows / kWave && (FORM != kWideGroupRows || s_is_a);
    const uint8_t *s_base = nullptr;                 // of the tile's first row
    uint32_t s_row = 0, s_end = 0;                   // bytes from there: this row, the end of the array (no row of the tile is 4 GB away)
    uint32_t s_back = 0;                             // exponents by which the tile's last stage is moved back
    uint32_t words[kBlock];
    int moved = kBlock;                                   // the one of them that is moved by so many exponents
    uint32_t moved_by = 0;
    auto scale_tile = [&](const Tile &t) {
        s_blocks = (t.T + kBlock - 1) / kBlock;
        s_T = t.T;
        // (from where the first stage is copied, at least four exponents ahead of the row's end)
        const int begin = stage_at(t, 0);
        if (!kBlocked) s_back = (uint32_t)(begin + (t.T - 1) * kWideK - stage_at(t, t.T - 1)) >> 5;
        if (!s_there) return;
        const int64_t row0 = s_is_a ? t.m0 : FORM == kWideBlock ? t.n0 >> 7 : t.n0, pitch = s_is_a ? p.pitch_a : p.pitch_b;
        const int last = (int)((s_is_a ? t.rows_end - t.m0 : p.N - t.n0) < S::kRows ? (s_is_a ? t.rows_end - t.m0 : p.N - t.n0) : S::kRows) - 1;
        int r = s_is_a ? tid : tid - kBM;
        r = r < last ? r : last;
        if (FORM == kWideBlock && !s_is_a) r >>= 7;
        const int64_t skip = row0 * pitch + (FORM == kWideGroupDw ? begin >> 5 : 0), left = (s_is_a ? p.end_a : p.end_b) - skip;
        s_base = (s_is_a ? p.a_x : p.b_x) + skip;
        s_end = left < 0xFFFFFFFFll ? (uint32_t)left : 0xFFFFFFFFu;
        s_row = (uint32_t)r * (uint32_t)pitch;
    };
    auto scale_load = [&]() {
        if (s_there) {
#pragma unroll
            for (int f = 0; f < kBlock / 4; f++) {
                const uint32_t at = s_row + (uint32_t)s_block * (4 * kBlock) + 16 * f;
                if (at + 16 <= s_end) {
                    const u32x4_at1 v = *reinterpret_cast<const u32x4_at1 *>(s_base + at);
                    words[4 * f] = v.x; words[4 * f + 1] = v.y; words[4 * f + 2] = v.z; words[4 * f + 3] = v.w;
                } else {
                    // the array ends here: its last four bytes, moved to their place in the word
#pragma unroll
                    for (int u = 0; u < 4; u++) {
                        const uint32_t w = at + 4 * u, from = w + 4 <= s_end ? w : s_end - 4;
                        words[4 * f + u] = *reinterpret_cast<const u32_at1 *>(s_base + from) >> (8 * ((w - from) & 3));
                    }
                }
            }
        }
        if (!kBlocked) {
            moved = s_block == s_blocks - 1 ? (s_T - 1) % kBlock : kBlock;
            moved_by = 8 * s_back;
        }
        if (++s_block == s_blocks) {
            s_block = 0;
            if (++s_tile < n_tiles) scale_tile(tile_of(s_tile));
        }
    };
    auto scale_store = [&](int half) {
        if (s_there)
#pragma unroll
            for (int u = 0; u < kBlock; u++) {
                uint32_t w = words[u];
                if (!kBlocked && u == moved) w <<= moved_by;
                if (FORM == kWideBlock) w = __float_as_uint(shown_scale(__uint_as_float(w)));
                ring[(half * kBlock + u) * S::kRows + tid] = w;
            }
    };

    // ---- what is computed
    v4f acc[MI][NJ], part[kBlocked ? 4 : 1];
    v8i fa[2], fb[NJ];
    uint32_t sa[4] = {0, 0, 0, 0}, sb[NJ];           // exponent bytes (sb: of each fragment); scales of rows of a, of blocks of b
    using RowScales = float[FORM == kWideBlockRows ? NJ : 1][4];
    RowScales row_scale;
    float both[2];
    const int sw = (r16 >> 1) & 7;
    const uint32_t lane_at = (uint32_t)(r16 * kWideK + ((q ^ sw) << 4));
    const uint32_t a_at = lane_at + (uint32_t)(wm * 16 * MI * kWideK), b_at = lane_at + (uint32_t)((kBM + wn * 16 * NJ) * kWideK);
    // (chunk q + 4 of a row lies 64 bytes from chunk q, whichever way)
    auto read_fragment = [&](v8i &f, uint32_t at, uint32_t at64) {
        const uint4 lo = *reinterpret_cast<const uint4 *>(wide_smem + at), hi = *reinterpret_cast<const uint4 *>(wide_smem + at64);
        f[0] = (int)lo.x; f[1] = (int)lo.y; f[2] = (int)lo.z; f[3] = (int)lo.w;
        f[4] = (int)hi.x; f[5] = (int)hi.y; f[6] = (int)hi.z; f[7] = (int)hi.w;
    };
    auto a_fragment = [&](v8i &f, int i, uint32_t slot) { read_fragment(f, a_at + slot + (uint32_t)(i * 16 * kWideK), (a_at ^ 64) + slot + (uint32_t)(i * 16 * kWideK)); };
    auto b_fragment = [&](v8i &f, int j, uint32_t slot) { read_fragment(f, b_at + slot + (uint32_t)(j * 16 * kWideK), (b_at ^ 64) + slot + (uint32_t)(j * 16 * kWideK)); };
    auto a_scale = [&](int i, int stage) {
        const uint32_t *x = ring + stage * S::kRows + wm * 16 * MI + i * 16 + r16;
        return kBlocked ? *x : (uint32_t)reinterpret_cast<const uint8_t *>(x)[q];
    };
    auto b_scale = [&](uint32_t (&s)[NJ], RowScales &rows, int j, int stage) {
        const uint32_t *x = ring + stage * S::kRows + kBM + wn * 16 * NJ + j * 16;
        if constexpr (FORM == kWideBlock) {
            if (j == 0) s[0] = x[0];                             // (a wave's columns share it)
        } else if constexpr (FORM == kWideBlockRows) {
            const float4 v = *reinterpret_cast<const float4 *>(x + 4 * q);
            rows[j][0] = v.x; rows[j][1] = v.y; rows[j][2] = v.z; rows[j][3] = v.w;
        } else if constexpr (FORM == kWideGroupDw) {
            s[j] = (uint32_t)reinterpret_cast<const uint8_t *>(x + r16)[q];
        } else {
            s[j] = 127;
        }
    };
    auto read_a = [&](int i, uint32_t slot, int stage) {
        a_fragment(fa[i & 1], i, slot);
        sa[i & 3] = a_scale(i, stage);
    };
    // instruction number n of a stage is that of fragments (n / NJ, n % NJ); its part is n % 4
    constexpr int kAll = MI * NJ;
    auto add_part = [&](int n, uint32_t of_a, const RowScales &rows) {       // (of_a: the row's scale, or with that of the block of b)
        const int i = n / NJ, j = n % NJ;
        v4f &d = part[kBlocked ? n & 3 : 0];
        asm volatile("" : "+v"(d));
#pragma unroll
        for (int v = 0; v < 4; v++) {
            if (FORM == kWideBlockRows) acc[i][j][v] = __builtin_fmaf(d[v] * __uint_as_float(of_a), rows[FORM == kWideBlockRows ? j : 0][v], acc[i][j][v]);
            else acc[i][j][v] = __builtin_fmaf(d[v], __uint_as_float(of_a), acc[i][j][v]);
        }
        asm volatile("" : "+v"(acc[i][j]));          // (here, and not when the part's registers are needed again)
    };
    auto fold = [&](int n) { add_part(n, FORM == kWideBlockRows ? sa[n / NJ & 3] : __float_as_uint(both[n / NJ & 1]), row_scale); };

    // Tiles of up to 128 rows: a wave holds all fragments and scales of its stage and reads those of the next between its matrix
    // instructions.  The barrier is at the head of the stage: there every wave holds it, so that its slot is free, and the next has landed.
    // (Where the fragments of a are fetched one ahead instead, a stage of 64 x 128 took 0.65 us, most of it the trip to LDS.)
    constexpr bool kHolds = MI <= 4 && !(FORM == kWideBlockRows && NJ == 4);
    struct Held {
        v8i a[MI], b[NJ];
        uint32_t sa[MI], sb[NJ];
        RowScales rows;
    };
    Held held0, held1;
    auto read_held = [&](Held &f, int x, uint32_t to) {
        if (x < NJ) b_fragment(f.b[x], x, to);
        else a_fragment(f.a[x - NJ], x - NJ, to);
    };
    auto read_held_scales = [&](Held &f, int stage) {
#pragma unroll
        for (int i = 0; i < MI; i++) f.sa[i] = a_scale(i, stage);
#pragma unroll
        for (int j = 0; j < NJ; j++) b_scale(f.sb, f.rows, j, stage);
    };

    // ---- the first stages
    copy_tile();
#pragma unroll
    for (int s = 0; s < SLOTS; s++)
        if (c_tile < n_tiles) {
            copy_begin();
#pragma unroll
            for (int x = 0; x < kPieces; x++) copy_piece(x);
            copy_end();
        }
    scale_tile(tile_of(0));
    scale_load();
    scale_store(0);
    wait_vmcnt<0>();
    wait_lds_and_barrier();
    int half = 0;
    uint32_t slot = 0;
    if constexpr (kHolds) {
#pragma unroll
        for (int x = 0; x < MI + NJ; x++) read_held(held0, x, 0);
        read_held_scales(held0, 0);
    } else {
        read_a(0, 0, 0);
#pragma unroll
        for (int j = 0; j < NJ; j++) {
            b_fragment(fb[j], j, 0);
            b_scale(sb, row_scale, j, 0);
        }
    }

    for (int k = 0; k < n_tiles; k++) {
        const Tile t = tile_of(k);
#pragma unroll
        for (int i = 0; i < MI; i++)
#pragma unroll
            for (int j = 0; j < NJ; j++)
#pragma unroll
                for (int v = 0; v < 4; v++) acc[i][j][v] = 0.0f;
        if (kBlocked) {
            // what the first instructions fold is nothing, whatever the scales of the tile before
            both[1] = 0.0f;
            sa[(MI - 1) & 3] = held1.sa[MI - 1] = 0;
#pragma unroll
            for (int j = 2; j < 4; j++)
#pragma unroll
                for (int v = 0; v < 4; v++) part[kBlocked ? j : 0][v] = 0.0f;
#pragma unroll
            for (int j = FORM == kWideBlockRows ? NJ - 2 : 0; j < (FORM == kWideBlockRows ? NJ : 0); j++)
#pragma unroll
                for (int v = 0; v < 4; v++) row_scale[j][v] = held1.rows[j][v] = 0.0f;
        }
        // 16-byte chunks of the last stage that belong to the sum
        const int last_from = t.first + (t.T - 1) * kWideK, last_at = stage_at(t, t.T - 1);
        const int last_lo = (last_from - last_at) >> 4, last_hi = (t.end - last_at) >> 4;
        const bool last_whole = last_lo == 0 && last_hi == 8;
        // what of a fragment does not belong to the sum: zeros, and 2^0 for a block of 32
        auto cut = [&](v8i &f) {
#pragma unroll
            for (int v = 0; v < 8; v++) {
                const int c = q + (v < 4 ? 0 : 4);
                if (c < last_lo || c >= last_hi) f[v] = 0;
            }
        };
        auto cut_exponent = [&](uint32_t &e) {
            if (2 * q < last_lo || 2 * q >= last_hi) e = 127;
        };
        auto one_stage = [&](int P, Held &f, Held &next) {
            const bool block_ends = P % kBlock == kBlock - 1 || P == t.T - 1;
            if (P % kBlock == 0 && s_tile < n_tiles) scale_load();
            const int stage = half * kBlock + P % kBlock, next_stage = block_ends ? (half ^ 1) * kBlock : stage + 1;
            const uint32_t next_slot = slot + S::kSlot == SLOTS * S::kSlot ? 0 : slot + S::kSlot;
            const bool whole = P < t.T - 1 || last_whole;
            bool copies = false;
            if constexpr (kHolds) {
                copies = c_tile < n_tiles;
                if (SLOTS > 2 && copies) wait_vmcnt<(SLOTS - 2) * kPieces>();
                else wait_vmcnt<0>();
                if (block_ends) scale_store(half ^ 1);
                wait_lds_and_barrier();
                if (copies) copy_begin();
                if (!whole) {
#pragma unroll
                    for (int i = 0; i < MI; i++) {
                        cut(f.a[i]);
                        if (kGroupK) cut_exponent(f.sa[i]);
                    }
                    if (kGroupK)
#pragma unroll
                        for (int j = 0; j < NJ; j++) {
                            cut(f.b[j]);
                            cut_exponent(f.sb[j]);
                        }
                }
#pragma unroll
                for (int j = 0; j < (kGroupK ? NJ : 0); j++) asm volatile("" : "+v"(f.b[j]));
#pragma unroll
                for (int i = 0; i < MI; i++) {
                    if (FORM == kWideBlock) f.sa[i] = __float_as_uint(block_scales(__uint_as_float(f.sa[i]), __uint_as_float(f.sb[0])));
                    asm volatile("" : "+v"(f.a[i]), "+v"(f.sa[i]));
                }
                if (!kBlocked)
#pragma unroll
                    for (int j = 0; j < NJ; j++) asm volatile("" : "+v"(f.sb[j]));
                asm volatile("s_nop 4" ::: "memory");            // vector ALU write -> operand of a matrix instruction
#pragma unroll
                for (int n = 0; n < kAll; n++) {
                    const int i = n / NJ, j = n % NJ;
                    if (kBlocked) mfma16_from_zero(part[kBlocked ? n & 3 : 0], f.b[j], f.a[i]);
                    else mfma16_scaled(acc[i][j], f.b[j], f.a[i], f.sb[j], f.sa[i]);
                    if (kBlocked) {
                        // (the last two of a stage are folded in the next one, ahead of its reads of scales)
                        if (n >= 2) add_part(n - 2, f.sa[(n + kAll - 2) % kAll / NJ], f.rows);
                        else add_part(n + kAll - 2, next.sa[(n + kAll - 2) % kAll / NJ], next.rows);
                    }
#pragma unroll
                    for (int x = n * (MI + NJ) / kAll; x < (n + 1) * (MI + NJ) / kAll; x++) read_held(next, x, next_slot);
                    if (n == 2) read_held_scales(next, next_stage);
                    if (copies)
#pragma unroll
                        for (int x = n * kPieces / kAll; x < (n + 1) * kPieces / kAll; x++) copy_piece(x);
                    pin();
                }
            }
#pragma unroll
            for (int i = 0; i < (kHolds ? 0 : MI); i++) {
                if (!whole) {
                    cut(fa[i & 1]);
                    if (kGroupK) {
                        cut_exponent(sa[i & 3]);
                        if (i == 0)
#pragma unroll
                            for (int j = 0; j < NJ; j++) {
                                cut(fb[j]);
                                cut_exponent(sb[j]);
                                asm volatile("" : "+v"(fb[j]));
                            }
                    }
                    asm volatile("s_nop 4" : "+v"(fa[i & 1]));   // vector ALU write -> operand of a matrix instruction
                }
                if (!kBlocked) {
                    // vector ALU write (the byte of the exponent) -> operand of a matrix instruction
                    if (i == 0)
#pragma unroll
                        for (int j = 0; j < NJ; j++) asm volatile("" : "+v"(sb[j]));
                    asm volatile("s_nop 4" : "+v"(sa[i & 3]));
                }
                if (FORM == kWideBlock) both[i & 1] = block_scales(__uint_as_float(sa[i & 3]), __uint_as_float(sb[0]));
#pragma unroll
                for (int j = 0; j < NJ; j++) {
                    if (kBlocked) mfma16_from_zero(part[kBlocked ? (i * NJ + j) & 3 : 0], fb[j], fa[i & 1]);
                    else mfma16_scaled(acc[i][j], fb[j], fa[i & 1], sb[j], sa[i & 3]);
                    if (kBlocked) {
                        // (the last two of a stage are folded in the next one.  The scales of the next stage's rows of b are read
                        // when those of this one have been used)
                        const int n = i * NJ + j - 2, of = n >= 0 ? n : n + kAll;
                        fold(of);
                        if (of / NJ == MI - 1 && FORM == kWideBlockRows) b_scale(sb, row_scale, of % NJ, n >= 0 ? next_stage : stage);
                    }
                    if (i + 1 < MI && j == 0) read_a(i + 1, slot, stage);
                    if (i == MI - 1) {
                        if (j == 0) read_a(0, next_slot, next_stage);
                        b_fragment(fb[j], j, next_slot);
                        if (FORM != kWideBlockRows) b_scale(sb, row_scale, j, next_stage);
                        if (copies)
#pragma unroll
                            for (int x = j * kPieces / NJ; x < (j + 1) * kPieces / NJ; x++) copy_piece(x);
                    }
                    pin();
                }
                if (i == MI - 2) {
                    // every wave has read this stage, and the next has landed
                    copies = c_tile < n_tiles;
                    if (SLOTS > 2 && copies) wait_vmcnt<(SLOTS - 2) * kPieces>();
                    else wait_vmcnt<0>();
                    if (block_ends) scale_store(half ^ 1);
                    wait_lds_and_barrier();
                    if (copies) copy_begin();
                }
            }
            if (copies) copy_end();
            if (block_ends) half ^= 1;
            slot = next_slot;
        };
        if constexpr (kHolds) {
            for (int P = 0; P < t.T; P += 2) {
                one_stage(P, held0, held1);
                if (P + 1 < t.T) one_stage(P + 1, held1, held0);
            }
        } else {
            for (int P = 0; P < t.T; P++) one_stage(P, held0, held0);
        }
        // ---- epilogue: straight from the registers
        float scale = 1.0f;
        if (kBlocked) {
            asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");   // the last matrix instructions retire
#pragma unroll
            for (int n = kAll - 2; n < kAll; n++) {
                if constexpr (kHolds) {
                    if (t.T & 1) add_part(n, held0.sa[n / NJ], held0.rows);
                    else add_part(n, held1.sa[n / NJ], held1.rows);
                } else {
                    fold(n);
                }
            }
        } else {
            scale = *p.a_s * p.b_s[FORM == kWideGroupRows ? t.group * p.b_s_stride : 0];
            asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
            for (int i = 0; i < MI; i++)
#pragma unroll
                for (int j = 0; j < NJ; j++) asm volatile("" : "+v"(acc[i][j]));
        }
        if (kHolds && (t.T & 1)) held0 = held1;                  // (the next tile's first stage)
        void *out = p.out;
        if (FORM == kWideGroupDw) out = (uint8_t *)p.out + (int64_t)t.group * p.M * p.ld_out * (p.out_f32 ? 4 : 2);
#pragma unroll
        for (int i = 0; i < MI; i++)
#pragma unroll
            for (int j = 0; j < NJ; j += 2)
                store_pair(acc[i][j], acc[i][j + 1], scale, out, p.ld_out, t.m0 + wm * 16 * MI + i * 16 + r16, t.n0 + wn * 16 * NJ + j * 16, q, t.rows_end, p.N,
                           p.out_f32, p.accumulate);
    }
    wait_vmcnt<0>();   // no copy into LDS may be outstanding when the wave ends
}

template <WideForm FORM, int MI, int NJ, int SLOTS>
static int launch_wide(WideArgs p, hipStream_t st)
{
    using S = WideShape<MI, NJ, SLOTS>;
    // a stage lies inside a row, outputs are whole 16-byte pieces, offsets inside a tile have 32 bits
    constexpr int64_t kMaxLd = (int64_t)1 << 24;
    if (p.K < kWideK || p.K % kGroup || p.N % 8 || p.ld_out % 8 || p.K > kMaxLd || p.ld_b > kMaxLd || !p.a_x) return MOSS_ERR_UNSUPPORTED;
    if (S::lds_bytes(FORM, p.groups) > 160 * 1024) return MOSS_ERR_UNSUPPORTED;
    int cus = moss_internal_cu_count();
    cus = cus <= 0 ? 256 : cus >= 8 ? cus & ~7 : 8;
    const int64_t tiles_n = (p.N + S::kBN - 1) / S::kBN;
    int64_t tiles_m = (p.M + S::kBM - 1) / S::kBM, total = tiles_m * tiles_n;
    int64_t most = total;
    if (FORM == kWideGroupRows) {
        const int64_t some = p.groups < p.M ? p.groups : p.M;
        total = (p.M + some * (S::kBM - 1)) / S::kBM * tiles_n;
        most = tiles_m * p.groups * tiles_n;         // whatever the offsets are
    }
    if (FORM == kWideGroupDw) most = total * p.groups;
    if (most > 0x7FFFFFF) return MOSS_ERR_UNSUPPORTED;
    if (FORM == kWideGroupDw) {
        uint32_t longest = 0;
        for (uint32_t x = 0; x < 8; x++) {
            const uint32_t n = eighths_of((uint32_t)total, x, (uint32_t)p.groups);
            longest = n > longest ? n : longest;
        }
        total = 8 * (int64_t)longest;
    }
    p.tiles_m = (int)tiles_m;
    p.tiles_n = (int)tiles_n;
    const auto kern = k_gemm_wide<FORM, MI, NJ, SLOTS>;
    static std::atomic<bool> attr_set[64];           // per device: the LDS size it may ask for has been raised
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return MOSS_ERR_HIP;
    if (!attr_set[dev].load()) {
        if (hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != hipSuccess) {
            (void)hipGetLastError();
            return MOSS_ERR_UNSUPPORTED;
        }
        attr_set[dev].store(true);
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)(total < cus ? total : cus)), dim3(kWideThreads), (size_t)S::lds_bytes(FORM, p.groups), st, p);
    if (hipGetLastError() != hipSuccess) return MOSS_ERR_HIP;
    return MOSS_OK;
}

}  // namespace moss
