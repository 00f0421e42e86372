// What the block-scaled GEMM kernels share: vector types, direct global->LDS copies and their waits, BF16 rounding.
#pragma once
#include "moss_internal.h"

namespace moss {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

// wave-wide direct global->LDS copy: every lane moves 16 bytes from base + off to
// lds_addr + 16 * lane (lds_addr is wave-uniform and goes through M0).  A copy into LDS that follows a scalar write of M0 needs
// one wait state in between, or it may go where M0 pointed before; the compiler, which puts it there itself elsewhere, does not
// look into an asm block.
__device__ __forceinline__ void dma16(const uint8_t *base, uint32_t off, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                 :: "v"(off), "s"(base), "s"(lds_addr) : "memory", "m0");
}

// the same to lds_addr + at, which is added in the move to M0 (`at` is a constant once loops are unrolled)
__device__ __forceinline__ void dma16_at(const uint8_t *base, uint32_t off, uint32_t lds_addr, int at)
{
    asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                 :: "v"(off), "s"(base), "s"(lds_addr), "i"(at) : "memory", "m0", "scc");
}

template <int N> __device__ __forceinline__ void wait_vmcnt()
{
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory");
}

__device__ __forceinline__ void wait_lds_and_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Workgroups are dealt round-robin to the 8 XCDs: the tile of this one, so that each XCD gets a contiguous range of `total`
__device__ __forceinline__ uint32_t xcd_range_tile(uint32_t block, uint32_t total)
{
    const uint32_t q = total >> 3, r = total & 7, xcd = block & 7;
    return xcd * q + (xcd < r ? xcd : r) + (block >> 3);
}

// tile `pid` of a matrix walked in bands of 8 tile rows, column by column
__device__ __forceinline__ void band_tile(uint32_t pid, uint32_t tiles_m, uint32_t tiles_n, int &tm, int &tn)
{
    constexpr uint32_t kBand = 8;
    const uint32_t band = pid / (kBand * tiles_n), rem = pid - band * kBand * tiles_n;
    const uint32_t here = tiles_m - band * kBand < kBand ? tiles_m - band * kBand : kBand;
    tn = __builtin_amdgcn_readfirstlane((int)(rem / here));
    tm = __builtin_amdgcn_readfirstlane((int)(band * kBand + rem % here));
}

// Rows [first, end) of a group.  Offsets come from the device and cannot be checked ahead: whatever they are, the rows lie in [0, rows).
__device__ __forceinline__ void group_range(const int32_t *offsets, int group, int64_t rows, int64_t &first, int64_t &end)
{
    const int64_t a = offsets[group], b = offsets[group + 1];
    first = a < 0 ? 0 : a < rows ? a : rows;
    end = b < first ? first : b < rows ? b : rows;
}

struct GroupTile {
    int group, tm, tn;
    int64_t first, end;
};

// The tile of workgroup `block` among those of all groups, group by group, each in tiles of BM rows of its own: false if there are
// fewer.  Every wave counts for itself, a lane per group (64 groups at a time).
template <int BM>
__device__ __forceinline__ bool find_group_tile(GroupTile &t, const int32_t *offsets, int groups, int64_t rows, uint32_t tiles_n, uint32_t block)
{
    const int lane = threadIdx.x & 63;
    int64_t first = 0, end = 0;
    auto tiles_of = [&](int g) {
        first = end = 0;
        if (g < groups) group_range(offsets, g, rows, first, end);
        return (uint32_t)((end - first + BM - 1) / BM);
    };
    uint32_t total = 0;
    for (int g0 = 0; g0 < groups; g0 += kWave) total += wave_sum_u32(tiles_of(g0 + lane));
    total = (uint32_t)__builtin_amdgcn_readfirstlane((int)total) * tiles_n;
    if ((block >> 3) >= (total >> 3) + ((block & 7) < (total & 7) ? 1 : 0)) return false;
    const uint32_t pid = xcd_range_tile(block, total);
    uint32_t before = 0;                              // tiles of the groups ahead
    for (int g0 = 0; g0 < groups; g0 += kWave) {
        const uint32_t n = tiles_of(g0 + lane);
        uint32_t upto = n;                            // rows of tiles up to and with this lane's group
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const uint32_t o = (uint32_t)__shfl_up((int)upto, d, 64);
            if (lane >= d) upto += o;
        }
        const uint64_t behind = __ballot(before + upto * tiles_n > pid);
        if (behind) {
            const int at = __ffsll((unsigned long long)behind) - 1;
            auto of_lane = [&](uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, at); };
            const uint32_t rows_of_tiles = of_lane(n);
            t.group = g0 + at;
            t.first = of_lane((uint32_t)first);
            t.end = of_lane((uint32_t)end);
            band_tile(pid - (before + (of_lane(upto) - rows_of_tiles) * tiles_n), rows_of_tiles, tiles_n, t.tm, t.tn);
            return true;
        }
        before += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63) * tiles_n;
    }
    return false;
}

// Row tiles of the groups ahead of each, [groups + 1], by the first wave
template <int BM>
__device__ __forceinline__ void count_group_tiles(uint32_t *table, const int32_t *offsets, int groups, int64_t rows)
{
    const int lane = threadIdx.x & 63;
    uint32_t before = 0;
    for (int g0 = 0; g0 < groups; g0 += kWave) {
        uint32_t n = 0;
        if (g0 + lane < groups) {
            int64_t first, end;
            group_range(offsets, g0 + lane, rows, first, end);
            n = (uint32_t)((end - first + BM - 1) / BM);
        }
        uint32_t upto = n;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const uint32_t o = (uint32_t)__shfl_up((int)upto, d, 64);
            if (lane >= d) upto += o;
        }
        if (g0 + lane < groups) table[g0 + lane] = before + upto - n;
        before += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    }
    if (lane == 0) table[groups] = before;
}

// The group of tile `at` among those that `table` counts, rows of tiles ahead of it and its own
struct GroupTiles {
    int group;
    uint32_t ahead, count;
};
__device__ __forceinline__ GroupTiles group_of_tile(const uint32_t *table, int groups, uint32_t tiles_n, uint32_t at)
{
    const int lane = threadIdx.x & 63;
    int g = 0;
    for (int g0 = 0; g0 < groups; g0 += kWave) {      // groups that start at or ahead of this tile
        const int o = g0 + lane;
        g += __popcll(__ballot(o < groups && table[o < groups ? o : groups] * tiles_n <= at));
    }
    GroupTiles t;
    t.group = __builtin_amdgcn_readfirstlane(g - 1);
    t.ahead = (uint32_t)__builtin_amdgcn_readfirstlane((int)table[t.group]);
    t.count = (uint32_t)__builtin_amdgcn_readfirstlane((int)table[t.group + 1]) - t.ahead;
    return t;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// two FP32 -> two BF16 (round to nearest even), a in the low half: one V_CVT_PK_BF16_F32
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// The block-scaled matrix instruction as volatile inline assembly: volatile asm statements keep
// their program order, which is what pins "one matrix instruction, one LDS read, one global->LDS
// copy" in the main loop (compiler scheduling hints did not survive: all 16 matrix instructions
// of a substep were emitted first and the memory instructions after them in one burst).
// SEL = 0 / 2 picks scale byte 0 / 2 of both scale registers.  Independent accumulators back to
// back need no wait states; the places where results are consumed add their own (see callers).
template <int SEL>
__device__ __forceinline__ void mfma_scaled(v16f &acc, const v8i &x, const v8i &y, int sx, int sy)
{
    if (SEL == 0)
        asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]"
                     : "+a"(acc) : "v"(x), "v"(y), "v"(sx), "v"(sy));
    else
        asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[1,1,0]"
                     : "+a"(acc) : "v"(x), "v"(y), "v"(sx), "v"(sy));
}
// The unscaled instruction, from zero and on top of what is there.  Independent and accumulating instructions back to back need no
// wait states; whoever reads the result otherwise waits.
__device__ __forceinline__ void mfma_unscaled_from_zero(v16f &d, const v8i &x, const v8i &y)
{
    asm volatile("v_mfma_f32_32x32x64_f8f6f4 %0, %1, %2, 0" : "=&v"(d) : "v"(x), "v"(y));
}
__device__ __forceinline__ void mfma_unscaled(v16f &d, const v8i &x, const v8i &y)
{
    asm volatile("v_mfma_f32_32x32x64_f8f6f4 %0, %1, %2, %0" : "+v"(d) : "v"(x), "v"(y));
}
// The product of a block's two scales.  That of finite ones is kept finite, so that a block of zeros adds nothing whatever they are.  One
// that is NaN or infinite makes it NaN, so that it shows in all that it scales: scales come here with NaN for infinity
// (shown_scale, once for each that a tile loads), and these two hand NaN on.
__device__ __forceinline__ float shown_scale(float s) { return __builtin_fmaf(s, 0.0f, s); }
__device__ __forceinline__ float block_scales(float a, float b)
{
    constexpr float kMost = 3.402823466e38f;
    return __builtin_elementwise_maximum(__builtin_elementwise_minimum(a * b, kMost), -kMost);
}

__device__ __forceinline__ void pin() { asm volatile("" ::: "memory"); }

// Stores a 32 x 32 fragment of accumulators times `scale` without staging it.  Register v of lane (i32, h) is row i32, column
// 8 (v / 4) + 4 h + v % 4: four columns in a row, so that an FP32 output leaves in 16-byte pieces, 32 bytes of a row per
// instruction.  For BF16 the halves of the wave exchange every other group of four first and hold eight columns each.  The pieces
// of a line meet in the L2.  (2048 x 2048 x 512 in 128 x 128 tiles: 2.5 us to stage the
// tile in LDS and walk it and 2.0 to store it, 2.6 together this way, 10.7 -> 8.8; accumulating 17.3 -> 14.6.)  `row` is this lane's, `n` the fragment's first column.
__device__ __forceinline__ void store_fragment(const v16f &acc, float scale, void *out, int64_t ld, int64_t row, int64_t n, int h,
                                               int64_t M, int64_t N, int out_f32, int accumulate)
{
    float r[16];
#pragma unroll
    for (int v = 0; v < 16; v++) r[v] = acc[v] * scale;
    if (out_f32) {
        float *o = reinterpret_cast<float *>(out) + row * ld + n + 4 * h;
        if (n + 32 <= N && ld % 4 == 0) {            // (wave-uniform)
            if (row >= M) return;
            if (accumulate) {
                float4 q[4];
#pragma unroll
                for (int g = 0; g < 4; g++) q[g] = *reinterpret_cast<const float4 *>(o + 8 * g);
#pragma unroll
                for (int g = 0; g < 4; g++)
                    *reinterpret_cast<float4 *>(o + 8 * g) = make_float4(r[4 * g] + q[g].x, r[4 * g + 1] + q[g].y, r[4 * g + 2] + q[g].z, r[4 * g + 3] + q[g].w);
            } else {
#pragma unroll
                for (int g = 0; g < 4; g++) *reinterpret_cast<float4 *>(o + 8 * g) = make_float4(r[4 * g], r[4 * g + 1], r[4 * g + 2], r[4 * g + 3]);
            }
        } else if (row < M) {
            // the matrix ends inside the fragment, or its rows are not 16-byte aligned
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const int64_t left = N - (n + 4 * h + 8 * g);
                if (left >= 4 && ld % 4 == 0) {
                    float4 v = make_float4(r[4 * g], r[4 * g + 1], r[4 * g + 2], r[4 * g + 3]);
                    if (accumulate) {
                        const float4 q = *reinterpret_cast<const float4 *>(o + 8 * g);
                        v.x += q.x; v.y += q.y; v.z += q.z; v.w += q.w;
                    }
                    *reinterpret_cast<float4 *>(o + 8 * g) = v;
                } else {
#pragma unroll
                    for (int x = 0; x < 4; x++)
                        if (x < left) o[8 * g + x] = accumulate ? r[4 * g + x] + o[8 * g + x] : r[4 * g + x];
                }
            }
        }
        return;
    }
    uint32_t w[8];
#pragma unroll
    for (int v = 0; v < 8; v++) w[v] = pack_bf16(r[2 * v], r[2 * v + 1]);
    uint16_t *o = reinterpret_cast<uint16_t *>(out) + row * ld + n;
    if (n + 32 <= N && ld % 8 == 0) {                // (wave-uniform)
#pragma unroll
        for (int g = 0; g < 2; g++) {
            // words 4 g .. : columns 16 g + 4 h + 0 .. 3 in the first two, 16 g + 8 + 4 h in the others
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const auto both = __builtin_amdgcn_permlane32_swap(w[4 * g + k], w[4 * g + 2 + k], false, false);
                w[4 * g + k] = both[0];
                w[4 * g + 2 + k] = both[1];
            }
            if (row < M) *reinterpret_cast<uint4 *>(o + 16 * g + 8 * h) = make_uint4(w[4 * g], w[4 * g + 1], w[4 * g + 2], w[4 * g + 3]);
        }
    } else if (row < M) {
        // the matrix ends inside the fragment, or its rows are not 16-byte aligned
#pragma unroll
        for (int g = 0; g < 4; g++) {
            const int at = 8 * g + 4 * h;
            const int64_t left = N - (n + at);
            if (left >= 4 && ld % 4 == 0) {
                *reinterpret_cast<uint2 *>(o + at) = make_uint2(w[2 * g], w[2 * g + 1]);
            } else {
#pragma unroll
                for (int x = 0; x < 4; x++)
                    if (x < left) o[at + x] = (uint16_t)(w[2 * g + x / 2] >> (16 * (x & 1)));
            }
        }
    }
}

}  // namespace moss
