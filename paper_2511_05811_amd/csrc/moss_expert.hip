// The rows' way to the experts of a layer and back: a plan made from the experts that routing chose, the copy of each token's row to the
// rows of its experts (dispatch), their weighted sum (combine), and the gradients.  They surround the grouped products; rows of
// an expert are filled up with zeros to a multiple that the quantizer's groups along the rows need.
//
// Bound: HBM.  Everything goes by tokens: a token's row is read once and stays in registers while its k rows are written (dispatch) or
// multiplied (gradient of combine); rows of zeros between the experts' rows are items of their own behind the tokens.  16 bytes
// per thread, 32 to 256 threads per token by the width.  Sums and products in FP32, one rounding to BF16 at the end.  The tensors
// that a quantizer reads leave their maximum behind, as the other BF16 producers do.
#include "moss_internal.h"
#include "moss_producer.h"

namespace moss {
namespace {

constexpr int kExThreads = 256;
constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kMaxExperts = 1024;

typedef unsigned short ex_u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 ex_bf16x2 __attribute__((ext_vector_type(2)));
typedef float ex_f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t ex_pk_max(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ex_u16x2, a), __builtin_bit_cast(ex_u16x2, b)));
}
__device__ __forceinline__ uint32_t ex_pack(float a, float b)     // two FP32 -> two BF16 (RNE), a in the low half
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(ex_f32x2{a, b}, ex_bf16x2));
}
__device__ __forceinline__ float ex_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float ex_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t ex_top(uint32_t m, uint4 v)
{
    m = ex_pk_max(m, v.x & 0x7FFF7FFFu);
    m = ex_pk_max(m, v.y & 0x7FFF7FFFu);
    m = ex_pk_max(m, v.z & 0x7FFF7FFFu);
    return ex_pk_max(m, v.w & 0x7FFF7FFFu);
}

// The plan, by one workgroup.  Every wave has a contiguous part of the assignments and counts it per expert; a scan over
// experts and waves gives each (wave, expert) its first row; then every wave walks its part again.  Of 64 assignments at a time, those of the
// same expert are found bit by bit of its number with ballots, so that each knows how many are ahead of it and the order is kept.
__global__ __launch_bounds__(kPlanThreads) void k_expert_plan(const int32_t *__restrict__ experts, int64_t n, int E, int bits, int multiple, int64_t rows,
                                                              int32_t *__restrict__ row_of, int32_t *__restrict__ source, int32_t *__restrict__ offsets)
{
    extern __shared__ int32_t first[];                // [waves][E]: counts, then first rows
    __shared__ int32_t sums[kPlanWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t steps = (n + kWave - 1) / kWave, per = (steps + kPlanWaves - 1) / kPlanWaves;
    const int64_t from = wave * per * kWave, to = from + per * kWave < n ? from + per * kWave : n;
    for (int i = tid; i < kPlanWaves * E; i += kPlanThreads) first[i] = 0;
    __syncthreads();
    auto expert_at = [&](int64_t a) {
        const int e = a < to ? experts[a] : -1;
        return e >= 0 && e < E ? e : -1;
    };
    // lanes of the wave with the same expert (those without one are with each other)
    auto same = [&](int e) {
        uint64_t m = __ballot(e >= 0);
        if (e < 0) m = ~m;
        for (int b = 0; b < bits; b++) {
            const uint64_t set = __ballot((e >> b) & 1);
            m &= (e >> b) & 1 ? set : ~set;
        }
        return m;
    };
    for (int64_t a0 = from; a0 < to; a0 += kWave) {
        const int e = expert_at(a0 + lane);
        if (e >= 0) atomicAdd(&first[wave * E + e], 1);           // (the wave's own counters)
    }
    __syncthreads();
    // thread e: rows of expert e, filled up; scan over the threads
    int count = 0, filled = 0;
    if (tid < E) {
        for (int w = 0; w < kPlanWaves; w++) {
            const int c = first[w * E + tid];
            first[w * E + tid] = count;
            count += c;
        }
        filled = (count + multiple - 1) / multiple * multiple;
    }
    int upto = filled;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int o = __shfl_up(upto, d, 64);
        if (lane >= d) upto += o;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; w++) upto += sums[w];
    if (tid < E) {
        const int start = upto - filled;
        for (int w = 0; w < kPlanWaves; w++) first[w * E + tid] += start;
        offsets[tid] = start;
        if (tid == E - 1) offsets[E] = (int32_t)rows;
        for (int r = start + count; r < upto; r++) source[r] = -1;
    }
    __syncthreads();
    int all = 0;
    for (int w = 0; w < kPlanWaves; w++) all += sums[w];
    for (int64_t r = all + tid; r < rows; r += kPlanThreads) source[r] = -1;
    for (int64_t a0 = from; a0 < to; a0 += kWave) {
        const int64_t a = a0 + lane;
        const int e = expert_at(a);
        const uint64_t mine = same(e);
        const int ahead = __popcll(mine & ((1ull << lane) - 1));
        int row = -1;
        if (e >= 0) {
            row = first[wave * E + e] + ahead;
            source[row] = (int32_t)a;
        }
        if (a < to) row_of[a] = row;
        __builtin_amdgcn_wave_barrier();                          // (all lanes have read their counters)
        if (e >= 0 && ahead == 0) first[wave * E + e] += __popcll(mine);
        __builtin_amdgcn_wave_barrier();
    }
}

__global__ void k_expert_clear(uint32_t *a)
{
    if (threadIdx.x == 0) *a = 0;
}

__device__ __forceinline__ void finish_max(uint32_t m, uint32_t *word, int look, const MaxSlots &slots)
{
    __shared__ uint32_t red[kExThreads / kWave];
    m = (m & 0xFFFFu) > (m >> 16) ? (m & 0xFFFFu) : (m >> 16);
    m = wave_max_u32(m);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int i = 1; i < kExThreads / kWave; i++) m = red[i] > m ? red[i] : m;
    if (slots.call) {
        const uint32_t top[1] = {m};
        uint32_t *const out[1] = {word};
        finish_max_in_slots<1, kExThreads>(slots, top, out, red);
        return;
    }
    if (threadIdx.x == 0) merge_max_word(word, m, look_at_word(word, look));
}

struct ExArgs {
    const uint16_t *x;               // dispatch: token rows; combine: the experts' rows; gradient of combine: d_out
    const uint16_t *y;               // gradient of combine: the experts' rows
    const int32_t *row_of, *source;
    const float *weights;
    int64_t tokens, rows;
    int k, chunks;                   // choices per token, 16-byte chunks per row
    int64_t ld_x, ld_y, ld_out;
    uint16_t *out;
    float *d_weights;
    uint32_t *top;
    int flags;
};

__device__ __forceinline__ bool row_ok(int r, int64_t rows) { return r >= 0 && r < rows; }

// Tokens, then rows without one (zeros).  GRAD: gradient of combine, else dispatch.
template <bool GRAD, int LANES>
__global__ __launch_bounds__(kExThreads) void k_expert_scatter(const ExArgs p, MaxSlots slots)
{
    constexpr int kItems = kExThreads / LANES;
    __shared__ float part[GRAD && LANES > kWave ? kExThreads / kWave : 1];
    const int sub = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    uint32_t m = 0;
    for (int64_t i0 = (int64_t)blockIdx.x * kItems; i0 < p.tokens + p.rows; i0 += (int64_t)gridDim.x * kItems) {
        const int64_t i = i0 + slot;
        if (i >= p.tokens) {
            const int64_t r = i - p.tokens;
            if (r < p.rows) {
                const int a = p.source[r];
                if (!(a >= 0 && a < p.tokens * p.k))
                    for (int c = sub; c < p.chunks; c += LANES) st_producer16(p.out + r * p.ld_out + (int64_t)c * 8, make_uint4(0, 0, 0, 0), p.flags & kProducerStream);
            }
        }
        const bool token = i < p.tokens;
        if (!GRAD) {
            if (!token) continue;
            for (int c = sub; c < p.chunks; c += LANES) {
                const uint4 v = ld_stream16(p.x + i * p.ld_x + (int64_t)c * 8);
                bool used = false;
                for (int j = 0; j < p.k; j++) {
                    const int r = p.row_of[i * p.k + j];
                    if (!row_ok(r, p.rows)) continue;
                    used = true;
                    st_producer16(p.out + (int64_t)r * p.ld_out + (int64_t)c * 8, v, p.flags & kProducerStream);
                }
                if (used) m = ex_top(m, v);
            }
            continue;
        }
        for (int j = 0; j < p.k; j++) {
            float dot = 0.0f;
            if (token) {
                const int r = p.row_of[i * p.k + j];
                if (row_ok(r, p.rows)) {
                    const float w = p.weights[i * p.k + j];
                    for (int c = sub; c < p.chunks; c += LANES) {
                        const uint4 g = *reinterpret_cast<const uint4 *>(p.x + i * p.ld_x + (int64_t)c * 8);
                        const uint4 v = ld_stream16(p.y + (int64_t)r * p.ld_y + (int64_t)c * 8);
                        const uint32_t a[4] = {g.x, g.y, g.z, g.w}, b[4] = {v.x, v.y, v.z, v.w};
                        uint32_t o[4];
#pragma unroll
                        for (int q = 0; q < 4; q++) {
                            dot += ex_lo(a[q]) * ex_lo(b[q]) + ex_hi(a[q]) * ex_hi(b[q]);
                            o[q] = ex_pack(w * ex_lo(a[q]), w * ex_hi(a[q]));
                        }
                        const uint4 d = make_uint4(o[0], o[1], o[2], o[3]);
                        m = ex_top(m, d);
                        st_producer16(p.out + (int64_t)r * p.ld_out + (int64_t)c * 8, d, p.flags & kProducerStream);
                    }
                }
            }
#pragma unroll
            for (int d = (LANES < kWave ? LANES : kWave) / 2; d > 0; d >>= 1) dot += __shfl_xor(dot, d, 64);
            if (LANES > kWave) {
                __syncthreads();
                if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = dot;
                __syncthreads();
                dot = 0.0f;
#pragma unroll
                for (int w = 0; w < LANES / kWave; w++) dot += part[slot * (LANES / kWave) + w];
            }
            if (token && sub == 0) p.d_weights[i * p.k + j] = dot;
        }
    }
    finish_max(m, p.top, p.flags & kProducerLook, slots);
}

// out[t] = sum over j of weights[t, j] * x[row_of[t, j]], in the order of j; WEIGHTS false: the plain sum (gradient of dispatch)
template <bool WEIGHTS, int LANES>
__global__ __launch_bounds__(kExThreads) void k_expert_combine(const ExArgs p)
{
    constexpr int kItems = kExThreads / LANES;
    const int sub = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    for (int64_t i = (int64_t)blockIdx.x * kItems + slot; i < p.tokens; i += (int64_t)gridDim.x * kItems) {
        for (int c = sub; c < p.chunks; c += LANES) {
            float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            for (int j = 0; j < p.k; j++) {
                const int r = p.row_of[i * p.k + j];
                if (!row_ok(r, p.rows)) continue;
                const uint4 v = ld_stream16(p.x + (int64_t)r * p.ld_x + (int64_t)c * 8);
                const uint32_t a[4] = {v.x, v.y, v.z, v.w};
                const float w = WEIGHTS ? p.weights[i * p.k + j] : 1.0f;
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    s[2 * q] += w * ex_lo(a[q]);
                    s[2 * q + 1] += w * ex_hi(a[q]);
                }
            }
            const uint4 o = make_uint4(ex_pack(s[0], s[1]), ex_pack(s[2], s[3]), ex_pack(s[4], s[5]), ex_pack(s[6], s[7]));
            st_producer16(p.out + i * p.ld_out + (int64_t)c * 8, o, p.flags & kProducerStream);
        }
    }
}

int lanes_for(int chunks) { return chunks <= 32 ? 32 : chunks <= 64 ? 64 : chunks <= 128 ? 128 : 256; }

int64_t device_cus()
{
    const int cus = moss_internal_cu_count();
    return cus <= 0 ? 256 : cus;
}

int items_grid(int64_t items, int lanes)
{
    const int64_t wgs = (items + kExThreads / lanes - 1) / (kExThreads / lanes), most = device_cus() * 4;
    return (int)(wgs < most ? wgs : most);
}

// what every call over rows and tokens checks
int check_rows(int64_t tokens, int64_t k, int64_t rows, int64_t cols, int64_t ld_tokens, int64_t ld_rows)
{
    if (tokens <= 0 || k <= 0 || rows <= 0 || cols <= 0 || cols % 8 || ld_tokens < cols || ld_rows < cols) return MOSS_ERR_SHAPE;
    if (tokens > 0x7FFFFFFF / k || rows > 0x7FFFFFFF || cols > ((int64_t)1 << 30)) return MOSS_ERR_SHAPE;
    return ld_tokens % 8 || ld_rows % 8 ? MOSS_ERR_ALIGN : MOSS_OK;
}

#define MOSS_EX_LANES(kernel_of, ...)                                                    \
    switch (lanes) {                                                                      \
        case 32: hipLaunchKernelGGL((kernel_of(32)), __VA_ARGS__); break;                  \
        case 64: hipLaunchKernelGGL((kernel_of(64)), __VA_ARGS__); break;                  \
        case 128: hipLaunchKernelGGL((kernel_of(128)), __VA_ARGS__); break;                \
        default: hipLaunchKernelGGL((kernel_of(256)), __VA_ARGS__); break;                 \
    }

template <bool GRAD>
int launch_scatter(ExArgs p, void *workspace, size_t workspace_bytes, hipStream_t st)
{
    const int lanes = lanes_for(p.chunks), grid = items_grid(p.tokens + p.rows, lanes);
    p.flags = producer_flags(p.rows, (int64_t)p.chunks * 8, true);
    const MaxSlots slots = max_slots(workspace, workspace_bytes, grid, 1, st);
    if (!slots.call) {
        hipLaunchKernelGGL(k_expert_clear, dim3(1), dim3(64), 0, st, p.top);
        MOSS_LAUNCH_CHECK();
    }
#define MOSS_EX_KERNEL(L) k_expert_scatter<GRAD, L>
    MOSS_EX_LANES(MOSS_EX_KERNEL, dim3(grid), dim3(kExThreads), 0, st, p, slots)
#undef MOSS_EX_KERNEL
    MOSS_LAUNCH_CHECK();
    return MOSS_OK;
}

template <bool WEIGHTS>
int launch_combine(ExArgs p, hipStream_t st)
{
    const int lanes = lanes_for(p.chunks), grid = items_grid(p.tokens, lanes);
    p.flags = producer_flags(p.tokens, (int64_t)p.chunks * 8, false);
#define MOSS_EX_KERNEL(L) k_expert_combine<WEIGHTS, L>
    MOSS_EX_LANES(MOSS_EX_KERNEL, dim3(grid), dim3(kExThreads), 0, st, p)
#undef MOSS_EX_KERNEL
    MOSS_LAUNCH_CHECK();
    return MOSS_OK;
}

}  // namespace
}  // namespace moss

extern "C" int64_t moss_expert_rows(int64_t tokens, int64_t k, int64_t experts, int64_t multiple)
{
    if (tokens <= 0 || k <= 0 || experts <= 0 || multiple <= 0 || tokens > 0x7FFFFFFF / k || experts > 0x7FFFFFFF || multiple > 0x7FFFFFFF) return 0;
    const int64_t n = tokens * k;
    return (n + (experts < n ? experts : n) * (multiple - 1)) / multiple * multiple;
}

extern "C" int moss_expert_plan(const int32_t *experts, int64_t tokens, int64_t k, int64_t n_experts, int64_t multiple, int64_t rows,
                                int32_t *row_of, int32_t *source, int32_t *offsets, void *stream)
{
    using namespace moss;
    if (!experts || !row_of || !source || !offsets) return MOSS_ERR_NULL;
    if (rows <= 0 || rows > 0x7FFFFFFF || moss_expert_rows(tokens, k, n_experts, multiple) == 0) return MOSS_ERR_SHAPE;
    if (n_experts > kMaxExperts || multiple > 4096) return MOSS_ERR_UNSUPPORTED;
    if (rows < moss_expert_rows(tokens, k, n_experts, multiple) || rows % multiple) return MOSS_ERR_SHAPE;
    if (((uintptr_t)experts | (uintptr_t)row_of | (uintptr_t)source | (uintptr_t)offsets) & 3) return MOSS_ERR_ALIGN;
    int bits = 0;
    while ((1 << bits) < n_experts) bits++;
    const size_t lds = (size_t)kPlanWaves * n_experts * 4;
    hipStream_t st = (hipStream_t)stream;
    if (lds > 48 * 1024) {
        if (hipFuncSetAttribute((const void *)k_expert_plan, hipFuncAttributeMaxDynamicSharedMemorySize, kPlanWaves * kMaxExperts * 4) != hipSuccess) {
            (void)hipGetLastError();
            return MOSS_ERR_HIP;
        }
    }
    hipLaunchKernelGGL(k_expert_plan, dim3(1), dim3(kPlanThreads), lds, st, experts, tokens * k, (int)n_experts, bits, (int)multiple, rows,
                       row_of, source, offsets);
    MOSS_LAUNCH_CHECK();
    return MOSS_OK;
}

extern "C" int moss_expert_dispatch_bf16(const void *x, const int32_t *row_of, const int32_t *source, int64_t tokens, int64_t k, int64_t rows,
                                         int64_t cols, int64_t ld_x, int64_t ld_y, void *y, uint32_t *y_absmax_bits, void *stream)
{
    return moss_internal_expert_dispatch_bf16(x, row_of, source, tokens, k, rows, cols, ld_x, ld_y, y, y_absmax_bits, nullptr, 0, stream);
}

extern "C" int moss_internal_expert_dispatch_bf16(const void *x, const int32_t *row_of, const int32_t *source, int64_t tokens, int64_t k,
                                                  int64_t rows, int64_t cols, int64_t ld_x, int64_t ld_y, void *y, uint32_t *y_absmax_bits,
                                                  void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace moss;
    if (!x || !row_of || !source || !y || !y_absmax_bits) return MOSS_ERR_NULL;
    const int rc = check_rows(tokens, k, rows, cols, ld_x, ld_y);
    if (rc) return rc;
    if (!moss_aligned16(x) || !moss_aligned16(y) || (((uintptr_t)row_of | (uintptr_t)source | (uintptr_t)y_absmax_bits) & 3)) return MOSS_ERR_ALIGN;
    ExArgs p{};
    p.x = (const uint16_t *)x; p.row_of = row_of; p.source = source;
    p.tokens = tokens; p.rows = rows; p.k = (int)k; p.chunks = (int)(cols / 8);
    p.ld_x = ld_x; p.ld_out = ld_y;
    p.out = (uint16_t *)y; p.top = y_absmax_bits;
    return launch_scatter<false>(p, workspace, workspace_bytes, (hipStream_t)stream);
}

extern "C" int moss_expert_combine_bf16(const void *y, const int32_t *row_of, const float *weights, int64_t tokens, int64_t k, int64_t rows,
                                        int64_t cols, int64_t ld_y, int64_t ld_out, void *out, void *stream)
{
    using namespace moss;
    if (!y || !row_of || !out) return MOSS_ERR_NULL;
    const int rc = check_rows(tokens, k, rows, cols, ld_out, ld_y);
    if (rc) return rc;
    if (!moss_aligned16(y) || !moss_aligned16(out) || (((uintptr_t)row_of | (uintptr_t)weights) & 3)) return MOSS_ERR_ALIGN;
    ExArgs p{};
    p.x = (const uint16_t *)y; p.row_of = row_of; p.weights = weights;
    p.tokens = tokens; p.rows = rows; p.k = (int)k; p.chunks = (int)(cols / 8);
    p.ld_x = ld_y; p.ld_out = ld_out;
    p.out = (uint16_t *)out;
    return weights ? launch_combine<true>(p, (hipStream_t)stream) : launch_combine<false>(p, (hipStream_t)stream);
}

extern "C" int moss_expert_combine_bf16_backward(const void *d_out, const void *y, const int32_t *row_of, const int32_t *source, const float *weights,
                                                 int64_t tokens, int64_t k, int64_t rows, int64_t cols, int64_t ld_out, int64_t ld_y, void *d_y,
                                                 float *d_weights, uint32_t *d_y_absmax_bits, void *stream)
{
    return moss_internal_expert_combine_bf16_backward(d_out, y, row_of, source, weights, tokens, k, rows, cols, ld_out, ld_y, d_y, d_weights,
                                                      d_y_absmax_bits, nullptr, 0, stream);
}

extern "C" int moss_internal_expert_combine_bf16_backward(const void *d_out, const void *y, const int32_t *row_of, const int32_t *source,
                                                          const float *weights, int64_t tokens, int64_t k, int64_t rows, int64_t cols,
                                                          int64_t ld_out, int64_t ld_y, void *d_y, float *d_weights, uint32_t *d_y_absmax_bits,
                                                          void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace moss;
    if (!d_out || !y || !row_of || !source || !weights || !d_y || !d_weights || !d_y_absmax_bits) return MOSS_ERR_NULL;
    const int rc = check_rows(tokens, k, rows, cols, ld_out, ld_y);
    if (rc) return rc;
    if (!moss_aligned16(d_out) || !moss_aligned16(y) || !moss_aligned16(d_y)) return MOSS_ERR_ALIGN;
    if (((uintptr_t)row_of | (uintptr_t)source | (uintptr_t)weights | (uintptr_t)d_weights | (uintptr_t)d_y_absmax_bits) & 3) return MOSS_ERR_ALIGN;
    ExArgs p{};
    p.x = (const uint16_t *)d_out; p.y = (const uint16_t *)y; p.row_of = row_of; p.source = source; p.weights = weights;
    p.tokens = tokens; p.rows = rows; p.k = (int)k; p.chunks = (int)(cols / 8);
    p.ld_x = ld_out; p.ld_y = ld_y; p.ld_out = ld_y;
    p.out = (uint16_t *)d_y; p.d_weights = d_weights; p.top = d_y_absmax_bits;
    return launch_scatter<true>(p, workspace, workspace_bytes, (hipStream_t)stream);
}
