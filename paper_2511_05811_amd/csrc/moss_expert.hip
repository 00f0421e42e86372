// The rows' way to the experts of a layer and back: a plan made from the experts that routing chose, the copy of each token's row to the
// rows of its experts (dispatch), their weighted sum (combine), and the gradients.  They surround the grouped products; rows of
// an expert are filled up with zeros to a multiple that the quantizer's groups along the rows need.
//
// Bound: HBM.  Everything goes by tokens: a token's row is read once and stays in registers while its k rows are written (dispatch) or
// multiplied (gradient of combine); rows of zeros between the experts' rows are items of their own behind the tokens.  16 bytes
// per thread, half a wave or a wave per token.  Sums and products in FP32, one rounding to BF16 at the end.  The tensors
// that a quantizer reads leave their maximum behind, as the other BF16 producers do.
//
// 8192 tokens of 4096 columns, two of 64 experts each, one behind the other again and again (median, and the fastest of twelve): plan 9.1 us (8.6),
// dispatch 47.4 (41.0), combine 39.3 (35.4), its gradient 77.4 (75.9), that of dispatch 39.5 (36.4): 213 (197) for what is 940 MB at
// least, 4.4 TB/s (4.8), a large copy 5.1; the five calls take 214.  (Four chunks of a row under way per thread, two or eight are slower.)
// 64 tokens of 256: 3 to 5 us each, a launch and two or three trips to memory behind one another.
#include "moss_internal.h"
#include "moss_producer.h"

namespace moss {
namespace {

constexpr int kExThreads = 256;
constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kPlanMaxWgs = 64;
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

// The rows of an expert with `total` assignments.  They fit 31 bits (moss_expert_rows, which the capacity is held to), the sum on the
// way there does not.
__host__ __device__ __forceinline__ int filled_rows(int total, int multiple)
{
    const uint32_t m = (uint32_t)multiple;
    return (int)(((uint32_t)total + m - 1) / m * m);
}

// The plan.  A workgroup places a contiguous part of the assignments, and counts all of them per expert for itself: those ahead of its
// part, its own wave by wave, and those behind.  So the workgroups need nothing of each other.  A scan over experts and waves gives
// each (wave, expert) its first row; then every wave walks its part again.  Of 64 assignments at a time, those of the same expert are
// found bit by bit of its number with ballots, so that each knows how many are ahead of it and the order is kept.
// (One workgroup for all: 16384 assignments 16 us.)
__global__ __launch_bounds__(kPlanThreads) void k_expert_plan(const int32_t *__restrict__ experts, int64_t n, int E, int bits, int multiple, int64_t rows,
                                                              int64_t part, int32_t *__restrict__ row_of, int32_t *__restrict__ source,
                                                              int32_t *__restrict__ offsets)
{
    extern __shared__ int32_t first[];                // [waves][E]: counts, then first rows
    int32_t *ahead_of_us = first + kPlanWaves * E, *behind_us = ahead_of_us + E;
    __shared__ int32_t sums[kPlanWaves];
    constexpr int kAhead = 8;                         // (a step is a trip to memory: eight are under way together)
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t begin = (int64_t)blockIdx.x * part, end = begin + part < n ? begin + part : n;
    const int64_t per = ((end - begin + kWave - 1) / kWave + kPlanWaves - 1) / kPlanWaves * kWave;
    const int64_t from = begin + wave * per < end ? begin + wave * per : end, to = from + per < end ? from + per : end;
    for (int i = tid; i < (kPlanWaves + 2) * E; i += kPlanThreads) first[i] = 0;
    __syncthreads();
    // the experts of assignments a0, a0 + stride, ..., -1 for none
    auto load_experts = [&](int (&e)[kAhead], int64_t a0, int stride, int64_t stop) {
#pragma unroll
        for (int u = 0; u < kAhead; u++) e[u] = a0 + u * stride < stop ? experts[a0 + u * stride] : -1;
#pragma unroll
        for (int u = 0; u < kAhead; u++) e[u] = e[u] < E && e[u] >= 0 ? e[u] : -1;
    };
    auto count = [&](int32_t *into, int64_t start, int64_t stop, int stride, int64_t batch) {
        for (int64_t a = start; a < stop; a += batch) {
            int e[kAhead];
            load_experts(e, a, stride, stop);
#pragma unroll
            for (int u = 0; u < kAhead; u++)
                if (e[u] >= 0) atomicAdd(&into[e[u]], 1);
        }
    };
    count(ahead_of_us, tid, begin, kPlanThreads, (int64_t)kPlanThreads * kAhead);
    count(behind_us, end + tid, n, kPlanThreads, (int64_t)kPlanThreads * kAhead);
    count(first + wave * E, from + lane, to, kWave, (int64_t)kWave * kAhead);
    __syncthreads();
    // thread e: rows of expert e, filled up; scan over the threads
    int total = 0, filled = 0;
    if (tid < E) {
        total = ahead_of_us[tid];
        for (int w = 0; w < kPlanWaves; w++) {
            const int c = first[w * E + tid];
            first[w * E + tid] = total;
            total += c;
        }
        total += behind_us[tid];
        filled = filled_rows(total, multiple);
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
        if (blockIdx.x == 0) {
            offsets[tid] = start;
            if (tid == E - 1) offsets[E] = (int32_t)rows;
        }
        if (tid % gridDim.x == blockIdx.x)
            for (int r = start + total; r < upto; r++) source[r] = -1;
    }
    __syncthreads();
    int all = 0;
    for (int w = 0; w < kPlanWaves; w++) all += sums[w];
    for (int64_t r = all + (int64_t)blockIdx.x * kPlanThreads + tid; r < rows; r += (int64_t)gridDim.x * kPlanThreads) source[r] = -1;
    for (int64_t a0 = from; a0 < to; a0 += kWave * kAhead) {
        int es[kAhead];
        load_experts(es, a0 + lane, kWave, to);
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            if (a0 + u * kWave >= to) break;
            const int64_t a = a0 + u * kWave + lane;
            const int e = es[u];
            // lanes of the wave with the same expert (those without one are with each other)
            uint64_t mine = __ballot(e >= 0);
            if (e < 0) mine = ~mine;
            for (int b = 0; b < bits; b++) {
                const uint64_t set = __ballot((e >> b) & 1);
                mine &= (e >> b) & 1 ? set : ~set;
            }
            const int ahead = __popcll(mine & ((1ull << lane) - 1));
            int row = -1;
            if (e >= 0) {
                row = first[wave * E + e] + ahead;
                source[row] = (int32_t)a;
            }
            if (a < to) row_of[a] = row;
            __builtin_amdgcn_wave_barrier();                      // (all lanes have read their counters)
            if (e >= 0 && ahead == 0) first[wave * E + e] += __popcll(mine);
            __builtin_amdgcn_wave_barrier();
        }
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

__device__ __forceinline__ int row_or_none(int r, int64_t rows) { return r >= 0 && r < rows ? r : -1; }

// A token is worked on by LANES threads of one wave, which have kDeep chunks of each row under way; of its choices K at a time.
constexpr int kDeep = 4;

template <int K>
__device__ __forceinline__ void load_rows(int (&r)[K], const ExArgs &p, int64_t token, int j0)
{
#pragma unroll
    for (int j = 0; j < K; j++) r[j] = j0 + j < p.k ? row_or_none(p.row_of[token * p.k + j0 + j], p.rows) : -1;
}

// Tokens, then rows without one (zeros).  GRAD: gradient of combine, else dispatch.
template <bool GRAD, int LANES, int K>
__global__ __launch_bounds__(kExThreads) void k_expert_scatter(const ExArgs p, MaxSlots slots)
{
    constexpr int kItems = kExThreads / LANES;
    const int sub = threadIdx.x % LANES, slot = threadIdx.x / LANES, stream = p.flags & kProducerStream;
    uint32_t m = 0;
    for (int64_t i = (int64_t)blockIdx.x * kItems + slot; i < p.tokens + p.rows; i += (int64_t)gridDim.x * kItems) {
        if (i >= p.tokens) {
            const int64_t r = i - p.tokens;
            const int a = p.source[r];
            if (!(a >= 0 && a < p.tokens * p.k))
                for (int c = sub; c < p.chunks; c += LANES) st_producer16(p.out + r * p.ld_out + (int64_t)c * 8, make_uint4(0, 0, 0, 0), stream);
            continue;
        }
        const uint16_t *x = p.x + i * p.ld_x;
        for (int j0 = 0; j0 < p.k; j0 += K) {
            int r[K];
            load_rows(r, p, i, j0);
            float w[K], dot[K];
#pragma unroll
            for (int j = 0; j < K; j++) {
                w[j] = GRAD && r[j] >= 0 ? p.weights[i * p.k + j0 + j] : 0.0f;
                dot[j] = 0.0f;
            }
            for (int c0 = sub; c0 < p.chunks; c0 += LANES * kDeep) {
                uint4 g[kDeep], v[kDeep][GRAD ? K : 1];
#pragma unroll
                for (int u = 0; u < kDeep; u++) {
                    const int c = c0 + u * LANES;
                    if (c >= p.chunks) continue;
                    g[u] = *reinterpret_cast<const uint4 *>(x + (int64_t)c * 8);
                    if (GRAD)
#pragma unroll
                        for (int j = 0; j < K; j++)
                            if (r[j] >= 0) v[u][GRAD ? j : 0] = ld_stream16(p.y + (int64_t)r[j] * p.ld_y + (int64_t)c * 8);
                }
#pragma unroll
                for (int u = 0; u < kDeep; u++) {
                    const int c = c0 + u * LANES;
                    if (c >= p.chunks) continue;
#pragma unroll
                    for (int j = 0; j < K; j++) {
                        if (r[j] < 0) continue;
                        uint4 d = g[u];
                        if (GRAD) {
                            const uint4 t = v[u][GRAD ? j : 0];
                            const uint32_t a[4] = {g[u].x, g[u].y, g[u].z, g[u].w}, b[4] = {t.x, t.y, t.z, t.w};
                            uint32_t o[4];
#pragma unroll
                            for (int q = 0; q < 4; q++) {
                                dot[j] += ex_lo(a[q]) * ex_lo(b[q]) + ex_hi(a[q]) * ex_hi(b[q]);
                                o[q] = ex_pack(w[j] * ex_lo(a[q]), w[j] * ex_hi(a[q]));
                            }
                            d = make_uint4(o[0], o[1], o[2], o[3]);
                        }
                        m = ex_top(m, d);
                        st_producer16(p.out + (int64_t)r[j] * p.ld_out + (int64_t)c * 8, d, stream);
                    }
                }
            }
            if (GRAD) {
#pragma unroll
                for (int j = 0; j < K; j++) {
#pragma unroll
                    for (int d = LANES / 2; d > 0; d >>= 1) dot[j] += __shfl_xor(dot[j], d, 64);
                    if (sub == 0 && j0 + j < p.k) p.d_weights[i * p.k + j0 + j] = dot[j];
                }
            }
        }
    }
    finish_max(m, p.top, p.flags & kProducerLook, slots);
}

// out[t] = sum over j of weights[t, j] * x[row_of[t, j]], in the order of j; WEIGHTS false: the plain sum (gradient of dispatch)
template <bool WEIGHTS, int LANES, int K>
__global__ __launch_bounds__(kExThreads) void k_expert_combine(const ExArgs p)
{
    constexpr int kItems = kExThreads / LANES;
    const int sub = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    for (int64_t i = (int64_t)blockIdx.x * kItems + slot; i < p.tokens; i += (int64_t)gridDim.x * kItems) {
        for (int c0 = sub; c0 < p.chunks; c0 += LANES * kDeep) {
            float s[kDeep][8];
#pragma unroll
            for (int u = 0; u < kDeep; u++)
#pragma unroll
                for (int q = 0; q < 8; q++) s[u][q] = 0.0f;
            for (int j0 = 0; j0 < p.k; j0 += K) {
                int r[K];
                load_rows(r, p, i, j0);
                uint4 v[kDeep][K];
#pragma unroll
                for (int j = 0; j < K; j++)
#pragma unroll
                    for (int u = 0; u < kDeep; u++)
                        if (r[j] >= 0 && c0 + u * LANES < p.chunks) v[u][j] = ld_stream16(p.x + (int64_t)r[j] * p.ld_x + (int64_t)(c0 + u * LANES) * 8);
#pragma unroll
                for (int j = 0; j < K; j++) {
                    if (r[j] < 0) continue;
                    const float w = WEIGHTS ? p.weights[i * p.k + j0 + j] : 1.0f;
#pragma unroll
                    for (int u = 0; u < kDeep; u++) {
                        if (c0 + u * LANES >= p.chunks) continue;
                        const uint32_t a[4] = {v[u][j].x, v[u][j].y, v[u][j].z, v[u][j].w};
#pragma unroll
                        for (int q = 0; q < 4; q++) {
                            s[u][2 * q] += w * ex_lo(a[q]);
                            s[u][2 * q + 1] += w * ex_hi(a[q]);
                        }
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kDeep; u++) {
                const int c = c0 + u * LANES;
                if (c >= p.chunks) continue;
                const uint4 o = make_uint4(ex_pack(s[u][0], s[u][1]), ex_pack(s[u][2], s[u][3]), ex_pack(s[u][4], s[u][5]), ex_pack(s[u][6], s[u][7]));
                st_producer16(p.out + i * p.ld_out + (int64_t)c * 8, o, p.flags & kProducerStream);
            }
        }
    }
}

int64_t device_cus()
{
    const int cus = moss_internal_cu_count();
    return cus <= 0 ? 256 : cus;
}

int items_grid(int64_t items, int lanes)
{
    const int64_t wgs = (items + kExThreads / lanes - 1) / (kExThreads / lanes), most = device_cus() * 8;
    return (int)(wgs < most ? wgs : most);
}

// what every call over rows and tokens checks
int check_rows(int64_t tokens, int64_t k, int64_t rows, int64_t cols, int64_t ld_tokens, int64_t ld_rows)
{
    if (tokens <= 0 || k <= 0 || rows <= 0 || cols <= 0 || cols % 8 || ld_tokens < cols || ld_rows < cols) return MOSS_ERR_SHAPE;
    if (tokens > 0x7FFFFFFF / k || rows > 0x7FFFFFFF || cols > ((int64_t)1 << 30)) return MOSS_ERR_SHAPE;
    return ld_tokens % 8 || ld_rows % 8 ? MOSS_ERR_ALIGN : MOSS_OK;
}

// the kernel of a width and a number of choices
#define MOSS_EX_PICK(kernel, flag)                                                                                             \
    (p.k == 1 ? (lanes == 32 ? kernel<flag, 32, 1> : kernel<flag, 64, 1>)                                                       \
              : p.k == 2 ? (lanes == 32 ? kernel<flag, 32, 2> : kernel<flag, 64, 2>) : (lanes == 32 ? kernel<flag, 32, 4> : kernel<flag, 64, 4>))

template <bool GRAD>
int launch_scatter(ExArgs p, void *workspace, size_t workspace_bytes, hipStream_t st)
{
    const int lanes = p.chunks <= 32 ? 32 : 64, grid = items_grid(p.tokens + p.rows, lanes);
    p.flags = producer_flags(p.rows, (int64_t)p.chunks * 8, true);
    const MaxSlots slots = max_slots(workspace, workspace_bytes, grid, 1, st);
    if (!slots.call) {
        hipLaunchKernelGGL(k_expert_clear, dim3(1), dim3(64), 0, st, p.top);
        MOSS_LAUNCH_CHECK();
    }
    hipLaunchKernelGGL(MOSS_EX_PICK(k_expert_scatter, GRAD), dim3(grid), dim3(kExThreads), 0, st, p, slots);
    MOSS_LAUNCH_CHECK();
    return MOSS_OK;
}

template <bool WEIGHTS>
int launch_combine(ExArgs p, hipStream_t st)
{
    const int lanes = p.chunks <= 32 ? 32 : 64, grid = items_grid(p.tokens, lanes);
    p.flags = producer_flags(p.tokens, (int64_t)p.chunks * 8, false);
    hipLaunchKernelGGL(MOSS_EX_PICK(k_expert_combine, WEIGHTS), dim3(grid), dim3(kExThreads), 0, st, p);
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

// The rows that the plan gives an expert with so many assignments (asked by the tests)
extern "C" int64_t moss_internal_expert_filled(int64_t total, int64_t multiple) { return moss::filled_rows((int)total, (int)multiple); }

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
    const size_t lds = (size_t)(kPlanWaves + 2) * n_experts * 4;
    hipStream_t st = (hipStream_t)stream;
    if (lds > 48 * 1024) {
        if (hipFuncSetAttribute((const void *)k_expert_plan, hipFuncAttributeMaxDynamicSharedMemorySize, (kPlanWaves + 2) * kMaxExperts * 4) != hipSuccess) {
            (void)hipGetLastError();
            return MOSS_ERR_HIP;
        }
    }
    // a thousand assignments each, but no more workgroups than it pays to count everything for
    const int64_t n = tokens * k, wanted = (n + kPlanThreads - 1) / kPlanThreads, wgs = wanted < kPlanMaxWgs ? wanted : kPlanMaxWgs;
    const int64_t part = (n + wgs - 1) / wgs;
    hipLaunchKernelGGL(k_expert_plan, dim3((unsigned)((n + part - 1) / part)), dim3(kPlanThreads), lds, st, experts, n, (int)n_experts, bits, (int)multiple,
                       rows, part, row_of, source, offsets);
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
