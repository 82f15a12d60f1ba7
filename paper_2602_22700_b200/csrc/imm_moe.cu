// Expert dispatch and combine (sm_100a) and their C ABI (declared in imm.h).
//
//   imm_moe_dispatch   rows of the tokens sorted by expert: the ragged left operands of the experts' products
//   imm_moe_combine    the experts' output rows back in token order, weighted and added up
//
// Both move rows of some KiB and are bound by HBM.  The order is a stable counting sort of the (token, slot) pairs:
// pairs are cut into runs of RUN; a counting launch writes how many pairs of every run go to every expert (no such
// launch when there is one run only); a moving launch then gives every block the tokens of a part of one run: the
// block works out the first row of its pairs from the counts of the runs before and by counting the pairs of its
// own run that come first, so no scan launch and no waiting between blocks is needed.  Counting uses integer
// atomics in shared memory, whose order does not matter; ranks among the pairs of one expert follow the pair's
// number, so the result is the same on every run.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/imm.h"
#include "imm_kernels.h"

namespace imm_moe {

constexpr int NT = 256;
constexpr int RUN = 2048;                     // pairs per counted run
constexpr int MAX_E = IMM_MOE_MAX_EXPERTS;

struct Dispatch {
    const char* x;
    const float* scale;
    const int32_t* expert;
    char* out;
    float* out_scale;
    int64_t* offsets;
    int32_t *position, *status;
    int32_t* counts;                          // nruns x experts (nullptr: one run)
    int64_t tokens, pairs, ldx, ldo;          // ld in bytes
    int64_t row_bytes;
    int32_t top, experts, nruns;
    int32_t tokens_per_block;
};

// expert of a pair as a histogram bin; -1: not routed
__device__ __forceinline__ int bin_of(int32_t e, int experts) { return (e >= 0 && e < experts) ? e : -1; }

__global__ void __launch_bounds__(NT) count_kernel(const Dispatch d)
{
    __shared__ int hist[MAX_E];
    for (int e = threadIdx.x; e < d.experts; e += NT) hist[e] = 0;
    __syncthreads();
    const int64_t b = (int64_t)blockIdx.x * RUN, end = min(d.pairs, b + RUN);
    for (int64_t p = b + threadIdx.x; p < end; p += NT) {
        const int e = bin_of(d.expert[p], d.experts);
        if (e >= 0) atomicAdd(&hist[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < d.experts; e += NT) d.counts[(int64_t)blockIdx.x * d.experts + e] = hist[e];
}

// W: bytes per copy word (16 when both sides allow it)
template <typename W>
__global__ void __launch_bounds__(NT) move_kernel(const Dispatch d)
{
    __shared__ int total[MAX_E], before[MAX_E];       // pairs of an expert in all runs / before this block's pairs
    __shared__ int first[MAX_E];                      // first output row of an expert
    __shared__ int warp_sum[NT / 32];
    __shared__ int bad;
    __shared__ int rows[IMM_MOE_MAX_TOP];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, E = d.experts;
    const int64_t t0 = (int64_t)blockIdx.x * d.tokens_per_block, t1 = min(d.tokens, t0 + d.tokens_per_block);
    const int64_t p0 = t0 * d.top;
    const int run = (int)(p0 / RUN);
    const int64_t r0 = (int64_t)run * RUN;
    for (int e = tid; e < E; e += NT) { total[e] = 0; before[e] = 0; }
    if (tid == 0) bad = 0;
    __syncthreads();
    if (d.counts) {
        for (int e = tid; e < E; e += NT) {
            int s = 0, b = 0;
            for (int r = 0; r < d.nruns; r++) {
                const int c = d.counts[(int64_t)r * E + e];
                if (r < run) b += c;
                s += c;
            }
            total[e] = s; before[e] = b;
        }
        __syncthreads();
        for (int64_t p = r0 + tid; p < p0; p += NT) {
            const int e = bin_of(d.expert[p], E);
            if (e >= 0) atomicAdd(&before[e], 1);
        }
    } else {
        for (int64_t p = tid; p < d.pairs; p += NT) {
            const int e = bin_of(d.expert[p], E);
            if (e >= 0) {
                atomicAdd(&total[e], 1);
                if (p < p0) atomicAdd(&before[e], 1);
            }
        }
    }
    __syncthreads();
    // exclusive scan of the totals: first rows
    {
        int carry = 0;
        for (int e0 = 0; e0 < E; e0 += NT) {
            const int e = e0 + tid;
            const int v = e < E ? total[e] : 0;
            int s = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_up_sync(0xFFFFFFFFu, s, o); if (lane >= o) s += t; }
            if (lane == 31) warp_sum[warp] = s;
            __syncthreads();
            int base = carry, all = 0;
            for (int w = 0; w < NT / 32; w++) { if (w < warp) base += warp_sum[w]; all += warp_sum[w]; }
            if (e < E) first[e] = base + s - v;
            carry += all;
            __syncthreads();
        }
        if (blockIdx.x == 0) {
            for (int e = tid; e < E; e += NT) d.offsets[e] = first[e];
            if (tid == 0) d.offsets[E] = carry;
        }
    }
    if (blockIdx.x == 0) {                            // an expert that does not exist?
        int wrong = 0;
        for (int64_t p = tid; p < d.pairs; p += NT) { const int e = d.expert[p]; wrong |= (e < -1 || e >= E) ? 1 : 0; }
        if (wrong) bad = 1;
        __syncthreads();
        if (tid == 0) *d.status = bad ? IMM_ERR_ARG : IMM_OK;
    }
    __syncthreads();
    for (int64_t t = t0; t < t1; t++) {
        if (tid == 0) {
            int n = 0;
            for (int j = 0; j < d.top; j++) {
                const int64_t p = t * d.top + j;
                const int e = bin_of(d.expert[p], E);
                int row = -1;
                if (e >= 0) {
                    row = first[e] + before[e]++;
                    rows[n++] = row;
                    if (d.out_scale) d.out_scale[row] = d.scale[t];
                }
                d.position[p] = row;
            }
            warp_sum[0] = n;
        }
        __syncthreads();
        const int n = warp_sum[0];
        const char* src = d.x + t * d.ldx;
        const int64_t words = d.row_bytes / (int64_t)sizeof(W);
        if (n)
            for (int64_t i = tid; i < words; i += NT) {
                const W v = *reinterpret_cast<const W*>(src + i * sizeof(W));
                for (int k = 0; k < n; k++) *reinterpret_cast<W*>(d.out + rows[k] * d.ldo + i * sizeof(W)) = v;
            }
        __syncthreads();
    }
}

// ---- combine ----

struct Combine {
    const void* y;
    const float* row_scale;
    const int32_t* position;
    const float* weight;
    void* out;
    int64_t tokens, y_rows, ldy, ldo;
    int32_t top, cols;
};

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(int32_t v) { return (float)v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(__half* p, float v) { *p = __float2half_rn(v); }

template <typename T, typename O>
__global__ void __launch_bounds__(NT) combine_kernel(const Combine c)
{
    const int64_t t = blockIdx.x;
    const int32_t* pos = c.position + t * c.top;
    const float* wt = c.weight ? c.weight + t * c.top : nullptr;
    O* out = (O*)c.out + t * c.ldo;
    for (int j = threadIdx.x; j < c.cols; j += NT) {
        float acc = 0.f;
        for (int k = 0; k < c.top; k++) {
            const int32_t r = pos[k];
            if (r < 0 || r >= c.y_rows) continue;
            float f = wt ? wt[k] : 1.f;
            if (c.row_scale) f *= c.row_scale[r];
            acc = fmaf(to_f(((const T*)c.y)[(int64_t)r * c.ldy + j]), f, acc);
        }
        put(out + j, acc);
    }
}

template <typename T>
cudaError_t launch_combine(const Combine& c, int out_dtype, cudaStream_t st)
{
    const unsigned grid = (unsigned)c.tokens;
    if (out_dtype == IMM_F32) combine_kernel<T, float><<<grid, NT, 0, st>>>(c);
    else if (out_dtype == IMM_BF16) combine_kernel<T, __nv_bfloat16><<<grid, NT, 0, st>>>(c);
    else combine_kernel<T, __half><<<grid, NT, 0, st>>>(c);
    return cudaGetLastError();
}

bool valid(int64_t tokens, int top, int experts)
{
    return tokens >= 0 && top > 0 && top <= IMM_MOE_MAX_TOP && experts > 0 && experts <= IMM_MOE_MAX_EXPERTS &&
           tokens <= IMM_MOE_MAX_PAIRS / top;
}

int runs_of(int64_t pairs) { return (int)((pairs + RUN - 1) / RUN); }

}  // namespace imm_moe

extern "C" {

size_t imm_moe_dispatch_workspace(int64_t tokens, int top, int experts)
{
    using namespace imm_moe;
    if (!valid(tokens, top, experts)) return 0;
    const int n = runs_of(tokens * top);
    return n > 1 ? (size_t)n * experts * sizeof(int32_t) : 0;
}

int imm_moe_dispatch(const void* d_x, const float* d_scale, const int32_t* d_expert, int64_t tokens, int top, int experts,
                     int64_t cols, int elem_bytes, int64_t ldx, int64_t ldo, int64_t out_rows, void* d_out, float* d_out_scale,
                     int64_t* d_offsets, int32_t* d_position, int32_t* d_status, void* d_ws, size_t ws_bytes, void* stream)
{
    using namespace imm_moe;
    if (!d_offsets || !d_status || (tokens > 0 && (!d_x || !d_expert || !d_out || !d_position))) return IMM_ERR_ARG;
    if ((d_scale == nullptr) != (d_out_scale == nullptr)) return IMM_ERR_ARG;
    if (elem_bytes != 1 && elem_bytes != 2 && elem_bytes != 4) return IMM_ERR_ARG;
    if (!valid(tokens, top, experts)) return IMM_ERR_SHAPE;
    if (cols <= 0 || cols > IMM_NORM_MAX_COLS || ldx < cols || ldo < cols || out_rows < tokens * top) return IMM_ERR_SHAPE;
    if ((uintptr_t)d_x % elem_bytes || (uintptr_t)d_out % elem_bytes || (uintptr_t)d_scale % 4 || (uintptr_t)d_out_scale % 4 ||
        (uintptr_t)d_expert % 4 || (uintptr_t)d_offsets % 8 || (uintptr_t)d_position % 4 || (uintptr_t)d_status % 4 || (uintptr_t)d_ws % 16)
        return IMM_ERR_ALIGN;
    const size_t need = imm_moe_dispatch_workspace(tokens, top, experts);
    if (need && (!d_ws || ws_bytes < need)) return IMM_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)stream;
    Dispatch d{};
    d.x = (const char*)d_x; d.scale = d_scale; d.expert = d_expert; d.out = (char*)d_out; d.out_scale = d_out_scale;
    d.offsets = d_offsets; d.position = d_position; d.status = d_status; d.counts = need ? (int32_t*)d_ws : nullptr;
    d.tokens = tokens; d.pairs = tokens * top; d.ldx = ldx * elem_bytes; d.ldo = ldo * elem_bytes; d.row_bytes = cols * elem_bytes;
    d.top = top; d.experts = experts; d.nruns = runs_of(d.pairs);
    // a block's tokens lie in one run: RUN / top tokens per run would not be whole, so a run's part is cut at pairs
    d.tokens_per_block = 1;
    const unsigned grid = (unsigned)(tokens ? tokens : 1);
    if (need) {
        count_kernel<<<(unsigned)d.nruns, NT, 0, st>>>(d);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return imm::cuda_failed(e);
    }
    const uintptr_t all = (uintptr_t)d_x | (uintptr_t)d_out | (uintptr_t)d.ldx | (uintptr_t)d.ldo | (uintptr_t)d.row_bytes;
    if (all % 16 == 0) move_kernel<uint4><<<grid, NT, 0, st>>>(d);
    else if (all % 4 == 0) move_kernel<uint32_t><<<grid, NT, 0, st>>>(d);
    else if (all % 2 == 0) move_kernel<uint16_t><<<grid, NT, 0, st>>>(d);
    else move_kernel<uint8_t><<<grid, NT, 0, st>>>(d);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? IMM_OK : imm::cuda_failed(e);
}

int imm_moe_combine(const void* d_y, int dtype, const float* d_row_scale, const int32_t* d_position, const float* d_weight,
                    int64_t tokens, int top, int64_t cols, int64_t y_rows, int64_t ldy, int64_t ldo, int out_dtype, void* d_out,
                    void* stream)
{
    using namespace imm_moe;
    if (tokens > 0 && (!d_position || !d_out || (y_rows > 0 && !d_y))) return IMM_ERR_ARG;
    if (dtype != IMM_I32 && dtype != IMM_F32 && dtype != IMM_BF16 && dtype != IMM_F16) return IMM_ERR_ARG;
    if (out_dtype != IMM_F32 && out_dtype != IMM_BF16 && out_dtype != IMM_F16) return IMM_ERR_ARG;
    if (!valid(tokens, top, 1)) return IMM_ERR_SHAPE;
    if (cols <= 0 || cols > IMM_NORM_MAX_COLS || y_rows < 0 || y_rows > IMM_MOE_MAX_PAIRS || ldy < cols || ldo < cols) return IMM_ERR_SHAPE;
    const uintptr_t es = dtype == IMM_I32 || dtype == IMM_F32 ? 4 : 2, os = out_dtype == IMM_F32 ? 4 : 2;
    if ((uintptr_t)d_y % es || (uintptr_t)d_out % os || (uintptr_t)d_row_scale % 4 || (uintptr_t)d_position % 4 || (uintptr_t)d_weight % 4)
        return IMM_ERR_ALIGN;
    if (tokens == 0) return IMM_OK;
    const Combine c{d_y, d_row_scale, d_position, d_weight, d_out, tokens, y_rows, ldy, ldo, top, (int32_t)cols};
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
    if (dtype == IMM_I32) e = launch_combine<int32_t>(c, out_dtype, st);
    else if (dtype == IMM_F32) e = launch_combine<float>(c, out_dtype, st);
    else if (dtype == IMM_BF16) e = launch_combine<__nv_bfloat16>(c, out_dtype, st);
    else e = launch_combine<__half>(c, out_dtype, st);
    return e == cudaSuccess ? IMM_OK : imm::cuda_failed(e);
}

}  // extern "C"
